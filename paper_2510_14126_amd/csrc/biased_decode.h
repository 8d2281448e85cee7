// One new token per sequence against its paged context with capped, biased or
// masked scores, for up to eight query heads per KV head (biased_body.h has the
// formulas and the form for more).
//
// The tiles, lane maps and merge are those of the plain decode (decode_body.h):
// a workgroup takes one partition of one (sequence, KV head), its wavefronts the
// 16-token blocks round-robin, each with NBUF tiles in a register ring; the 16
// columns of the 16x16 MFMA tiles hold the heads' queries twice, and the high
// and low parts of each weight ride in one PV step.  Here the columns stand for
// GP = 4 or 8 heads, of which p.group exist (the others repeat the last and are
// not written), and a block's scores are shaped before the running max:
//     y = cap tanh(x / cap),  e = y - slope (n - 1 - t),
// hidden tokens by select, in the blocks that hold some (the first and last of
// the tokens the row sees).  All heads of a sequence see the same tokens, so V of
// hidden ones is replaced by zeros.
//
// Against the 32x32 form a block's chain is half as long: half the scores per
// lane, QK^T in two accumulation chains of two instead of one of eight.  32x32 /
// this form, capped, 32 heads over 8: one sequence of 4096 tokens 12.0 / 9.4 us,
// 32 of 500 14.4 / 10.3, 64 of 2500 111 / 105, 256 of 64..8192 271 / 265 (5.9 TB/s;
// the tail of the longest contexts holds it: 64 of 8192, two heads over one, run at
// 6.6 TB/s, and reading tiles without arithmetic reaches 6.8).
#pragma once

#include "biased_body.h"
#include "decode_body.h"

namespace pa {
namespace biased {

using decode::KvTile;
using decode::WaveState;
using decode::lds_u32x2_t;
using decode::load_rows;
using decode::stage_off;
using decode::u32x2_t;
using mfma::column_value;
using mfma::floatx2_t;
using mfma::k_arow;
using mfma::lds_floatx2_t;
using mfma::short4_t;

template <int D, int GP>
constexpr int kDecodeLdsBytes = (kWaves * 16 * D * 2 > (2 * kWaves * GP + kWaves * GP * D) * 4)
                                    ? kWaves * 16 * D * 2 : (2 * kWaves * GP + kWaves * GP * D) * 4;

// One block.  t0: its first token; tokens lo <= t < hi are seen, all 16 unless
// `edge`; lo_part: 1 in the columns that carry the low parts, else 0.  keep(e): is
// given the block's scores in log2 units, register r that of token t0 + 4r + q.
struct KeepNone {
  __device__ __forceinline__ void operator()(const float (&)[4]) const {}
};
template <int D, bool CAP, bool BIAS, typename Keep = KeepNone>
__device__ __forceinline__ void decode_tile(const BiasedParams& p, WaveState<D>& S, KvTile<D>& T,
                                            const uint4 (&qb)[D / 32], lds_u8_t* stage, int t0, int lo, int hi,
                                            bool edge, int q, int n, float lo_part, float scale, int pos, float slope,
                                            const Keep& keep = Keep()) {
  constexpr int VW = D / 32;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if constexpr (D == 128) {
      *reinterpret_cast<lds_u32x4_t*>(stage + stage_off<D>(4 * u + q, n)) =
          u32x4_t{T.k[u][0], T.k[u][1], T.k[u][2], T.k[u][3]};
    } else {
      *reinterpret_cast<lds_u32x2_t*>(stage + stage_off<D>(4 * u + q, n >> 1) + ((n & 1) << 3)) =
          u32x2_t{T.k[u][0], T.k[u][1]};
    }
  }
  u32x4_t ka[D / 32];
#pragma unroll
  for (int s = 0; s < D / 32; ++s)
    ka[s] = *reinterpret_cast<const lds_u32x4_t*>(stage + stage_off<D>(k_arow(n), 4 * s + q));
  const floatx4_t z = {0.f, 0.f, 0.f, 0.f};
  floatx4_t st[2];
#pragma unroll
  for (int s = 0; s < D / 32; ++s)
    st[s & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ka[s]),
                                                        __builtin_bit_cast(bf16x8_t, qb[s]),
                                                        s < 2 ? z : st[s & 1], 0, 0, 0);
  const floatx4_t raw = st[0] + st[1];

  // Register r is token t0 + 4r + q.
  float e[4];
  if constexpr (CAP) {
    const float most = fmaxf(fmaxf(fabsf(raw[0]), fabsf(raw[1])), fmaxf(fabsf(raw[2]), fabsf(raw[3])));
    const bool far = __builtin_amdgcn_ballot_w64(!(most <= p.raw_max)) != 0;
    if (far) {
#pragma unroll
      for (int r = 0; r < 4; ++r) e[r] = cap_any(p, raw[r]);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) e[r] = cap_near(p, raw[r]);
    }
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) e[r] = raw[r] * scale;
  }
  if constexpr (BIAS) {
    const float d0 = (float)(pos - t0 - q);
#pragma unroll
    for (int r = 0; r < 4; ++r) e[r] = fmaf(-slope, fabsf(d0 - (float)(4 * r)), e[r]);
  }
  if (edge) {
    const int t_lane = t0 + q;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = t_lane + 4 * r;
      const bool seen = t >= lo && t < hi;
      e[r] = seen ? e[r] : -__builtin_inff();
#pragma unroll
      for (int w = 0; w < VW; ++w) T.v[r][w] = seen ? T.v[r][w] : 0u;    // V row 4r + q
    }
  }

  keep(e);

  const float xmax = fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3]));
  if (__builtin_amdgcn_ballot_w64(xmax > S.m + kLazyRescale) != 0) {
    const float bm = group_max4(xmax);
    const float mn = bm > S.m + kLazyRescale ? bm : S.m;
    const float alpha = mn == -__builtin_inff() ? 1.f : fast_exp2(S.m - mn);
    S.l *= alpha;
    if (__builtin_amdgcn_ballot_w64(S.m != -__builtin_inff()) != 0) {
      float ar[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) ar[r] = column_value(alpha, q, r);
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) S.o[j][r] *= ar[r];
    }
    S.m = mn;
    S.neg = mn == -__builtin_inff() ? 0.f : -mn;
  }

  float w[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) w[r] = fast_exp2(e[r] + S.neg);
  S.l += (w[0] + w[1]) + (w[2] + w[3]);
  const uint32_t h01 = pack_bf16(w[0], w[1]), h23 = pack_bf16(w[2], w[3]);
  const uint32_t w01 = pack_bf16(fmaf(-lo_part, bf16_lo(h01), w[0]), fmaf(-lo_part, bf16_hi(h01), w[1]));
  const uint32_t w23 = pack_bf16(fmaf(-lo_part, bf16_lo(h23), w[2]), fmaf(-lo_part, bf16_hi(h23), w[3]));
  const short4_t pw = __builtin_bit_cast(short4_t, make_uint2(w01, w23));
#pragma unroll
  for (int j = 0; j < D / 16; ++j) {
    const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
    const uint32_t b0 = __builtin_amdgcn_perm(T.v[1][j >> 1], T.v[0][j >> 1], sel);
    const uint32_t b1 = __builtin_amdgcn_perm(T.v[3][j >> 1], T.v[2][j >> 1], sel);
    S.o[j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(pw, __builtin_bit_cast(short4_t, make_uint2(b0, b1)),
                                                       S.o[j], 0, 0, 0);
  }
}

// The wavefronts' states become the rows' results: the low parts' output rows (GP ..
// 2GP-1) are added to the high parts' (0 .. GP-1), then the wavefronts are merged
// through LDS, as in the plain decode.  store(r, d, o0, o1, lt, mref): dims d and d+1
// of row r < rows, normalised; lt: the sum of its weights 2^(e - mref), 0 where it saw
// nothing.
template <int D, int GP, typename Store>
__device__ __forceinline__ void decode_merge(const WaveState<D>& S, lds_u8_t* smem, int wave, int q, int n, int rows,
                                             const Store& store) {
  constexpr int DPL = D / 16;   // dims per lane and token row
  const float lrow = group_sum4(S.l);
  floatx4_t sum[DPL / 2];
#pragma unroll
  for (int j = 0; j < DPL / 2; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float x = S.o[j][r], y = S.o[j + DPL / 2][r];
      if constexpr (GP == 8) swap32(x, y); else swap16(x, y);
      sum[j][r] = x + y;
    }
  const int half = GP == 8 ? q >> 1 : q & 1;          // which half of the lane's dims
  const int qrow = GP == 8 ? q & 1 : q >> 1;          // merge rows 4 * qrow + r
  const bool keeps = GP == 8 || q < 2;                // else groups 2 and 3 hold copies
  __syncthreads();
  lds_f32_t* sm = reinterpret_cast<lds_f32_t*>(smem);       // [kWaves][GP]
  lds_f32_t* sl = sm + kWaves * GP;                          // [kWaves][GP]
  lds_f32_t* sacc = sl + kWaves * GP;                        // [kWaves][GP][D]
  if (q == 0 && n < GP) {
    sm[wave * GP + n] = S.m;
    sl[wave * GP + n] = lrow;
  }
  if (keeps) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      lds_f32_t* row = sacc + (wave * GP + 4 * qrow + r) * D + DPL * n + (DPL / 2) * half;
      if constexpr (D == 128) {
        *reinterpret_cast<lds_floatx4_t*>(row) = floatx4_t{sum[0][r], sum[1][r], sum[2][r], sum[3][r]};
      } else {
        row[0] = sum[0][r];
        row[1] = sum[1][r];
      }
    }
  }
  __syncthreads();
  constexpr int kRowThreads = D / 2;                  // two output dims of a row per thread
  constexpr int kRowsPerPass = 64 * kWaves / kRowThreads;
  const int d = 2 * (threadIdx.x % kRowThreads);
#pragma unroll
  for (int r0 = 0; r0 < GP; r0 += kRowsPerPass) {
    const int r = r0 + threadIdx.x / kRowThreads;
    if (r >= rows) return;
    float mx = sm[r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mx = fmaxf(mx, sm[w * GP + r]);
    const float mref = mx == -__builtin_inff() ? 0.f : mx;
    float lt = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = fast_exp2(sm[w * GP + r] - mref);
      lt = fmaf(sl[w * GP + r], f, lt);
      const floatx2_t a = *reinterpret_cast<const lds_floatx2_t*>(sacc + (w * GP + r) * D + d);
      o0 = fmaf(a[0], f, o0);
      o1 = fmaf(a[1], f, o1);
    }
    const float inv = lt == 0.f ? 0.f : 1.0f / lt;
    store(r, d, o0 * inv, o1 * inv, lt, mref);
  }
}

template <int D, int GP, bool CAP, bool BIAS, int AUX>
__device__ __forceinline__ void decode_body(const BiasedParams& p, int wg, lds_u8_t* smem) {
  constexpr int DPL = D / 16;   // dims per lane and token row
  // Tiles of the ring.  With two a wavefront needs 156 registers and three run
  // per SIMD, with three 190 and two; two / three, capped, D = 128: 32 sequences of
  // 1024 tokens 20.4 / 21.1 us, 64 of 2500 105 / 109, 64 of 8192 325 / 326.
  constexpr int NBUF = 2;
  static_assert(GP == 4 || GP == 8, "columns of a tile");
  const int lane = threadIdx.x & 63;
  const int wave = wave_uniform(threadIdx.x >> 6);
  const int q = lane >> 4;
  const int n = lane & 15;

  const int g = wg % p.num_kv_heads;
  wg /= p.num_kv_heads;
  const int b = wg % p.batch;
  const int part = wg / p.batch;
  const int head0 = g * p.group;
  const int32_t* table = p.block_tables + (size_t)b * p.bt_stride;

  // Where nothing but the context length bounds what the row sees, the
  // partition's first block ids are loaded with it instead of after it.
  const bool whole = p.window == 0 && p.first_tokens == nullptr && p.bt_stride > 0;
  int ids_first = 0;
  if (whole) ids_first = table[min((int64_t)part * p.part_blocks + lane, (int64_t)p.bt_stride - 1)];
  const int first_token = p.first_tokens ? p.first_tokens[b] : 0;
  const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
  const int head = min(n & (GP - 1), p.group - 1);
  uint4 qb[D / 32];
  {
    const uint16_t* q_row = p.q + ((size_t)b * p.num_q_heads + head0 + head) * D;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const uint4 x = *reinterpret_cast<const uint4*>(q_row + (4 * s + q) * 8);
      qb[s] = make_uint4(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
    }
  }
  const float slope = BIAS ? p.slopes[head0 + head] * kLog2e : 0.f;
  int ctx = p.context_lens[b];
  ctx = ctx < 0 ? 0 : (ctx > p.max_ctx ? p.max_ctx : ctx);

  const int hi = ctx;
  int lo = p.window > 0 ? max(0, ctx - p.window) : 0;
  lo = min(max(lo, first_token), hi);
  const int first = lo >> 4;
  const int nblk = hi > lo ? ((hi + 15) >> 4) - first : 0;
  const int per = p.parts == 1 ? nblk : p.part_blocks;
  const int j0 = first + part * per;
  const int cnt = min(per, nblk - part * per);
  const size_t slot = ((size_t)b * p.num_kv_heads + g) * p.parts + part;
  const bool split = p.parts > 1 && nblk > per;         // else the first partition writes the output
  if (cnt <= 0 && part > 0) {
    if (threadIdx.x < p.tile_rows) p.part_lse[slot * p.tile_rows + threadIdx.x] = -__builtin_inff();
    return;
  }

  WaveState<D> S;
  S.m = -__builtin_inff();
  S.neg = 0.f;
  S.l = 0.f;
#pragma unroll
  for (int j = 0; j < DPL; ++j) S.o[j] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  const float scale = p.scale_log2 == 0.f ? 1.1754944e-38f : fabsf(p.scale_log2);
  const float lo_part = (n & GP) ? 1.f : 0.f;
  lds_u8_t* stage = smem + wave * (16 * D * 2);

  constexpr size_t kTile = 16 * D;
  const size_t blk_stride = (size_t)p.num_kv_heads * kTile;
  const uint16_t* kbase = p.k_pool + (size_t)g * kTile;
  const uint16_t* vbase = p.v_pool + (size_t)g * kTile;
  const uint32_t lane_off = (uint32_t)(q * D + DPL * n) * 2u;

  for (int c0 = 0; c0 < cnt; c0 += 64) {
    const int cn = min(64, cnt - c0);
    const int raw = c0 == 0 && whole ? ids_first : (lane < cn ? table[j0 + c0 + lane] : 0);
    const int ids = lane < cn ? min(max(raw, 0), p.num_blocks - 1) : 0;
    auto load = [&](KvTile<D>& T, int i) {
      const bool ok = i < cn;
      const size_t id = (size_t)__builtin_amdgcn_readlane(ids, ok ? i : 0);
      const int bytes = ok ? (int)(kTile * 2) : 0;        // none past the last: zeros
      load_rows<D, AUX>(T.k, kbase + id * blk_stride, lane_off, bytes);
      load_rows<D, AUX>(T.v, vbase + id * blk_stride, lane_off, bytes);
    };
    KvTile<D> T[NBUF];
    int i = wave, ld = wave;
#pragma unroll
    for (int s = 0; s < NBUF - 1; ++s) {
      load(T[s], ld);
      ld += kWaves;
    }
    bool done = i >= cn;
    while (!done) {
#pragma unroll
      for (int s = 0; s < NBUF; ++s) {
        if (!done) {
          load(T[(s + NBUF - 1) % NBUF], ld);
          ld += kWaves;
          const int t0 = (j0 + c0 + i) * 16;
          decode_tile<D, CAP, BIAS>(p, S, T[s], qb, stage, t0, lo, hi, t0 < lo || t0 + 16 > hi, q, n, lo_part, scale,
                                    ctx - 1, slope);
          i += kWaves;
          done = i >= cn;
        }
      }
    }
  }

  decode_merge<D, GP>(S, smem, wave, q, n, p.group, [&](int r, int d, float o0, float o1, float lt, float mref) {
    if (split) {
      store_partial2(p.part_o + (slot * p.tile_rows + r) * D + d, o0, o1);
      if (d == 0) p.part_lse[slot * p.tile_rows + r] = lt == 0.f ? -__builtin_inff() : mref + log2f(lt);
    } else {
      const size_t row = (size_t)b * p.num_q_heads + head0 + r;
      *reinterpret_cast<uint32_t*>(p.out + row * D + d) = pack_bf16(o0, o1);
      if (d == 0 && p.parts > 1) p.part_lse[slot * p.tile_rows + r] = kWhole;
    }
  });
}

}  // namespace biased
}  // namespace pa
