// One new token per sequence against chosen blocks of its paged context, or against
// all of it with the weights kept (gfx950, head_dim 64 or 128).
//
// Tiles, lane maps and merge are those of the biased decode (biased_decode.h): a
// workgroup takes one partition of one (sequence, KV head, tile of GP query heads),
// its wavefronts the 16-token blocks round-robin, each with two tiles in a register
// ring.  KV heads of more than eight query heads take several tiles of eight, each of which
// reads the K and V (without the streaming hint; 256 sequences of 8192 tokens over one KV head
// of 128, 8 / 16 query heads: chosen blocks 175 / 306 us, weights 234 / 366; 32 over 8 KV heads,
// 64 / 128: 171 / 203, 219 / 285).
//
// LISTED: the blocks come from a list per (sequence, KV head).  A wavefront's lanes
// load 64 entries and then their table entries; an entry that names no block of the
// context becomes a tile of zeros whose tokens lie behind the context.
//
// WEIGHTS: the scores (log2 units, -inf behind the context) go to memory as
// [token][GP] beside the partitions' log-sum-exps, from which weights_body makes the
// weights; the two are 8 GP bytes a token and KV head of traffic against the 4 D of
// its K and V, where a second pass over the keys would be 2 D and its products again.
// These stores cost more than their bytes (128 sequences of 64..8192 tokens, 32 heads
// over 8, 782 MB of K and V and 24 MB of scores: 172 us, 150 without the stores), so they
// are kept down.  A wavefront gathers scores in LDS, up to kRoomBlocks a workgroup; a
// row whose blocks are no more than that is one partition, and ends with its log-sum-exps at
// hand, and what goes to memory is one sum over the tile's heads a token, a fourth or an
// eighth (164 us; 128 of 64..2000 118 / 106).  The others' scores are stored 64 blocks at a time.
#pragma once

#include "biased_decode.h"
#include "tokens.h"

namespace pa {
namespace chosen {

using biased::decode_merge;
using biased::decode_tile;
using biased::kDecodeLdsBytes;
using decode::KvTile;
using decode::WaveState;
using decode::load_rows;
using mfma::floatx4_t;
using mfma::kWaves;
using mfma::pack_bf16;

__device__ __forceinline__ int clamped(int x, int most) { return x < 0 ? 0 : (x > most ? most : x); }

// Index of a workgroup's row tile: (b * head_tiles + tile) * num_kv_heads + g.
struct Place {
  int g, tile, b, part;
};
__device__ __forceinline__ Place place_of(const TokensParams& p, int wg) {
  Place x;
  x.g = wg % p.num_kv_heads;
  wg /= p.num_kv_heads;
  x.tile = wg % p.head_tiles;
  wg /= p.head_tiles;
  x.b = wg % p.batch;
  x.part = wg / p.batch;
  return x;
}

// The scores' place in LDS: behind the stages, and the merge's floats with the rows'
// log-sum-exps, which take their room (GP is a multiple of 4: whole 16 bytes).
template <int D, int GP>
constexpr int kScoreRoom = ((2 * kWaves * GP + kWaves * GP * D + GP) * 4 > kDecodeLdsBytes<D, GP>
                                ? (2 * kWaves * GP + kWaves * GP * D + GP) * 4 : kDecodeLdsBytes<D, GP>);
static_assert((kScoreRoom<64, 4> | kScoreRoom<64, 8> | kScoreRoom<128, 4> | kScoreRoom<128, 8>) % 16 == 0, "16-byte records");
template <int GP> constexpr int kRoomBlocks = GP == 4 ? 128 : 64;    // three workgroups fit a CU
template <int GP> constexpr int kScoreBytes = kRoomBlocks<GP> * 16 * GP * 4;
// Whether a sequence's rows keep their scores in LDS (weights): its blocks are one
// partition then.
template <int GP>
__device__ __forceinline__ bool kept_whole(const TokensParams& p, int nblk) {
  return nblk <= min(p.whole_blocks, kRoomBlocks<GP>);
}
template <int D, int GP> constexpr int kLsePlace = 2 * kWaves * GP + kWaves * GP * D;         // floats: behind the merge's
template <int D, int GP, bool WEIGHTS>
constexpr int kChosenLdsBytes = WEIGHTS ? kScoreRoom<D, GP> + kScoreBytes<GP> : kDecodeLdsBytes<D, GP>;

template <int D, int GP, bool LISTED, bool WEIGHTS, int AUX>
__device__ __forceinline__ void decode_body(const TokensParams& p, int wg, lds_u8_t* smem) {
  constexpr int DPL = D / 16;
  constexpr int NBUF = 2;
  constexpr int kNowhere = 1 << 26;                     // a block behind every context
  const int lane = threadIdx.x & 63;
  const int wave = wave_uniform(threadIdx.x >> 6);
  const int q = lane >> 4;
  const int n = lane & 15;

  const Place at = place_of(p, wg);
  const int head0 = at.g * p.group + at.tile * GP;      // the tile's heads: rows of them
  const int rows = min(GP, p.group - at.tile * GP);
  const int32_t* table = p.block_tables + (size_t)at.b * p.bt_stride;
  const int32_t* list = LISTED ? p.selected + ((size_t)at.b * p.num_kv_heads + at.g) * p.max_blocks : table;
  const int list_len = LISTED ? p.max_blocks : p.bt_stride;

  // the partition's first entries are loaded with the context length, not after it
  const int j0 = at.part * p.part_blocks;
  const int first_entry = j0 + lane < list_len ? list[j0 + lane] : -1;
  const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
  uint4 qb[D / 32];
  {
    const uint16_t* q_row = p.q + ((size_t)at.b * p.num_q_heads + head0 + min(n & (GP - 1), rows - 1)) * D;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const uint4 x = *reinterpret_cast<const uint4*>(q_row + (4 * s + q) * 8);
      qb[s] = make_uint4(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
    }
  }
  const int ctx = clamped(p.context_lens[at.b], p.max_ctx);
  const int nblk = (ctx + 15) >> 4;
  const int all = LISTED ? (ctx > 0 ? p.max_blocks : 0) : nblk;
  const bool whole = WEIGHTS && kept_whole<GP>(p, nblk);
  const int cnt = whole ? (at.part == 0 ? nblk : 0) : min(p.part_blocks, all - j0);
  const int tile_index = (at.b * p.head_tiles + at.tile) * p.num_kv_heads + at.g;
  const size_t slot = (size_t)tile_index * p.parts + at.part;
  if (cnt <= 0 && at.part > 0) {
    if (threadIdx.x < GP) p.part_lse[slot * GP + threadIdx.x] = -__builtin_inff();
    return;
  }
  float* scores = WEIGHTS ? p.scores + (size_t)tile_index * p.score_tokens * GP : nullptr;
  lds_f32_t* room = reinterpret_cast<lds_f32_t*>(smem + kScoreRoom<D, GP> + wave * (kScoreBytes<GP> / kWaves));

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
  const uint16_t* kbase = p.k_pool + (size_t)at.g * kTile;
  const uint16_t* vbase = p.v_pool + (size_t)at.g * kTile;
  const uint32_t lane_off = (uint32_t)(q * D + DPL * n) * 2u;
  const BiasedParams none{};                            // nothing of it is read without CAP and BIAS

  for (int c0 = 0; c0 < cnt; c0 += 64) {
    const int cn = min(64, cnt - c0);
    int entry = c0 == 0 ? first_entry : (lane < cn ? list[j0 + c0 + lane] : -1);
    int where = j0 + c0 + lane;                          // block of the context
    if constexpr (LISTED) {
      where = lane < cn && entry >= 0 && entry < nblk ? entry : kNowhere;
      entry = where != kNowhere ? table[where] : 0;
    }
    const int ids = lane < cn ? clamped(entry, p.num_blocks - 1) : 0;
    auto block_at = [&](int i) { return LISTED ? __builtin_amdgcn_readlane(where, i) : j0 + c0 + i; };
    auto load = [&](KvTile<D>& T, int i) {
      const bool in = i < cn;
      const size_t id = (size_t)__builtin_amdgcn_readlane(ids, in ? i : 0);
      const bool ok = in && block_at(in ? i : 0) != kNowhere;
      const int bytes = ok ? (int)(kTile * 2) : 0;
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
          const int t0 = block_at(i) * 16;
          auto keep = [&](const float (&e)[4]) {
            if constexpr (WEIGHTS) {
              // Columns n and n ^ GP (and at GP = 4 all four fours) hold the same scores: each
              // stores another register's, 64 floats side by side per instruction.
              lds_f32_t* dst = room + ((whole ? c0 : 0) + i) / kWaves * (16 * GP);
              if constexpr (GP == 4) {
                const int r = n >> 2;
                const float x = r == 0 ? e[0] : (r == 1 ? e[1] : (r == 2 ? e[2] : e[3]));
                dst[(4 * r + q) * GP + (n & 3)] = x;
              } else {
                const bool odd = n >= 8;
                dst[(4 * (int)odd + q) * GP + (n & 7)] = odd ? e[1] : e[0];
                dst[(4 * (2 + (int)odd) + q) * GP + (n & 7)] = odd ? e[3] : e[2];
              }
            }
          };
          decode_tile<D, false, false>(none, S, T[s], qb, stage, t0, 0, ctx, t0 + 16 > ctx, q, n, lo_part, scale, 0,
                                       0.f, keep);
          i += kWaves;
          done = i >= cn;
        }
      }
    }
    if (WEIGHTS && !whole) {
      __builtin_amdgcn_wave_barrier();
      constexpr int kLanes = 4 * GP;                    // lanes that hold a block's scores, four each
      for (int k = lane / kLanes; wave + kWaves * k < cn; k += 64 / kLanes) {
        const floatx4_t x = *reinterpret_cast<const mfma::lds_floatx4_t*>(room + k * (16 * GP) + lane % kLanes * 4);
        *reinterpret_cast<floatx4_t*>(scores + (size_t)(j0 + c0 + wave + kWaves * k) * (16 * GP) + lane % kLanes * 4) = x;
      }
      __builtin_amdgcn_wave_barrier();
    }
  }

  decode_merge<D, GP>(S, smem, wave, q, n, rows, [&](int r, int d, float o0, float o1, float lt, float mref) {
    if (p.parts > 1)
      store_partial2(p.part_o + (slot * GP + r) * D + d, o0, o1);
    else
      *reinterpret_cast<uint32_t*>(p.out + ((size_t)at.b * p.num_q_heads + head0 + r) * D + d) = pack_bf16(o0, o1);
    if (d == 0 && (p.parts > 1 || WEIGHTS)) {
      const float lse = lt == 0.f ? -__builtin_inff() : mref + log2f(lt);
      p.part_lse[slot * GP + r] = lse;
      if constexpr (WEIGHTS) reinterpret_cast<lds_f32_t*>(smem)[kLsePlace<D, GP> + r] = lt == 0.f ? __builtin_inff() : lse;
    }
  });
  if (WEIGHTS && whole) {
    __syncthreads();
    float lse[GP];
#pragma unroll
    for (int r = 0; r < GP; ++r) lse[r] = r < rows ? reinterpret_cast<lds_f32_t*>(smem)[kLsePlace<D, GP> + r] : __builtin_inff();
    const lds_f32_t* all = reinterpret_cast<const lds_f32_t*>(smem + kScoreRoom<D, GP>);
    for (int t = threadIdx.x; t < ctx; t += 64 * kWaves) {
      const int j = t >> 4;
      const lds_f32_t* e = all + (j % kWaves) * (kScoreBytes<GP> / kWaves / 4) + (j / kWaves * 16 + (t & 15)) * GP;
      float sum = 0.f;
#pragma unroll
      for (int r4 = 0; r4 < GP; r4 += 4) {
        const floatx4_t x = *reinterpret_cast<const mfma::lds_floatx4_t*>(e + r4);
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += fast_exp2(x[r] - lse[r4 + r]);
      }
      scores[t] = sum;
    }
  }
}

// One row (query head) of a sequence from its partitions: one wavefront, weights
// 2^(lse - max lse), D / 64 dims per lane, eight partitions' rows loaded together.
template <int D>
__device__ __forceinline__ void merge_row(const TokensParams& p, int64_t row) {
  constexpr int DPL = D / 64, kTogether = 8;
  const int lane = threadIdx.x & 63;
  const int b = (int)(row / p.num_q_heads), h = (int)(row % p.num_q_heads);
  const int g = h / p.group, tile = h % p.group / p.tile_heads, r = h % p.group % p.tile_heads;
  const size_t slot = ((size_t)(b * p.head_tiles + tile) * p.num_kv_heads + g) * p.parts;
  const float* lse = p.part_lse + slot * p.tile_heads + r;
  const float* po = p.part_o + (slot * p.tile_heads + r) * D + DPL * lane;
  float mx = -__builtin_inff();
  for (int c = lane; c < p.parts; c += 64) mx = fmaxf(mx, lse[(size_t)c * p.tile_heads]);
  mx = group_max4(row_max16(mx));
  const float mref = mx == -__builtin_inff() ? 0.f : mx;
  float sum = 0.f, acc[DPL];
#pragma unroll
  for (int d = 0; d < DPL; ++d) acc[d] = 0.f;
  for (int c0 = 0; c0 < p.parts; c0 += 64) {
    const float x = c0 + lane < p.parts ? lse[(size_t)(c0 + lane) * p.tile_heads] : -__builtin_inff();
    const uint64_t some = __builtin_amdgcn_ballot_w64(x != -__builtin_inff());
    if (some == 0) continue;
    const int last = 64 - __builtin_clzll(some);
    const int wl = __float_as_int(fast_exp2(x - mref));
    for (int j0 = 0; j0 < last; j0 += kTogether) {
      float v[kTogether][DPL];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        const bool has = (some >> (j0 + k)) & 1;         // an empty partition's outputs are never written
#pragma unroll
        for (int d = 0; d < DPL; ++d) v[k][d] = has ? po[(size_t)(c0 + j0 + k) * p.tile_heads * D + d] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        const float w = __int_as_float(__builtin_amdgcn_readlane(wl, j0 + k));
        sum += w;
#pragma unroll
        for (int d = 0; d < DPL; ++d) acc[d] = fmaf(w, v[k][d], acc[d]);
      }
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  uint16_t* dst = p.out + (size_t)row * D;
  if constexpr (DPL == 2)
    *reinterpret_cast<uint32_t*>(dst + 2 * lane) = pack_bf16(acc[0] * inv, acc[1] * inv);
  else
    dst[lane] = (uint16_t)pack_bf16(acc[0] * inv, 0.f);
}

// Weights of 256 tokens of a sequence, summed over its heads in a fixed order: the
// heads' log-sum-exps over the partitions go to LDS, kHeads at a time, and a thread
// per token adds 2^(score - lse) over its GP-float records, which lie side by side.
constexpr int kHeads = 512;
constexpr int kEarly = 8;
template <int GP>
__device__ __forceinline__ void weights_body(const TokensParams& p, int b, int chunk, lds_f32_t* lds) {
  const int ctx = clamped(p.context_lens[b], p.max_ctx);
  const int t = chunk * 256 + threadIdx.x;
  if (chunk * 256 >= ctx) return;                       // whole workgroup
  const int planes = p.head_tiles * p.num_kv_heads;     // of GP heads (those past the group's are not read)
  const size_t at = (size_t)b * p.totals_stride + t;
  const float before = p.totals && t < ctx ? p.totals[at] : 0.f;
  if (kept_whole<GP>(p, (ctx + 15) >> 4)) {                 // a sum per plane and token
    const float* s = p.scores + (size_t)b * planes * p.score_tokens * GP + min(t, ctx - 1);
    float sum = 0.f;
#pragma unroll 8
    for (int i = 0; i < planes; ++i) sum += s[(size_t)i * p.score_tokens * GP];
    if (t < ctx) p.totals_out[at] = fmaf(p.decay, before, sum);
    return;
  }
  const int nparts = p.parts == 1 ? 1 : min(p.parts, ((ctx + 15) / 16 + p.part_blocks - 1) / p.part_blocks);
  const size_t plane0 = (size_t)b * planes;
  float sum = 0.f;
  for (int c0 = 0; c0 < planes; c0 += kHeads / GP) {
    const int cn = min(kHeads / GP, planes - c0);
    if (c0 > 0) __syncthreads();
    // the first planes' scores are loaded before the log-sum-exps that they wait for
    const float* s = p.scores + ((plane0 + c0) * p.score_tokens + min(t, ctx - 1)) * GP;
    const size_t step = (size_t)p.score_tokens * GP;
    floatx4_t early[kEarly][GP / 4];
#pragma unroll
    for (int i = 0; i < kEarly; ++i)
#pragma unroll
      for (int r = 0; r < GP / 4; ++r) early[i][r] = *reinterpret_cast<const floatx4_t*>(s + min(i, cn - 1) * step + 4 * r);
    for (int i = threadIdx.x; i < cn * GP; i += 256) {
      const int plane = c0 + i / GP, r = i % GP;
      float y = __builtin_inff();                       // no such head: weight 0
      if (plane / p.num_kv_heads * GP + r < p.group) {
        const float* lse = p.part_lse + (plane0 + plane) * p.parts * GP + r;
        float m = -__builtin_inff(), l = 0.f;
        for (int k0 = 0; k0 < nparts; k0 += 16) {
          float x[16], most = m;
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            x[k] = k0 + k < nparts ? lse[(size_t)(k0 + k) * GP] : -__builtin_inff();
            most = fmaxf(most, x[k]);
          }
          const float mref = most == -__builtin_inff() ? 0.f : most;
          l *= fast_exp2(m - mref);
          m = most;
#pragma unroll
          for (int k = 0; k < 16; ++k) l += fast_exp2(x[k] - mref);
        }
        y = l == 0.f ? __builtin_inff() : m + log2f(l);
      }
      lds[i] = y;
    }
    __syncthreads();
    auto add = [&](int i, int r4, const floatx4_t& e) {
#pragma unroll
      for (int r = 0; r < 4; ++r) sum += fast_exp2(e[r] - lds[i * GP + r4 + r]);
    };
#pragma unroll
    for (int i = 0; i < kEarly; ++i)
      if (i < cn)
#pragma unroll
        for (int r = 0; r < GP / 4; ++r) add(i, 4 * r, early[i][r]);
#pragma unroll 4
    for (int i = kEarly; i < cn; ++i)
#pragma unroll
      for (int r = 0; r < GP / 4; ++r) add(i, 4 * r, *reinterpret_cast<const floatx4_t*>(s + i * step + 4 * r));
  }
  if (t < ctx) p.totals_out[at] = fmaf(p.decay, before, sum);
}

}  // namespace chosen
}  // namespace pa
