// Attention of query rows over a paged context with capped, biased or masked
// scores, on 32x32 MFMA tiles (gfx950, head_dim 64 or 128).
//
// For KV head g the (new token i, head j) pairs of sequence b form rows
// R = i * G + j, at position p = n - L + i (n: context with the L new tokens).
// In log2 units, x = |scale| log2(e) <q, K[t]> (a negative scale rides on the
// sign of Q),
//     y = cap tanh(x / cap)      (CAP)        y = x            (else)
//     e = y - slope |p - t|      (BIAS)
// for the tokens lo <= t < hi that the row sees, and out = sum 2^e V / sum 2^e.
//
// tanh: tanh(z) / z is even, so while |z| <= 1/2 a polynomial of degree three in
// raw^2 (minimax, relative error 5.5e-7) gives y in four FMAs and one product,
// without the transcendental unit that the softmax keeps busy; a stage with any
// larger score (rare: caps are chosen well above ordinary scores) takes cap -
// 2 cap / (2^(2 z log2 e) + 1) for those.
//
// Lanes: h = lane >> 5, n = lane & 31.  v_mfma_f32_32x32x16_bf16 takes A row n
// / B column n at contraction indices 8h .. 8h+7 and leaves in register r of
// its result row 8(r/4) + 4h + r%4 of column n.  A stage is 32 tokens, K rows
// then V rows in LDS.
//  * S^T = K Q^T: A = K rows (token i of the stage in row i), B = Q^T with query
//    row n in column n.  Lane (h, n) receives the scores of tokens 8a + 4h + b
//    (register 4a + b).
//  * O += P V: for block m of the stage the contraction index k = 8h + e
//    stands for token 16m + 8(e/4) + 4h + e%4, which makes the scores above
//    exactly the A operand; the B operand comes from the staged V through
//    transposing reads.  Each weight reaches the matrix core as a bf16 pair,
//    high part and rounded remainder (about 2^-17 relative); the row sum adds
//    the fp32 values.
//
// What hidden tokens hold must not matter.  Tokens that no row of the workgroup
// sees are staged as zeros.  Where some rows see a token and others do not its
// weight is an exact 0, but 0 times an infinity or NaN in V is NaN in an MFMA:
// in stages with masks, infinities and NaN of V are staged as zeros too, and a
// second pass over those stages (add_special, only where there were any) adds
// them to the rows that do see them.
#pragma once

#include "kernels.h"
#include "mfma_body.h"
#include "ops.h"
#include "pa_device.h"

namespace pa {
namespace biased {

using mfma::bf16x8_t;
using mfma::floatx16_t;
using mfma::floatx4_t;
using mfma::kLazyRescale;
using mfma::kWaves;
using mfma::lds_floatx4_t;
using mfma::lds_short4_t;
using mfma::lds_u32x4_t;
using mfma::pack_bf16;
using mfma::u32x4_t;
typedef __attribute__((address_space(3))) uint16_t lds_u16_t;
typedef __attribute__((address_space(3))) uint32_t lds_u32_t;

constexpr int kTokens = 32;                                 // per stage: two blocks
template <int D> constexpr int kStageBytes = 2 * kTokens * D * 2;   // K rows, then V rows
template <int D> constexpr int kVOffset = kTokens * D * 2;
template <int D> constexpr int kPieces = D / 32;            // 16-byte pieces of K (and of V) per lane and 16 tokens, x 2

// LDS byte offset of 16-byte chunk c of token row r of the staged K: chunk c at
// position c ^ r modulo the row's chunks.  Lanes read one chunk column of 32
// rows: eight consecutive ones touch eight different positions.
template <int D>
__device__ __forceinline__ int k_off(int r, int c) {
  return r * (2 * D) + ((c ^ (r & (D / 8 - 1))) << 4);
}

// The same of the staged V (from kVOffset): 32-byte windows of 16 dims.  The
// transposing reads of a half wavefront take windows 2j and 2j+1 of four
// consecutive rows; at D = 128 a row spans all 64 banks and window w is at
// w ^ 2(r % 4), at D = 64 two rows do and it is at w ^ 2(r / 2 % 2).
template <int D>
__device__ __forceinline__ int v_off(int r, int c) {
  const int swz = D == 128 ? (r & 3) << 1 : (r & 2);
  return r * (2 * D) + (((c >> 1) ^ swz) << 5) + ((c & 1) << 4);
}

// Maximum over the 32 columns; every lane receives it (both halves hold the
// same columns).
template <int CTRL>
__device__ __forceinline__ int dpp_i(int x) { return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ int max32(int x) {
  x = max(x, dpp_i<kDppQuadXor1>(x));
  x = max(x, dpp_i<kDppQuadXor2>(x));
  x = max(x, dpp_i<kDppRowRor4>(x));
  x = max(x, dpp_i<kDppRowRor8>(x));
  const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return wave_uniform(max((int)y[0], (int)y[1]));
}
__device__ __forceinline__ int min32(int x) { return -max32(-x); }

// Sequence b's new tokens: its first row in q and out, their number, the
// position of the first and the context length.  Device data, clamped.
struct Chunk {
  int start, len, first, ctx;
};
__device__ __forceinline__ Chunk chunk_of(const BiasedParams& p, int b) {
  int ctx = p.context_lens[b];
  ctx = ctx < 0 ? 0 : (ctx > p.max_ctx ? p.max_ctx : ctx);
  int qs = b, L = 1;
  if (p.q_start) {
    qs = p.q_start[b];
    qs = qs < 0 ? 0 : (qs > p.total_q ? p.total_q : qs);
    const int qe = p.q_start[b + 1];
    L = qe < qs ? 0 : (qe > p.total_q ? p.total_q : qe) - qs;
  }
  L = min(min(L, ctx), p.max_chunk);
  return {qs, L, ctx - L, ctx};
}

// What the row of column n sees, and its bias.
struct Row {
  int lo, hi;       // tokens lo <= t < hi; hi <= lo: none
  int pos;          // differences of positions become fp32, not positions: those pass 2^24
  float slope;      // log2 units per token of distance
};
template <bool BIAS>
__device__ __forceinline__ Row row_of(const BiasedParams& p, const Chunk& c, int b, int g, int R) {
  const int i = R / p.group;
  const int pos = c.first + i;
  Row r;
  r.lo = p.window > 0 ? max(0, pos - p.window + 1) : 0;
  if (p.first_tokens) r.lo = max(r.lo, min(p.first_tokens[c.start + i], c.ctx));
  r.hi = pos + 1;
  if (p.prefix_lens) r.hi = max(r.hi, min(p.prefix_lens[b], c.ctx));
  r.hi = max(r.hi, r.lo);
  r.pos = pos;
  r.slope = BIAS ? p.slopes[g * p.group + R % p.group] * kLog2e : 0.f;
  return r;
}

// A raw score capped, in log2 units: within the polynomial's range, and anywhere.
__device__ __forceinline__ float cap_factor(const BiasedParams& p, float x) {
  const float u = x * x;
  return fmaf(u, fmaf(u, fmaf(u, p.c3, p.c2), p.c1), p.c0);
}
__device__ __forceinline__ float cap_near(const BiasedParams& p, float x) { return x * cap_factor(p, x); }
__device__ __forceinline__ float cap_far(const BiasedParams& p, float x) {
  const float t = fast_exp2(x * p.two_z);
  return fmaf(-2.f * p.cap, __builtin_amdgcn_rcpf(t + 1.f), p.cap);
}
__device__ __forceinline__ bool cap_is_near(const BiasedParams& p, float x) { return fabsf(x) <= p.raw_max; }
__device__ __forceinline__ float cap_any(const BiasedParams& p, float x) {
  const float z = cap_far(p, x);
  return cap_is_near(p, x) ? cap_near(p, x) : z;
}

// Trees (TREE): a row sees the tokens before the chunk, and of the chunk the node's
// ancestors and itself: bit j of the row's kTreeWords words in LDS is node j (a word
// of zeros behind them takes the reads past the last node).  Rows are kTreePitch
// words apart: 32 lanes that read one word of 32 rows touch 32 banks.
constexpr int kTreeWords = kTreeMostNodes / 32;
constexpr int kTreePitch = kTreeWords + 1;
template <int ROWS> constexpr int kTreeBytes = ROWS * kTreePitch * 4;

// Fills the words of the workgroup's ROWS rows from row0 on and ends with a
// barrier.  The parents go through LDS (up: 2 kTreeMostNodes bytes that nobody reads
// yet), for a path is a chain of dependent reads.
template <int ROWS>
__device__ __forceinline__ void tree_rows(const BiasedParams& p, const Chunk& c, int row0, lds_u32_t* words, lds_u16_t* up) {
  constexpr int kNone = 0xffff;
  for (int j = threadIdx.x; j < c.len; j += 64 * kWaves) {          // c.len <= max_chunk <= kTreeMostNodes
    const int x = p.parents[c.start + j];
    up[j] = (uint16_t)(x >= 0 && x < j ? x : kNone);
  }
  __syncthreads();
  if (threadIdx.x < ROWS) {
    const int R = row0 + threadIdx.x;
    int j = R < c.len * p.group ? R / p.group : kNone;
    lds_u32_t* row = words + threadIdx.x * kTreePitch;
    row[kTreeWords] = 0u;
#pragma unroll 1
    for (int w = kTreeWords - 1; w >= 0; --w) {
      uint32_t bits = 0u;
      while (j != kNone && j >= 32 * w) {                           // nodes descend
        bits |= 1u << (j & 31);
        j = up[j];
      }
      row[w] = bits;
    }
  }
  __syncthreads();
}

// Bits of a row's nodes from `from` on (k: node from + k); the context before the
// chunk (from + k < 0) is seen.
__device__ __forceinline__ uint32_t tree_bits(const lds_u32_t* row, int from) {
  const int w = min(max(from, 0) >> 5, kTreeWords);
  const uint32_t a = row[w], b = row[min(w + 1, kTreeWords)];
  const int s = max(from, 0) & 31;
  const uint32_t x = s == 0 ? a : (a >> s) | (b << (32 - s));
  if (from <= -32) return 0xffffffffu;
  return from < 0 ? (x << -from) | (0xffffffffu >> (32 + from)) : x;
}

// The 32 columns of one wavefront: queries (Q^T operand of step s: dims 16s + 8h
// .. of column n), softmax state, outputs.
template <int D, bool CAP, bool BIAS, bool TREE = false>
struct Columns {
  Row row;
  const lds_u32_t* tree;        // TREE: the words of the wavefront's first row
  int drafted;                  // TREE: the chunk's first token
  float m, neg, l;              // running max, -m (0 while it is -inf), the lane's share of the sum
  floatx16_t o[D / 32];         // [j][r]: row 8(r/4) + 4h + r%4, dim 32j + n
  float scale;                  // |scale_log2|
  float base;                   // of the shaped stage (see shape)
  float most;                   // its largest |raw score| (CAP)

  // Operand of step s from the row's memory; bf16 negation is exact.
  static __device__ __forceinline__ u32x4_t query(const BiasedParams& p, const uint16_t* q_row, int s, int h) {
    const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
    const uint4 w = *reinterpret_cast<const uint4*>(q_row + (2 * s + h) * 8);
    return u32x4_t{w.x ^ flip, w.y ^ flip, w.z ^ flip, w.w ^ flip};
  }

  __device__ __forceinline__ void init(const BiasedParams& p, const Row& r) {
    // A scale of zero becomes the smallest normal number, so that a hidden
    // token's score stays -inf times it (ordinary scores weigh the same).
    scale = p.scale_log2 == 0.f ? 1.1754944e-38f : fabsf(p.scale_log2);
    row = r;
    m = -__builtin_inff();
    neg = 0.f;
    l = 0.f;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
  }

  // Raw scores of the stage at st; q(s): the operand of step s.
  template <typename Q>
  static __device__ __forceinline__ floatx16_t scores(const lds_u8_t* st, int h, int n, Q&& q) {
    floatx16_t a;
#pragma unroll
    for (int i = 0; i < 16; ++i) a[i] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const lds_u32x4_t*>(st + k_off<D>(n, 2 * s + h))),
          __builtin_bit_cast(bf16x8_t, q(s)), a, 0, 0, 0);
    return a;
  }

  // Shapes the raw scores of a stage whose first token is t0, in two parts.
  //
  // shape: what nearly every stage needs, without a branch, so that the compiler
  // can place it between the PV MFMAs of the stage before.  Without CAP and BIAS
  // the scores stay raw; with CAP alone they become log2 units less the running
  // max of the stages before, base, in the polynomial's last FMA; with BIAS log2
  // units without the part of the bias that all tokens of the stage share, base =
  // slope (t0 + 4h - p): one FMA per score adds slope (t - t0 - 4h), and base goes
  // where the running max does.
  //
  // reshape: in a stage with scores beyond the polynomial those alone anew, so that
  // no score's bits depend on another, which its row may not see; in one with
  // tokens after a row's position (not linear) base and the FMA's part for |p - t|
  // (small numbers both, as before: large ones would cost bits); then the masks, in a
  // stage with hidden tokens (edge).
  __device__ __forceinline__ floatx16_t shape(const BiasedParams& p, const floatx16_t& raw, int t0, int h) {
    floatx16_t a = raw;
    if constexpr (CAP) {
      most = fabsf(raw[0]);
#pragma unroll
      for (int r = 1; r < 16; ++r) most = fmaxf(most, fabsf(raw[r]));
    }
    if constexpr (CAP || BIAS) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float off = BIAS ? row.slope * (float)(8 * (r >> 2) + (r & 3)) : neg;
        a[r] = fmaf(raw[r], CAP ? cap_factor(p, raw[r]) : scale, off);
      }
    }
    base = BIAS ? row.slope * (float)(t0 + 4 * h - row.pos) : CAP ? -neg : 0.f;
    return a;
  }
  __device__ __forceinline__ void reshape(const BiasedParams& p, floatx16_t& a, const floatx16_t& raw, int t0, bool edge,
                                          bool linear, int h) {
    if (CAP && __builtin_amdgcn_ballot_w64(!(most <= p.raw_max)) != 0) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float z = cap_far(p, raw[r]) + (BIAS ? row.slope * (float)(8 * (r >> 2) + (r & 3)) : neg);
        a[r] = cap_is_near(p, raw[r]) ? a[r] : z;
      }
    }
    if (BIAS && !linear) {
      const float d0 = (float)(row.pos - t0 - 4 * h);
      base = -row.slope * fabsf(d0);                       // of the lane's first token, before the row or after it
#pragma unroll
      for (int r = 0; r < 16; ++r)
        a[r] = fmaf(2.f * row.slope, fminf(fmaxf(d0, 0.f) - (float)(8 * (r >> 2) + (r & 3)), 0.f), a[r]);
    }
    if (edge) {
      // bit k: the row sees token t0 + 4h + k
      const int from = max(row.lo - (t0 + 4 * h), 0), to = min(row.hi - (t0 + 4 * h), 32);
      uint32_t seen = to > from ? (0xffffffffu >> (32 - (to - from))) << from : 0u;
      if constexpr (TREE) seen &= tree_bits(tree + ((int)threadIdx.x & 31) * kTreePitch, t0 + 4 * h - drafted);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)seen, 8 * (r >> 2) + (r & 3), 1);
        a[r] = __uint_as_float((keep & __float_as_uint(a[r])) | (~keep & 0xff800000u));
      }
    }
  }

  // One value per row, from the lane (h, n) that holds it as column n to the
  // lanes that hold the row's outputs.  rowv: 32 floats of the wavefront's own.
  static __device__ __forceinline__ void per_row(lds_f32_t* rowv, int h, int n, float x, float (&out)[16]) {
    if (h == 0) rowv[n] = x;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const floatx4_t y = *reinterpret_cast<const lds_floatx4_t*>(rowv + 8 * a + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) out[4 * a + e] = y[e];
    }
    __builtin_amdgcn_wave_barrier();
  }

  // Running-max step before a stage's weights.  The test needs no cross-lane
  // reduction: any lane above its row's max + kLazyRescale triggers the rescale.
  // Scores that hold a running max (CAP alone) follow it.
  __device__ __forceinline__ void raise(floatx16_t& a, lds_f32_t* rowv, int h, int n) {
    float x = a[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) x = fmaxf(x, a[r]);
    if constexpr (CAP || BIAS)
      x += base;
    else
      x *= scale;
    if (__builtin_amdgcn_ballot_w64(x > m + kLazyRescale) != 0) {
      float y = x;
      swap32(x, y);
      const float bm = fmaxf(x, y);
      const float mn = bm > m + kLazyRescale ? bm : m;
      // 1 for rows that keep their max (or have attended to nothing yet)
      const float alpha = mn == -__builtin_inff() ? 1.f : fast_exp2(m - mn);
      l *= alpha;
      if (__builtin_amdgcn_ballot_w64(m != -__builtin_inff()) != 0) {
        float ar[16];
        per_row(rowv, h, n, alpha, ar);
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[j][r] *= ar[r];
      }
      m = mn;
      neg = mn == -__builtin_inff() ? 0.f : -mn;
      if constexpr (CAP && !BIAS) {
#pragma unroll
        for (int r = 0; r < 16; ++r) a[r] += neg + base;
      }
    }
  }

  // Weights of the shaped scores a and their PV with the stage at st.
  __device__ __forceinline__ void attend(const floatx16_t& a, const lds_u8_t* st, int lane) {
    float w[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) w[r] = fast_exp2(BIAS ? a[r] + (neg + base) : CAP ? a[r] : fmaf(a[r], scale, neg));
    u32x4_t hi[2], lo[2];
    float sum[2];
#pragma unroll
    for (int mb = 0; mb < 2; ++mb)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float p0 = w[8 * mb + e], p1 = w[8 * mb + e + 1];
        const uint32_t x = pack_bf16(p0, p1);
        hi[mb][e / 2] = x;
        lo[mb][e / 2] = pack_bf16(p0 - bf16_lo(x), p1 - bf16_hi(x));
        sum[mb] = e == 0 ? p0 + p1 : sum[mb] + (p0 + p1);
      }
    l += sum[0] + sum[1];
    // Transposing reads: lane i = lane % 16 of group (h, f = bit 4 of lane)
    // addresses row 4h + i/4 (+ 8u, + 16m), dims 32j + 16f + 4(i%4) .. +3.
    const int vr = 4 * (lane >> 5) + ((lane & 15) >> 2);
    const int vf = (lane >> 4) & 1;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
      u32x4_t vb[D / 32];
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        uint2 b[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          b[u] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                     (lds_short4_t*)(st + kVOffset<D> + mb * 16 * D * 2 + v_off<D>(vr + 8 * u, 2 * (2 * j + vf)) +
                                     ((lane & 3) << 3))));
        vb[j] = u32x4_t{b[0].x, b[0].y, b[1].x, b[1].y};
      }
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
        o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, hi[mb]),
                                                       __builtin_bit_cast(bf16x8_t, vb[j]), o[j], 0, 0, 0);
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
        o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, lo[mb]),
                                                       __builtin_bit_cast(bf16x8_t, vb[j]), o[j], 0, 0, 0);
    }
  }

  // Adds what stood in V where a masked stage was given zeros for infinities and
  // NaN, to the rows that see it (its weight is above 0: it makes them infinite
  // or NaN).  v: the stage's V as it is, first token t0.  rowv: 32 floats of LDS
  // of the wavefront's own.
  __device__ __forceinline__ void add_special(int t0, const lds_u8_t* v, lds_f32_t* rowv, int h, int n) {
    float from[16], to[16];
    per_row(rowv, h, n, __int_as_float(row.lo), from);
    per_row(rowv, h, n, __int_as_float(row.hi), to);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
#pragma unroll 1
      for (int t = 0; t < kTokens; ++t) {
        const uint32_t x = *reinterpret_cast<const lds_u16_t*>(v + v_off<D>(t, (32 * j + n) >> 3) + ((n & 7) << 1));
        const float y = (x & 0x7f80u) == 0x7f80u ? bf16_lo(x) : 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t0 + t >= __float_as_int(from[r]) && t0 + t < __float_as_int(to[r]) &&
              (!TREE || (tree_bits(tree + (8 * (r >> 2) + 4 * h + (r & 3)) * kTreePitch, t0 + t - drafted) & 1u) != 0))
            o[j][r] += y;
      }
    }
  }
};

// The order of a range's stages: with a distance bias from the nearest tokens to
// the farthest, so that the running max is found first (upwards it rises with
// every stage of a steep head, and each rise rescales the outputs: a prompt of
// 8191 tokens upwards 841 us, downwards 728).  at(s): stage of step s (past the last step
// the last stage again); chunk(s): which 64 blocks hold it.
template <bool DOWN>
struct Walk {
  int n;
  static constexpr int kStep = DOWN ? -1 : 1;
  __device__ __forceinline__ int at(int s) const {
    const int t = max(min(s, n - 1), 0);
    return DOWN ? max(n - 1, 0) - t : t;
  }
  __device__ __forceinline__ int chunk(int s) const { return 2 * at(s) >> 6; }
};

// Zeros for the infinities and NaN among N x 8 bf16; marks in `odd` that there
// were any.  An exponent of all ones carries into the sign's place.
template <int N>
__device__ __forceinline__ void keep_finite(u32x4_t (&v)[N], uint32_t& odd) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) any |= (v[i][e] & 0x7f807f80u) + 0x00800080u;
  if (__builtin_amdgcn_ballot_w64((any & 0x80008000u) != 0) == 0) return;
  odd = 1;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t bad = (((v[i][e] & 0x7f807f80u) + 0x00800080u) >> 15) & 0x00010001u;
      v[i][e] &= ~(bad * 0xffffu);
    }
}

// add_special over the masked ones of a wavefront's stages (steps from, from +
// step, ... of the walk) of cnt blocks that begin at block j0 with table entries
// bt: all its lanes, for its own columns.  v: LDS for a stage's V of the wavefront's own.
template <int D, typename C, typename W>
__device__ __forceinline__ void special_pass(C& cols, const BiasedParams& p, const int32_t* bt, const uint16_t* vbase,
                                             const W& walk, int cnt, int j0, int from, int step, int all_lo, int all_hi,
                                             lds_u8_t* v, lds_f32_t* rowv) {
  constexpr int kChunks = D / 8;
  const int lane = threadIdx.x & 63;
#pragma unroll 1
  for (int i = from; i < walk.n; i += step) {
    const int s = walk.at(i);
    const int t0 = (j0 + 2 * s) * 16;
    if (t0 >= all_lo && t0 + kTokens <= all_hi) continue;
#pragma unroll 1
    for (int r = lane / kChunks; r < kTokens; r += 64 / kChunks) {
      const int j = 2 * s + (r >> 4);
      uint4 x = make_uint4(0, 0, 0, 0);
      if (j < cnt) {
        const size_t id = (size_t)min(max(bt[j], 0), p.num_blocks - 1);
        x = *reinterpret_cast<const uint4*>(vbase + id * p.num_kv_heads * (16 * D) + (r & 15) * D + lane % kChunks * 8);
      }
      *reinterpret_cast<lds_u32x4_t*>(v + v_off<D>(r, lane % kChunks)) = u32x4_t{x.x, x.y, x.z, x.w};
    }
    __builtin_amdgcn_wave_barrier();
    cols.add_special(t0, v, rowv, lane >> 5, lane & 31);
    __builtin_amdgcn_wave_barrier();
  }
}

// --------------------------------------------------------------------------
// One row tile per workgroup, its tokens split over the wavefronts (and over
// workgroups, `parts`): for decode, short chunks and small grids.
// --------------------------------------------------------------------------
template <int D> constexpr int kSwapBytes = 4 * 64 * (D / 32) * 4;     // one wavefront's outputs for another at the merge
template <int D> constexpr int kSplitStats = kWaves * kStageBytes<D>;
template <int D> constexpr int kSplitQuery = kSplitStats<D> + 3 * kWaves * kBiasedTileRows * 4;   // the tile's queries
template <int D> constexpr int kSplitLdsBytes = kSplitQuery<D> + kBiasedTileRows * D * 2;
static_assert(kWaves * (kWaves - 1) * kSwapBytes<128> <= kSplitStats<128>, "the merge reuses the stages");
static_assert(kWaves * (kWaves - 1) * kSwapBytes<64> <= kSplitStats<64>, "the merge reuses the stages");

// In place of the log-sum-exp of a row tile's first partition: it was the only
// one and the output is written.  (A row's own is at most finite, or NaN.)
constexpr float kWhole = __builtin_inff();

// AUX: cache policy of the tiles' loads.
// TREE: kTreeBytes<kBiasedTileRows> of LDS follow kSplitLdsBytes.
template <int D, bool CAP, bool BIAS, int AUX, bool TREE = false>
__device__ __forceinline__ void split_body(const BiasedParams& p, int wg, lds_u8_t* smem) {
  using Cols = Columns<D, CAP, BIAS, TREE>;
  constexpr int kRows = kBiasedTileRows;
  const int lane = threadIdx.x & 63;
  const int wave = wave_uniform(threadIdx.x >> 6);
  const int h = lane >> 5;
  const int n = lane & 31;

  const int g = wg % p.num_kv_heads;
  wg /= p.num_kv_heads;
  const int tile = wg % p.tiles;
  wg /= p.tiles;
  const int b = wg % p.batch;
  const int part = wg / p.batch;

  // Where nothing but the context length bounds what rows see, the partition's
  // first block ids are loaded with it instead of after it.
  const bool whole = p.window == 0 && p.first_tokens == nullptr && p.bt_stride > 0;
  int ids_first = 0;
  if (whole) {
    const int64_t j = (int64_t)part * p.part_blocks + lane;
    ids_first = p.block_tables[(size_t)b * p.bt_stride + min(j, (int64_t)p.bt_stride - 1)];
  }
  const Chunk c = chunk_of(p, b);
  const int rows = c.len * p.group;
  const int row0 = tile * kRows;
  if (row0 >= rows && !(p.q_start == nullptr && c.len == 0 && part == 0)) return;   // whole workgroup: no rows here
  if (c.len == 0) {
    // an empty sequence of a decode: its rows are zeros
    for (int i = threadIdx.x; i < min(kRows, p.group - row0) * D; i += 64 * kWaves)
      p.out[((size_t)b * p.num_q_heads + g * p.group + row0 + i / D) * D + i % D] = 0;
    return;
  }

  // A column without a row repeats the tile's first and is not written.
  const int R = row0 + n < rows ? row0 + n : row0;
  u32x4_t q_mine[D / 64];                              // this wavefront's share of the queries
  {
    const uint16_t* q_row = p.q + ((size_t)(c.start + R / p.group) * p.num_q_heads + g * p.group + R % p.group) * D;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) q_mine[i] = Cols::query(p, q_row, wave * (D / 64) + i, h);
  }
  const Row row = row_of<BIAS>(p, c, b, g, R);
  const bool none = row.hi <= row.lo;
  const int lo = min32(none ? 0x3fffffff : row.lo);     // tokens that some row sees
  const int hi = max32(none ? 0 : row.hi);
  const int all_lo = max32(row.lo);                     // tokens that every row sees
  const int all_hi = TREE ? c.first : min32(none ? 0 : row.hi);

  const int from_pos = c.first + row0 / p.group;        // position of the tile's first row
  // This partition's blocks.
  const int first = lo >> 4;
  const int nblk = hi > lo ? ((hi + 15) >> 4) - first : 0;
  const int per = partition_blocks(p, nblk);
  const int j0 = first + part * per;
  const int cnt = min(per, nblk - part * per);          // <= 0: nothing in this partition
  const size_t slot = (((size_t)b * p.tiles + tile) * p.num_kv_heads + g) * p.parts + part;
  const bool split = p.parts > 1 && nblk > per;         // else the first partition writes the output
  if (cnt <= 0 && p.parts > 1) {
    if (threadIdx.x < p.tile_rows) p.part_lse[slot * p.tile_rows + threadIdx.x] = -__builtin_inff();
    return;
  }

  Cols C;
  C.init(p, row);
  if constexpr (TREE) {
    lds_u32_t* words = reinterpret_cast<lds_u32_t*>(smem + kSplitLdsBytes<D>);
    tree_rows<kRows>(p, c, row0, words, reinterpret_cast<lds_u16_t*>(smem));
    C.tree = words;
    C.drafted = c.first;
  }
  // The queries stay in LDS (all wavefronts have the same rows): in registers
  // they would not fit beside a stage in flight.
  lds_u32x4_t* ql = reinterpret_cast<lds_u32x4_t*>(smem + kSplitQuery<D>) + lane;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) ql[64 * (wave * (D / 64) + i)] = q_mine[i];

  constexpr size_t kTile = 16 * D;
  const size_t blk_stride = (size_t)p.num_kv_heads * kTile;
  const uint16_t* kbase = p.k_pool + (size_t)g * kTile;
  const uint16_t* vbase = p.v_pool + (size_t)g * kTile;
  const int32_t* bt = p.block_tables + (size_t)b * p.bt_stride + j0;

  // A wavefront's stage: kLoads pieces of K and of V per lane, piece i of token
  // row i * kRowsPerLoad + lane / (D/8).
  constexpr int kChunks = D / 8;
  constexpr int kRowsPerLoad = 64 / kChunks;
  constexpr int kLoads = kTokens / kRowsPerLoad;
  const int lrow = lane / kChunks, lchunk = lane % kChunks;
  const int lane_off = lane * 16;
  u32x4_t rk[kLoads], rv[kLoads];
  const int nstage = (cnt + 1) >> 1;
  // Block ids, one per lane: those of the 64 blocks being loaded and the next 64.
  auto ids_of = [&](int chunk) {
    const int j = 64 * chunk + lane;
    return j >= 0 && j < cnt ? min(max(bt[j], 0), p.num_blocks - 1) : 0;
  };
  const Walk<BIAS> walk{nstage};
  int chunk = walk.chunk(wave);
  int ids = whole && chunk == 0 ? (lane < cnt ? min(max(ids_first, 0), p.num_blocks - 1) : 0) : ids_of(chunk);
  int ids_next = ids_of(chunk + walk.kStep);
  auto load = [&](int s) {
    if (walk.chunk(s) != chunk) {                         // uniform; a wavefront's stages skip no chunk
      ids = ids_next;
      chunk += walk.kStep;
      ids_next = ids_of(chunk + walk.kStep);
    }
    const int j = 2 * walk.at(s);
    int id[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) id[e] = __builtin_amdgcn_readlane(ids, (j + e) & 63);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int bytes = s < nstage && j + e < cnt ? (int)kTile * 2 : 0;      // none past the last block: zeros
      const __amdgpu_buffer_rsrc_t dk = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint16_t*>(kbase + (size_t)id[e] * blk_stride), 0, bytes, kBufferDescWord3);
      const __amdgpu_buffer_rsrc_t dv = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint16_t*>(vbase + (size_t)id[e] * blk_stride), 0, bytes, kBufferDescWord3);
#pragma unroll
      for (int i = 0; i < kLoads / 2; ++i) {
        rk[e * kLoads / 2 + i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(dk, lane_off + i * 1024, 0, AUX));
        rv[e * kLoads / 2 + i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(dv, lane_off + i * 1024, 0, AUX));
      }
    }
  };

  lds_u8_t* st = smem + wave * kStageBytes<D>;
  lds_f32_t* sm = reinterpret_cast<lds_f32_t*>(smem + kSplitStats<D>);   // [kWaves][32]
  lds_f32_t* sl = sm + kWaves * kRows;                                   // [kWaves][32]
  lds_f32_t* rowv = sl + kWaves * kRows + wave * kRows;

  uint32_t odd = 0;                                               // infinities or NaN among V where there are masks
  load(wave);
  __syncthreads();
  for (int s = wave; s < nstage; s += kWaves) {
    const int t0 = (j0 + 2 * walk.at(s)) * 16;
    const bool edge = t0 < all_lo || t0 + kTokens > all_hi;       // uniform
    if (edge) {
      if (t0 < lo || t0 + kTokens > hi) {
        const int t_lane = t0 + lrow;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int t = t_lane + i * kRowsPerLoad;
          if (t < lo || t >= hi) {
            rk[i] = u32x4_t{0, 0, 0, 0};
            rv[i] = u32x4_t{0, 0, 0, 0};
          }
        }
      }
      keep_finite(rv, odd);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = i * kRowsPerLoad + lrow;
      *reinterpret_cast<lds_u32x4_t*>(st + k_off<D>(r, lchunk)) = rk[i];
      *reinterpret_cast<lds_u32x4_t*>(st + kVOffset<D> + v_off<D>(r, lchunk)) = rv[i];
    }
    load(s + kWaves);
    const floatx16_t raw = C.scores(st, h, n, [&](int i) { return ql[64 * i]; });
    floatx16_t a = C.shape(p, raw, t0, h);
    C.reshape(p, a, raw, t0, edge, t0 + kTokens <= from_pos + 1, h);
    C.raise(a, rowv, h, n);
    C.attend(a, st, lane);
  }

  if (__builtin_amdgcn_ballot_w64(odd != 0) != 0)
    special_pass<D>(C, p, bt, vbase, walk, cnt, j0, wave, kWaves, all_lo, all_hi, st, rowv);

  // Merge.  Row n's maximum and sum over the wavefronts, then each wavefront
  // scales its outputs to the common maximum and the final sum; wavefront d
  // adds up rows 8d + 4h + b (b = 0..3).
  {
    float x = C.l, y = C.l;
    swap32(x, y);
    if (h == 0) {
      sm[wave * kRows + n] = C.m;
      sl[wave * kRows + n] = x + y;
    }
  }
  __syncthreads();
  float mx = sm[n];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) mx = fmaxf(mx, sm[w * kRows + n]);
  const float mref = mx == -__builtin_inff() ? 0.f : mx;
  float lt = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) lt = fmaf(sl[w * kRows + n], fast_exp2(sm[w * kRows + n] - mref), lt);
  const float inv = lt == 0.f ? 0.f : 1.0f / lt;
  if (p.parts > 1 && wave == 0 && lane < p.tile_rows)
    p.part_lse[slot * p.tile_rows + lane] = !split ? kWhole : (lt == 0.f ? -__builtin_inff() : mref + log2f(lt));
  float f[16];
  Cols::per_row(rowv, h, n, fast_exp2(C.m - mref) * inv, f);
  constexpr int kJ = D / 32;
  auto at = [&](int dst, int src) {   // outputs of wavefront src for wavefront dst
    return reinterpret_cast<lds_f32_t*>(smem + (dst * (kWaves - 1) + (src > dst ? src - 1 : src)) * kSwapBytes<D>) +
           lane * kJ;
  };
#pragma unroll
  for (int d = 0; d < kWaves; ++d)
    if (d != wave) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < kJ; ++j) at(d, wave)[e * 64 * kJ + j] = C.o[j][4 * d + e] * f[4 * d + e];
    }
  __syncthreads();
#pragma unroll
  for (int d = 0; d < kWaves; ++d)
    if (d == wave) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 8 * d + 4 * h + e;
        float acc[kJ];
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          acc[j] = C.o[j][4 * d + e] * f[4 * d + e];
#pragma unroll
          for (int w = 0; w < kWaves; ++w)
            if (w != d) acc[j] += at(d, w)[e * 64 * kJ + j];
        }
        const int Rr = row0 + r;
        if (Rr < rows) {
          if (split) {
#pragma unroll
            for (int j = 0; j < kJ; ++j) store_partial(p.part_o + (slot * p.tile_rows + r) * D + 32 * j + n, acc[j]);
          } else {
            uint16_t* dst = p.out + ((size_t)(c.start + Rr / p.group) * p.num_q_heads + g * p.group + Rr % p.group) * D;
#pragma unroll
            for (int j = 0; j < kJ; j += 2) {
              const uint32_t x = pack_bf16(acc[j], acc[j + 1]);
              dst[32 * j + n] = (uint16_t)x;
              dst[32 * j + 32 + n] = (uint16_t)(x >> 16);
            }
          }
        }
      }
    }
}

// --------------------------------------------------------------------------
// 128 rows per workgroup, 32 per wavefront, over one stream of stages through
// LDS that all of them read: for long chunks.
//
// The loop is software-pipelined by one stage: iteration j publishes stage j+2
// to LDS, loads stage j+3 and computes the scores of stage j+1, the weights of
// stage j and their PV; every slot is read only between the barriers that follow
// its writing and precede its next writing.  Publishing first leaves scores and
// weights in one run of instructions without a branch (masked stages have one
// while they are published), exponentials between the MFMAs of the scores: scores
// before it / after, 8191 tokens with slopes 740 / 728 us, 16 chunks of 600 over
// 2904 capped 733 / 727, four of 3001..4096 tokens in documents of 61..1500 206 / 205.
// --------------------------------------------------------------------------
constexpr int kSlots = 3;
template <int D> constexpr int kBigRow = kSlots * kStageBytes<D>;         // one value per row, per wavefront
template <int D> constexpr int kBigRange = kBigRow<D> + kWaves * kBiasedTileRows * 4;   // ranges of the wavefronts
template <int D> constexpr int kBigLdsBytes = kBigRange<D> + 4 * kWaves * 4;
static_assert(kWaves * kBiasedTileRows * 128 * 2 <= kBigRow<128> && kWaves * kBiasedTileRows * 64 * 2 <= kBigRow<64>,
              "the stages' room holds the outputs, and a V tile per wavefront");

// F over the wavefront, of two values at a time; every lane receives it.
template <typename F>
__device__ __forceinline__ int all64(int x, F&& f) {
  x = f(x, dpp_i<kDppQuadXor1>(x));
  x = f(x, dpp_i<kDppQuadXor2>(x));
  x = f(x, dpp_i<kDppRowRor4>(x));
  x = f(x, dpp_i<kDppRowRor8>(x));
  const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = f((int)y[0], (int)y[1]);
  const auto z = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return wave_uniform(f((int)z[0], (int)z[1]));
}

// The order of the row tiles of a call that the GPU holds all at once (ranked):
// its CUs take one or two workgroups each, and the one with the most work ends the
// call.  Workgroup w and the one a CU further, w + kCus, share a CU (the
// dispatcher deals them out in turn), so the tiles that see the most tokens go to
// the CUs with one and the others in pairs of the longest with the shortest.
// Sequence after sequence / ranked, capped, D = 128: chunks of 128, 576 and 1024
// tokens over 2304 resident ones (432 workgroups) 165 / 152 us, four of 600 over
// 1000, 16 heads over 16 (304), 78 / 65, 17 of 168 over 2432, 12 over 2 (272), 122 /
// 117.  With more workgroups than slots the sequences' own order is kept:
// neighbours share their tokens in L2 (four chunks of 3001..4096 tokens in
// documents ranked by length 201 -> 229 us).
//
// Here tile i of a KV head: sequence b, its chunk and tile, false: there are fewer.
// One sequence per lane; a tile's length counts in tiles, `first` before its chunk.
__device__ __forceinline__ bool ranked_tile(const BiasedParams& p, int i, int& b, Chunk& c, int& tile) {
  const int lane = threadIdx.x & 63;
  const Chunk own = chunk_of(p, min(lane, p.batch - 1));
  const int tiles = lane < p.batch ? (int)(((int64_t)own.len * p.group + kBiasedWgRows - 1) / kBiasedWgRows) : 0;
  const int first = (int)min((int64_t)own.first * p.group / kBiasedWgRows, (int64_t)1 << 29);
  auto sum = [](int x, int y) { return x + y; };
  const int n = all64(tiles, sum);
  if (i >= n) return false;
  const int cus = kCus / p.num_kv_heads;               // tiles of a head until each CU has a workgroup
  if (n > cus) {
    const int alone = max(2 * cus - n, 0);             // CUs (tiles of a head) with one workgroup
    i = i >= cus ? n - 1 - (i - cus) : (i < cus - alone ? alone + i : i - (cus - alone));
  }
  auto at_least = [&](int v) { return all64(min(max(first + tiles - v + 1, 0), tiles), sum); };
  // the largest length v that more than i tiles reach
  int v = 1, past = all64(first + tiles, [](int x, int y) { return max(x, y); }) + 1;
  while (past - v > 1) {
    const int mid = v + (past - v) / 2;
    if (at_least(mid) > i)
      v = mid;
    else
      past = mid;
  }
  uint64_t with = __builtin_amdgcn_ballot_w64(first < v && v <= first + tiles);
  for (int j = i - at_least(v + 1); j > 0; --j) with &= with - 1;
  b = __builtin_ctzll(with);
  tile = v - 1 - __builtin_amdgcn_readlane(first, b);
  c = {__builtin_amdgcn_readlane(own.start, b), __builtin_amdgcn_readlane(own.len, b),
       __builtin_amdgcn_readlane(own.first, b), __builtin_amdgcn_readlane(own.ctx, b)};
  return true;
}

// TREE: kTreeBytes<kBiasedWgRows> of LDS follow kBigLdsBytes, and the tokens may be
// split over workgroups (parts).
template <int D, bool CAP, bool BIAS, bool TREE = false>
__device__ __forceinline__ void big_body(const BiasedParams& p, int wg, lds_u8_t* smem) {
  using Cols = Columns<D, CAP, BIAS, TREE>;
  const int lane = threadIdx.x & 63;
  const int wave = wave_uniform(threadIdx.x >> 6);
  const int h = lane >> 5;
  const int n = lane & 31;

  const int g = wg % p.num_kv_heads;
  wg /= p.num_kv_heads;
  // A chunk's last rows see the most tokens: they start first.
  int tile = p.tiles - 1 - wg % p.tiles;
  int b = wg / p.tiles;
  int part = 0;
  if constexpr (TREE) {
    part = b / p.batch;
    b = b % p.batch;
  }
  Chunk c;
  if (!TREE && p.ranked) {
    if (!ranked_tile(p, wg, b, c, tile)) return;       // whole workgroup
  } else {
    c = chunk_of(p, b);
  }
  const int rows = c.len * p.group;
  if (tile * kBiasedWgRows >= rows) return;            // whole workgroup: no rows here
  // Which 32 of the rows the wavefront takes.  A tree's tile is seldom full: a
  // wavefront without rows computes nothing, and since wavefront i of either of a CU's
  // two workgroups runs on its SIMD i, every other workgroup turns the rows by two, so
  // that its idle wavefronts meet the other's busy ones.
  const int turn = TREE ? (wave + 2 * (int)(blockIdx.x / kCus & 1)) & 3 : wave;
  const int row0 = tile * kBiasedWgRows + kBiasedTileRows * turn;
  const bool busy = !TREE || row0 < rows;

  // A column without a row repeats the workgroup's first and is not written.
  const int R = row0 + n < rows ? row0 + n : tile * kBiasedWgRows;
  u32x4_t q[D / 16];
  {
    const uint16_t* q_row = p.q + ((size_t)(c.start + R / p.group) * p.num_q_heads + g * p.group + R % p.group) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) q[s] = Cols::query(p, q_row, s, h);
  }
  const Row row = row_of<BIAS>(p, c, b, g, R);
  int lo, hi, all_lo, all_hi;                          // tokens that some row, that every row of the workgroup sees
  {
    const bool none = row.hi <= row.lo;
    lds_i32_t* range = reinterpret_cast<lds_i32_t*>(smem + kBigRange<D>);
    const int x[4] = {-min32(none ? 0x3fffffff : row.lo), max32(none ? 0 : row.hi), max32(row.lo),
                      -min32(none ? 0 : row.hi)};
    if (lane < 4) range[4 * wave + lane] = lane == 0 ? x[0] : (lane == 1 ? x[1] : (lane == 2 ? x[2] : x[3]));
    __syncthreads();
    int y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = range[i];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) y[i] = max(y[i], range[4 * w + i]);
      y[i] = wave_uniform(y[i]);
    }
    lo = -y[0];
    hi = y[1];
    all_lo = y[2];
    all_hi = TREE ? c.first : -y[3];
    __syncthreads();                                   // `range` is used again
  }
  const int from_pos = c.first + tile * kBiasedWgRows / p.group;   // position of the workgroup's first row
  int j0 = lo >> 4;
  int cnt = hi > lo ? ((hi + 15) >> 4) - j0 : 0;
  bool split = false;                                  // else the first partition writes the output
  size_t slot = 0;                                     // of its first row's partial results
  if constexpr (TREE) {
    slot = ((((size_t)b * p.tiles + tile) * p.num_kv_heads + g) * p.parts + part) * p.tile_rows + turn * kBiasedTileRows;
    const int per = p.parts > 1 ? p.part_blocks : cnt;
    split = cnt > per;
    j0 += part * per;
    cnt = min(per, cnt - part * per);
    if (cnt <= 0 && part > 0) {
      if (lane < kBiasedTileRows && turn * kBiasedTileRows + lane < p.tile_rows) p.part_lse[slot + lane] = -__builtin_inff();
      return;                                          // whole workgroup
    }
  }

  Cols C;
  C.init(p, row);
  if constexpr (TREE) {
    lds_u32_t* words = reinterpret_cast<lds_u32_t*>(smem + kBigLdsBytes<D>);
    tree_rows<kBiasedWgRows>(p, c, tile * kBiasedWgRows, words, reinterpret_cast<lds_u16_t*>(smem));
    C.tree = words + turn * kBiasedTileRows * kTreePitch;
    C.drafted = c.first;
  }
  auto query = [&](int s) { return q[s]; };

  constexpr size_t kTile = 16 * D;
  const size_t blk_stride = (size_t)p.num_kv_heads * kTile;
  const uint16_t* kbase = p.k_pool + (size_t)g * kTile;
  const uint16_t* vbase = p.v_pool + (size_t)g * kTile;
  const int32_t* bt = p.block_tables + (size_t)b * p.bt_stride + j0;
  const int nstage = (cnt + 1) >> 1;
  auto ids_of = [&](int chunk) {
    const int j = 64 * chunk + lane;
    return j >= 0 && j < cnt ? min(max(bt[j], 0), p.num_blocks - 1) : 0;
  };
  const Walk<BIAS> walk{nstage};
  int chunk = walk.chunk(0);
  int ids = ids_of(chunk), ids_next = ids_of(chunk + walk.kStep);

  // The workgroup's share of a stage: 256 threads take 16 bytes each of K and V,
  // D / 64 times: whole blocks (D = 128) or both halves at once (D = 64).
  constexpr int kLoads = D / 64;
  constexpr int kChunks = D / 8;
  const int lrow = threadIdx.x / kChunks, lchunk = threadIdx.x % kChunks;
  const int lane_off = (D == 128 ? threadIdx.x : threadIdx.x & 127) * 16;
  u32x4_t rk[kLoads], rv[kLoads];
  auto load = [&](int s) {
    if (walk.chunk(s) != chunk) {                      // uniform
      ids = ids_next;
      chunk += walk.kStep;
      ids_next = ids_of(chunk + walk.kStep);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int j = 2 * walk.at(s) + (D == 128 ? i : wave >> 1);
      const size_t id = (size_t)__builtin_amdgcn_readlane(ids, j & 63);
      const int bytes = s < nstage && j < cnt ? (int)kTile * 2 : 0;  // none past the last block: zeros
      const __amdgpu_buffer_rsrc_t dk = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint16_t*>(kbase + id * blk_stride), 0, bytes, kBufferDescWord3);
      const __amdgpu_buffer_rsrc_t dv = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint16_t*>(vbase + id * blk_stride), 0, bytes, kBufferDescWord3);
      rk[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(dk, lane_off, 0, 0));
      rv[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(dv, lane_off, 0, 0));
    }
  };
  auto first_of = [&](int s) { return (j0 + 2 * walk.at(s)) * 16; };
  auto edge = [&](int s) { return first_of(s) < all_lo || first_of(s) + kTokens > all_hi; };
  uint32_t odd = 0;                                    // infinities or NaN among V where there are masks
  auto publish = [&](int s, int slot) {
    if (edge(s)) {
      const int t0 = first_of(s);
      if (t0 < lo || t0 + kTokens > hi) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int t = t0 + lrow + 16 * i;
          if (t < lo || t >= hi) {
            rk[i] = u32x4_t{0, 0, 0, 0};
            rv[i] = u32x4_t{0, 0, 0, 0};
          }
        }
      }
      keep_finite(rv, odd);
    }
    lds_u8_t* st = smem + slot * kStageBytes<D>;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      *reinterpret_cast<lds_u32x4_t*>(st + k_off<D>(16 * i + lrow, lchunk)) = rk[i];
      *reinterpret_cast<lds_u32x4_t*>(st + kVOffset<D> + v_off<D>(16 * i + lrow, lchunk)) = rv[i];
    }
  };
  lds_f32_t* rowv = reinterpret_cast<lds_f32_t*>(smem + kBigRow<D>) + wave * kBiasedTileRows;

  load(0);
  publish(0, 0);
  load(1);
  publish(1, 1);
  load(2);
  __syncthreads();
  auto linear = [&](int s) { return first_of(s) + kTokens <= from_pos + 1; };
  floatx16_t raw, a;
  if (busy) {
    raw = C.scores(smem, h, n, query);
    a = C.shape(p, raw, first_of(0), h);
    C.reshape(p, a, raw, first_of(0), edge(0), linear(0), h);
    C.raise(a, rowv, h, n);
  }
  for (int s0 = 0; s0 < nstage; s0 += kSlots) {
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      const int s = s0 + u;
      if (s < nstage) {                                // uniform over the workgroup
        publish(s + 2, (u + 2) % kSlots);
        load(s + 3);
        if (busy) {
          // trees: at raised priority, so that the SIMD's other wavefront publishes and loads
          // beside the products (64 trees of 13..32 nodes over 2300 tokens 118 -> 115 us)
          if constexpr (TREE) __builtin_amdgcn_s_setprio(1);
          raw = C.scores(smem + (u + 1) % kSlots * kStageBytes<D>, h, n, query);
          C.attend(a, smem + u * kStageBytes<D>, lane);
          if constexpr (TREE) __builtin_amdgcn_s_setprio(0);
          a = C.shape(p, raw, first_of(s + 1), h);
          if (s + 1 < nstage) {
            C.reshape(p, a, raw, first_of(s + 1), edge(s + 1), linear(s + 1), h);
            C.raise(a, rowv, h, n);
          }
        }
        __syncthreads();
      }
    }
  }

  // Every wavefront is past the last barrier: the stages are free.
  {
    lds_i32_t* flag = reinterpret_cast<lds_i32_t*>(smem + kBigRange<D>);
    if (lane == 0) flag[wave] = 0;
    if (__builtin_amdgcn_ballot_w64(odd != 0) != 0 && lane == 0) flag[wave] = 1;
    __syncthreads();
    if (wave_uniform(flag[0] | flag[1] | flag[2] | flag[3]) != 0)
      special_pass<D>(C, p, bt, vbase, walk, cnt, j0, 0, 1, all_lo, all_hi, smem + wave * (kBiasedTileRows * D * 2), rowv);
  }

  // Normalise, transpose through LDS and write bf16 rows in 16-byte pieces.
  float lx = C.l, ly = C.l;
  swap32(lx, ly);
  const float lcol = lx + ly;
  float inv[16];
  Cols::per_row(rowv, h, n, lcol == 0.f ? 0.f : 1.0f / lcol, inv);
  if constexpr (TREE) {
    if (p.parts > 1 && h == 0 && turn * kBiasedTileRows + n < p.tile_rows)
      p.part_lse[slot + n] = !split ? kWhole : (lcol == 0.f ? -__builtin_inff() : C.m + log2f(lcol));
    if (split) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int at = 8 * (r >> 2) + 4 * h + (r & 3);
        if (row0 + at < rows)
#pragma unroll
          for (int j = 0; j < D / 32; ++j) store_partial(p.part_o + (slot + at) * D + 32 * j + n, C.o[j][r] * inv[r]);
      }
      return;
    }
  }
  lds_u8_t* out = smem + wave * (kBiasedTileRows * D * 2);
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int j = 0; j < D / 32; j += 2) {
      const uint32_t x = pack_bf16(C.o[j][r] * inv[r], C.o[j + 1][r] * inv[r]);
      lds_u16_t* dst = reinterpret_cast<lds_u16_t*>(out + (8 * (r >> 2) + 4 * h + (r & 3)) * (D * 2) + (32 * j + n) * 2);
      dst[0] = (uint16_t)x;
      dst[32] = (uint16_t)(x >> 16);
    }
  __builtin_amdgcn_wave_barrier();
  constexpr int kRowsPerStore = 64 / kChunks;
#pragma unroll
  for (int i = 0; i < kBiasedTileRows / kRowsPerStore; ++i) {
    const int r = row0 + kRowsPerStore * i + lane / kChunks;
    const u32x4_t x = *reinterpret_cast<const lds_u32x4_t*>(out + i * 1024 + lane * 16);
    if (r < rows)
      *reinterpret_cast<u32x4_t*>(p.out + ((size_t)(c.start + r / p.group) * p.num_q_heads + g * p.group + r % p.group) * D +
                                  lane % kChunks * 8) = x;
  }
}

// Merge of the partitions of row `r` of a row tile: weights 2^(lse - max lse),
// NW wavefronts per row, D / 64 dims per lane.  Lane q loads lse_q (64
// partitions per round); the rows of the partitions that hold something are
// dealt to the wavefronts in groups of kGroup that are loaded together, and the
// wavefronts' sums are added in order through LDS.
constexpr int kGroup = 8;
template <int D, int NW, int ROWS = kBiasedTileRows>
__device__ __forceinline__ void merge_body(const BiasedParams& p, int slot0, int r, int wave, lds_f32_t* smem) {
  constexpr int DPL = D / 64;
  const int lane = threadIdx.x & 63;
  int wg = slot0;
  const int g = wg % p.num_kv_heads;
  wg /= p.num_kv_heads;
  const int tile = wg % p.tiles;
  const int b = wg / p.tiles;
  const float* lse = p.part_lse + (size_t)slot0 * p.parts * p.tile_rows + r;
  const float x0 = lane < p.parts ? lse[lane * p.tile_rows] : -__builtin_inff();
  const float* po = p.part_o + ((size_t)slot0 * p.parts * p.tile_rows + r) * D + DPL * lane;
  // Where rows are few (NW > 1) the first group is loaded before lse tells which
  // partitions hold something; what the others' slots hold is not used.
  float v[kGroup][DPL];
  auto load_group = [&](int first, uint64_t some) {
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const bool has = (some >> k) & 1;                           // uniform
#pragma unroll
      for (int d = 0; d < DPL; ++d) v[k][d] = has ? po[(size_t)(first + k) * p.tile_rows * D + d] : 0.f;
    }
  };
  if constexpr (NW > 1) load_group(wave * kGroup, p.parts > wave * kGroup ? ~0ull >> (64 - min(p.parts - wave * kGroup, 64)) : 0);
  const Chunk c = chunk_of(p, b);
  const int R = tile * ROWS + r;
  if (R >= c.len * p.group) return;                             // all wavefronts of the row
  if (__int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x0))) == kWhole) return;
  float mx = x0;
  for (int c0 = 64; c0 < p.parts; c0 += 64)
    if (c0 + lane < p.parts) mx = fmaxf(mx, lse[(c0 + lane) * p.tile_rows]);
  mx = group_max4(row_max16(mx));
  const float mref = mx == -__builtin_inff() ? 0.f : mx;
  float sum = 0.f, acc[DPL];
#pragma unroll
  for (int d = 0; d < DPL; ++d) acc[d] = 0.f;
  for (int c0 = 0; c0 < p.parts; c0 += 64) {
    float x = x0;
    if (c0 > 0) x = c0 + lane < p.parts ? lse[(c0 + lane) * p.tile_rows] : -__builtin_inff();
    // partitions that hold something come first: the others begin past the row's last token
    const uint64_t some = __builtin_amdgcn_ballot_w64(x != -__builtin_inff());
    if (some == 0) continue;
    const int cnt = 64 - __builtin_clzll(some);
    const int wl = __float_as_int(fast_exp2(x - mref));
    for (int j0 = wave * kGroup; j0 < cnt; j0 += NW * kGroup) {
      const uint64_t here = some >> j0;
      if (NW == 1 || c0 + j0 > wave * kGroup) load_group(c0 + j0, here);
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        if (!((here >> k) & 1)) continue;
        const float w = __int_as_float(__builtin_amdgcn_readlane(wl, j0 + k));
        sum += w;
#pragma unroll
        for (int d = 0; d < DPL; ++d) acc[d] = fmaf(w, v[k][d], acc[d]);
      }
    }
  }
  if constexpr (NW > 1) {
    lds_f32_t* so = smem;                                       // [NW][D], then [NW] sums
    lds_f32_t* sw = smem + NW * D;
#pragma unroll
    for (int d = 0; d < DPL; ++d) so[wave * D + DPL * lane + d] = acc[d];
    if (lane == 0) sw[wave] = sum;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      sum += sw[w];
#pragma unroll
      for (int d = 0; d < DPL; ++d) acc[d] += so[w * D + DPL * lane + d];
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  uint16_t* dst = p.out + ((size_t)(c.start + R / p.group) * p.num_q_heads + g * p.group + R % p.group) * D;
  if constexpr (DPL == 2)
    *reinterpret_cast<uint32_t*>(dst + 2 * lane) = pack_bf16(acc[0] * inv, acc[1] * inv);
  else
    dst[lane] = (uint16_t)pack_bf16(acc[0] * inv, 0.f);
}

}  // namespace biased
}  // namespace pa
