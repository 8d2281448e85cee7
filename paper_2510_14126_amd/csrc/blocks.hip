// Bounds of the keys of blocks, and the choice of each query's blocks by them
// (gfx950, head_dim 64 or 128).
#include "choose_body.h"
#include "tokens.h"

#include <algorithm>

namespace pa {
namespace {

__device__ __forceinline__ int clamped(int x, int most) { return x < 0 ? 0 : (x > most ? most : x); }

// ---- bounds ----------------------------------------------------------------
// One wavefront per (sequence, block of its new tokens, KV head): 16 bytes of a key
// row per lane, 1 KiB of rows per load, all of the tile at once; least and greatest
// over the lanes' rows, then over the lanes that hold the same dims.  It reads 4 KiB
// (D = 128) and writes 512 bytes: a step's newest blocks are launch-bound.
template <int D>
__global__ void __launch_bounds__(256) bounds_kernel(const BlocksParams p, int blocks) {
  constexpr int kRowLanes = D / 8;                 // lanes per key row
  constexpr int kRows = 64 / kRowLanes;            // rows per load
  const int lane = threadIdx.x & 63;
  int64_t item = (int64_t)blockIdx.x * 4 + wave_uniform(threadIdx.x >> 6);
  if (item >= (int64_t)p.batch * blocks * p.num_kv_heads) return;
  const int g = (int)(item % p.num_kv_heads);
  item /= p.num_kv_heads;
  const int j = (int)(item % blocks), b = (int)(item / blocks);
  const int ctx = clamped(p.context_lens[b], p.max_ctx);
  int first = p.first_tokens ? clamped(p.first_tokens[b], ctx) : 0;
  first = max(first, ctx - p.max_new);
  const int block = (first >> 4) + j;
  const int valid = min(16, ctx - 16 * block);     // tokens of the block
  if (first >= ctx || valid <= 0) return;
  const int id = clamped(p.block_tables[(size_t)b * p.bt_stride + block], p.num_blocks - 1);
  const uint16_t* tile = p.k_pool + ((size_t)id * p.num_kv_heads + g) * (16 * D);
  uint4 x[16 / kRows];
#pragma unroll
  for (int i = 0; i < 16 / kRows; ++i) x[i] = *reinterpret_cast<const uint4*>(tile + (size_t)i * 512 + lane * 8);
  float lo[8], hi[8];
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    lo[d] = __builtin_inff();
    hi[d] = -__builtin_inff();
  }
#pragma unroll
  for (int i = 0; i < 16 / kRows; ++i) {
    if (i * kRows + lane / kRowLanes >= valid) continue;
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const float y = d & 1 ? bf16_hi(w[d / 2]) : bf16_lo(w[d / 2]);
      lo[d] = fminf(lo[d], y);                     // of a NaN and a number the number
      hi[d] = fmaxf(hi[d], y);
    }
  }
#pragma unroll
  for (int m = kRowLanes; m < 64; m <<= 1)
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      lo[d] = fminf(lo[d], __shfl_xor(lo[d], m));
      hi[d] = fmaxf(hi[d], __shfl_xor(hi[d], m));
    }
  if (lane < 2 * kRowLanes) {
    const bool upper = lane >= kRowLanes;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {                  // the values are bf16 as they are
      const uint32_t a = __float_as_uint(upper ? hi[2 * k] : lo[2 * k]), c = __float_as_uint(upper ? hi[2 * k + 1] : lo[2 * k + 1]);
      w[k] = (a >> 16) | (c & 0xffff0000u);
    }
    *reinterpret_cast<uint4*>(p.bounds + ((size_t)id * p.num_kv_heads + g) * (2 * D) + lane * 8) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ---- scores ----------------------------------------------------------------
// max(q lo, q hi) is q hi for q >= 0 and q lo for q < 0, so a block's score over the
// heads of a KV head is one product of its 2 D bounds with the sums of the heads'
// negative and positive parts.  Products and sums are fp64: products of bf16 and
// their sums are then exact up to parts of 2^-53, so that the choice between two
// close blocks does not hang on the order of a sum.  The vector unit's fp64 rate is
// that of its scalar fp32, and what bounds the pass is reading the bounds, 4 D bytes
// a block and KV head, a sixteenth of its keys and values.
//
// D / 4 lanes read a block's bounds, 16 bytes each, with the non-temporal hint (the
// step of 64 sequences below 159 -> 153 us); a wavefront has kLoads loads in
// flight for its next round while it sums the blocks of this one.  The lanes' partial
// sums are exchanged so that each step halves the blocks a lane still holds.
constexpr int kLoads = 8;
template <int D> constexpr int kGroups = 64 / (D / 4);                // blocks per load
template <int D> constexpr int kRoundBlocks = kLoads * kGroups<D>;    // blocks per wavefront and round
constexpr int kWaves = 4;
// Rounds of a wavefront: as many as leave the GPU full (kFillWaves), so that the chain
// of loads before a wavefront's first round (length, table, bounds) and its sums of q
// are paid once for several, and few, so that the last ones end together.  Whole steps,
// 64 sequences of 4097..28672 tokens, 32 heads over 8 (28 rounds to fill), with 1 / 2 / 3
// / 4 / 8 / 11: 174 / 176 / 153 / 154 / 157 / 159 us; 16 of them (7) 64.5 / 59.5 with 2.
// Four / two / one wavefronts per SIMD to fill: one of 131003 tokens, 64 heads over 8, 43.8 /
// 43.8 / 42.9, four, heads over 4, D = 64, 50.5 / 44.7 / 45.4, four of 32000, 32 over 8, 25.8 /
// 24.9 / 26.4.
constexpr int kFillWaves = 2 * 1024, kMostRounds = 4;
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef short i16x2_t __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ double moved(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xf, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
constexpr int kDppHalfMirror = 0x141;   // lane i of eight gets lane 7 - i's

// a of the lanes with the bit M clear and b of those with it set, each plus the same
// value of a lane that has the bit the other way round.  (Which one does not matter:
// the lanes below M are summed later.)
template <int M>
__device__ __forceinline__ double folded(double a, double b, int lane) {
  if constexpr (M == 16) {
    const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
    const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)y, false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(x >> 32), (uint32_t)(y >> 32), false, false);
    return __builtin_bit_cast(double, ((uint64_t)hi[0] << 32) | lo[0]) + __builtin_bit_cast(double, ((uint64_t)hi[1] << 32) | lo[1]);
  } else {
    constexpr int kCtrl = M == 8 ? kDppRowRor8 : (M == 4 ? kDppHalfMirror : (M == 2 ? kDppQuadXor2 : kDppQuadXor1));
    const bool up = (lane & M) != 0;
    return (up ? b : a) + moved<kCtrl>(up ? a : b);
  }
}

// Candidates of a sequence: how many blocks lie between its first and last ones;
// 0 where it attends to all of them.
__device__ __forceinline__ int candidates(const BlocksParams& p, int nblk) {
  return nblk <= p.max_blocks ? 0 : nblk - p.first_blocks - p.last_blocks;
}

// One wavefront's candidates of (sequence b, KV head g), `rounds` rounds from `base` on.
// store(i, key): candidate i.
template <int D, typename Store>
__device__ __forceinline__ void score_blocks(const BlocksParams& p, int b, int g, int base, int rounds, const Store& store) {
  constexpr int kLanes = D / 4;                    // lanes per block
  constexpr int kPer = kRoundBlocks<D>;
  const int lane = threadIdx.x & 63;
  const int part = lane / kLanes, piece = lane % kLanes;
  // the lane's side: pieces of the least values meet the negative parts of q
  const bool upper = piece >= kLanes / 2;
  const uint16_t* q_row = p.q + ((size_t)b * p.num_kv_heads + g) * p.group * D + piece % (kLanes / 2) * 8;
  // the first heads' q before all else: it is summed while the bounds are on their way (one
  // sequence of 131003 tokens, 64 heads over 8, 43.8 -> 36.5 us, of 300 14.9 -> 13.3; read four
  // heads at a time behind the bounds before)
  constexpr int kEarly = 8;
  uint4 early[kEarly];
#pragma unroll
  for (int h = 0; h < kEarly; ++h) early[h] = *reinterpret_cast<const uint4*>(q_row + (size_t)min(h, p.group - 1) * D);
  // 64 table entries at a time, and the 64 behind them; the first before the length is there
  const int32_t* table = p.block_tables + (size_t)b * p.bt_stride + p.first_blocks;
  const int most = min(p.key_blocks - p.first_blocks, base + rounds * kPer);
  auto ids_from = [&](int at) { return at + lane < most ? clamped(table[at + lane], p.num_blocks - 1) : 0; };
  int ids = ids_from(base), ids_next = ids_from(base + 64);
  const int ctx = clamped(p.context_lens[b], p.max_ctx);
  const int n = candidates(p, (ctx + 15) >> 4);
  const int end = min(n, base + rounds * kPer);
  if (base >= end) return;
  const uint16_t* bounds = p.bounds + (size_t)g * (2 * D) + piece * 8;
  const size_t stride = (size_t)p.num_kv_heads * (2 * D);

  auto load = [&](u32x4_t (&x)[kLoads], int at) {    // at - base: a multiple of kPer, which divides 64
    if (at > base && ((at - base) & 63) == 0) {
      ids = ids_next;
      ids_next = ids_from(at + 64);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const size_t id = (size_t)__shfl(ids, ((at - base) & 63) + i * kGroups<D> + part);
      x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(bounds + id * stride));
    }
  };
  u32x4_t x[2][kLoads];
  load(x[0], base);

  // Sums of the parts' magnitudes: with the lower side's signs flipped, bf16 that are
  // negative as 16-bit integers have no part.  (So has a NaN on one of the sides.)
  const uint32_t flip = upper ? 0u : 0x80008000u;
  double q[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  auto add = [&](const uint4& y) {
    const uint32_t w[4] = {y.x ^ flip, y.y ^ flip, y.z ^ flip, y.w ^ flip};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t z = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2_t, w[k]), i16x2_t{0, 0}));
      q[2 * k] += (double)bf16_lo(z);
      q[2 * k + 1] += (double)bf16_hi(z);
    }
  };
#pragma unroll
  for (int h = 0; h < kEarly; ++h)
    if (h < p.group) add(early[h]);                // uniform
#pragma unroll 4
  for (int h = kEarly; h < p.group; ++h) add(*reinterpret_cast<const uint4*>(q_row + (size_t)h * D));
#pragma unroll
  for (int d = 0; d < 8; ++d) q[d] = upper ? q[d] : -q[d];

  auto score = [&](u32x4_t (&y)[kLoads], int at) {
    double v[kLoads];
    int i;
    for (bool again = false;; again = true) {
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        const uint32_t w[4] = {y[k][0], y[k][1], y[k][2], y[k][3]};
        v[k] = 0.0;
#pragma unroll
        for (int d = 0; d < 8; ++d) v[k] = fma(q[d], (double)(d & 1 ? bf16_hi(w[d / 2]) : bf16_lo(w[d / 2])), v[k]);
      }
      // lane bits from the block's highest on choose which half stays
      if constexpr (kLanes == 32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = folded<16>(v[k], v[k + 4], lane);
#pragma unroll
        for (int k = 0; k < 2; ++k) v[k] = folded<8>(v[k], v[k + 2], lane);
        v[0] = folded<4>(v[0], v[1], lane);
        v[0] += moved<kDppQuadXor2>(v[0]);
        i = ((lane & 16) >> 2) | ((lane & 8) >> 2) | ((lane & 4) >> 2);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = folded<8>(v[k], v[k + 4], lane);
#pragma unroll
        for (int k = 0; k < 2; ++k) v[k] = folded<4>(v[k], v[k + 2], lane);
        v[0] = folded<2>(v[0], v[1], lane);
        i = ((lane & 8) >> 1) | ((lane & 4) >> 1) | ((lane & 2) >> 1);
      }
      v[0] += moved<kDppQuadXor1>(v[0]);
      // A bound that no head's q looks at (no positive part over the greatest, no negative
      // one over the least) may be infinite, and 0 times it is NaN: once more without those.
      if (again || __builtin_amdgcn_ballot_w64(v[0] != v[0]) == 0) break;
#pragma unroll
      for (int d = 0; d < 8; ++d)
        if (q[d] == 0.0)
#pragma unroll
          for (int k = 0; k < kLoads; ++k) y[k][d / 2] &= d & 1 ? 0x0000ffffu : 0xffff0000u;
    }
    const int block = at + i * kGroups<D> + part;
    if (block < end && lane % (kLanes / kLoads) == 0) store(block, choose::key_of(v[0]));
  };
  for (int at = base; at < end; at += 2 * kPer) {
    if (at + kPer < end) load(x[1], at + kPer);    // uniform
    score(x[0], at);
    if (at + kPer >= end) break;
    if (at + 2 * kPer < end) load(x[0], at + 2 * kPer);
    score(x[1], at + kPer);
  }
}

template <int D>
__global__ void __launch_bounds__(64 * kWaves) score_kernel(const BlocksParams p, int rounds) {
  const int wave = wave_uniform(threadIdx.x >> 6);
  int wg = blockIdx.x;
  const int g = wg % p.num_kv_heads;
  wg /= p.num_kv_heads;
  const int b = wg % p.batch;
  uint64_t* keys = p.keys + ((size_t)b * p.num_kv_heads + g) * p.key_blocks;
  score_blocks<D>(p, b, g, (wg / p.batch * kWaves + wave) * rounds * kRoundBlocks<D>, rounds,
                  [&](int i, uint64_t key) { keys[i] = key; });
}

// ---- choice ----------------------------------------------------------------
// One workgroup per (sequence, KV head): of 512 threads up to kFewKeys candidates, else of
// 1024 (256 / 512 / 1024 threads, one sequence of 1000 blocks 18.1 / 17.7 us, of 2000 20.0 /
// 18.5; of 4000 - / 21.6 / 20.8, of 8100 - / 28.3 / 25.6).
//
// Up to kFewKeys it can make the keys itself: a launch less, no keys through memory, and
// while some workgroups choose others still read, but four wavefronts to a row.  It does
// where the rows fill the GPU (kManyRows), or the candidates are few (kOwnRounds of each
// wavefront).  Whole steps, 32 heads over 8, scores in a launch of their own / here: one
// sequence of 256 / 320 / 500 blocks 16.4 / 17.9, 17.0 / 19.3, 17.2 / 22.7 us, four of 256 /
// 320 17.2 / 18.6, 17.5 / 19.9 (before q was summed ahead of the bounds one of 64 / 128 17.7 /
// 15.8, 18.3 / 17.2; 32, that is 256 rows, of 500 / 2000 32.2 / 30.9, 70.3 / 67.0; 128 of 500 /
// 1000 / 2000 82.8 / 75.4, 130.7 / 115, 228 / 195).  Eight wavefronts to a row from
// kLongRounds rounds on (four / eight: 32 of 500 / 1000 / 2000 31.0 / 30.3, 43.4 / 41.1, 67.3 /
// 62.8; 128 of 256 / 500 / 1000 / 2000 55.2 / 60.3, 75.4 / 77.4, 115.5 / 115.9, 195 / 193.5; 32
// of 125..2000 58.1 / 49.7).
constexpr int kFewKeys = 2048, kManyKeys = 16384;
constexpr int kOwnRounds = 3, kManyRows = 256, kLongRounds = 33;
template <int THREADS, int CAPACITY, typename Keys>
__device__ __forceinline__ void select_row(const BlocksParams& p, int b, int g, int n, int nblk, choose::Scratch& scratch,
                                           uint64_t* room, const Keys& keys) {
  int32_t* out = p.selected + ((size_t)b * p.num_kv_heads + g) * p.max_blocks;
  const int bound = p.key_blocks > p.max_blocks ? p.key_blocks - p.first_blocks - p.last_blocks : 0;
  const int want = n > 0 ? p.max_blocks - p.first_blocks - p.last_blocks : 0;     // < n
  choose::choose<uint64_t, THREADS, CAPACITY>(bound, n, want, scratch, room, keys,
                                              [&](int rank, int i) { out[p.first_blocks + rank] = p.first_blocks + i; });
  if (n <= 0) {                                                       // all of them
    for (int i = threadIdx.x; i < p.max_blocks; i += THREADS) out[i] = i < nblk ? i : -1;
    return;
  }
  for (int i = threadIdx.x; i < p.first_blocks; i += THREADS) out[i] = i;
  for (int i = threadIdx.x; i < p.last_blocks; i += THREADS)
    out[p.max_blocks - p.last_blocks + i] = nblk - p.last_blocks + i;
}

template <int D, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) select_own_kernel(const BlocksParams p, int rounds) {
  __shared__ choose::Scratch scratch;
  __shared__ uint64_t room[kFewKeys];
  const int g = blockIdx.x % p.num_kv_heads, b = blockIdx.x / p.num_kv_heads;
  const int wave = wave_uniform(threadIdx.x >> 6);
  score_blocks<D>(p, b, g, wave * rounds * kRoundBlocks<D>, rounds, [&](int i, uint64_t key) { room[i] = key; });
  const int nblk = (clamped(p.context_lens[b], p.max_ctx) + 15) >> 4;
  __syncthreads();
  select_row<64 * WAVES, kFewKeys>(p, b, g, candidates(p, nblk), nblk, scratch, room, [&](int i) { return room[i]; });
}

template <int THREADS, int CAPACITY>
__global__ void __launch_bounds__(THREADS) select_kernel(const BlocksParams p) {
  __shared__ choose::Scratch scratch;
  __shared__ uint64_t room[CAPACITY];
  const int g = blockIdx.x % p.num_kv_heads, b = blockIdx.x / p.num_kv_heads;
  const uint64_t* keys = p.keys + ((size_t)b * p.num_kv_heads + g) * p.key_blocks;
  const int nblk = (clamped(p.context_lens[b], p.max_ctx) + 15) >> 4;
  select_row<THREADS, CAPACITY>(p, b, g, candidates(p, nblk), nblk, scratch, room, [&](int i) { return keys[i]; });
}

}  // namespace

hipError_t launch_bounds(const BlocksParams& p, hipStream_t stream) {
  const int blocks = (p.max_new + 14) / 16 + 1;        // that max_new tokens can lie in
  const int64_t items = (int64_t)p.batch * blocks * p.num_kv_heads;
  const dim3 grid((unsigned)((items + 3) / 4));
  if (p.head_dim == 128)
    hipLaunchKernelGGL(bounds_kernel<128>, grid, dim3(256), 0, stream, p, blocks);
  else
    hipLaunchKernelGGL(bounds_kernel<64>, grid, dim3(256), 0, stream, p, blocks);
  return hipGetLastError();
}

hipError_t launch_select(const BlocksParams& p, hipStream_t stream) {
  const int64_t rows = (int64_t)p.batch * p.num_kv_heads;
  const int n = p.key_blocks > p.max_blocks ? p.key_blocks - p.first_blocks - p.last_blocks : 0;   // candidates at most
  const int per = p.head_dim == 128 ? kRoundBlocks<128> : kRoundBlocks<64>;
  const int n_rounds = (n + per - 1) / per;
  const dim3 all((unsigned)rows), wg(64 * kWaves);
  if (n > 0 && n <= kFewKeys && (n_rounds <= kOwnRounds * kWaves || rows >= kManyRows)) {
    auto go = [&](auto kernel, int waves) {
      hipLaunchKernelGGL(kernel, all, dim3(64 * waves), 0, stream, p, (n_rounds + waves - 1) / waves);
    };
    if (n_rounds >= kLongRounds)
      go(p.head_dim == 128 ? select_own_kernel<128, 8> : select_own_kernel<64, 8>, 8);
    else
      go(p.head_dim == 128 ? select_own_kernel<128, 4> : select_own_kernel<64, 4>, 4);
    return hipGetLastError();
  }
  if (n > 0) {
    const int rounds = (int)std::min<int64_t>(kMostRounds, std::max<int64_t>(1, rows * n_rounds / kFillWaves));
    const dim3 grid((unsigned)(rows * ((n_rounds + kWaves * rounds - 1) / (kWaves * rounds))));
    if (p.head_dim == 128)
      hipLaunchKernelGGL(score_kernel<128>, grid, wg, 0, stream, p, rounds);
    else
      hipLaunchKernelGGL(score_kernel<64>, grid, wg, 0, stream, p, rounds);
  }
  if (n <= kFewKeys)
    hipLaunchKernelGGL((select_kernel<512, kFewKeys>), all, dim3(512), 0, stream, p);
  else
    hipLaunchKernelGGL((select_kernel<1024, kManyKeys>), all, dim3(1024), 0, stream, p);
  return hipGetLastError();
}

}  // namespace pa
