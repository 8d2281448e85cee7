// Bounds of the keys of blocks, and the choice of each query's blocks by them
// (gfx950, head_dim 64 or 128).
#include "choose_body.h"
#include "tokens.h"

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
// D / 4 lanes read a block's bounds, 16 bytes each, kLoads loads in flight per
// wavefront; their partial sums are exchanged so that each step halves the blocks a
// lane still holds: 16 additions for 16 blocks.
constexpr int kLoads = 16;
template <int D> constexpr int kGroups = 64 / (D / 4);                // blocks per load
template <int D> constexpr int kWaveBlocks = kLoads * kGroups<D>;     // blocks per wavefront and round

__device__ __forceinline__ double exchanged(double x, int m) {
  return __builtin_bit_cast(double, __shfl_xor(__builtin_bit_cast(unsigned long long, x), m));
}

// Candidates of a sequence: how many blocks lie between its first and last ones;
// 0 where it attends to all of them.
__device__ __forceinline__ int candidates(const BlocksParams& p, int nblk) {
  return nblk <= p.max_blocks ? 0 : nblk - p.first_blocks - p.last_blocks;
}

template <int D>
__global__ void __launch_bounds__(256) score_kernel(const BlocksParams p) {
  constexpr int kLanes = D / 4;                    // lanes per block
  const int lane = threadIdx.x & 63;
  const int wave = wave_uniform(threadIdx.x >> 6);
  int wg = blockIdx.x;
  const int g = wg % p.num_kv_heads;
  wg /= p.num_kv_heads;
  const int b = wg % p.batch;
  const int base = (wg / p.batch * 4 + wave) * kWaveBlocks<D>;
  const int ctx = clamped(p.context_lens[b], p.max_ctx);
  const int n = candidates(p, (ctx + 15) >> 4);
  if (base >= n) return;
  const int32_t* table = p.block_tables + (size_t)b * p.bt_stride + p.first_blocks + base;
  const int ids = lane < kWaveBlocks<D> && base + lane < n ? clamped(table[lane], p.num_blocks - 1) : 0;
  const int part = lane / kLanes, piece = lane % kLanes;
  uint4 x[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const size_t id = (size_t)__shfl(ids, i * kGroups<D> + part);
    x[i] = *reinterpret_cast<const uint4*>(p.bounds + (id * p.num_kv_heads + g) * (2 * D) + piece * 8);
  }
  // the lane's side: pieces of the least values meet the negative parts of q
  const bool upper = piece >= kLanes / 2;
  double q[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const uint16_t* q_row = p.q + ((size_t)b * p.num_kv_heads + g) * p.group * D + piece % (kLanes / 2) * 8;
  for (int h = 0; h < p.group; ++h) {
    const uint4 y = *reinterpret_cast<const uint4*>(q_row + (size_t)h * D);
    const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const float z = d & 1 ? bf16_hi(w[d / 2]) : bf16_lo(w[d / 2]);
      q[d] += (double)((upper ? z < 0.f : z > 0.f) ? 0.f : z);        // NaN stays
    }
  }
  double v[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    v[i] = 0.0;
#pragma unroll
    for (int d = 0; d < 8; ++d) v[i] = fma(q[d], (double)(d & 1 ? bf16_hi(w[d / 2]) : bf16_lo(w[d / 2])), v[i]);
  }
  int load = 0, m = kLanes / 2;
#pragma unroll
  for (int half = kLoads / 2; half >= 1; half /= 2) {
    const bool up = (lane & m) != 0;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const double keep = up ? v[i + half] : v[i], give = up ? v[i] : v[i + half];
      v[i] = keep + exchanged(give, m);
    }
    load += up ? half : 0;
    m >>= 1;
  }
  if constexpr (kLanes == 32) v[0] += exchanged(v[0], 1);
  const int block = load * kGroups<D> + part;
  if (base + block < n && (kLanes < 32 || (lane & 1) == 0))
    p.keys[((size_t)b * p.num_kv_heads + g) * p.key_blocks + base + block] = choose::key_of(v[0]);
}

// ---- choice ----------------------------------------------------------------
// One workgroup per (sequence, KV head); the keys come from L2 once per digit.
__global__ void __launch_bounds__(choose::kThreads) select_kernel(const BlocksParams p) {
  __shared__ choose::Scratch scratch;
  const int g = blockIdx.x % p.num_kv_heads, b = blockIdx.x / p.num_kv_heads;
  const size_t row = (size_t)b * p.num_kv_heads + g;
  const int ctx = clamped(p.context_lens[b], p.max_ctx);
  const int nblk = (ctx + 15) >> 4;
  int32_t* out = p.selected + row * p.max_blocks;
  const int n = candidates(p, nblk);
  if (n <= 0) {
    for (int i = threadIdx.x; i < p.max_blocks; i += choose::kThreads) out[i] = i < nblk ? i : -1;
    return;
  }
  const int want = p.max_blocks - p.first_blocks - p.last_blocks;     // < n
  for (int i = threadIdx.x; i < p.first_blocks; i += choose::kThreads) out[i] = i;
  for (int i = threadIdx.x; i < p.last_blocks; i += choose::kThreads)
    out[p.max_blocks - p.last_blocks + i] = nblk - p.last_blocks + i;
  const uint64_t* keys = p.keys + row * p.key_blocks;
  choose::choose<uint64_t>(n, want, scratch, [&](int i) { return keys[i]; },
                           [&](int rank, int i) { out[p.first_blocks + rank] = p.first_blocks + i; });
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
  if (p.key_blocks > p.max_blocks) {                   // else every sequence attends to all of its blocks
    const int per = 4 * (p.head_dim == 128 ? kWaveBlocks<128> : kWaveBlocks<64>);
    const int64_t n = p.key_blocks - p.first_blocks - p.last_blocks;
    const dim3 grid((unsigned)(rows * ((n + per - 1) / per)));
    if (p.head_dim == 128)
      hipLaunchKernelGGL(score_kernel<128>, grid, dim3(256), 0, stream, p);
    else
      hipLaunchKernelGGL(score_kernel<64>, grid, dim3(256), 0, stream, p);
  }
  hipLaunchKernelGGL(select_kernel, dim3((unsigned)rows), dim3(choose::kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace pa
