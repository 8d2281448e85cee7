// The tokens that stay in a cache, and their move to the front of their sequences
// (gfx950).
#include "choose_body.h"
#include "tokens.h"

namespace pa {
namespace {

__device__ __forceinline__ int clamped(int x, int most) { return x < 0 ? 0 : (x > most ? most : x); }

// ---- choice ----------------------------------------------------------------
// One workgroup per sequence: of 512 threads up to kFewKeys candidates, else of 1024 (256 /
// 512 / 1024 threads, choice and move of one sequence of 1000 tokens 12.4 / 11.9 us, of 2000
// 14.1 / 12.3; of 4000 - / 15.0 / 13.7, of 8000 - / 19.7 / 17.1).
constexpr int kFewKeys = 2048, kManyKeys = 32768;
template <int THREADS, int CAPACITY>
__global__ void __launch_bounds__(THREADS) keep_kernel(const KeepParams p) {
  __shared__ choose::Scratch scratch;
  __shared__ uint32_t room[CAPACITY];
  const int b = blockIdx.x;
  const int ctx = clamped(p.context_lens[b], p.max_ctx);
  const int first = p.first_tokens ? clamped(p.first_tokens[b], ctx) : 0;
  const int recent = min(p.recent, ctx - first);
  const int n = ctx - first - recent;                                   // candidates
  const int want = min(max(p.keep - first - recent, 0), n);
  int32_t* out = p.kept + (size_t)b * p.kept_stride;
  for (int i = threadIdx.x; i < recent; i += THREADS) out[want + i] = n + i;
  for (int i = want + recent + threadIdx.x; i < p.kept_stride; i += THREADS) out[i] = -1;
  if (threadIdx.x == 0) p.kept_lens[b] = want + recent;
  const float* totals = p.totals + (size_t)b * p.totals_stride + first;
  choose::choose<uint32_t, THREADS, CAPACITY>(p.max_ctx - first, n, want, scratch, room, [&](int i) { return choose::key_of(totals[i]); },
                                              [&](int rank, int i) { out[rank] = i; });
}

// ---- move ------------------------------------------------------------------
// A workgroup moves the rows of one (sequence, KV head, pool), kMovePasses x 256 pieces
// of 16 bytes at a time: all of them loaded, a barrier, all of them stored.  In place
// that is enough.  A row moves to a slot at or before its own, and what a later
// round reads lies behind every slot that this one writes (kept ascends, so row j's
// source is at least slot j), so only the rows of one round can stand in each
// other's way.  To other blocks the rounds are workgroups of their own (chunks).  In place
// they wait for one another: right for an accepted path, slow for a few long lists, whose
// workgroups are few (8 KV heads of 128, 16384 of 30000 tokens of one sequence 837 us, to
// other blocks 41; 4096 each of 64 sequences 529 / 450).
//
// The rows are read and written once; nothing but their traffic bounds the move.  It
// reads and writes them with the non-temporal hint, and the KV heads run fastest over
// the workgroups, then the rounds: neighbouring workgroups then move the rows of
// the same tokens, 256 bytes of each block's neighbouring tiles.  64 sequences of
// 3001..15000 tokens cut to 4096, 1.5 GB read and written: rounds fastest 640 us, heads
// fastest 505, with the hint on loads / stores / both 347 / 343 / 337 (4.6 TB/s, a copy of
// 1 GiB runs at 5.0); one of 30000 cut to 16384, with its choice, 117 / 93 / 89 / 81 (no hint
// / ...; 66 with the later choice, the move alone 41).
constexpr int kPasses = kMovePasses;
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// The loads before this line have arrived in every thread of the workgroup.
__device__ __forceinline__ void all_loaded() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// What a sequence keeps: its first tokens, and how many of its list move behind them.  A
// sequence that is shorter than its first tokens keeps what it has, and nothing moves: it must
// not grow to tokens that it never held.
//
// new_lens may be context_lens, so another workgroup may have written first + moved there
// already: that gives the same two numbers again (first <= context: first is below the sum,
// and moved does not depend on the context; else the sum is the context and moved 0).
struct Stay {
  int first, moved;
};
__device__ __forceinline__ Stay stay_of(const CompactParams& p, int b) {
  const int lists = p.kept_lens[b], given = p.first_tokens ? p.first_tokens[b] : 0, len = p.context_lens[b];   // together
  const int ctx = clamped(len, p.max_ctx), first = clamped(given, p.max_ctx);
  const int moved = clamped(lists, min(p.kept_stride, p.max_ctx - first));
  return {min(first, ctx), first <= ctx ? moved : 0};
}

// AHEAD: the first round's entries of the list are loaded before its length is there.
// That is a link less in the chain of loads (lengths, list, table, rows), which is the
// time of a small move, and registers, which large ones miss: four sequences cut to 256
// tokens 12.5 -> 10.9 us (66 workgroups), two cut to 2048 26.6 -> 25.6 (514); 100 trees of
// 8..32 nodes 10.7 -> 11.1 (1700), 64 cut to 4096 364 -> 381.
constexpr int64_t kAheadWorkgroups = 1024;
template <int D, bool AHEAD>
__device__ __forceinline__ void move_rows(const CompactParams& p, int wg) {
  constexpr int kRowThreads = D / 8;
  constexpr int kRows = kMoveThreads / kRowThreads;                     // per pass
  const int g = wg % p.num_kv_heads;
  wg /= p.num_kv_heads;
  const int chunk = wg % p.chunks;
  wg /= p.chunks;
  uint16_t* pool = wg & 1 ? p.v_pool : p.k_pool;
  const int b = wg >> 1;
  const int32_t* kept = p.kept + (size_t)b * p.kept_stride;
  const int row = threadIdx.x / kRowThreads, piece = threadIdx.x % kRowThreads;
  const int own0 = chunk * kPasses * kRows;
  int early[AHEAD ? kPasses : 1];
  if constexpr (AHEAD) {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) early[i] = own0 + i * kRows + row < p.kept_stride ? kept[own0 + i * kRows + row] : 0;
  }
  const auto [first, m] = stay_of(p, b);
  const int32_t* from = p.block_tables + (size_t)b * p.bt_stride;
  const int32_t* to = p.dst_tables ? p.dst_tables + (size_t)b * p.dst_stride : from;
  const int to_blocks = p.dst_tables ? p.dst_stride : p.bt_stride;
  auto slot = [&](int id, int t) {
    return pool + (((size_t)clamped(id, p.num_blocks - 1) * p.num_kv_heads + g) * 16 + (t & 15)) * D + piece * 8;
  };
  for (int j0 = own0; j0 < m; j0 += p.chunks * kPasses * kRows) {   // uniform
    u32x4_t x[kPasses];
    uint16_t* dst[kPasses];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int j = j0 + i * kRows + row;
      dst[i] = nullptr;
      if (j < m && (first + j) >> 4 < to_blocks) {
        const int at = AHEAD && j0 == own0 ? early[AHEAD ? i : 0] : kept[j];
        const int s = clamped(at, p.max_ctx - 1 - first) + first;
        const uint16_t* src = slot(from[s >> 4], s);
        dst[i] = slot(to[(first + j) >> 4], first + j);
        if (dst[i] == src)
          dst[i] = nullptr;                                             // it stays where it is
        else
          x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(src));
      }
    }
    all_loaded();
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
      if (dst[i]) __builtin_nontemporal_store(x[i], reinterpret_cast<u32x4_t*>(dst[i]));
  }
}

// A sequence's totals, in the same way, and its new length.
__device__ __forceinline__ void move_totals(const CompactParams& p, int b) {
  const auto [first, m] = stay_of(p, b);
  const int ctx = clamped(p.context_lens[b], p.max_ctx);
  if (p.totals_out) {
    const int32_t* kept = p.kept + (size_t)b * p.kept_stride;
    const float* in = p.totals + (size_t)b * p.totals_stride;
    float* out = p.totals_out + (size_t)b * p.totals_stride;
    if (in != out)
      for (int t = threadIdx.x; t < min(first, ctx); t += kMoveThreads) out[t] = in[t];
    for (int j0 = 0; j0 < m; j0 += kPasses * kMoveThreads) {
      float x[kPasses];
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const int j = j0 + i * kMoveThreads + threadIdx.x;
        x[i] = j < m ? in[first + clamped(kept[j], p.max_ctx - 1 - first)] : 0.f;
      }
      all_loaded();
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const int j = j0 + i * kMoveThreads + threadIdx.x;
        if (j < m) out[first + j] = x[i];
      }
    }
    for (int t = first + m + threadIdx.x; t < ctx; t += kMoveThreads) out[t] = 0.f;
  }
  all_loaded();                                                         // new_lens may be context_lens
  if (threadIdx.x == 0 && p.new_lens) p.new_lens[b] = first + m;
}

template <int D, bool AHEAD>
__global__ void __launch_bounds__(kMoveThreads) compact_kernel(const CompactParams p) {
  if ((int)blockIdx.x < p.batch)
    move_totals(p, blockIdx.x);
  else
    move_rows<D, AHEAD>(p, blockIdx.x - p.batch);
}

}  // namespace

hipError_t launch_keep(const KeepParams& p, hipStream_t stream) {
  const dim3 grid((unsigned)p.batch);
  if (p.max_ctx <= kFewKeys)
    hipLaunchKernelGGL((keep_kernel<512, kFewKeys>), grid, dim3(512), 0, stream, p);
  else
    hipLaunchKernelGGL((keep_kernel<1024, kManyKeys>), grid, dim3(1024), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_compact(const CompactParams& p, hipStream_t stream) {
  const int64_t grid = p.batch + (int64_t)p.batch * 2 * p.num_kv_heads * p.chunks;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kMoveThreads), 0, stream, p); };
  if (grid <= kAheadWorkgroups)
    go(p.head_dim == 128 ? compact_kernel<128, true> : compact_kernel<64, true>);
  else
    go(p.head_dim == 128 ? compact_kernel<128, false> : compact_kernel<64, false>);
  return hipGetLastError();
}

}  // namespace pa
