// The `want` largest of n keys, by one workgroup of kChooseThreads: their ranks in
// the keys' own order.  Equal keys: the first ones.
//
// The threshold is found from the top: the highest bit in which any two keys differ,
// then eight bits of it and those below at a time, a histogram in LDS of the keys
// that share all higher ones, until the keys of one digit are exactly those that are
// still wanted, or no bit is left.  (Starting at the first differing bit spares the
// digits that all keys share, as sign and exponent nearly do, whose histogram would
// be one counter that every thread adds to.)  Then every wavefront counts its
// stretch of keys above and on the threshold, and writes them behind those of the
// stretches before.  Nothing depends on the order of the atomics.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pa_device.h"

namespace pa {
namespace choose {

constexpr int kThreads = 1024;
constexpr int kWavesHere = kThreads / 64;

struct Scratch {
  uint64_t any[kWavesHere];
  uint32_t hist[256];
  int32_t above[kWavesHere], equal[kWavesHere];
  int32_t digit, need, exact;
};

// Keys that order as the values do, NaN above all, -0 as 0.
__device__ __forceinline__ uint64_t key_of(double x) {
  if (x != x) return ~0ull;
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return ~0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// load(i): key i < n.  emit(rank, i): key i is one of the chosen, rank < want.  Every
// thread of the workgroup calls it, with the same n and 0 < want < n.
template <typename Key, typename Load, typename Emit>
__device__ __forceinline__ void choose_some(int n, int want, Scratch& s, const Load& load, const Emit& emit) {
  const int lane = threadIdx.x & 63;
  const int wave = wave_uniform(threadIdx.x >> 6);
  constexpr int kBits = 8 * sizeof(Key);
  const Key key0 = load(0);
  // a wavefront's stretch of the keys, whole groups of 64
  const int stretch = (n + kThreads - 1) / kThreads * 64;
  const int from = min(n, wave * stretch), to = min(n, from + stretch);
  // f(i, key, in) for the lane's keys, all lanes together; in: there is a key i
  auto each = [&](const auto& f) {
    for (int i0 = from; i0 < to; i0 += 64) f(i0 + lane, i0 + lane < to ? load(i0 + lane) : (Key)0, i0 + lane < to);
  };
  uint64_t any = 0;
  each([&](int, Key k, bool in) { any |= in ? (uint64_t)(k ^ key0) : 0; });
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) any |= __shfl_xor((unsigned long long)any, m);
  if (lane == 0) s.any[wave] = any;
  __syncthreads();
  any = 0;
#pragma unroll
  for (int w = 0; w < kWavesHere; ++w) any |= s.any[w];
  // bits from `hi` on are decided: the threshold's are `fixed`
  int hi = any == 0 ? 0 : 64 - __builtin_clzll(any);
  auto top = [&](Key k) { return hi == kBits ? (Key)0 : (Key)(k >> hi); };
  Key fixed = top(key0);
  int need = want;
  bool exact = false;
  while (hi > 0 && !exact) {
    const int bits = hi < 8 ? hi : 8;
    const int lo = hi - bits;
    if (threadIdx.x < 256) s.hist[threadIdx.x] = 0;
    __syncthreads();
    each([&](int, Key k, bool in) {
      if (in && top(k) == fixed) atomicAdd(&s.hist[(uint32_t)(k >> lo) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    if (wave == 0) {
      // lane: digits 255 - 4 lane down to 252 - 4 lane, and the count of those above
      int c[4], mine = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[j] = (int)s.hist[255 - 4 * lane - j];
        mine += c[j];
      }
      int before = mine;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const int x = __shfl_up(before, m);
        if (lane >= m) before += x;
      }
      before -= mine;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < need && need <= before + c[j]) {          // one lane, one digit
          s.digit = 255 - 4 * lane - j;
          s.need = need - before;
          s.exact = need - before == c[j];
        }
        before += c[j];
      }
    }
    __syncthreads();
    fixed = (Key)(hi == kBits ? (Key)0 : (Key)(fixed << bits)) | (Key)s.digit;
    need = s.need;
    exact = s.exact != 0;
    hi = lo;
  }

  int above = 0, equal = 0;
  each([&](int, Key k, bool in) {
    above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && top(k) > fixed));
    equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && top(k) == fixed));
  });
  if (lane == 0) {
    s.above[wave] = above;
    s.equal[wave] = equal;
  }
  __syncthreads();
  above = 0;
  equal = 0;
  for (int w = 0; w < wave; ++w) {
    above += s.above[w];
    equal += s.equal[w];
  }
  const uint64_t below = (1ull << lane) - 1;
  each([&](int i, Key k, bool in) {
    const Key t = top(k);
    const uint64_t a = __builtin_amdgcn_ballot_w64(in && t > fixed), e = __builtin_amdgcn_ballot_w64(in && t == fixed);
    const int a_rank = above + __builtin_popcountll(a & below), e_rank = equal + __builtin_popcountll(e & below);
    if (in && (t > fixed || (t == fixed && e_rank < need))) emit(a_rank + min(e_rank, need), i);
    above += __builtin_popcountll(a);
    equal += __builtin_popcountll(e);
  });
}

// The same for 0 <= want <= n.  Up to CAPACITY keys wait in LDS (`room`), which takes
// the passes' loads from L2 out of the chain.
// (In registers they are slower: the unrolled passes are code that is fetched from L2
// as it runs, once, 11.7 / 9.3 us for 512 rows of 250..1800 keys.)
template <typename Key, int CAPACITY, typename Load, typename Emit>
__device__ __forceinline__ void choose(int n, int want, Scratch& s, Key* room, const Load& load, const Emit& emit) {
  if (want <= 0) return;
  if (want >= n) {
    for (int i = threadIdx.x; i < n; i += kThreads) emit(i, i);
    return;
  }
  if (n > CAPACITY) {
    choose_some<Key>(n, want, s, load, emit);
    return;
  }
  const int stretch = (n + kThreads - 1) / kThreads * 64;
  const int from = min(n, wave_uniform(threadIdx.x >> 6) * stretch), to = min(n, from + stretch);
#pragma unroll 4
  for (int i = from + (threadIdx.x & 63); i < to; i += 64) room[i] = load(i);
  __syncthreads();
  choose_some<Key>(n, want, s, [&](int i) { return room[i]; }, emit);
}

}  // namespace choose
}  // namespace pa
