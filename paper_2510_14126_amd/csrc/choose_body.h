// The `want` largest of n keys, by one workgroup: their ranks in the keys' own order.
// Equal keys: the first ones.
//
// The threshold is found from the top: the highest bit in which any two keys differ,
// then eight bits of it and those below at a time, a histogram in LDS of the keys
// that share all higher ones, until the keys of one digit are exactly those that are
// still wanted, or a wavefront's lanes hold them, or no bit is left.  (Starting at the
// first differing bit spares the digits that all keys share, as sign and exponent nearly
// do, whose histogram would be one counter that every thread adds to.)  Then every
// wavefront goes once more through its stretch of the keys: those above the threshold
// become a bit each in words that its lanes keep, and those on it go to a list, from
// which every wavefront takes the wanted ones for itself, by comparing all with all.
// It writes its own behind those of the stretches before.  Nothing depends on the order
// of the atomics.
//
// A short chain bounds it: a handful of passes with a barrier after each.  So the keys
// wait in LDS; every wavefront reads a digit's histogram for itself, and each digit has
// one of its own, zeroed beforehand; and of 64-bit keys the passes look at the 32 bits
// from the first differing one on (the others decide only between keys that are equal
// in those).  Unrolled over registers the passes were slower: code that is fetched from
// L2 as it runs, once.
//
// Up to kListFrom keys, where more are equal than the list takes, or where LDS does not
// hold them, all digits are gone through instead, and the stretches twice at the end, to
// count and to write.  Whole steps with all digits / with the list: the blocks of one
// sequence of 131003 tokens, 64 heads over 8, 36.4 / 33.5 us, of 32000 20.8 / 20.2, 64
// sequences' tokens 365.5 / 363.5; of 300 tokens 13.3 / 14.2 if the list were used there.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pa_device.h"

namespace pa {
namespace choose {

constexpr int kMostWaves = 16;
constexpr int kDigits = 8;                // of a 64-bit key
constexpr int kList = 64;                 // keys on the threshold that a wavefront holds
constexpr int kListFrom = 1024;           // keys

struct Scratch {
  uint64_t any[kMostWaves];
  int32_t above[kMostWaves], equal[kMostWaves];
  uint64_t list[kList];
  int32_t place[kList];
  uint32_t listed;
  alignas(16) uint32_t hist[kDigits][256];
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

// x >> s for 0 <= s <= the type's bits.
template <typename T>
__device__ __forceinline__ T shifted(T x, int s) {
  return s >= (int)(8 * sizeof(T)) ? (T)0 : (T)(x >> s);
}

// Sums over this lane and those before it, and the bits of all lanes together: DPP
// moves within the rows of 16, then each row's last lane to the rows behind it.  (The
// same through the LDS crossbar was half of a digit's time, sixteen wavefronts at it.)
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
constexpr int kDppRowShr1 = 0x111, kDppRowBcast15 = 0x142, kDppRowBcast31 = 0x143;
__device__ __forceinline__ uint32_t sum_before(uint32_t x) {
  x += moved<kDppRowShr1, 0xf>(x);
  x += moved<kDppRowShr1 + 1, 0xf>(x);
  x += moved<kDppRowShr1 + 3, 0xf>(x);
  x += moved<kDppRowShr1 + 7, 0xf>(x);
  x += moved<kDppRowBcast15, 0xa>(x);
  x += moved<kDppRowBcast31, 0xc>(x);
  return x;
}
__device__ __forceinline__ uint32_t any_bits(uint32_t x) {
  x |= moved<kDppRowShr1, 0xf>(x);
  x |= moved<kDppRowShr1 + 1, 0xf>(x);
  x |= moved<kDppRowShr1 + 3, 0xf>(x);
  x |= moved<kDppRowShr1 + 7, 0xf>(x);
  x |= moved<kDppRowBcast15, 0xa>(x);
  x |= moved<kDppRowBcast31, 0xc>(x);
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// Keys of which `bits` bits are undecided, seen as U values of that many bits at most:
// the threshold's bits from `hi` on (fixed), how many keys share them (all), and how
// many of those are wanted (need).
template <typename U>
struct Threshold {
  int hi, need, all;
  U fixed;
  __device__ __forceinline__ bool exact() const { return all == need; }
};
// each(f): f(key, there) for the lane's keys, n in all.  Ends with no more than `few` of
// them on the threshold, where that many bits tell them apart.
template <typename U, typename Each>
__device__ __forceinline__ Threshold<U> threshold(Scratch& s, int bits, int n, int want, int few, const Each& each) {
  const int lane = threadIdx.x & 63;
  Threshold<U> t{bits, want, n, (U)0};
  for (int digit = 0; t.hi > 0 && !t.exact() && t.all > few; ++digit) {
    const int width = t.hi < 8 ? t.hi : 8;
    const int lo = t.hi - width;
    uint32_t* hist = s.hist[digit];
    each([&](U k, bool in) {
      if (in && shifted(k, t.hi) == t.fixed) atomicAdd(&hist[(uint32_t)(k >> lo) & ((1u << width) - 1)], 1u);
    });
    __syncthreads();
    // lane: digits 255 - 4 lane down to 252 - 4 lane, and the count of those above
    const uint4 four = *reinterpret_cast<const uint4*>(hist + 252 - 4 * lane);
    const int c[4] = {(int)four.w, (int)four.z, (int)four.y, (int)four.x};
    const int mine = c[0] + c[1] + c[2] + c[3];
    int before = (int)sum_before((uint32_t)mine) - mine;
    int found = -1, rest = 0, all = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (before < t.need && t.need <= before + c[j]) {          // one lane, one digit
        found = 255 - 4 * lane - j;
        rest = t.need - before;
        all = c[j];
      }
      before += c[j];
    }
    const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(found >= 0));
    t.fixed = (U)(t.fixed << width) | (U)__builtin_amdgcn_readlane(found, who);
    t.need = __builtin_amdgcn_readlane(rest, who);
    t.all = __builtin_amdgcn_readlane(all, who);
    t.hi = lo;
  }
  return t;
}

// Lanes of a mask below this one.
__device__ __forceinline__ int below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Writes the chosen keys of the workgroup's stretches.  each(f): f(i, key, there).
template <typename U, typename Each, typename Emit>
__device__ __forceinline__ void write_chosen(Scratch& s, const Threshold<U>& t, int wave, const Each& each, const Emit& emit) {
  const int lane = threadIdx.x & 63;
  int above = 0, equal = 0;
  each([&](int, U k, bool in) {
    const U x = shifted(k, t.hi);
    above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && x > t.fixed));
    equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && x == t.fixed));
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
  each([&](int i, U k, bool in) {
    const U x = shifted(k, t.hi);
    const uint64_t a = __builtin_amdgcn_ballot_w64(in && x > t.fixed), e = __builtin_amdgcn_ballot_w64(in && x == t.fixed);
    if ((a | e) == 0) return;                                    // uniform
    const int e_rank = equal + below(e);
    if (in && (x > t.fixed || (x == t.fixed && e_rank < t.need))) emit(above + below(a) + min(e_rank, t.need), i);
    above += __builtin_popcountll(a);
    equal += __builtin_popcountll(e);
  });
}

__device__ __forceinline__ int bits_in(uint64_t mask) { return __builtin_popcountll(mask); }

// The same where no more than kList keys are on the threshold, and no stretch has more
// than 64 words of 64 keys.  key_at(i): all bits; of those, the ones from `drop` on and
// below `mask` are the threshold's.
template <typename Key, typename At, typename Emit>
__device__ __forceinline__ void write_few(Scratch& s, const Threshold<uint32_t>& t, int drop, uint32_t mask, int wave,
                                          int from, int to, const At& key_at, const Emit& emit) {
  const int lane = threadIdx.x & 63;
  uint64_t mine = 0;                                               // lane: of its word of the stretch
  int above = 0;
  Key next = from + lane < to ? key_at(from + lane) : (Key)0;
  for (int i0 = from, w = 0; i0 < to; i0 += 64, ++w) {
    const Key k = next;
    const bool in = i0 + lane < to;
    next = i0 + 64 + lane < to ? key_at(i0 + 64 + lane) : (Key)0;  // on its way during this one
    const uint32_t x = shifted((uint32_t)shifted(k, drop) & mask, t.hi);
    const uint64_t a = __builtin_amdgcn_ballot_w64(in && (x > t.fixed || (t.exact() && x == t.fixed)));
    const uint64_t on = t.exact() ? 0 : __builtin_amdgcn_ballot_w64(in && x == t.fixed);
    if (on != 0) {                                                 // uniform
      uint32_t at = 0;
      if (lane == 0) at = atomicAdd(&s.listed, (uint32_t)bits_in(on));   // t.all <= kList in all
      at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at) + below(on);
      if ((on >> lane) & 1) {
        s.list[at] = k;
        s.place[at] = i0 + lane;
      }
    }
    if (lane == w) mine = a;
    above += bits_in(a);
  }
  if (lane == 0) s.above[wave] = above;
  __syncthreads();
  above = 0;
  for (int w = 0; w < wave; ++w) above += s.above[w];
  if (!t.exact()) {
    const uint64_t k = s.list[lane];                               // zeros behind the listed ones: below all keys
    const int i = s.place[lane];
    int rank = 0;
    for (int j0 = 0; j0 < t.all; j0 += 8)
#pragma unroll
      for (int j = 0; j < 8; ++j) rank += s.list[j0 + j] > k;
    bool chosen = lane < t.all && rank < t.need;
    if (bits_in(__builtin_amdgcn_ballot_w64(chosen)) != t.need) {  // equal ones on both sides: the first of them
      int equal = 0, before = 0;
      for (int j = 0; j < t.all; ++j) {
        equal += s.list[j] == k;
        before += s.list[j] == k && s.place[j] < i;
      }
      chosen = chosen && rank + (rank + equal > t.need ? before : 0) < t.need;
    }
    above += bits_in(__builtin_amdgcn_ballot_w64(chosen && i < from));
    for (uint64_t own = __builtin_amdgcn_ballot_w64(chosen && i >= from && i < to); own != 0; own &= own - 1) {
      const int at = __builtin_amdgcn_readlane(i, __builtin_ctzll(own)) - from;
      if (lane == at >> 6) mine |= 1ull << (at & 63);
    }
  }
  for (int i0 = from, w = 0; i0 < to; i0 += 64, ++w) {
    const uint64_t a = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(mine >> 32), w) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, w);
    if ((a >> lane) & 1) emit(above + below(a), i0 + lane);
    above += bits_in(a);
  }
}

// load(i): key i < bound, of which the first n <= bound count (bound is known before
// n arrives, and the first loads need not wait for it).  emit(rank, i): key i is one of
// the chosen, rank < want.  All THREADS of the workgroup call it, with the same n and
// 0 <= want <= n.  Up to CAPACITY keys wait in `room`; more are loaded anew by each pass.
template <typename Key, int THREADS, int CAPACITY, typename Load, typename Emit>
__device__ __forceinline__ void choose(int bound, int n, int want, Scratch& s, Key* room, const Load& load, const Emit& emit) {
  const int lane = threadIdx.x & 63;
  const int wave = wave_uniform(threadIdx.x >> 6);
  constexpr int kFirst = THREADS == 1024 ? 8 : 4;
  const Key key0 = bound > 0 ? load(0) : (Key)0;
  Key first[kFirst];
#pragma unroll
  for (int k = 0; k < kFirst; ++k) first[k] = (int)threadIdx.x + k * THREADS < bound ? load(threadIdx.x + k * THREADS) : (Key)0;
  if (want <= 0) return;
  if (want >= n) {
    for (int i = threadIdx.x; i < n; i += THREADS) emit(i, i);
    return;
  }
  for (int i = threadIdx.x; i < kDigits * 256; i += THREADS) (&s.hist[0][0])[i] = 0;
  if (threadIdx.x < kList) s.list[threadIdx.x] = 0;
  if (threadIdx.x == 0) s.listed = 0;
  // a wavefront's stretch of the keys, whole groups of 64
  const int stretch = (n + THREADS - 1) / THREADS * 64;
  const int from = min(n, wave * stretch), to = min(n, from + stretch);
  uint64_t any = 0;
  static_assert(CAPACITY <= 64 * THREADS, "a stretch's words: one per lane");
  const bool held = n <= CAPACITY, listing = held && n > kListFrom;
  auto seen = [&](int i, Key k) {
    if (held) room[i] = k;
    any |= (uint64_t)(k ^ key0);
  };
#pragma unroll
  for (int k = 0; k < kFirst; ++k)
    if ((int)threadIdx.x + k * THREADS < n) seen(threadIdx.x + k * THREADS, first[k]);
#pragma unroll 4
  for (int i = threadIdx.x + kFirst * THREADS; i < n; i += THREADS) seen(i, load(i));
  any = (uint64_t)any_bits((uint32_t)(any >> 32)) << 32 | any_bits((uint32_t)any);
  if (lane == 0) s.any[wave] = any;
  __syncthreads();
  any = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) any |= s.any[w];
  const int bits = any == 0 ? 0 : 64 - __builtin_clzll(any);          // that are not the same in all keys

  auto passes = [&](const auto& key_at) {
    // the 32 highest of those bits
    const int drop = max(0, bits - 32);
    const uint32_t mask = bits - drop >= 32 ? ~0u : (1u << (bits - drop)) - 1;
    auto each = [&](const auto& f) {
      Key k = from + lane < to ? key_at(from + lane) : (Key)0;
      for (int i0 = from; i0 < to; i0 += 64) {
        const Key next = i0 + 64 + lane < to ? key_at(i0 + 64 + lane) : (Key)0;    // on its way during this one
        f(i0 + lane, (uint32_t)shifted(k, drop) & mask, i0 + lane < to);
        k = next;
      }
    };
    const auto t = threshold<uint32_t>(s, bits - drop, n, want, listing ? kList : 0, [&](const auto& f) {
#pragma unroll 4
      for (int i = from + lane; i < to; i += 64) f((uint32_t)shifted(key_at(i), drop) & mask, true);
    });
    if (listing && (t.exact() || t.all <= kList)) {
      write_few<Key>(s, t, drop, mask, wave, from, to, key_at, emit);
      return;
    }
    if (t.exact() || drop == 0) {
      write_chosen<uint32_t>(s, t, wave, each, emit);
      return;
    }
    // keys equal in all of those stand on both sides: all bits
    __syncthreads();
    for (int i = threadIdx.x; i < kDigits * 256; i += THREADS) (&s.hist[0][0])[i] = 0;
    __syncthreads();
    const uint64_t wide = bits >= 64 ? ~0ull : (1ull << bits) - 1;
    auto each_wide = [&](const auto& f) {
      for (int i0 = from; i0 < to; i0 += 64) {
        const bool in = i0 + lane < to;
        f(i0 + lane, (uint64_t)(in ? key_at(i0 + lane) : (Key)0) & wide, in);
      }
    };
    const auto u = threshold<uint64_t>(s, bits, n, want, 0, [&](const auto& f) {
      each_wide([&](int, uint64_t k, bool in) { f(k, in); });
    });
    write_chosen<uint64_t>(s, u, wave, each_wide, emit);
  };
  if (held)
    passes([&](int i) { return room[i]; });
  else
    passes(load);
}

}  // namespace choose
}  // namespace pa
