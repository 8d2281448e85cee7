// What paged_attn_keep_heaviest and paged_attn_compact hand to their kernels, under the
// sanitizers: launchers that launch nothing but look at it, arrays told apart.
#include "kernels.h"
#include "ops.h"
#include "paged_attn_tokens.h"
#include "tokens.h"

#include <algorithm>
#include <cstdio>
#include <random>

namespace {
int g_bad = 0;
long g_keep = 0, g_apart = 0, g_in_place = 0, g_same = 0;
bool g_same_tables = false;

void need(bool ok, const char* what) {
  if (!ok && g_bad++ < 10) std::printf("%s\n", what);
}
}  // namespace

namespace pa {
hipError_t launch_rope(const RopeParams&, const double*, int, bool, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_biased(const BiasedParams&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_tree(const BiasedParams&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_selected(const TokensParams&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_weights(const TokensParams&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_bounds(const BlocksParams&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_select(const BlocksParams&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_keep(const KeepParams& p, hipStream_t) {
  ++g_keep;
  const int64_t most = std::min<int64_t>(std::max(p.keep, p.recent), p.max_ctx);
  need(p.kept_stride >= most, "room for the kept");
  need(p.totals_stride >= p.max_ctx && p.max_ctx < 1 << 30, "totals of every token");
  need((int64_t)p.batch * 1024 <= 0xffffffffLL, "keep's grid");
  return hipErrorNotSupported;
}
hipError_t launch_compact(const CompactParams& p, hipStream_t) {
  if (g_same_tables) {
    // several workgroups to a sequence's rows may only write blocks that none of them reads
    ++g_same;
    need(p.chunks == 1, "rounds of a move within one table are in order");
  } else if (p.dst_tables) {
    ++g_apart;
    const int64_t per = (int64_t)kMovePasses * kMoveThreads / (p.head_dim / 8);
    need(p.chunks * per >= std::min(p.kept_stride, p.max_ctx), "rounds of a move apart");
  } else {
    ++g_in_place;
    need(p.chunks == 1, "rounds of a move in place are in order");
  }
  return hipErrorNotSupported;
}
}  // namespace pa

int main() {
  std::mt19937_64 rng(5);
  auto upto = [&](int64_t n) { return (int64_t)(rng() % (uint64_t)(n + 1)); };
  auto at = [](int i) { return reinterpret_cast<int32_t*>((uintptr_t)(i + 1) << 32); };
  float* totals = reinterpret_cast<float*>(at(20));
  for (int round = 0; round < 2000; ++round) {
    const int32_t hkv = (int32_t)(1 + upto(63)), d = rng() % 2 ? 64 : 128;
    pa_kv_pool* pool = nullptr;
    if (kv_pool_create(100, 16, hkv, d, at(30), at(31), &pool) != PA_OK) return 1;
    for (int i = 0; i < 20; ++i) {
      const int32_t batch = (int32_t)(1 + upto(300)), ctx = (int32_t)upto((int64_t)1 << upto(29)), stride = (ctx + 15) / 16 + (int32_t)upto(3);
      const int32_t recent = (int32_t)upto(ctx), keep = (int32_t)upto((int64_t)1 << upto(30));
      const int32_t wide = (int32_t)std::min<int64_t>(std::max(keep, recent), ctx) + (int32_t)upto(2);
      const int rc = paged_attn_keep_heaviest(totals, ctx + upto(5), rng() % 2 ? at(0) : nullptr, at(1), batch, ctx, recent, keep,
                                              at(2), wide, at(3), nullptr);
      need(rc == PA_EHIP, "the choice reaches its launcher");
      auto move = [&](const int32_t* to, int32_t to_stride) {
        const int m = paged_attn_compact(pool, at(4), stride, to, to_stride, at(0), at(1), batch, ctx, at(2), wide, at(3),
                                         totals, totals, ctx, rng() % 2 ? at(1) : at(6), nullptr);
        need(m == PA_EHIP || m == PA_EINVAL, "status");       // (a grid may be too large)
      };
      move(nullptr, 0);
      move(at(5), stride + 1);
      g_same_tables = stride > 0;
      if (g_same_tables) move(at(4), stride);                  // the table itself, given as the second one
      g_same_tables = false;
    }
    kv_pool_destroy(pool);
  }
  for (long n : {g_keep, g_apart, g_in_place, g_same})
    if (n < 1000) {
      std::printf("too few calls reached a launcher: %ld\n", n);
      return 1;
    }
  if (g_bad) return 1;
  std::printf("choices and moves hold: %ld %ld %ld %ld\n", g_keep, g_apart, g_in_place, g_same);
  return 0;
}
