// Host paths of the operators in paged_attn_tokens.h under the sanitizers: random
// arguments, with launchers that launch nothing but look at what they are given.
// Whatever a kernel takes from its plan must hold: partitions that reach every
// block, tiles that hold every row and head, partial results and scores inside a
// workspace of exactly the size that was asked for, and grids of 32 bits of threads.
#include "kernels.h"
#include "ops.h"
#include "paged_attn_tokens.h"
#include "tokens.h"

#include <cstdio>
#include <cstdlib>
#include <random>

namespace {
uint8_t* const kWorkspace = reinterpret_cast<uint8_t*>(0x7f0000000000);
size_t g_bytes = 0;
int g_bad = 0;
long g_seen[6] = {};

void need(bool ok, const char* what) {
  if (!ok && g_bad++ < 10) std::printf("plan: %s\n", what);
}
void inside(const void* p, size_t bytes, const char* what) {
  if (bytes == 0) return;
  const uint8_t* x = static_cast<const uint8_t*>(p);
  need(x >= kWorkspace && x + bytes <= kWorkspace + g_bytes && reinterpret_cast<uintptr_t>(x) % 16 == 0, what);
}
bool grid_fits(int64_t workgroups, int threads) { return workgroups * threads <= 0xffffffffLL; }

void look(const pa::TokensParams& p, bool weights) {
  const int64_t tiles = (int64_t)p.batch * p.head_tiles * p.num_kv_heads, rows = tiles * p.tile_heads;
  const int64_t blocks = weights ? ((int64_t)p.max_ctx + 15) / 16 : p.max_blocks;
  need((int64_t)p.parts * p.part_blocks >= blocks && p.parts >= 1, "partitions reach every block");
  need(p.head_tiles * p.tile_heads >= p.group && (p.tile_heads == 4 || p.tile_heads == 8), "tiles hold every head");
  need(grid_fits(tiles * p.parts, 256), "grid");
  if (p.parts > 1) inside(p.part_o, (size_t)rows * p.parts * p.head_dim * 4, "partial outputs");
  if (p.parts > 1 || weights) inside(p.part_lse, (size_t)rows * p.parts * 4, "log-sum-exps");
  if (weights) {
    need(p.score_tokens % 16 == 0 && p.score_tokens >= p.max_ctx, "scores of whole blocks");
    inside(p.scores, (size_t)rows * p.score_tokens * 4, "scores");
    need(p.parts == 1 || (uint8_t*)p.part_o >= (uint8_t*)p.scores + (size_t)rows * p.score_tokens * 4, "scores and partial outputs apart");
    need(grid_fits((int64_t)p.batch * ((p.max_ctx + 255) / 256) + ((int64_t)p.batch * p.num_q_heads + 3) / 4, 256), "weights' grid");
  }
  if (p.parts > 1) need((uint8_t*)p.part_lse >= (uint8_t*)p.part_o + (size_t)rows * p.parts * p.head_dim * 4, "partials apart");
}
}  // namespace

namespace pa {
hipError_t launch_rope(const RopeParams&, const double*, int, bool, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_biased(const BiasedParams&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_tree(const BiasedParams& p, hipStream_t) {
  ++g_seen[0];
  const int64_t rows = (int64_t)p.max_chunk * p.group, tile = p.big ? kBiasedWgRows : kBiasedTileRows;
  const int64_t tiles = (int64_t)p.batch * p.tiles * p.num_kv_heads;
  need(p.tiles * tile >= rows && (p.tiles > 1 ? p.tile_rows == tile : p.tile_rows >= rows), "tiles hold every row");
  need((int64_t)p.parts * p.part_blocks >= ((int64_t)p.max_ctx + 15) / 16, "partitions reach every block");
  need(grid_fits(tiles * p.parts, 256) && (p.parts == 1 || tiles * p.tile_rows <= 0x7fffffffLL), "grid");
  need(p.max_chunk <= kTreeMostNodes && p.parents && p.q_start && !p.slopes && !p.prefix_lens && p.window == 0, "a tree's arguments");
  if (p.parts > 1) {
    inside(p.part_o, (size_t)tiles * p.parts * p.tile_rows * p.head_dim * 4, "partial outputs");
    inside(p.part_lse, (size_t)tiles * p.parts * p.tile_rows * 4, "log-sum-exps");
  }
  return hipErrorNotSupported;
}
hipError_t launch_selected(const TokensParams& p, hipStream_t) { ++g_seen[1]; look(p, false); return hipErrorNotSupported; }
hipError_t launch_weights(const TokensParams& p, hipStream_t) { ++g_seen[2]; look(p, true); return hipErrorNotSupported; }
hipError_t launch_bounds(const BlocksParams& p, hipStream_t) {
  ++g_seen[3];
  need(grid_fits(((int64_t)p.batch * ((p.max_new + 14) / 16 + 1) * p.num_kv_heads + 3) / 4, 256), "bounds' grid");
  return hipErrorNotSupported;
}
hipError_t launch_select(const BlocksParams& p, hipStream_t) {
  ++g_seen[4];
  const int64_t rows = (int64_t)p.batch * p.num_kv_heads;
  need(p.first_blocks >= 0 && p.last_blocks >= 1 && (int64_t)p.first_blocks + p.last_blocks <= p.max_blocks, "forced blocks");
  if (p.key_blocks > p.max_blocks) inside(p.keys, (size_t)rows * p.key_blocks * 8, "keys");
  need(grid_fits(rows, 1024) && grid_fits(rows * ((p.key_blocks + 63) / 64), 256), "select's grid");
  return hipErrorNotSupported;
}
hipError_t launch_keep(const KeepParams& p, hipStream_t) {
  const int64_t most = p.keep > p.recent ? p.keep : p.recent;
  need(p.kept_stride >= (most < p.max_ctx ? most : p.max_ctx), "room for the kept");
  return hipErrorNotSupported;
}
hipError_t launch_compact(const CompactParams& p, hipStream_t) {
  ++g_seen[5];
  const int64_t per = (int64_t)kMovePasses * kMoveThreads / (p.head_dim / 8);
  const int64_t most = p.kept_stride < p.max_ctx ? p.kept_stride : p.max_ctx;
  need(p.dst_tables ? p.chunks * per >= most : p.chunks == 1, "rounds of a move");
  need(grid_fits((int64_t)p.batch * (1 + 2 * (int64_t)p.num_kv_heads * p.chunks), 256), "move's grid");
  return hipErrorNotSupported;
}
}  // namespace pa

int main() {
  std::mt19937_64 rng(11);
  auto pick = [&](std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); };
  auto upto = [&](int64_t n) { return (int64_t)(rng() % (uint64_t)(n + 1)); };
  // sizes from one to large ones, and values that must be refused
  auto size = [&](int64_t most) -> int64_t {
    const int64_t x = (int64_t)1 << upto(31);
    const int64_t y = upto(x < most ? x : most);
    return rng() % 40 == 0 ? pick({-1, 0, 2147483647, -2147483648LL}) : y;
  };
  void* dev = reinterpret_cast<void*>(0x10000);
  float* fdev = static_cast<float*>(dev);
  int32_t* idev = static_cast<int32_t*>(dev);
  for (int round = 0; round < 60; ++round) {
    const int32_t hkv = (int32_t)(1 + upto(63)), d = rng() % 2 ? 64 : 128;
    pa_kv_pool* pool = nullptr;
    if (kv_pool_create(100, 16, hkv, d, dev, dev, &pool) != PA_OK) return 1;
    for (int i = 0; i < 4000; ++i) {
      const int32_t hq = (int32_t)(hkv * (rng() % 50 == 0 ? upto(1 << 22) : 1 + upto(20)) + (rng() % 40 == 0)), batch = (int32_t)size(1 << 20);
      const int32_t ctx = (int32_t)size((1 << 30) - 1), nodes = (int32_t)pick({0, 1, 7, 31, 64, 200, 256, 257, upto(300), -1});
      const int32_t stride = rng() % 20 ? (int32_t)((ctx + 15LL) / 16 + upto(3)) : (int32_t)size(1 << 27);
      const int32_t most = (int32_t)size(1 << 26), first = (int32_t)pick({0, 1, 2, upto(most > 0 ? most : 0)}), last = (int32_t)pick({1, 2, 0, upto(most > 0 ? most : 0)});
      const int32_t total = (int32_t)size(1 << 26), fresh = (int32_t)size(1 << 27);
      const int64_t ts = ctx + pick({0, 1, -1, 1 << 20, (int64_t)1 << 60});
      auto ok = [&](int rc) { need(rc == PA_OK || rc == PA_EINVAL || rc == PA_EUNSUPPORTED || rc == PA_EHIP, "status"); };
      auto with = [&](int rc, size_t bytes, auto call) {
        ok(rc);
        if (rc != PA_OK) bytes = upto(1 << 30);
        g_bytes = bytes;
        ok(call(bytes));
        if (rc == PA_OK && bytes > 0) need(call(bytes - 1) == PA_EINVAL || batch == 0 || total == 0 || nodes == 0, "a short workspace");
      };
      size_t bytes = 0;
      int rc = paged_attn_tree_workspace_size(pool, batch, hq, ctx, nodes, &bytes);
      if (total > 0 && nodes > 0)
        with(rc, bytes, [&](size_t n) {
          return paged_attn_extend_tree(pool, dev, idev, total, idev, idev, stride, idev, batch, hq, 0.1f, (float)pick({0, 30}), ctx,
                                        nodes, kWorkspace, n, dev, nullptr);
        });
      bytes = 0;
      rc = paged_attn_selected_workspace_size(pool, batch, hq, most, &bytes);
      with(rc, bytes, [&](size_t n) {
        return paged_attn_decode_selected(pool, dev, idev, stride, idev, batch, hq, 0.1f, ctx, idev, most, kWorkspace, n, dev, nullptr);
      });
      bytes = 0;
      rc = paged_attn_select_workspace_size(pool, batch, ctx, most, &bytes);
      with(rc, bytes, [&](size_t n) {
        return paged_attn_select_blocks(pool, dev, dev, idev, stride, idev, batch, hq, ctx, first, last, most, kWorkspace, n, idev, nullptr);
      });
      bytes = 0;
      rc = paged_attn_weights_workspace_size(pool, batch, hq, ctx, &bytes);
      with(rc, bytes, [&](size_t n) {
        return paged_attn_decode_weights(pool, dev, idev, stride, idev, batch, hq, 0.1f, ctx, 1.f, fdev, fdev, ts, kWorkspace, n, dev, nullptr);
      });
      ok(paged_attn_block_bounds(pool, dev, idev, stride, rng() % 2 ? idev : nullptr, idev, batch, ctx, total, nullptr));
      ok(paged_attn_keep_heaviest(fdev, ts, idev, idev, batch, ctx, first, most, idev, (int32_t)size(1 << 30), idev, nullptr));
      const bool apart = rng() % 2 != 0;
      ok(paged_attn_compact(pool, idev, stride, apart ? idev : nullptr, apart ? fresh : 0, nullptr, idev, batch, ctx, idev, most, idev,
                            fdev, fdev, ts, nullptr, nullptr));
    }
    kv_pool_destroy(pool);
  }
  for (long n : g_seen)
    if (n < 1000) {
      std::printf("too few calls reached a launcher: %ld\n", n);
      return 1;
    }
  if (g_bad) return 1;
  std::printf("plans hold: %ld %ld %ld %ld %ld %ld\n", g_seen[0], g_seen[1], g_seen[2], g_seen[3], g_seen[4], g_seen[5]);
  return 0;
}
