// Plans of the biased attention's calls: the launcher keeps its parameters, and
// every plan is held against what the kernels take from it -- that a tile's
// partitions reach all the tokens its rows may see, that the row tiles reach all
// rows, that the partial results lie in the workspace that was asked for and that
// the grids can be launched.
#include "ops.h"
#include "paged_attn_ops.h"

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <memory>
#include <random>
#include <vector>

namespace pa {
BiasedParams g_last;
bool g_launched = false;
hipError_t launch_rope(const RopeParams&, const double*, int, bool, bool, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_biased(const BiasedParams& p, hipStream_t) {
  g_last = p;
  g_launched = true;
  return hipSuccess;
}
}  // namespace pa

namespace {

using pa::BiasedParams;

#define NEED(x)                                                                                               \
  do {                                                                                                        \
    if (!(x)) {                                                                                               \
      std::printf("%s\n  batch %d heads %d over %d D %d max_ctx %d max_chunk %d window %d prefix %d total %d: " \
                  "%d tiles, %d partitions of %d blocks, big %d\n",                                           \
                  #x, p.batch, p.num_q_heads, p.num_kv_heads, p.head_dim, p.max_ctx, p.max_chunk, p.window,   \
                  p.prefix_lens != nullptr, p.total_q, p.tiles, p.parts, p.part_blocks, p.big);               \
      return false;                                                                                           \
    }                                                                                                         \
  } while (0)

// The widest range of blocks that a row tile of a chunk of L of n tokens may see lies in its partitions.
bool covers(const BiasedParams& p, int64_t n, int64_t L, int64_t prefix) {
  const int64_t rows = L * p.group, per_tile = pa::kBiasedTileRows;
  const int64_t tiles = (rows + per_tile - 1) / per_tile;
  for (int64_t tile = 0; tile < tiles; tile += std::max<int64_t>(1, tile < tiles - 1 ? std::min(tiles / 7, tiles - 1 - tile) : 1)) {
    const int64_t first = n - L + tile * per_tile / p.group;
    const int64_t last = n - L + (std::min(rows, (tile + 1) * per_tile) - 1) / p.group;
    const int64_t lo = p.window > 0 ? std::max<int64_t>(0, first - p.window + 1) : 0;
    const int64_t hi = std::max(last + 1, p.prefix_lens ? std::min(prefix, n) : 0);
    const int64_t blocks = (hi + 15) / 16 - lo / 16;
    const int64_t per = pa::partition_blocks(p, (int)blocks);
    NEED(blocks <= p.parts * per && (p.parts == 1 || per % 2 == 0));
    NEED(p.parts == 1 || p.part_blocks == per || (p.window > 0 && p.prefix_lens));
  }
  return true;
}

bool plan_holds(const BiasedParams& p, const void* workspace, size_t bytes, std::mt19937& rng) {
  const int64_t rows = (int64_t)p.max_chunk * p.group;
  const int64_t per_tile = p.big ? pa::kBiasedWgRows : pa::kBiasedTileRows;
  const int64_t row_tiles = (int64_t)p.batch * p.tiles * p.num_kv_heads;
  NEED((int64_t)p.tiles * per_tile >= rows);
  NEED(p.parts >= 1 && row_tiles * p.parts * 256 <= 0xffffffffLL);         // threads of a launch: 32 bits
  NEED(!p.ranked || (p.big && p.batch <= 64));
  if (p.parts > 1) {
    NEED(!p.big && p.part_blocks > 0 && p.part_blocks % 2 == 0);
    NEED(p.tile_rows >= std::min<int64_t>(rows, pa::kBiasedTileRows) && p.tile_rows <= pa::kBiasedTileRows);
    NEED((row_tiles * p.tile_rows + 3) / 4 * 256 <= 0xffffffffLL);         // the merge, one wavefront per row
    const uint8_t* ws = static_cast<const uint8_t*>(workspace);
    const int64_t slots = row_tiles * p.parts * p.tile_rows;
    NEED(reinterpret_cast<const uint8_t*>(p.part_o) == ws);
    NEED(reinterpret_cast<const uint8_t*>(p.part_lse) >= ws + slots * p.head_dim * 4);
    NEED(reinterpret_cast<const uint8_t*>(p.part_lse + slots) <= ws + bytes);
  }
  for (int i = 0; i < 24; ++i) {
    const int64_t n = i % 3 == 0 ? p.max_ctx : rng() % ((uint64_t)p.max_ctx + 1);
    const int64_t most = std::min<int64_t>(n, p.max_chunk), L = i % 2 == 0 ? most : rng() % (most + 1);
    if (!covers(p, n, L, i % 4 < 2 ? n : rng() % (n + 1))) return false;
  }
  return true;
}

int32_t spread(std::mt19937& rng, double lo, double hi) {
  return (int32_t)std::lround(std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng)));
}

}  // namespace

int main() {
  void* dev = reinterpret_cast<void*>(0x10000);
  int32_t* idev = static_cast<int32_t*>(dev);
  std::mt19937 rng(11);
  struct Call { int d, hq, hkv, batch, ctx, chunk, window; bool prefix; };
  std::vector<Call> calls = {
      // a window's blocks are fewer than a prefix that sees itself whole may add
      {64, 8, 2, 1, 900, 900, 700, true},    {128, 8, 2, 1, 2000, 300, 700, true},
      {128, 8, 1, 1, 2000, 500, 1024, true}, {128, 8, 2, 1, 1500, 200, 640, true},
      {128, 32, 8, 1, 2000, 100, 1024, true}, {64, 3, 1, 2, 100000, 1, 1000, true},
      {128, 64, 1, 3, 30000, 7, 30000, true},
  };
  const int heads[][2] = {{1, 1}, {2, 1}, {3, 1}, {5, 1}, {8, 1}, {12, 2}, {15, 5}, {28, 4}, {32, 8}, {16, 16}, {64, 8}, {71, 1}, {64, 64}};
  for (int i = 0; i < 40000; ++i) {
    const auto& h = heads[rng() % (sizeof heads / sizeof heads[0])];
    Call c = {rng() % 2 ? 64 : 128, h[0], h[1], spread(rng, 1, 300), spread(rng, 1, 300000), 1, 0, rng() % 2 == 0};
    if (rng() % 3) c.chunk = std::min(c.ctx, spread(rng, 1, 20000));
    if (rng() % 2) c.window = spread(rng, 1, 1.3 * c.ctx);
    calls.push_back(c);
  }
  int split = 0, both = 0, whole = 0, decodes = 0;
  for (const Call& c : calls) {
    pa_kv_pool* made = nullptr;
    if (kv_pool_create(100, 16, c.hkv, c.d, dev, dev, &made) != PA_OK) return 1;
    const std::unique_ptr<pa_kv_pool, int (*)(pa_kv_pool*)> held(made, kv_pool_destroy);
    const pa_kv_pool* pool = made;
    size_t bytes = 0;
    if (paged_attn_biased_workspace_size(pool, c.batch, c.hq, c.ctx, c.chunk, c.window, &bytes) == PA_OK) {
      const int32_t stride = (c.ctx + 15) / 16, total = (int32_t)std::min<int64_t>((int64_t)c.batch * c.chunk, 2000000000);
      const bool decode = c.chunk == 1 && !c.prefix;
      pa::g_launched = false;
      const int rc = decode
          ? paged_attn_decode_biased(pool, dev, idev, stride, idev, c.batch, c.hq, 0.1f, 0.f, nullptr, c.window,
                                     rng() % 2 ? idev : nullptr, c.ctx, dev, bytes, dev, nullptr)
          : paged_attn_extend_biased(pool, dev, idev, rng() % 2 ? total : 1 + rng() % total, idev, stride, idev, c.batch, c.hq,
                                     0.1f, 0.f, nullptr, c.window, rng() % 2 ? idev : nullptr, c.prefix ? idev : nullptr,
                                     c.ctx, c.chunk, dev, bytes, dev, nullptr);
      if (rc != PA_OK || !pa::g_launched) {
        std::printf("a call whose workspace has a size was refused: %s\n", pa_last_error());
        return 1;
      }
      const BiasedParams& p = pa::g_last;
      if (!plan_holds(p, dev, bytes, rng)) return 1;
      split += p.parts > 1;
      both += p.parts > 1 && c.window > 0 && c.prefix && c.chunk > 1;
      whole += p.big;
      decodes += decode;
    }
  }
  std::printf("%d plans hold: %d split (%d with a window and a prefix), %d of 128 rows, %d decodes\n", (int)calls.size(), split, both, whole, decodes);
  return split > 1000 && both > 100 && whole > 1000 && decodes > 1000 ? 0 : 1;
}
