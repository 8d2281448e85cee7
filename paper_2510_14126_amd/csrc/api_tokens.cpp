// C ABI of the operators that choose tokens of a paged context
// (paged_attn_tokens.h): argument validation and launch planning.  Every check
// runs on the host before any HIP call.
#include "kernels.h"
#include "ops.h"
#include "paged_attn_tokens.h"
#include "pool.h"
#include "tokens.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

static_assert(PA_TREE_MAX_NODES == pa::kTreeMostNodes, "the header's bound is the kernels'");

namespace {
using pa::fail;

constexpr double kLog2e = 1.4426950408889634;
// A launch's threads are counted in 32 bits.
constexpr int64_t kMostThreads = 0xffffffffLL;
constexpr int64_t kMostBytes = (int64_t)1 << 62;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
int64_t blocks_of(int64_t tokens) { return (tokens + PA_BLOCK_SIZE - 1) / PA_BLOCK_SIZE; }

int check_batch(const pa_kv_pool* pool, int32_t batch, int32_t max_context_len, const char* fn) {
  if (!pool) return fail(PA_EINVAL, "%s: pool is NULL", fn);
  if (batch < 0) return fail(PA_EINVAL, "%s: batch = %d < 0", fn, batch);
  if (max_context_len < 0 || max_context_len >= 1 << 30)
    return fail(PA_EINVAL, "%s: max_context_len = %d outside [0, 2^30)", fn, max_context_len);
  return PA_OK;
}

int check_heads(const pa_kv_pool* pool, int32_t num_q_heads, const char* fn) {
  if (num_q_heads <= 0 || num_q_heads % pool->num_kv_heads != 0)
    return fail(PA_EINVAL, "%s: num_q_heads = %d is not a positive multiple of num_kv_heads = %d", fn, num_q_heads,
                pool->num_kv_heads);
  return PA_OK;
}

int check_tables(int32_t bt_stride, int32_t max_context_len, const char* fn) {
  const int64_t need = blocks_of(max_context_len);
  if (bt_stride < need || bt_stride < 0)
    return fail(PA_EINVAL, "%s: bt_stride = %d < ceil(max_context_len / 16) = %lld", fn, bt_stride, (long long)need);
  return PA_OK;
}

int check_workspace(const void* workspace, size_t bytes, size_t need, const char* fn) {
  if (bytes < need) return fail(PA_EINVAL, "%s: workspace of %zu bytes, %zu are needed", fn, bytes, need);
  if (need > 0 && (!workspace || !aligned(workspace, 16)))
    return fail(PA_EINVAL, "%s: workspace is NULL or not 16-byte aligned", fn);
  return PA_OK;
}

int check_grid(int64_t workgroups, int threads, const char* fn) {
  if (workgroups > kMostThreads / threads) return fail(PA_EINVAL, "%s: grid too large", fn);
  return PA_OK;
}

int launched(hipError_t e, const char* fn) {
  if (e != hipSuccess) return fail(PA_EHIP, "%s: kernel launch failed: %s", fn, hipGetErrorString(e));
  return PA_OK;
}

// How the rows of a decode and their blocks are dealt to workgroups: tiles of four or
// eight heads of a KV head, and partitions of a row's blocks as in the biased decode:
// as many as make a workgroup a CU (kFill64: two), or twice that rather than partitions of
// more than kMostBlocks.  Capped at kMostBlocks / twice as many, 32 heads over 8: weights of
// four sequences of 15000..30000 tokens 81 / 74.5 us, of one of 130000, 64 heads, 120 / 113;
// 1500 chosen blocks of four 100 / 96; three of 64..30000 43 / 45.
//
// Where the rows fill the GPU, those with kept weights are split at kMostBlocks (whose
// scores LDS holds), but into pieces of kLongBlocks: a workgroup takes a hundred
// microseconds for 128 blocks, and the last ones' end is what the others wait for.  Split
// at 128 into 128 / at 128 into 64 / at 64 into 64 / at 128 into 32: 128 sequences of 64..8192
// tokens 169 / 160 / 167 / 162 us, 64 of 64..16000 92 / 85 / 88 / 86; 128 of an equal
// distribution of 64..8192 438 / 432 / 435 / 440, 64 of 4096 201 / 203 / 203 / 207.
constexpr int64_t kFill128 = 256, kFill64 = 512;
constexpr int64_t kWholeBlocks = 40, kLeastBlocks = 16, kMostBlocks = 128, kLongBlocks = 64;

struct Plan {
  int32_t tile_heads, head_tiles, parts, part_blocks, whole_blocks;
  int64_t tiles;                          // row tiles: batch x head tiles x KV heads
  size_t o_bytes, lse_bytes, score_bytes;
  size_t bytes() const { return o_bytes + lse_bytes + score_bytes; }
};

// blocks: bound of a row's.  weights: the blocks' scores are kept, and every row's
// log-sum-exp.
int plan_decode(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads, int64_t blocks, bool weights, Plan* pl,
                const char* fn) {
  const int64_t score_tokens = weights ? blocks * PA_BLOCK_SIZE : 0;
  const int32_t group = num_q_heads / pool->num_kv_heads;
  pl->tile_heads = group <= 4 ? 4 : 8;
  pl->head_tiles = (group + pl->tile_heads - 1) / pl->tile_heads;
  pl->tiles = (int64_t)batch * pl->head_tiles * pool->num_kv_heads;
  if (pl->tiles > 0x7fffffffLL) return fail(PA_EINVAL, "%s: grid too large", fn);
  int64_t per = std::max<int64_t>(blocks, 1);
  if (blocks > kWholeBlocks) {
    const int64_t fill = pool->head_dim == 64 ? kFill64 : kFill128;
    auto deal = [&](int64_t workgroups) {
      const int64_t parts = std::max<int64_t>(1, workgroups / std::max<int64_t>(pl->tiles, 1));
      per = std::max(kLeastBlocks, (blocks + 2 * parts - 1) / (2 * parts) * 2);
    };
    deal(fill);
    if (per > kMostBlocks) deal(2 * fill);
  }
  pl->whole_blocks = (int32_t)std::min(per, kMostBlocks);
  if (per > kMostBlocks) per = weights ? kLongBlocks : kMostBlocks;
  const int64_t parts = std::max<int64_t>(1, (blocks + per - 1) / per);
  pl->part_blocks = (int32_t)per;
  pl->parts = (int32_t)parts;
  const int64_t rows = pl->tile_heads * std::max<int64_t>(pl->tiles, 1);
  if (parts > 0x7fffffffLL / rows || score_tokens > kMostBytes / 8 / rows)
    return fail(PA_EINVAL, "%s: grid too large", fn);
  pl->o_bytes = parts > 1 ? (size_t)(pl->tiles * pl->tile_heads * parts) * pool->head_dim * sizeof(float) : 0;
  pl->lse_bytes = parts > 1 || weights ? (size_t)(pl->tiles * pl->tile_heads * parts) * sizeof(float) : 0;
  pl->score_bytes = (size_t)(pl->tiles * pl->tile_heads) * score_tokens * sizeof(float);
  return PA_OK;
}

// What the two decodes check and hand on alike.
int decode_params(const pa_kv_pool* pool, const void* q, const int32_t* block_tables, int32_t bt_stride,
                  const int32_t* context_lens, int32_t batch, int32_t num_q_heads, float scale, int32_t max_context_len,
                  const Plan& pl, void* workspace, size_t workspace_bytes, void* out, pa::TokensParams* p, const char* fn) {
  if (!q || !block_tables || !context_lens || !out)
    return fail(PA_EINVAL, "%s: q, block_tables, context_lens and out must be non-NULL", fn);
  if (!aligned(q, 16) || !aligned(out, 16)) return fail(PA_EINVAL, "%s: q/out are not 16-byte aligned", fn);
  if (!aligned(block_tables, 4) || !aligned(context_lens, 4))
    return fail(PA_EINVAL, "%s: block_tables/context_lens are not 4-byte aligned", fn);
  int rc = check_grid(pl.tiles * pl.parts, 256, fn);
  if (rc || (rc = check_workspace(workspace, workspace_bytes, pl.bytes(), fn))) return rc;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p->k_pool = pool->k;
  p->v_pool = pool->v;
  p->q = static_cast<const uint16_t*>(q);
  p->block_tables = block_tables;
  p->context_lens = context_lens;
  p->out = static_cast<uint16_t*>(out);
  // the scores first, whose records are read 16 bytes at a time
  p->scores = pl.score_bytes ? reinterpret_cast<float*>(ws) : nullptr;
  p->part_o = pl.o_bytes ? reinterpret_cast<float*>(ws + pl.score_bytes) : nullptr;
  p->part_lse = pl.lse_bytes ? reinterpret_cast<float*>(ws + pl.score_bytes + pl.o_bytes) : nullptr;
  p->num_blocks = pool->num_blocks;
  p->num_kv_heads = pool->num_kv_heads;
  p->num_q_heads = num_q_heads;
  p->group = num_q_heads / pool->num_kv_heads;
  p->head_dim = pool->head_dim;
  p->head_tiles = pl.head_tiles;
  p->tile_heads = pl.tile_heads;
  p->batch = batch;
  p->bt_stride = bt_stride;
  p->max_ctx = max_context_len;
  p->parts = pl.parts;
  p->part_blocks = pl.part_blocks;
  p->whole_blocks = pl.whole_blocks;
  p->stream_tiles = pl.head_tiles == 1 && pool->shared_blocks == 0;
  p->scale_log2 = (float)(scale * kLog2e);
  return PA_OK;
}

int check_scale(float scale, const char* fn) {
  if (!std::isfinite((float)(scale * kLog2e)))
    return fail(PA_EINVAL, "%s: scale is not finite, or not in log2 units", fn);
  return PA_OK;
}

int check_totals(const void* totals, const void* totals_out, int64_t totals_stride, int64_t batch, int32_t max_context_len,
                 const char* fn) {
  if (totals_stride < max_context_len)
    return fail(PA_EINVAL, "%s: totals_stride = %lld < max_context_len = %d", fn, (long long)totals_stride, max_context_len);
  if (totals_stride > kMostBytes / 8 / std::max<int64_t>(batch, 1))
    return fail(PA_EINVAL, "%s: totals_stride = %lld is too large", fn, (long long)totals_stride);
  if (!aligned(totals, 4) || !aligned(totals_out, 4)) return fail(PA_EINVAL, "%s: totals are not 4-byte aligned", fn);
  return PA_OK;
}

int plan_weights(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads, int32_t max_context_len, Plan* pl, const char* fn) {
  int rc = check_batch(pool, batch, max_context_len, fn);
  if (rc || (rc = check_heads(pool, num_q_heads, fn))) return rc;
  return plan_decode(pool, batch, num_q_heads, blocks_of(max_context_len), true, pl, fn);
}

int plan_selected(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads, int32_t max_blocks, Plan* pl, const char* fn) {
  int rc = check_batch(pool, batch, 0, fn);
  if (rc || (rc = check_heads(pool, num_q_heads, fn))) return rc;
  if (max_blocks < 0) return fail(PA_EINVAL, "%s: max_blocks = %d < 0", fn, max_blocks);
  return plan_decode(pool, batch, num_q_heads, max_blocks, false, pl, fn);
}

int select_bytes(const pa_kv_pool* pool, int32_t batch, int32_t max_context_len, int32_t max_blocks, size_t* bytes,
                 const char* fn) {
  const int rc = check_batch(pool, batch, max_context_len, fn);
  if (rc) return rc;
  if (max_blocks < 1) return fail(PA_EINVAL, "%s: max_blocks = %d < 1", fn, max_blocks);
  const int64_t blocks = blocks_of(max_context_len), rows = (int64_t)batch * pool->num_kv_heads;
  if (blocks > max_blocks && rows > kMostBytes / 8 / blocks) return fail(PA_EINVAL, "%s: grid too large", fn);
  *bytes = blocks > max_blocks ? (size_t)rows * blocks * sizeof(uint64_t) : 0;
  return PA_OK;
}

}  // namespace

extern "C" {

int paged_attn_tree_workspace_size(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads, int32_t max_context_len,
                                   int32_t max_nodes, size_t* bytes_out) {
  const char* fn = "paged_attn_tree_workspace_size";
  if (max_nodes > PA_TREE_MAX_NODES)
    return fail(PA_EUNSUPPORTED, "%s: max_nodes = %d > %d", fn, max_nodes, PA_TREE_MAX_NODES);
  return pa::biased_size(pool, batch, num_q_heads, max_context_len, max_nodes, 0, true, bytes_out, fn);
}

int paged_attn_extend_tree(const pa_kv_pool* pool, const void* q, const int32_t* q_start, int32_t total_q,
                           const int32_t* parents, const int32_t* block_tables, int32_t bt_stride,
                           const int32_t* context_lens, int32_t batch, int32_t num_q_heads, float scale, float softcap,
                           int32_t max_context_len, int32_t max_nodes, void* workspace, size_t workspace_bytes, void* out,
                           void* stream) {
  const char* fn = "paged_attn_extend_tree";
  if (max_nodes > PA_TREE_MAX_NODES)
    return fail(PA_EUNSUPPORTED, "%s: max_nodes = %d > %d", fn, max_nodes, PA_TREE_MAX_NODES);
  if (batch > 0 && total_q > 0 && max_nodes > 0 && (!q_start || !parents))
    return fail(PA_EINVAL, "%s: q_start or parents is NULL", fn);
  return pa::biased_call(pool, q, q_start, total_q, parents, block_tables, bt_stride, context_lens, batch, num_q_heads,
                         scale, softcap, nullptr, 0, nullptr, nullptr, max_context_len, max_nodes, workspace,
                         workspace_bytes, out, stream, pa::launch_tree, fn);
}

int paged_attn_block_bounds(const pa_kv_pool* pool, void* bounds, const int32_t* block_tables, int32_t bt_stride,
                            const int32_t* first_tokens, const int32_t* context_lens, int32_t batch,
                            int32_t max_context_len, int32_t max_new, void* stream) {
  const char* fn = "paged_attn_block_bounds";
  int rc = check_batch(pool, batch, max_context_len, fn);
  if (rc || (rc = check_tables(bt_stride, max_context_len, fn))) return rc;
  if (max_new < 0) return fail(PA_EINVAL, "%s: max_new = %d < 0", fn, max_new);
  max_new = std::min(max_new, max_context_len);
  if (batch == 0 || max_new == 0) return PA_OK;
  if (!bounds || !block_tables || !context_lens)
    return fail(PA_EINVAL, "%s: bounds, block_tables and context_lens must be non-NULL", fn);
  if (!aligned(bounds, 16)) return fail(PA_EINVAL, "%s: bounds are not 16-byte aligned", fn);
  if (!aligned(block_tables, 4) || !aligned(context_lens, 4) || !aligned(first_tokens, 4))
    return fail(PA_EINVAL, "%s: block_tables/context_lens/first_tokens are not 4-byte aligned", fn);
  if ((rc = check_grid(((int64_t)batch * ((max_new + 14) / 16 + 1) * pool->num_kv_heads + 3) / 4, 256, fn))) return rc;
  pa::BlocksParams p{};
  p.k_pool = pool->k;
  p.bounds = static_cast<uint16_t*>(bounds);
  p.block_tables = block_tables;
  p.context_lens = context_lens;
  p.first_tokens = first_tokens;
  p.num_blocks = pool->num_blocks;
  p.num_kv_heads = pool->num_kv_heads;
  p.head_dim = pool->head_dim;
  p.batch = batch;
  p.bt_stride = bt_stride;
  p.max_ctx = max_context_len;
  p.max_new = max_new;
  return launched(pa::launch_bounds(p, static_cast<hipStream_t>(stream)), fn);
}

int paged_attn_select_workspace_size(const pa_kv_pool* pool, int32_t batch, int32_t max_context_len, int32_t max_blocks,
                                     size_t* bytes_out) {
  const char* fn = "paged_attn_select_workspace_size";
  if (!bytes_out) return fail(PA_EINVAL, "%s: NULL output pointer", fn);
  size_t bytes = 0;
  const int rc = select_bytes(pool, batch, max_context_len, max_blocks, &bytes, fn);
  if (!rc) *bytes_out = bytes;
  return rc;
}

int paged_attn_select_blocks(const pa_kv_pool* pool, const void* q, const void* bounds, const int32_t* block_tables,
                             int32_t bt_stride, const int32_t* context_lens, int32_t batch, int32_t num_q_heads,
                             int32_t max_context_len, int32_t first_blocks, int32_t last_blocks, int32_t max_blocks,
                             void* workspace, size_t workspace_bytes, int32_t* selected, void* stream) {
  const char* fn = "paged_attn_select_blocks";
  size_t need = 0;
  int rc = select_bytes(pool, batch, max_context_len, max_blocks, &need, fn);
  if (rc || (rc = check_heads(pool, num_q_heads, fn)) || (rc = check_tables(bt_stride, max_context_len, fn))) return rc;
  if (first_blocks < 0 || last_blocks < 1 || (int64_t)first_blocks + last_blocks > max_blocks)
    return fail(PA_EINVAL, "%s: first_blocks = %d >= 0, last_blocks = %d >= 1 and together at most max_blocks = %d are needed",
                fn, first_blocks, last_blocks, max_blocks);
  if (batch == 0) return PA_OK;
  if (!q || !bounds || !block_tables || !context_lens || !selected)
    return fail(PA_EINVAL, "%s: q, bounds, block_tables, context_lens and selected must be non-NULL", fn);
  if (!aligned(q, 16) || !aligned(bounds, 16)) return fail(PA_EINVAL, "%s: q/bounds are not 16-byte aligned", fn);
  if (!aligned(block_tables, 4) || !aligned(context_lens, 4) || !aligned(selected, 4))
    return fail(PA_EINVAL, "%s: block_tables/context_lens/selected are not 4-byte aligned", fn);
  const int64_t rows = (int64_t)batch * pool->num_kv_heads, blocks = blocks_of(max_context_len);
  if ((rc = check_grid(rows, 1024, fn)) || (rc = check_grid(rows * ((blocks + 63) / 64), 256, fn)) ||
      (rc = check_workspace(workspace, workspace_bytes, need, fn)))
    return rc;
  pa::BlocksParams p{};
  p.bounds = static_cast<uint16_t*>(const_cast<void*>(bounds));
  p.q = static_cast<const uint16_t*>(q);
  p.block_tables = block_tables;
  p.context_lens = context_lens;
  p.keys = static_cast<uint64_t*>(workspace);
  p.selected = selected;
  p.num_blocks = pool->num_blocks;
  p.num_kv_heads = pool->num_kv_heads;
  p.group = num_q_heads / pool->num_kv_heads;
  p.head_dim = pool->head_dim;
  p.batch = batch;
  p.bt_stride = bt_stride;
  p.max_ctx = max_context_len;
  p.key_blocks = (int32_t)blocks;
  p.first_blocks = first_blocks;
  p.last_blocks = last_blocks;
  p.max_blocks = max_blocks;
  return launched(pa::launch_select(p, static_cast<hipStream_t>(stream)), fn);
}

int paged_attn_selected_workspace_size(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads, int32_t max_blocks,
                                       size_t* bytes_out) {
  const char* fn = "paged_attn_selected_workspace_size";
  if (!bytes_out) return fail(PA_EINVAL, "%s: NULL output pointer", fn);
  Plan pl;
  const int rc = plan_selected(pool, batch, num_q_heads, max_blocks, &pl, fn);
  if (!rc) *bytes_out = pl.bytes();
  return rc;
}

int paged_attn_decode_selected(const pa_kv_pool* pool, const void* q, const int32_t* block_tables, int32_t bt_stride,
                               const int32_t* context_lens, int32_t batch, int32_t num_q_heads, float scale,
                               int32_t max_context_len, const int32_t* selected, int32_t max_blocks, void* workspace,
                               size_t workspace_bytes, void* out, void* stream) {
  const char* fn = "paged_attn_decode_selected";
  int rc = check_batch(pool, batch, max_context_len, fn);
  if (rc) return rc;
  Plan pl;
  if ((rc = plan_selected(pool, batch, num_q_heads, max_blocks, &pl, fn)) ||
      (rc = check_tables(bt_stride, max_context_len, fn)) || (rc = check_scale(scale, fn)))
    return rc;
  if (batch == 0) return PA_OK;
  if (max_blocks > 0 && !selected) return fail(PA_EINVAL, "%s: selected is NULL", fn);
  if (!aligned(selected, 4)) return fail(PA_EINVAL, "%s: selected is not 4-byte aligned", fn);
  pa::TokensParams p{};
  if ((rc = decode_params(pool, q, block_tables, bt_stride, context_lens, batch, num_q_heads, scale, max_context_len, pl,
                          workspace, workspace_bytes, out, &p, fn)))
    return rc;
  p.selected = selected;
  p.max_blocks = max_blocks;
  return launched(pa::launch_selected(p, static_cast<hipStream_t>(stream)), fn);
}

int paged_attn_weights_workspace_size(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads, int32_t max_context_len,
                                      size_t* bytes_out) {
  const char* fn = "paged_attn_weights_workspace_size";
  if (!bytes_out) return fail(PA_EINVAL, "%s: NULL output pointer", fn);
  Plan pl;
  const int rc = plan_weights(pool, batch, num_q_heads, max_context_len, &pl, fn);
  if (!rc) *bytes_out = pl.bytes();
  return rc;
}

int paged_attn_decode_weights(const pa_kv_pool* pool, const void* q, const int32_t* block_tables, int32_t bt_stride,
                              const int32_t* context_lens, int32_t batch, int32_t num_q_heads, float scale,
                              int32_t max_context_len, float decay, const float* totals, float* totals_out,
                              int64_t totals_stride, void* workspace, size_t workspace_bytes, void* out, void* stream) {
  const char* fn = "paged_attn_decode_weights";
  Plan pl;
  int rc = plan_weights(pool, batch, num_q_heads, max_context_len, &pl, fn);
  if (rc || (rc = check_tables(bt_stride, max_context_len, fn)) || (rc = check_scale(scale, fn))) return rc;
  if (!std::isfinite(decay)) return fail(PA_EINVAL, "%s: decay is not finite", fn);
  if ((rc = check_totals(totals, totals_out, totals_stride, batch, max_context_len, fn))) return rc;
  if (batch == 0) return PA_OK;
  if (!totals_out) return fail(PA_EINVAL, "%s: totals_out is NULL", fn);
  pa::TokensParams p{};
  if ((rc = decode_params(pool, q, block_tables, bt_stride, context_lens, batch, num_q_heads, scale, max_context_len, pl,
                          workspace, workspace_bytes, out, &p, fn)))
    return rc;
  if ((rc = check_grid((int64_t)batch * ((max_context_len + 255) / 256) + ((int64_t)batch * num_q_heads + 3) / 4, 256, fn)))
    return rc;
  p.totals = totals;
  p.totals_out = totals_out;
  p.totals_stride = totals_stride;
  p.decay = decay;
  p.score_tokens = (int32_t)(blocks_of(max_context_len) * PA_BLOCK_SIZE);
  return launched(pa::launch_weights(p, static_cast<hipStream_t>(stream)), fn);
}

int paged_attn_keep_heaviest(const float* totals, int64_t totals_stride, const int32_t* first_tokens,
                             const int32_t* context_lens, int32_t batch, int32_t max_context_len, int32_t recent,
                             int32_t keep, int32_t* kept, int32_t kept_stride, int32_t* kept_lens, void* stream) {
  const char* fn = "paged_attn_keep_heaviest";
  if (batch < 0) return fail(PA_EINVAL, "%s: batch = %d < 0", fn, batch);
  if (max_context_len < 0 || max_context_len >= 1 << 30)
    return fail(PA_EINVAL, "%s: max_context_len = %d outside [0, 2^30)", fn, max_context_len);
  if (recent < 0 || keep < 0) return fail(PA_EINVAL, "%s: recent = %d or keep = %d < 0", fn, recent, keep);
  int rc = check_totals(totals, nullptr, totals_stride, batch, max_context_len, fn);
  if (rc) return rc;
  const int32_t most = std::min(std::max(keep, recent), max_context_len);
  if (kept_stride < most)
    return fail(PA_EINVAL, "%s: kept_stride = %d < min(max(keep, recent), max_context_len) = %d", fn, kept_stride, most);
  if (batch == 0) return PA_OK;
  if (!totals || !context_lens || !kept || !kept_lens)
    return fail(PA_EINVAL, "%s: totals, context_lens, kept and kept_lens must be non-NULL", fn);
  if (!aligned(first_tokens, 4) || !aligned(context_lens, 4) || !aligned(kept, 4) || !aligned(kept_lens, 4))
    return fail(PA_EINVAL, "%s: an index or length array is not 4-byte aligned", fn);
  if ((rc = check_grid(batch, 1024, fn))) return rc;
  pa::KeepParams p{};
  p.totals = totals;
  p.totals_stride = totals_stride;
  p.first_tokens = first_tokens;
  p.context_lens = context_lens;
  p.kept = kept;
  p.kept_lens = kept_lens;
  p.batch = batch;
  p.max_ctx = max_context_len;
  p.recent = recent;
  p.keep = keep;
  p.kept_stride = kept_stride;
  return launched(pa::launch_keep(p, static_cast<hipStream_t>(stream)), fn);
}

int paged_attn_compact(const pa_kv_pool* pool, const int32_t* block_tables, int32_t bt_stride, const int32_t* dst_tables,
                       int32_t dst_stride, const int32_t* first_tokens, const int32_t* context_lens, int32_t batch,
                       int32_t max_context_len, const int32_t* kept, int32_t kept_stride, const int32_t* kept_lens,
                       const float* totals, float* totals_out, int64_t totals_stride, int32_t* new_lens, void* stream) {
  const char* fn = "paged_attn_compact";
  int rc = check_batch(pool, batch, max_context_len, fn);
  if (rc || (rc = check_tables(bt_stride, max_context_len, fn))) return rc;
  if (dst_stride < 0 || (dst_tables ? dst_stride == 0 : dst_stride != 0))
    return fail(PA_EINVAL, "%s: dst_stride = %d %s dst_tables", fn, dst_stride, dst_tables ? "with" : "without");
  if (kept_stride < 0) return fail(PA_EINVAL, "%s: kept_stride = %d < 0", fn, kept_stride);
  if (!totals != !totals_out) return fail(PA_EINVAL, "%s: totals and totals_out are given together or not at all", fn);
  if (totals && (rc = check_totals(totals, totals_out, totals_stride, batch, max_context_len, fn))) return rc;
  if (batch == 0) return PA_OK;
  if (!block_tables || !context_lens || !kept_lens || (kept_stride > 0 && !kept))
    return fail(PA_EINVAL, "%s: block_tables, context_lens, kept and kept_lens must be non-NULL", fn);
  if (!aligned(block_tables, 4) || !aligned(dst_tables, 4) || !aligned(first_tokens, 4) || !aligned(context_lens, 4) ||
      !aligned(kept, 4) || !aligned(kept_lens, 4) || !aligned(new_lens, 4))
    return fail(PA_EINVAL, "%s: an index or length array is not 4-byte aligned", fn);
  // one workgroup of a sequence writes its new length while the others read these
  if (new_lens && (new_lens == first_tokens || new_lens == kept_lens || new_lens == kept || new_lens == block_tables ||
                   new_lens == dst_tables))
    return fail(PA_EINVAL, "%s: new_lens is another of the call's arrays than context_lens", fn);
  // the table itself as the second one: several workgroups to a sequence's rows would read
  // what others of them write
  if (dst_tables == block_tables && dst_stride == bt_stride) {
    dst_tables = nullptr;
    dst_stride = 0;
  }
  pa::CompactParams p{};
  p.k_pool = pool->k;
  p.v_pool = pool->v;
  p.block_tables = block_tables;
  p.dst_tables = dst_tables;
  p.first_tokens = first_tokens;
  p.context_lens = context_lens;
  p.kept = kept;
  p.kept_lens = kept_lens;
  p.totals = totals;
  p.totals_out = totals_out;
  p.new_lens = new_lens;
  p.totals_stride = totals_stride;
  p.num_blocks = pool->num_blocks;
  p.num_kv_heads = pool->num_kv_heads;
  p.head_dim = pool->head_dim;
  p.batch = batch;
  p.bt_stride = bt_stride;
  p.dst_stride = dst_stride;
  p.max_ctx = max_context_len;
  p.kept_stride = kept_stride;
  p.chunks = dst_tables ? pa::compact_chunks(pool->head_dim, std::min(kept_stride, max_context_len)) : 1;
  if ((rc = check_grid((int64_t)batch * (1 + 2 * pool->num_kv_heads * (int64_t)p.chunks), 256, fn))) return rc;
  return launched(pa::launch_compact(p, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
