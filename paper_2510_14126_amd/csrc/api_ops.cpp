// C ABI of the operators around the cache's attention (paged_attn_ops.h):
// argument validation and launch planning.  Every check runs on the host
// before any HIP call.
#include "kernels.h"
#include "ops.h"
#include "paged_attn_ops.h"
#include "pool.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>

struct pa_rope {
  int32_t head_dim;
  int32_t rotary_dim;
  int32_t layout;
  double magnitude;
  double turns[pa::kRopeMaxDim / 2];   // revolutions per position
};

namespace {
using pa::fail;

// A launch's threads are counted in 32 bits.
constexpr int64_t kMostWorkgroups = 0xffffffffLL / 256;
constexpr int32_t kMostTokens = (1 << 26) - 64;       // of the row operators: one wavefront per token at least

constexpr double kTwoPi = 6.283185307179586476925286766559;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int64_t type_bytes(int32_t dtype) { return dtype == PA_FP32 ? 4 : 2; }

// Rows of one operand: pointer, stride and the values per token that it must hold.
int check_rows(const void* x, int64_t stride, int64_t width, int64_t tokens, int64_t elem, const char* name,
               const char* fn) {
  if (!x) return fail(PA_EINVAL, "%s: %s is NULL", fn, name);
  if (!aligned(x, 16)) return fail(PA_EINVAL, "%s: %s is not 16-byte aligned", fn, name);
  if (stride < width)
    return fail(PA_EINVAL, "%s: %s's stride %lld < heads * head_dim = %lld", fn, name, (long long)stride, (long long)width);
  if (stride > ((int64_t)1 << 60) / elem / tokens)
    return fail(PA_EINVAL, "%s: %s's stride %lld is too large", fn, name, (long long)stride);
  if (stride * elem % 16 != 0)
    return fail(PA_EINVAL, "%s: %s's stride %lld is not a multiple of 16 bytes", fn, name, (long long)stride);
  return PA_OK;
}

// What both row operators check, and what they hand on of the rotation.
int rope_params(const pa_rope* rope, int32_t num_q_heads, int32_t num_kv_heads, const float* q_weight,
                const float* k_weight, float eps, int32_t dtype, pa::RopeParams* p, const char* fn) {
  if (!rope) return fail(PA_EINVAL, "%s: rope is NULL", fn);
  if (num_q_heads < 0 || num_kv_heads < 0 || num_q_heads > 65536 || num_kv_heads > 65536)
    return fail(PA_EINVAL, "%s: %d query and %d KV heads outside [0, 65536]", fn, num_q_heads, num_kv_heads);
  if (dtype != PA_BF16 && dtype != PA_FP16 && dtype != PA_FP32)
    return fail(PA_EINVAL, "%s: dtype = %d is none of PA_BF16, PA_FP16, PA_FP32", fn, dtype);
  if (!(eps >= 0.f) || eps == __builtin_inff())
    return fail(PA_EINVAL, "%s: eps is negative or not finite", fn);
  if (!aligned(q_weight, 16) || !aligned(k_weight, 16))
    return fail(PA_EINVAL, "%s: q_weight/k_weight are not 16-byte aligned", fn);
  p->q_weight = q_weight;
  p->k_weight = k_weight;
  p->num_q_heads = num_q_heads;
  p->num_kv_heads = num_kv_heads;
  p->head_dim = rope->head_dim;
  p->rotary_dim = rope->rotary_dim;
  p->eps = eps;
  p->magnitude = (float)rope->magnitude;
  return PA_OK;
}

}  // namespace

extern "C" {

int pa_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_context,
                        double low, double high, double* freqs_out, double* magnitude_out) {
  const char* fn = "pa_rope_frequencies";
  if (rotary_dim < 0 || rotary_dim % 2 != 0 || rotary_dim > pa::kRopeMaxDim)
    return fail(PA_EINVAL, "%s: rotary_dim = %d is not even in [0, %d]", fn, rotary_dim, pa::kRopeMaxDim);
  if (!(base > 1.0) || !std::isfinite(base)) return fail(PA_EINVAL, "%s: base must be finite and above 1", fn);
  if (scaling < PA_ROPE_UNSCALED || scaling > PA_ROPE_YARN)
    return fail(PA_EINVAL, "%s: unknown scaling %d", fn, scaling);
  if (scaling != PA_ROPE_UNSCALED && (!(factor > 0.0) || !std::isfinite(factor)))
    return fail(PA_EINVAL, "%s: factor must be finite and positive", fn);
  const bool banded = scaling == PA_ROPE_BANDS || scaling == PA_ROPE_YARN;
  if (banded && (!(original_context > 0.0) || !(low > 0.0) || !(low < high) || !std::isfinite(original_context) ||
                 !std::isfinite(high)))
    return fail(PA_EINVAL, "%s: original_context > 0 and 0 < low < high are needed", fn);
  if ((rotary_dim > 0 && !freqs_out) || !magnitude_out) return fail(PA_EINVAL, "%s: NULL output pointer", fn);
  const double r = rotary_dim;
  const int n = rotary_dim / 2;
  // a single pair has no base to change: its frequency is 1 with any
  const double b = scaling == PA_ROPE_NTK && n > 1 ? base * std::pow(factor, r / (r - 2.0)) : base;
  // YaRN's ramp: from the pair that turns `high` times in the original context
  // to the one that turns `low` times
  double from = 0.0, to = 0.0;
  if (scaling == PA_ROPE_YARN && n > 0) {
    auto pair_of = [&](double turns) { return r * std::log(original_context / (turns * kTwoPi)) / (2.0 * std::log(base)); };
    from = std::max(std::floor(pair_of(high)), 0.0);
    to = std::min(std::ceil(pair_of(low)), r - 1.0);
  }
  for (int i = 0; i < n; ++i) {
    double f = std::pow(b, -2.0 * i / r);
    if (scaling == PA_ROPE_LINEAR) {
      f /= factor;
    } else if (scaling == PA_ROPE_BANDS) {
      const double turns = original_context * f / kTwoPi;
      const double keep = std::min(std::max((turns - low) / (high - low), 0.0), 1.0);
      f = f / factor * (1.0 - keep) + f * keep;
    } else if (scaling == PA_ROPE_YARN) {
      const double ramp = std::min(std::max((i - from) / std::max(to - from, 1e-3), 0.0), 1.0);
      f = f / factor * ramp + f * (1.0 - ramp);
    }
    freqs_out[i] = f;
  }
  *magnitude_out = scaling == PA_ROPE_YARN ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return PA_OK;
}

int pa_rope_create(int32_t head_dim, int32_t rotary_dim, int32_t layout, const double* freqs, double magnitude,
                   pa_rope** out) {
  const char* fn = "pa_rope_create";
  if (!out) return fail(PA_EINVAL, "%s: out is NULL", fn);
  if (head_dim < 16 || head_dim > pa::kRopeMaxDim || head_dim % 16 != 0)
    return fail(PA_EUNSUPPORTED, "%s: head_dim = %d is not a multiple of 16 in [16, %d]", fn, head_dim, pa::kRopeMaxDim);
  if (rotary_dim < 0 || rotary_dim > head_dim)
    return fail(PA_EINVAL, "%s: rotary_dim = %d outside [0, head_dim = %d]", fn, rotary_dim, head_dim);
  if (rotary_dim % 16 != 0)
    return fail(PA_EUNSUPPORTED, "%s: rotary_dim = %d is not a multiple of 16", fn, rotary_dim);
  if (layout != PA_ROPE_HALF && layout != PA_ROPE_INTERLEAVED)
    return fail(PA_EINVAL, "%s: unknown layout %d", fn, layout);
  if (rotary_dim > 0 && !freqs) return fail(PA_EINVAL, "%s: freqs is NULL", fn);
  for (int i = 0; i < rotary_dim / 2; ++i)
    if (!std::isfinite(freqs[i])) return fail(PA_EINVAL, "%s: freqs[%d] is not finite", fn, i);
  if (!(std::fabs(magnitude) <= FLT_MAX)) return fail(PA_EINVAL, "%s: magnitude is not finite in fp32", fn);
  pa_rope* r = new (std::nothrow) pa_rope{};
  if (!r) return fail(PA_ENOMEM, "%s: host allocation failed", fn);
  r->head_dim = head_dim;
  r->rotary_dim = rotary_dim;
  r->layout = layout;
  r->magnitude = magnitude;
  for (int i = 0; i < rotary_dim / 2; ++i) r->turns[i] = freqs[i] / kTwoPi;
  *out = r;
  return PA_OK;
}

int pa_rope_destroy(pa_rope* rope) {
  delete rope;
  return PA_OK;
}

int paged_attn_norm_rope(const pa_rope* rope, const void* q, int64_t q_stride, int32_t num_q_heads,
                         const float* q_weight, const void* k, int64_t k_stride, int32_t num_kv_heads,
                         const float* k_weight, float eps, int32_t dtype, const int32_t* positions, int32_t tokens,
                         void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
  const char* fn = "paged_attn_norm_rope";
  pa::RopeParams p{};
  int rc = rope_params(rope, num_q_heads, num_kv_heads, q_weight, k_weight, eps, dtype, &p, fn);
  if (rc) return rc;
  if (tokens < 0 || tokens > kMostTokens)
    return fail(PA_EINVAL, "%s: tokens = %d outside [0, 2^26 - 64]", fn, tokens);
  if (tokens == 0 || num_q_heads + num_kv_heads == 0) return PA_OK;
  const int64_t elem = type_bytes(dtype);
  const struct { const void* x; int64_t stride; int32_t heads; const char* name; } rows[] = {
      {q, q_stride, num_q_heads, "q"}, {q_out, q_out_stride, num_q_heads, "q_out"},
      {k, k_stride, num_kv_heads, "k"}, {k_out, k_out_stride, num_kv_heads, "k_out"}};
  for (const auto& r : rows)
    if (r.heads > 0 && (rc = check_rows(r.x, r.stride, (int64_t)r.heads * rope->head_dim, tokens, elem, r.name, fn))) return rc;
  if (!positions || !aligned(positions, 4))
    return fail(PA_EINVAL, "%s: positions is NULL or not 4-byte aligned", fn);
  p.q = q;
  p.k = k;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.q_out = q_out;
  p.k_out = k_out;
  p.q_out_stride = q_out_stride;
  p.k_out_stride = k_out_stride;
  p.positions = positions;
  p.tokens = tokens;
  const hipError_t e = pa::launch_rope(p, rope->turns, dtype, rope->layout == PA_ROPE_INTERLEAVED, false,
                                       static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(PA_EHIP, "%s: kernel launch failed: %s", fn, hipGetErrorString(e));
  return PA_OK;
}

int paged_attn_rope_append(const pa_kv_pool* pool, const pa_rope* rope, const void* q, int64_t q_stride,
                           int32_t num_q_heads, const float* q_weight, const void* k, int64_t k_stride,
                           const float* k_weight, const void* v, int64_t v_stride, float eps, int32_t dtype,
                           const int32_t* positions, const int32_t* q_start, int32_t total_q,
                           const int32_t* block_tables, int32_t bt_stride, const int32_t* context_lens,
                           int32_t batch, void* q_out, void* stream) {
  const char* fn = "paged_attn_rope_append";
  if (!pool) return fail(PA_EINVAL, "%s: pool is NULL", fn);
  pa::RopeParams p{};
  int rc = rope_params(rope, num_q_heads, pool->num_kv_heads, q_weight, k_weight, eps, dtype, &p, fn);
  if (rc) return rc;
  if (rope->head_dim != pool->head_dim)
    return fail(PA_EINVAL, "%s: the rotation's head_dim = %d, the pool's %d", fn, rope->head_dim, pool->head_dim);
  if (batch < 0) return fail(PA_EINVAL, "%s: batch = %d < 0", fn, batch);
  if (total_q < 0 || total_q > kMostTokens)
    return fail(PA_EINVAL, "%s: total_q = %d outside [0, 2^26 - 64]", fn, total_q);
  if (bt_stride < 1 || (int64_t)bt_stride * PA_BLOCK_SIZE > 0x7fffffffLL)
    return fail(PA_EINVAL, "%s: bt_stride = %d outside [1, 2^27)", fn, bt_stride);
  if (batch == 0 || total_q == 0) return PA_OK;
  const int64_t elem = type_bytes(dtype);
  const int64_t q_width = (int64_t)num_q_heads * pool->head_dim, kv_width = (int64_t)pool->num_kv_heads * pool->head_dim;
  if (num_q_heads > 0 && (rc = check_rows(q, q_stride, q_width, total_q, elem, "q", fn))) return rc;
  if (num_q_heads > 0 && (!q_out || !aligned(q_out, 16)))
    return fail(PA_EINVAL, "%s: q_out is NULL or not 16-byte aligned", fn);
  if ((rc = check_rows(k, k_stride, kv_width, total_q, elem, "k", fn))) return rc;
  if ((rc = check_rows(v, v_stride, kv_width, total_q, elem, "v", fn))) return rc;
  if (!block_tables || !context_lens)
    return fail(PA_EINVAL, "%s: block_tables and context_lens must be non-NULL", fn);
  if (!aligned(block_tables, 4) || !aligned(context_lens, 4) || !aligned(q_start, 4) || !aligned(positions, 4))
    return fail(PA_EINVAL, "%s: block_tables/context_lens/q_start/positions are not 4-byte aligned", fn);
  p.q = q;
  p.k = k;
  p.v = v;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.q_out = q_out;
  p.q_out_stride = q_width;
  p.positions = positions;
  p.tokens = total_q;
  p.k_pool = pool->k;
  p.v_pool = pool->v;
  p.q_start = q_start;
  p.block_tables = block_tables;
  p.context_lens = context_lens;
  p.batch = batch;
  p.bt_stride = bt_stride;
  p.num_blocks = pool->num_blocks;
  const hipError_t e = pa::launch_rope(p, rope->turns, dtype, rope->layout == PA_ROPE_INTERLEAVED, true,
                                       static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(PA_EHIP, "%s: kernel launch failed: %s", fn, hipGetErrorString(e));
  return PA_OK;
}

namespace {

constexpr double kLog2e = 1.4426950408889634;

// How a call's rows and tokens are dealt to workgroups.
//
// Rows: 128 per workgroup over one stream of its tokens (big), or 32 whose
// tokens its wavefronts split, a chain four times shorter per workgroup: while
// those, weighed by the tokens a chunk's average row sees against the longest
// context, are few, or while they are at most twice the others, whose tiles are
// then mostly empty.  32-row / 128-row form, capped, 32 heads over 8, weighed
// workgroups in brackets: D = 128, three chunks of 100 over 2404 tokens (306) 47 /
// 81 us, of 300 over 2604 (859) 97 / 93, of 600 over 2904 (1614) 186 / 144, one
// prompt of 1500 (752) 57 / 56, 2000 (1000) 89 / 74, 8191 (4096) 1149 / 845; D = 64,
// three of 400 over 2704 (1111) 77 / 91, 500 over 2804 (1377) 91 / 95, one prompt of
// 2000 (1000) 58 / 55, 2600 (1300) 90 / 76, 3000 (1500) 112 / 91.
//
// A call's chunks are the bounds max_chunk and max_context_len, or what total_q
// leaves of them with half a tile more per sequence: ragged chunks hold fewer
// rows.  128-row form, taken by the bounds alone / 32-row: three chunks of 82, 230
// and 380 over 2064 tokens, capped, 122 / 84 us; 19 of at most 80 over 7.7K with
// slopes, 8 heads over 8, 311 / 238 us.
//
// Tokens of a 32-row tile: one partition, or several, merged by a second launch
// (2.5 us), where the tiles alone are few workgroups and hold more than
// kWholeBlocks blocks each.  One / several partitions, decode, 32 heads over 8: one
// sequence of 512 tokens 7.0 / 8.7 us, 768 8.9 / 8.5, 1024 10.9 / 8.6.  As many as
// keep the grid within one workgroup per CU, at D = 64, whose workgroups read half
// as much, within two; at most 256 / 512 / 768 workgroups, decode: D = 128, four
// sequences of 16384 tokens, 32 heads over 8, 43.2 / 44.4 / 45.6 us, 4096 13.6 /
// 13.9 / 14.2, three of 10000, 16 over 8, 22.0 / 22.6 / 23.4 (27.1 at 264, a few
// more than the CUs); D = 64, eight of 8192, 32 over 8, 28.0 / 23.5 / 25.2, 16 of
// 4096, 32 over 4, 16.4 / 14.3 / 15.9, four of 9000, 12 over 12, 25.4 / 20.6 / 21.5.
// The bounds alone decide them, as they decide the workspace.
//
// In a decode, whose contexts differ, a partition holds at most kMostBlocks: 256
// of 64..8192 tokens in partitions of at most 64 / 96 / 128 blocks 269 / 265 / 265
// us, 64 with a window of 4096 169 / 168 / 167, of 32 blocks 303 / 175.
constexpr int64_t kFillWorkgroups128 = 256, kFillWorkgroups64 = 512;
constexpr int64_t kWholeBlocks = 40, kLeastBlocks = 16, kMostBlocks = 128;

pa::BiasedPlan biased_plan(int batch, int num_kv_heads, int group, int head_dim, int max_ctx, int max_chunk, int window,
                           int64_t total_q) {
  pa::BiasedPlan pl;
  const int64_t rows = (int64_t)std::max(max_chunk, 1) * group;
  const int64_t tiles = (rows + pa::kBiasedTileRows - 1) / pa::kBiasedTileRows;
  const int64_t big_tiles = (rows + pa::kBiasedWgRows - 1) / pa::kBiasedWgRows;
  const int64_t wgs = std::max<int64_t>(1, batch * tiles * num_kv_heads), big_wgs = batch * big_tiles * num_kv_heads;
  auto long_chunks = [&](int64_t n32, int64_t n128) {
    return max_chunk > 1 && n32 > 2 * n128 &&
           n32 * (2.0 * max_ctx - max_chunk) > 2.0 * (head_dim == 64 ? 1280 : 768) * max_ctx;
  };
  auto tiles_of = [&](int64_t rows_per) { return (total_q * group / rows_per + (batch + 1) / 2) * num_kv_heads; };
  pl.big = long_chunks(wgs, big_wgs) &&
           long_chunks(std::min(wgs, tiles_of(pa::kBiasedTileRows)), std::min(big_wgs, tiles_of(pa::kBiasedWgRows)));
  pl.tiles = (int32_t)(pl.big ? big_tiles : tiles);
  pl.tile_rows = (int32_t)std::min<int64_t>(rows, pa::kBiasedTileRows);
  const int64_t all = ((int64_t)max_ctx + PA_BLOCK_SIZE - 1) / PA_BLOCK_SIZE;
  // a window spans its own tokens and those between a tile's first and last row, wherever they begin in a block
  // (what a prefix adds to it lengthens the partitions in the kernel, see partition_blocks)
  const int64_t blocks = window > 0 ? std::min(all, ((int64_t)window + pa::kBiasedTileRows / group + PA_BLOCK_SIZE - 1) / PA_BLOCK_SIZE + 1) : all;
  int64_t per = blocks;
  if (!pl.big && blocks > kWholeBlocks) {
    const int64_t fill = head_dim == 64 ? kFillWorkgroups64 : kFillWorkgroups128;
    const int64_t parts = std::max<int64_t>(1, fill / wgs);
    per = std::max(kLeastBlocks, (blocks + 2 * parts - 1) / (2 * parts) * 2);
    if (max_chunk <= 1) per = std::min(per, kMostBlocks);
  }
  per = std::max<int64_t>(per, 1);
  pl.parts = (int32_t)std::max<int64_t>(1, (blocks + per - 1) / per);
  pl.part_blocks = (int32_t)std::min<int64_t>(per, 0x7fffffff);
  return pl;
}

size_t biased_part_o_bytes(const pa::BiasedPlan& pl, int64_t slots, int32_t head_dim) {
  return pl.parts > 1 ? (size_t)slots * pl.parts * pl.tile_rows * head_dim * sizeof(float) : 0;
}
size_t biased_lse_bytes(const pa::BiasedPlan& pl, int64_t slots) {
  return pl.parts > 1 ? ((size_t)slots * pl.parts * pl.tile_rows * sizeof(float) + 15) / 16 * 16 : 0;
}

// Geometry and plan of a biased call, and its number of row tiles.
int plan_biased(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads, int32_t max_context_len,
                int32_t max_chunk, int32_t window, int64_t total_q, pa::BiasedPlan* pl, int64_t* slots, const char* fn) {
  if (!pool) return fail(PA_EINVAL, "%s: pool is NULL", fn);
  if (batch < 0) return fail(PA_EINVAL, "%s: batch = %d < 0", fn, batch);
  if (num_q_heads <= 0 || num_q_heads % pool->num_kv_heads != 0)
    return fail(PA_EINVAL, "%s: num_q_heads = %d is not a positive multiple of num_kv_heads = %d", fn, num_q_heads,
                pool->num_kv_heads);
  // the kernels' token indexes stay below the mark of a row that sees nothing, 2^30 - 1
  if (max_context_len < 0 || max_context_len >= 1 << 30)
    return fail(PA_EINVAL, "%s: max_context_len = %d outside [0, 2^30)", fn, max_context_len);
  if (max_chunk < 0 || max_chunk > std::max(max_context_len, 1))
    return fail(PA_EINVAL, "%s: max_chunk = %d outside [0, max_context_len = %d]", fn, max_chunk, max_context_len);
  if (window < 0) return fail(PA_EINVAL, "%s: window = %d < 0", fn, window);
  const int32_t group = num_q_heads / pool->num_kv_heads;
  const int64_t rows = (int64_t)std::max(max_chunk, 1) * group;
  if (rows > 0x7fffffffLL) return fail(PA_EINVAL, "%s: max_chunk * heads per KV head = %lld is too large", fn, (long long)rows);
  const int64_t tiles = (rows + pa::kBiasedTileRows - 1) / pa::kBiasedTileRows;
  *slots = (int64_t)batch * tiles;
  if (*slots > 0x7fffffffLL / pool->num_kv_heads) return fail(PA_EINVAL, "%s: grid too large", fn);
  *slots *= pool->num_kv_heads;
  *pl = biased_plan(batch, pool->num_kv_heads, group, pool->head_dim, max_context_len, max_chunk, window,
                    total_q);
  if (*slots * pl->parts > 0x7fffffffLL || (pl->parts > 1 && *slots * pl->tile_rows > 0x7fffffffLL))
    return fail(PA_EINVAL, "%s: grid too large", fn);
  return PA_OK;
}

int biased_impl(const pa_kv_pool* pool, const void* q, const int32_t* q_start, int32_t total_q,
                const int32_t* block_tables, int32_t bt_stride, const int32_t* context_lens, int32_t batch,
                int32_t num_q_heads, float scale, float softcap, const float* slopes, int32_t window,
                const int32_t* first_tokens, const int32_t* prefix_lens, int32_t max_context_len, int32_t max_chunk,
                void* workspace, size_t workspace_bytes, void* out, void* stream, const char* fn) {
  pa::BiasedPlan pl;
  int64_t slots = 0;
  int rc = plan_biased(pool, batch, num_q_heads, max_context_len, max_chunk, window, total_q, &pl, &slots, fn);
  if (rc) return rc;
  if (total_q < 0) return fail(PA_EINVAL, "%s: total_q = %d < 0", fn, total_q);
  const int64_t need_bt = ((int64_t)max_context_len + PA_BLOCK_SIZE - 1) / PA_BLOCK_SIZE;
  if (bt_stride < need_bt || bt_stride < 0)
    return fail(PA_EINVAL, "%s: bt_stride = %d < ceil(max_context_len / 16) = %lld", fn, bt_stride, (long long)need_bt);
  if (!std::isfinite((float)(scale * kLog2e)))
    return fail(PA_EINVAL, "%s: scale is not finite, or not in log2 units", fn);
  if (!(softcap >= 0.f) || !std::isfinite(softcap))
    return fail(PA_EINVAL, "%s: softcap is negative or not finite", fn);
  if (batch == 0 || total_q == 0 || max_chunk == 0) return PA_OK;
  if (!q || !block_tables || !context_lens || !out)
    return fail(PA_EINVAL, "%s: q, block_tables, context_lens and out must be non-NULL", fn);
  if (!aligned(q, 16) || !aligned(out, 16)) return fail(PA_EINVAL, "%s: q/out are not 16-byte aligned", fn);
  if (!aligned(block_tables, 4) || !aligned(context_lens, 4) || !aligned(q_start, 4) || !aligned(slopes, 4) ||
      !aligned(first_tokens, 4) || !aligned(prefix_lens, 4))
    return fail(PA_EINVAL, "%s: an index, length or slope array is not 4-byte aligned", fn);
  const int64_t row_tiles = (int64_t)batch * pl.tiles * pool->num_kv_heads;
  if (row_tiles * pl.parts > kMostWorkgroups || (pl.parts > 1 && (row_tiles * pl.tile_rows + 3) / 4 > kMostWorkgroups))
    return fail(PA_EINVAL, "%s: grid too large", fn);
  const size_t o_bytes = biased_part_o_bytes(pl, slots, pool->head_dim);
  const size_t need = o_bytes + biased_lse_bytes(pl, slots);
  if (workspace_bytes < need)
    return fail(PA_EINVAL, "%s: workspace of %zu bytes, %zu are needed", fn, workspace_bytes, need);
  if (need > 0 && (!workspace || !aligned(workspace, 16)))
    return fail(PA_EINVAL, "%s: workspace is NULL or not 16-byte aligned", fn);
  pa::BiasedParams p{};
  p.k_pool = pool->k;
  p.v_pool = pool->v;
  p.q = static_cast<const uint16_t*>(q);
  p.q_start = q_start;
  p.block_tables = block_tables;
  p.context_lens = context_lens;
  p.slopes = slopes;
  p.first_tokens = first_tokens;
  p.prefix_lens = prefix_lens;
  p.out = static_cast<uint16_t*>(out);
  p.part_o = static_cast<float*>(workspace);
  p.part_lse = need > 0 ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + o_bytes) : nullptr;
  p.num_blocks = pool->num_blocks;
  p.num_kv_heads = pool->num_kv_heads;
  p.num_q_heads = num_q_heads;
  p.group = num_q_heads / pool->num_kv_heads;
  p.head_dim = pool->head_dim;
  p.batch = batch;
  p.bt_stride = bt_stride;
  p.max_ctx = max_context_len;
  p.max_chunk = max_chunk;
  p.total_q = total_q;
  p.window = window;
  p.big = pl.big;
  // more than one workgroup per CU and at most two; a chunk's last tile may be part of one
  const int64_t full = (int64_t)total_q * p.group / pa::kBiasedWgRows, cus = pa::kCus / pool->num_kv_heads;
  p.ranked = pl.big && batch <= 64 && cus > 0 && full > cus && full + batch <= 2 * cus;
  p.tiles = pl.tiles;
  p.parts = pl.parts;
  p.part_blocks = pl.part_blocks;
  p.tile_rows = pl.tile_rows;
  p.stream_tiles = !q_start && pl.tiles == 1 && pool->shared_blocks == 0;
  p.scale_log2 = (float)(scale * kLog2e);
  if (softcap > 0.f) {
    // tanh(z) / z on |z| <= 1/2 as a polynomial in z^2, z = raw * |scale| / softcap
    constexpr double kT[4] = {0.9999994557709386, -0.33326317935941446, 0.1319029660321076, -0.04440222612772746};
    const double s = std::fabs((double)scale), z = s / softcap;
    double c[4], reach = 0.5;
    for (int i = 3; i >= 0; --i) {
      c[i] = kT[i] * s * kLog2e * std::pow(z, 2 * i);
      // a coefficient below fp32's normal numbers: only as far as its term is below 2^-23
      if (i > 0 && std::fabs(c[i]) < FLT_MIN) reach = std::pow(0x1p-23 / std::fabs(kT[i]), 0.5 / i);
    }
    constexpr double kMostRaw = 1e19;                  // its square is finite in fp32
    p.cap = (float)(softcap * kLog2e);
    p.c0 = (float)c[0];
    p.c1 = (float)c[1];
    p.c2 = (float)c[2];
    p.c3 = (float)c[3];
    p.raw_max = (float)std::min(reach / std::max(z, 1e-30), kMostRaw);
    p.two_z = (float)(2.0 * kLog2e * z);
    if (!std::isfinite(p.cap) || !std::isfinite(p.c1) || !std::isfinite(p.c2) || !std::isfinite(p.c3) ||
        !std::isfinite(p.two_z) || (s > 0.0 && reach / z > kMostRaw))
      return fail(PA_EUNSUPPORTED, "%s: softcap = %g with scale = %g leaves the range of fp32", fn, softcap, scale);
  }
  const hipError_t e = pa::launch_biased(p, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(PA_EHIP, "%s: kernel launch failed: %s", fn, hipGetErrorString(e));
  return PA_OK;
}

}  // namespace

int paged_attn_biased_workspace_size(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads,
                                     int32_t max_context_len, int32_t max_chunk, int32_t window, size_t* bytes_out) {
  const char* fn = "paged_attn_biased_workspace_size";
  if (!bytes_out) return fail(PA_EINVAL, "%s: NULL output pointer", fn);
  pa::BiasedPlan pl;
  int64_t slots = 0;
  const int rc = plan_biased(pool, batch, num_q_heads, max_context_len, max_chunk, window, 0, &pl, &slots, fn);
  if (rc) return rc;
  *bytes_out = biased_part_o_bytes(pl, slots, pool->head_dim) + biased_lse_bytes(pl, slots);
  return PA_OK;
}

int paged_attn_decode_biased(const pa_kv_pool* pool, const void* q, const int32_t* block_tables, int32_t bt_stride,
                             const int32_t* context_lens, int32_t batch, int32_t num_q_heads, float scale,
                             float softcap, const float* slopes, int32_t window, const int32_t* first_tokens,
                             int32_t max_context_len, void* workspace, size_t workspace_bytes, void* out,
                             void* stream) {
  return biased_impl(pool, q, nullptr, batch, block_tables, bt_stride, context_lens, batch, num_q_heads, scale,
                     softcap, slopes, window, first_tokens, nullptr, max_context_len, 1, workspace, workspace_bytes,
                     out, stream, "paged_attn_decode_biased");
}

int paged_attn_extend_biased(const pa_kv_pool* pool, const void* q, const int32_t* q_start, int32_t total_q,
                             const int32_t* block_tables, int32_t bt_stride, const int32_t* context_lens,
                             int32_t batch, int32_t num_q_heads, float scale, float softcap, const float* slopes,
                             int32_t window, const int32_t* first_tokens, const int32_t* prefix_lens,
                             int32_t max_context_len, int32_t max_chunk, void* workspace, size_t workspace_bytes,
                             void* out, void* stream) {
  const char* fn = "paged_attn_extend_biased";
  if (batch > 0 && total_q > 0 && max_chunk > 0 && !q_start) return fail(PA_EINVAL, "%s: q_start is NULL", fn);
  return biased_impl(pool, q, q_start, total_q, block_tables, bt_stride, context_lens, batch, num_q_heads, scale,
                     softcap, slopes, window, first_tokens, prefix_lens, max_context_len, max_chunk, workspace,
                     workspace_bytes, out, stream, fn);
}

}  // extern "C"
