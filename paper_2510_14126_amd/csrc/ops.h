// Kernel parameter blocks and launchers of the operators around the cache's
// attention (paged_attn_ops.h): head norms with rotary positions, the rotated
// append, and attention with capped, biased or masked scores.  Host code fills
// these after validating every argument.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

struct pa_kv_pool;

namespace pa {

constexpr int kRopeMaxDim = 256;        // largest head_dim of the row operators

// Rows of q and k (and, for the append, v) of a batch of tokens.
struct RopeParams {
  const void* q;                 // [tokens] rows of num_q_heads x head_dim, q_stride elements apart
  const void* k;
  const void* v;                 // append only
  int64_t q_stride, k_stride, v_stride;
  void* q_out;
  void* k_out;                   // not for the append
  int64_t q_out_stride, k_out_stride;
  const float* q_weight;         // [head_dim], or NULL: no norm
  const float* k_weight;
  const int32_t* positions;      // [tokens]; append: or NULL, the token's slot
  int32_t tokens;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;              // a multiple of 16, at most kRopeMaxDim
  int32_t rotary_dim;            // a multiple of 16, at most head_dim
  int32_t waves;                 // wavefronts per token (set by the launcher)
  float eps;
  float magnitude;
  // append: the paged cache
  uint16_t* k_pool;              // bf16 [num_blocks][num_kv_heads][16][head_dim]
  uint16_t* v_pool;
  const int32_t* q_start;        // [batch + 1], or NULL: one token per sequence
  const int32_t* block_tables;   // [batch][bt_stride]
  const int32_t* context_lens;   // [batch], the chunk included
  int32_t batch;
  int32_t bt_stride;
  int32_t num_blocks;
};
// turns: revolutions per position of each of the rotary_dim / 2 pairs (host
// memory); dtype: PA_BF16, PA_FP16 or PA_FP32; interleaved: pairs (2i, 2i + 1).
hipError_t launch_rope(const RopeParams& p, const double* turns, int dtype, bool interleaved, bool append,
                       hipStream_t stream);

// Attention of new tokens over their sequences' paged context with capped,
// biased or masked scores.
struct BiasedParams {
  const uint16_t* k_pool;        // bf16 [num_blocks][num_kv_heads][16][head_dim]
  const uint16_t* v_pool;
  const uint16_t* q;             // bf16 [total_q][num_q_heads][head_dim]
  const int32_t* q_start;        // [batch + 1], or NULL: row b is sequence b's one new token
  const int32_t* block_tables;   // [batch][bt_stride]
  const int32_t* context_lens;   // [batch], the new tokens included
  const float* slopes;           // [num_q_heads], or NULL
  const int32_t* first_tokens;   // [total_q], or NULL
  const int32_t* prefix_lens;    // [batch], or NULL
  uint16_t* out;                 // bf16 [total_q][num_q_heads][head_dim]
  float* part_o;                 // parts > 1: fp32 [row tiles][parts][tile_rows][head_dim]
  float* part_lse;               // fp32 [row tiles][parts][tile_rows], log2 units
  int32_t num_blocks;
  int32_t num_kv_heads;
  int32_t num_q_heads;
  int32_t group;                 // query heads per KV head
  int32_t head_dim;              // 64 or 128
  int32_t batch;
  int32_t bt_stride;
  int32_t max_ctx;
  int32_t max_chunk;
  int32_t total_q;
  int32_t window;                // 0: none
  int32_t big;                   // 1: kBiasedWgRows rows per workgroup, 0: kBiasedTileRows
  int32_t ranked;                // big: 1: the GPU holds all workgroups at once, paired by length (batch <= 64)
  int32_t tiles;                 // row tiles (of that many rows) per sequence in the grid
  int32_t parts;                 // partitions of a tile's tokens in the grid
  int32_t part_blocks;           // blocks of a partition (even), where there are several; see partition_blocks
  int32_t tile_rows;             // rows of a tile that the partial buffers hold
  int32_t stream_tiles;          // 1: load the tiles with the streaming cache hint
  float scale_log2;              // scale * log2(e)
  // softcap > 0, scores in log2 units x = raw * |scale_log2|: y = raw * (c0 + c1 raw^2
  // + c2 raw^4 + c3 raw^6) while |raw| <= raw_max (|z| <= 1/2, or as far as coefficients
  // that fp32 holds reach), cap - 2 cap / (2^(raw * two_z) + 1) above
  float cap;                     // softcap * log2(e), or 0
  float c0, c1, c2, c3;
  float raw_max;
  float two_z;                   // 2 log2(e) |scale| / softcap
  const int32_t* parents;        // [total_q], trees only
};
constexpr int kBiasedTileRows = 32;     // query rows (token x head) of a row tile
constexpr int kBiasedWgRows = 128;      // rows of a workgroup in the form for long chunks
constexpr int kCus = 256;               // compute units of the GPU
constexpr int kTreeMostNodes = 256;     // of one sequence's tree

// Blocks of one partition of a row tile that sees nblk blocks.  The plan's
// part_blocks reach a window and the positions of a tile's rows; a prefix that sees
// itself whole adds up to the rest of the chunk, and its tiles take longer
// partitions, in the same number.
__host__ __device__ inline int partition_blocks(const BiasedParams& p, int nblk) {
  if (p.parts == 1) return nblk;
  if (p.prefix_lens == nullptr || p.window == 0) return p.part_blocks;
  const uint32_t two = 2u * (uint32_t)p.parts;          // parts < 2^24, blocks <= 2^27: no overflow
  const int even = (int)(((uint32_t)nblk + two - 1) / two) * 2;
  return even > p.part_blocks ? even : p.part_blocks;
}

// Rows and token partitions of a call (kernel launch and workspace size).
struct BiasedPlan {
  int32_t tiles, tile_rows, parts, part_blocks, big;
};
hipError_t launch_biased(const BiasedParams& p, hipStream_t stream);

// A tree of drafted tokens (paged_attn_tokens.h) is planned, checked and
// dispatched as a biased extend with its parents and its own kernels.
using BiasedLaunch = hipError_t (*)(const BiasedParams&, hipStream_t);
hipError_t launch_tree(const BiasedParams& p, hipStream_t stream);
int biased_size(const pa_kv_pool* pool, int32_t batch, int32_t num_q_heads, int32_t max_context_len,
                int32_t max_chunk, int32_t window, bool tree, size_t* bytes_out, const char* fn);
int biased_call(const pa_kv_pool* pool, const void* q, const int32_t* q_start, int32_t total_q, const int32_t* parents,
                const int32_t* block_tables, int32_t bt_stride, const int32_t* context_lens, int32_t batch,
                int32_t num_q_heads, float scale, float softcap, const float* slopes, int32_t window,
                const int32_t* first_tokens, const int32_t* prefix_lens, int32_t max_context_len, int32_t max_chunk,
                void* workspace, size_t workspace_bytes, void* out, void* stream, BiasedLaunch launch, const char* fn);

}  // namespace pa
