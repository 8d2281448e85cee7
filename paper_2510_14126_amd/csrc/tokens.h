// Kernel parameter blocks and launchers of the operators that choose tokens of a
// paged context (paged_attn_tokens.h).  Host code fills these after validating
// every argument.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pa {

// Decode attention over listed blocks (selected), or over the whole context with
// the weights added to totals (scores).
struct TokensParams {
  const uint16_t* k_pool;        // bf16 [num_blocks][num_kv_heads][16][head_dim]
  const uint16_t* v_pool;
  const uint16_t* q;             // bf16 [batch][num_q_heads][head_dim]
  const int32_t* block_tables;   // [batch][bt_stride]
  const int32_t* context_lens;   // [batch]
  const int32_t* selected;       // [batch][num_kv_heads][max_blocks], or NULL: all blocks
  uint16_t* out;                 // bf16 [batch][num_q_heads][head_dim]
  float* part_o;                 // parts > 1: fp32 [batch][head tiles][kv heads][parts][tile_heads][head_dim]
  float* part_lse;               // fp32 [batch][head tiles][kv heads][parts][tile_heads], log2 units
  float* scores;                 // weights: fp32 [batch][head tiles][kv heads][score_tokens][tile_heads], log2 units
  const float* totals;           // weights: [batch][totals_stride], or NULL
  float* totals_out;
  int64_t totals_stride;
  float decay;
  int32_t num_blocks;
  int32_t num_kv_heads;
  int32_t num_q_heads;
  int32_t group;                 // query heads per KV head
  int32_t head_dim;              // 64 or 128
  int32_t head_tiles;            // tiles of tile_heads query heads of a KV head
  int32_t tile_heads;            // 4 or 8: columns of a matrix tile
  int32_t batch;
  int32_t bt_stride;
  int32_t max_ctx;
  int32_t max_blocks;            // selected
  int32_t score_tokens;          // max_ctx rounded up to whole blocks
  int32_t parts;                 // partitions of a row's blocks
  int32_t part_blocks;           // blocks of one
  int32_t whole_blocks;          // weights: rows of no more are one partition, if LDS holds their scores
  int32_t stream_tiles;          // 1: load the tiles with the streaming cache hint
  float scale_log2;              // scale * log2(e)
};
hipError_t launch_selected(const TokensParams& p, hipStream_t stream);
hipError_t launch_weights(const TokensParams& p, hipStream_t stream);

// Bounds of blocks' keys, and the choice of blocks by them.
struct BlocksParams {
  const uint16_t* k_pool;
  uint16_t* bounds;              // bf16 [num_blocks][num_kv_heads][2][head_dim]: written by the bounds, else read
  const uint16_t* q;             // bf16 [batch][num_q_heads][head_dim]
  const int32_t* block_tables;
  const int32_t* context_lens;
  const int32_t* first_tokens;   // bounds: [batch], or NULL
  uint64_t* keys;                // select: [batch][num_kv_heads][key_blocks], ascending with the score
  int32_t* selected;             // [batch][num_kv_heads][max_blocks]
  int32_t num_blocks;
  int32_t num_kv_heads;
  int32_t group;
  int32_t head_dim;
  int32_t batch;
  int32_t bt_stride;
  int32_t max_ctx;
  int32_t max_new;               // bounds: tokens
  int32_t key_blocks;            // blocks of max_ctx
  int32_t first_blocks, last_blocks, max_blocks;
};
hipError_t launch_bounds(const BlocksParams& p, hipStream_t stream);
hipError_t launch_select(const BlocksParams& p, hipStream_t stream);

// The tokens with the largest totals.
struct KeepParams {
  const float* totals;           // [batch][totals_stride]
  int64_t totals_stride;
  const int32_t* first_tokens;   // [batch], or NULL
  const int32_t* context_lens;
  int32_t* kept;                 // [batch][kept_stride]
  int32_t* kept_lens;
  int32_t batch;
  int32_t max_ctx;
  int32_t recent, keep;
  int32_t kept_stride;
};
hipError_t launch_keep(const KeepParams& p, hipStream_t stream);

// Moves of chosen tokens.
struct CompactParams {
  uint16_t* k_pool;
  uint16_t* v_pool;
  const int32_t* block_tables;
  const int32_t* dst_tables;     // or NULL: block_tables, in place
  const int32_t* first_tokens;   // or NULL
  const int32_t* context_lens;
  const int32_t* kept;
  const int32_t* kept_lens;
  const float* totals;           // or NULL, with totals_out
  float* totals_out;
  int32_t* new_lens;             // or NULL
  int64_t totals_stride;
  int32_t num_blocks;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t batch;
  int32_t bt_stride, dst_stride;
  int32_t max_ctx;
  int32_t kept_stride;
  int32_t chunks;                // workgroups per (sequence, KV head, pool): 1 in place
};
// Rows that a workgroup of a move has in flight, and the workgroups for `rows` of them
// of a (sequence, KV head, pool).
constexpr int kMoveThreads = 256, kMovePasses = 8;
inline int compact_chunks(int head_dim, int rows) {
  const int per = kMovePasses * kMoveThreads / (head_dim / 8);
  return rows > per ? (int)(((int64_t)rows + per - 1) / per) : 1;
}
hipError_t launch_compact(const CompactParams& p, hipStream_t stream);

}  // namespace pa
