// Host-side state of a KV block pool handle, shared by the sources of the C
// ABI.
#pragma once

#include "paged_attn.h"

#include <vector>

struct pa_kv_pool {
  int32_t num_blocks;
  int32_t num_kv_heads;
  int32_t head_dim;
  uint16_t* k;                     // caller-owned device pools (the append writes them)
  uint16_t* v;
  std::vector<int32_t> refcount;  // 0 = free
  std::vector<int32_t> free_stack; // top = back(); ids pop in ascending order initially
  int64_t shared_blocks = 0;       // blocks whose reference count is 2 or more
  int64_t shared_refs = 0;         // references of those blocks
};
