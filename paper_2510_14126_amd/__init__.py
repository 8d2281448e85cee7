"""MI355X (gfx950) paged decode attention.

The compute lives in the HIP library ``libpaged_attn.so`` behind the C ABI in
``include/paged_attn.h``, ``include/paged_attn_ops.h`` and ``include/paged_attn_tokens.h``; ``binding`` is its
ctypes binding and ``device`` moves one decode step's inputs into device memory with torch.  Importing the
package fails if the library has not been built.
"""
from . import binding  # noqa: F401  (raises ImportError when the library is missing)
from .binding import (  # noqa: F401
    KVPool, PagedAttnError, kv_pool_alloc, kv_pool_claim, kv_pool_create, kv_pool_destroy,
    kv_pool_layout, kv_pool_num_free, kv_pool_num_shared, kv_pool_refcount, kv_pool_release, kv_pool_retain,
    pa_last_error, pa_stream_copy, pa_version, paged_attn_decode, paged_attn_decode_trace,
    paged_attn_num_partitions, paged_attn_reduce, paged_attn_workspace_size,
    paged_attn_cascade_workspace_size, paged_attn_decode_cascade, paged_attn_reduce_cascade,
    PA_BF16, PA_FP16, PA_FP32, PA_ROPE_HALF, PA_ROPE_INTERLEAVED, PA_ROPE_UNSCALED, PA_ROPE_LINEAR, PA_ROPE_NTK,
    PA_ROPE_BANDS, PA_ROPE_YARN, Rope, pa_rope_frequencies, pa_rope_create, pa_rope_destroy, paged_attn_norm_rope,
    paged_attn_rope_append, paged_attn_biased_workspace_size, paged_attn_decode_biased, paged_attn_extend_biased,
    PA_TREE_MAX_NODES, paged_attn_tree_workspace_size, paged_attn_extend_tree, paged_attn_block_bounds,
    paged_attn_select_workspace_size, paged_attn_select_blocks, paged_attn_selected_workspace_size,
    paged_attn_decode_selected, paged_attn_weights_workspace_size, paged_attn_decode_weights,
    paged_attn_keep_heaviest, paged_attn_compact,
)
