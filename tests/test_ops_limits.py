"""Sizes at which the operators of paged_attn_ops.h refuse a call.  No kernel is
launched."""
import pytest

torch = pytest.importorskip("torch")

from paper_2510_14126_amd import binding as pa  # noqa: E402

A = 0x10000                       # an aligned placeholder device address (never dereferenced)


@pytest.mark.parametrize("top", [2 ** 30, 2 ** 30 + 1, 2 ** 31 - 1])
def test_biased_contexts_beyond_the_kernels_integers(top):
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    for call in (lambda: pa.paged_attn_biased_workspace_size(pool, 1, 8, top),
                 lambda: pa.paged_attn_decode_biased(pool, A, A, 2 ** 27, A, 1, 8, 0.1, 0.0, None, 64, None, top, A,
                                                     1 << 40, A),
                 lambda: pa.paged_attn_extend_biased(pool, A, A, 3, A, 2 ** 27, A, 1, 8, 0.1, 0.0, None, 64, A, A, top,
                                                     3, A, 1 << 40, A)):
        with pytest.raises(pa.PagedAttnError) as e:
            call()
        assert e.value.code == pa.PA_EINVAL and "max_context_len" in str(e.value)
    assert pa.paged_attn_biased_workspace_size(pool, 1, 8, 2 ** 30 - 1) > 0


def test_rows_beyond_the_threads_of_a_launch():
    """A launch's threads are counted in 32 bits: one wavefront per token at least."""
    rope = pa.pa_rope_create(64, 64, pa.PA_ROPE_HALF, [1.0] * 32)
    pool = pa.kv_pool_create(8, 16, 1, 64, A, A)
    for tokens in (2 ** 26, 2 ** 31 - 1):
        for call in (lambda: pa.paged_attn_norm_rope(rope, A, 64, 1, None, A, 64, 1, None, 0.0, pa.PA_BF16, A, tokens, A,
                                                     64, A, 64),
                     lambda: pa.paged_attn_rope_append(pool, rope, A, 64, 1, None, A, 64, None, A, 64, 0.0, pa.PA_BF16,
                                                       None, A, tokens, A, 4, A, 2, A)):
            with pytest.raises(pa.PagedAttnError) as e:
                call()
            assert e.value.code == pa.PA_EINVAL and "2^26" in str(e.value)


def test_biased_grids_beyond_the_threads_of_a_launch():
    pool = pa.kv_pool_create(8, 16, 64, 64, A, A)
    big = 1 << 40
    for call in (lambda: pa.paged_attn_decode_biased(pool, A, A, 4, A, 2 ** 18, 64, 0.1, 0.0, None, 0, None, 50, A, big, A),
                 lambda: pa.paged_attn_extend_biased(pool, A, A, 9, A, 4, A, 2 ** 18, 64, 0.1, 0.0, None, 0, None, None,
                                                     50, 2, A, big, A),
                 # the merge: a wavefront per row
                 lambda: pa.paged_attn_decode_biased(pool, A, A, 256, A, 2 ** 16, 64 * 32, 0.1, 0.0, None, 0, None, 4096,
                                                     A, big, A)):
        with pytest.raises(pa.PagedAttnError) as e:
            call()
        assert e.value.code == pa.PA_EINVAL and "grid too large" in str(e.value)


@pytest.mark.parametrize("magnitude", [1e39, -1e300])
def test_magnitudes_beyond_fp32(magnitude):
    with pytest.raises(pa.PagedAttnError) as e:
        pa.pa_rope_create(64, 16, pa.PA_ROPE_HALF, [1.0] * 8, magnitude)
    assert e.value.code == pa.PA_EINVAL and "magnitude" in str(e.value)
