"""Arrays that a move of kept tokens may not be given twice: its workgroups read the
first tokens, the lists and their lengths while one of them writes the new lengths.
Host checks alone: every call is refused or is a no-op."""
import pytest

pytest.importorskip("torch")

from paper_2510_14126_amd import binding as pa  # noqa: E402

AT = {name: 0x10000 * (i + 1) for i, name in enumerate(
    ["block_tables", "dst_tables", "first_tokens", "context_lens", "kept", "kept_lens", "totals", "new_lens"])}


def compact(batch=3, **kw):
    pool = pa.kv_pool_create(8, 16, 2, 64, 0x10000, 0x10000)
    args = dict(bt_stride=8, dst_stride=8, batch=batch, max_context_len=100, kept_stride=40, totals_stride=100,
                totals_out=AT["totals"], **AT)
    return pa.paged_attn_compact(pool, **{**args, **kw})


@pytest.mark.parametrize("name", ["first_tokens", "kept_lens", "kept", "block_tables", "dst_tables"])
def test_new_lens_is_no_other_array(name):
    with pytest.raises(pa.PagedAttnError) as e:
        compact(new_lens=AT[name])
    assert e.value.code == pa.PA_EINVAL and "new_lens" in str(e.value)
    compact(batch=0, new_lens=AT[name])          # an empty batch writes none
