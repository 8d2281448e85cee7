"""Host-side tests of the operators in paged_attn_tokens.h: exports, refusals,
no-ops, workspace sizes, and the oracle's own pins.  No kernel is launched: every
call is refused or is a no-op."""
import ctypes
import os
import re
from fractions import Fraction

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tokens as oracle  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "include", "paged_attn_tokens.h")
A = 0x10000                       # an aligned placeholder device address (never dereferenced)
BIG = 2 ** 31 - 1


def test_header_library_and_binding_agree():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"^\s*int\s+([a-z_0-9]+)\s*\(", src, flags=re.M)))
    assert names == sorted(pa.TOKENS_SIGNATURES) and len(names) == 11
    import paper_2510_14126_amd
    for n in names:
        assert hasattr(pa.library(), n) and hasattr(pa, n) and hasattr(paper_2510_14126_amd, n)
        declared = re.search(rf"\b{n}\s*\((.*?)\);", src, flags=re.S).group(1)
        assert len(declared.split(",")) == len(pa.TOKENS_SIGNATURES[n][1])
    for n, v in re.findall(r"\b(PA_[A-Z0-9_]+) = (\d+)", src):
        assert getattr(pa, n) == int(v)


POOL = dict(blocks=8, hkv=2, d=64)
SEQ = dict(block_tables=A, bt_stride=8, context_lens=A, batch=3)
CALLS = {
    "paged_attn_extend_tree": dict(q=A, q_start=A, total_q=9, parents=A, **SEQ, num_q_heads=8, scale=0.1, softcap=0.0,
                                   max_context_len=100, max_nodes=8, workspace=A, workspace_bytes=1 << 40, out=A),
    "paged_attn_block_bounds": dict(bounds=A, first_tokens=A, **SEQ, max_context_len=100, max_new=5),
    "paged_attn_select_blocks": dict(q=A, bounds=A, **SEQ, num_q_heads=8, max_context_len=100, first_blocks=1,
                                     last_blocks=1, max_blocks=4, workspace=A, workspace_bytes=1 << 40, selected=A),
    "paged_attn_decode_selected": dict(q=A, **SEQ, num_q_heads=8, scale=0.1, max_context_len=100, selected=A,
                                       max_blocks=100, workspace=A, workspace_bytes=1 << 40, out=A),
    "paged_attn_decode_weights": dict(q=A, **SEQ, num_q_heads=8, scale=0.1, max_context_len=100, decay=1.0, totals=A,
                                      totals_out=A, totals_stride=100, workspace=A, workspace_bytes=1 << 40, out=A),
    "paged_attn_keep_heaviest": dict(totals=A, totals_stride=100, first_tokens=A, context_lens=A, batch=3,
                                     max_context_len=100, recent=10, keep=40, kept=A, kept_stride=40, kept_lens=A),
    "paged_attn_compact": dict(**SEQ, dst_tables=A, dst_stride=4, first_tokens=A, max_context_len=100, kept=A,
                               kept_stride=40, kept_lens=A, totals=A, totals_out=A, totals_stride=100, new_lens=A),
}


def call(name, **kw):
    args = {**CALLS[name], **kw}
    if name == "paged_attn_keep_heaviest":
        return pa.paged_attn_keep_heaviest(**args)
    pool = pa.kv_pool_create(POOL["blocks"], 16, POOL["hkv"], POOL["d"], A, A)
    return getattr(pa, name)(pool, **args)


REFUSALS = [
    ("paged_attn_extend_tree", k, v, c) for k, v, c in [
        ("max_nodes", 257, pa.PA_EUNSUPPORTED), ("max_nodes", -1, pa.PA_EINVAL), ("max_nodes", 101, pa.PA_EINVAL),
        ("num_q_heads", 9, pa.PA_EINVAL), ("num_q_heads", 0, pa.PA_EINVAL), ("batch", -1, pa.PA_EINVAL),
        ("total_q", -1, pa.PA_EINVAL), ("max_context_len", 1 << 30, pa.PA_EINVAL), ("max_context_len", -1, pa.PA_EINVAL),
        ("bt_stride", 6, pa.PA_EINVAL), ("scale", float("nan"), pa.PA_EINVAL), ("scale", 3e38, pa.PA_EINVAL),
        ("softcap", -1.0, pa.PA_EINVAL), ("softcap", float("inf"), pa.PA_EINVAL), ("softcap", 1e-30, pa.PA_EUNSUPPORTED),
        ("q", None, pa.PA_EINVAL), ("q", A + 8, pa.PA_EINVAL), ("q_start", None, pa.PA_EINVAL),
        ("parents", None, pa.PA_EINVAL), ("parents", A + 2, pa.PA_EINVAL), ("block_tables", None, pa.PA_EINVAL),
        ("context_lens", None, pa.PA_EINVAL), ("out", None, pa.PA_EINVAL), ("out", A + 4, pa.PA_EINVAL)]
] + [
    ("paged_attn_block_bounds", k, v, pa.PA_EINVAL) for k, v in [
        ("bounds", None), ("bounds", A + 8), ("block_tables", None), ("block_tables", A + 1), ("context_lens", None),
        ("first_tokens", A + 2), ("batch", -1), ("max_context_len", -1), ("max_context_len", 1 << 30), ("bt_stride", 6),
        ("max_new", -1)]
] + [
    ("paged_attn_select_blocks", k, v, pa.PA_EINVAL) for k, v in [
        ("q", None), ("q", A + 2), ("bounds", None), ("bounds", A + 4), ("selected", None), ("selected", A + 1),
        ("block_tables", None), ("context_lens", None), ("num_q_heads", 3), ("first_blocks", -1), ("last_blocks", 0),
        ("first_blocks", 4), ("max_blocks", 0), ("first_blocks", BIG), ("bt_stride", 6), ("batch", -1),
        ("max_context_len", -1), ("workspace", None), ("workspace", A + 8), ("workspace_bytes", 100)]
] + [
    ("paged_attn_decode_selected", k, v, pa.PA_EINVAL) for k, v in [
        ("q", None), ("q", A + 2), ("selected", None), ("selected", A + 2), ("max_blocks", -1), ("num_q_heads", 7),
        ("scale", float("inf")), ("bt_stride", 6), ("batch", -1), ("max_context_len", 1 << 30), ("workspace", None),
        ("workspace_bytes", 100), ("out", None), ("out", A + 8), ("context_lens", A + 1), ("block_tables", None)]
] + [
    ("paged_attn_decode_weights", k, v, pa.PA_EINVAL) for k, v in [
        ("q", None), ("out", None), ("totals_out", None), ("totals", A + 2), ("totals_out", A + 1),
        ("totals_stride", 99), ("totals_stride", 1 << 60), ("decay", float("nan")), ("decay", float("inf")),
        ("scale", float("nan")), ("num_q_heads", 0), ("bt_stride", 6), ("batch", -1), ("max_context_len", 1 << 30),
        ("workspace", None), ("workspace", A + 4), ("workspace_bytes", 100), ("context_lens", None)]
] + [
    ("paged_attn_keep_heaviest", k, v, pa.PA_EINVAL) for k, v in [
        ("totals", None), ("totals", A + 2), ("totals_stride", 99), ("totals_stride", 1 << 60), ("context_lens", None),
        ("kept", None), ("kept", A + 1), ("kept_lens", None), ("kept_stride", 39), ("recent", -1), ("keep", -1),
        ("recent", 41), ("batch", -1), ("max_context_len", -1), ("max_context_len", 1 << 30), ("first_tokens", A + 3)]
] + [
    ("paged_attn_compact", k, v, pa.PA_EINVAL) for k, v in [
        ("block_tables", None), ("bt_stride", 6), ("dst_stride", 0), ("dst_stride", -1), ("dst_tables", None),
        ("dst_tables", A + 2), ("context_lens", None), ("kept", None), ("kept", A + 2), ("kept_lens", None),
        ("kept_stride", -1), ("totals", None), ("totals_out", None), ("totals_stride", 99), ("batch", -1),
        ("max_context_len", -1), ("new_lens", A + 2)]
]


@pytest.mark.parametrize("name,key,value,code", REFUSALS)
def test_refusals(name, key, value, code):
    with pytest.raises(pa.PagedAttnError) as e:
        call(name, **{key: value})
    assert e.value.code == code and name in str(e.value)


def test_short_workspace_is_refused():
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    need = pa.paged_attn_tree_workspace_size(pool, 1, 8, 65536, 8)
    with pytest.raises(pa.PagedAttnError) as e:
        call("paged_attn_extend_tree", batch=1, bt_stride=4096, max_context_len=65536, workspace_bytes=need - 1)
    assert e.value.code == pa.PA_EINVAL and need > 0


@pytest.mark.parametrize("name", sorted(CALLS))
def test_no_ops(name):
    """An empty batch reads no pointer."""
    nulls = {k: None for k, v in CALLS[name].items() if v == A}
    if name == "paged_attn_compact":
        nulls["dst_stride"] = 0
    call(name, batch=0, **nulls)
    if name == "paged_attn_extend_tree":
        call(name, total_q=0, **nulls)
        call(name, max_nodes=0, **nulls)
    if name == "paged_attn_block_bounds":
        call(name, max_new=0, **nulls)


def test_workspace_sizes():
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    assert pa.paged_attn_tree_workspace_size(pool, 4, 8, 100, 8) == 0
    assert pa.paged_attn_tree_workspace_size(pool, 1, 8, 65536, 8) > 0
    assert pa.paged_attn_select_workspace_size(pool, 3, 1600, 100) == 0          # all blocks are taken
    assert pa.paged_attn_select_workspace_size(pool, 3, 1601, 100) == 3 * 2 * 101 * 8
    assert pa.paged_attn_selected_workspace_size(pool, 3, 8, 40) == 0
    assert pa.paged_attn_selected_workspace_size(pool, 0, 8, 4000) == 0
    assert pa.paged_attn_selected_workspace_size(pool, 1, 8, 4000) > 0
    one = pa.paged_attn_weights_workspace_size(pool, 1, 8, 100)
    assert one >= 2 * 4 * 112 * 4                                                # scores of 7 blocks
    assert pa.paged_attn_weights_workspace_size(pool, 1, 10, 100) >= 2 * one - 64    # five heads take a tile of eight
    for bad in ((-1, 8, 100), (1, 9, 100), (1, 8, -1), (1, 8, 1 << 30), (BIG, 8 * 10 ** 6, (1 << 30) - 1)):
        with pytest.raises(pa.PagedAttnError) as e:
            pa.paged_attn_weights_workspace_size(pool, *bad)
        assert e.value.code == pa.PA_EINVAL
    for fn, bad in ((pa.paged_attn_selected_workspace_size, (1, 8, -1)), (pa.paged_attn_select_workspace_size, (1, 10, 0)),
                    (pa.paged_attn_selected_workspace_size, (BIG, 8 * 10 ** 6, 10)),
                    (pa.paged_attn_tree_workspace_size, (1, 8, 1000, 300))):
        with pytest.raises(pa.PagedAttnError):
            fn(pool, *bad)
    many = pa.kv_pool_create(8, 16, 64, 64, A, A)                                # 2^66 bytes: no size_t holds them
    with pytest.raises(pa.PagedAttnError):
        pa.paged_attn_select_workspace_size(many, BIG, 2 ** 30 - 1, 5)


# --------------------------------------------------------------------------
# native calls
# --------------------------------------------------------------------------

NATIVE = {
    "paged_attn_extend_tree": ["pool", "t", "t", 0, "t", "t", 8, "t", 0, 8, 0.1, 30.0, 100, 7, "t", 0, "t", None],
    "paged_attn_block_bounds": ["pool", "t", "t", 8, "t", "t", 0, 100, 5, None],
    "paged_attn_select_blocks": ["pool", "t", "t", "t", 8, "t", 0, 8, 100, 1, 1, 4, "t", 0, "t", None],
    "paged_attn_decode_selected": ["pool", "t", "t", 8, "t", 0, 8, 0.1, 100, "t", 4, "t", 0, "t", None],
    "paged_attn_decode_weights": ["pool", "t", "t", 8, "t", 0, 8, 0.1, 100, 1.0, "t", "t", 100, "t", 0, "t", None],
    "paged_attn_keep_heaviest": ["t", 100, "t", "t", 0, 100, 10, 40, "t", 40, "t", None],
    "paged_attn_compact": ["pool", "t", 8, "t", 4, "t", "t", 0, 100, "t", 40, "t", "t", "t", 100, "t", None],
}


def test_every_native_operator_is_listed():
    assert set(pa._pycall.TOKENS_NAMES) == set(NATIVE)
    assert set(pa.PER_STEP) == set(pa._pycall.NAMES) | set(pa._pycall.OPS_NAMES) | set(pa._pycall.TOKENS_NAMES)


@pytest.mark.parametrize("name", sorted(NATIVE))
def test_same_status_as_ctypes(name):
    t = torch.zeros(64, dtype=torch.int32)
    pool = pa.kv_pool_create(4, 16, 2, 64, t, t)
    fill = {"pool": pool.handle, "t": t}
    args = [fill.get(a, a) if isinstance(a, str) else a for a in NATIVE[name]]
    native, plain = getattr(pa._pycall, name), getattr(pa._lib, name)

    def both(a):
        rc = native(*a)
        said = pa.pa_last_error()
        assert rc == plain(*[x.data_ptr() if hasattr(x, "data_ptr") else x for x in a])
        assert rc == pa.PA_OK or said == pa.pa_last_error()
        return rc

    assert both(args) == pa.PA_OK
    refused = 0
    for i, a in enumerate(args):
        if type(a) is int and NATIVE[name][i] != "pool":
            refused += both(args[:i] + [-1] + args[i + 1:]) != pa.PA_OK
        elif type(a) is float:
            refused += both(args[:i] + [float("nan")] + args[i + 1:]) != pa.PA_OK
    assert refused >= 2
    with pytest.raises(TypeError):
        native(*args[:-1])
    with pytest.raises(ctypes.ArgumentError):
        native(*[1.5 if type(a) is int else a for a in args])


# --------------------------------------------------------------------------
# the oracle's own pins
# --------------------------------------------------------------------------

def test_oracle_paths():
    parents = [-1, 0, 0, 1, -1, 4, 3]
    assert [oracle.path(parents, i) for i in range(7)] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5], [0, 1, 3, 6]]
    assert oracle.path([0, 5, 1], 2) == [1, 2] and oracle.path([-7], 0) == [0]     # parents that are none


def test_oracle_tree_is_attention_over_each_path():
    from oracle import extend_attention  # noqa: F401  (a chain is an ordinary chunk)
    from oracle.ops import biased_attention
    rng = np.random.default_rng(1)
    k, v = (rng.integers(0x3F00, 0x4040, (4, 2, 16, 8)).astype(np.uint16) for _ in range(2))
    q = rng.standard_normal((5, 4, 8))
    tables, start, ctx = np.array([[2, 0], [3, 1]]), np.array([0, 3, 5]), np.array([20, 2])
    chain = oracle.tree_attention(q, start, [-1, 0, 1, -1, 0], k, v, tables, ctx, 0.3, 5.0)
    assert np.allclose(chain, biased_attention(q, start, k, v, tables, ctx, 0.3, 5.0))
    roots = oracle.tree_attention(q, start, [-1] * 5, k, v, tables, ctx, 0.3)
    for i in range(3):      # siblings: each as the only new token
        from oracle.attention import gather_sequence
        K, V = gather_sequence(k, v, tables[0], 20)
        seen = list(range(17)) + [17 + i]
        for h in range(4):
            s = np.exp(0.3 * K[h // 2][seen] @ q[i, h])
            assert np.allclose(roots[i, h], (s / s.sum()) @ V[h // 2][seen])


def test_oracle_choice_pins():
    q = np.array([[1.0, -2.0], [0.5, 0.0]])
    assert oracle.block_score(q, np.array([[-1.0, -3.0], [2.0, 1.0]])) == Fraction(2 + 6 + 1)
    rows = np.array([[1.0, np.nan], [-2.0, 5.0], [0.0, 3.0]])
    assert np.array_equal(oracle.block_bounds(rows), [[-2.0, 3.0], [1.0, 5.0]])
    s = [9, 1, 5, 5, 5, 7, 0, 2]
    assert oracle.select_blocks(s, 1, 2, 5) == [0, 2, 5, 6, 7]           # 7, then the first 5
    assert oracle.select_blocks(s, 0, 1, 8) == list(range(8))
    rng = np.random.default_rng(2)      # the score bounds every key of the block
    k, q = rng.standard_normal((16, 8)), rng.standard_normal((3, 8))
    assert float(oracle.block_score(q, oracle.block_bounds(k))) >= (q @ k.T).sum(0).max()


def test_oracle_eviction_pins():
    t = np.array([1.0, 0.0, 3.0, 3.0, 0.5, 3.0, np.nan, 0.0])
    assert oracle.keep_heaviest(t, 0, 0, 3) == [2, 3, 6]                 # NaN, then the first of the equal ones
    assert oracle.keep_heaviest(t, 2, 1, 5) == [0, 4, 5]                 # tokens 2, 6 and 7 behind the first two
    assert oracle.keep_heaviest(t, 6, 4, 3) == [0, 1]                    # the first and the last ones alone
    assert oracle.keep_heaviest(t, 0, 0, 0) == [] and oracle.keep_heaviest(t, 0, 0, 99) == list(range(8))
    pool = np.arange(3 * 16).reshape(3, 1, 16, 1)
    got = oracle.compact(pool, [2, 0], [2, 0], 1, [0, 4, 20])
    assert got[2, 0, 1:4, 0].tolist() == [33, 37, 5] and (np.delete(got.ravel(), [33, 34, 35]) == np.delete(pool.ravel(), [33, 34, 35])).all()


def test_oracle_weights_pins():
    rng = np.random.default_rng(3)
    k, v = (rng.integers(0x3F00, 0x4040, (3, 2, 16, 8)).astype(np.uint16) for _ in range(2))
    out, w = oracle.decode_weights(rng.standard_normal((2, 4, 8)), k, v, np.array([[0, 1], [2, 2]]), np.array([23, 0]), 0.3)
    assert w[0].shape == (23,) and w[0].sum() == pytest.approx(4.0) and w[1].size == 0 and (out[1] == 0).all()
    zero, w = oracle.decode_weights(np.zeros((1, 2, 8)), k, v, np.array([[0, 1]]), np.array([23]), 0.3)
    assert np.allclose(w[0], 2 / 23)
