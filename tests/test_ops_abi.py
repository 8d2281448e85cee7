"""Host-side tests of the operators in paged_attn_ops.h: exports, frequencies,
refusals and no-ops.  No kernel is launched: every call is refused, is a no-op,
or handles host metadata."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle.ops import biased_rows, head_rows  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "include", "paged_attn_ops.h")
A = 0x10000                       # an aligned placeholder device address (never dereferenced)


def test_header_library_and_binding_agree():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"^\s*int\s+([a-z_0-9]+)\s*\(", src, flags=re.M)))
    assert names == sorted(pa.OPS_SIGNATURES) and len(names) == 8
    for n in names:
        assert hasattr(pa.library(), n) and hasattr(pa, n)
    for n, v in re.findall(r"\b(PA_[A-Z0-9_]+) = (\d+)", src):
        assert getattr(pa, n) == int(v)


# --------------------------------------------------------------------------
# frequencies and handles
# --------------------------------------------------------------------------

def expected(r, base, kind, factor, original, low, high):
    f = np.array([base ** (-2 * i / r) for i in range(r // 2)])
    if kind == pa.PA_ROPE_LINEAR:
        f = f / factor
    if kind == pa.PA_ROPE_NTK:
        f = np.array([(base * factor ** (r / (r - 2))) ** (-2 * i / r) for i in range(r // 2)])
    if kind == pa.PA_ROPE_BANDS:
        for i, x in enumerate(f):
            turns = original / (2 * math.pi / x)
            if turns < low:
                f[i] = x / factor
            elif turns <= high:
                s = (turns - low) / (high - low)
                f[i] = (1 - s) * x / factor + s * x
    if kind == pa.PA_ROPE_YARN:
        def pair(turns):
            return r * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), r - 1)
        for i, x in enumerate(f):
            ramp = min(max((i - a) / max(b - a, 1e-3), 0), 1)
            f[i] = x / factor * ramp + x * (1 - ramp)
    return f, 0.1 * math.log(factor) + 1 if kind == pa.PA_ROPE_YARN else 1.0


@pytest.mark.parametrize("r", [16, 64, 128, 256])
@pytest.mark.parametrize("kind", range(5))
def test_frequencies(r, kind):
    args = (r, 10000.0, kind, 8.0, 8192.0, 1.0, 32.0)
    got, magnitude = pa.pa_rope_frequencies(*args)
    want, m = expected(*args)
    assert len(got) == r // 2 and magnitude == pytest.approx(m, rel=1e-15)
    assert np.allclose(got, want, rtol=1e-13, atol=0)


def test_frequencies_small_dims():
    assert pa.pa_rope_frequencies(0, 10000.0)[0] == []
    assert pa.pa_rope_frequencies(2, 10000.0, pa.PA_ROPE_NTK, 4.0)[0] == [1.0]


@pytest.mark.parametrize("args", [(3, 1e4), (-2, 1e4), (258, 1e4), (16, 1.0), (16, float("inf")), (16, float("nan")),
                                  (16, 1e4, 5), (16, 1e4, -1), (16, 1e4, 1, 0.0), (16, 1e4, 2, float("nan")),
                                  (16, 1e4, 3, 2.0, 0.0, 1.0, 4.0), (16, 1e4, 3, 2.0, 10.0, 4.0, 4.0),
                                  (16, 1e4, 4, 2.0, 10.0, 0.0, 4.0), (16, 1e4, 4, 2.0, 10.0, 1.0, float("inf"))])
def test_frequencies_refusals(args):
    with pytest.raises(pa.PagedAttnError) as e:
        pa.pa_rope_frequencies(*args)
    assert e.value.code == pa.PA_EINVAL and "pa_rope_frequencies" in str(e.value)


@pytest.mark.parametrize("args,code", [
    ((72, 16, 0, [1.0] * 8), pa.PA_EUNSUPPORTED), ((272, 16, 0, [1.0] * 8), pa.PA_EUNSUPPORTED),
    ((64, 20, 0, [1.0] * 10), pa.PA_EUNSUPPORTED), ((64, 80, 0, [1.0] * 40), pa.PA_EINVAL),
    ((64, -16, 0, []), pa.PA_EINVAL), ((64, 16, 2, [1.0] * 8), pa.PA_EINVAL), ((64, 16, 0, [1.0] * 7), pa.PA_EINVAL),
    ((64, 16, 0, [float("nan")] * 8), pa.PA_EINVAL), ((64, 16, 0, [1.0] * 8, float("inf")), pa.PA_EINVAL)])
def test_rope_create_refusals(args, code):
    with pytest.raises(pa.PagedAttnError) as e:
        pa.pa_rope_create(*args)
    assert e.value.code == code


def test_rope_handle_closes():
    r = pa.pa_rope_create(64, 0, pa.PA_ROPE_HALF, [])
    pa.pa_rope_destroy(r)
    r.close()
    with pytest.raises(pa.PagedAttnError):
        pa.paged_attn_norm_rope(r, A, 64, 1, None, A, 64, 1, None, 0.0, 0, A, 1, A, 64, A, 64)


# --------------------------------------------------------------------------
# refusals of the device calls
# --------------------------------------------------------------------------

NORM = dict(q=A, q_stride=512, num_q_heads=8, q_weight=A, k=A, k_stride=128, num_kv_heads=2, k_weight=None, eps=1e-6,
            dtype=pa.PA_BF16, positions=A, tokens=3, q_out=A, q_out_stride=512, k_out=A, k_out_stride=128)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(q=A + 8), dict(q_stride=504), dict(q_stride=516), dict(q_stride=-512), dict(num_q_heads=-1),
    dict(num_q_heads=9), dict(num_q_heads=65537), dict(q_weight=A + 4), dict(k_weight=A + 8), dict(k=None), dict(k=A + 2),
    dict(k_stride=64), dict(num_kv_heads=-2), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(dtype=3), dict(dtype=-1), dict(positions=None), dict(positions=A + 2), dict(tokens=-1), dict(q_out=None),
    dict(q_out=A + 4), dict(q_out_stride=8), dict(k_out=None), dict(k_out_stride=2 ** 62), dict(k_out_stride=130),
    dict(tokens=2 ** 31 - 1, q_stride=2 ** 40)], ids=str)
def test_norm_rope_refusals(bad):
    rope = pa.pa_rope_create(64, 64, pa.PA_ROPE_HALF, [1.0] * 32)
    with pytest.raises(pa.PagedAttnError) as e:
        pa.paged_attn_norm_rope(rope, **{**NORM, **bad})
    assert e.value.code == pa.PA_EINVAL and "paged_attn_norm_rope" in str(e.value)


def test_norm_rope_no_ops():
    rope = pa.pa_rope_create(64, 64, pa.PA_ROPE_HALF, [1.0] * 32)
    pa.paged_attn_norm_rope(rope, **{**NORM, "tokens": 0, "q": None, "positions": None})
    pa.paged_attn_norm_rope(rope, **{**NORM, "num_q_heads": 0, "num_kv_heads": 0, "q": None, "k": None})


APPEND = dict(q=A, q_stride=512, num_q_heads=8, q_weight=None, k=A, k_stride=128, k_weight=A, v=A, v_stride=128,
              eps=1e-6, dtype=pa.PA_BF16, positions=None, q_start=A, total_q=5, block_tables=A, bt_stride=4,
              context_lens=A, batch=2, q_out=A)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(q_stride=500), dict(q_out=None), dict(q_out=A + 8), dict(k=None), dict(k_stride=127), dict(v=None),
    dict(v=A + 1), dict(v_stride=0), dict(eps=-1.0), dict(dtype=7), dict(positions=A + 1), dict(q_start=A + 2),
    dict(total_q=-1), dict(block_tables=None), dict(block_tables=A + 2), dict(bt_stride=0), dict(bt_stride=1 << 27),
    dict(context_lens=None), dict(context_lens=A + 3), dict(batch=-1), dict(num_q_heads=-8)], ids=str)
def test_rope_append_refusals(bad):
    rope = pa.pa_rope_create(64, 64, pa.PA_ROPE_HALF, [1.0] * 32)
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    with pytest.raises(pa.PagedAttnError) as e:
        pa.paged_attn_rope_append(pool, rope, **{**APPEND, **bad})
    assert e.value.code == pa.PA_EINVAL and "paged_attn_rope_append" in str(e.value)


def test_rope_append_head_dims_and_no_ops():
    rope = pa.pa_rope_create(128, 64, pa.PA_ROPE_HALF, [1.0] * 32)
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    with pytest.raises(pa.PagedAttnError) as e:
        pa.paged_attn_rope_append(pool, rope, **APPEND)
    assert e.value.code == pa.PA_EINVAL
    rope = pa.pa_rope_create(64, 64, pa.PA_ROPE_HALF, [1.0] * 32)
    for empty in (dict(batch=0), dict(total_q=0)):
        pa.paged_attn_rope_append(pool, rope, **{**APPEND, "q": None, "k": None, "block_tables": None, **empty})


DECODE = dict(q=A, block_tables=A, bt_stride=8, context_lens=A, batch=2, num_q_heads=8, scale=0.1, softcap=30.0,
              slopes=None, window=0, first_tokens=None, max_context_len=100, workspace=A, workspace_bytes=1 << 30, out=A)
EXTEND = dict(q=A, q_start=A, total_q=9, block_tables=A, bt_stride=8, context_lens=A, batch=2, num_q_heads=8, scale=0.1,
              softcap=0.0, slopes=A, window=5, first_tokens=A, prefix_lens=A, max_context_len=100, max_chunk=7,
              workspace=A, workspace_bytes=1 << 30, out=A)
COMMON = [dict(q=None), dict(q=A + 8), dict(block_tables=None), dict(block_tables=A + 1), dict(bt_stride=6),
          dict(bt_stride=-1), dict(context_lens=None), dict(context_lens=A + 2), dict(batch=-1), dict(num_q_heads=0),
          dict(num_q_heads=7), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-3.0e38), dict(softcap=-1.0),
          dict(softcap=float("nan")), dict(softcap=float("inf")), dict(slopes=A + 2), dict(window=-1),
          dict(first_tokens=A + 1), dict(max_context_len=-1), dict(out=None), dict(out=A + 4)]
LONG = dict(bt_stride=4096, max_context_len=65536)      # split: needs a workspace


@pytest.mark.parametrize("bad", COMMON + [dict(LONG, workspace=None), dict(LONG, workspace=A + 8),
                                          dict(LONG, workspace_bytes=100)], ids=str)
def test_decode_biased_refusals(bad):
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    with pytest.raises(pa.PagedAttnError) as e:
        pa.paged_attn_decode_biased(pool, **{**DECODE, **bad})
    assert e.value.code == pa.PA_EINVAL and "paged_attn_decode_biased" in str(e.value)


@pytest.mark.parametrize("bad", COMMON + [dict(q_start=None), dict(q_start=A + 2), dict(total_q=-1), dict(max_chunk=-1),
                                          dict(max_chunk=101), dict(prefix_lens=A + 3),
                                          dict(LONG, window=0, workspace=None), dict(LONG, window=0, workspace_bytes=0)],
                         ids=str)
def test_extend_biased_refusals(bad):
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    with pytest.raises(pa.PagedAttnError) as e:
        pa.paged_attn_extend_biased(pool, **{**EXTEND, **bad})
    assert e.value.code == pa.PA_EINVAL and "paged_attn_extend_biased" in str(e.value)


@pytest.mark.parametrize("cap,scale", [(1e-30, 0.1), (3.0e38, 0.1), (1e-3, 1e30)])
def test_biased_refuses_caps_beyond_fp32(cap, scale):
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    with pytest.raises(pa.PagedAttnError) as e:
        pa.paged_attn_decode_biased(pool, **{**DECODE, "softcap": cap, "scale": scale})
    assert e.value.code == pa.PA_EUNSUPPORTED


def test_biased_no_ops():
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    pa.paged_attn_decode_biased(pool, **{**DECODE, "batch": 0, "q": None, "out": None})
    for empty in (dict(batch=0), dict(total_q=0), dict(max_chunk=0)):
        pa.paged_attn_extend_biased(pool, **{**EXTEND, "q": None, "q_start": None, "out": None, **empty})


def test_biased_workspace_size():
    pool = pa.kv_pool_create(8, 16, 2, 64, A, A)
    size = pa.paged_attn_biased_workspace_size
    assert size(pool, 0, 8, 100) == 0 and size(pool, 4, 8, 100) == 0 and size(pool, 1, 8, 0) == 0
    assert size(pool, 1, 8, 65536) > 0
    assert size(pool, 1, 8, 65536, 1, 4096) < size(pool, 1, 8, 65536)
    assert size(pool, 100000, 8, 65536, 64) == 0              # the row tiles alone fill the GPU
    for bad in ((-1, 8, 100), (1, 9, 100), (1, 8, -1), (1, 8, 100, 101), (1, 8, 100, 1, -1), (2 ** 31 - 1, 8, 100)):
        with pytest.raises(pa.PagedAttnError) as e:
            size(pool, *bad)
        assert e.value.code == pa.PA_EINVAL
    with pytest.raises(pa.PagedAttnError):
        size(pool, 1, 2 ** 30, 2 ** 31 - 1, 2 ** 31 - 1)


# --------------------------------------------------------------------------
# native calls
# --------------------------------------------------------------------------

NATIVE = {
    "paged_attn_norm_rope": ["rope", "t", 512, 8, "t", "t", 128, 2, None, 1e-6, 0, "t", 0, "t", 512, "t", 128, None],
    "paged_attn_rope_append": ["pool", "rope", "t", 512, 8, None, "t", 128, None, "t", 128, 1e-6, 0, None, "t", 0, "t",
                               4, "t", 0, "t", None],
    "paged_attn_decode_biased": ["pool", "t", "t", 8, "t", 0, 8, 0.1, 30.0, None, 0, None, 100, "t", 0, "t", None],
    "paged_attn_extend_biased": ["pool", "t", "t", 0, "t", 8, "t", 0, 8, 0.1, 30.0, None, 0, None, None, 100, 7, "t", 0,
                                 "t", None],
}


def test_every_native_operator_is_listed():
    assert set(pa._pycall.OPS_NAMES) == set(NATIVE)


@pytest.mark.parametrize("name", sorted(NATIVE))
def test_same_status_as_ctypes(name):
    t = torch.zeros(64, dtype=torch.int32)
    pool = pa.kv_pool_create(4, 16, 2, 64, t, t)
    rope = pa.pa_rope_create(64, 64, pa.PA_ROPE_HALF, [1.0] * 32)
    fill = {"pool": pool.handle, "rope": rope.handle, "t": t}
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
        if type(a) is int and NATIVE[name][i] not in ("pool", "rope"):
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

@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_rotation_pins(interleaved):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 3, 32))
    f = [1.0, 0.5, 0.25, 0.125]
    y = head_rows(x, None, 0.0, [0, 1, 7, 100], f, 1.0, interleaved)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 8:], x[..., 8:])
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))            # turns keep lengths
    a, b = (2, 3) if interleaved else (1, 5)                          # pair 1 of token 2, by hand
    t = 7 * 0.5
    assert y[2, 1, a] == pytest.approx(x[2, 1, a] * math.cos(t) - x[2, 1, b] * math.sin(t))
    assert y[2, 1, b] == pytest.approx(x[2, 1, b] * math.cos(t) + x[2, 1, a] * math.sin(t))
    # scores of turned rows depend on the distance alone
    q, k = head_rows(x[:1], None, 0.0, [50], f, 1.0, interleaved), head_rows(x[1:2], None, 0.0, [47], f, 1.0, interleaved)
    q2, k2 = head_rows(x[:1], None, 0.0, [3], f, 1.0, interleaved), head_rows(x[1:2], None, 0.0, [0], f, 1.0, interleaved)
    assert np.allclose((q * k).sum(-1), (q2 * k2).sum(-1))
    n = head_rows(x, np.full(32, 2.0), 1e-6, [0] * 4, [], 1.0, interleaved)
    assert np.allclose((n ** 2).mean(-1), 4.0, rtol=1e-5)


def test_oracle_attention_pins():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 8)), rng.standard_normal((20, 8)), rng.standard_normal((20, 4))
    pos, zero = np.array([4, 9, 19]), np.zeros(3)
    one = biased_rows(q, k, v, 0.3, 0.0, zero, pos, pos, pos + 1)
    assert np.allclose(one, v[pos])                                   # a row that sees one token
    assert (biased_rows(q, k, v, 0.3, 5.0, zero, pos, pos, pos) == 0).all()
    mean = biased_rows(q, k, v, 0.0, 5.0, zero, pos, zero, pos + 1)
    assert np.allclose(mean[1], v[:10].mean(0))                       # equal scores
    near = biased_rows(q, k, v, 0.3, 0.0, np.full(3, 1e6), pos, zero, np.full(3, 20))
    assert np.allclose(near, v[pos])                                  # a steep distance bias
    tiny = biased_rows(q, k, v, 0.3, 1e6, zero, pos, zero, pos + 1)
    assert np.allclose(tiny, biased_rows(q, k, v, 0.3, 0.0, zero, pos, zero, pos + 1))   # a cap far above
    s = 3.0 * np.tanh(0.3 * (k[:5] @ q[0]) / 3.0) - 0.2 * np.abs(4 - np.arange(5))
    w = np.exp(s) / np.exp(s).sum()
    assert np.allclose(biased_rows(q, k, v, 0.3, 3.0, np.full(3, 0.2), pos, zero, pos + 1)[0], w @ v[:5])
