"""Norm and rotation of head rows, and the rotated append, against the float64
oracle on the same inputs.

Tolerance of one output value, from the roundings on its way (u = 2^-24, half
a step of the rows' type e = finfo.eps / 2): the row's sum of squares, the
inverse root, two products with inverse and weight, and the two products and a
sum of the turn, with cos and sin off by at most 4 u each, stay below 24 u of
the pair's length (a row without norm and turn: 0); then the rounding to the
type, e of the value.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle.ops import head_rows  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, pa.PA_BF16), "fp16": (torch.float16, pa.PA_FP16), "fp32": (torch.float32, pa.PA_FP32)}
EPS = 1e-5


def half_step(t):
    return torch.finfo(t).eps / 2


def rotation(d, rot, layout, scaling=pa.PA_ROPE_UNSCALED):
    extra = (8.0, 4096.0, 1.0, 32.0) if scaling else (1.0, 0.0, 0.0, 0.0)
    freqs, magnitude = pa.pa_rope_frequencies(rot, 10000.0, scaling, *extra)
    return pa.pa_rope_create(d, rot, layout, freqs, magnitude), freqs, magnitude


def check(got, x, weight, positions, freqs, magnitude, interleaved, out_type, steps=24):
    """got, x: [n][heads][d] tensors."""
    ref = head_rows(x.double().cpu().numpy(), None if weight is None else weight.double().cpu().numpy(),
                    np.float64(np.float32(EPS)), np.asarray(positions), freqs, magnitude, interleaved)
    y = got.double().cpu().numpy()
    half = len(freqs)
    length = np.abs(ref)
    if half:
        i = np.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        pair = np.hypot(ref[..., a], ref[..., b])
        length[..., a], length[..., b] = pair, pair
    limit = steps * 2.0 ** -24 * length + half_step(out_type) * np.abs(ref) * (1 + 2.0 ** -10)
    if out_type == torch.float16:
        limit += 2.0 ** -25            # below the normal numbers the step is 2^-24
    bad = ~(np.abs(y - ref) <= limit)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3], y[bad][:3], ref[bad][:3])


def rows_of(gen, n, width, t, stride):
    x = torch.full((max(n, 1), stride), float("nan"), device=DEV, dtype=t)
    x[:, :width] = torch.randn(max(n, 1), width, generator=gen, device=DEV).to(t)
    return x


CASES = [
    # tokens, hq, hkv, d, rotary, layout, scaling, norm, type, reach, spare
    (1, 8, 2, 64, 64, 0, 0, False, "bf16", 300, 0),
    (1, 1, 1, 16, 16, 1, 0, True, "fp32", 10, 0),
    (3, 5, 1, 128, 64, 0, 4, True, "bf16", 100000, 8),
    (7, 32, 8, 128, 128, 1, 3, False, "fp16", 1 << 20, 24),
    (129, 40, 5, 128, 112, 0, 2, True, "fp32", 1 << 20, 4),
    (33, 3, 3, 80, 32, 1, 1, True, "bf16", 50, 16),
    (65, 2, 1, 256, 256, 0, 0, True, "fp16", 4096, 0),
    (64, 6, 2, 192, 48, 0, 0, False, "bf16", 9, 40),
    (2, 9, 3, 96, 96, 1, 4, True, "bf16", 70000, 8),
    (2500, 8, 4, 64, 0, 0, 0, True, "bf16", 3, 0),
    (9001, 7, 1, 64, 16, 0, 0, True, "bf16", 9001, 8),
    (5, 4, 0, 64, 64, 0, 0, True, "bf16", 100, 0),
    (5, 0, 4, 64, 64, 0, 0, True, "bf16", 100, 0),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_norm_rope(case):
    n, hq, hkv, d, rot, layout, scaling, norm, type_, reach, spare = case
    t, code = TYPES[type_]
    print(f"[gpu case] norm_rope {case}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(n * 31 + hq)
    rope, freqs, magnitude = rotation(d, rot, layout, scaling)
    q, k = rows_of(gen, n, hq * d, t, hq * d + spare), rows_of(gen, n, hkv * d, t, hkv * d + spare)
    wq = torch.randn(d, generator=gen, device=DEV) if norm else None
    wk = torch.randn(d, generator=gen, device=DEV) if norm else None
    pos = torch.randint(0, reach, (n,), generator=gen, device=DEV, dtype=torch.int32)
    guard = 7.0
    q_out = torch.full((n + 1, hq * d + 16), guard, device=DEV, dtype=t)
    k_out = torch.full((n + 1, hkv * d + 32), guard, device=DEV, dtype=t)
    pa.paged_attn_norm_rope(rope, q if hq else None, q.stride(0), hq, wq, k if hkv else None, k.stride(0), hkv, wk,
                            EPS, code, pos, n, q_out, q_out.stride(0), k_out, k_out.stride(0))
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    for x, out, w, heads in ((q, q_out, wq, hq), (k, k_out, wk, hkv)):
        if heads:
            check(out[:n, :heads * d].reshape(n, heads, d), x[:n, :heads * d].reshape(n, heads, d), w, p, freqs,
                  magnitude, bool(layout), t)
        assert (out[:, heads * d:] == guard).all() and (out[n] == guard).all()


@pytest.mark.parametrize("layout", [0, 1])
def test_norm_rope_in_place_on_packed_rows(layout):
    """q and k of a packed projection, each its own output; v beside them stays."""
    n, hq, hkv, d = 77, 8, 2, 128
    print(f"[gpu case] norm_rope in place {layout}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(5)
    rope, freqs, magnitude = rotation(d, 64, layout)
    x = torch.randn(n, (hq + 2 * hkv) * d, generator=gen, device=DEV).to(torch.bfloat16)
    was = x.clone()
    pos = torch.arange(n, device=DEV, dtype=torch.int32) * 5
    q, k, s = x.data_ptr(), x.data_ptr() + hq * d * 2, x.stride(0)
    pa.paged_attn_norm_rope(rope, q, s, hq, None, k, s, hkv, None, EPS, pa.PA_BF16, pos, n, q, s, k, s)
    torch.cuda.synchronize()
    heads = x.view(n, -1, d)
    check(heads[:, :hq + hkv], was.view(n, -1, d)[:, :hq + hkv], None, pos.cpu().numpy(), freqs, magnitude,
          bool(layout), torch.bfloat16)
    assert torch.equal(heads[:, hq + hkv:], was.view(n, -1, d)[:, hq + hkv:])
    assert torch.equal(heads[..., 64:].view(torch.int16), was.view(n, -1, d)[..., 64:].view(torch.int16))


def test_norm_rope_far_positions_and_large_values():
    """Positions to 2^31 - 1 in the angle, rows whose squares are near the ends of fp32."""
    d = 128
    print("[gpu case] norm_rope far", flush=True)
    rope, freqs, magnitude = rotation(d, d, 0)
    pos = torch.tensor([0, 1, 12345678, 2 ** 30 + 12345, 2 ** 31 - 1, 2 ** 31 - 2], dtype=torch.int32, device=DEV)
    n = pos.numel()
    gen = torch.Generator(device=DEV).manual_seed(9)
    x = torch.randn(n, d, generator=gen, device=DEV)
    x *= torch.tensor([1e-15, 1e15, 1.0, 1.0, 1e-3, 1e17], device=DEV)[:, None]
    out = torch.zeros_like(x)
    w = torch.ones(d, device=DEV)
    pa.paged_attn_norm_rope(rope, x, d, 1, w, None, 0, 0, None, EPS, pa.PA_FP32, pos, n, out, d, None, 0)
    torch.cuda.synchronize()
    # Roundings to 53 bits of products near 2^31: 2^31 2^-53 radians for the frequency in revolutions and as much
    # for its product with the position, half of it for the oracle's product: 10 u more.
    check(out.view(n, 1, d), x.view(n, 1, d), w, pos.cpu().numpy(), freqs, magnitude, False, torch.float32, 34)


# --------------------------------------------------------------------------
# append
# --------------------------------------------------------------------------

APPENDS = [
    # lengths of chunks, resident tokens, hq, hkv, d, rotary, layout, norm, type, pad, positions
    ([1], [0], 8, 2, 64, 64, 0, False, "bf16", 0, False),
    ([1, 1, 1, 1], [3, 15, 16, 300], 8, 2, 64, 32, 1, True, "bf16", 3, False),
    ([17, 0, 1, 33, 64], [5, 7, 0, 31, 16], 32, 8, 128, 128, 0, True, "bf16", 9, False),
    ([100, 3], [0, 1000], 7, 7, 128, 96, 0, True, "fp16", 0, True),
    ([5, 250], [1, 0], 12, 2, 64, 48, 1, False, "fp32", 1, False),
    ([1] * 200 + [2], [4] * 201, 4, 1, 128, 128, 0, True, "bf16", 2, False),
    ([1] * 70 + [0] * 30 + [3] * 4200, [1] * 4300, 2, 1, 64, 64, 0, True, "bf16", 5, False),
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
@pytest.mark.parametrize("single", [False, True])
def test_rope_append(case, single):
    lens, old, hq, hkv, d, rot, layout, norm, type_, pad, given = APPENDS[case]
    if single:                                  # one token per sequence, no q_start
        lens = [1] * len(lens)
    t, code = TYPES[type_]
    print(f"[gpu case] rope_append {case} single={single}", flush=True)
    rng = np.random.default_rng(case)
    gen = torch.Generator(device=DEV).manual_seed(case)
    batch, rows = len(lens), sum(lens)
    total = rows + pad
    ctx = np.array(old) + np.array(lens)
    nb = (ctx + 15) // 16
    blocks = int(nb.sum()) + 3
    ids = rng.permutation(blocks)
    width = max(1, int(nb.max())) + 2
    table = np.full((batch, width), -7, np.int32)
    at = 0
    for b in range(batch):
        table[b, :nb[b]] = ids[at:at + nb[b]]
        at += nb[b]
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    rope, freqs, magnitude = rotation(d, rot, layout, pa.PA_ROPE_YARN if norm else 0)
    x = torch.randn(total, (hq + 2 * hkv) * d, generator=gen, device=DEV).to(t)
    wq = torch.randn(d, generator=gen, device=DEV) if norm else None
    wk = torch.randn(d, generator=gen, device=DEV) if norm else None
    kp = torch.randn(blocks, hkv, 16, d, generator=gen, device=DEV).to(torch.bfloat16)
    vp = torch.randn(blocks, hkv, 16, d, generator=gen, device=DEV).to(torch.bfloat16)
    k_was, v_was = kp.clone(), vp.clone()
    guard = 7.0
    q_out = torch.full((total, hq, d), guard, device=DEV, dtype=torch.bfloat16)
    pos = torch.randint(0, 10000, (total,), generator=gen, device=DEV, dtype=torch.int32) if given else None
    dev = lambda a: torch.tensor(a, device=DEV, dtype=torch.int32)  # noqa: E731
    bt, cl, qs = dev(table), dev(ctx), dev(start)
    pool = pa.kv_pool_create(blocks, 16, hkv, d, kp, vp)
    e, s = x.element_size(), x.stride(0)
    q, k, v = x.data_ptr(), x.data_ptr() + hq * d * e, x.data_ptr() + (hq + hkv) * d * e
    pa.paged_attn_rope_append(pool, rope, q, s, hq, wq, k, s, wk, v, s, EPS, code, pos, None if single else qs, total,
                              bt, width, cl, batch, q_out)
    torch.cuda.synchronize()
    seq = np.repeat(np.arange(batch), lens)
    slot = np.concatenate([np.arange(ctx[b] - lens[b], ctx[b]) for b in range(batch)])
    p = pos.cpu().numpy()[:rows] if given else slot
    heads = x[:rows].view(rows, -1, d)
    check(q_out[:rows], heads[:, :hq], wq, p, freqs, magnitude, bool(layout), torch.bfloat16)
    assert (q_out[rows:] == guard).all()
    block, line = dev(table[seq, slot // 16]).long(), dev(slot % 16).long()
    check(kp[block, :, line], heads[:, hq:hq + hkv], wk, p, freqs, magnitude, bool(layout), torch.bfloat16)
    assert torch.equal(vp[block, :, line], heads[:, hq + hkv:].to(torch.bfloat16))
    kp[block, :, line], vp[block, :, line] = k_was[block, :, line], v_was[block, :, line]
    assert torch.equal(kp, k_was) and torch.equal(vp, v_was)      # nothing else was written


def test_rope_append_keeps_bits_and_matches_append_kv():
    """Without norm and rotation a step's append is paged_attn_append_kv's, NaN payloads and all."""
    print("[gpu case] rope_append raw", flush=True)
    batch, hkv, d, blocks = 5, 4, 64, 20
    gen = torch.Generator(device=DEV).manual_seed(1)
    bits = torch.randint(-32768, 32768, (2, batch, hkv, d), generator=gen, device=DEV, dtype=torch.int16)
    rope = pa.pa_rope_create(d, 0, pa.PA_ROPE_HALF, [])
    table = torch.randperm(blocks, generator=gen, device=DEV)[:batch * 3].view(batch, 3).int().contiguous()
    ctx = torch.tensor([1, 16, 17, 0, 48], device=DEV, dtype=torch.int32)
    got = []
    for ours in (False, True):
        kp, vp = (torch.zeros(blocks, hkv, 16, d, device=DEV, dtype=torch.int16) for _ in range(2))
        pool = pa.kv_pool_create(blocks, 16, hkv, d, kp, vp)
        if ours:
            pa.paged_attn_rope_append(pool, rope, None, 0, 0, None, bits[0], hkv * d, None, bits[1], hkv * d, EPS,
                                      pa.PA_BF16, None, None, batch, table, 3, ctx, batch, None)
        else:
            pa.paged_attn_append_kv(pool, bits[0], bits[1], table, 3, ctx, batch)
        torch.cuda.synchronize()
        got.append((kp, vp))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_rope_append_bad_device_data_stays_inside():
    """Lengths, tables and starts that lie: nothing outside the pool or q_out is written."""
    print("[gpu case] rope_append bad device data", flush=True)
    batch, hq, hkv, d, blocks, total = 4, 4, 2, 64, 6, 40
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(total, (hq + 2 * hkv) * d, generator=gen, device=DEV).to(torch.bfloat16)
    rope, _, _ = rotation(d, d, 0)
    guard = torch.full((2, blocks + 2, hkv, 16, d), 3.0, device=DEV, dtype=torch.bfloat16)
    pool = pa.kv_pool_create(blocks, 16, hkv, d, guard[0, 1:], guard[1, 1:])
    s, e = x.stride(0), 2
    q, k, v = x.data_ptr(), x.data_ptr() + hq * d * e, x.data_ptr() + (hq + hkv) * d * e
    big = 2 ** 31 - 1
    for start in ([0, 10, 20, 30, 40], [0, -5, 50, big, 40], [-big - 1, -3, -2, -1, big], [7, 3, 9, 1, 2]):
        for ctx in ([10, 10, 10, 10], [big, -big - 1, 5, 0], [1000, 3, 48, 49]):
            for ids in (-5, big, 3):
                q_out = torch.full((total + 2, hq, d), 3.0, device=DEV, dtype=torch.bfloat16)
                dev = lambda a: torch.tensor(a, device=DEV, dtype=torch.int32)  # noqa: E731
                keep = dev(start), dev(ctx), torch.full((batch, 3), ids, device=DEV, dtype=torch.int32)
                pa.paged_attn_rope_append(pool, rope, q, s, hq, None, k, s, None, v, s, EPS, pa.PA_BF16, None, keep[0],
                                          total, keep[2], 3, keep[1], batch, q_out[1:])
                torch.cuda.synchronize()
                assert (q_out[0] == 3.0).all() and (q_out[-1] == 3.0).all()
                assert (guard[:, 0] == 3.0).all() and (guard[:, -1] == 3.0).all()
