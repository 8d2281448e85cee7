"""Decode and extend attention with capped, biased or masked scores, against
the float64 oracle over the same bf16 inputs.

Tolerance of one output row.  u = 2^-24.  A raw score is off by at most D u of
sum |q k| (fp32 accumulation; bf16 products are exact), its cap by 6e-7 of it
(the polynomial) or 3 u of the cap (the exponential form, two roundings and the
reciprocal), the distance bias by 2 u of it: with |scores| S in natural units
the weight 2^e is off by a factor of at most 1 +- w,
    w = 2^-17 + S 10^-6 + 2^-20
(2^-17: the bf16 pair; 2^-20: the exponential and fp32 sums).  An output is a
weighted mean, so its error is at most 2 w max |V|, and then half a step of
bf16, 2^-8 of the value.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle.attention import bf16_to_f64  # noqa: E402
from oracle.ops import biased_attention  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN, INF, NINF = 0x7FC0, 0x7F80, 0xFF80


def bits(rng, shape, scale=1.0):
    x = (rng.standard_normal(shape) * scale).astype(np.float32).view(np.uint32)
    return ((x + 0x7FFF + ((x >> 16) & 1)) >> 16).astype(np.uint16)


def dev16(a):
    return torch.from_numpy(a.view(np.int16).copy()).to(DEV)


def dev32(a):
    return None if a is None else torch.from_numpy(np.asarray(a, np.int32).copy()).to(DEV)


class Case:
    """Inputs of a call; every slot that no row may read holds NaN."""

    def __init__(self, seed, ctx, chunk, hq, hkv, d, cap=0.0, alibi=False, window=0, docs=None, prefix=None, pad=0,
                 qscale=1.0, scale=None, poison=True):
        rng = np.random.default_rng(seed)
        self.ctx, self.chunk = np.array(ctx), np.array(chunk)
        self.hq, self.hkv, self.d, self.cap, self.window = hq, hkv, d, cap, window
        self.scale = d ** -0.5 if scale is None else scale
        self.batch = len(ctx)
        nb = (self.ctx + 15) // 16
        self.blocks = int(nb.sum()) + 2
        ids = rng.permutation(self.blocks)
        self.width = max(1, int(nb.max(initial=0))) + 1
        self.table = np.full((self.batch, self.width), -9, np.int32)
        self.k = np.full((self.blocks, hkv, 16, d), NAN, np.uint16)
        self.v = np.full((self.blocks, hkv, 16, d), NAN if poison else 0, np.uint16)
        at = 0
        for b in range(self.batch):
            self.table[b, :nb[b]] = ids[at:at + nb[b]]
            at += nb[b]
            for j in range(nb[b]):
                m = min(16, self.ctx[b] - 16 * j)
                self.k[self.table[b, j], :, :m] = bits(rng, (hkv, m, d))
                self.v[self.table[b, j], :, :m] = bits(rng, (hkv, m, d))
        self.start = np.concatenate([[0], np.cumsum(self.chunk)])
        self.rows = int(self.start[-1])
        self.total = self.rows + pad
        self.q = bits(rng, (self.total, hq, d), qscale)
        self.slopes = 2.0 ** (-8.0 * (np.arange(hq) + 1) / hq) if alibi else None
        self.first = docs(self, rng) if docs else None
        self.prefix = None if prefix is None else np.array(prefix)

    def reference(self):
        return biased_attention(bf16_to_f64(self.q[:self.rows]), self.start, self.k, self.v, self.table, self.ctx,
                                np.float64(np.float32(self.scale)), self.cap, self.slopes, self.window, self.first,
                                self.prefix)

    def run(self, decode=False, stream=None, spare=0, out=None, workspace=None):
        t = self.t = dict(k=dev16(self.k), v=dev16(self.v), q=dev16(self.q), table=dev32(self.table),
                          ctx=dev32(self.ctx), start=dev32(self.start), first=dev32(self.first),
                          prefix=dev32(self.prefix),
                          slopes=None if self.slopes is None else torch.tensor(self.slopes, dtype=torch.float32,
                                                                               device=DEV))
        pool = self.pool = pa.kv_pool_create(self.blocks, 16, self.hkv, self.d, t["k"], t["v"])
        top = int(self.ctx.max(initial=0)) + spare
        most = 1 if decode else int(self.chunk.max(initial=0)) + min(spare, 3)
        size = pa.paged_attn_biased_workspace_size(pool, self.batch, self.hq, top, most, self.window)
        ws = torch.full((max(size, 16),), 255, dtype=torch.uint8, device=DEV) if workspace is None else workspace
        out = torch.full((self.total, self.hq, self.d), 0x4242, dtype=torch.int16, device=DEV) if out is None else out
        if decode:
            def call(stream=stream):
                pa.paged_attn_decode_biased(pool, t["q"], t["table"], self.width, t["ctx"], self.batch, self.hq,
                                            self.scale, self.cap, t["slopes"], self.window, t["first"], top, ws, size,
                                            out, stream)
        else:
            def call(stream=stream):
                pa.paged_attn_extend_biased(pool, t["q"], t["start"], self.total, t["table"], self.width, t["ctx"],
                                            self.batch, self.hq, self.scale, self.cap, t["slopes"], self.window,
                                            t["first"], t["prefix"], top, most, ws, size, out, stream)
        self.call, self.out, self.ws, self.size = call, out, ws, size
        call()
        torch.cuda.synchronize()
        return out.cpu().numpy().view(np.uint16)

    def check(self, got, ref=None, score=None):
        assert (got[self.rows:] == 0x4242).all()       # rows behind the last sequence
        ref = self.reference() if ref is None else ref
        x = bf16_to_f64(got[:self.rows])
        fin = np.isfinite(ref)
        # an infinity may come out as NaN: the weight's low part may be 0 or negative
        assert (np.isfinite(x) == fin).all(), "infinities and NaN are where they should be"
        s = 40.0 if score is None else score           # largest |score|: |q| |k| scale, N(0, 1) rows
        vmax = np.abs(bf16_to_f64(self.v)[np.isfinite(bf16_to_f64(self.v))]).max(initial=0.0)
        limit = 2 * (2.0 ** -17 + s * 1e-6 + 2.0 ** -20) * vmax + 2.0 ** -8 * np.abs(ref)
        with np.errstate(invalid="ignore"):
            bad = fin & ~(np.abs(x - ref) <= limit)
        assert not bad.any(), (int(bad.sum()), bad.size, np.argwhere(bad)[:4], x[bad][:4], ref[bad][:4])
        empty = (ref == 0).all(-1)
        assert (x[empty] == 0).all()


def documents(lo, hi):
    def build(c, rng):
        first = np.zeros(c.rows, np.int64)
        for b in range(c.batch):
            begins = np.concatenate([[0], np.cumsum(rng.integers(lo, hi + 1, size=c.ctx[b] // lo + 2))])
            p = np.arange(c.ctx[b] - c.chunk[b], c.ctx[b])
            first[c.start[b]:c.start[b + 1]] = begins[np.searchsorted(begins, p, side="right") - 1]
        return first
    return build


DECODES = {
    "one_token": dict(ctx=[1], hq=8, hkv=2, d=64, cap=30.0),
    "plain": dict(ctx=[1, 15, 16, 17, 100, 0, 333], hq=8, hkv=2, d=64),
    "cap": dict(ctx=[31, 32, 33, 1000, 0, 4097], hq=32, hkv=8, d=128, cap=30.0, qscale=4.0),
    "cap_far": dict(ctx=[700, 65], hq=4, hkv=4, d=128, cap=3.0, qscale=6.0),
    "alibi": dict(ctx=[300, 5, 2111], hq=12, hkv=12, d=64, alibi=True),
    "alibi_cap": dict(ctx=[129, 2048], hq=14, hkv=2, d=128, alibi=True, cap=20.0, qscale=4.0),
    "window": dict(ctx=[1, 99, 100, 101, 2000, 0, 640], hq=16, hkv=8, d=128, window=100, cap=50.0),
    "window_one": dict(ctx=[50, 16, 1], hq=8, hkv=1, d=64, window=1),
    "documents": dict(ctx=[700, 33, 1], hq=28, hkv=4, d=128, docs=documents(3, 200)),
    "many_heads": dict(ctx=[77, 600], hq=71, hkv=1, d=64, alibi=True),
    "long": dict(ctx=[9001, 20000], hq=16, hkv=2, d=128, cap=50.0, qscale=4.0),
    "odd_group": dict(ctx=[45, 3, 260], hq=15, hkv=5, d=64, cap=15.0, window=64),
    "negative_scale": dict(ctx=[200, 17], hq=8, hkv=2, d=128, scale=-0.1, cap=9.0, qscale=3.0),
    "zero_scale": dict(ctx=[200, 17], hq=8, hkv=2, d=128, scale=0.0, cap=9.0),
    "zero_scale_plain": dict(ctx=[200, 17], hq=8, hkv=2, d=128, scale=0.0),
}


@pytest.mark.parametrize("spare", [0, 5000])
@pytest.mark.parametrize("name", sorted(DECODES))
def test_decode(name, spare):
    print(f"[gpu case] decode_biased {name} {spare}", flush=True)
    kw = dict(DECODES[name])
    c = Case(len(name), chunk=[1] * len(kw["ctx"]), **kw)
    if 0 in kw["ctx"]:                       # rows of empty sequences: no chunk in the oracle, zeros here
        keep = [i for i, n in enumerate(kw["ctx"]) if n]
        got = _wide(c, spare)
        assert (got[[i for i, n in enumerate(kw["ctx"]) if not n]] == 0).all()
        full = c.chunk
        c.chunk = np.array([1 if n else 0 for n in kw["ctx"]])
        c.start = np.concatenate([[0], np.cumsum(c.chunk)])
        q, first = c.q, c.first
        c.q, c.rows = q[keep], len(keep)
        c.first = None if first is None else first[keep]
        ref = c.reference()
        c.total = c.rows
        c.check(got[keep], ref, 40.0 * kw.get("qscale", 1.0))
        c.chunk = full
    else:
        c.check(_wide(c, spare), None, 40.0 * kw.get("qscale", 1.0))


def _wide(c, spare):
    """A decode whose host bound of the lengths is `spare` above the longest."""
    if spare:
        c.table = np.concatenate([c.table, np.full((c.batch, spare // 16 + 2), -9, np.int32)], axis=1)
        c.width = c.table.shape[1]
    return c.run(decode=True, spare=spare)


EXTENDS = {
    "one": dict(ctx=[1], chunk=[1], hq=8, hkv=2, d=64, cap=30.0),
    "plain": dict(ctx=[40, 16, 100, 333], chunk=[40, 1, 17, 130], hq=8, hkv=2, d=128, pad=3),
    "cap": dict(ctx=[700, 33, 256], chunk=[300, 33, 7], hq=16, hkv=4, d=128, cap=30.0, qscale=4.0),
    "cap_64": dict(ctx=[500, 64], chunk=[129, 64], hq=12, hkv=2, d=64, cap=5.0, qscale=4.0, pad=1),
    "alibi": dict(ctx=[600, 90], chunk=[600, 31], hq=6, hkv=6, d=128, alibi=True),
    "alibi_cap_64": dict(ctx=[257], chunk=[257], hq=14, hkv=2, d=64, alibi=True, cap=25.0, qscale=3.0),
    "window": dict(ctx=[900, 50, 131], chunk=[400, 50, 131], hq=8, hkv=2, d=128, window=70, cap=50.0),
    "window_one": dict(ctx=[100], chunk=[100], hq=4, hkv=2, d=128, window=1),
    "documents": dict(ctx=[800, 200], chunk=[700, 200], hq=8, hkv=2, d=128, docs=documents(1, 90)),
    "documents_window_64": dict(ctx=[300], chunk=[300], hq=10, hkv=2, d=64, docs=documents(5, 150), window=40),
    "prefix": dict(ctx=[300, 64, 20, 90], chunk=[300, 64, 20, 10], hq=8, hkv=2, d=128, prefix=[120, 64, 500, 7]),
    "prefix_alibi_window": dict(ctx=[400, 33], chunk=[400, 33], hq=4, hkv=1, d=64, prefix=[200, 32], alibi=True,
                                window=100),
    "empty_chunks": dict(ctx=[30, 0, 50, 0], chunk=[0, 0, 20, 0], hq=8, hkv=2, d=128, cap=30.0, pad=2),
    "many": dict(ctx=[20 + i for i in range(60)], chunk=[1 + i % 19 for i in range(60)], hq=8, hkv=2, d=128, cap=30.0),
    "big_group": dict(ctx=[120], chunk=[50], hq=48, hkv=1, d=128, cap=30.0),
    "long_tail": dict(ctx=[9000], chunk=[5], hq=8, hkv=2, d=128, cap=50.0),
    "beyond_8192": dict(ctx=[8700], chunk=[140], hq=4, hkv=1, d=128, window=8300),
    "many_tiles": dict(ctx=[500] * 12, chunk=[260] * 12, hq=32, hkv=8, d=128, cap=30.0, qscale=4.0),
    "many_tiles_64": dict(ctx=[420] * 12, chunk=[200] * 12, hq=32, hkv=8, d=64, alibi=True, docs=documents(20, 300)),
    "many_tiles_rising": dict(ctx=[600] * 12, chunk=[260] * 12, hq=32, hkv=8, d=128, cap=50.0, qscale=8.0),
    "paired_tiles": dict(ctx=[900, 700, 0, 1300, 40], chunk=[500, 330, 0, 650, 3], hq=32, hkv=8, d=128, cap=30.0, qscale=4.0),
    "paired_tiles_64": dict(ctx=[2500, 200, 2400], chunk=[900, 90, 880], hq=30, hkv=6, d=64, alibi=True, pad=9),
    "paired_tiles_window": dict(ctx=[800] * 7, chunk=[500, 450, 1, 480, 380, 422, 199], hq=16, hkv=16, d=128, window=333),
    "one_long_of_four": dict(ctx=[900, 5, 700, 2], chunk=[600, 1, 3, 0], hq=32, hkv=8, d=128, cap=50.0, qscale=8.0, pad=2),
    "negative_scale": dict(ctx=[150], chunk=[150], hq=8, hkv=2, d=128, scale=-0.1),
    "zero_scale": dict(ctx=[150], chunk=[150], hq=8, hkv=2, d=128, scale=0.0, window=33),
}


@pytest.mark.parametrize("spare", [0, 700])
@pytest.mark.parametrize("name", sorted(EXTENDS))
def test_extend(name, spare):
    print(f"[gpu case] extend_biased {name} {spare}", flush=True)
    kw = dict(EXTENDS[name])
    c = Case(len(name) + 100, **kw)
    if spare:
        c.table = np.concatenate([c.table, np.full((c.batch, spare // 16 + 2), -9, np.int32)], axis=1)
        c.width = c.table.shape[1]
    c.check(c.run(spare=spare), None, 40.0 * kw.get("qscale", 1.0))


def test_rows_that_see_nothing():
    """First tokens past the row: zeros, beside rows that do see tokens."""
    print("[gpu case] empty rows", flush=True)

    def docs(c, rng):
        p = np.concatenate([np.arange(n - m, n) for n, m in zip(c.ctx, c.chunk)])
        return np.where(rng.random(c.rows) < 0.4, p + rng.integers(1, 50, c.rows), np.maximum(p - 20, -3))
    for hkv, chunk in ((2, [90, 33]), (8, [1, 1])):
        c = Case(4, ctx=[300, 33], chunk=chunk, hq=16, hkv=hkv, d=128, docs=docs, cap=20.0)
        c.check(c.run(decode=chunk == [1, 1]))
    c = Case(5, ctx=[64], chunk=[64], hq=4, hkv=2, d=64, docs=lambda c, rng: np.full(c.rows, 2 ** 31 - 1))
    assert (c.run() == 0).all()


@pytest.mark.parametrize("alibi", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("decode", [True, False])
def test_infinities_and_nan_in_hidden_places(d, decode, alibi):
    """K and V of tokens that some or all rows do not see hold infinities and NaN; rows that see one show it."""
    print(f"[gpu case] special values {d} {decode} {alibi}", flush=True)
    rng = np.random.default_rng(8)
    chunk = [1, 1, 1] if decode else [70, 200, 33]
    c = Case(6, ctx=[150, 400, 33], chunk=chunk, hq=8, hkv=2, d=d, window=60, cap=0.0 if d == 64 else 30.0, alibi=alibi)
    for b, n in enumerate(c.ctx):
        hidden = n - chunk[b] - 60 + 1                    # below it nobody looks
        for t in range(max(0, hidden)):
            block, line = c.table[b, t // 16], t % 16
            c.k[block, :, line] = rng.choice([NAN, INF, NINF], size=(2, d))
            c.v[block, :, line] = rng.choice([NAN, INF, NINF], size=(2, d))
    if not decode:                                        # tokens that later rows see, earlier ones do not
        for b, t, what in ((0, 120, INF), (1, 300, NAN), (1, 333, NINF), (2, 32, NAN)):
            c.v[c.table[b, t // 16], b % 2, t % 16, 3::7] = what
        c.k[c.table[0, 140 // 16], 0, 140 % 16, 5] = NAN
    got = c.run(decode=decode)
    with np.errstate(all="ignore"):
        ref = c.reference()
    c.check(got, ref)
    assert decode or (np.isfinite(ref).any() and np.isnan(ref).any() and np.isinf(ref).any())


def test_lowest_values_in_visible_places():
    """Keys of the type's lowest value (scores of -3e38 and below) weigh nothing beside ordinary ones."""
    print("[gpu case] lowest values", flush=True)
    c = Case(7, ctx=[100, 40], chunk=[100, 40], hq=4, hkv=2, d=128)
    c.q[:] = np.uint16(0x3F80)                            # ones: the score is the sum of the key's values
    for b, t in ((0, 0), (0, 50), (0, 51), (1, 39), (1, 17)):
        c.k[c.table[b, t // 16], :, t % 16] = 0xFF7F if t else 0xFF80
    got = c.run()
    with np.errstate(all="ignore"):
        ref = c.reference()
    fin = np.isfinite(ref).all(-1)
    assert fin.sum() > 500
    x = bf16_to_f64(got[:c.rows])
    assert np.isnan(x[~fin]).all() or (x[~fin] == 0).all()      # a row that sees -inf alone has no softmax
    ref[~fin] = x[~fin]
    c.check(got, ref, 60.0)


@pytest.mark.parametrize("alibi", [False, True])
@pytest.mark.parametrize("hq,chunks", [(8, [12] * 40), (64, [3, 5, 2])])     # 128 rows per workgroup, 32 over several stages
def test_special_values_in_both_forms(hq, chunks, alibi):
    """Infinities and NaN that some rows of a tile see and others do not, in every stage of long contexts."""
    print(f"[gpu case] special values in both forms {hq} {alibi}", flush=True)
    ctx = [700 + 17 * i for i in range(len(chunks))] if hq == 64 else [n + 40 for n in chunks]
    c = Case(15, ctx=ctx, chunk=chunks, hq=hq, hkv=8, d=128, alibi=alibi,
             docs=lambda c, rng: np.concatenate([rng.integers(0, n - m, m) for n, m in zip(c.ctx, c.chunk)]))
    rng = np.random.default_rng(3)
    for b, n in enumerate(c.ctx):
        for t in rng.integers(0, n, 2):
            c.v[c.table[b, t // 16], rng.integers(0, 8), t % 16, rng.integers(0, 128)] = rng.choice([NAN, INF, NINF])
    got = c.run()
    with np.errstate(all="ignore"):
        ref = c.reference()
    assert 0 < (~np.isfinite(ref)).sum() < ref.size // 2
    c.check(got, ref)


@pytest.mark.parametrize("decode", [True, False])
def test_bad_device_data_stays_inside(decode):
    """Lengths, starts, tables, documents and prefixes that lie: nothing outside out is written."""
    print(f"[gpu case] bad device data {decode}", flush=True)
    big = 2 ** 31 - 1
    batch, hq, hkv, d, total, blocks = 4, 8, 2, 64, 40, 6
    gen = torch.Generator(device=DEV).manual_seed(3)
    k, v = (torch.randn(blocks, hkv, 16, d, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(total, hq, d, generator=gen, device=DEV).to(torch.bfloat16)
    pool = pa.kv_pool_create(blocks, 16, hkv, d, k, v)
    width, top = 5, 70
    for start in ([0, 10, 20, 30, 40], [0, -5, 50, big, 40], [-big - 1, -3, -2, -1, big], [7, 3, 9, 1, 2]):
        for ctx in ([10, 70, 33, 10], [big, -big - 1, 5, 0]):
            for ids, lie in ((-5, -big - 1), (big, big), (3, 20)):
                out = torch.full((total + 2, hq, d), 3.0, device=DEV, dtype=torch.bfloat16)
                table, ctxd, qs = dev32(np.full((batch, width), ids)), dev32(ctx), dev32(start)
                first, prefix = dev32(np.full(total, lie)), dev32(np.full(batch, lie))
                size = pa.paged_attn_biased_workspace_size(pool, batch, hq, top, 1 if decode else 20, 0)
                ws = torch.full((size + 32,), 7, dtype=torch.uint8, device=DEV)
                if decode:
                    pa.paged_attn_decode_biased(pool, q, table, width, ctxd, batch, hq, 0.1, 30.0, None, 0, first, top,
                                                ws, size, out[1:])
                else:
                    pa.paged_attn_extend_biased(pool, q, qs, total, table, width, ctxd, batch, hq, 0.1, 30.0, None, 0,
                                                first, prefix, top, 20, ws, size, out[1:])
                torch.cuda.synchronize()
                assert (out[0] == 3.0).all() and (out[-1] == 3.0).all() and (ws[size:] == 7).all()


@pytest.mark.parametrize("hq", [8, 32])                  # both decode forms
def test_decode_of_empty_sequences_alone(hq):
    """No sequence holds a token, and the table has no columns: zeros."""
    print(f"[gpu case] empty decode {hq}", flush=True)
    k = torch.full((2, 2, 16, 64), float("nan"), device=DEV, dtype=torch.bfloat16)
    pool = pa.kv_pool_create(2, 16, 2, 64, k, k)
    q = torch.ones(3, hq, 64, device=DEV, dtype=torch.bfloat16)
    ctx, table = dev32([0, 5, -1]), torch.zeros(4, dtype=torch.int32, device=DEV)
    out = torch.full((3, hq, 64), 7.0, device=DEV, dtype=torch.bfloat16)
    pa.paged_attn_decode_biased(pool, q, table, 0, ctx, 3, hq, 0.1, 0.0, None, 0, None, 0, None, 0, out)
    torch.cuda.synchronize()
    assert (out == 0).all()


def test_side_stream_and_two_calls_at_once():
    """Two calls on two streams, each with its workspace, give what each gives alone."""
    print("[gpu case] streams", flush=True)
    cases = [Case(11, ctx=[3000, 900], chunk=[1, 1], hq=32, hkv=8, d=128, cap=30.0, qscale=4.0),
             Case(12, ctx=[2500], chunk=[9], hq=8, hkv=2, d=128, alibi=True)]
    alone = [c.run(decode=i == 0).copy() for i, c in enumerate(cases)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in cases:
        c.out.fill_(0x4242)
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(cases, streams):
            c.call(s.cuda_stream)
    torch.cuda.synchronize()
    for c, want in zip(cases, alone):
        assert (c.out.cpu().numpy().view(np.uint16) == want).all()


@pytest.mark.parametrize("window", [500, 1200])          # one partition, several
def test_captured_and_replayed(window):
    """A step of norm, rotation, append and attention captured into a graph, replayed over changing inputs."""
    print(f"[gpu case] graph {window}", flush=True)
    hq, hkv, d, batch, steps = 16, 4, 128, 3, 6
    gen = torch.Generator(device=DEV).manual_seed(13)
    ctx = np.array([70, 1500, 31])
    blocks, width = 130, 110
    table = torch.randperm(blocks, generator=gen, device=DEV)[:120].view(-1).int()
    rows = torch.zeros(batch, width, dtype=torch.int32, device=DEV)
    rows[0, :8], rows[1, :100], rows[2, :8] = table[:8], table[8:108], table[108:116]
    freqs, magnitude = pa.pa_rope_frequencies(d, 10000.0)
    rope = pa.pa_rope_create(d, d, pa.PA_ROPE_HALF, freqs, magnitude)

    def fresh():
        g = torch.Generator(device=DEV).manual_seed(14)
        st = dict(k=torch.randn(blocks, hkv, 16, d, generator=g, device=DEV).to(torch.bfloat16),
                  v=torch.randn(blocks, hkv, 16, d, generator=g, device=DEV).to(torch.bfloat16),
                  x=torch.zeros(batch, (hq + 2 * hkv) * d, device=DEV, dtype=torch.bfloat16),
                  q=torch.zeros(batch, hq, d, device=DEV, dtype=torch.bfloat16),
                  out=torch.zeros(batch, hq, d, device=DEV, dtype=torch.bfloat16),
                  ctx=torch.tensor(ctx, dtype=torch.int32, device=DEV))
        st["pool"] = pa.kv_pool_create(blocks, 16, hkv, d, st["k"], st["v"])
        size = pa.paged_attn_biased_workspace_size(st["pool"], batch, hq, 16 * width, 1, window)
        assert (size > 0) == (window == 1200)
        st["ws"] = torch.zeros(max(size, 16), dtype=torch.uint8, device=DEV)

        def step(stream):
            x, s = st["x"].data_ptr(), st["x"].stride(0)
            pa.paged_attn_rope_append(st["pool"], rope, x, s, hq, None, x + 2 * hq * d, s, None,
                                      x + 2 * (hq + hkv) * d, s, 1e-6, pa.PA_BF16, None, None, batch, rows, width,
                                      st["ctx"], batch, st["q"], stream)
            pa.paged_attn_decode_biased(st["pool"], st["q"], rows, width, st["ctx"], batch, hq, d ** -0.5, 30.0, None,
                                        window, None, 16 * width, st["ws"], size, st["out"], stream)
        st["step"] = step
        return st

    xs = [torch.randn(batch, (hq + 2 * hkv) * d, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(steps)]
    eager = fresh()
    want = []
    for x in xs:
        eager["x"].copy_(x)
        eager["ctx"] += 1
        eager["step"](None)
        want.append(eager["out"].clone())
    torch.cuda.synchronize()
    st = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st["step"](torch.cuda.current_stream().cuda_stream)
    for i, x in enumerate(xs):
        st["x"].copy_(x)
        st["ctx"] += 1
        graph.replay()
        torch.cuda.synchronize()
        eager["step"](None)                              # the program's own work between replays
        torch.cuda.synchronize()
        assert torch.equal(st["out"], want[i])
    assert torch.equal(st["k"], eager["k"]) and torch.equal(st["v"], eager["v"])


def test_repeatable_and_independent_of_placement():
    print("[gpu case] bits", flush=True)
    c = Case(21, ctx=[2000, 333], chunk=[1, 1], hq=8, hkv=2, d=128, cap=30.0, alibi=True)
    a = c.run(decode=True)
    perm = np.random.default_rng(0).permutation(c.blocks)
    k, v, t = np.empty_like(c.k), np.empty_like(c.v), c.table.copy()
    k[perm], v[perm] = c.k, c.v
    t[c.table >= 0] = perm[c.table[c.table >= 0]]
    c.k, c.v, c.table = k, v, t
    assert (c.run(decode=True) == a).all()


def test_serving_steps_prompt_then_tokens():
    """A run of the operators together: a prompt appended and attended as a chunk, then tokens one by one, equal the
    whole sequence as one chunk."""
    print("[gpu case] prompt then tokens", flush=True)
    hq, hkv, d, n, prompt = 8, 2, 128, 150, 120
    gen = torch.Generator(device=DEV).manual_seed(31)
    x = torch.randn(n, (hq + 2 * hkv) * d, generator=gen, device=DEV).to(torch.bfloat16)
    w = torch.rand(d, generator=gen, device=DEV) + 0.5
    freqs, magnitude = pa.pa_rope_frequencies(d, 10000.0, pa.PA_ROPE_BANDS, 8.0, 64.0, 1.0, 4.0)
    rope = pa.pa_rope_create(d, d, pa.PA_ROPE_INTERLEAVED, freqs, magnitude)
    table = torch.randperm(12, generator=gen, device=DEV)[:10].int().view(1, 10).contiguous()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731

    def pass_over(pieces):
        k, v = (torch.zeros(12, hkv, 16, d, device=DEV, dtype=torch.bfloat16) for _ in range(2))
        pool = pa.kv_pool_create(12, 16, hkv, d, k, v)
        outs, at = [], 0
        for m in pieces:
            rows = x[at:at + m]
            at += m
            base, s = rows.data_ptr(), rows.stride(0)
            q, out = (torch.zeros(m, hq, d, device=DEV, dtype=torch.bfloat16) for _ in range(2))
            start, ctx = i32(0, m), i32(at)
            pa.paged_attn_rope_append(pool, rope, base, s, hq, w, base + 2 * hq * d, s, w, base + 2 * (hq + hkv) * d,
                                      s, 1e-6, pa.PA_BF16, None, None if m == 1 else start, m, table, 10, ctx, 1, q)
            size = pa.paged_attn_biased_workspace_size(pool, 1, hq, 160, m, 0)
            ws = torch.zeros(max(size, 16), dtype=torch.uint8, device=DEV)
            if m == 1:
                pa.paged_attn_decode_biased(pool, q, table, 10, ctx, 1, hq, d ** -0.5, 30.0, None, 0, None, 160, ws,
                                            size, out)
            else:
                pa.paged_attn_extend_biased(pool, q, start, m, table, 10, ctx, 1, hq, d ** -0.5, 30.0, None, 0, None,
                                            None, 160, m, ws, size, out)
            outs.append(out)
        torch.cuda.synchronize()
        return torch.cat(outs).double(), k, v

    a, ka, va = pass_over([n])
    b, kb, vb = pass_over([prompt] + [1] * (n - prompt))
    assert torch.equal(ka, kb) and torch.equal(va, vb)
    # each within half a bf16 step of the same value, and the weights' 2^-17
    assert ((a - b).abs() <= 2.0 ** -7 * a.abs() + 2 * (2.0 ** -16) * va.double().abs().max()).all()
