"""The tokens that stay and their move, exactly as the oracle has them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tokens as oracle  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import DEV, dev16, dev32  # noqa: E402

pytestmark = pytest.mark.gpu


def choose(totals, ctx, first, recent, keep, spare=0):
    """(kept, kept_lens) of rows of totals [batch][width]."""
    batch, width = totals.shape
    top = max(ctx) if len(ctx) else 0
    stride = min(max(keep, recent), top) + spare
    kept = torch.full((batch, max(stride, 1)), 55, dtype=torch.int32, device=DEV)
    lens = torch.full((batch,), 55, dtype=torch.int32, device=DEV)
    pa.paged_attn_keep_heaviest(torch.tensor(totals, device=DEV), width, None if first is None else dev32(first), dev32(ctx),
                                batch, top, recent, keep, kept, stride, lens)
    torch.cuda.synchronize()
    return kept.cpu().numpy()[:, :stride], lens.cpu().numpy()


def values(kind, rng, shape):
    if kind == "equal":
        return np.full(shape, 0.25, np.float32)
    if kind == "few":
        return rng.integers(0, 3, shape).astype(np.float32)
    if kind == "signed":
        x = rng.standard_normal(shape).astype(np.float32)
        x[rng.random(shape) < 0.1] = -0.0
        x[rng.random(shape) < 0.1] = 0.0
        return x
    if kind == "special":
        x = rng.standard_normal(shape).astype(np.float32)
        at = rng.random(shape)
        x[at < 0.1], x[(at > 0.1) & (at < 0.2)], x[at > 0.9] = np.nan, np.inf, -np.inf
        return x
    if kind == "close":       # neighbouring floats: only the last bits differ
        return (np.uint32(0x3F800000) + rng.integers(0, 500, shape).astype(np.uint32)).view(np.float32)
    return (rng.random(shape) ** 8).astype(np.float32)


@pytest.mark.parametrize("kind", ["heavy", "equal", "few", "signed", "special", "close"])
@pytest.mark.parametrize("keep,recent", [(0, 0), (1, 0), (40, 8), (64, 64), (10, 100), (1000, 17), (1023, 0), (5000, 1)])
def test_choice(kind, keep, recent):
    print(f"[gpu case] keep {kind} {keep} {recent}", flush=True)
    rng = np.random.default_rng(keep + recent)
    ctx = [0, 1, 2, 63, 64, 65, 1000, 1023, 1024, 1025, 1300, 4097, 41]
    totals = values(kind, rng, (len(ctx), max(ctx) + 5))
    for first in (None, [0, 5, 1, 10, 64, 0, 999, 512, 1, 1025, 7, 100, -3]):
        kept, lens = choose(totals, ctx, first, recent, keep, spare=3)
        for b, n in enumerate(ctx):
            want = oracle.keep_heaviest(totals[b, :n], 0 if first is None else first[b], recent, keep)
            assert lens[b] == len(want) and kept[b, :len(want)].tolist() == want and (kept[b, len(want):] == -1).all()


@pytest.mark.parametrize("equal", [1, 2, 63, 64, 65, 300])
@pytest.mark.parametrize("n", [1025, 1100, 2048, 2049, 9000, 32768, 32769])
def test_equal_totals_on_the_threshold(n, equal):
    """Groups of equal totals that the cut goes through, as many as a wavefront's lanes and more, among others close by."""
    print(f"[gpu case] keep on the threshold {n} {equal}", flush=True)
    rng = np.random.default_rng(n + equal)
    above = 400
    totals = np.zeros((4, n), np.float32)
    cuts = [1, equal // 2, equal, equal + 1]
    for b in range(4):
        x = (np.uint32(0x3F000000) - rng.integers(1, 1 << 20, n).astype(np.uint32)).view(np.float32)    # below 0.5
        at = rng.permutation(n)
        x[at[:above]] = 0.5 + rng.random(above, np.float32) + np.float32(0.001)
        x[at[above:above + equal]] = 0.5
        if b == 1:
            x[at[-1]] = -1e30                              # the first bit that differs is the sign
        totals[b] = x
    for cut in cuts:
        kept, lens = choose(totals, [n] * 4, None, 0, above + cut)
        for b in range(4):
            assert kept[b, :lens[b]].tolist() == oracle.keep_heaviest(totals[b], 0, 0, above + cut)


def test_choice_of_long_sequences():
    print("[gpu case] keep long", flush=True)
    rng = np.random.default_rng(3)
    ctx = [100001, 33000]
    totals = values("heavy", rng, (2, max(ctx)))
    totals[1] = np.round(totals[1], 2)                # many equal ones
    kept, lens = choose(totals, ctx, [16, 0], 300, 20001)
    for b, n in enumerate(ctx):
        assert kept[b, :lens[b]].tolist() == oracle.keep_heaviest(totals[b, :n], [16, 0][b], 300, 20001)


class Move:
    """A pool, tables, and for each sequence the first tokens and an ascending list of those that stay."""

    def __init__(self, seed, ctx, hkv, d, share=0.5, first=None, fresh=False, own_first_block=False):
        rng = np.random.default_rng(seed)
        self.ctx, self.hkv, self.d, self.batch = ctx, hkv, d, len(ctx)
        nb = [(n + 15) // 16 for n in ctx]
        self.first = [int(rng.integers(0, n // 2 + 1)) for n in ctx] if first is None else first
        if fresh and not own_first_block:
            self.first = [f // 16 * 16 for f in self.first]
        self.kept = [sorted(rng.choice(n - f, int(round(share * (n - f))), replace=False).tolist()) if n > f else []
                     for n, f in zip(ctx, self.first)]
        blocks = 2 * sum(nb) + 3
        ids = rng.permutation(blocks).tolist()
        self.width = max(nb + [1])
        self.table = np.full((self.batch, self.width), -9, np.int32)
        self.to = np.full((self.batch, self.width), -9, np.int32)
        for b in range(self.batch):
            for j in range(nb[b]):
                self.table[b, j] = ids.pop()
                keeps = 16 * j < self.first[b] if own_first_block else 16 * j + 15 < self.first[b]
                self.to[b, j] = self.table[b, j] if keeps else ids.pop()
        if not fresh:
            self.to = self.table
        self.fresh, self.blocks = fresh, blocks
        self.k, self.v = (rng.integers(0, 65536, (blocks, hkv, 16, d)).astype(np.uint16) for _ in range(2))
        self.totals = rng.random((self.batch, max(ctx + [0]) + 2)).astype(np.float32)

    def run(self, totals="in place", alias=True, stream=None):
        t = self.t = dict(k=dev16(self.k), v=dev16(self.v), table=dev32(self.table), to=dev32(self.to),
                          first=dev32(self.first), ctx=dev32(self.ctx), lens=dev32([len(x) for x in self.kept]),
                          totals=torch.tensor(self.totals, device=DEV))
        stride = max([len(x) for x in self.kept] + [1]) + 1
        kept = np.full((self.batch, stride), -1, np.int64)
        for b, x in enumerate(self.kept):
            kept[b, :len(x)] = x
        t["kept"] = dev32(kept)
        t["after"] = t["totals"] if totals == "in place" else torch.full_like(t["totals"], -7.0)
        t["new"] = t["ctx"] if alias else torch.zeros_like(t["ctx"])
        self.pool = pa.kv_pool_create(self.blocks, 16, self.hkv, self.d, t["k"], t["v"])

        def call(stream=stream):
            pa.paged_attn_compact(self.pool, t["table"], self.width, t["to"] if self.fresh else None,
                                  self.width if self.fresh else 0, t["first"], t["ctx"], self.batch, max(self.ctx + [0]),
                                  t["kept"], stride, t["lens"], t["totals"] if totals else None,
                                  t["after"] if totals else None, self.totals.shape[1] if totals else 0, t["new"], stream)
        self.call = call
        call()
        torch.cuda.synchronize()
        k, v = self.k, self.v
        for b in range(self.batch):
            k = oracle.compact(k, self.table[b], self.to[b], self.first[b], self.kept[b])
            v = oracle.compact(v, self.table[b], self.to[b], self.first[b], self.kept[b])
        assert np.array_equal(t["k"].cpu().numpy().view(np.uint16), k)
        assert np.array_equal(t["v"].cpu().numpy().view(np.uint16), v)
        assert t["new"].tolist() == [f + len(x) for f, x in zip(self.first, self.kept)]
        if totals:
            want = self.totals.copy() if totals == "in place" else np.full_like(self.totals, -7.0)
            for b, n in enumerate(self.ctx):
                f, m = self.first[b], len(self.kept[b])
                row = self.totals[b, f:n][self.kept[b]]
                want[b, :n] = 0
                want[b, :min(f, n)] = self.totals[b, :min(f, n)]
                want[b, f:f + m] = row
            assert np.array_equal(t["after"].cpu().numpy(), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("share", [0.0, 0.02, 0.5, 0.97, 1.0])
def test_move(share, fresh, d):
    print(f"[gpu case] compact {share} {fresh} {d}", flush=True)
    ctx = [0, 1, 15, 16, 17, 100, 333, 1000, 2049]
    Move(int(share * 100) + d, ctx, 3, d, share, fresh=fresh).run()
    Move(int(share * 100) + d + 1, ctx, 2, d, share, fresh=fresh).run(totals="apart", alias=False)
    Move(int(share * 100) + d + 2, ctx, 1, d, share, fresh=fresh, first=[0] * 9).run(totals=None)


def test_move_with_the_first_block_shared_by_both_tables():
    """The block in which the first tokens end may stay the sequence's own."""
    print("[gpu case] compact own first block", flush=True)
    for seed in range(4):
        Move(seed, [200, 37, 640, 17], 2, 128, 0.6, fresh=True, own_first_block=True, first=[23, 5, 500, 16]).run()


def test_move_of_long_sequences():
    print("[gpu case] compact long", flush=True)
    Move(1, [20011], 2, 128, 0.7, first=[33]).run()
    Move(2, [20011], 2, 64, 0.7, first=[32], fresh=True).run()


def test_move_repeats():
    """What overlaps in place comes out the same every time."""
    print("[gpu case] compact repeated", flush=True)
    for i in range(10):
        Move(7, [3000, 2999, 1500, 800], 8, 128, 0.8, first=[0, 7, 16, 31]).run()


def test_tokens_beyond_the_second_table_stay():
    print("[gpu case] compact short table", flush=True)
    m = Move(5, [200], 2, 64, 1.0, first=[0], fresh=True)
    t = dict(k=dev16(m.k), v=dev16(m.v), table=dev32(m.table), to=dev32(m.to[:, :3]), lens=dev32([200]),
             kept=dev32([list(range(200))]), ctx=dev32([200]))
    pool = pa.kv_pool_create(m.blocks, 16, 2, 64, t["k"], t["v"])
    pa.paged_attn_compact(pool, t["table"], m.width, t["to"], 3, None, t["ctx"], 1, 200, t["kept"], 200, t["lens"], None,
                          None, 0, None)
    torch.cuda.synchronize()
    assert np.array_equal(t["k"].cpu().numpy().view(np.uint16),
                          oracle.compact(m.k, m.table[0], m.to[0], 0, list(range(48))))


def test_bad_device_data_stays_inside():
    """Lengths, tables and lists that lie: nothing outside the pool, the totals and the lists is written."""
    print("[gpu case] keep bad device data", flush=True)
    big = 2 ** 31 - 1
    batch, hkv, d, blocks, width, top = 3, 2, 64, 6, 5, 70
    for ctx in ([10, 70, 33], [big, -big - 1, 5]):
        for ids, lie in ((-5, -big - 1), (big, big), (3, 20)):
            k = torch.full((blocks + 2, hkv, 16, d), 7, dtype=torch.int16, device=DEV)
            v = k.clone()
            pool = pa.kv_pool_create(blocks, 16, hkv, d, k[1:], v[1:])
            totals = torch.full((batch + 2, top), 7.0, device=DEV)
            kept = torch.full((batch + 2, 40), 7, dtype=torch.int32, device=DEV)
            lens = torch.full((batch + 2,), 7, dtype=torch.int32, device=DEV)
            k[1:-1], v[1:-1], totals[1:-1] = 1, 1, 1.0
            table, first, what = dev32(np.full((batch, width), ids)), dev32(np.full(batch, lie)), dev32(ctx)
            pa.paged_attn_keep_heaviest(totals[1:], top, first, what, batch, top, 5, 40, kept[1:], 40, lens[1:])
            for to in (None, table):
                for lists, counts in ((kept[1:], lens[1:]), (dev32(np.full((batch, 40), lie)), dev32(np.full(batch, lie)))):
                    pa.paged_attn_compact(pool, table, width, to, 0 if to is None else width, first, what, batch, top,
                                          lists, 40, counts, totals[1:], totals[1:], top, None)
            torch.cuda.synchronize()
            for x in (k, v, totals, kept, lens):
                assert (x[0] == 7).all() and (x[-1] == 7).all()
            assert ((k == 1) | (k == 7)).all()
