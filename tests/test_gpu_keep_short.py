"""Sequences that are shorter than their first tokens (padded slots of a captured step
among them) through the choice of the tokens that stay and their move: they keep what
they have and nothing moves."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tokens as oracle  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import DEV, dev16, dev32  # noqa: E402

pytestmark = pytest.mark.gpu


class Cut:
    """A pool with tables that hold `width` blocks of every sequence's own, and other blocks to move to."""

    def __init__(self, seed, ctx, first, hkv, d, fresh):
        rng = np.random.default_rng(seed)
        self.ctx, self.first, self.hkv, self.d, self.fresh, self.batch = ctx, first, hkv, d, fresh, len(ctx)
        self.top = max(ctx + first)
        self.width = (self.top + 15) // 16
        self.blocks = 2 * self.batch * self.width
        ids = rng.permutation(self.blocks).reshape(2, self.batch, self.width).astype(np.int32)
        self.table, self.to = ids
        if fresh:       # tokens before the first block that moves stay where they are
            for b, f in enumerate(first):
                self.to[b, :f // 16] = self.table[b, :f // 16]
        else:
            self.to = self.table
        self.k, self.v = (rng.integers(0, 65536, (self.blocks, hkv, 16, d)).astype(np.uint16) for _ in range(2))
        self.totals = rng.random((self.batch, self.top)).astype(np.float32)
        self.t = dict(k=dev16(self.k), v=dev16(self.v), table=dev32(self.table), to=dev32(self.to), ctx=dev32(ctx),
                      first=dev32(first), totals=torch.tensor(self.totals, device=DEV))
        self.pool = pa.kv_pool_create(self.blocks, 16, hkv, d, self.t["k"], self.t["v"])

    def compact(self, kept, stride, lens, after, new):
        t = self.t
        pa.paged_attn_compact(self.pool, t["table"], self.width, t["to"] if self.fresh else None,
                              self.width if self.fresh else 0, t["first"], t["ctx"], self.batch, self.top, kept, stride,
                              lens, None if after is None else t["totals"], after, 0 if after is None else self.top, new)

    def check(self, kept, after, new, untouched):
        """kept: the lists that hold.  untouched: what rows apart hold behind the context."""
        torch.cuda.synchronize()
        k, v = self.k.copy(), self.v.copy()
        want = np.full_like(self.totals, untouched) if after is not self.t["totals"] else self.totals.copy()
        for b, n in enumerate(self.ctx):
            f, m = min(self.first[b], n), len(kept[b])
            source, goal = f + np.array(kept[b], int), f + np.arange(m)
            for x, before in ((k, self.k), (v, self.v)):       # (blocks are a sequence's own)
                x[self.to[b, goal // 16], :, goal % 16] = before[self.table[b, source // 16], :, source % 16]
            want[b, :n] = 0
            want[b, :f] = self.totals[b, :f]
            want[b, f:f + m] = self.totals[b, f:n][kept[b]]
        assert new.tolist() == [min(f, n) + len(x) for f, n, x in zip(self.first, self.ctx, kept)]
        assert np.array_equal(self.t["k"].cpu().numpy().view(np.uint16), k)
        assert np.array_equal(self.t["v"].cpu().numpy().view(np.uint16), v)
        if after is not None:
            assert np.array_equal(after.cpu().numpy(), want)


CTX, FIRST = [0, 5, 16, 40, 300, 17, 0, 33, 700], [16, 16, 16, 64, 32, 17, 0, 1000, 0]


@pytest.mark.parametrize("totals", ["in place", "apart", None])
@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("fresh", [False, True])
@pytest.mark.parametrize("times,hkv,d", [(1, 2, 64), (1, 1, 128), (24, 2, 64)])
def test_choice_and_move(times, hkv, d, fresh, alias, totals):
    """As the choice gives them; up to 1024 workgroups and more."""
    print(f"[gpu case] short sequences {times} {hkv} {d} {fresh} {alias} {totals}", flush=True)
    c = Cut(times + hkv, CTX * times, FIRST * times, hkv, d, fresh)
    keep, recent = 120, 9
    kept = torch.full((c.batch, keep), 55, dtype=torch.int32, device=DEV)
    lens = torch.full((c.batch,), 55, dtype=torch.int32, device=DEV)
    pa.paged_attn_keep_heaviest(c.t["totals"], c.top, c.t["first"], c.t["ctx"], c.batch, c.top, recent, keep, kept, keep, lens)
    after = None if totals is None else c.t["totals"] if totals == "in place" else torch.full_like(c.t["totals"], -7.0)
    new = c.t["ctx"] if alias else torch.full_like(c.t["ctx"], 55)
    c.compact(kept, keep, lens, after, new)
    c.check([oracle.keep_heaviest(c.totals[b, :n], c.first[b], recent, keep) for b, n in enumerate(c.ctx)], after, new, -7.0)


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("fresh", [False, True])
def test_stale_lists(fresh, alias):
    """Lists of an earlier step, in slots whose sequence has gone: nothing of them moves."""
    print(f"[gpu case] short sequences stale lists {fresh} {alias}", flush=True)
    c = Cut(3, CTX, FIRST, 2, 128, fresh)
    lists = [sorted(set(range(0, n - f, 3))) if n >= f else [1, 2, 5] for n, f in zip(c.ctx, c.first)]
    stride = max(len(x) for x in lists)
    kept = np.full((c.batch, stride), -1)
    for b, x in enumerate(lists):
        kept[b, :len(x)] = x
    after, new = torch.full_like(c.t["totals"], -7.0), c.t["ctx"] if alias else torch.full_like(c.t["ctx"], 55)
    c.compact(dev32(kept), stride, dev32([len(x) for x in lists]), after, new)
    c.check([x if n >= f else [] for x, n, f in zip(lists, c.ctx, c.first)], after, new, -7.0)
