"""Bounds of blocks, the choice by them, attention over chosen blocks, and decode
attention whose weights are added to totals, against the float64 oracle.

Bounds and choices are exact.  Outputs have the tolerance of test_gpu_biased: with
|scores| at most S a weight is off by a factor 1 +- w, w = 2^-17 + S 10^-6 + 2^-20, an
output by 2 w max |V| and half a step of bf16.  A total has no bf16 in it: weights off
by 1 +- 2 (S 10^-6 + 2^-20) (score and log-sum-exp), a sum over Hq heads by Hq 2^-23 of
itself, the product with the decay and the addition by 2^-23 of their values.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tokens as oracle  # noqa: E402
from oracle.attention import bf16_to_f64  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import DEV, INF, NAN, Case, bits, dev16, dev32  # noqa: E402

pytestmark = pytest.mark.gpu


def exact_bits(rng, shape):
    """bf16 bits of multiples of 1/16 up to 8: their products and sums are exact in 64 bits, and many are equal."""
    x = (rng.integers(-127, 128, shape) / 16.0).astype(np.float32).view(np.uint32)
    assert ((x & 0xffff) == 0).all()
    return (x >> 16).astype(np.uint16)


class Sparse(Case):
    def __init__(self, seed, ctx, hq, hkv, d, first, last, most, exact=True, **kw):
        super().__init__(seed, ctx, [1] * len(ctx), hq, hkv, d, **kw)
        self.first, self.last, self.most = first, last, most
        rng = np.random.default_rng(seed + 7)
        if exact:
            for b, n in enumerate(self.ctx):
                for t0 in range(0, n, 16):
                    m = min(16, n - t0)
                    self.k[self.table[b, t0 // 16], :, :m] = exact_bits(rng, (hkv, m, d))
            self.q = exact_bits(rng, (self.batch, hq, d))

    def oracle_picks(self):
        picks = np.full((self.batch, self.hkv, self.most), -1)
        group = self.hq // self.hkv
        k, q = bf16_to_f64(self.k), bf16_to_f64(self.q)
        for b, n in enumerate(self.ctx):
            nb = (n + 15) // 16
            for g in range(self.hkv):
                rows = q[b, g * group:(g + 1) * group]
                scores = []
                for j in range(nb):
                    bounds = oracle.block_bounds(k[self.table[b, j], g, :min(16, n - 16 * j)])
                    with np.errstate(all="ignore"):
                        scores.append(np.maximum(rows * bounds[0], rows * bounds[1]).sum())
                chosen = oracle.select_blocks(scores, self.first, self.last, self.most)
                picks[b, g, :len(chosen)] = chosen
        return picks

    def setup(self, spare=0):
        t = self.t = dict(k=dev16(self.k), v=dev16(self.v), q=dev16(self.q), ctx=dev32(self.ctx))
        self.top = int(self.ctx.max(initial=0)) + spare
        if self.width * 16 < self.top:
            self.table = np.concatenate([self.table, np.full((self.batch, self.top // 16 + 1), -9, np.int32)], axis=1)
            self.width = self.table.shape[1]
        t["table"] = dev32(self.table)
        self.pool = pa.kv_pool_create(self.blocks, 16, self.hkv, self.d, t["k"], t["v"])
        t["bounds"] = torch.full((self.blocks, self.hkv, 2, self.d), 0x4242, dtype=torch.int16, device=DEV)
        t["picked"] = torch.full((self.batch, self.hkv, self.most), 77, dtype=torch.int32, device=DEV)
        t["out"] = torch.full((self.batch, self.hq, self.d), 0x4242, dtype=torch.int16, device=DEV)
        self.select_bytes = pa.paged_attn_select_workspace_size(self.pool, self.batch, self.top, self.most)
        self.attend_bytes = pa.paged_attn_selected_workspace_size(self.pool, self.batch, self.hq, self.most)
        t["ws"] = torch.full((max(self.select_bytes, self.attend_bytes, 16),), 255, dtype=torch.uint8, device=DEV)
        return t

    def bound(self, new=None, first=None, stream=None):
        t = self.t
        pa.paged_attn_block_bounds(self.pool, t["bounds"], t["table"], self.width, first, t["ctx"], self.batch, self.top,
                                   self.top if new is None else new, stream)

    def select(self, stream=None):
        t = self.t
        pa.paged_attn_select_blocks(self.pool, t["q"], t["bounds"], t["table"], self.width, t["ctx"], self.batch, self.hq,
                                    self.top, self.first, self.last, self.most, t["ws"], self.select_bytes, t["picked"],
                                    stream)

    def attend(self, picked=None, most=None, stream=None):
        t = self.t
        pa.paged_attn_decode_selected(self.pool, t["q"], t["table"], self.width, t["ctx"], self.batch, self.hq, self.scale,
                                      self.top, t["picked"] if picked is None else picked,
                                      self.most if most is None else most, t["ws"], self.attend_bytes, t["out"], stream)

    def check_out(self, picks, qscale=1.0):
        torch.cuda.synchronize()
        ref = oracle.selected_attention(bf16_to_f64(self.q), picks, self.k, self.v, self.table, self.ctx,
                                        np.float64(np.float32(self.scale)))
        self.check(self.t["out"].cpu().numpy().view(np.uint16), ref, 40.0 * qscale)


SPARSE = {
    "one_token": dict(ctx=[1], hq=8, hkv=2, d=64, first=0, last=1, most=1),
    "all_taken": dict(ctx=[0, 1, 16, 17, 100], hq=8, hkv=2, d=128, first=1, last=1, most=8),
    "ragged": dict(ctx=[333, 16, 0, 700, 129, 128, 127], hq=32, hkv=8, d=128, first=1, last=2, most=8),
    "one_free": dict(ctx=[2000, 1999], hq=8, hkv=2, d=64, first=2, last=5, most=8),
    "none_free": dict(ctx=[500, 90], hq=8, hkv=2, d=64, first=2, last=2, most=4),
    "all_but_one": dict(ctx=[1000], hq=8, hkv=1, d=128, first=0, last=1, most=62),
    "odd_group": dict(ctx=[1500, 40], hq=15, hkv=5, d=64, first=0, last=3, most=20),
    "seven_heads": dict(ctx=[1200, 800], hq=28, hkv=4, d=128, first=3, last=1, most=11),
    "many_heads": dict(ctx=[900, 300], hq=71, hkv=1, d=128, first=1, last=1, most=13),
    "many": dict(ctx=[20 + 41 * i for i in range(60)], hq=8, hkv=2, d=128, first=1, last=1, most=17),
    "long": dict(ctx=[30000, 9001], hq=8, hkv=2, d=64, first=1, last=4, most=150),
    "very_long": dict(ctx=[70001], hq=4, hkv=1, d=64, first=4, last=16, most=256),
    "long_lists": dict(ctx=[6500, 5000] + [300, 17, 0] * 5, hq=8, hkv=8, d=128, first=1, last=1, most=390),
    "negative_scale": dict(ctx=[700], hq=8, hkv=2, d=128, first=0, last=1, most=9, scale=-0.1),
    "many_rows": dict(ctx=[30 + 61 * i for i in range(65)], hq=8, hkv=4, d=64, first=0, last=1, most=10),
    "many_long_rows": dict(ctx=[5 + 141 * i for i in range(65)], hq=8, hkv=4, d=128, first=1, last=1, most=30),
}


@pytest.mark.parametrize("spare", [0, 5000])
@pytest.mark.parametrize("name", sorted(SPARSE))
def test_sparse(name, spare):
    """Bounds, choice and attention of one step."""
    print(f"[gpu case] sparse {name} {spare}", flush=True)
    c = Sparse(len(name) + 20, **SPARSE[name])
    t = c.setup(spare)
    c.bound()
    c.select()
    c.attend()
    torch.cuda.synchronize()
    got = t["bounds"].cpu().numpy().view(np.uint16)
    k = bf16_to_f64(c.k)
    done = set()
    for b, n in enumerate(c.ctx):
        for j in range((n + 15) // 16):
            done.add(c.table[b, j])
            for g in range(c.hkv):
                ref = oracle.block_bounds(k[c.table[b, j], g, :min(16, n - 16 * j)])
                assert np.array_equal(bf16_to_f64(got[c.table[b, j], g]), ref)
    rest = [i for i in range(c.blocks) if i not in done]
    assert (got[rest] == 0x4242).all()
    picks = c.oracle_picks()
    assert np.array_equal(t["picked"].cpu().numpy(), picks)
    # exact inputs are larger than N(0, 1) ones: |q|, |k| <= 8
    c.check_out(picks, 8.0)


def test_bounds_of_new_tokens():
    """first_tokens and max_new choose the blocks that are done anew."""
    print("[gpu case] bounds of new tokens", flush=True)
    c = Sparse(5, ctx=[100, 33, 16, 0, 47], hq=8, hkv=2, d=128, first=0, last=1, most=4)
    t = c.setup()

    def done():
        torch.cuda.synchronize()
        x = t["bounds"].cpu().numpy().view(np.uint16)
        t["bounds"].fill_(0x4242)
        return [[j for j in range((n + 15) // 16) if (x[c.table[b, j]] != 0x4242).any()] for b, n in enumerate(c.ctx)]
    c.bound(new=1)
    assert done() == [[6], [2], [0], [], [2]]
    c.bound(new=2)
    assert done() == [[6], [1, 2], [0], [], [2]]
    c.bound(new=20)
    assert done() == [[5, 6], [0, 1, 2], [0], [], [1, 2]]
    c.bound(first=dev32([99, 16, 16, 0, -5]))
    assert done() == [[6], [1, 2], [], [], [0, 1, 2]]
    c.bound(new=17, first=dev32([0, 16, 15, 3, 2 ** 31 - 1]))
    assert done() == [[5, 6], [1, 2], [0], [], []]


def test_bounds_of_special_keys():
    """NaN is left out, infinities are kept, a dimension of NaN alone gives an empty range."""
    print("[gpu case] bounds of special keys", flush=True)
    c = Sparse(6, ctx=[20], hq=4, hkv=1, d=64, first=0, last=1, most=2)
    c.k[c.table[0, 0], 0, 3, 5] = NAN
    c.k[c.table[0, 0], 0, 4, 6] = INF
    c.k[c.table[0, 0], 0, 5, 8], c.k[c.table[0, 0], 0, 6, 9] = 0x7F81, 0xFF81     # signalling ones
    c.k[c.table[0, 0], 0, :, 7] = NAN
    t = c.setup()
    c.bound()
    torch.cuda.synchronize()
    got = bf16_to_f64(t["bounds"].cpu().numpy().view(np.uint16)[c.table[0, 0], 0])
    ref = oracle.block_bounds(bf16_to_f64(c.k[c.table[0, 0], 0]))
    assert np.array_equal(got, ref) and got[0, 7] == np.inf and got[1, 7] == -np.inf and got[1, 6] == np.inf


@pytest.mark.parametrize("hkv,d,ctx,most", [(64, 64, 70001, 99), (32, 128, 70001, 2500), (300, 64, 33000, 200), (2, 64, 300000, 64)])
def test_choice_among_many(hkv, d, ctx, most):
    """Rounds of several per wavefront, choices beyond the keys that LDS holds: against sorted 64-bit scores (exact inputs)."""
    print(f"[gpu case] choice among many {hkv} {d} {ctx}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(5)
    nb, group = (ctx + 15) // 16, 2
    table = torch.randperm(nb, generator=gen, device=DEV)
    bounds = torch.randint(-127, 128, (nb, hkv, 2, d), generator=gen, device=DEV).float().div_(16).to(torch.bfloat16)
    bounds = torch.stack([bounds.amin(2), bounds.amax(2)], 2)
    q = torch.randint(-127, 128, (1, hkv * group, d), generator=gen, device=DEV).float().div_(16).to(torch.bfloat16)
    scores = torch.zeros((hkv, nb), dtype=torch.float64, device=DEV)
    for g in range(hkv):
        lo, hi = (bounds[table, g, i].double() for i in range(2))
        for h in range(group):
            x = q[0, g * group + h].double()
            scores[g] += torch.maximum(x * lo, x * hi).sum(1)
    first, last = 3, 5
    order = torch.sort(scores[:, first:nb - last], dim=1, descending=True, stable=True).indices[:, :most - first - last] + first
    want = torch.cat([torch.arange(first, device=DEV).expand(hkv, -1), torch.sort(order, dim=1).values,
                      torch.arange(nb - last, nb, device=DEV).expand(hkv, -1)], 1)
    k = torch.zeros(16, dtype=torch.int16, device=DEV)         # the choice reads no key
    pool = pa.kv_pool_create(nb, 16, min(hkv, 64), d, k, k)
    if hkv > 64:                                               # rows by sequences instead: 64 heads are a pool's most
        batch, heads = hkv // 50, 50
        pool = pa.kv_pool_create(nb * batch, 16, heads, d, k, k)
        shuffled = bounds.view(nb, batch, heads, 2, d).transpose(0, 1).reshape(batch * nb, heads, 2, d).contiguous()
        tables = torch.stack([table + b * nb for b in range(batch)]).int()
    else:
        batch, heads, shuffled, tables = 1, hkv, bounds, table.int()[None]
    size = pa.paged_attn_select_workspace_size(pool, batch, ctx, most)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    picked = torch.zeros((batch, heads, most), dtype=torch.int32, device=DEV)
    pa.paged_attn_select_blocks(pool, q, shuffled, tables.contiguous(), nb, dev32([ctx] * batch), batch, heads * group, ctx,
                                first, last, most, ws, size, picked)
    torch.cuda.synchronize()
    assert torch.equal(picked.view(hkv, most), want.int())


@pytest.mark.parametrize("d", [64, 128])
def test_choice_of_close_and_equal_scores(d):
    """Scores that fp32 sums cannot tell apart are told apart; equal ones go to the lower block."""
    print(f"[gpu case] close scores {d}", flush=True)
    n, hkv = 200, 2
    c = Sparse(8, ctx=[16 * n], hq=2, hkv=hkv, d=d, first=0, last=1, most=40)
    rng = np.random.default_rng(1)
    c.k[:] = 0
    c.q[:] = 0
    c.q[0, :, 0], c.q[0, :, d - 1], c.q[0, 1, 9] = 0x4580, 0x3B80, 0xBF80        # 4096, 2^-8, -1
    order = rng.permutation(n)
    for j in range(n):
        block = c.table[0, j]
        c.k[block, :, 2, 0] = 0x4580                                             # 4096: every score begins with 2^24
        c.k[block, :, 5, d - 1] = bits_of(float(order[j] // 3))                  # triples are equal
    t = c.setup()
    c.bound()
    c.select()
    torch.cuda.synchronize()
    scores = [(order[j] // 3) / 256 for j in range(n)]
    want = oracle.select_blocks(scores, 0, 1, 40)
    assert np.array_equal(t["picked"].cpu().numpy()[0], [want] * hkv)
    # all equal: the first ones
    c.q[:] = 0
    t["q"].copy_(dev16(c.q))
    c.select()
    torch.cuda.synchronize()
    assert np.array_equal(t["picked"].cpu().numpy()[0, 0], list(range(39)) + [n - 1])


@pytest.mark.parametrize("n,coarse,fine", [(1500, 30, 3), (1500, 64, 1), (1500, 65, 5), (5000, 60, 64), (5000, 50, 100), (1030, 1, 1)])
def test_choice_by_bits_far_below_the_first_that_differ(n, coarse, fine):
    """Groups of scores that only bits 2^-32 of the largest tell apart, and within them groups of equal ones."""
    print(f"[gpu case] low bits {n} {coarse} {fine}", flush=True)
    c = Sparse(9, ctx=[16 * n], hq=1, hkv=1, d=64, first=0, last=1, most=n // 3)
    rng = np.random.default_rng(n)
    c.k[:] = 0
    c.q[:] = 0
    c.q[0, 0, 0], c.q[0, 0, 5], c.q[0, 0, 63] = 0x4580, 0x4580, 0x3B80           # 4096, 4096, 2^-8
    order = rng.permutation(n)
    scores = np.zeros(n)
    for j in range(2, n):                                                        # the first two: 0
        block, hi, lo = c.table[0, j], order[j] // coarse % 200, order[j] % coarse // fine
        c.k[block, :, 2, 0] = 0x4580
        c.k[block, :, 7, 5] = bits_of(float(hi))
        c.k[block, :, 5, 63] = bits_of(float(lo))
        scores[j] = 2.0 ** 24 + 4096.0 * hi + lo / 256
    t = c.setup()
    c.bound()
    c.select()
    torch.cuda.synchronize()
    assert t["picked"].cpu().numpy()[0, 0].tolist() == oracle.select_blocks(scores, 0, 1, n // 3)


def bits_of(x):
    return int(np.float32(x).view(np.uint32) >> 16)


def test_choice_of_infinite_and_nan_scores():
    """A score of NaN counts as the highest, then +infinity; -infinity is the lowest."""
    print("[gpu case] infinite scores", flush=True)
    c = Sparse(11, ctx=[16 * 20], hq=1, hkv=1, d=64, first=0, last=1, most=4)
    c.q[:] = 0
    c.q[0, 0, 0], c.q[0, 0, 1] = 0x3F80, 0xBF80
    t = c.setup()
    c.bound()
    lo, hi = np.zeros((20, 64), np.float32), np.ones((20, 64), np.float32)
    hi[3, 0] = np.inf
    hi[7, 0], lo[7, 1] = np.inf, np.inf                                         # inf - inf
    hi[0, 0] = -np.inf
    x = torch.tensor(np.stack([lo, hi], 1)[:, None], device=DEV).to(torch.bfloat16).view(torch.int16)
    for j in range(20):
        t["bounds"][int(c.table[0, j])] = x[j]
    c.select()
    torch.cuda.synchronize()
    assert t["picked"].cpu().numpy()[0, 0].tolist() == [1, 3, 7, 19]


@pytest.mark.parametrize("nan", [0x7FC0, 0xFFC0])
def test_choice_of_a_query_that_is_nan(nan):
    """All scores of its KV head are NaN, the highest: the lowest blocks.  The others choose as ever."""
    print(f"[gpu case] nan in q {nan:x}", flush=True)
    c = Sparse(22, ctx=[900, 2000], hq=22, hkv=2, d=128, first=1, last=2, most=30)
    want = c.oracle_picks()
    c.q[1, 15, 77] = nan                                                        # the fifth of eleven heads
    c.q[0, 10, 0] = nan                                                         # the last
    c.setup()
    c.bound()
    c.select()
    torch.cuda.synchronize()
    for b, g, n in ((1, 1, 125), (0, 0, 57)):
        want[b, g] = list(range(28)) + [n - 2, n - 1]
    assert np.array_equal(c.t["picked"].cpu().numpy(), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [1, 3, 8])
def test_choice_past_bounds_that_no_head_looks_at(heads, d):
    """q > 0 looks at the greatest values, q < 0 at the least, q = 0 at none: infinities elsewhere do not count."""
    print(f"[gpu case] infinite bounds on the other side {heads} {d}", flush=True)
    n = 150
    c = Sparse(21, ctx=[16 * n], hq=heads, hkv=1, d=d, first=0, last=1, most=41)
    rng = np.random.default_rng(heads + d)
    sign = rng.integers(-1, 2, d)                                               # of all heads, so that a side is unused
    q = sign * rng.integers(1, 9, (heads, d)).astype(np.float64)
    q[0, :3] = [2, -2, 0]
    q[1:, :3] = rng.integers(0, 3, (heads - 1, 3)) * np.array([1, -1, 0])
    c.q[0] = (q.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    lo = rng.integers(-99, 0, (n, d)).astype(np.float64)
    hi = rng.integers(0, 99, (n, d)).astype(np.float64)
    for j in rng.permutation(n)[:90]:                                           # sides that are not looked at
        lo[j, 0], hi[j, 1] = -np.inf, np.inf
        lo[j, 2], hi[j, 2] = rng.choice([-np.inf, -1.0]), np.inf
    lo[5, 3:], hi[5, 3:] = -np.inf, np.inf                                      # looked at: the highest
    lo[6], hi[6] = np.inf, -np.inf                                              # no number in any dimension: the lowest
    t = c.setup()
    c.bound()
    x = torch.tensor(np.stack([lo, hi], 1)[:, None], device=DEV).to(torch.bfloat16).view(torch.int16)
    for j in range(n):
        t["bounds"][int(c.table[0, j])] = x[j]
    c.select()
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        part = np.where(q > 0, q * hi[:, None], np.where(q < 0, q * lo[:, None], 0.0))
    scores = part.sum((1, 2))
    assert not np.isnan(scores).any() and scores[5] == np.inf and scores[6] == -np.inf
    assert t["picked"].cpu().numpy()[0, 0].tolist() == oracle.select_blocks(scores, 0, 1, 41)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (32, 4, 64), (71, 1, 64), (3, 3, 128)])
def test_lists_of_the_callers_own(hq, hkv, d):
    """Any order, entries that name no block, blocks listed twice, lists of none."""
    print(f"[gpu case] own lists {hq} {hkv} {d}", flush=True)
    rng = np.random.default_rng(2)
    c = Sparse(12, ctx=[700, 35, 0, 160], hq=hq, hkv=hkv, d=d, first=0, last=1, most=90, exact=False)
    c.setup()
    picks = rng.integers(-3, 50, (4, hkv, 90))
    picks[3] = rng.choice([-1, 10, 11, 2 ** 31 - 1, -2 ** 31, 1 << 26], (hkv, 90))    # 10 blocks: none of these
    c.attend(dev32(picks))
    c.check_out(picks)
    assert (c.t["out"][2:] == 0).all()
    c.attend(None, 0)
    torch.cuda.synchronize()
    assert (c.t["out"] == 0).all()
    # a single list entry, and one partition more than the blocks fill
    one = rng.integers(0, 2, (4, hkv, 1))
    c.attend(dev32(one), 1)
    c.check_out(one)


def test_unlisted_blocks_do_not_matter():
    print("[gpu case] unlisted blocks", flush=True)
    c = Sparse(13, ctx=[500, 64], hq=16, hkv=8, d=128, first=0, last=1, most=6, exact=False)
    picks = np.broadcast_to(np.array([30, 0, 31, 7, -1, 3]), (2, 8, 6))
    for b, n in enumerate(c.ctx):
        for j in range((n + 15) // 16):
            if j not in picks[0, 0]:
                c.k[c.table[b, j]] = NAN
                c.v[c.table[b, j]] = INF
    c.setup()
    c.attend(dev32(picks))
    c.check_out(picks)


WEIGHTS = {
    "one_token": dict(ctx=[1], hq=8, hkv=2, d=64),
    "ragged": dict(ctx=[1, 15, 16, 17, 100, 0, 333, 257, 256], hq=8, hkv=2, d=64),
    "groups_of_four": dict(ctx=[31, 1000, 0, 4097], hq=32, hkv=8, d=128),
    "groups_of_eight": dict(ctx=[700, 65], hq=64, hkv=8, d=128),
    "no_groups": dict(ctx=[300, 5, 2111], hq=12, hkv=12, d=64),
    "seven_heads": dict(ctx=[129, 2048], hq=28, hkv=4, d=128),
    "many_heads": dict(ctx=[77, 600], hq=71, hkv=1, d=64),
    "heads_beyond_lds": dict(ctx=[100, 40], hq=1040, hkv=52, d=64),      # 52 heads of 20: three tiles of eight each
    "long": dict(ctx=[9001, 20000], hq=16, hkv=2, d=128),
    "one_long_64": dict(ctx=[33333], hq=4, hkv=1, d=64),
    "zero_scale": dict(ctx=[200, 17], hq=8, hkv=2, d=128, scale=0.0),
    "negative_scale": dict(ctx=[200, 17], hq=8, hkv=2, d=128, scale=-0.1),
    "two_a_cu": dict(ctx=[6000, 4097, 2500] + [20, 1030, 700, 1] * 3 + [0], hq=8, hkv=8, d=128),
    # rows that fill the GPU: some kept whole, some split
    "filled": dict(ctx=[2048, 2049, 1024, 1025, 2500, 0, 1, 2047, 2064, 4000] + [9, 40, 70] * 10, hq=32, hkv=8, d=128),
    "filled_eights": dict(ctx=[1024, 1025, 2048, 2049, 3000, 0, 513] + [3, 31, 65] * 11, hq=48, hkv=8, d=128),
    "filled_64": dict(ctx=[2048, 2049, 1025, 2100, 0, 1008] + [2, 16, 90] * 20, hq=8, hkv=8, d=64),
}


class Weights(Case):
    def go(self, spare=0, decay=1.0, start=True, in_place=False, stride=3, stream=None):
        t = self.t = dict(k=dev16(self.k), v=dev16(self.v), q=dev16(self.q), ctx=dev32(self.ctx))
        top = int(self.ctx.max(initial=0)) + spare
        if self.width * 16 < top:
            self.table = np.concatenate([self.table, np.full((self.batch, top // 16 + 1), -9, np.int32)], axis=1)
            self.width = self.table.shape[1]
        t["table"] = dev32(self.table)
        pool = self.pool = pa.kv_pool_create(self.blocks, 16, self.hkv, self.d, t["k"], t["v"])
        rng = np.random.default_rng(5)
        self.before = rng.random((self.batch, top + stride)).astype(np.float32) * 4
        t["totals"] = torch.tensor(self.before, device=DEV)
        after = t["totals"] if in_place else torch.full_like(t["totals"], -7.0)
        out = torch.full((self.batch, self.hq, self.d), 0x4242, dtype=torch.int16, device=DEV)
        size = pa.paged_attn_weights_workspace_size(pool, self.batch, self.hq, top)
        ws = torch.full((max(size, 16) + 64,), 255, dtype=torch.uint8, device=DEV)

        def call(stream=stream):
            pa.paged_attn_decode_weights(pool, t["q"], t["table"], self.width, t["ctx"], self.batch, self.hq, self.scale,
                                         top, decay, t["totals"] if start else None, after, top + stride, ws, size, out,
                                         stream)
        self.call, self.out, self.after = call, out, after
        call()
        torch.cuda.synchronize()
        assert (ws[size:] == 255).all()
        return out.cpu().numpy().view(np.uint16), after.cpu().numpy()

    def check_all(self, out, after, decay, start, rest, score=40.0):
        ref, weights = oracle.decode_weights(bf16_to_f64(self.q), self.k, self.v, self.table, self.ctx,
                                             np.float64(np.float32(self.scale)))
        self.check(out, ref, score)
        for b, n in enumerate(self.ctx):
            old = self.before[b, :n].astype(np.float64) * np.float64(np.float32(decay)) if start else np.zeros(n)
            limit = weights[b] * (2 * (score * 1e-6 + 2.0 ** -20) + self.hq * 2.0 ** -23) + 2.0 ** -23 * np.abs(old + weights[b])
            assert (np.abs(after[b, :n] - (old + weights[b])) <= limit + 1e-30).all()
            assert np.array_equal(after[b, n:], rest[b, n:])


@pytest.mark.parametrize("spare", [0, 5000])
@pytest.mark.parametrize("name", sorted(WEIGHTS))
def test_weights(name, spare):
    print(f"[gpu case] weights {name} {spare}", flush=True)
    kw = WEIGHTS[name]
    c = Weights(len(name), chunk=[1] * len(kw["ctx"]), **kw)
    decay = 0.75 if spare else 1.0
    out, after = c.go(spare, decay, in_place=spare > 0)
    c.check_all(out, after, decay, True, c.before if spare else np.full_like(c.before, -7.0))


def test_weights_without_totals_and_repeated():
    """No totals before; the sums of a step are the same bits every time."""
    print("[gpu case] weights without totals", flush=True)
    c = Weights(3, ctx=[3000, 40, 777], chunk=[1] * 3, hq=32, hkv=8, d=128)
    out, after = c.go(start=False, decay=0.0)
    c.check_all(out, after, 0.0, False, np.full_like(c.before, -7.0))
    for b, n in enumerate(c.ctx):
        assert abs(after[b, :n].sum(dtype=np.float64) - 32) < 1e-3
    for _ in range(3):
        c.after.fill_(-7.0)
        c.call()
        torch.cuda.synchronize()
        assert np.array_equal(c.after.cpu().numpy(), after) and np.array_equal(c.out.cpu().numpy().view(np.uint16), out)


def test_contexts_of_none():
    """A bound of no tokens at all: zeros, and no total is touched."""
    print("[gpu case] weights of empty contexts", flush=True)
    c = Weights(14, ctx=[0, 0, 0], chunk=[1] * 3, hq=8, hkv=2, d=128)
    out, after = c.go(in_place=True)
    assert (out == 0).all() and np.array_equal(after, c.before)
    s = Sparse(15, ctx=[0, 0], hq=8, hkv=2, d=64, first=1, last=2, most=5)
    t = s.setup()
    s.bound()
    s.select()
    s.attend()
    torch.cuda.synchronize()
    assert (t["picked"] == -1).all() and (t["out"] == 0).all() and (t["bounds"] == 0x4242).all()


def test_weights_of_special_values():
    """What stands behind the context does not matter; a NaN among the scores shows in the sequence's totals alone."""
    print("[gpu case] weights of special values", flush=True)
    kw = dict(ctx=[300, 40], chunk=[1, 1], hq=8, hkv=2, d=128)
    out0, after0 = Weights(4, **kw).go()
    c = Weights(4, **kw)
    c.k[c.table[0, 5], 1, 3, 9] = NAN
    out, after = c.go()
    assert np.isnan(after[0, :300]).all() and np.array_equal(after[1], after0[1])
    assert np.array_equal(out[1], out0[1]) and np.array_equal(out[0, :4], out0[0, :4])
    assert np.isnan(bf16_to_f64(out[0, 4:])).all()


def test_bad_device_data_stays_inside():
    """Lengths, tables and lists that lie: nothing outside the outputs is written."""
    print("[gpu case] chosen bad device data", flush=True)
    big = 2 ** 31 - 1
    batch, hq, hkv, d, blocks, width, top, most = 4, 8, 2, 64, 6, 5, 70, 3
    gen = torch.Generator(device=DEV).manual_seed(3)
    k, v = (torch.randn(blocks, hkv, 16, d, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(batch, hq, d, generator=gen, device=DEV).to(torch.bfloat16)
    pool = pa.kv_pool_create(blocks, 16, hkv, d, k, v)
    for ctx in ([10, 70, 33, 10], [big, -big - 1, 5, 0]):
        for ids, lie in ((-5, -big - 1), (big, big), (3, 20)):
            table, lens, first = dev32(np.full((batch, width), ids)), dev32(ctx), dev32(np.full(batch, lie))
            bounds = torch.full((blocks + 2, hkv, 2, d), 3.0, device=DEV, dtype=torch.bfloat16)
            pa.paged_attn_block_bounds(pool, bounds[1:], table, width, first, lens, batch, top, 40)
            size = pa.paged_attn_select_workspace_size(pool, batch, top, most)
            ws = torch.full((size + 32,), 7, dtype=torch.uint8, device=DEV)
            picked = torch.full((batch + 2, hkv, most), 9, device=DEV, dtype=torch.int32)
            pa.paged_attn_select_blocks(pool, q, bounds[1:], table, width, lens, batch, hq, top, 1, 1, most, ws, size,
                                        picked[1:])
            out = torch.full((batch + 2, hq, d), 3.0, device=DEV, dtype=torch.bfloat16)
            pa.paged_attn_decode_selected(pool, q, table, width, lens, batch, hq, 0.1, top,
                                          dev32(np.full((batch, hkv, most), lie)), most, None, 0, out[1:])
            totals = torch.full((batch + 2, top), 3.0, device=DEV)
            need = pa.paged_attn_weights_workspace_size(pool, batch, hq, top)
            ws2 = torch.full((need + 32,), 7, dtype=torch.uint8, device=DEV)
            pa.paged_attn_decode_weights(pool, q, table, width, lens, batch, hq, 0.1, top, 1.0, None, totals[1:], top, ws2,
                                         need, out[1:])
            torch.cuda.synchronize()
            assert all((x[0] == x[0].flatten()[0]).all() and (x[-1] == 3.0).all() for x in (bounds, out, totals))
            assert (picked[0] == 9).all() and (picked[-1] == 9).all()
            assert (ws[size:] == 7).all() and (ws2[need:] == 7).all()
