"""Attention of trees of drafted tokens against the float64 oracle over the same
bf16 inputs; tolerance and case builder are those of test_gpu_biased."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle.attention import bf16_to_f64  # noqa: E402
from oracle.tokens import tree_attention  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import DEV, INF, NAN, NINF, Case, dev16, dev32  # noqa: E402

pytestmark = pytest.mark.gpu


class Tree(Case):
    """reach: a node's parent is among the `reach` before it, or the context."""

    def __init__(self, seed, ctx, chunk, hq, hkv, d, reach=4, parents=None, **kw):
        super().__init__(seed, ctx, chunk, hq, hkv, d, **kw)
        rng = np.random.default_rng(seed + 1000)
        node = np.concatenate([np.arange(m) for m in self.chunk]) if self.rows else np.zeros(0, int)
        self.parents = np.full(self.total, -1, np.int64)
        self.parents[:self.rows] = np.maximum(node - rng.integers(1, reach + 1, self.rows), -1)
        if parents is not None:
            self.parents[:self.rows] = parents

    def reference(self):
        with np.errstate(all="ignore"):
            return tree_attention(bf16_to_f64(self.q[:self.rows]), self.start, self.parents, self.k, self.v, self.table,
                                  self.ctx, np.float64(np.float32(self.scale)), self.cap)

    def run(self, stream=None, spare=0, nodes=0):
        t = self.t = dict(k=dev16(self.k), v=dev16(self.v), q=dev16(self.q), table=dev32(self.table),
                          ctx=dev32(self.ctx), start=dev32(self.start), parents=dev32(self.parents))
        pool = self.pool = pa.kv_pool_create(self.blocks, 16, self.hkv, self.d, t["k"], t["v"])
        most = max(int(self.chunk.max(initial=0)), nodes)
        top = max(int(self.ctx.max(initial=0)), most) + spare
        if self.width * 16 < top:
            self.table = np.concatenate([self.table, np.full((self.batch, top // 16 + 1), -9, np.int32)], axis=1)
            self.width = self.table.shape[1]
            t["table"] = dev32(self.table)
        size = pa.paged_attn_tree_workspace_size(pool, self.batch, self.hq, top, most)
        ws = torch.full((max(size, 16),), 255, dtype=torch.uint8, device=DEV)
        out = torch.full((self.total, self.hq, self.d), 0x4242, dtype=torch.int16, device=DEV)

        def call(stream=stream):
            pa.paged_attn_extend_tree(pool, t["q"], t["start"], self.total, t["parents"], t["table"], self.width, t["ctx"],
                                      self.batch, self.hq, self.scale, self.cap, top, most, ws, size, out, stream)
        self.call, self.out = call, out
        call()
        torch.cuda.synchronize()
        return out.cpu().numpy().view(np.uint16)


TREES = {
    "one_token": dict(ctx=[1], chunk=[1], hq=8, hkv=2, d=64),
    "one_node": dict(ctx=[200, 17, 16, 33], chunk=[1, 1, 1, 1], hq=8, hkv=2, d=128),
    "no_context": dict(ctx=[8, 33, 256], chunk=[8, 33, 256], hq=8, hkv=2, d=128, reach=3),
    "chain": dict(ctx=[100, 70], chunk=[40, 64], hq=16, hkv=8, d=128, reach=1),
    "siblings": dict(ctx=[100, 70], chunk=[40, 64], hq=16, hkv=8, d=64, parents=-1),
    "ragged": dict(ctx=[300, 47, 16, 0, 900, 90], chunk=[31, 32, 16, 0, 33, 0], hq=32, hkv=8, d=128, pad=5),
    "cap": dict(ctx=[500, 64], chunk=[65, 30], hq=28, hkv=4, d=128, cap=20.0, qscale=4.0),
    "cap_64": dict(ctx=[333], chunk=[97], hq=24, hkv=3, d=64, cap=5.0, qscale=4.0, pad=2),
    "most_nodes": dict(ctx=[700, 256], chunk=[256, 255], hq=8, hkv=8, d=128, reach=64),
    "most_nodes_64": dict(ctx=[300], chunk=[256], hq=8, hkv=1, d=64, reach=200),
    "many": dict(ctx=[60 + 7 * i for i in range(70)], chunk=[1 + i % 37 for i in range(70)], hq=32, hkv=8, d=128),
    "many_wide": dict(ctx=[600] * 12, chunk=[200] * 12, hq=32, hkv=8, d=128, reach=16, cap=50.0, qscale=8.0),
    "many_wide_64": dict(ctx=[420] * 12, chunk=[180] * 12, hq=32, hkv=8, d=64, reach=16),
    "long": dict(ctx=[9001, 20000], chunk=[61, 13], hq=16, hkv=2, d=128, reach=8),
    "long_64": dict(ctx=[12000], chunk=[40], hq=12, hkv=4, d=64, reach=8),
    "big_group": dict(ctx=[150], chunk=[9], hq=71, hkv=1, d=128),
    "negative_scale": dict(ctx=[150], chunk=[50], hq=8, hkv=2, d=128, scale=-0.1),
    "zero_scale": dict(ctx=[150], chunk=[50], hq=8, hkv=2, d=128, scale=0.0),
}


@pytest.mark.parametrize("spare", [0, 5000])
@pytest.mark.parametrize("name", sorted(TREES))
def test_tree(name, spare):
    print(f"[gpu case] tree {name} {spare}", flush=True)
    kw = dict(TREES[name])
    c = Tree(len(name) + 40, **kw)
    c.check(c.run(spare=spare), None, 40.0 * kw.get("qscale", 1.0))


@pytest.mark.parametrize("name", ["one_node", "ragged", "cap_64", "many", "long", "long_64", "big_group"])
def test_small_trees_under_a_large_bound(name):
    """max_nodes far above the trees: most tiles of the plan, and most rows of the others, are empty."""
    print(f"[gpu case] tree under 256 nodes {name}", flush=True)
    c = Tree(len(name) + 60, **TREES[name])
    c.check(c.run(nodes=256))
    c.check(c.run(nodes=256, spare=30000))


def test_sequences_that_share_blocks():
    """Trees over a context whose blocks several tables hold."""
    print("[gpu case] tree over shared blocks", flush=True)
    c = Tree(21, ctx=[300, 290, 305], chunk=[20, 9, 31], hq=32, hkv=8, d=128, parents=None)
    c.table[1:, :16] = c.table[0, :16]
    c.check(c.run())


def test_parents_that_are_none():
    """A parent at or behind its node, or negative, stands for the context."""
    print("[gpu case] tree bad parents", flush=True)
    parents = [0, 1, 0, 2 ** 31 - 1, -2 ** 31, 4, 99, 5, 7, 9]
    c = Tree(3, ctx=[50], chunk=[10], hq=8, hkv=2, d=128, parents=parents)
    got = c.run()
    c.check(got)
    c.parents[:10] = [-1, -1, 0, -1, -1, 4, -1, 5, 7, -1]
    assert np.array_equal(c.run(), got)


def test_chain_equals_extend():
    """A chain is an ordinary chunk.  The two calls may take their rows and tokens in other forms, whose sums have other
    orders: each is within the tolerance of the chunk's oracle, and so they are within twice it of each other."""
    print("[gpu case] tree chain against extend", flush=True)
    c = Tree(5, ctx=[300, 90, 45], chunk=[40, 64, 45], hq=16, hkv=4, d=128, reach=1)
    c.parents[:] = np.concatenate([np.arange(m) - 1 for m in c.chunk])
    ref = Case.reference(c)
    c.check(c.run(), ref)
    out = torch.full_like(c.out, 0x4242)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    pa.paged_attn_extend_biased(c.pool, c.t["q"], c.t["start"], c.total, c.t["table"], c.width, c.t["ctx"], 3, 16,
                                c.scale, 0.0, None, 0, None, None, 300, 64, ws, 1 << 20, out)
    torch.cuda.synchronize()
    c.check(out.cpu().numpy().view(np.uint16), ref)


@pytest.mark.parametrize("hq,d", [(8, 128), (8, 64), (64, 128)])
def test_special_values_of_unseen_nodes(hq, d):
    """Infinities and NaN in K and V of nodes: the nodes' descendants show them, the others do not change a bit."""
    print(f"[gpu case] tree special values {hq} {d}", flush=True)
    kw = dict(ctx=[333, 70, 600], chunk=[60, 70, 33], hq=hq, hkv=8, d=d, reach=5)
    clean = Tree(9, **kw).run()
    c = Tree(9, **kw)
    rng = np.random.default_rng(4)
    for b, i in ((0, 20), (0, 41), (1, 33), (2, 7), (2, 32)):
        t = c.ctx[b] - c.chunk[b] + i
        block, line = c.table[b, t // 16], t % 16
        c.k[block, :, line, 3] = NAN
        c.v[block, :, line] = rng.choice([NAN, INF, NINF], size=(8, d))
    got = c.run()
    ref = c.reference()
    fin = np.isfinite(ref).all(-1)
    assert 0.2 < fin.mean() < 1.0
    assert np.array_equal(got[:c.rows][fin], clean[:c.rows][fin])
    assert np.isnan(bf16_to_f64(got[:c.rows])[~fin]).all()


def test_values_that_a_row_sees():
    """An infinity in V alone, in the context and in a node, reaches the rows that see it."""
    print("[gpu case] tree visible infinities", flush=True)
    for hq, chunk in ((8, [60, 30]), (64, [13, 8])):
        c = Tree(10, ctx=[400, 90], chunk=chunk, hq=hq, hkv=8, d=128)
        for b, t in ((0, 400 - chunk[0] + 2), (1, 10), (1, 90 - chunk[1] + 5)):
            c.v[c.table[b, t // 16], b, t % 16, 5::9] = INF
        c.check(c.run())


def test_bad_device_data_stays_inside():
    """Lengths, starts, tables and parents that lie: nothing outside out is written."""
    print("[gpu case] tree bad device data", flush=True)
    big = 2 ** 31 - 1
    batch, hq, hkv, d, total, blocks = 4, 8, 2, 64, 40, 6
    gen = torch.Generator(device=DEV).manual_seed(3)
    k, v = (torch.randn(blocks, hkv, 16, d, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(total, hq, d, generator=gen, device=DEV).to(torch.bfloat16)
    pool = pa.kv_pool_create(blocks, 16, hkv, d, k, v)
    width, top = 5, 70
    size = pa.paged_attn_tree_workspace_size(pool, batch, hq, top, 20)
    ws = torch.full((size + 32,), 7, dtype=torch.uint8, device=DEV)
    for start in ([0, 10, 20, 30, 40], [0, -5, 50, big, 40], [-big - 1, -3, -2, -1, big], [7, 3, 9, 1, 2]):
        for ctx in ([10, 70, 33, 10], [big, -big - 1, 5, 0]):
            for ids, lie in ((-5, -big - 1), (big, big), (3, 20)):
                out = torch.full((total + 2, hq, d), 3.0, device=DEV, dtype=torch.bfloat16)
                pa.paged_attn_extend_tree(pool, q, dev32(start), total, dev32(np.full(total, lie)),
                                          dev32(np.full((batch, width), ids)), width, dev32(ctx), batch, hq, 0.1, 0.0, top,
                                          20, ws, size, out[1:])
                torch.cuda.synchronize()
                assert (out[0] == 3.0).all() and (out[-1] == 3.0).all() and (ws[size:] == 7).all()
