"""The operators of paged_attn_tokens.h together, as a serving loop calls them: a step
of drafted tokens, an eviction and sparse steps over what stays; captured into a
graph; on two streams; over shared blocks; and beyond 4 GiB of cache."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tokens as oracle  # noqa: E402
from oracle.attention import bf16_to_f64  # noqa: E402
from oracle.ops import head_rows  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import DEV, bits, dev16, dev32  # noqa: E402
from test_gpu_chosen import SPARSE, WEIGHTS, Sparse, Weights  # noqa: E402
from test_gpu_keep import Move  # noqa: E402
from test_gpu_tree import TREES, Tree  # noqa: E402

pytestmark = pytest.mark.gpu


def u16(t):
    return t.cpu().numpy().view(np.uint16)


def close(got, ref, vmax, score=40.0):
    """Within the outputs' tolerance (test_gpu_biased)."""
    limit = 2 * (2.0 ** -17 + score * 1e-6 + 2.0 ** -20) * vmax + 2.0 ** -8 * np.abs(ref)
    assert (np.abs(bf16_to_f64(got) - ref) <= limit).all()


class Engine:
    """A small engine's cache: a pool, a table per sequence, and the host's copy of each sequence's rows."""

    def __init__(self, seed, ctx, room, hq=16, hkv=4, d=128):
        self.rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.batch = hq, hkv, d, len(ctx)
        self.width = (max(ctx) + room + 15) // 16
        self.blocks = self.batch * self.width * 2
        self.k, self.v = (torch.from_numpy(bits(self.rng, (self.blocks, hkv, 16, d)).view(np.int16)).to(DEV) for _ in range(2))
        self.pool = pa.kv_pool_create(self.blocks, 16, hkv, d, self.k, self.v)
        self.table = np.array([pa.kv_pool_alloc(self.pool, self.width) for _ in ctx], np.int32)
        self.ctx = np.array(ctx)
        k, v = u16(self.k), u16(self.v)
        t = [np.arange(n) for n in ctx]
        self.rows = [[x[self.table[b, t[b] // 16], :, t[b] % 16].copy() for x in (k, v)] for b in range(self.batch)]
        self.top = self.width * 16

    def host_rows(self):
        k, v = u16(self.k), u16(self.v)
        out = []
        for b, n in enumerate(self.ctx):
            t = np.arange(n)
            out.append([x[self.table[b, t // 16], :, t % 16] for x in (k, v)])
        return out

    def attention(self, q, b, t):
        """Oracle of query heads [hq][d] over sequence b's rows t."""
        k, v = (bf16_to_f64(x[t]) for x in self.rows[b])
        g = self.hq // self.hkv
        return np.concatenate([oracle.rows_over(q[i * g:(i + 1) * g], k[:, i], v[:, i], self.d ** -0.5)[0]
                               for i in range(self.hkv)])


def test_speculation():
    """Three steps: drafted rows rotated to their depths and appended, the tree's attention, the accepted path kept."""
    print("[gpu case] speculation", flush=True)
    e = Engine(1, [37, 200, 64, 5], 64)
    hq, hkv, d = e.hq, e.hkv, e.d
    freqs, magnitude = pa.pa_rope_frequencies(d, 10000.0)
    rope = pa.pa_rope_create(d, d, pa.PA_ROPE_HALF, freqs, magnitude)
    for step in range(3):
        nodes = e.rng.integers(1, 16, e.batch)
        start = np.concatenate([[0], np.cumsum(nodes)])
        parents = np.concatenate([np.maximum(np.arange(m) - e.rng.integers(1, 4, m), -1) for m in nodes])
        paths = [[oracle.path(parents[start[b]:start[b + 1]], i) for i in range(nodes[b])] for b in range(e.batch)]
        depth = np.concatenate([[e.ctx[b] + len(p) - 1 for p in paths[b]] for b in range(e.batch)])
        total = int(start[-1])
        raw = bits(e.rng, (total, hq + 2 * hkv, d))
        rows = dev16(raw)
        stride, base = (hq + 2 * hkv) * d, rows.data_ptr()
        table, ctx = dev32(e.table), dev32(e.ctx + nodes)
        q = torch.zeros((total, hq, d), dtype=torch.int16, device=DEV)
        pa.paged_attn_rope_append(e.pool, rope, base, stride, hq, None, base + 2 * hq * d, stride, None,
                                  base + 2 * (hq + hkv) * d, stride, 0.0, pa.PA_BF16, dev32(depth), dev32(start), total,
                                  table, e.width, ctx, e.batch, q)
        size = pa.paged_attn_tree_workspace_size(e.pool, e.batch, hq, e.top, 16)
        ws, out = torch.empty(size + 16, dtype=torch.uint8, device=DEV), torch.zeros_like(q)
        pa.paged_attn_extend_tree(e.pool, q, dev32(start), total, dev32(parents), table, e.width, ctx, e.batch, hq,
                                  d ** -0.5, 0.0, e.top, 16, ws, size, out)
        accepted = [paths[b][e.rng.integers(nodes[b])][:e.rng.integers(0, 5)] for b in range(e.batch)]
        kept = np.full((e.batch, 16), -1)
        for b, x in enumerate(accepted):
            kept[b, :len(x)] = x
        lens = torch.zeros(e.batch, dtype=torch.int32, device=DEV)
        pa.paged_attn_compact(e.pool, table, e.width, None, 0, dev32(e.ctx), ctx, e.batch, e.top, dev32(kept), 16,
                              dev32([len(x) for x in accepted]), None, None, 0, lens)
        torch.cuda.synchronize()
        # the same on the host: the rotated rows come back in q and the pool
        x = bf16_to_f64(raw)
        turned = head_rows(x[:, hq:hq + hkv], None, 0.0, depth, freqs, magnitude, False)
        qt = bf16_to_f64(u16(q))
        assert np.abs(qt - head_rows(x[:, :hq], None, 0.0, depth, freqs, magnitude, False)).max() < 0.04
        got = u16(out)
        for b in range(e.batch):
            n = int(e.ctx[b])
            a = slice(start[b], start[b + 1])
            drafted = [raw[a, hq:hq + hkv], raw[a, hq + hkv:]]
            e.rows[b] = [np.concatenate([e.rows[b][i], drafted[i]]) for i in range(2)]
            # keys: as the pool holds them (rounded once from the oracle's), those that were moved among the kept ones
            kept_keys = u16(e.k)[e.table[b, (n + np.arange(len(accepted[b]))) // 16], :, (n + np.arange(len(accepted[b]))) % 16]
            assert np.abs(bf16_to_f64(kept_keys) - turned[a][accepted[b]]).max(initial=0.0) < 0.04
            exact = turned[a]
            f = exact.astype(np.float32).view(np.uint32)
            e.rows[b][0][n:] = ((f + 0x7FFF + ((f >> 16) & 1)) >> 16).astype(np.uint16)
            for i in range(nodes[b]):
                t = list(range(n)) + [n + j for j in paths[b][i]]
                # a key's rounding may fall to the other side here: a step of bf16 in it, 2^-8 of |k| |q| scale in a score
                close(got[start[b] + i], e.attention(qt[start[b] + i], b, t), 5.0, 40.0 + 2.0 ** -8 * 40.0 * 1e6 / 64)
            stay = np.concatenate([np.arange(n), n + np.array(accepted[b], int)]).astype(int)
            e.rows[b] = [r[stay] for r in e.rows[b]]
            e.rows[b][0][n:] = kept_keys
        e.ctx = e.ctx + [len(x) for x in accepted]
        assert lens.tolist() == e.ctx.tolist()
        for (k, v), (hk, hv) in zip(e.host_rows(), e.rows):
            assert np.array_equal(k, hk) and np.array_equal(v, hv)


def test_eviction_and_sparse_steps():
    """Weights over some steps, a cut to fresh blocks, the old ones released, bounds of what stays, sparse steps."""
    print("[gpu case] eviction flow", flush=True)
    e = Engine(2, [300, 700, 90, 511], 40)
    hq, hkv, d, keep, recent = e.hq, e.hkv, e.d, 256, 30
    totals = torch.zeros((e.batch, e.top), device=DEV)
    want = [np.zeros(e.top) for _ in range(e.batch)]
    table = dev32(e.table)
    size = pa.paged_attn_weights_workspace_size(e.pool, e.batch, hq, e.top)
    ws = torch.empty(size + 16, dtype=torch.uint8, device=DEV)

    def append():
        k, v = bits(e.rng, (2, e.batch, hkv, d))
        e.ctx = e.ctx + 1
        pa.paged_attn_append_kv(e.pool, dev16(k), dev16(v), table, e.width, dev32(e.ctx), e.batch)
        for b in range(e.batch):
            e.rows[b] = [np.concatenate([e.rows[b][0], k[b:b + 1]]), np.concatenate([e.rows[b][1], v[b:b + 1]])]
        return bits(e.rng, (e.batch, hq, d))

    for _ in range(3):
        q = append()
        out = torch.zeros((e.batch, hq, d), dtype=torch.int16, device=DEV)
        pa.paged_attn_decode_weights(e.pool, dev16(q), table, e.width, dev32(e.ctx), e.batch, hq, d ** -0.5, e.top, 0.9,
                                     totals, totals, e.top, ws, size, out)
        torch.cuda.synchronize()
        for b, n in enumerate(e.ctx):
            close(u16(out)[b], e.attention(bf16_to_f64(q[b]), b, np.arange(n)), 5.0)
            g = hq // hkv
            k = bf16_to_f64(e.rows[b][0])
            w = sum(oracle.rows_over(bf16_to_f64(q[b, i * g:(i + 1) * g]), k[:, i], k[:, i], d ** -0.5)[1].sum(0) for i in range(hkv))
            want[b][:n] = want[b][:n] * np.float64(np.float32(0.9)) + w
        got = totals.cpu().numpy().astype(np.float64)
        for b, n in enumerate(e.ctx):
            assert (np.abs(got[b] - want[b]) <= want[b] * 3 * (1e-4 + 20 * 2.0 ** -23)).all()
    # the cut: shared prompts of 16 tokens stay where they are
    first = np.full(e.batch, 16)
    kept = torch.zeros((e.batch, keep), dtype=torch.int32, device=DEV)
    lens, new = (torch.zeros(e.batch, dtype=torch.int32, device=DEV) for _ in range(2))
    old = e.table.copy()
    fresh = np.array([np.concatenate([old[b, :1], pa.kv_pool_alloc(e.pool, e.width - 1)]) for b in range(e.batch)], np.int32)
    before = totals.clone()
    pa.paged_attn_keep_heaviest(totals, e.top, dev32(first), dev32(e.ctx), e.batch, e.top, recent, keep, kept, keep, lens)
    pa.paged_attn_compact(e.pool, table, e.width, dev32(fresh), e.width, dev32(first), dev32(e.ctx), e.batch, e.top, kept,
                          keep, lens, totals, totals, e.top, new)
    torch.cuda.synchronize()
    for b in range(e.batch):
        row = before[b].cpu().numpy()
        stay = oracle.keep_heaviest(row[:e.ctx[b]], 16, recent, keep)
        assert kept[b, :len(stay)].tolist() == stay and int(lens[b]) == len(stay)
        t = np.concatenate([np.arange(16), 16 + np.array(stay)])
        e.rows[b] = [x[t] for x in e.rows[b]]
        assert np.array_equal(totals[b, :len(t)].cpu().numpy(), row[t]) and (totals[b, len(t):] == 0).all()
        pa.kv_pool_release(e.pool, [int(i) for i in old[b, 1:]])
    e.table, e.ctx = fresh, new.cpu().numpy().astype(np.int64)
    assert e.ctx.tolist() == [256, 256, 93, 256]
    for (k, v), (hk, hv) in zip(e.host_rows(), e.rows):
        assert np.array_equal(k, hk) and np.array_equal(v, hv)
    # sparse steps: bounds of all that stays, then of each step's newest block
    table = dev32(e.table)
    bounds = torch.zeros((e.blocks, hkv, 2, d), dtype=torch.int16, device=DEV)
    pa.paged_attn_block_bounds(e.pool, bounds, table, e.width, None, dev32(e.ctx), e.batch, e.top, e.top)
    most = 9
    picked = torch.zeros((e.batch, hkv, most), dtype=torch.int32, device=DEV)
    size = max(pa.paged_attn_select_workspace_size(e.pool, e.batch, e.top, most),
               pa.paged_attn_selected_workspace_size(e.pool, e.batch, hq, most))
    ws = torch.empty(size + 16, dtype=torch.uint8, device=DEV)
    for _ in range(20):
        q = append()
        ctx, qd = dev32(e.ctx), dev16(q)
        out = torch.zeros((e.batch, hq, d), dtype=torch.int16, device=DEV)
        pa.paged_attn_block_bounds(e.pool, bounds, table, e.width, None, ctx, e.batch, e.top, 1)
        pa.paged_attn_select_blocks(e.pool, qd, bounds, table, e.width, ctx, e.batch, hq, e.top, 1, 2, most, ws, size, picked)
        pa.paged_attn_decode_selected(e.pool, qd, table, e.width, ctx, e.batch, hq, d ** -0.5, e.top, picked, most, ws, size,
                                      out)
        torch.cuda.synchronize()
        for b, n in enumerate(e.ctx):
            x, g = bf16_to_f64(q[b]), hq // hkv
            ref = np.zeros((hq, d))
            for i in range(hkv):
                keys, heads = bf16_to_f64(e.rows[b][0][:, i]), slice(i * g, (i + 1) * g)
                scores = [np.maximum(x[heads] * lo, x[heads] * hi).sum() for lo, hi in
                          (oracle.block_bounds(keys[j:j + 16]) for j in range(0, n, 16))]
                chosen = oracle.select_blocks(scores, 1, 2, most)
                assert picked[b, i, :len(chosen)].tolist() == chosen
                t = [t for j in chosen for t in range(16 * j, min(n, 16 * j + 16))]
                ref[heads] = oracle.rows_over(x[heads], keys[t], bf16_to_f64(e.rows[b][1][t, i]), d ** -0.5)[0]
            close(u16(out)[b], ref, 5.0)


def cases():
    """Each operator's call on inputs of its own, and what it writes."""
    tree = Tree(3, **TREES["long"])
    tree.run()
    small = Tree(4, **TREES["ragged"])
    small.run()
    sparse = Sparse(5, **SPARSE["ragged"])
    sparse.setup()

    def steps(stream=None):
        sparse.bound(stream=stream)
        sparse.select(stream=stream)
        sparse.attend(stream=stream)
    steps()
    weights = Weights(6, chunk=[1, 1], **WEIGHTS["long"])
    weights.go()
    move = Move(7, [700, 60, 300], 4, 128, 0.6, fresh=True)
    move.run(totals="apart", alias=False)
    t = sparse.t
    return [(tree.call, [tree.out]), (small.call, [small.out]), (steps, [t["bounds"], t["picked"], t["out"]]),
            (weights.call, [weights.out, weights.after]),
            (move.call, [move.t["k"], move.t["v"], move.t["after"], move.t["new"]])]


def test_captured_into_a_graph():
    """Replays give what the eager calls gave, with other work between them."""
    print("[gpu case] tokens graph", flush=True)
    every = cases()
    torch.cuda.synchronize()
    want = [[x.clone() for x in outs] for _, outs in every]
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for call, _ in every:
            call(stream=torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        for _, outs in every[:-1]:
            for x in outs:
                x.fill_(i)
        if i == 0:
            every[3][1][1].fill_(-7.0)
        every[3][1][1][:] = want[3][1].where(want[3][1] == -7.0, torch.full_like(want[3][1], float(i)))
        x = torch.randn(1000, 1000, device=DEV)
        (x @ x).sum()
        torch.cuda.synchronize()
        # rows that the calls leave alone: as they were
        every[0][1][0][:], every[1][1][0][:] = 0x4242, 0x4242
        every[2][1][0][:] = 0x4242
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for (_, outs), ref in zip(every, want):
            for a, b in zip(outs, ref):
                assert torch.equal(a, b)


def test_two_streams_at_once():
    """Each call has its workspace: two of them side by side give the same bits."""
    print("[gpu case] tokens on two streams", flush=True)
    one, two = cases(), cases()
    torch.cuda.synchronize()
    want = [[x.clone() for x in outs] for _, outs in one]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        for i in range(len(one)):
            one[i][0](stream=a.cuda_stream)
            two[-1 - i][0](stream=b.cuda_stream)
    torch.cuda.synchronize()
    for every in (one, two):
        for (_, outs), ref in zip(every, want):
            for x, y in zip(outs, ref):
                assert torch.equal(x, y)


@pytest.mark.parametrize("name", ["groups_of_four", "groups_of_eight", "one_long_64"])
def test_shared_blocks_change_no_bit(name):
    """Blocks that the allocator knows as shared are loaded with another cache policy."""
    print(f"[gpu case] tokens over shared blocks {name}", flush=True)
    kw = WEIGHTS[name]
    w = Weights(8, chunk=[1] * len(kw["ctx"]), **kw)
    w.go()
    s = Sparse(9, exact=False, first=1, last=1, most=20, **kw)
    s.setup()
    s.bound()
    s.select()
    s.attend()
    torch.cuda.synchronize()
    want = [x.clone() for x in (w.out, w.after, s.t["out"])]
    for c in (w, s):
        pa.kv_pool_claim(c.pool, [0])
        pa.kv_pool_retain(c.pool, [0])
        assert pa.kv_pool_num_shared(c.pool) == 1
    w.call()
    s.attend()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, (w.out, w.after, s.t["out"])))


def test_beyond_4_gib():
    """Blocks, bounds and moves at offsets that 32 bits do not hold."""
    print("[gpu case] tokens beyond 4 GiB", flush=True)
    hkv, hq, d, blocks = 8, 32, 128, 150000                   # 4.9 GB a pool
    k, v = (torch.zeros((blocks, hkv, 16, d), dtype=torch.int16, device=DEV) for _ in range(2))
    bounds = torch.zeros((blocks, hkv, 2, d), dtype=torch.int16, device=DEV)
    pool = pa.kv_pool_create(blocks, 16, hkv, d, k, v)
    rng = np.random.default_rng(1)
    n = 600
    ids = [blocks - 1 - 7 * j if j % 2 else 5 * j for j in range(38)]
    fresh = [blocks - 3 - 7 * j if j % 3 else 5 * j + 1 for j in range(38)]
    rows = [bits(rng, (38, hkv, 16, d)) for _ in range(2)]
    for pool_t, x in ((k, rows[0]), (v, rows[1])):
        pool_t[torch.tensor(ids, device=DEV)] = torch.from_numpy(x.view(np.int16)).to(DEV)
    q = bits(rng, (1, hq, d))
    table, to, ctx, qd = dev32([ids]), dev32([fresh]), dev32([n]), dev16(q)
    pa.paged_attn_block_bounds(pool, bounds, table, 38, None, ctx, 1, n, n)
    most = 12
    picked = torch.zeros((1, hkv, most), dtype=torch.int32, device=DEV)
    out, tree, plain = (torch.zeros((1, hq, d), dtype=torch.int16, device=DEV) for _ in range(3))
    size = 1 << 22
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    pa.paged_attn_select_blocks(pool, qd, bounds, table, 38, ctx, 1, hq, n, 1, 1, most, ws, size, picked)
    pa.paged_attn_decode_selected(pool, qd, table, 38, ctx, 1, hq, d ** -0.5, n, picked, most, ws, size, out)
    pa.paged_attn_extend_tree(pool, qd, dev32([0, 1]), 1, dev32([-1]), table, 38, ctx, 1, hq, d ** -0.5, 0.0, n, 1, ws, size,
                              tree)
    totals = torch.zeros((1, n), device=DEV)
    pa.paged_attn_decode_weights(pool, qd, table, 38, ctx, 1, hq, d ** -0.5, n, 1.0, totals, totals, n, ws, size, plain)
    torch.cuda.synchronize()
    logical = [x.transpose(0, 2, 1, 3).reshape(-1, hkv, d)[:n] for x in rows]
    kf, vf, x = bf16_to_f64(logical[0]), bf16_to_f64(logical[1]), bf16_to_f64(q[0])
    for g in range(hkv):
        h = slice(4 * g, 4 * g + 4)
        scores = [np.maximum(x[h] * lo, x[h] * hi).sum() for lo, hi in (oracle.block_bounds(kf[j:j + 16, g]) for j in range(0, n, 16))]
        chosen = oracle.select_blocks(scores, 1, 1, most)
        assert picked[0, g].tolist() == chosen
        t = [t for j in chosen for t in range(16 * j, min(n, 16 * j + 16))]
        close(u16(out)[0, h], oracle.rows_over(x[h], kf[t, g], vf[t, g], d ** -0.5)[0], 5.0)
        ref = oracle.rows_over(x[h], kf[:, g], vf[:, g], d ** -0.5)[0]
        close(u16(tree)[0, h], ref, 5.0)
        close(u16(plain)[0, h], ref, 5.0)
    kept = sorted(rng.choice(n, 300, replace=False).tolist())
    pa.paged_attn_compact(pool, table, 38, to, 38, None, ctx, 1, n, dev32([kept]), 300, dev32([300]), None, None, 0, None)
    torch.cuda.synchronize()
    for pool_t, x in ((k, logical[0]), (v, logical[1])):
        got = u16(pool_t[torch.tensor(fresh, device=DEV)].transpose(1, 2).reshape(-1, hkv, d))
        assert np.array_equal(got[:300], x[kept])
