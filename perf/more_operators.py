"""The operators that choose tokens of a paged context, as cases to prepare, run, price and check:

  kind "tree"     attention of each sequence's tree of drafted tokens over its resident context and their ancestors
       "commit"   a step's drafted rows written into the cache, and the accepted path's moved behind the resident ones
       "sparse"   one new token per sequence over the blocks that the bounds of their keys choose: the bounds of the
                  newest block, the choice, the attention
       "weights"  one new token per sequence, its attention weights added to running totals per resident token
       "evict"    the tokens with the smallest totals leave the cache: the choice, and the kept ones' move to fresh blocks

A case is a dict of plain values:

  hq, hkv, d     query heads, KV heads, head_dim
  batch          sequences
  shared         tokens that all sequences share as the same blocks
  lo, hi         each sequence's own resident tokens, spread evenly over [lo, hi], or lognormal (mean 1500, sigma 0.8)
                 clipped to it
  nodes_lo, nodes_hi  tree and commit: drafted tokens per sequence
  reach          how near a drafted token's parent is: among the `reach` tokens before it (1: a chain)
  pad            rows behind the last sequence's
  cap            the scores' cap (0: none), tree
  blocks         sparse: blocks that a token attends to, of them `sink` first ones and `local` last ones always
  decay          weights: factor of the totals before
  keep, recent   evict: tokens that stay of a sequence, of them the last `recent` always (and the shared ones)

The lengths of a case are fixed; a seed draws their order, the blocks' places in the pool, the trees and the values.
"""
import math
from statistics import NormalDist

import numpy as np
import torch

own = False

BLOCK = 16
DEVICE = "cuda:0"


def _case(name, kind, hq, hkv, d, **kw):
    c = dict(name=name, kind=kind, hq=hq, hkv=hkv, d=d, batch=1, shared=0, lo=0, hi=0, lengths="even", nodes_lo=1,
             nodes_hi=1, reach=4, pad=0, cap=0.0, blocks=0, sink=1, local=2, decay=1.0, keep=0, recent=0)
    c.update(kw)
    return c


def listed():
    return [
        # A small model's step with a few drafted tokens for each of four calls: launch-bound.
        _case("tree_tiny", "tree", 8, 2, 64, batch=4, lo=100, hi=300, nodes_lo=8, nodes_hi=8),
        # A stage's batch over its schema prompt, a tree of 13 to 32 drafts for each call.
        _case("tree_stage", "tree", 32, 8, 128, batch=64, shared=2048, lo=64, hi=512, nodes_lo=13, nodes_hi=32, pad=9),
        # One call alone over a long context with a wide tree, capped scores.
        _case("tree_single_long", "tree", 64, 8, 128, batch=1, lo=30011, hi=30011, nodes_lo=61, nodes_hi=61, reach=16,
              cap=30.0),
        # The cache after the small model's step.
        _case("commit_tiny", "commit", 8, 2, 64, batch=4, lo=100, hi=300, nodes_lo=8, nodes_hi=8),
        # The cache after a step of one engine pool of mixed lengths, large trees.
        _case("commit_pool", "commit", 32, 8, 128, batch=256, lo=64, hi=4096, lengths="lognormal", nodes_lo=17,
              nodes_hi=64),
        # The small model's batch, some contexts shorter than what is attended to.
        _case("sparse_tiny", "sparse", 8, 2, 64, batch=4, lo=90, hi=1300, blocks=16),
        # A batch over long contexts, 2048 tokens attended to of each.
        _case("sparse_batch", "sparse", 32, 8, 128, batch=64, lo=4097, hi=28672, blocks=128, local=8),
        # One call alone over a very long context.
        _case("sparse_single_long", "sparse", 64, 8, 128, batch=1, lo=131003, hi=131003, blocks=256, sink=4, local=16),
        # One call alone over a long context whose tokens' weights are kept.
        _case("weights_single", "weights", 64, 8, 128, batch=1, lo=30011, hi=30011),
        # One engine pool of mixed lengths, the weights of older steps fading.
        _case("weights_pool", "weights", 32, 8, 128, batch=128, lo=64, hi=8192, lengths="lognormal", decay=0.98),
        # The small model's contexts cut to a budget, one of them shorter than it.
        _case("evict_tiny", "evict", 8, 2, 64, batch=4, lo=200, hi=700, keep=256, recent=32),
        # Long contexts behind a shared prompt cut to a quarter or so.
        _case("evict_batch", "evict", 32, 8, 128, batch=64, shared=1024, lo=3001, hi=15000, keep=4096, recent=512),
    ]


HEADS = [(32, 8, 128), (64, 8, 128), (16, 16, 128), (16, 8, 128), (28, 4, 128), (8, 1, 128), (40, 5, 128), (16, 1, 128),
         (8, 2, 64), (32, 4, 64), (24, 3, 64), (12, 12, 64), (15, 5, 64)]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _cost(c):
    w = work(c)
    return w["bytes"] / 5e12 + w["flops"] / 5e14


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        c = _draw_one(rng)
        s = _structure(c, 0)
        tokens = c["batch"] * s["table"].shape[1] * BLOCK
        rows = int(s["nodes"].max()) if c["kind"] == "tree" else 1
        if tokens * c["hq"] * rows > 2.1e9 or tokens * c["hkv"] * c["d"] > 2.2e9:
            continue   # the plain form's scores and gathered tokens
        if _cost(c) <= most[c["kind"]]:
            return c


def _draw_one(rng):
    kind = rng.choice(["tree", "tree", "commit", "sparse", "sparse", "weights", "evict"])
    hq, hkv, d = rng.choice(HEADS)
    c = _case("", kind, hq, hkv, d)
    del c["name"]
    c["batch"] = _logint(rng, 1, 256)
    c["hi"] = _logint(rng, 1, 131072 if c["batch"] == 1 else 32768)
    c["lo"] = rng.choice([c["hi"], _logint(rng, 1, c["hi"])])
    if kind in ("tree", "commit"):
        c["nodes_hi"] = _logint(rng, 1, 256)
        c["nodes_lo"] = rng.choice([c["nodes_hi"], _logint(rng, 1, c["nodes_hi"])])
        c["reach"] = rng.choice([1, 2, 4, 8, 64])
        c["pad"] = rng.choice([0, rng.randint(1, 64)])
        c["shared"] = BLOCK * rng.choice([0, rng.randint(1, 128)])
        c["cap"] = rng.choice([0.0, 0.0, 30.0]) if kind == "tree" else 0.0
        if rng.random() < 0.1:
            c["lo"] = 0
    if kind == "sparse":
        c["sink"], c["local"] = rng.randint(0, 4), rng.randint(1, 16)
        c["blocks"] = c["sink"] + c["local"] + _logint(rng, 1, 256)
    if kind == "weights":
        c["decay"] = rng.choice([1.0, 0.9, 0.5])
    if kind == "evict":
        c["shared"] = BLOCK * rng.choice([0, 0, rng.randint(1, 64)])
        c["recent"] = rng.choice([0, _logint(rng, 1, 256)])
        c["keep"] = c["shared"] + c["recent"] + _logint(rng, 1, 8192)
    return c


# --------------------------------------------------------------------------
# lengths, tables, trees and work
# --------------------------------------------------------------------------

def _spread(n, lo, hi, how):
    u = (np.arange(n) + 0.5) / max(n, 1)
    if how == "lognormal":
        mu = math.log(1500.0) - 0.8 * 0.8 / 2
        x = np.array([math.exp(mu + 0.8 * NormalDist().inv_cdf(v)) for v in u])
    else:
        x = lo + u * (hi - lo)
    return np.clip(np.rint(x), lo, hi).astype(np.int64)


def _structure(c, seed):
    """Lengths in the seed's order, block tables over a shuffled pool 1.2 times as large as needed, trees."""
    rng = np.random.default_rng(seed)
    n = c["batch"]
    old = rng.permutation(_spread(n, c["lo"], c["hi"], c["lengths"]))
    nodes = np.zeros(n, np.int64)
    if c["kind"] in ("tree", "commit"):
        nodes = rng.permutation(_spread(n, c["nodes_lo"], c["nodes_hi"], "even"))
    ctx = c["shared"] + old + nodes
    n_pre = c["shared"] // BLOCK
    tail = (ctx - c["shared"] + BLOCK - 1) // BLOCK
    fresh = np.zeros(n, np.int64)
    if c["kind"] == "evict":
        fresh = (np.minimum(ctx, c["keep"]) - c["shared"] + BLOCK - 1) // BLOCK
    # (by the lengths alone, not by which trees they meet)
    needed = n_pre + int(((old + BLOCK - 1) // BLOCK + (nodes + BLOCK - 1) // BLOCK).sum()) + int(fresh.sum())
    blocks = max(1, math.ceil(1.2 * needed))
    ids = rng.permutation(blocks)
    at = n_pre

    def tables(count):
        nonlocal at
        t = np.zeros((n, max(1, int(n_pre + count.max()))), np.int32)
        t[:, :n_pre] = ids[:n_pre]
        for b in range(n):
            t[b, n_pre:n_pre + count[b]] = ids[at:at + count[b]]
            at += count[b]
        return t

    table = tables(tail)
    to = tables(fresh) if c["kind"] == "evict" else None
    start = np.concatenate([[0], np.cumsum(nodes)])
    # a node's parent: one of the `reach` before it, or the resident context (-1); the trees are wide at the root
    node = np.arange(start[-1]) - np.repeat(start[:-1], nodes)
    back = 1 + np.floor(rng.random(start[-1]) * c["reach"]).astype(np.int64)
    parents = np.maximum(node - back, -1)
    return dict(ctx=ctx, nodes=nodes, table=table, to=to, blocks=blocks, start=start, parents=parents, node=node)


def _depth(s):
    """Ancestors of each node, itself included."""
    up = np.where(s["parents"] < 0, -1, np.arange(len(s["node"])) - s["node"] + s["parents"])
    depth = np.ones(len(up), np.int64)
    for i in np.flatnonzero(up >= 0):
        depth[i] = depth[up[i]] + 1
    return depth


def _accepted(c, s, seed):
    """Nodes of a path from the context to one of each tree's nodes, in their order, and their number."""
    rng = np.random.default_rng(seed + 1)
    kept = np.full((c["batch"], max(1, int(s["nodes"].max()))), -1, np.int32)
    count = np.zeros(c["batch"], np.int32)
    for b in range(c["batch"]):
        path, i = [], int(rng.integers(-1, s["nodes"][b]))
        while i >= 0:
            path.append(i)
            i = int(s["parents"][s["start"][b] + i])
        count[b] = len(path)
        kept[b, :len(path)] = path[::-1]
    return kept, count


def work(c):
    s = _structure(c, 0)
    kv, hq, d, n = 2 * 2 * c["hkv"] * c["d"], c["hq"], c["d"], c["batch"]
    own_tokens = int((s["ctx"] - c["shared"]).sum())
    if c["kind"] == "tree":
        rows = int(s["start"][-1])
        seen = int(((s["ctx"] - s["nodes"]) * s["nodes"]).sum() + _depth(s).sum())
        return {"bytes": (c["shared"] + own_tokens) * kv + 4 * rows * hq * d + 4 * s["table"].size + 4 * rows,
                "flops": 4 * hq * d * seen}
    if c["kind"] == "commit":
        rows = int(s["start"][-1])
        kept, count = _accepted(c, s, 0)
        moved = int((kept > np.arange(kept.shape[1])).sum())
        return {"bytes": 2 * kv * (rows + moved) + 4 * int(count.sum()) + 8 * n, "flops": 0}
    if c["kind"] == "sparse":
        blocks = (s["ctx"] + BLOCK - 1) // BLOCK
        scored = int(np.where(blocks > c["blocks"], blocks - c["sink"] - c["local"], 0).sum())
        tokens = int(np.minimum(s["ctx"], c["blocks"] * BLOCK).sum())
        return {"bytes": scored * kv + n * kv * (BLOCK // 2 + 1) + tokens * kv + 4 * n * hq * d
                + 4 * int(np.minimum(blocks, c["blocks"]).sum()) * c["hkv"],
                "flops": 4 * scored * c["hkv"] * d + 4 * tokens * hq * d}
    if c["kind"] == "weights":
        tokens = int(s["ctx"].sum())
        return {"bytes": tokens * (kv + 8) + 4 * n * hq * d + 4 * s["table"].size, "flops": 4 * tokens * hq * d}
    stay = int(np.minimum(s["ctx"], c["keep"]).sum()) - n * c["shared"]
    return {"bytes": stay * (2 * kv + 4 + 12) + 4 * own_tokens + 4 * n * c["shared"] * 2, "flops": 0}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def prepare(case, seed):
    c, hq, hkv, d, n = case, case["hq"], case["hkv"], case["d"], case["batch"]
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 7919 + 17)

    def normal(shape, dtype, scale=1.0):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).mul_(scale).to(dtype)

    s = _structure(c, seed)
    st = {"c": c, "blocks": s["blocks"], "rows": int(s["start"][-1]), "total": int(s["start"][-1]) + c["pad"],
          "max_ctx": int(s["ctx"].max()), "max_nodes": int(s["nodes"].max())}
    for name in ("ctx", "table", "to", "start", "parents"):
        st[name] = None if s[name] is None else torch.tensor(s[name], dtype=torch.int32, device=DEVICE)
    shape = (s["blocks"], hkv, BLOCK, d)
    k = torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)
    if c["kind"] == "sparse":   # neighbouring tokens resemble each other
        k.mul_(0.8).add_(torch.randn((s["blocks"], hkv, 1, d), generator=gen, device=DEVICE), alpha=0.6)
    st["k_pool"] = k.to(torch.bfloat16)
    del k
    st["v_pool"] = normal(shape, torch.bfloat16)
    if c["kind"] == "tree":
        st["q"] = normal((st["total"], hq, d), torch.bfloat16, 4.0 if c["cap"] else 1.0)
        st["out"] = torch.zeros((st["total"], hq, d), dtype=torch.bfloat16, device=DEVICE)
    if c["kind"] in ("sparse", "weights"):
        st["q"] = normal((n, hq, d), torch.bfloat16, 2.0)
        st["out"] = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=DEVICE)
    if c["kind"] == "commit":
        st["rows_kv"] = normal((st["total"], 2, hkv, d), torch.bfloat16)
        kept, count = _accepted(c, s, seed)
        st["kept"] = torch.tensor(kept, device=DEVICE)
        st["count"] = torch.tensor(count, device=DEVICE)
        st["first"] = torch.tensor(s["ctx"] - s["nodes"], dtype=torch.int32, device=DEVICE)
        st["lens"] = torch.zeros(n, dtype=torch.int32, device=DEVICE)
    if c["kind"] == "sparse":
        # bounds as the steps before left them: those of full blocks
        st["bounds"] = torch.stack([st["k_pool"].amin(2), st["k_pool"].amax(2)], 2)
        st["picked"] = torch.zeros((n, hkv, c["blocks"]), dtype=torch.int32, device=DEVICE)
    if c["kind"] in ("weights", "evict"):
        # what many steps added: few tokens have most of it, some have none
        u = torch.rand((n, st["max_ctx"]), generator=gen, device=DEVICE)
        st["totals"] = torch.where(u < 0.02, 0.0, u.clamp(min=1e-6).pow(6).mul(4.0))
        st["totals_out"] = torch.zeros_like(st["totals"])
    if c["kind"] == "evict":
        st["first"] = torch.full((n,), c["shared"], dtype=torch.int32, device=DEVICE)
        st["kept"] = torch.zeros((n, min(c["keep"], st["max_ctx"])), dtype=torch.int32, device=DEVICE)
        st["count"] = torch.zeros(n, dtype=torch.int32, device=DEVICE)
        st["lens"] = torch.zeros(n, dtype=torch.int32, device=DEVICE)
    if own:
        _prepare_own(st)
    return st


def _prepare_own(st):
    """The handles and the workspace that a program keeps beside its cache."""
    from paper_2510_14126_amd import binding as pa
    c = st["c"]
    st["pool"] = pa.kv_pool_create(st["blocks"], BLOCK, c["hkv"], c["d"], st["k_pool"], st["v_pool"])
    if c["kind"] == "commit":
        st["rope"] = pa.pa_rope_create(c["d"], 0, pa.PA_ROPE_HALF, [], 1.0)
    size = 0
    if c["kind"] == "tree":
        size = pa.paged_attn_tree_workspace_size(st["pool"], c["batch"], c["hq"], st["max_ctx"], st["max_nodes"])
    if c["kind"] == "sparse":
        size = max(pa.paged_attn_select_workspace_size(st["pool"], c["batch"], st["max_ctx"], c["blocks"]),
                   pa.paged_attn_selected_workspace_size(st["pool"], c["batch"], c["hq"], c["blocks"]))
    if c["kind"] == "weights":
        size = pa.paged_attn_weights_workspace_size(st["pool"], c["batch"], c["hq"], st["max_ctx"])
    st["workspace"] = torch.empty(max(size, 1), dtype=torch.uint8, device=DEVICE)
    st["workspace_bytes"] = size


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(st):
    if own:
        return _run_own(st)
    return {"tree": _tree_plain, "commit": _commit_plain, "sparse": _sparse_plain, "weights": _weights_plain,
            "evict": _evict_plain}[st["c"]["kind"]](st)


def _gathered(st, table):
    """K as [n][hkv][d][tokens] and V as [n][hkv][tokens][d] of the tables' blocks [n][blocks], in 32 bits."""
    c = st["c"]
    n, tokens = table.shape[0], table.shape[1] * BLOCK
    k = st["k_pool"][table].permute(0, 2, 4, 1, 3).reshape(n, c["hkv"], c["d"], tokens).float()
    v = st["v_pool"][table].permute(0, 2, 1, 3, 4).reshape(n, c["hkv"], tokens, c["d"]).float()
    return k, v


def _softmax(s):
    """Weights of scores (in place), and 1 over their sum: 0 where nothing is seen."""
    peak = s.amax(-1, keepdim=True)
    w = s.sub_(torch.where(peak == -math.inf, 0.0, peak)).exp_()
    total = w.sum(-1, keepdim=True)
    return w, torch.where(total > 0, 1.0 / total, 0.0)


def _tree_plain(st):
    c = st["c"]
    n, hq, hkv, d, most = c["batch"], c["hq"], c["hkv"], c["d"], st["max_nodes"]
    group = hq // hkv
    row = torch.arange(st["rows"], device=DEVICE, dtype=torch.int32)
    b = torch.searchsorted(st["start"], row, right=True) - 1
    i = row - st["start"][b]
    first = st["ctx"] - (st["start"][1:] - st["start"][:-1])
    # one step to the parent, then every path by doubling
    up = torch.zeros((n, most, most), device=DEVICE)
    up[b, i, st["parents"].clamp(min=0)] = (st["parents"] >= 0).float()
    seen = up + torch.eye(most, device=DEVICE)
    for _ in range(max(1, most - 1).bit_length()):
        seen = torch.matmul(seen, seen).clamp_(max=1.0)
    k, v = _gathered(st, st["table"].long())
    tokens = k.shape[-1]
    t = torch.arange(tokens, device=DEVICE)
    node = t - first[:, None]                                        # [n][tokens]
    drafted = (node >= 0) & (node < most)
    mask = torch.gather(seen > 0, 2, node.clamp(0, most - 1)[:, None, :].expand(n, most, tokens)) & drafted[:, None, :]
    mask |= (node < 0)[:, None, :]
    q = torch.zeros((n, most, hkv, group, d), device=DEVICE)
    q[b, i] = st["q"][:st["rows"]].float().view(-1, hkv, group, d)
    s = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(n, hkv, most * group, d), k)
    s = s.view(n, hkv, most, group, tokens).mul_(d ** -0.5)
    if c["cap"]:
        s = s.div_(c["cap"]).tanh_().mul_(c["cap"])
    s.masked_fill_(~mask[:, None, :, None, :], -math.inf)
    w, inverse = _softmax(s)
    out = torch.matmul(w.view(n, hkv, most * group, tokens), v).view(n, hkv, most, group, d) * inverse
    st["out"][:st["rows"]] = out.permute(0, 2, 1, 3, 4)[b, i].reshape(-1, hq, d).to(torch.bfloat16)
    return {"out": st["out"]}


def _slots(table, b, t):
    return table[b, t // BLOCK].long(), t % BLOCK


def _commit_plain(st):
    row = torch.arange(st["rows"], device=DEVICE)
    b = torch.searchsorted(st["start"], row, right=True) - 1
    block, slot = _slots(st["table"], b, (st["first"] - st["start"][:-1])[b] + row)
    st["k_pool"][block, :, slot] = st["rows_kv"][:st["rows"], 0]
    st["v_pool"][block, :, slot] = st["rows_kv"][:st["rows"], 1]
    j = torch.arange(st["kept"].shape[1], device=DEVICE)
    b, j = torch.nonzero(j < st["count"][:, None], as_tuple=True)
    source = _slots(st["table"], b, (st["first"][b] + st["kept"][b, j]).long())
    goal = _slots(st["table"], b, st["first"][b] + j)
    for pool in (st["k_pool"], st["v_pool"]):
        pool[goal[0], :, goal[1]] = pool[source[0], :, source[1]]
    st["lens"].copy_(st["first"] + st["count"])
    return {"k_pool": st["k_pool"], "v_pool": st["v_pool"], "lens": st["lens"]}


def _sparse_plain(st):
    c = st["c"]
    n, hq, hkv, d, most = c["batch"], c["hq"], c["hkv"], c["d"], c["blocks"]
    ctx, b = st["ctx"].long(), torch.arange(n, device=DEVICE)
    # the newest block's bounds, of the rows that it has
    newest = st["table"][b, (ctx - 1) // BLOCK].long()
    have = (torch.arange(BLOCK, device=DEVICE) <= ((ctx - 1) % BLOCK)[:, None])[:, None, :, None]
    rows = st["k_pool"][newest].float()
    st["bounds"][newest, :, 0] = rows.masked_fill(~have, math.inf).amin(2).to(torch.bfloat16)
    st["bounds"][newest, :, 1] = rows.masked_fill(~have, -math.inf).amax(2).to(torch.bfloat16)
    # the largest score that a key within the bounds could have, over the heads of a KV head: in 64 bits, for
    # neighbouring scores decide which block is taken
    q = st["q"].double().view(n, hkv, hq // hkv, d)
    above, below = q.clamp(min=0).sum(2), q.clamp(max=0).sum(2)
    sides = st["bounds"][st["table"].long()].double()                # [n][blocks][hkv][2][d]
    score = (torch.matmul(sides[..., 1, :].permute(0, 2, 1, 3).contiguous(), above[..., None])
             + torch.matmul(sides[..., 0, :].permute(0, 2, 1, 3).contiguous(), below[..., None]))[..., 0]
    del sides
    count = ((ctx + BLOCK - 1) // BLOCK)[:, None, None]
    j = torch.arange(score.shape[2], device=DEVICE)
    always = (j < c["sink"]) | (j >= count - c["local"])
    score = score.masked_fill(always, math.inf).masked_fill(j >= count, -math.inf)
    order = torch.sort(score, dim=2, descending=True, stable=True).indices[..., :most]
    taken = torch.where(torch.arange(order.shape[2], device=DEVICE) < count, order, 1 << 30)
    taken = torch.sort(taken, dim=2).values
    there = taken < (1 << 30)
    st["picked"].fill_(-1)
    st["picked"][..., :taken.shape[2]] = torch.where(there, taken, -1)
    # attention over them
    head = torch.arange(hkv, device=DEVICE)[:, None]
    ids = st["table"].long()[b[:, None, None], torch.where(there, taken, 0)]
    k = st["k_pool"][ids, head].float().flatten(2, 3)                # [n][hkv][tokens][d]
    v = st["v_pool"][ids, head].float().flatten(2, 3)
    at = (torch.where(there, taken, 1 << 30)[..., None] * BLOCK + torch.arange(BLOCK, device=DEVICE)).flatten(2)
    s = torch.matmul(st["q"].float().view(n, hkv, hq // hkv, d), k.transpose(2, 3).contiguous()).mul_(d ** -0.5)
    s.masked_fill_((at >= ctx[:, None, None])[:, :, None, :], -math.inf)
    w, inverse = _softmax(s)
    st["out"].copy_((torch.matmul(w, v) * inverse).view(n, hq, d))
    return {"bounds": st["bounds"], "picked": st["picked"], "out": st["out"]}


def _weights_plain(st):
    c = st["c"]
    n, hq, hkv, d = c["batch"], c["hq"], c["hkv"], c["d"]
    k, v = _gathered(st, st["table"].long())
    s = torch.matmul(st["q"].float().view(n, hkv, hq // hkv, d), k).mul_(d ** -0.5)
    hidden = torch.arange(k.shape[-1], device=DEVICE) >= st["ctx"][:, None]
    s.masked_fill_(hidden[:, None, None, :], -math.inf)
    w, inverse = _softmax(s)
    st["out"].copy_((torch.matmul(w, v) * inverse).view(n, hq, d))
    added = st["totals"] * c["decay"] + (w * inverse).sum((1, 2))[:, :st["max_ctx"]]
    st["totals_out"].copy_(torch.where(hidden[:, :st["max_ctx"]], st["totals_out"], added))
    return {"out": st["out"], "totals": st["totals_out"]}


def _evict_plain(st):
    c = st["c"]
    n, ctx, first, width = c["batch"], st["ctx"].long(), c["shared"], st["kept"].shape[1]
    t = torch.arange(st["max_ctx"], device=DEVICE)
    x = st["totals"].masked_fill(t >= (ctx - c["recent"])[:, None], math.inf)
    x = x.masked_fill(t < first, math.inf).masked_fill(t >= ctx[:, None], -math.inf)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    stay = torch.zeros_like(x, dtype=torch.bool)
    stay.scatter_(1, order[:, :c["keep"]], True)
    stay &= (t >= first) & (t < ctx[:, None])
    b, at = torch.nonzero(stay, as_tuple=True)
    count = stay.sum(1)
    j = torch.arange(len(b), device=DEVICE) - (torch.cumsum(count, 0) - count)[b]
    st["kept"].fill_(-1)
    st["kept"][b, j] = (at - first).int()
    st["count"].copy_(count)
    st["lens"].copy_(first + count)
    source, goal = _slots(st["table"], b, at), _slots(st["to"], b, first + j)
    for pool in (st["k_pool"], st["v_pool"]):
        pool[goal[0], :, goal[1]] = pool[source[0], :, source[1]]
    st["totals_out"].masked_fill_(t < ctx[:, None], 0.0)
    st["totals_out"][:, :first] = st["totals"][:, :first]
    st["totals_out"][b, first + j] = st["totals"][b, at]
    return {"kept": st["kept"], "count": st["count"], "lens": st["lens"], "totals": st["totals_out"],
            "k_pool": st["k_pool"], "v_pool": st["v_pool"]}


def _run_own(st):
    from paper_2510_14126_amd import binding as pa
    c = st["c"]
    n, hq, hkv, d, width = c["batch"], c["hq"], c["hkv"], c["d"], st["table"].shape[1]
    if c["kind"] == "tree":
        pa.paged_attn_extend_tree(st["pool"], st["q"], st["start"], st["total"], st["parents"], st["table"], width,
                                  st["ctx"], n, hq, d ** -0.5, c["cap"], st["max_ctx"], st["max_nodes"],
                                  st["workspace"], st["workspace_bytes"], st["out"])
        return {"out": st["out"]}
    if c["kind"] == "commit":
        rows = st["rows_kv"].data_ptr()
        pa.paged_attn_rope_append(st["pool"], st["rope"], None, 0, 0, None, rows, 2 * hkv * d, None, rows + 2 * hkv * d,
                                  2 * hkv * d, 0.0, pa.PA_BF16, None, st["start"], st["total"], st["table"], width,
                                  st["ctx"], n, None)
        pa.paged_attn_compact(st["pool"], st["table"], width, None, 0, st["first"], st["ctx"], n, st["max_ctx"],
                              st["kept"], st["kept"].shape[1], st["count"], None, None, 0, st["lens"])
        return {"k_pool": st["k_pool"], "v_pool": st["v_pool"], "lens": st["lens"]}
    if c["kind"] == "sparse":
        pa.paged_attn_block_bounds(st["pool"], st["bounds"], st["table"], width, None, st["ctx"], n, st["max_ctx"], 1)
        pa.paged_attn_select_blocks(st["pool"], st["q"], st["bounds"], st["table"], width, st["ctx"], n, hq,
                                    st["max_ctx"], c["sink"], c["local"], c["blocks"], st["workspace"],
                                    st["workspace_bytes"], st["picked"])
        pa.paged_attn_decode_selected(st["pool"], st["q"], st["table"], width, st["ctx"], n, hq, d ** -0.5,
                                      st["max_ctx"], st["picked"], c["blocks"], st["workspace"], st["workspace_bytes"],
                                      st["out"])
        return {"bounds": st["bounds"], "picked": st["picked"], "out": st["out"]}
    if c["kind"] == "weights":
        pa.paged_attn_decode_weights(st["pool"], st["q"], st["table"], width, st["ctx"], n, hq, d ** -0.5,
                                     st["max_ctx"], c["decay"], st["totals"], st["totals_out"], st["max_ctx"],
                                     st["workspace"], st["workspace_bytes"], st["out"])
        return {"out": st["out"], "totals": st["totals_out"]}
    pa.paged_attn_keep_heaviest(st["totals"], st["max_ctx"], st["first"], st["ctx"], n, st["max_ctx"], c["recent"],
                                c["keep"], st["kept"], st["kept"].shape[1], st["count"])
    pa.paged_attn_compact(st["pool"], st["table"], width, st["to"], st["to"].shape[1], st["first"], st["ctx"], n,
                          st["max_ctx"], st["kept"], st["kept"].shape[1], st["count"], st["totals"], st["totals_out"],
                          st["max_ctx"], st["lens"])
    return {"kept": st["kept"], "count": st["count"], "lens": st["lens"], "totals": st["totals_out"],
            "k_pool": st["k_pool"], "v_pool": st["v_pool"]}


# --------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"tree": _exact_tree, "commit": _exact_commit, "sparse": _exact_sparse, "weights": _exact_weights,
            "evict": _exact_evict}[case["kind"]](st, case, _structure(case, seed), seed)


def _exact_heads(st, ids, n, q, cap=0.0, hidden=None):
    """Outputs and weights of query rows [m][hq][d] over the first n tokens of the blocks `ids`; hidden: [m][n]."""
    c = st["c"]
    hkv, d = c["hkv"], c["d"]
    k = st["k_pool"][ids].double().transpose(1, 2).reshape(-1, hkv, d)[:n].permute(1, 2, 0).contiguous()
    v = st["v_pool"][ids].double().transpose(1, 2).reshape(-1, hkv, d)[:n].transpose(0, 1).contiguous()
    m = q.shape[0]
    x = torch.bmm(q.double().view(m, hkv, -1, d).permute(1, 2, 0, 3).reshape(hkv, -1, d), k) / math.sqrt(d)
    if cap:
        x = cap * torch.tanh(x / cap)
    x = x.view(hkv, -1, m, n)
    if hidden is not None:
        x = x.masked_fill(hidden, -math.inf)
    w = torch.softmax(x, -1)
    o = torch.bmm(w.reshape(hkv, -1, n), v).view(hkv, -1, m, d)
    return o.permute(2, 0, 1, 3).reshape(m, -1, d), w


def _exact_tree(st, c, s, seed):
    out = torch.zeros((st["total"], c["hq"], c["d"]), dtype=torch.float64, device=DEVICE)
    for b in range(c["batch"]):
        a, e, n, m = int(s["start"][b]), int(s["start"][b + 1]), int(s["ctx"][b]), int(s["nodes"][b])
        hidden = np.zeros((m, n), bool)
        hidden[:, n - m:] = True
        for i in range(m):
            j = i
            while j >= 0:
                hidden[i, n - m + j] = False
                j = int(s["parents"][a + j])
        ids = st["table"][b, :(n + BLOCK - 1) // BLOCK].long()
        out[a:e] = _exact_heads(st, ids, n, st["q"][a:e], c["cap"], torch.tensor(hidden, device=DEVICE))[0]
    return {"out": out}


def _exact_commit(st, c, s, seed):
    kept, count = _accepted(c, s, seed)
    pools = [st["k_pool"], st["v_pool"]]
    for b in range(c["batch"]):
        first = int(s["ctx"][b] - s["nodes"][b])
        row = np.arange(s["nodes"][b])
        row[:count[b]] = kept[b, :count[b]]
        t = torch.arange(first, int(s["ctx"][b]), device=DEVICE)
        block = st["table"][b, t // BLOCK].long()
        row = torch.tensor(row + s["start"][b], device=DEVICE)
        for i, pool in enumerate(pools):
            pool[block, :, t % BLOCK] = st["rows_kv"][row, i]
    lens = torch.tensor(s["ctx"] - s["nodes"] + count, dtype=torch.int32, device=DEVICE)
    return {"k_pool": pools[0].double(), "v_pool": pools[1].double(), "lens": lens}


def _exact_sparse(st, c, s, seed):
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    out = torch.zeros((c["batch"], hq, d), dtype=torch.float64, device=DEVICE)
    picked = torch.full((c["batch"], hkv, c["blocks"]), -1, dtype=torch.int32, device=DEVICE)
    bounds = st["bounds"].double()
    for b in range(c["batch"]):
        n = int(s["ctx"][b])
        count = (n + BLOCK - 1) // BLOCK
        ids = st["table"][b, :count].long()
        rows = st["k_pool"][ids[-1], :, :n - (count - 1) * BLOCK].double()
        bounds[ids[-1], :, 0], bounds[ids[-1], :, 1] = rows.min(1).values, rows.max(1).values
        q = st["q"][b].double().view(hkv, hq // hkv, d)
        for g in range(hkv):
            lo, hi = bounds[ids, g, 0], bounds[ids, g, 1]
            best = torch.zeros(count, dtype=torch.float64, device=DEVICE)
            for h in range(hq // hkv):
                best += torch.maximum(q[g, h] * lo, q[g, h] * hi).sum(1)
            free = torch.arange(min(c["sink"], count), max(count - c["local"], min(c["sink"], count)), device=DEVICE)
            forced = torch.ones(count, dtype=torch.bool, device=DEVICE)
            forced[free] = False
            want = min(c["blocks"], count) - int(forced.sum())
            ranked = free[torch.sort(best[free], descending=True, stable=True).indices][:want]
            take = torch.sort(torch.cat([torch.nonzero(forced)[:, 0], ranked])).values
            picked[b, g, :len(take)] = take.int()
            t = (take[:, None] * BLOCK + torch.arange(BLOCK, device=DEVICE)).flatten()
            k = st["k_pool"][ids[take], g].double().view(-1, d)[t < n]
            v = st["v_pool"][ids[take], g].double().view(-1, d)[t < n]
            w = torch.softmax(torch.mm(q[g], k.t().contiguous()) / math.sqrt(d), -1)
            out[b, g * (hq // hkv):(g + 1) * (hq // hkv)] = torch.mm(w, v)
    return {"bounds": bounds, "picked": picked, "out": out}


def _exact_weights(st, c, s, seed):
    out = torch.zeros((c["batch"], c["hq"], c["d"]), dtype=torch.float64, device=DEVICE)
    totals = torch.zeros(st["totals"].shape, dtype=torch.float64, device=DEVICE)
    for b in range(c["batch"]):
        n = int(s["ctx"][b])
        o, w = _exact_heads(st, st["table"][b, :(n + BLOCK - 1) // BLOCK].long(), n, st["q"][b:b + 1])
        out[b] = o[0]
        totals[b, :n] = c["decay"] * st["totals"][b, :n].double() + w.sum((0, 1, 2))
    return {"out": out, "totals": totals}


def _exact_evict(st, c, s, seed):
    pools = [st["k_pool"], st["v_pool"]]
    totals = torch.zeros(st["totals"].shape, dtype=torch.float64, device=DEVICE)
    kept = torch.full(st["kept"].shape, -1, dtype=torch.int32, device=DEVICE)
    count = torch.zeros(c["batch"], dtype=torch.int32, device=DEVICE)
    f = c["shared"]
    for b in range(c["batch"]):
        n = int(s["ctx"][b])
        end = max(f, n - c["recent"])
        want = max(0, min(c["keep"], n) - f - (n - end))
        free = st["totals"][b, f:end]
        best = torch.sort(free, descending=True, stable=True).indices[:want]
        stay = torch.cat([torch.sort(best).values, torch.arange(end - f, n - f, device=DEVICE)])
        m = len(stay)
        kept[b, :m], count[b] = stay.int(), m
        totals[b, :f] = st["totals"][b, :f].double()
        totals[b, f:f + m] = st["totals"][b, f:n][stay].double()
        t, u = f + stay, torch.arange(f, f + m, device=DEVICE)
        source, goal = st["table"][b, t // BLOCK].long(), st["to"][b, u // BLOCK].long()
        for pool in pools:
            pool[goal, :, u % BLOCK] = pool[source, :, t % BLOCK]
    return {"kept": kept, "count": count, "lens": count + f, "totals": totals, "k_pool": pools[0].double(),
            "v_pool": pools[1].double()}
