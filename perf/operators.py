"""The operators around the cache's attention, as cases to prepare, run, price and check:

  kind "rope"    the rows of q and k after their projection: normed per head, rotated to their positions
       "append"  the same on a batch's chunks of new tokens (or single tokens), k and v written into the paged cache
       "decode"  attention of one new token per sequence, its scores capped by a tanh, biased by distance, or masked
       "extend"  the same for chunks of new tokens

A case is a dict of plain values:

  hq, hkv, d     query heads, KV heads, head_dim
  batch          sequences
  tokens, reach  rope: rows, and the bound of their positions
  shared         tokens that all sequences share as the same blocks
  lo, hi         each sequence's own resident tokens, spread evenly over [lo, hi], or lognormal (mean 1500,
                 sigma 0.8) clipped to it; decode: the new token included
  chunk_lo, chunk_hi  new tokens per sequence
  pad            rows behind the last sequence's
  dtype, rotary, layout, scaling, norm        of rope and append
  cap, alibi, window, doc_lo, doc_hi, prefix  of decode and extend: the scores' cap (0: none), a slope per head,
                 the tokens a row sees back (0: all), lengths of the documents that a sequence is packed from
                 (0: one), tokens at a sequence's start that all of its rows see

The lengths of a case are fixed; a seed draws their order, the blocks' places in the pool, the documents, the
positions and the values.
"""
import math
from statistics import NormalDist

import numpy as np
import torch

own = False

BLOCK = 16
DEVICE = "cuda:0"
BASE = 500000.0
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# scaling -> (kind, factor, original context, low, high)
SCALINGS = {"none": (0, 1.0, 0.0, 0.0, 0.0), "linear": (1, 4.0, 0.0, 0.0, 0.0), "ntk": (2, 4.0, 0.0, 0.0, 0.0),
            "bands": (3, 8.0, 8192.0, 1.0, 4.0), "yarn": (4, 16.0, 4096.0, 1.0, 32.0)}


def _case(name, kind, hq, hkv, d, **kw):
    c = dict(name=name, kind=kind, hq=hq, hkv=hkv, d=d, batch=0, tokens=0, reach=0, shared=0, lo=0, hi=0,
             lengths="even", chunk_lo=1, chunk_hi=1, pad=0, dtype="bf16", rotary=d, layout="half", scaling="none",
             norm=False, cap=0.0, alibi=False, window=0, doc_lo=0, doc_hi=0, prefix=0)
    c.update(kw)
    return c


def listed():
    return [
        # A small model's decode step, four calls in flight: launch-bound.
        _case("rope_tiny_step", "rope", 8, 2, 64, tokens=4, reach=300, layout="interleaved"),
        # The rows of one long prompt, heads normed, positions scaled for a long context.
        _case("rope_long_prompt", "rope", 64, 8, 128, tokens=8191, reach=131072, scaling="yarn", norm=True),
        # A step of a stage's batch: one token per sequence into the cache, half of the head rotated.
        _case("append_step", "append", 32, 8, 128, batch=64, shared=2048, lo=64, hi=512, rotary=64, norm=True),
        # The new prompts of a retry stage's whole batch, in the engine's padded row buffer.
        _case("append_prompts", "append", 32, 8, 128, batch=93, shared=2304, chunk_lo=128, chunk_hi=1024, pad=117,
              scaling="bands", norm=True),
        # The small model's step with a distance bias instead of rotated positions.
        _case("decode_tiny_alibi", "decode", 8, 2, 64, batch=4, lo=100, hi=300, alibi=True),
        # One call alone over a long context, capped scores.
        _case("decode_single_long", "decode", 64, 8, 128, batch=1, lo=30011, hi=30011, cap=50.0),
        # One engine pool of mixed lengths, capped scores.
        _case("decode_pool_capped", "decode", 32, 8, 128, batch=256, lo=64, hi=8192, lengths="lognormal", cap=50.0),
        # A sliding-window layer over long contexts, two query heads per KV head.
        _case("decode_window", "decode", 16, 8, 128, batch=64, lo=4097, hi=28672, cap=30.0, window=4096),
        # The retries of one request as they arrive, capped scores over a resident context.
        _case("extend_retries_capped", "extend", 32, 8, 128, batch=3, shared=2304, chunk_lo=128, chunk_hi=1024, cap=30.0),
        # A long-context stage's first prompt, distance bias, nothing resident.
        _case("extend_prompt_alibi", "extend", 32, 8, 128, batch=1, chunk_lo=8191, chunk_hi=8191, alibi=True),
        # Packed documents that must not see each other.
        _case("extend_documents", "extend", 32, 8, 128, batch=4, chunk_lo=3001, chunk_hi=4096, doc_lo=61, doc_hi=1500),
        # Short inputs with a prefix that sees itself whole, a small model.
        _case("extend_prefix_small", "extend", 24, 3, 64, batch=5, chunk_lo=17, chunk_hi=301, prefix=200, pad=5),
    ]


HEADS = [(32, 8, 128), (64, 8, 128), (16, 16, 128), (16, 8, 128), (28, 4, 128), (8, 1, 128), (40, 5, 128), (12, 2, 128),
         (8, 2, 64), (32, 4, 64), (24, 3, 64), (12, 12, 64), (15, 5, 64)]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = max(most.get(c["kind"], 0.0), w["bytes"] / 5e12 + w["flops"] / 5e14)
    while True:
        c = _draw_one(rng)
        if c["kind"] in ("decode", "extend"):
            s = _structure(c, 0)
            tokens = c["batch"] * s["table"].shape[1] * BLOCK
            if tokens * c["hq"] * int(s["chunk"].max()) > 2.1e9 or tokens * c["hkv"] * c["d"] > 2.2e9:
                continue   # the plain form's scores and gathered tokens
        w = work(c)
        if w["bytes"] / 5e12 + w["flops"] / 5e14 <= most[c["kind"]]:
            return c


def _draw_one(rng):
    kind = rng.choice(["rope", "append", "decode", "extend"])
    hq, hkv, d = rng.choice(HEADS)
    c = _case("", kind, hq, hkv, d)
    del c["name"]
    if kind in ("rope", "append"):
        c.update(dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), layout=rng.choice(["half", "interleaved"]),
                 rotary=rng.choice([d, d, d // 2, d // 4, d - 16, 0]), scaling=rng.choice(sorted(SCALINGS)),
                 norm=rng.random() < 0.5)
    if kind == "rope":
        c.update(tokens=_logint(rng, 1, 16384), reach=_logint(rng, 16, 1 << 20))
        return c
    c["batch"] = _logint(rng, 1, 256)
    if kind in ("append", "extend"):
        c["chunk_hi"] = _logint(rng, 1, 8192)
        c["chunk_lo"] = _logint(rng, 1, c["chunk_hi"])
        c["pad"] = rng.choice([0, rng.randint(1, 64)])
        c["shared"] = BLOCK * rng.choice([0, rng.randint(1, 256)])
        c["hi"] = rng.choice([0, _logint(rng, 1, 16384)])
        c["lo"] = rng.choice([0, c["hi"]])
    if kind == "append":
        return c
    if kind == "decode":
        c["hi"] = _logint(rng, 1, 32768)
        c["lo"] = _logint(rng, 1, c["hi"])
    how = rng.choice(["cap", "cap", "alibi", "window", "both", "documents", "prefix" if kind == "extend" else "cap"])
    if how in ("cap", "both"):
        c["cap"] = rng.choice([20.0, 30.0, 50.0])
    if how in ("alibi", "both"):
        c["alibi"] = True
    if how == "window":
        c.update(window=_logint(rng, 1, 8192), cap=rng.choice([0.0, 50.0]))
    if how == "documents":
        c["doc_hi"] = _logint(rng, 8, 4096)
        c["doc_lo"] = _logint(rng, 4, c["doc_hi"])
    if how == "prefix":
        c["prefix"] = _logint(rng, 1, 2048)
    return c


# --------------------------------------------------------------------------
# lengths, tables and work
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
    """Lengths in the seed's order, block tables over a shuffled pool 1.2 times as large as needed, and the masks."""
    rng = np.random.default_rng(seed)
    n = c["batch"]
    old = rng.permutation(_spread(n, c["lo"], c["hi"], c["lengths"]))
    if c["kind"] == "decode":
        chunk = np.ones(n, np.int64)
        ctx = c["shared"] + old
    elif c["chunk_lo"] == c["chunk_hi"] == 1:      # a step: the new token is the last of lo .. hi
        chunk = np.ones(n, np.int64)
        ctx = c["shared"] + np.maximum(old, 1)
    else:
        chunk = rng.permutation(_spread(n, c["chunk_lo"], c["chunk_hi"], "even"))
        ctx = c["shared"] + old + chunk
    n_pre = c["shared"] // BLOCK
    tail = (ctx - c["shared"] + BLOCK - 1) // BLOCK
    needed = n_pre + int(tail.sum())
    blocks = max(1, math.ceil(1.2 * needed))
    ids = rng.permutation(blocks)
    table = np.zeros((n, max(1, int(n_pre + tail.max()))), np.int32)
    table[:, :n_pre] = ids[:n_pre]
    at = n_pre
    for b in range(n):
        table[b, n_pre:n_pre + tail[b]] = ids[at:at + tail[b]]
        at += tail[b]
    start = np.concatenate([[0], np.cumsum(chunk)])
    first = None
    if c["doc_hi"]:
        first = np.zeros(start[-1], np.int64)
        for b in range(n):
            most = int(ctx[b])
            ends = np.cumsum(rng.integers(c["doc_lo"], c["doc_hi"] + 1, size=most // c["doc_lo"] + 1))
            begins = np.concatenate([[0], ends])
            p = np.arange(most - chunk[b], most)
            first[start[b]:start[b + 1]] = begins[np.searchsorted(begins, p, side="right") - 1]
    prefix = np.minimum(ctx, rng.integers(1, c["prefix"] + 1, size=n)) if c["prefix"] else None
    return dict(ctx=ctx, chunk=chunk, table=table, blocks=blocks, start=start, first=first, prefix=prefix)


def _visible(c, s):
    """(first, end) of the tokens that each row sees."""
    row = np.arange(s["start"][-1])
    b = np.searchsorted(s["start"], row, side="right") - 1
    p = s["ctx"][b] - s["chunk"][b] + row - s["start"][b]
    lo = np.zeros_like(p) if s["first"] is None else s["first"].copy()
    if c["window"]:
        lo = np.maximum(lo, p - c["window"] + 1)
    hi = p + 1 if s["prefix"] is None else np.maximum(p + 1, s["prefix"][b])
    return b, lo, hi


def work(c):
    size = 4 if c["dtype"] == "fp32" else 2
    if c["kind"] == "rope":
        n = c["tokens"] * (c["hq"] + c["hkv"]) * c["d"]
        return {"bytes": 2 * n * size + 4 * c["tokens"], "flops": 8 * n}
    s = _structure(c, 0)
    rows = int(s["start"][-1])
    if c["kind"] == "append":
        n = rows * c["d"]
        return {"bytes": n * (c["hq"] + 2 * c["hkv"]) * (size + 2) + 4 * rows, "flops": 8 * n * (c["hq"] + c["hkv"])}
    b, lo, hi = _visible(c, s)
    seen = np.full(c["batch"], 1 << 40)
    np.minimum.at(seen, b, lo)
    tokens = int(np.maximum(s["ctx"] - np.maximum(seen, c["shared"]), 0).sum()) + max(0, c["shared"] - int(seen.min()))
    nbytes = tokens * 2 * c["hkv"] * c["d"] * 2 + 2 * rows * c["hq"] * c["d"] * 2 + s["table"].size * 4
    return {"bytes": nbytes, "flops": int(4 * c["hq"] * c["d"] * int((hi - lo).sum()))}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def prepare(case, seed):
    c, hq, hkv, d = case, case["hq"], case["hkv"], case["d"]
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed * 7919 + 17)

    def normal(shape, dtype, scale=1.0):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).mul_(scale).to(dtype)

    st = {"c": c}
    if c["kind"] in ("rope", "append"):
        t = TYPES[c["dtype"]]
        if c["norm"]:
            st["wq"] = 1.0 + 0.2 * normal((d,), torch.float32)
            st["wk"] = 1.0 + 0.2 * normal((d,), torch.float32)
        else:
            st["wq"] = st["wk"] = None
        st["freqs"], st["magnitude"] = _frequencies(c["rotary"], c["scaling"])
        st["freqs"] = torch.tensor(st["freqs"], dtype=torch.float64, device=DEVICE)
    if c["kind"] == "rope":
        n = c["tokens"]
        # one projection's output: q, k and v of a token side by side
        st["rows"] = normal((n, (hq + 2 * hkv) * d), t)
        st["positions"] = torch.randint(0, c["reach"], (n,), generator=gen, device=DEVICE, dtype=torch.int32)
        st["q_out"] = torch.zeros((n, hq, d), dtype=t, device=DEVICE)
        st["k_out"] = torch.zeros((n, hkv, d), dtype=t, device=DEVICE)
    else:
        s = _structure(c, seed)
        for name in ("ctx", "table", "start", "first", "prefix"):
            st[name] = None if s[name] is None else torch.tensor(s[name], dtype=torch.int32, device=DEVICE)
        st.update(blocks=s["blocks"], rows_in=int(s["start"][-1]), total=int(s["start"][-1]) + c["pad"],
                  max_ctx=int(s["ctx"].max()), max_chunk=int(s["chunk"].max()))
        shape = (s["blocks"], hkv, BLOCK, d)
        st["k_pool"] = normal(shape, torch.bfloat16)
        st["v_pool"] = normal(shape, torch.bfloat16)
        if c["kind"] == "append":
            st["rows"] = normal((st["total"], (hq + 2 * hkv) * d), t)
        else:
            # scores of a few units, as trained heads have them: some reach the cap
            st["q"] = normal((st["total"], hq, d), torch.bfloat16, 4.0 if c["cap"] else 1.0)
            st["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32,
                                        device=DEVICE) if c["alibi"] else None
        st["out"] = torch.zeros((st["total"], hq, d), dtype=torch.bfloat16, device=DEVICE)
    if own:
        _prepare_own(st)
    return st


def _prepare_own(st):
    """The handles and the workspace that a program keeps beside its cache."""
    from paper_2510_14126_amd import binding as pa
    c = st["c"]
    if "freqs" in st:
        kind, factor, original, low, high = SCALINGS[c["scaling"]]
        freqs, magnitude = pa.pa_rope_frequencies(c["rotary"], BASE, kind, factor, original, low, high)
        st["rope"] = pa.pa_rope_create(c["d"], c["rotary"], pa.PA_ROPE_HALF if c["layout"] == "half"
                                       else pa.PA_ROPE_INTERLEAVED, freqs, magnitude)
        st["type"] = {"bf16": pa.PA_BF16, "fp16": pa.PA_FP16, "fp32": pa.PA_FP32}[c["dtype"]]
    if c["kind"] != "rope":
        st["pool"] = pa.kv_pool_create(st["blocks"], BLOCK, c["hkv"], c["d"], st["k_pool"], st["v_pool"])
    if c["kind"] in ("decode", "extend"):
        size = pa.paged_attn_biased_workspace_size(st["pool"], c["batch"], c["hq"], st["max_ctx"], st["max_chunk"],
                                                   c["window"])
        st["workspace"] = torch.empty(max(size, 1), dtype=torch.uint8, device=DEVICE)
        st["workspace_bytes"] = size


def _frequencies(r, scaling):
    """Angle per position of each rotated pair, and the rotated values' factor."""
    kind, factor, original, low, high = SCALINGS[scaling]
    i = np.arange(r // 2)
    f = BASE ** (-2.0 * i / max(r, 1))
    if kind == 1:
        return f / factor, 1.0
    if kind == 2:
        return (BASE * factor ** (r / (r - 2)) if r > 2 else BASE) ** (-2.0 * i / max(r, 1)), 1.0
    if kind == 3:
        smooth = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return f / factor * (1 - smooth) + f * smooth, 1.0
    if kind == 4:
        at = [r * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(BASE)) for turns in (high, low)]
        a, b = max(math.floor(at[0]), 0), min(math.ceil(at[1]), max(r - 1, 0))
        ramp = np.clip((i - a) / max(b - a, 1e-3), 0.0, 1.0)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1.0
    return f, 1.0


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(st):
    c = st["c"]
    if own:
        return _run_own(st)
    if c["kind"] == "rope":
        hq, hkv, d = c["hq"], c["hkv"], c["d"]
        rows = st["rows"].view(c["tokens"], hq + 2 * hkv, d)
        st["q_out"].copy_(_rotate(st, rows[:, :hq], st["wq"], st["positions"]))
        st["k_out"].copy_(_rotate(st, rows[:, hq:hq + hkv], st["wk"], st["positions"]))
        return {"q": st["q_out"], "k": st["k_out"]}
    if c["kind"] == "append":
        return _append_plain(st)
    return {"out": _attention_plain(st)}


def _rotate(st, x, weight, positions):
    """The rows [n][heads][d], normed and rotated, in 32 bits (the angles in 64)."""
    c, r = st["c"], st["c"]["rotary"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    angle = positions.double()[:, None] * st["freqs"]
    cos, sin = ((f(angle) * st["magnitude"]).float()[:, None, :] for f in (torch.cos, torch.sin))
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _places(st):
    """Sequence and position of each row that a sequence has."""
    row = torch.arange(st["rows_in"], device=DEVICE, dtype=torch.int32)
    b = torch.searchsorted(st["start"], row, right=True) - 1
    return row, b, st["ctx"][b] - st["start"][b + 1] + row


def _append_plain(st):
    c = st["c"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    row, b, p = _places(st)
    rows = st["rows"][:st["rows_in"]].view(-1, hq + 2 * hkv, d)
    st["out"][:st["rows_in"]] = _rotate(st, rows[:, :hq], st["wq"], p).to(torch.bfloat16)
    block = st["table"][b, p // BLOCK].long()
    slot = (p % BLOCK).long()
    st["k_pool"][block, :, slot] = _rotate(st, rows[:, hq:hq + hkv], st["wk"], p).to(torch.bfloat16)
    st["v_pool"][block, :, slot] = rows[:, hq + hkv:].float().to(torch.bfloat16)
    return {"q": st["out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"]}


def _attention_plain(st):
    c = st["c"]
    n, hq, hkv, d, most = c["batch"], c["hq"], c["hkv"], c["d"], st["max_chunk"]
    group = hq // hkv
    _, b, p = _places(st)
    i = p - (st["ctx"] - (st["start"][1:] - st["start"][:-1]))[b]
    table = st["table"].long()
    tokens = table.shape[1] * BLOCK
    k = st["k_pool"][table].permute(0, 2, 4, 1, 3).reshape(n, hkv, d, tokens).float()
    v = st["v_pool"][table].permute(0, 2, 1, 3, 4).reshape(n, hkv, tokens, d).float()
    q = torch.zeros((n, most, hkv, group, d), device=DEVICE)
    q[b, i] = st["q"][:st["rows_in"]].float().view(-1, hkv, group, d)
    s = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(n, hkv, most * group, d), k)
    s = s.view(n, hkv, most, group, tokens).mul_(d ** -0.5)
    if c["cap"]:
        s = s.div_(c["cap"]).tanh_().mul_(c["cap"])
    # position of chunk token i, and what it sees
    at = (st["ctx"] - (st["start"][1:] - st["start"][:-1]))[:, None] + torch.arange(most, device=DEVICE, dtype=torch.int32)
    t = torch.arange(tokens, device=DEVICE, dtype=torch.int32)
    if c["alibi"]:
        away = (at[:, :, None] - t).abs().float()
        s -= st["slopes"].view(1, hkv, 1, group, 1) * away[:, None, :, None, :]
    low = torch.zeros((n, most), device=DEVICE, dtype=torch.int32)
    if st["first"] is not None:
        low[b, i] = st["first"]
    if c["window"]:
        low = torch.maximum(low, at - c["window"] + 1)
    end = at + 1
    if st["prefix"] is not None:
        end = torch.maximum(end, st["prefix"][:, None])
    end = torch.minimum(end, st["ctx"][:, None])
    seen = (t >= low[:, :, None]) & (t < end[:, :, None])
    s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    peak = s.amax(-1, keepdim=True)
    s = s.sub_(torch.where(peak == -math.inf, 0.0, peak)).exp_()
    total = s.sum(-1)
    out = torch.matmul(s.view(n, hkv, most * group, tokens), v).view(n, hkv, most, group, d)
    out = torch.where(total[..., None] > 0, out / total[..., None], 0.0)
    st["out"][:st["rows_in"]] = out.permute(0, 2, 1, 3, 4)[b, i].reshape(-1, hq, d).to(torch.bfloat16)
    return st["out"]


def _run_own(st):
    from paper_2510_14126_amd import binding as pa
    c = st["c"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] in ("rope", "append"):
        rows = st["rows"]
        stride = rows.shape[1]
        base, step = rows.data_ptr(), d * rows.element_size()
        q, k, v = base, base + hq * step, base + (hq + hkv) * step
    if c["kind"] == "rope":
        pa.paged_attn_norm_rope(st["rope"], q, stride, hq, st["wq"], k, stride, hkv, st["wk"], EPS, st["type"],
                                st["positions"], c["tokens"], st["q_out"], hq * d, st["k_out"], hkv * d)
        return {"q": st["q_out"], "k": st["k_out"]}
    if c["kind"] == "append":
        pa.paged_attn_rope_append(st["pool"], st["rope"], q, stride, hq, st["wq"], k, stride, st["wk"], v, stride, EPS,
                                  st["type"], None, st["start"], st["total"], st["table"], st["table"].shape[1],
                                  st["ctx"], c["batch"], st["out"])
        return {"q": st["out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"]}
    if c["kind"] == "decode":
        pa.paged_attn_decode_biased(st["pool"], st["q"], st["table"], st["table"].shape[1], st["ctx"], c["batch"], hq,
                                    d ** -0.5, c["cap"], st["slopes"], c["window"], st["first"], st["max_ctx"],
                                    st["workspace"], st["workspace_bytes"], st["out"])
    else:
        pa.paged_attn_extend_biased(st["pool"], st["q"], st["start"], st["total"], st["table"], st["table"].shape[1],
                                    st["ctx"], c["batch"], hq, d ** -0.5, c["cap"], st["slopes"], c["window"],
                                    st["first"], st["prefix"], st["max_ctx"], st["max_chunk"], st["workspace"],
                                    st["workspace_bytes"], st["out"])
    return {"out": st["out"]}


# --------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    c = case
    if c["kind"] in ("rope", "append"):
        return _exact_rows(st, c)
    return {"out": _exact_attention(st, c, seed)}


def _exact_head_rows(x, weight, position, freqs, magnitude, r, half):
    """One head's rows [n][d] at their positions."""
    y = x.double()
    if weight is not None:
        y = y / ((y * y).sum(-1, keepdim=True) / y.shape[-1] + EPS).sqrt() * weight.double()
    z = y.clone()
    turn = torch.polar(torch.full((), magnitude, dtype=torch.float64, device=DEVICE),
                       position.double().unsqueeze(-1) * freqs)
    first = slice(0, r // 2) if half else slice(0, r, 2)
    second = slice(r // 2, r) if half else slice(1, r, 2)
    pair = torch.complex(y[..., first], y[..., second]) * turn
    z[..., first], z[..., second] = pair.real, pair.imag
    return z


def _exact_rows(st, c):
    hq, hkv, d, r, half = c["hq"], c["hkv"], c["d"], c["rotary"], c["layout"] == "half"
    if c["kind"] == "rope":
        n, pos = c["tokens"], st["positions"]
        q_out = torch.zeros((n, hq, d), dtype=torch.float64, device=DEVICE)
        k_out = torch.zeros((n, hkv, d), dtype=torch.float64, device=DEVICE)
    else:
        n = st["rows_in"]
        start, ctx = st["start"].tolist(), st["ctx"].tolist()
        pos = torch.cat([torch.arange(ctx[b] - (start[b + 1] - start[b]), ctx[b], device=DEVICE)
                         for b in range(c["batch"])])
        seq = torch.repeat_interleave(torch.arange(c["batch"], device=DEVICE), (st["start"][1:] - st["start"][:-1]).long())
        q_out = torch.zeros((st["total"], hq, d), dtype=torch.float64, device=DEVICE)
        kp, vp = st["k_pool"].double(), st["v_pool"].double()
        where = (st["table"].long()[seq, pos // BLOCK], pos % BLOCK)
    for h in range(hq + 2 * hkv):
        x = st["rows"][:n, h * d:(h + 1) * d]
        if h < hq:
            q_out[:n, h] = _exact_head_rows(x, st["wq"], pos, st["freqs"], st["magnitude"], r, half)
        elif h < hq + hkv:
            y = _exact_head_rows(x, st["wk"], pos, st["freqs"], st["magnitude"], r, half)
            if c["kind"] == "rope":
                k_out[:, h - hq] = y
            else:
                kp[where[0], h - hq, where[1]] = y
        elif c["kind"] == "append":
            vp[where[0], h - hq - hkv, where[1]] = x.double()
    return {"q": q_out, "k": k_out} if c["kind"] == "rope" else {"q": q_out, "k_pool": kp, "v_pool": vp}


def _exact_attention(st, c, seed):
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    s = _structure(c, seed)
    _, lo, hi = _visible(c, s)
    out = torch.zeros((st["total"], hq, d), dtype=torch.float64, device=DEVICE)
    slopes = [0.0] * hq if st["slopes"] is None else st["slopes"].double().tolist()
    slopes = torch.tensor(slopes, dtype=torch.float64, device=DEVICE).view(hkv, hq // hkv, 1, 1)
    lo, hi = torch.tensor(lo, device=DEVICE), torch.tensor(hi, device=DEVICE)
    for b in range(c["batch"]):
        n, length = int(s["ctx"][b]), int(s["chunk"][b])
        ids = st["table"][b, :(n + BLOCK - 1) // BLOCK].long()
        k = st["k_pool"][ids].double().transpose(1, 2).reshape(-1, hkv, d)[:n].permute(1, 2, 0).contiguous()
        v = st["v_pool"][ids].double().transpose(1, 2).reshape(-1, hkv, d)[:n].transpose(0, 1).contiguous()
        t = torch.arange(n, device=DEVICE)
        for i0 in range(0, length, 1024):
            rows = slice(int(s["start"][b]) + i0, int(s["start"][b]) + min(length, i0 + 1024))
            m = rows.stop - rows.start
            q = st["q"][rows].double().view(m, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
            x = (torch.bmm(q, k) / math.sqrt(d)).view(hkv, hq // hkv, m, n)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            p = n - length + i0 + torch.arange(m, device=DEVICE)
            x = x - slopes * (p[:, None] - t).abs()
            hidden = (t < lo[rows, None]) | (t >= hi[rows, None])
            x = x.masked_fill(hidden, -math.inf)
            w = torch.softmax(x, -1)
            w = torch.where(hidden.all(-1)[:, None], 0.0, w)
            o = torch.bmm(w.reshape(hkv, -1, n), v).view(hkv, hq // hkv, m, d)
            out[rows] = o.permute(2, 0, 1, 3).reshape(m, hq, d)
    return out
