"""Distances between positions beyond 2^24, which fp32 does not hold one by one:
a window's rows at the end of a context of millions of tokens (whose table names
few blocks) give bit for bit what they give near the start."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import DEV, Case, dev32  # noqa: E402

pytestmark = pytest.mark.gpu
WINDOW = 100
FORMS = {
    "decode": dict(ctx=[997, 300], chunk=[1, 1], hq=32, hkv=8, d=128),
    "decode_8_heads_64": dict(ctx=[997, 300], chunk=[1, 1], hq=8, hkv=1, d=64),
    "decode_many_heads": dict(ctx=[997, 300], chunk=[1, 1], hq=24, hkv=2, d=128),
    "rows_32": dict(ctx=[500, 333], chunk=[200, 31], hq=8, hkv=2, d=128),
    "rows_128": dict(ctx=[500] * 4, chunk=[260] * 4, hq=64, hkv=16, d=64),
}


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_far_positions(form, cap):
    print(f"[gpu case] far positions {form} {cap}", flush=True)
    decode = form.startswith("decode")
    c = Case(70, cap=cap, alibi=True, window=WINDOW, **FORMS[form])
    near = c.run(decode=decode)
    c.check(near)
    t, more = c.t, 1 << 21                                # blocks of 16 tokens in front
    table = torch.zeros(c.batch, more + c.width, dtype=torch.int32, device=DEV)
    table[:, more:] = t["table"]
    top, most = int(c.ctx.max()) + 16 * more, int(c.chunk.max())
    ctx = dev32(c.ctx + 16 * more)
    size = pa.paged_attn_biased_workspace_size(c.pool, c.batch, c.hq, top, most, WINDOW)
    assert size == c.size
    out = torch.full_like(c.out, 0x4242)
    if decode:
        pa.paged_attn_decode_biased(c.pool, t["q"], table, table.shape[1], ctx, c.batch, c.hq, c.scale, cap,
                                    t["slopes"], WINDOW, None, top, c.ws, size, out)
    else:
        pa.paged_attn_extend_biased(c.pool, t["q"], t["start"], c.total, table, table.shape[1], ctx, c.batch, c.hq,
                                    c.scale, cap, t["slopes"], WINDOW, None, None, top, most, c.ws, size, out)
    torch.cuda.synchronize()
    assert (out.cpu().numpy().view(np.uint16) == near).all()


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("hq,hkv,d,chunks", [(4, 2, 128, [1500, 70]), (6, 2, 64, [1500]), (32, 8, 128, [700] * 3)])
def test_rows_that_see_only_tokens_far_after_them(hq, hkv, d, chunks, cap):
    """A prefix that sees itself whole and first tokens past the row: every distance is to a later token."""
    print(f"[gpu case] far after {hq} {hkv} {d} {chunks} {cap}", flush=True)

    def first(c, rng):
        p = np.concatenate([np.arange(n) for n in c.ctx])
        return np.minimum(p + 600, np.repeat(c.ctx, c.chunk) - 40)
    c = Case(71, ctx=chunks, chunk=chunks, hq=hq, hkv=hkv, d=d, cap=cap, alibi=True, docs=first, prefix=chunks)
    # a score's size is the bias of its row's nearest tokens too, at most slope * 1500
    c.check(c.run(), None, 40.0 + 1500 * float(c.slopes.max()))
