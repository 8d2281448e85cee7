"""What tokens hold that a row does not see changes no bit of the row's output,
also where other rows of its tile see them: keys far beyond the cap's ordinary
range, infinities and NaN in K and V of every second document."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_biased import INF, NAN, NINF, Case, bits  # noqa: E402

pytestmark = pytest.mark.gpu
DOC = 24                      # tokens of a document: borders inside blocks and stages


def first_of(c, rng):
    p = np.concatenate([np.arange(n - m, n) for n, m in zip(c.ctx, c.chunk)])
    return p // DOC * DOC


FORMS = {
    "decode": dict(ctx=[30, 100, 333, 48, 55], chunk=[1] * 5, hq=32, hkv=8, d=128),
    "decode_64": dict(ctx=[30, 100, 333, 48, 55], chunk=[1] * 5, hq=8, hkv=1, d=64),
    "decode_many_heads": dict(ctx=[30, 100, 333], chunk=[1] * 3, hq=24, hkv=2, d=128),
    "rows_32": dict(ctx=[400, 90], chunk=[400, 31], hq=8, hkv=2, d=128),
    "rows_32_64": dict(ctx=[400, 90], chunk=[400, 31], hq=6, hkv=2, d=64),
    "rows_128": dict(ctx=[500] * 12, chunk=[260] * 12, hq=32, hkv=8, d=128),
    "rows_128_64": dict(ctx=[420] * 12, chunk=[200] * 12, hq=32, hkv=8, d=64),
}


@pytest.mark.parametrize("what", ["large", "special"])
@pytest.mark.parametrize("alibi", [False, True])
@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_other_documents_change_no_bit(form, cap, alibi, what):
    print(f"[gpu case] other documents {form} {cap} {alibi} {what}", flush=True)
    decode = form.startswith("decode")
    c = Case(40, cap=cap, alibi=alibi, docs=first_of, **FORMS[form])
    if decode:                                            # a document of the last few tokens, beside others' in its blocks
        c.first = np.maximum(c.ctx - 7, 0)
    before = c.run(decode=decode)
    rng = np.random.default_rng(41)
    p = np.concatenate([np.arange(n - m, n) for n, m in zip(c.ctx, c.chunk)])
    for b, n in enumerate(c.ctx):
        for t in range(n):
            if (t < n - 7) if decode else (t // DOC % 2 == 1):
                block, line, shape = c.table[b, t // 16], t % 16, (c.hkv, c.d)
                if what == "large":
                    c.k[block, :, line] = bits(rng, shape, 40.0)
                    c.v[block, :, line] = bits(rng, shape, 1000.0)
                else:
                    c.k[block, :, line] = rng.choice([NAN, INF, NINF], size=shape)
                    c.v[block, :, line] = rng.choice([NAN, INF, NINF], size=shape)
    after = c.run(decode=decode)
    rows = np.ones(len(p), bool) if decode else p // DOC % 2 == 0
    differ = before[:c.rows][rows] != after[:c.rows][rows]
    assert not differ.any(), (int(differ.sum()), differ.size)
    assert decode or (before[:c.rows][~rows] != after[:c.rows][~rows]).any()


@pytest.mark.parametrize("alibi", [False, True])
@pytest.mark.parametrize("form", ["rows_32", "rows_128", "rows_128_64"])
def test_later_tokens_change_no_bit(form, alibi):
    """Causal rows before a token with keys beyond the cap's ordinary range."""
    print(f"[gpu case] later tokens {form} {alibi}", flush=True)
    c = Case(42, cap=30.0, alibi=alibi, **FORMS[form])
    before = c.run()
    rng = np.random.default_rng(43)
    from_t = c.ctx - c.chunk // 2
    for b, n in enumerate(c.ctx):
        for t in range(from_t[b], n):
            c.k[c.table[b, t // 16], :, t % 16] = bits(rng, (c.hkv, c.d), 40.0)
    after = c.run()
    p = np.concatenate([np.arange(n - m, n) for n, m in zip(c.ctx, c.chunk)])
    rows = p < np.repeat(from_t, c.chunk)
    assert (before[:c.rows][rows] == after[:c.rows][rows]).all()
