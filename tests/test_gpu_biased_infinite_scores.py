"""Infinite scores of visible tokens: under a cap they are the cap itself; without
one +infinity makes the row NaN, -infinity weighs nothing, and a row of -infinities
alone gives zeros.  Oracle and tolerance are those of test_gpu_biased."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle.attention import bf16_to_f64  # noqa: E402
from test_gpu_biased import INF, NINF, Case  # noqa: E402

pytestmark = pytest.mark.gpu
FORMS = {
    "decode": dict(ctx=[300, 40, 5, 2], chunk=[1] * 4, hq=32, hkv=8, d=128),
    "decode_64": dict(ctx=[300, 40, 5, 2], chunk=[1] * 4, hq=8, hkv=1, d=64),
    "decode_many_heads": dict(ctx=[300, 5], chunk=[1] * 2, hq=24, hkv=2, d=128),
    "decode_split": dict(ctx=[5000, 5], chunk=[1] * 2, hq=8, hkv=2, d=128),
    "rows_32": dict(ctx=[200, 40], chunk=[100, 40], hq=8, hkv=2, d=128),
    "rows_128": dict(ctx=[300] * 12, chunk=[260] * 12, hq=32, hkv=8, d=64),
    "rows_128_short": dict(ctx=[40] * 60, chunk=[40] * 60, hq=32, hkv=8, d=128),
}


@pytest.mark.parametrize("alibi", [False, True])
@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_infinite_scores(form, cap, alibi):
    print(f"[gpu case] infinite scores {form} {cap} {alibi}", flush=True)
    decode = form.startswith("decode")
    c = Case(80, cap=cap, alibi=alibi, **FORMS[form])
    rng = np.random.default_rng(81)
    for b, n in enumerate(c.ctx):
        # an infinity in one dimension: the score's sign is the query's there; every token of the shorter contexts
        for t in (range(n) if n <= 40 else rng.integers(0, n, 3)):
            c.k[c.table[b, t // 16], :, t % 16, 7] = INF if b % 2 == 0 else NINF
    got = c.run(decode=decode)
    with np.errstate(all="ignore"):
        ref = c.reference()
    x = bf16_to_f64(got[:c.rows])
    if cap:
        assert np.isfinite(ref).all()
    else:
        alone = np.isnan(ref).all(-1) & (x == 0).all(-1)
        sign = bf16_to_f64(c.q)[..., 7]
        for b, n in enumerate(c.ctx):
            for r in range(c.start[b], c.start[b + 1]):
                if n <= 40:
                    assert (alone[r] == (sign[r] < 0 if b % 2 == 0 else sign[r] > 0)).all()
                else:
                    assert not alone[r].any()
        assert np.isnan(ref).any() and alone.any() == (c.ctx <= 40).any()
        ref[alone] = 0
    c.check(got, ref, 60.0)
