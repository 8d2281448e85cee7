"""Capped scores of large rows with a small scale: the coefficients of the cap's
polynomial in the raw score pass the smallest numbers of fp32 (scale^7 / cap^6
and so on), while the scores themselves are ordinary ones.  Oracle and tolerance
are those of test_gpu_biased; the largest |score| is 5.5 scale |q| |k|."""
import pytest

torch = pytest.importorskip("torch")

from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import Case  # noqa: E402

gpu = pytest.mark.gpu
FORMS = {
    "decode": dict(ctx=[300, 1500, 7], chunk=[1] * 3, hq=32, hkv=8, d=128),
    "decode_64": dict(ctx=[300, 1500, 7], chunk=[1] * 3, hq=8, hkv=2, d=64),
    "rows_32": dict(ctx=[400, 90], chunk=[200, 31], hq=8, hkv=2, d=128),
    "rows_128": dict(ctx=[300] * 12, chunk=[260] * 12, hq=32, hkv=8, d=128),
    "rows_32_64": dict(ctx=[400, 90], chunk=[200, 31], hq=6, hkv=2, d=64),
}


@gpu
@pytest.mark.parametrize("alibi", [False, True])
@pytest.mark.parametrize("scale", [1e-4, 2e-6, 1e-8, 1e-12, 1e-20])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_small_scales(form, scale, alibi):
    print(f"[gpu case] small scale {form} {scale} {alibi}", flush=True)
    kw = FORMS[form]
    c = Case(60, cap=20.0, scale=scale, qscale=8.0 / (scale * kw["d"] ** 0.5), alibi=alibi, **kw)
    c.check(c.run(decode=form.startswith("decode")), None, 60.0)


@pytest.mark.parametrize("cap,scale", [(1e24, 0.1), (1e30, 1e-5), (1e35, 1.0)])
def test_caps_beyond_the_square_of_any_score(cap, scale):
    pool = pa.kv_pool_create(8, 16, 2, 64, 0x10000, 0x10000)
    with pytest.raises(pa.PagedAttnError) as e:
        pa.paged_attn_decode_biased(pool, 0x10000, 0x10000, 8, 0x10000, 2, 8, scale, cap, None, 0, None, 100, 0x10000,
                                    1 << 30, 0x10000)
    assert e.value.code == pa.PA_EUNSUPPORTED
