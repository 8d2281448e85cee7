"""Extend attention where a window and a prefix that sees itself whole meet and
a tile's tokens are split over workgroups: a row's tokens then reach from its
window's first to the prefix's end, more blocks than the window alone.  Oracle
and tolerance are those of test_gpu_biased."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_biased import Case, documents  # noqa: E402

pytestmark = pytest.mark.gpu

RANGES = {
    "d64": dict(ctx=[900], chunk=[900], hq=8, hkv=2, d=64, window=700, prefix=[900]),
    "d128": dict(ctx=[2000], chunk=[300], hq=8, hkv=2, d=128, window=700, prefix=[2000]),
    "one_kv_head": dict(ctx=[2000], chunk=[500], hq=8, hkv=1, d=128, window=1024, prefix=[2000], cap=30.0, qscale=4.0),
    "eight_kv_heads": dict(ctx=[2000], chunk=[100], hq=32, hkv=8, d=128, window=1024, prefix=[2000], pad=3),
    "ragged": dict(ctx=[1500, 40, 0, 2222, 733], chunk=[90, 40, 0, 1, 33], hq=8, hkv=2, d=128, window=700,
                   prefix=[1500, 30, 0, 5000, 733], alibi=True),
    "prefix_inside_the_chunk": dict(ctx=[1800], chunk=[800], hq=5, hkv=1, d=64, window=900, prefix=[1407], cap=20.0,
                                    qscale=3.0, alibi=True),
    "documents_too": dict(ctx=[1600], chunk=[600], hq=12, hkv=2, d=64, window=800, prefix=[1555],
                          docs=documents(100, 900)),
    "prefix_behind_the_window": dict(ctx=[3000], chunk=[64], hq=8, hkv=2, d=128, window=700, prefix=[500]),
}


@pytest.mark.parametrize("spare", [0, 700])
@pytest.mark.parametrize("name", sorted(RANGES))
def test_window_and_prefix_over_partitions(name, spare):
    print(f"[gpu case] window and prefix {name} {spare}", flush=True)
    kw = dict(RANGES[name])
    c = Case(len(name) + 200, **kw)
    if spare:
        c.table = np.concatenate([c.table, np.full((c.batch, spare // 16 + 2), -9, np.int32)], axis=1)
        c.width = c.table.shape[1]
    got = c.run(spare=spare)
    assert c.size > 0, "the tokens are split over workgroups"
    c.check(got, None, 40.0 * kw.get("qscale", 1.0))
