"""A move whose second table is the first itself: in place, in order, however long."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tokens as oracle  # noqa: E402
from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import dev16, dev32  # noqa: E402
from test_gpu_keep import Move  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_move_within_the_table_itself(d):
    print(f"[gpu case] compact within the same table {d}", flush=True)
    m = Move(d, [6011, 700, 0, 2049], 2, d, 0.8, first=[33, 0, 0, 16])
    stride = max(len(x) for x in m.kept)
    kept = np.full((m.batch, stride), -1)
    for b, x in enumerate(m.kept):
        kept[b, :len(x)] = x
    k, v, table, new = dev16(m.k), dev16(m.v), dev32(m.table), dev32([0] * m.batch)
    pool = pa.kv_pool_create(m.blocks, 16, m.hkv, d, k, v)
    pa.paged_attn_compact(pool, table, m.width, table, m.width, dev32(m.first), dev32(m.ctx), m.batch, max(m.ctx),
                          dev32(kept), stride, dev32([len(x) for x in m.kept]), None, None, 0, new)
    torch.cuda.synchronize()
    want = [m.k, m.v]
    for b in range(m.batch):
        want = [oracle.compact(x, m.table[b], m.table[b], m.first[b], m.kept[b]) for x in want]
    assert np.array_equal(k.cpu().numpy().view(np.uint16), want[0]) and np.array_equal(v.cpu().numpy().view(np.uint16), want[1])
    assert new.tolist() == [f + len(x) for f, x in zip(m.first, m.kept)]
