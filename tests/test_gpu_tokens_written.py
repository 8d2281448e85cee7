"""That the calls of paged_attn_tokens.h write what they return: again over buffers and
workspaces that hold other values, and with rows before and behind every output that
nothing may touch."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2510_14126_amd import binding as pa  # noqa: E402
from test_gpu_biased import DEV, dev16, dev32  # noqa: E402
from test_gpu_chosen import WEIGHTS, Sparse, Weights  # noqa: E402
from test_gpu_tokens_flow import cases  # noqa: E402

pytestmark = pytest.mark.gpu


def workspace_of(call):
    """The workspace that a case's call (a closure) hands on."""
    return dict(zip(call.__code__.co_freevars, (c.cell_contents for c in call.__closure__)))["ws"]


@pytest.mark.parametrize("name", ["groups_of_four", "groups_of_eight", "one_long_64", "no_groups", "filled", "filled_64"])
def test_shared_blocks_change_no_bit(name):
    """Blocks that the allocator knows as shared are loaded with another cache policy: all is written anew, alike."""
    print(f"[gpu case] tokens over shared blocks, written anew {name}", flush=True)
    kw = WEIGHTS[name]
    w = Weights(8, chunk=[1] * len(kw["ctx"]), **kw)
    w.go()
    s = Sparse(9, exact=False, first=1, last=1, most=60, **kw)
    s.setup()
    s.bound()
    s.select()
    s.attend()
    torch.cuda.synchronize()
    want = [x.clone() for x in (w.out, w.after, s.t["out"])]
    assert all((x != y).any() for x, y in zip(want, (0x4242, -7.0, 0x4242)))
    for c in (w, s):
        pa.kv_pool_claim(c.pool, [0])
        pa.kv_pool_retain(c.pool, [0])
        assert pa.kv_pool_num_shared(c.pool) == 1
    for fill in (255, 0):
        for x, value in ((w.out, 0x4242), (w.after, -7.0), (s.t["out"], 0x4242), (workspace_of(w.call), fill), (s.t["ws"], fill)):
            x.fill_(value)
        w.call()
        s.attend()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, (w.out, w.after, s.t["out"])))


def test_two_streams_at_once():
    """Calls side by side, each with its workspace, write all of their outputs anew."""
    print("[gpu case] tokens on two streams, written anew", flush=True)
    one, two = cases(), cases()
    torch.cuda.synchronize()
    want = [[x.clone() for x in outs] for _, outs in one]
    # what the outputs held before their first call: trees, bounds and picks and outputs, weights, the move's new places
    before = [[0x4242], [0x4242], [0x4242, 77, 0x4242], [0x4242, -7.0], [None, None, -7.0, 0]]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for fill in (255, 0, 255):
        for every in (one, two):
            for (call, outs), values in zip(every, before):
                for x, value in zip(outs, values):
                    if value is not None:
                        x.fill_(value)
            for call, _ in (every[0], every[1], every[3]):
                workspace_of(call).fill_(fill)
        torch.cuda.synchronize()
        for i in range(len(one)):
            one[i][0](stream=a.cuda_stream)
            two[-1 - i][0](stream=b.cuda_stream)
        torch.cuda.synchronize()
        for every in (one, two):
            for (_, outs), ref in zip(every, want):
                for x, y in zip(outs, ref):
                    assert torch.equal(x, y)


def guarded(shape, value, dtype):
    """A tensor of `value`s whose first and last row stand around an output."""
    return torch.full((shape[0] + 2, *shape[1:]), value, dtype=dtype, device=DEV)


@pytest.mark.parametrize("ctx", [[10, 70, 33, 10], [0, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 5, 0]])
@pytest.mark.parametrize("ids,lie", [(-5, -2 ** 31), (2 ** 31 - 1, 2 ** 31 - 1), (3, 20), (0, 0)])
def test_rows_around_the_outputs_stay(ctx, ids, lie):
    """True and lying lengths, tables and lists: the rows before and behind every output hold what they held."""
    print(f"[gpu case] rows around {ctx} {ids} {lie}", flush=True)
    batch, hq, hkv, d, blocks, width, top, most = 4, 8, 2, 64, 6, 5, 70, 3
    gen = torch.Generator(device=DEV).manual_seed(3)
    k, v = (torch.randn(blocks, hkv, 16, d, generator=gen, device=DEV).to(torch.bfloat16).view(torch.int16) for _ in range(2))
    q = torch.randn(batch, hq, d, generator=gen, device=DEV).to(torch.bfloat16)
    pool = pa.kv_pool_create(blocks, 16, hkv, d, k, v)
    table, lens, first = dev32(np.full((batch, width), ids)), dev32(ctx), dev32(np.full(batch, lie))
    lists = dev32(np.full((batch, hkv, most), lie))
    bounds = guarded((blocks, hkv, 2, d), 0x4242, torch.int16)
    picked = guarded((batch, hkv, most), 9, torch.int32)
    out, apart, tree = (guarded((batch, hq, d), 0x4242, torch.int16) for _ in range(3))
    totals = guarded((batch, top), 3.0, torch.float32)
    kept, kept_lens, new = guarded((batch, 40), 9, torch.int32), guarded((batch,), 9, torch.int32), guarded((batch,), 9, torch.int32)
    moved_k, moved_v = guarded((blocks, hkv, 16, d), 0x4242, torch.int16), guarded((blocks, hkv, 16, d), 0x4242, torch.int16)
    moved_k[1:-1], moved_v[1:-1] = k, v
    moved_pool = pa.kv_pool_create(blocks, 16, hkv, d, moved_k[1:], moved_v[1:])
    sizes = [pa.paged_attn_select_workspace_size(pool, batch, top, most), pa.paged_attn_selected_workspace_size(pool, batch, hq, most),
             pa.paged_attn_weights_workspace_size(pool, batch, hq, top), pa.paged_attn_tree_workspace_size(pool, batch, hq, top, 4)]
    spaces = [torch.full((n + 32,), 7, dtype=torch.uint8, device=DEV) for n in sizes]
    pa.paged_attn_block_bounds(pool, bounds[1:], table, width, first, lens, batch, top, 40)
    pa.paged_attn_select_blocks(pool, q, bounds[1:], table, width, lens, batch, hq, top, 1, 1, most, spaces[0], sizes[0], picked[1:])
    pa.paged_attn_decode_selected(pool, q, table, width, lens, batch, hq, 0.1, top, lists, most, spaces[1], sizes[1], apart[1:])
    pa.paged_attn_decode_weights(pool, q, table, width, lens, batch, hq, 0.1, top, 1.0, None, totals[1:], top, spaces[2], sizes[2],
                                 out[1:])
    pa.paged_attn_extend_tree(pool, q, dev32(np.arange(batch + 1)), batch, first, table, width, lens, batch, hq, 0.1, 0.0, top, 4,
                              spaces[3], sizes[3], tree[1:])
    pa.paged_attn_keep_heaviest(totals[1:], top, first, lens, batch, top, 5, 40, kept[1:], 40, kept_lens[1:])
    pa.paged_attn_compact(moved_pool, table, width, None, 0, first, lens, batch, top, kept[1:], 40, kept_lens[1:], totals[1:],
                          totals[1:], top, new[1:])
    torch.cuda.synchronize()
    for x, value in ((bounds, 0x4242), (out, 0x4242), (apart, 0x4242), (tree, 0x4242), (totals, 3.0), (picked, 9), (kept, 9),
                     (kept_lens, 9), (new, 9), (moved_k, 0x4242), (moved_v, 0x4242)):
        assert (x[0] == value).all() and (x[-1] == value).all()
    assert all((x[n:] == 7).all() for x, n in zip(spaces, sizes))
