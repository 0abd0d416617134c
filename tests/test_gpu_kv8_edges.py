"""Calls of the 8-bit cache at the ends of what its header allows: addresses, batches, heads, queries that are not finite,
workspaces in turn."""
import math

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.gpu_helpers import device
from tests.kv8_helpers import DT, filled, shape_of
from tests.test_gpu_kv8 import decoded, rows_of
from tests.test_gpu_kv8_bounds import excess

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def shifted(x, dev, by=16):
    """x at an address that is a multiple of 16 bytes and of nothing larger; what is around it is 0xee."""
    n = x.numel() * x.element_size()
    room = torch.full((n + 256,), 0xEE, dtype=torch.uint8, device=dev)
    at = (by - room.data_ptr()) % 128
    y = room[at:at + n].view(x.dtype).view(x.shape)
    y.copy_(x.to(dev))
    assert y.data_ptr() % 128 == by
    return y, room


@pytest.mark.parametrize("heads,kv_heads,d,page,dtype", [(8, 2, 128, 16, "bf16"), (16, 1, 64, 32, "fp16")])
def test_everything_at_16_bytes(dev, heads, kv_heads, d, page, dtype):
    lens = [300, 1, 47]
    c, table = filled(110, lens, kv_heads, page, d)
    q = rows_of(111, 3, heads * d, 0, DT[dtype], dev)
    want, want_z, _ = decoded(dev, c, table, q, heads, dtype, lens, 300)
    shape = shape_of(3, heads, kv_heads, d, page, c.blocks, table.shape[1], dtype)
    cache, _ = shifted(c.image(), dev)
    qs, _ = shifted(q[:3], dev)
    o, room = shifted(torch.zeros(3, heads * d, dtype=DT[dtype]), dev)
    need = hs.hs_kv8_decode_workspace_bytes(shape, 300)
    ws, ws_room = shifted(torch.zeros(max(need, 16), dtype=torch.uint8), dev)
    lens_d = torch.tensor(lens, dtype=torch.int32, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    hs.hs_kv8_decode(shape, qs, cache, table.to(dev), lens_d, 300, o, None, ws, need, err)
    torch.cuda.synchronize()
    assert err.item() == 0 and torch.equal(o.cpu(), want)
    used = torch.zeros_like(room, dtype=torch.bool)
    at = o.data_ptr() - room.data_ptr()
    used[at:at + o.numel() * 2] = True
    assert (room[~used] == 0xEE).all()
    # appended to and read back at such addresses: the bytes of those at others
    rows = rows_of(112, 40, 2 * kv_heads * d, 0, DT[dtype], dev)[:40]
    slots = torch.arange(40, device=dev)
    images, outs = [], []
    for place in (lambda x: shifted(x, dev)[0], lambda x: x.to(dev)):
        kv, x = place(c.image()), place(rows)
        hs.hs_kv8_append(shape, x, x[:, kv_heads * d:], 2 * kv_heads * d, slots, 40, kv, err)
        out = place(torch.zeros(c.blocks, 2, page, kv_heads, d, dtype=DT[dtype]))
        hs.hs_kv8_read(shape, kv, table.to(dev), lens_d, 300, out, c.blocks, table.to(dev), err)
        images.append(kv.cpu())
        outs.append(out.cpu().view(torch.int16))
    assert err.item() == 0 and torch.equal(*images) and torch.equal(*outs)


@pytest.mark.parametrize("unsplit", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_queries_that_are_not_finite_keep_to_their_rows(dev, dtype, unsplit):
    lens, heads, d = [700, 90], 8, 128
    c, table = filled(113, lens, 2, 16, d)
    q = rows_of(114, 2, heads * d, 0, DT[dtype], dev)
    o, z, _ = decoded(dev, c, table, q, heads, dtype, lens, 700, unsplit=unsplit)
    bad = q.clone()
    bad[0, 1 * d + 5], bad[0, 6 * d + 77], bad[1, 3 * d] = math.inf, math.nan, -math.inf
    o1, z1, err = decoded(dev, c, table, bad, heads, dtype, lens, 700, unsplit=unsplit)
    hit = torch.zeros(2, heads, dtype=torch.bool)
    hit[0, [1, 6]] = hit[1, 3] = True
    assert err == 0
    assert not torch.isfinite(o1.unflatten(1, (heads, d))[hit]).any()
    assert torch.isfinite(o1.unflatten(1, (heads, d))[~hit]).all() and torch.isfinite(z1[~hit]).all()
    if unsplit:
        assert torch.equal(o1.unflatten(1, (heads, d))[~hit], o.unflatten(1, (heads, d))[~hit])
        assert torch.equal(z1[~hit], z[~hit])


@pytest.mark.parametrize("heads,kv_heads,d,lens", [(4, 2, 64, [33, 0, 700] * 128), (1024, 1024, 64, [40, 17]),
                                                   (2048, 16, 128, [5, 300])])
def test_the_most_requests_and_heads(dev, heads, kv_heads, d, lens):
    c, table = filled(115, lens, kv_heads, 16, d)
    q = rows_of(116, len(lens), heads * d, 0, torch.bfloat16, dev, loud=0.5)
    for unsplit in (False, True):
        o, z, err = decoded(dev, c, table, q, heads, "bf16", lens, max(lens), unsplit=unsplit)
        assert err == 0
        for b in {0, 1, len(lens) // 2, len(lens) - 1}:
            if lens[b] == 0:
                assert (o[b] == 0).all() and (z[b] == -math.inf).all()
                continue
            over, over_z = excess(c, table, q, heads, "bf16", b, lens[b], o, z, d ** -0.5)
            assert over <= 1 and over_z <= 1


def test_two_captured_steps_with_one_workspace(dev):
    """Two graphs of steps with different shapes whose workspace is one, replayed in turn on one stream."""
    cases = []
    for seed, lens, heads, hk, d in ((117, [3000, 5, 900], 8, 2, 128), (118, [2500] * 4, 16, 1, 64)):
        c, table = filled(seed, lens, hk, 16, d)
        shape = shape_of(len(lens), heads, hk, d, 16, c.blocks, table.shape[1], "bf16")
        q = rows_of(seed, len(lens), heads * d, 0, torch.bfloat16, dev)
        want = decoded(dev, c, table, q, heads, "bf16", lens, max(lens))[0]
        cases.append(dict(shape=shape, bound=max(lens), size=hs.hs_kv8_decode_workspace_bytes(shape, max(lens)), want=want,
                          args=[x.to(dev) for x in (q, c.image(), table, torch.tensor(lens, dtype=torch.int32))],
                          o=torch.zeros(len(lens), heads * d, dtype=torch.bfloat16, device=dev)))
    size = max(x["size"] for x in cases)
    ws = torch.empty(size, dtype=torch.uint8, device=dev)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for x in cases:
            x["graph"] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(x["graph"], stream=stream):
                hs.hs_kv8_decode(x["shape"], *x["args"], x["bound"], x["o"], None, ws, size)
        for _ in range(20):
            for x in cases:
                x["o"].zero_()
                x["graph"].replay()
        stream.synchronize()
    for x in cases:
        assert torch.equal(x["o"].cpu(), x["want"])
