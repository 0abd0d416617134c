"""The full-attention calls and hs_kv_append on the GPU, through the C ABI, against float64.

Bounds are per output element, from the roundings that the calls document (tests/attn_helpers.py:
Problem.row): half a step of the element type for each weight and for the output, float32 steps
for scores and sums.  Everything outside a request's keys is NaN, so that a masked place that
reaches a result shows.
"""
import math

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.attn_helpers import (DT, HSDT, Problem, cu_of, guarded, run_decode, run_prefill, workspace)
from tests.gpu_helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


# ---- append --------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kv_heads,d,page,rows,pad", [
    (1, 64, 16, 1, 0), (2, 64, 16, 33, 8), (4, 128, 16, 257, 512), (8, 128, 32, 1000, 0),
    (3, 128, 64, 77, 24), (4, 64, 256, 600, 0), (72, 128, 16, 5, 8), (200, 64, 16, 40, 0)])
def test_append_writes_each_row_to_its_slot(dev, dtype, kv_heads, d, page, rows, pad):
    g = torch.Generator().manual_seed(rows)
    dt = DT[dtype]
    blocks = -(-rows // page) + 2
    inner = kv_heads * d
    kv = torch.randn(2, rows, inner + pad, generator=g).to(dt)
    kv[0, 0, :2] = torch.tensor([math.nan, math.inf])      # moved, not computed on
    slots = torch.randperm(blocks * page, generator=g)[:rows]
    slots[rows // 2] = -1                                  # padding
    cache = torch.full((blocks, 2, page, kv_heads, d), -3.0, dtype=dt)
    want = cache.clone()
    for r, s in enumerate(slots.tolist()):
        if s >= 0:
            for i in range(2):
                want[s // page, i, s % page] = kv[i, r, :inner].reshape(kv_heads, d)
    got, kv_d, err = cache.to(dev), kv.to(dev), torch.zeros(1, dtype=torch.int32, device=dev)
    shape = hs.make_attn_shape(0, kv_heads, kv_heads, d, page, blocks, 0, HSDT[dtype])
    hs.hs_kv_append(shape, kv_d[0], kv_d[1], inner + pad, slots.to(dev), rows, got, err)
    torch.cuda.synchronize()
    assert err.item() == 0
    assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))


def test_append_reports_slots_beyond_the_cache(dev):
    k = torch.ones(3, 1, 64, dtype=torch.bfloat16, device=dev)
    cache = torch.zeros(2, 2, 16, 1, 64, dtype=torch.bfloat16, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    shape = hs.make_attn_shape(0, 1, 1, 64, 16, 2, 0)
    slots = torch.tensor([32, 5, 1 << 40], device=dev)
    hs.hs_kv_append(shape, k, k, 0, slots, 3, cache, err)
    torch.cuda.synchronize()
    assert err.item() == hs.HS_DEVERR_BLOCK_OOB
    assert cache[0, :, 5].eq(1).all() and cache.sum().item() == 2 * 64


# ---- prefill -------------------------------------------------------------------------------

LENGTHS = {
    "one token": ([0], [1]),
    "small": ([0, 5, 0, 3, 130], [1, 1, 2, 0, 3]),
    "tile edges": ([0, 0, 0, 63, 128], [127, 128, 129, 65, 1]),
    "ragged": ([200, 0, 17, 1000], [61, 40, 0, 7]),
    "page edges": ([15, 16, 17, 31], [1, 16, 15, 2]),
}


@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv_heads,d,page,dtype", [
    (1, 1, 64, 16, "bf16"), (4, 1, 128, 16, "bf16"), (6, 2, 128, 32, "fp16"), (8, 4, 64, 64, "fp16"),
    (14, 2, 128, 128, "bf16"), (16, 1, 64, 256, "bf16"), (2, 2, 128, 16, "fp16")])
def test_prefill(dev, lengths, heads, kv_heads, d, page, dtype):
    pos0, n = LENGTHS[lengths]
    p = Problem(1, heads, kv_heads, d, page, dtype, [a + b for a, b in zip(pos0, n)], sum(n))
    run_prefill(p, pos0, n, dev).check(p.prefill_rows(pos0, n, cu_of(n)))


@pytest.mark.parametrize("unsplit", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,dtype,pos0,n", [
    (4, 1, 128, "bf16", [1500], [300]),          # few rows, many keys
    (2, 2, 128, "fp16", [0], [700]),             # a whole prompt, a head per KV head
    (8, 2, 64, "bf16", [4000, 0, 900], [5, 333, 130]),
    (128, 1, 64, "fp16", [100, 700], [3, 2]),    # a group as tall as a tile
    (5, 1, 128, "bf16", [2100], [70])])          # a group that divides no tile
def test_prefill_over_many_keys(dev, unsplit, heads, kv_heads, d, dtype, pos0, n):
    p = Problem(2, heads, kv_heads, d, 16, dtype, [a + b for a, b in zip(pos0, n)], sum(n))
    run_prefill(p, pos0, n, dev, unsplit=unsplit).check(p.prefill_rows(pos0, n, cu_of(n)))


def test_prefill_strides_gaps_and_no_lse(dev):
    """Rows with gaps between requests and elements between rows; nothing else is written."""
    pos0, n, cu = [30, 7], [20, 9], [2, 25, 40]
    p = Problem(3, 6, 2, 128, 16, "bf16", [50, 16], 40, pad=72)
    out = run_prefill(p, pos0, n, dev, cu=cu)
    out.check(p.prefill_rows(pos0, n, cu))
    q, cache, table, _ = out.keep
    o = torch.full_like(out.o, math.nan)
    shape = p.shape(2)
    size = hs.hs_attn_prefill_workspace_bytes(shape, pos0, n)
    ws = workspace(size, dev)
    hs.hs_attn_prefill(shape, q, cache, table, o, None, pos0, n, cu, ws, size, out.err)
    torch.cuda.synchronize()
    assert torch.equal(o.view(torch.int16), out.o.view(torch.int16))


@pytest.mark.parametrize("sharp,slope", [(30.0, 0.0), (1.0, 60.0), (1.0, -60.0), (0.01, 0.0)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_prefill_of_sharp_rising_and_falling_scores(dev, sharp, slope, dtype):
    """The running maximum jumps, climbs along all keys, or never moves again."""
    p = Problem(4, 4, 1, 128, 16, dtype, [900], 60, sharp=sharp, slope=slope)
    run_prefill(p, [840], [60], dev).check(p.prefill_rows([840], [60], [0, 60]))


@pytest.mark.parametrize("heads,kv_heads,d,page", [(4, 1, 128, 16), (3, 1, 64, 32), (8, 8, 128, 64)])
def test_unsplit_tails_equal_the_recomputation_bitwise(dev, heads, kv_heads, d, page):
    N = 611
    p = Problem(5, heads, kv_heads, d, page, "bf16", [N], N)
    full = run_prefill(p, [0], [N], dev, unsplit=True)
    for c in (64, 128, 200, 384, 555, 610):
        tail = Problem(5, heads, kv_heads, d, page, "bf16", [N], N)
        out = run_prefill(tail, [c], [N - c], dev, cu=[c, N], unsplit=True)
        assert torch.equal(out.o[c:N].view(torch.int16), full.o[c:N].view(torch.int16)), c
        assert torch.equal(out.lse[c:N], full.lse[c:N]), c


def test_equal_calls_give_equal_bits(dev):
    pos0, n = [1900, 0, 60], [70, 200, 1]
    p = Problem(6, 8, 2, 128, 16, "bf16", [a + b for a, b in zip(pos0, n)], sum(n))
    first, again = (run_prefill(p, pos0, n, dev) for _ in range(2))
    assert torch.equal(first.o.view(torch.int16), again.o.view(torch.int16))
    assert torch.equal(first.lse[:-1], again.lse[:-1])


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [0, 40, 127, 128, 140, 149])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_keeps_later_values_out_of_earlier_rows(dev, bad, at, d):
    """A value that is not finite reaches the rows at and behind its position, in its column."""
    n = 150
    p = Problem(7, 2, 1, d, 16, "bf16", [n], n)
    clean = run_prefill(p, [0], [n], dev)
    blk, off = p.table[0, at // 16].item(), at % 16
    p.cache[blk, 1, off, 0, 5] = bad
    out = run_prefill(p, [0], [n], dev)
    o, ref = (x.o[:n, :2 * d].reshape(n, 2, d).cpu() for x in (out, clean))
    assert torch.equal(o[:at].view(torch.int16), ref[:at].view(torch.int16))
    keep = torch.arange(d) != 5
    assert torch.equal(o[:, :, keep].view(torch.int16), ref[:, :, keep].view(torch.int16))
    assert not torch.isfinite(o[at:, :, 5]).any()


@pytest.mark.parametrize("heads,kv_heads,d,dtype", [(2, 2, 128, "bf16"), (2, 2, 64, "fp16"), (6, 2, 128, "fp16"),
                                                    (6, 2, 64, "bf16")])
@pytest.mark.parametrize("n", [128, 300])
def test_every_place_of_a_diagonal_tile_is_searched(dev, n, heads, kv_heads, d, dtype):
    """One value that is not finite at a time, walking over the rows and columns (and so over the chunks
    that the searching lanes hold) in the places that only some rows see: the rows in front keep their
    values, those at and behind it lose that column alone."""
    p = Problem(31, heads, kv_heads, d, 16, dtype, [n], n)
    clean = run_prefill(p, [0], [n], dev).o.cpu()[:n, :heads * d].reshape(n, kv_heads, heads // kv_heads, d)
    good = p.cache.clone()
    for i in range(40):
        at, col, kvh, bad = (1 + 37 * i) % n, (11 * i) % d, i % kv_heads, (math.nan, math.inf, -math.inf)[i % 3]
        p.cache = good.clone()
        p.cache[p.table[0, at // 16].long(), 1, at % 16, kvh, col] = bad
        o = run_prefill(p, [0], [n], dev).o.cpu()[:n, :heads * d].reshape(n, kv_heads, heads // kv_heads, d)
        hit = torch.zeros(n, kv_heads, 1, d, dtype=torch.bool)
        hit[at:, kvh, :, col] = True
        hit = hit.expand_as(o)
        assert not torch.isfinite(o[hit]).any(), (at, col, kvh)
        assert torch.equal(o[~hit], clean[~hit]), (at, col, kvh)


def test_prefill_reports_pages_outside_the_cache(dev):
    """Rows that do not attend to the bad page keep their values; nothing faults."""
    p = Problem(8, 2, 1, 128, 16, "bf16", [100, 50], 150)
    p.table[0, 3] = p.blocks
    out = run_prefill(p, [0, 0], [100, 50], dev)
    assert out.err.item() == hs.HS_DEVERR_BLOCK_OOB
    out.err.zero_()
    good = {r[0]: r for r in p.prefill_rows([0, 0], [100, 50], [0, 100, 150])}
    o = out.o.cpu()
    for r in list(range(48)) + list(range(100, 150)):
        got = o[r, :256].double().reshape(2, 128)
        assert ((got - good[r][1]).abs() <= good[r][3]).all(), r
    p.table[0, 3] = -7
    assert run_prefill(p, [0, 0], [100, 50], dev).err.item() == hs.HS_DEVERR_BLOCK_OOB


@pytest.mark.parametrize("at", [0, 100, 140])
def test_prefill_keeps_later_keys_out_of_earlier_rows(dev, at):
    """A key of NaN reaches the rows at and behind its position."""
    n = 150
    p = Problem(21, 2, 1, 128, 16, "fp16", [n], n)
    clean = run_prefill(p, [0], [n], dev)
    p.cache[p.table[0, at // 16].item(), 0, at % 16] = math.nan
    out = run_prefill(p, [0], [n], dev)
    assert torch.equal(out.o[:at].view(torch.int16), clean.o[:at].view(torch.int16))
    assert torch.equal(out.lse[:at], clean.lse[:at])
    assert torch.isnan(out.o[at:n, :256]).all()


def test_prefill_keeps_a_bad_query_to_itself(dev):
    p = Problem(22, 4, 2, 128, 16, "bf16", [300], 40)
    clean = run_prefill(p, [260], [40], dev)
    p.q[7, 130] = math.nan            # token 7, head 1
    p.q[20, 0] = math.inf             # token 20, head 0
    out = run_prefill(p, [260], [40], dev)
    o, ref = (x.o[:40, :512].reshape(40, 4, 128).cpu() for x in (out, clean))
    bad = torch.zeros(40, 4, dtype=torch.bool)
    bad[7, 1] = bad[20, 0] = True
    assert torch.isnan(o[bad]).all()
    assert torch.equal(o[~bad].view(torch.int16), ref[~bad].view(torch.int16))


@pytest.mark.parametrize("unsplit", [False, True])
def test_prefill_of_the_largest_batch(dev, unsplit):
    """384 requests of 0 to 3 tokens, the first and last without one, some tables sharing pages."""
    n = [0] + [(5 * b) % 4 for b in range(1, 383)] + [0]
    pos0 = [(41 * b) % 150 for b in range(384)]
    p = Problem(23, 6, 2, 64, 16, "bf16", [a + b for a, b in zip(pos0, n)], sum(n))
    for b in range(4, 384, 4):        # the pages in front of the new tokens are another request's
        whole = min(pos0[b], pos0[b - 1]) // 16
        p.table[b, :whole] = p.table[b - 1, :whole]
        for x in (p.K, p.V):
            x[b][:whole * 16] = x[b - 1][:whole * 16]
    run_prefill(p, pos0, n, dev, unsplit=unsplit).check(p.prefill_rows(pos0, n, cu_of(n)))


@pytest.mark.parametrize("scale", [0.003, 0.7])
def test_scales(dev, scale):
    p = Problem(24, 4, 2, 64, 16, "fp16", [333, 20], 25)
    p.scale = scale
    run_prefill(p, [310, 18], [23, 2], dev, scale=scale).check(p.prefill_rows([310, 18], [23, 2], [0, 23, 25]))


def test_captured_prefill_and_shared_decode_replay_with_new_contents(dev):
    """The lists of a captured prefill are part of the graph; queries, pages and tables are read anew."""
    pos0, n = [700, 3], [90, 40]
    a, b = (Problem(25 + i, 8, 2, 128, 16, "bf16", [790, 43], 130, prefix_len=200) for i in range(2))
    shape, side = a.shape(2), torch.cuda.Stream()
    size = max(hs.hs_attn_prefill_workspace_bytes(shape, pos0, n),
               hs.hs_attn_decode_shared_workspace_bytes(shape, 200, 790))
    q, cache, table, pre = (x.to(dev) for x in (a.q, a.cache, a.table, a.prefix_table))
    lens = torch.tensor([790, 43], dtype=torch.int32, device=dev)
    ws, err = workspace(size, dev), torch.zeros(1, dtype=torch.int32, device=dev)
    o, o2 = torch.zeros_like(q), torch.zeros_like(q)
    lse, lse2 = (torch.zeros(131, 8, device=dev) for _ in range(2))

    def calls():
        hs.hs_attn_prefill(shape, q, cache, table, o, lse, pos0, n, [0, 90, 130], ws, size, err, side)
        hs.hs_attn_decode_shared(shape, q, cache, pre, 200, table, lens, 790, o2, lse2, ws, size, err, side)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for p in (a, b, a):
        for x, y in ((q, p.q), (cache, p.cache), (table, p.table), (pre, p.prefix_table)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert err.item() == 0
        for got, rows in ((o, p.prefill_rows(pos0, n, [0, 90, 130])), (o2, p.decode_rows([790, 43]))):
            for r, want, _, bound, _ in rows:
                assert ((got[r, :1024].cpu().double().reshape(8, 128) - want).abs() <= bound).all(), r
    assert guarded(ws, size)


# ---- decode --------------------------------------------------------------------------------


@pytest.mark.parametrize("unsplit", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,page,dtype", [
    (1, 1, 64, 16, "bf16"), (16, 4, 128, 16, "bf16"), (6, 2, 128, 32, "fp16"), (8, 8, 64, 64, "fp16"),
    (14, 2, 128, 128, "bf16"), (32, 1, 64, 256, "bf16"), (128, 1, 128, 16, "fp16")])
@pytest.mark.parametrize("kv_len", [[1], [0], [5000], [0, 1, 15, 16, 17, 127, 128, 129, 300, 0, 1030]],
                         ids=lambda x: "-".join(map(str, x)))
def test_decode(dev, unsplit, heads, kv_heads, d, page, dtype, kv_len):
    p = Problem(9, heads, kv_heads, d, page, dtype, kv_len, len(kv_len))
    run_decode(p, kv_len, max(kv_len), dev, shared=False, unsplit=unsplit).check(p.decode_rows(kv_len))


def test_decode_of_the_largest_batch(dev):
    kv_len = [(37 * b) % 70 for b in range(384)]
    p = Problem(10, 4, 2, 64, 16, "bf16", kv_len, 384, pad=8)
    run_decode(p, kv_len, 80, dev, shared=False).check(p.decode_rows(kv_len))


def test_decode_bound_above_the_lengths(dev):
    """The bound is a bound: any one at or above the lengths gives the same values."""
    kv_len = [3, 700, 64]
    p = Problem(11, 8, 2, 128, 16, "bf16", kv_len, 3)
    p.table = torch.cat((p.table, torch.full((3, 400), -1, dtype=torch.int32)), dim=1)
    for bound in (700, 701, 5000):
        run_decode(p, kv_len, bound, dev, shared=False).check(p.decode_rows(kv_len))


@pytest.mark.parametrize("shared", [False, True])
def test_decode_reports_lengths_outside_the_bound(dev, shared):
    """The request is skipped; the others are answered."""
    p = Problem(12, 4, 2, 128, 16, "bf16", [40, 40, 40, 40], 4, prefix_len=100 if shared else 0)
    out = run_decode(p, [40, 41, -1, 20], 40, dev, shared=shared)
    assert out.err.item() == hs.HS_DEVERR_LENGTH
    out.err.zero_()
    rows = list(p.decode_rows([40, 0, 0, 20]))
    out.check([rows[0], rows[3]])


@pytest.mark.parametrize("shared", [False, True])
def test_decode_reports_pages_outside_the_cache(dev, shared):
    kv_len = [40, 33]
    p = Problem(13, 4, 2, 128, 16, "bf16", kv_len, 2, prefix_len=50 if shared else 0)
    p.table[1, 2] = p.blocks + 5
    out = run_decode(p, kv_len, 40, dev, shared=shared)
    assert out.err.item() == hs.HS_DEVERR_BLOCK_OOB
    out.err.zero_()
    got = out.o.cpu()[0, :512].double().reshape(4, 128)
    want = next(p.decode_rows(kv_len))
    assert ((got - want[1]).abs() <= want[3]).all()


def test_captured_decode_replays_as_lengths_grow(dev):
    """Three steps from one graph: the lengths, the table, q and the cache change in place."""
    steps = [[5, 130, 0], [6, 131, 1], [300, 17, 2]]
    top = [max(x) for x in zip(*steps)]
    p = Problem(14, 8, 2, 128, 16, "bf16", top, 3)
    p.table = torch.cat((p.table, torch.full((3, 20 - p.table.shape[1]), -1, dtype=torch.int32)), dim=1)
    shape = p.shape(3)
    size = hs.hs_attn_decode_workspace_bytes(shape, 320)
    q, cache, table, ws = p.q.to(dev), p.cache.to(dev), p.table.to(dev), workspace(size, dev)
    lens = torch.zeros(3, dtype=torch.int32, device=dev)
    o, lse = torch.zeros_like(q), torch.zeros(3, 8, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    side = torch.cuda.Stream()

    def step(stream):
        hs.hs_attn_decode(shape, q, cache, table, lens, 320, o, lse, ws, size, err, stream)
    step(None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for kv_len in steps:
        lens.copy_(torch.tensor(kv_len, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert err.item() == 0
        for r, want, want_lse, bound, bound_lse in p.decode_rows(kv_len):
            got = o[r, :1024].cpu().double().reshape(8, 128)
            assert ((got - want).abs() <= bound).all(), (kv_len, r)
    assert guarded(ws, size)


# ---- decode behind a shared prefix ---------------------------------------------------------


@pytest.mark.parametrize("unsplit", [False, True])
@pytest.mark.parametrize("prefix", [0, 1, 16, 100, 129, 2500])
@pytest.mark.parametrize("heads,kv_heads,d,page,dtype,kv_len", [
    (4, 4, 64, 16, "bf16", [0, 1, 17]),
    (16, 4, 128, 16, "bf16", [1, 0, 64, 129, 33, 700, 2, 16]),
    (10, 2, 128, 32, "fp16", [(13 * b) % 47 for b in range(70)]),
    (16, 1, 64, 64, "bf16", [(29 * b) % 90 for b in range(33)]),
    (2, 1, 128, 16, "fp16", [5])])
def test_decode_shared(dev, unsplit, prefix, heads, kv_heads, d, page, dtype, kv_len):
    p = Problem(15, heads, kv_heads, d, page, dtype, kv_len, len(kv_len), prefix_len=prefix)
    run_decode(p, kv_len, max(kv_len), dev, unsplit=unsplit).check(p.decode_rows(kv_len))


def test_shared_prefix_without_suffixes(dev):
    p = Problem(16, 8, 2, 128, 16, "bf16", [0] * 9, 9, prefix_len=777)
    run_decode(p, [0] * 9, 0, dev).check(p.decode_rows([0] * 9))


@pytest.mark.parametrize("sharp,slope", [(30.0, 0.0), (1.0, 60.0)])
def test_decode_shared_of_sharp_and_rising_scores(dev, sharp, slope):
    kv_len = [90, 1, 300]
    p = Problem(17, 8, 2, 128, 16, "bf16", kv_len, 3, prefix_len=1000, sharp=sharp, slope=slope)
    run_decode(p, kv_len, 300, dev).check(p.decode_rows(kv_len))


# ---- streams -------------------------------------------------------------------------------


def test_calls_at_once_on_two_streams(dev):
    """Each with a workspace of its own, on streams that are not the current one."""
    kv = [[900, 40], [77, 2000]]
    ps = [Problem(18 + i, 8, 2, 128, 16, "bf16", kv[i], 2) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in ps]
    outs, held = [], []
    for p, s, k in zip(ps, streams, kv):
        pos0, n = [x - 1 for x in k], [1, 1]
        from tests.attn_helpers import Outputs
        out = Outputs(p, dev)
        shape = p.shape(2)
        size = hs.hs_attn_prefill_workspace_bytes(shape, pos0, n)
        held.append((shape, p.q.to(dev), p.cache.to(dev), p.table.to(dev), workspace(size, dev), size, pos0, n, s))
        outs.append(out)
    torch.cuda.synchronize()
    for _ in range(20):
        for out, (shape, q, cache, table, ws, size, pos0, n, s) in zip(outs, held):
            hs.hs_attn_prefill(shape, q, cache, table, out.o, out.lse, pos0, n, [0, 1, 2], ws, size,
                               out.err, s)
    for p, out, h in zip(ps, outs, held):
        out.check(p.prefill_rows(h[6], h[7], [0, 1, 2]))


# ---- small weights -------------------------------------------------------------------------


@pytest.mark.parametrize("at", [0, 2500, 4999])
@pytest.mark.parametrize("call", ["prefill", "unsplit", "decode", "shared"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_many_small_weights_beside_a_large_one(dev, dtype, call, at):
    """4,999 keys with 2^-25.5 of the weight of one more each, below half the smallest fp16 number: the
    values of the small ones are 1, of the large one 0.  Weights are rounded with 2^8 of room below the
    largest, so that one of 2^-25.5 is off by at most half a step of 2^-24 beside 2^-17.5, which is 2^-7.5 of
    it; the output, near 2^-13.2, is rounded in steps of 2^-24 in fp16, by 2^-8 of it in bf16.  lse: the
    scale's two roundings and the result's, each at most 2^-24 of 25.5."""
    n, d, dt = 5000, 64, DT[dtype]
    cache = torch.zeros(20, 2, 256, 1, d, dtype=dt, device=dev)
    cache[:, 1] = 1
    cache[at // 256, 0, at % 256, 0, 0] = 16
    cache[at // 256, 1, at % 256] = 0
    q, o = torch.zeros(1, d, dtype=dt, device=dev), torch.full((1, d), math.nan, dtype=dt, device=dev)
    q[0, 0] = 1
    lse = torch.zeros(1, 1, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    table = torch.arange(20, dtype=torch.int32, device=dev)[None]
    scale = 25.5 * math.log(2) / 16
    shape = hs.make_attn_shape(1, 1, 1, d, 256, 20, 20, HSDT[dtype], scale=scale, unsplit=call == "unsplit")
    if call in ("prefill", "unsplit"):
        size = hs.hs_attn_prefill_workspace_bytes(shape, [n - 1], [1])
        hs.hs_attn_prefill(shape, q, cache, table, o, lse, [n - 1], [1], [0, 1], workspace(size, dev), size,
                           err)
    elif call == "decode":
        size = hs.hs_attn_decode_workspace_bytes(shape, n)
        lens = torch.tensor([n], dtype=torch.int32, device=dev)
        hs.hs_attn_decode(shape, q, cache, table, lens, n, o, lse, workspace(size, dev), size, err)
    else:
        front = 2048
        size = hs.hs_attn_decode_shared_workspace_bytes(shape, front, n - front)
        lens = torch.tensor([n - front], dtype=torch.int32, device=dev)
        own = torch.zeros_like(table)
        own[0, :12] = table[0, 8:]
        hs.hs_attn_decode_shared(shape, q, cache, table[0], front, own, lens, n - front, o, lse,
                                 workspace(size, dev), size, err)
    torch.cuda.synchronize()
    assert err.item() == 0
    small = (n - 1) * 2.0 ** -25.5
    want = small / (1 + small)
    assert (o.double() / want - 1).abs().max().item() <= 2.0 ** -7.5 + 2.0 ** -8 + 2.0 ** -16
    assert abs(lse.item() - (scale * 16 + math.log1p(small))) <= 2.0 ** -17
