"""Rotary positions and the 8-bit cache on the GPU against their definitions (tests/kv8_helpers.py): every byte of
the cache, every output within bounds of the roundings on its way."""
import math

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.gpu_helpers import device
from tests.kv8_helpers import DT, G, TINY, U, VALUES, Cache, attended, filled, keys_of, shape_of, turned

pytestmark = pytest.mark.gpu

PLAIN = dict(base=10000.0)


@pytest.fixture(scope="module")
def dev():
    return device()


def fresh_err(dev):
    return torch.zeros(1, dtype=torch.int32, device=dev)


def rows_of(seed, n, width, pad, dt, dev, loud=1.0):
    """n random rows of `width` with `pad` elements of NaN behind each, and a row of NaN behind the last."""
    g = torch.Generator().manual_seed(seed)
    x = torch.full((n + 1, width + pad), math.nan, dtype=dt)
    x[:n, :width] = (torch.randn(n, width, generator=g) * loud).to(dt)
    return x


# ---- positions ---------------------------------------------------------------------------

ROPE = [  # heads, kv heads, d, dims, layout, dtype, rows, pad
    (4, 4, 64, 64, 0, "bf16", 1, 0), (16, 4, 128, 128, 0, "fp16", 33, 8), (32, 8, 128, 64, 1, "bf16", 7, 0),
    (3, 1, 128, 96, 1, "fp16", 19, 24), (14, 2, 64, 16, 0, "fp16", 5, 0), (5, 5, 128, 32, 0, "bf16", 700, 8),
    (8, 8, 64, 48, 1, "bf16", 2500, 0), (128, 1, 128, 112, 0, "bf16", 3, 0)]


@pytest.mark.parametrize("heads,kv_heads,d,dims,layout,dtype,rows,pad", ROPE)
def test_rope(dev, heads, kv_heads, d, dims, layout, dtype, rows, pad):
    rope = hs.hs_rope_plan(dims, layout, 500000.0, hs.HS_ROPE_TURNS, 8.0, 8192, 1.0, 32.0, 1.2)
    width = (heads + kv_heads) * d
    x = rows_of(1, rows, width, pad, DT[dtype], dev)
    g = torch.Generator().manual_seed(2)
    pos = torch.randint(-200000, 2000000, (rows,), generator=g)
    pos[:3] = torch.tensor([0, 1, 2 ** 31 - 1])[:rows]
    shape = shape_of(0, heads, kv_heads, d, 16, 1, 1, dtype)
    xd, pd = x.to(dev), pos.to(dev)
    q = torch.full((rows + 1, heads * d + 16), math.nan, dtype=DT[dtype], device=dev)
    k = torch.full((rows + 1, kv_heads * d), math.nan, dtype=DT[dtype], device=dev)
    hs.hs_rope_apply(shape, rope, xd, xd[:, heads * d:], width + pad, pd, rows, q, heads * d + 16, k, 0)
    torch.cuda.synchronize()
    want, err = turned(rope, x[:rows, :width].double().reshape(rows, -1, d), pos.tolist())
    got = torch.cat((q.cpu()[:rows, :heads * d], k.cpu()[:rows]), dim=1).double().reshape(rows, -1, d)
    bound = err + U[dtype] * (want.abs() + err) + TINY[dtype]
    bound[..., dims:] = 0
    off = (got - want).abs()
    assert (off <= bound).all(), (off - bound).max()
    assert torch.isnan(q[rows:]).all() and torch.isnan(k[rows:]).all() and torch.isnan(q[:, heads * d:]).all()
    # in place, and each alone, give the same bits
    hs.hs_rope_apply(shape, rope, xd, None, width + pad, pd, rows, xd, width + pad, None, 0)
    hs.hs_rope_apply(shape, rope, None, xd[:, heads * d:], width + pad, pd, rows, None, 0, xd[:, heads * d:], width + pad)
    torch.cuda.synchronize()
    assert torch.equal(xd[:rows, :heads * d], q[:rows, :heads * d])
    assert torch.equal(xd[:rows, heads * d:width], k[:rows])
    assert torch.isnan(xd[:rows, width:]).all() and torch.isnan(xd[rows]).all()


def test_rope_keeps_what_is_not_finite_in_its_pair(dev):
    shape, rope = shape_of(0, 2, 1, 64, 16, 1, 1, "bf16"), hs.hs_rope_plan(64, hs.HS_ROPE_HALF, **PLAIN)
    x = rows_of(3, 4, 128, 0, torch.bfloat16, dev)
    bad = x.clone()
    bad[1, 5], bad[2, 64 + 40] = math.inf, math.nan
    pos = torch.tensor([3, 4, 5, 6], device=dev)
    out = []
    for y in (x, bad):
        q = torch.empty(4, 128, dtype=torch.bfloat16, device=dev)
        hs.hs_rope_apply(shape, rope, y.to(dev), None, 0, pos, 4, q, 0, None, 0)
        out.append(q.cpu())
    hit = torch.zeros(4, 128, dtype=torch.bool)
    hit[1, [5, 37]] = hit[2, [64 + 8, 64 + 40]] = True
    assert not torch.isfinite(out[1][hit]).any()
    assert torch.equal(out[0][~hit], out[1][~hit])


# ---- appending ---------------------------------------------------------------------------


class Layer:
    """A cache on the GPU and its definition beside it, appended to alike."""

    def __init__(self, dev, kv_heads, d, page, dtype, blocks, heads=None):
        self.dev, self.dtype, self.d, self.hk, self.page = dev, dtype, d, kv_heads, page
        self.heads = heads or kv_heads
        self.ref = Cache(blocks, kv_heads, page, d)
        self.shape = shape_of(0, self.heads, kv_heads, d, page, blocks, 1, dtype)
        assert hs.hs_kv8_block_bytes(self.shape) == self.ref.size()
        self.cache = self.ref.image().to(dev)
        self.err = fresh_err(dev)

    def append(self, seed, slots, loud=1.0, pad=0, change=None):
        n, w = len(slots), self.hk * self.d
        x = rows_of(seed, n, 2 * w, pad, DT[self.dtype], self.dev, loud)
        if change:
            change(x)
        xd = x.to(self.dev)
        hs.hs_kv8_append(self.shape, xd, xd[:, w:], 2 * w + pad, torch.tensor(slots, device=self.dev), n, self.cache,
                         self.err)
        y = x[:n, :2 * w].double().reshape(n, 2, self.hk, self.d)
        self.ref.append(torch.where(torch.isfinite(y), y, torch.full_like(y, math.nan)), slots)

    def check(self, err=0):
        torch.cuda.synchronize()
        assert self.err.item() == err
        got, want = self.cache.cpu(), self.ref.image()
        # NaN may have either sign
        n = self.ref.kv_heads * 2 * self.page * self.d
        for x in (got, want):
            x[:, :n] = torch.where(x[:, :n] % 128 == 127, torch.full_like(x[:, :n], 127), x[:, :n])
        assert torch.equal(got, want)


APPEND = [(1, 64, 16, "bf16"), (4, 128, 16, "bf16"), (2, 64, 32, "fp16"), (8, 128, 32, "fp16"), (3, 128, 256, "bf16"),
          (5, 64, 64, "bf16")]


@pytest.mark.parametrize("kv_heads,d,page,dtype", APPEND)
def test_append_step_by_step(dev, kv_heads, d, page, dtype):
    """Prompts of odd lengths and then single tokens that grow and shrink, so that groups take larger scales: every byte."""
    y = Layer(dev, kv_heads, d, page, dtype, 12 if page < 64 else 4)
    rooms = [(0, 19), (3 * page, 1), (2 * page, 15)]                # first slot, tokens
    slots = [a + i for a, n in rooms for i in range(n)]
    y.append(1, slots, pad=8)
    y.check()
    ends = [a + n for a, n in rooms]
    for step in range(20):
        y.append(10 + step, ends, loud=2.0 ** ((step * 7) % 11 - 5))
        ends = [e + 1 for e in ends]
        if step % 6 == 0:
            y.check()
    y.check()


@pytest.mark.parametrize("kv_heads,d,page,dtype", APPEND)
@pytest.mark.parametrize("rows", [1, 16, 17, 200, 1500])
def test_append_of_many_rows(dev, kv_heads, d, page, dtype, rows):
    """Requests of odd lengths at odd places of their groups, rows of a group in any order, padding between requests."""
    blocks = max(3, 3 * -(-rows // page) + 3)
    y = Layer(dev, kv_heads, d, page, dtype, blocks)
    g = torch.Generator().manual_seed(rows)
    y.append(5, list(range(0, blocks * page, 16)), loud=0.25)           # every group is begun
    order = torch.randperm(blocks, generator=g).tolist()
    slots = []
    while len(slots) < rows and order:
        n = int(torch.randint(1, 2 * page, (1,), generator=g))
        begin = int(torch.randint(0, page, (1,), generator=g))
        pages = [order.pop() for _ in range(min(len(order), -(-(begin + n) // page)))]
        one = [b * page + i for b in pages for i in range(page)][begin:begin + n]
        # any order inside a group
        by = {}
        for s in one:
            by.setdefault(s // G, []).append(s)
        for part in by.values():
            slots += [part[i] for i in torch.randperm(len(part), generator=g).tolist()]
        slots += [-1] * int(torch.randint(0, 3, (1,), generator=g))
    y.append(6, slots, loud=3.0, pad=16)
    y.check()


def test_append_scales_at_their_borders(dev):
    """Largest magnitudes at 448 2^e and one step around it, zeros, the type's smallest and largest."""
    for dtype in ("bf16", "fp16"):
        info = torch.finfo(DT[dtype])
        step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -10
        tops = [448.0, 448.0 * (1 + step / 1.75), 448.0 * (1 - step / 1.75), 0.0, 7.0, 3.5, 0.875, 1.75 * 2.0 ** -14, info.max,
                info.smallest_normal, info.smallest_normal * info.eps, 2.0 ** -20, 448.0 * 2.0 ** -6, 1.0]
        y = Layer(dev, 2, 64, 16, dtype, len(tops))

        def change(x):
            for i, t in enumerate(tops):
                x[i, :256] = 0.0
                x[i, 3] = -t
                x[i, 128 + 70] = t
                x[i, 1] = t / 3
        y.append(1, [16 * i for i in range(len(tops))], change=change)
        y.check()
        for i, t in enumerate(tops):
            s = y.ref.scales[i, 0, 0, 0].item()
            assert s == 2.0 ** -126 or s / 2 < torch.tensor(t, dtype=DT[dtype]).item() / 448 <= s


def test_append_of_values_that_are_not_finite(dev):
    y = Layer(dev, 2, 128, 16, "fp16", 4)

    def change(x):
        x[0, 5], x[3, 256 + 7], x[20, 130] = math.inf, math.nan, -math.inf
    y.append(1, list(range(40)), change=change)
    y.check()
    assert torch.isnan(VALUES[y.ref.bytes[0, 0, 0, 0, 5]]) and torch.isfinite(y.ref.scales[:2]).all()
    y.append(2, [40], loud=50.0, change=lambda x: x[:1, 60].fill_(math.inf))
    y.check()


def test_append_skips_what_it_must(dev):
    """Negative slots, slots behind the cache (reported), a group next to them."""
    y = Layer(dev, 1, 64, 32, "bf16", 3)
    y.append(0, [80])
    y.append(1, [-1, 95, -7, 96, 97, 0, 1, 1 << 40, -1])
    y.check(hs.HS_DEVERR_BLOCK_OOB)


@pytest.mark.parametrize("heads,kv_heads,d,dims,layout,dtype,page,rows,start", [
    (16, 4, 128, 128, 0, "bf16", 16, 32, "steps"), (32, 8, 128, 64, 0, "fp16", 32, 64, "steps"),
    (14, 2, 64, 64, 1, "bf16", 16, 7, "steps"), (6, 3, 128, 96, 0, "bf16", 64, 300, "tails"),
    (8, 8, 64, 16, 0, "fp16", 256, 3000, "tails"), (4, 1, 128, 32, 1, "bf16", 16, 5500, "tails"),
    (16, 4, 128, 128, 0, "fp16", 16, 5500, "tails"), (1, 1, 64, 48, 0, "bf16", 32, 1, "tails")])
def test_append_with_positions(dev, heads, kv_heads, d, dims, layout, dtype, page, rows, start):
    rope = hs.hs_rope_plan(dims, layout, 500000.0, hs.HS_ROPE_INDEX, 4.0, 8192, 1.0, 32.0, 1.14)
    w, g = (heads + 2 * kv_heads) * d, torch.Generator().manual_seed(3)
    blocks = rows + 2 if start == "steps" else -(-rows // page) + 8
    y = Layer(dev, kv_heads, d, page, dtype, blocks, heads)
    order = torch.randperm(blocks, generator=g)
    if start == "steps":
        n = torch.randint(0, page, (rows,), generator=g)
        slots = order[:rows] * page + n
        # what the tokens before them left
        y.append(4, [int(s) // G * G + i for s in slots for i in range(int(s) % G)], loud=0.3)
        pos = torch.randint(0, 100000, (rows,), generator=g)
    else:
        first = 5
        flat = (order[:, None] * page + torch.arange(page)).flatten()
        slots = flat[first:first + rows]
        y.append(4, flat[:first].tolist(), loud=0.3)
        pos = torch.arange(rows) + 77777
    if rows > 1:
        slots[-1] = -1
    x = rows_of(7, rows, w, 8, DT[dtype], dev)
    xd, q = x.to(dev), torch.full((rows + 1, heads * d), math.nan, dtype=DT[dtype], device=dev)
    hs.hs_kv8_append_rope(y.shape, rope, xd, xd[:, heads * d:], xd[:, (heads + kv_heads) * d:], w + 8, pos.to(dev),
                          slots.to(dev), rows, q, 0, y.cache, y.err)
    torch.cuda.synchronize()
    assert y.err.item() == 0
    v = x[:rows, :w].double().reshape(rows, -1, d)
    z, err = turned(rope, v[:, :heads + kv_heads], pos.tolist())
    got = q.cpu().double()
    skipped = slots < 0
    assert torch.isnan(got[:rows][skipped]).all() and torch.isnan(got[rows]).all()
    want, err_q = z[:, :heads], err[:, :heads]
    bound = err_q + U[dtype] * (want.abs() + err_q) + TINY[dtype]
    bound[..., dims:] = 0
    off = (got[:rows].reshape(rows, heads, d) - want).abs()
    assert (off <= bound)[~skipped].all()
    # the cache: every byte as of the exactly turned keys
    y.ref.append(torch.stack((z[:, heads:], v[:, heads + kv_heads:]), dim=1), slots.tolist())
    y.check()


def test_a_turned_key_at_a_border(dev):
    """Keys whose largest turned value is 448 but for a few steps of float32: the scale goes by float64."""
    for layout in (0, 1):
        rope = hs.hs_rope_plan(64, layout, 10000.0)
        n = 600
        y = Layer(dev, 1, 64, 16, "fp16", n)
        g = torch.Generator().manual_seed(layout)
        pos = torch.randint(1, 50000, (n,), generator=g)
        # one pair (a, 0): its larger turned value near 448 only where a cos or a sin is; theta of pair 0 is set for it
        x = torch.zeros(n, 128, dtype=torch.float16)
        x[:, 0] = 449.5 + torch.arange(n) % 7 * 0.25
        cases = []
        for i in range(0, n, 20):
            a = x[i, 0].double().item()
            # the angle with a cos(angle) = 448 (1 + k 2^-26), one position
            k = (i // 20 % 9 - 4) * 2.0 ** -26
            rope.theta[0] = math.acos(448.0 * (1 + k) / a)
            xd = x[i:i + 1].to(dev)
            slot = torch.tensor([16 * i], device=dev)
            hs.hs_kv8_append_rope(y.shape, rope, None, xd, xd[:, 64:], 128, torch.tensor([1], device=dev), slot, 1,
                                  None, 0, y.cache, y.err)
            c = a * math.cos(rope.theta[0])
            if abs(c / 448.0 - 1) > 2.0 ** -40:          # theta itself is rounded
                cases.append((i, 1.0 if c < 448.0 else 2.0))
        torch.cuda.synchronize()
        got = y.cache.cpu()
        scales = got[:, 2048:2052].contiguous().view(torch.float32)[:, 0]
        assert len(cases) > 20
        for i, want in cases:
            assert scales[i].item() == want, i


def append_keys(dev, y, rope, x, slots, pos):
    w, n = y.hk * y.d, len(slots)
    xd = x.to(dev)
    hs.hs_kv8_append_rope(y.shape, rope, None, xd, xd[:, w:], x.shape[1], torch.tensor(pos, device=dev),
                          torch.tensor(slots, device=dev), n, None, 0, y.cache, y.err)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("amplitude", [0, -20, 20])          # powers of two: the bytes are those of 1
@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "bf16")])
def test_keys_at_position_zero_are_rounded_as_they_are(dev, layout, amplitude, d, dtype):
    """Position 0 turns by nothing, so that keys that lie halfway between two bytes stay there: one in 16 of bf16."""
    rope = hs.hs_rope_plan(d, layout, 10000.0, hs.HS_ROPE_PLAIN, 1.0, 1, 1.0, 2.0, 2.0 ** amplitude)
    y, n, w = Layer(dev, 2, d, 16, dtype, 6), 61, 2 * d
    x = rows_of(5, n, 2 * w, 0, DT[dtype], dev)[:n]
    slots = list(range(16, 16 + n))
    append_keys(dev, y, rope, x, slots, [0] * n)
    z = x.double().reshape(n, 2, 2, d)
    z[:, 0] *= 2.0 ** amplitude
    y.ref.append(z, slots)
    y.check()


@pytest.mark.parametrize("layout", [0, 1])
def test_zeros_turned(dev, layout):
    """Rows of zeros among others, groups of zeros, pairs of zeros: zeros, of either sign."""
    rope = hs.hs_rope_plan(128, layout, 10000.0)
    y, n, w = Layer(dev, 1, 128, 32, "bf16", 8), 200, 128
    x = rows_of(6, n, 2 * w, 0, torch.bfloat16, dev)[:n]
    x[3], x[32:64], x[70:75, :w] = 0.0, 0.0, -0.0
    x[100:, 7:9], x[100:, 64 + 7:64 + 9] = 0.0, -0.0
    slots, pos = list(range(n)), list(range(1000, 1000 + n))
    append_keys(dev, y, rope, x, slots, pos)
    z = x.double().reshape(n, 2, 1, 128)
    z[:, 0] = turned(rope, z[:, 0], pos)[0]
    y.ref.append(z, slots)
    unsigned = y.ref.bytes.clone()
    got = y.cache.cpu()
    m = unsigned[0].numel()
    flat = got[:, :m]
    got[:, :m] = torch.where(flat == 128, torch.zeros_like(flat), flat)
    y.ref.bytes = torch.where(unsigned == 128, torch.zeros_like(unsigned), unsigned)
    y.cache = got
    y.check()


@pytest.mark.parametrize("amplitude", [2.0 ** -20, 2.0 ** 20])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_smallest_and_largest_values_at_the_ends_of_the_amplitude(dev, amplitude, dtype):
    """Groups of zeros alone, of the type's smallest and of its largest values, whose scales are at their ends."""
    rope = hs.hs_rope_plan(64, 0, 10000.0, hs.HS_ROPE_PLAIN, 1.0, 1, 1.0, 2.0, amplitude)
    y, n, info = Layer(dev, 1, 64, 16, dtype, 4), 64, torch.finfo(DT[dtype])
    x = rows_of(11, n, 128, 0, DT[dtype], dev)[:n]
    x[:16, :64] = 0.0
    x[16:32, :64] = info.smallest_normal * info.eps * torch.randint(0, 3, (16, 64), generator=torch.Generator().manual_seed(0))
    x[32:48, :64] = (x[32:48, :64].sign().double() * info.max * min(1.0, 1.0 / amplitude) / 2).to(DT[dtype])
    slots, pos = list(range(n)), [0] * 8 + list(range(1, n - 7))
    append_keys(dev, y, rope, x, slots, pos)
    z = x.double().reshape(n, 2, 1, 64)
    z[:, 0] = turned(rope, z[:, 0], pos)[0]
    y.ref.append(z, slots)
    # a zero's sign is not compared
    got = y.cache.cpu()
    m = y.ref.bytes[0].numel()
    got[:, :m] = torch.where(got[:, :m] == 128, torch.zeros_like(got[:, :m]), got[:, :m])
    y.ref.bytes = torch.where(y.ref.bytes == 128, torch.zeros_like(y.ref.bytes), y.ref.bytes)
    y.cache = got
    y.check()


@pytest.mark.parametrize("times", [1, 30])
@pytest.mark.parametrize("kv_heads,d,dtype,dims", [(3, 64, "bf16", 64), (1, 128, "fp16", 32), (9, 128, "bf16", 128),
                                                   (24, 64, "fp16", 16)])
def test_steps_beside_prompts(dev, kv_heads, d, dtype, dims, times):
    """Single tokens, short runs and prompts in one call: windows of rows that begin 16 groups, some and none."""
    g = torch.Generator().manual_seed(kv_heads)
    runs = [1] * 20 + [2, 3, 40, 1, 17, 5, 1, 1, 33, 16, 16, 1] * times + [1] * 17
    slots, at = [], 0
    for n in runs:
        at = -(-at // G) * G
        first = at + int(torch.randint(0, G, (1,), generator=g))
        slots += list(range(first, first + n))
        at = first + n
        if n == 5:
            slots.append(-1)
    n, w = len(slots), kv_heads * d
    y = Layer(dev, kv_heads, d, 32, dtype, -(-at // 32) + 1)
    held = sorted({s // G * G for s in slots if s >= 0})
    y.append(8, [b + i for b in held for i in range(G)], loud=0.5)
    y.append(9, slots)
    y.check()
    rope = hs.hs_rope_plan(dims, 0, 10000.0)
    x = rows_of(10, n, 2 * w, 0, DT[dtype], dev, loud=3.0)[:n]
    pos = torch.randint(0, 70000, (n,), generator=g).tolist()
    append_keys(dev, y, rope, x, slots, pos)
    z = x.double().reshape(n, 2, kv_heads, d)
    z[:, 0] = turned(rope, z[:, 0], pos)[0]
    y.ref.append(z, slots)
    y.check()


@pytest.mark.parametrize("kv_heads,d", [(1024, 64), (511, 128)])
def test_append_of_the_most_heads(dev, kv_heads, d):
    slots = [3, 16, 40, 41, 42] + list(range(50, 75)) + [96]
    n, w = len(slots), kv_heads * d
    y = Layer(dev, kv_heads, d, 16, "bf16", 7)
    y.append(11, list(range(7 * 16)), loud=0.5)       # a group that goes on has begun
    y.append(12, slots)
    y.append(13, [4, 17, 97], loud=4.0)
    rope = hs.hs_rope_plan(d, 1, 10000.0)
    x, pos = rows_of(14, n, 2 * w, 0, torch.bfloat16, dev, loud=9.0)[:n], list(range(500, 500 + n))
    append_keys(dev, y, rope, x, slots, pos)
    z = x.double().reshape(n, 2, kv_heads, d)
    z[:, 0] = turned(rope, z[:, 0], pos)[0]
    y.ref.append(z, slots)
    y.check()


# ---- reading back ------------------------------------------------------------------------

READ = [(4, 128, 16, "bf16", [300, 0, 1, 16, 17, 999]), (2, 64, 32, "fp16", [31, 33]), (8, 128, 32, "fp16", [2000]),
        (1, 64, 256, "bf16", [700, 255, 256, 257]), (3, 128, 64, "bf16", [5] * 50), (5, 64, 16, "fp16", [90, 1] * 120)]


@pytest.mark.parametrize("shift", [0, 8])       # elements: a cache at a multiple of 16 bytes, not of 32
@pytest.mark.parametrize("kv_heads,d,page,dtype,lens", READ)
def test_read(dev, kv_heads, d, page, dtype, lens, shift):
    c, table = filled(1, lens, kv_heads, page, d, width=-(-max(lens) // page) + 2)
    blocks = c.blocks + 5
    g = torch.Generator().manual_seed(9)
    to = torch.randperm(blocks, generator=g).int()
    out_table = torch.where(table >= 0, to[table.clamp(min=0).long()], -1).int()
    room = torch.full((blocks * 2 * page * kv_heads * d + 16,), math.nan, dtype=DT[dtype], device=dev)
    out = room[shift:shift - 16].view(blocks, 2, page, kv_heads, d)
    want = out.cpu().contiguous()
    vals = c.values()
    for b, n in enumerate(lens):
        for j in range(n):
            src, dst = table[b, j // page], out_table[b, j // page]
            want[dst, :, j % page] = vals[src, :, :, j % page].transpose(0, 1).to(DT[dtype])
    shape = shape_of(len(lens), kv_heads, kv_heads, d, page, c.blocks, table.shape[1], dtype)
    err = fresh_err(dev)
    for bound in (max(lens), table.shape[1] * page):
        hs.hs_kv8_read(shape, c.image().to(dev), table.to(dev), torch.tensor(lens, dtype=torch.int32, device=dev), bound,
                       out, blocks, out_table.to(dev), err)
        torch.cuda.synchronize()
        assert err.item() == 0
        assert torch.equal(out.cpu().nan_to_num(7.0), want.nan_to_num(7.0))
        assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want))
        assert torch.isnan(room[:shift]).all() and torch.isnan(room[shift - 16:]).all()


def test_read_of_every_byte_and_the_largest_values(dev):
    for dtype, top in (("bf16", 2.0 ** 120), ("fp16", 256.0)):
        c, table = filled(2, [48], 1, 16, 128)
        c.bytes[table[0, 0], 0, 0] = torch.arange(16 * 128).reshape(16, 128) % 256
        c.bytes[table[0, 1], 0, 0] = torch.arange(16 * 128).reshape(16, 128) % 256
        c.scales[table[0, 0]] = top
        c.scales[table[0, 1]] = 2.0 ** -12
        out = torch.zeros(4, 2, 16, 1, 128, dtype=DT[dtype], device=dev)
        shape = shape_of(1, 1, 1, 128, 16, c.blocks, 3, dtype)
        hs.hs_kv8_read(shape, c.image().to(dev), table.to(dev), torch.tensor([48], dtype=torch.int32, device=dev), 48,
                       out, 4, torch.tensor([[2, 0, 3]], dtype=torch.int32, device=dev))
        most = torch.finfo(DT[dtype]).max
        for src, dst in ((0, 2), (1, 0)):
            want = c.values()[table[0, src], 0].clamp(-most, most).to(DT[dtype])
            got = out.cpu()[dst, :, :, 0]
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(got.nan_to_num(1.0), want.nan_to_num(1.0))


def test_read_reports_pages_and_lengths(dev):
    c, table = filled(3, [64, 64, 64], 2, 16, 64)
    out_table = torch.arange(12, dtype=torch.int32).reshape(3, 4)
    shape = shape_of(3, 2, 2, 64, 16, c.blocks, 4, "bf16")
    for name, code in (("from", hs.HS_DEVERR_BLOCK_OOB), ("to", hs.HS_DEVERR_BLOCK_OOB), ("len", hs.HS_DEVERR_LENGTH),
                       ("long", hs.HS_DEVERR_LENGTH)):
        t, o, lens = table.clone(), out_table.clone(), [64, 64, 64]
        if name == "from":
            t[1, 2] = c.blocks
        elif name == "to":
            o[1, 2] = -1
        else:
            lens[1] = -1 if name == "len" else 65
        out = torch.full((12, 2, 16, 2, 64), math.nan, dtype=torch.bfloat16, device=dev)
        err = fresh_err(dev)
        hs.hs_kv8_read(shape, c.image().to(dev), t.to(dev), torch.tensor(lens, dtype=torch.int32, device=dev), 64, out, 12,
                       o.to(dev), err)
        torch.cuda.synchronize()
        assert err.item() == code
        left = torch.isnan(out.cpu()).flatten(1).all(dim=1)
        skipped = {6} if name in ("from", "to") else {4, 5, 6, 7}
        assert {i for i in range(12) if left[i]} == skipped


# ---- a decode step -----------------------------------------------------------------------


def decoded(dev, c, table, q, heads, dtype, lens, bound, ostride=0, lse=True, **kw):
    """(o, lse, status) of a call; q [row][heads d + pad] on the CPU."""
    B, d = len(lens), c.d
    shape = shape_of(B, heads, c.kv_heads, d, c.page, c.blocks, table.shape[1], dtype, q_stride=q.shape[1],
                     o_stride=ostride, **kw)
    o = torch.full((B + 1, ostride or heads * d), math.nan, dtype=DT[dtype], device=dev)
    z = torch.full((B + 1, heads), math.nan, device=dev)
    size = hs.hs_kv8_decode_workspace_bytes(shape, bound)
    ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device=dev)
    err = fresh_err(dev)
    hs.hs_kv8_decode(shape, q.to(dev), c.image().to(dev), table.to(dev), torch.tensor(lens, dtype=torch.int32, device=dev),
                     bound, o, z if lse else None, ws, size, err)
    torch.cuda.synchronize()
    assert (ws[size:] == 0xFF).all()
    assert torch.isnan(o[B:]).all() and torch.isnan(z[B:]).all() and torch.isnan(o[:, heads * d:]).all()
    return o[:B, :heads * d].cpu(), z[:B].cpu(), err.item()


def near(c, table, q, heads, dtype, lens, o, z, scale, only=None):
    d, hk = c.d, c.kv_heads
    for b, n in enumerate(lens):
        if only is not None and b not in only:
            continue
        k, v = keys_of(c, table, b, n)
        x = q[b, :heads * d].double().reshape(hk, heads // hk, d)
        want, want_z, bound, bound_z = attended(x, k, v, scale, dtype)
        off = (o[b].double().reshape(want.shape) - want).abs()
        assert (off <= bound).all(), (b, n, (off / bound).max().item())
        got = z[b].double().reshape(want_z.shape)
        if n == 0:
            assert (got == -math.inf).all()
        else:
            assert ((got - want_z).abs() <= bound_z).all(), (b, n)


DECODE = [  # heads, kv heads, d, page, dtype, lengths
    (4, 1, 128, 16, "bf16", [1]), (16, 4, 128, 16, "bf16", [4608]), (14, 2, 64, 16, "bf16", [0, 1, 15, 16, 17, 300, 45] * 9),
    (16, 4, 128, 16, "fp16", [0, 1, 2000, 31, 32, 33, 777, 5, 1200]), (32, 8, 128, 32, "bf16", [3000, 2900, 10, 0]),
    (8, 8, 64, 32, "fp16", [511, 512, 513]), (12, 1, 128, 64, "bf16", [100, 900]), (16, 1, 64, 256, "fp16", [1, 255, 700]),
    (9, 1, 128, 128, "fp16", [640, 3]), (24, 1, 64, 16, "bf16", [50, 0, 400]), (128, 1, 128, 16, "bf16", [300, 1100]),
    (48, 3, 128, 32, "fp16", [64, 65, 1000]), (3, 3, 128, 16, "bf16", [7] * 300), (5, 5, 64, 16, "fp16", [600] * 30)]


@pytest.mark.parametrize("unsplit", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,page,dtype,lens", DECODE)
def test_decode(dev, heads, kv_heads, d, page, dtype, lens, unsplit):
    c, table = filled(4, lens, kv_heads, page, d, width=-(-max(lens) // page) + 70)
    q = rows_of(5, len(lens), heads * d, 8, DT[dtype], dev, loud=0.5)
    first = None
    for bound in (max(lens), table.shape[1] * page):
        o, z, err = decoded(dev, c, table, q, heads, dtype, lens, bound, heads * d + 16, unsplit=unsplit)
        assert err == 0
        near(c, table, q, heads, dtype, lens, o, z, d ** -0.5)
        if unsplit and first is not None:
            assert torch.equal(o, first[0]) and torch.equal(z, first[1])
        first = (o, z)
        again = decoded(dev, c, table, q, heads, dtype, lens, bound, heads * d + 16, lse=False, unsplit=unsplit)
        assert torch.equal(again[0], o)


def test_decode_unsplit_rows_know_nothing_of_the_others(dev):
    lens = [700, 33, 1500, 0, 260]
    c, table = filled(6, lens, 2, 16, 128)
    q = rows_of(7, 5, 8 * 128, 0, torch.bfloat16, dev)
    o, z, _ = decoded(dev, c, table, q, 8, "bf16", lens, 1500, unsplit=True)
    for b, n in enumerate(lens):
        o1, z1, _ = decoded(dev, c, table[b:b + 1], q[b:b + 1], 8, "bf16", [n], n, unsplit=True)
        assert torch.equal(o1[0], o[b]) and torch.equal(z1[0], z[b])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("scale,loud", [(1e-6, 1.0), (1.0, 1.0), (30.0, 4.0), (2.0 ** -40, 2.0 ** 10)])
def test_decode_scores_of_every_size(dev, dtype, scale, loud):
    """Flat, sharp and very sharp softmax; groups with scales 2^16 apart."""
    lens = [900, 40]
    c, table = filled(8, lens, 2, 32, 64, spread=8)
    q = rows_of(9, 2, 8 * 64, 0, DT[dtype], dev, loud=loud)
    o, z, err = decoded(dev, c, table, q, 8, dtype, lens, 900, scale=scale)
    assert err == 0
    near(c, table, q, 8, dtype, lens, o, z, scale)


def test_decode_of_queries_of_any_size(dev):
    """bf16 queries from 2^-120 to 2^100, a row of zeros: the keys' scales bring the scores back."""
    lens = [100] * 6
    c, table = filled(10, lens, 1, 16, 128)
    q = rows_of(11, 6, 128, 0, torch.bfloat16, dev)
    for i, e in enumerate((-120, -60, 0, 60, 100)):
        q[i, :128] *= 2.0 ** e
    q[5, :128] = 0.0
    o, z, err = decoded(dev, c, table, q, 1, "bf16", lens, 100, scale=1.0)
    assert err == 0
    near(c, table, q, 1, "bf16", lens, o, z, 1.0, only={0, 1, 2, 5})
    # scores of 2^60 and more: the largest alone counts
    for b in (3, 4):
        k, v = keys_of(c, table, b, 100)
        s = torch.einsum("d,nd->n", q[b, :128].double(), k[0])
        best = s.argmax()
        gap = s.max() - s[torch.arange(100) != best].max()
        assert gap > 2.0 ** -20 * s.abs().max()
        assert torch.equal(o[b].double(), v[0, best].bfloat16().double())
    c.scales[table[0].long()] *= 2.0 ** 100                     # tiny queries, huge keys
    q[0, :128] = rows_of(12, 1, 128, 0, torch.bfloat16, dev)[0] * 2.0 ** -100
    o, z, err = decoded(dev, c, table[:1], q[:1], 1, "bf16", [100], 100, scale=1.0)
    k, v = keys_of(c, table, 0, 100)
    want, want_z, bound, bound_z = attended(q[:1].double().reshape(1, 1, 128), k, v, 1.0, "bf16")
    assert ((o[0].double() - want[0, 0]).abs() <= bound[0, 0]).all() and ((z[0] - want_z[0]).abs() <= bound_z[0]).all()


def test_decode_of_values_at_the_types_end(dev):
    """Averages of values beyond the type's largest stay finite."""
    for dtype, e in (("fp16", 8), ("bf16", 120)):
        c, table = filled(12, [600], 1, 16, 64)
        c.bytes[:, :, 1] = 126                                   # 448
        c.scales[:, :, 1] = 2.0 ** e
        q = rows_of(13, 1, 64, 0, DT[dtype], dev)
        for unsplit in (False, True):
            for n in (5, 600):
                o, z, err = decoded(dev, c, table, q, 1, dtype, [n], 600, unsplit=unsplit)
                assert err == 0 and (o.double() == torch.finfo(DT[dtype]).max).all()


def test_decode_keeps_nan_to_its_heads(dev):
    lens = [800, 300]
    c, table = filled(14, lens, 3, 16, 128)
    q = rows_of(15, 2, 6 * 128, 0, torch.bfloat16, dev)
    o, z, _ = decoded(dev, c, table, q, 6, "bf16", lens, 800)
    blk = table[0, 20]
    for plane in (0, 1):
        old = c.bytes[blk, 1, plane, 3, 77].clone()
        c.bytes[blk, 1, plane, 3, 77] = 127
        o1, z1, err = decoded(dev, c, table, q, 6, "bf16", lens, 800)
        c.bytes[blk, 1, plane, 3, 77] = old
        assert err == 0
        hit = torch.zeros(2, 6 * 128, dtype=torch.bool)
        hit[0, 2 * 128:4 * 128] = True
        assert torch.equal(o1[~hit], o[~hit])
        bad = o1.reshape(2, 6, 128)[0, 2:4]
        assert torch.isnan(bad).all() if plane == 0 else torch.isnan(bad[:, 77]).all()


def test_decode_reports_pages_and_lengths(dev):
    lens = [100, 500, 50, 300]
    c, table = filled(16, lens, 2, 16, 64)
    q = rows_of(17, 4, 4 * 64, 0, torch.float16, dev)
    for unsplit in (False, True):
        for bad in (c.blocks, -1, 1 << 30, -(1 << 31)):
            t = table.clone()
            t[1, 13] = bad
            o, z, err = decoded(dev, c, t, q, 4, "fp16", lens, 512, unsplit=unsplit)
            assert err == hs.HS_DEVERR_BLOCK_OOB
            near(c, table, q, 4, "fp16", lens, o, z, 0.125, only={0, 2, 3})
        for n in (-1, 513, -(1 << 31)):
            o, z, err = decoded(dev, c, table, q, 4, "fp16", [100, n, 50, 300], 512, unsplit=unsplit)
            assert err == hs.HS_DEVERR_LENGTH
            near(c, table, q, 4, "fp16", lens, o, z, 0.125, only={0, 2, 3})
            assert torch.isnan(o[1]).all() and torch.isnan(z[1]).all()


# ---- together ----------------------------------------------------------------------------


@pytest.mark.parametrize("heads,kv_heads,d,page,dtype,layout", [(16, 4, 128, 16, "bf16", 0), (8, 2, 64, 32, "fp16", 1)])
def test_a_resumed_request(dev, heads, kv_heads, d, page, dtype, layout):
    """Pages saved and restored with their scales, the tail turned and appended, the prefix read back for a prefill of the
    tail, then captured decode steps that are replayed as the request grows."""
    prefix, tail, steps = 6 * page, 45, 20
    n = prefix + tail + steps
    w, blocks = (heads + 2 * kv_heads) * d, 64
    g = torch.Generator().manual_seed(20)
    rope = hs.hs_rope_plan(d, layout, 10000.0)
    width = -(-n // page)
    table = torch.randperm(blocks, generator=g)[:width].int().reshape(1, width).to(dev)
    shape = shape_of(1, heads, kv_heads, d, page, blocks, width, dtype, q_stride=w)
    size = hs.hs_kv8_block_bytes(shape)
    qkv = torch.randn(n, w, generator=g).to(DT[dtype]).to(dev)
    pos = torch.arange(n, device=dev)
    slots = table[0, pos // page].long() * page + pos % page
    err = fresh_err(dev)

    def views(x):
        return x, x[:, heads * d:], x[:, (heads + kv_heads) * d:]
    # the first run: every row at once, and its pages saved
    whole = torch.zeros(blocks, size, dtype=torch.uint8, device=dev)
    q_all = torch.empty(n, w, dtype=DT[dtype], device=dev)
    hs.hs_kv8_append_rope(shape, rope, *views(qkv), w, pos, slots, n, q_all, w, whole, err)
    staging = torch.zeros(prefix // page, size, dtype=torch.uint8, device=dev)
    hs.hs_save_kv_pages(hs.ptr_array([whole], dev), hs.ptr_array([staging], dev), 1, table[0], prefix // page, size,
                        blocks, err)
    # the resumed one
    cache = torch.full((blocks, size), 0xFF, dtype=torch.uint8, device=dev)
    hs.hs_restore_kv_pages(hs.ptr_array([staging], dev), hs.ptr_array([cache], dev), 1, table[0], prefix // page, size,
                           blocks, err)
    kv16 = torch.full((blocks, 2, page, kv_heads, d), math.nan, dtype=DT[dtype], device=dev)
    tail_q = torch.empty(tail, w, dtype=DT[dtype], device=dev)
    rows = slice(prefix, prefix + tail)
    hs.hs_kv8_append_rope(shape, rope, *views(qkv[rows]), w, pos[rows], slots[rows], tail, tail_q, w, cache, err)
    assert torch.equal(tail_q[:, :heads * d], q_all[rows, :heads * d])
    have = torch.tensor([prefix + tail], dtype=torch.int32, device=dev)
    hs.hs_kv8_read(shape, cache, table, have, width * page, kv16, blocks, table, err)
    o = torch.empty(tail, heads, d, dtype=DT[dtype], device=dev)
    need = hs.hs_attn_prefill_workspace_bytes(shape, [prefix], [tail])
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    hs.hs_attn_prefill(shape, tail_q, kv16, table, o, None, [prefix], [tail], [0, tail], ws, need, err)
    torch.cuda.synchronize()
    assert err.item() == 0
    ref = Cache(blocks, kv_heads, page, d)

    def of_device(x):
        y = x.cpu()
        m = kv_heads * 2 * page * d
        ref.bytes = y[:, :m].reshape(ref.bytes.shape).long()
        s = y[:, m:m + kv_heads * 2 * page // G * 4].contiguous().view(torch.float32)
        ref.scales = s.reshape(ref.scales.shape).double()
        return ref
    k, v = keys_of(of_device(cache), table.cpu(), 0, prefix + tail)
    for t in (0, 17, tail - 1):
        x = tail_q[t, :heads * d].double().cpu().reshape(kv_heads, heads // kv_heads, d)
        want, _, bound, _ = attended(x, k[:, :prefix + t + 1], v[:, :prefix + t + 1], d ** -0.5, dtype)
        # the prefill rounds its weights, whose sum is 1, to the element type
        bound = bound + U[dtype] * v.abs().amax()
        assert ((o[t].double().cpu().reshape(want.shape) - want).abs() <= bound).all()
    # decode steps, captured once
    need = hs.hs_kv8_decode_workspace_bytes(shape, width * page)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    step = qkv[prefix + tail:prefix + tail + 1].clone()
    at, slot, length = (torch.zeros(1, dtype=t, device=dev) for t in (torch.int64, torch.int64, torch.int32))
    q1, o1 = torch.empty(1, w, dtype=DT[dtype], device=dev), torch.empty(1, heads, d, dtype=DT[dtype], device=dev)

    def run():
        hs.hs_kv8_append_rope(shape, rope, *views(step), w, at, slot, 1, q1, w, cache, err)
        hs.hs_kv8_decode(shape, q1, cache, table, length, width * page, o1, None, ws, need, err)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        at.fill_(prefix + tail)
        slot.copy_(slots[prefix + tail:prefix + tail + 1])
        length.fill_(prefix + tail + 1)
        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
    for i in range(steps):
        j = prefix + tail + i
        step.copy_(qkv[j:j + 1])
        at.fill_(j)
        slot.copy_(slots[j:j + 1])
        length.fill_(j + 1)
        graph.replay()
        torch.cuda.synchronize()
        if i in (0, 1, steps - 1):
            k, v = keys_of(of_device(cache), table.cpu(), 0, j + 1)
            x = q1[0, :heads * d].double().cpu().reshape(kv_heads, heads // kv_heads, d)
            want, _, bound, _ = attended(x, k, v, d ** -0.5, dtype)
            assert ((o1[0].double().cpu().reshape(want.shape) - want).abs() <= bound).all()
    assert err.item() == 0


def test_pages_beyond_4_gib(dev):
    """The same keys in the last blocks of a large cache and in a small one: bytes, what is read back and answers."""
    heads, hk, d, page, n = 4, 2, 128, 256, 600
    g = torch.Generator().manual_seed(40)
    x = torch.randn(n, (heads + 2 * hk) * d, generator=g).bfloat16().to(dev)
    w = x.shape[1]
    rope, pos, got = hs.hs_rope_plan(d, hs.HS_ROPE_HALF, **PLAIN), torch.arange(n, device=dev), []
    size = hs.hs_kv8_block_bytes(shape_of(1, heads, hk, d, page, 1, 3, "bf16"))
    many = (5 << 30) // size
    for blocks, ids in ((4, [2, 0, 3]), (many, [many - 1, many - 7, many - 2])):
        shape = shape_of(1, heads, hk, d, page, blocks, 3, "bf16", q_stride=w)
        cache = torch.zeros(blocks, size, dtype=torch.uint8, device=dev)
        table = torch.tensor([ids], dtype=torch.int32, device=dev)
        slots = table[0, pos // page].long() * page + pos % page
        err, q = fresh_err(dev), x.clone()
        hs.hs_kv8_append_rope(shape, rope, q, q[:, heads * d:], q[:, (heads + hk) * d:], w, pos, slots, n, q, w, cache, err)
        out = torch.zeros(3, 2, page, hk, d, dtype=torch.bfloat16, device=dev)
        lens = torch.tensor([n], dtype=torch.int32, device=dev)
        hs.hs_kv8_read(shape, cache, table, lens, n, out, 3, torch.tensor([[0, 1, 2]], dtype=torch.int32, device=dev), err)
        need = hs.hs_kv8_decode_workspace_bytes(shape, n)
        ws, o = torch.empty(max(need, 16), dtype=torch.uint8, device=dev), torch.empty(1, heads * d, dtype=torch.bfloat16, device=dev)
        hs.hs_kv8_decode(shape, q[n - 1:], cache, table, lens, n, o, None, ws, need, err)
        torch.cuda.synchronize()
        assert err.item() == 0
        got.append((cache[torch.tensor(ids, device=dev)].cpu(), out.cpu(), o.cpu(), q.cpu()))
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("heads,d,dtype", [(2, 64, "bf16"), (1, 128, "fp16")])
def test_decode_of_a_long_context(dev, heads, d, dtype):
    lens = [200_003, 17]
    c, table = filled(41, lens, 1, 256, d)
    q = rows_of(42, 2, heads * d, 0, DT[dtype], dev)
    for unsplit in (False, True):
        o, z, err = decoded(dev, c, table, q, heads, dtype, lens, 200_003, unsplit=unsplit)
        assert err == 0
        near(c, table, q, heads, dtype, lens, o, z, d ** -0.5)


def test_decode_without_a_key(dev):
    c, table = filled(43, [0, 0, 0], 2, 16, 128)
    q = rows_of(44, 3, 4 * 128, 0, torch.bfloat16, dev)
    for bound in (0, 16):
        o, z, err = decoded(dev, c, table, q, 4, "bf16", [0, 0, 0], bound)
        assert err == 0 and (o == 0).all() and (z == -math.inf).all()


def test_calls_on_two_streams_at_once(dev):
    """Each with its own workspace and cache: the bits of the calls one by one."""
    cases = []
    for seed, lens, heads, hk in ((50, [3000, 5, 900], 8, 2), (51, [2500] * 4, 16, 1)):
        c, table = filled(seed, lens, hk, 16, 128)
        shape = shape_of(len(lens), heads, hk, 128, 16, c.blocks, table.shape[1], "bf16")
        bound = table.shape[1] * 16
        size = hs.hs_kv8_decode_workspace_bytes(shape, bound)
        q = rows_of(seed, len(lens), heads * 128, 0, torch.bfloat16, dev)
        cases.append(dict(shape=shape, q=q.to(dev), cache=c.image().to(dev), table=table.to(dev), size=size, bound=bound,
                          lens=torch.tensor(lens, dtype=torch.int32, device=dev),
                          ws=torch.empty(size, dtype=torch.uint8, device=dev),
                          o=[torch.zeros(len(lens), heads * 128, dtype=torch.bfloat16, device=dev) for _ in range(13)]))

    def run(x, i, stream=None):
        hs.hs_kv8_decode(x["shape"], x["q"], x["cache"], x["table"], x["lens"], x["bound"], x["o"][i], None, x["ws"], x["size"],
                         None, stream)
    for x in cases:
        run(x, 0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for i in range(1, 13):
        for x, s in zip(cases, streams):
            run(x, i, s)
    torch.cuda.synchronize()
    for x in cases:
        assert all(torch.equal(y, x["o"][0]) for y in x["o"][1:])
