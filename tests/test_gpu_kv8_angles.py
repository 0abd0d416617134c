"""Angles of far positions against integers: turned rows and the bytes of turned keys."""
import math

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.gpu_helpers import device
from tests.kv8_helpers import DT, TINY, U, shape_of
from tests.test_gpu_kv8 import Layer, append_keys, rows_of

pytestmark = pytest.mark.gpu
BITS = 400


@pytest.fixture(scope="module")
def dev():
    return device()


def turns_per_radian():
    """1 / (2 pi) in units of 2^-BITS, by Machin's formula."""
    one = 1 << (2 * BITS)

    def arctan(n):               # of 1 / n
        term = total = one // n
        k, sign = 1, -1
        while term:
            term //= n * n
            k += 2
            total += sign * (term // k)
            sign = -sign
        return total
    pi = 4 * (4 * arctan(5) - arctan(239))
    return (one * one // (2 * pi)) >> BITS


UNIT = turns_per_radian()


def spins(rope, pos):
    """cos and sin of pos theta, float64 [row][1][pair], from the exact product."""
    rows = []
    for p in pos:
        row = []
        for theta in rope.theta[:rope.dims // 2]:
            a, b = theta.as_integer_ratio()                  # b a power of two
            whole = b << BITS
            x = p * a * UNIT % whole
            row.append((x if 2 * x < whole else x - whole) / whole)
        rows.append(row)
    t = torch.tensor(rows, dtype=torch.float64)[:, None] * (2 * math.pi)
    return t.cos(), t.sin()


def exactly(rope, x, pos):
    """x float64 [row][head][d] turned; the sum of its pairs' magnitudes, laid out alike."""
    n = rope.dims // 2
    c, s = (y * rope.amplitude for y in spins(rope, pos))
    y, rest = x[..., :rope.dims], x[..., rope.dims:]
    half = rope.layout == hs.HS_ROPE_HALF
    a, b = (y[..., :n], y[..., n:]) if half else (y[..., 0::2], y[..., 1::2])
    sums = rope.amplitude * (a.abs() + b.abs())
    z = [(a * c - b * s, b * c + a * s), (sums, sums)]
    z = [torch.cat(t, dim=2) if half else torch.stack(t, dim=3).flatten(2) for t in z]
    return torch.cat((z[0], rest), dim=2), torch.cat((z[1], torch.zeros_like(rest)), dim=2)


def planned(dims, layout, kind):
    rope = hs.hs_rope_plan(dims, layout, 500000.0, amplitude=1.0)
    for i in range(dims // 2):
        if kind == "backwards":
            rope.theta[i] = -rope.theta[i]
        elif kind == "fast":                                 # many turns a position, up to 2^60 radians
            rope.theta[i] = rope.theta[i] * 2.0 ** (i % 61) * (1 - 2 * (i % 2))
    return rope


@pytest.mark.parametrize("kind", ["forwards", "backwards", "fast"])
@pytest.mark.parametrize("d,dims,layout", [(128, 128, 0), (64, 48, 1)])
def test_rope_at_far_positions(dev, d, dims, layout, kind):
    rope = planned(dims, layout, kind)
    rows = 200
    g = torch.Generator().manual_seed(80)
    e = torch.randint(0, 51, (rows,), generator=g).tolist()
    pos = [int(p * 2.0 ** k) for p, k in zip((torch.rand(rows, generator=g, dtype=torch.float64) * 2 - 1).tolist(), e)]
    pos[:4] = [0, 2 ** 50 + 1, -2 ** 50 - 12345, 2 ** 33]
    x = rows_of(81, rows, 3 * d, 0, torch.float16, dev)
    out = torch.empty(rows, 2 * d, dtype=torch.float16, device=dev)
    k_out = torch.empty(rows, d, dtype=torch.float16, device=dev)
    xd = x.to(dev)
    hs.hs_rope_apply(shape_of(0, 2, 1, d, 16, 1, 1, "fp16"), rope, xd, xd[:, 2 * d:], 3 * d, torch.tensor(pos, device=dev),
                     rows, out, 0, k_out, 0)
    want, size = exactly(rope, x[:rows].double().reshape(rows, 3, d), pos)
    got = torch.cat((out, k_out), dim=1).double().cpu().reshape(rows, 3, d)
    # theta's rounding; the angle's upper 32 bits as a float of a half turn; sine, cosine, products and their sum in float32
    angle = torch.tensor([abs(p) for p in pos], dtype=torch.float64)[:, None, None] * 2.0 ** -65 * 2 * math.pi
    err = size * (angle + math.pi * 2.0 ** -24 + 2.0 ** -29 + 2.0 ** -22 + 2.0 ** -22)
    assert ((got - want).abs() <= err + U["fp16"] * (want.abs() + err) + TINY["fp16"]).all()


@pytest.mark.parametrize("kind", ["forwards", "backwards", "fast"])
@pytest.mark.parametrize("d,dims,layout,dtype", [(128, 128, 0, "bf16"), (64, 64, 1, "fp16")])
def test_bytes_of_keys_at_far_positions(dev, d, dims, layout, dtype, kind):
    """Every byte as of the exactly turned keys, up to positions of 2^39."""
    rope = planned(dims, layout, kind)
    n, hk = 400, 4
    y = Layer(dev, hk, d, 16, dtype, n // 16)
    x = rows_of(82, n, 2 * hk * d, 0, DT[dtype], dev)[:n]
    g = torch.Generator().manual_seed(83)
    pos = torch.randint(2 ** 37, 2 ** 39, (n,), generator=g) * (1 - 2 * torch.randint(0, 2, (n,), generator=g))
    pos[::5] = torch.randint(0, 10 ** 6, (n // 5,), generator=g)
    slots, pos = list(range(n)), pos.tolist()
    append_keys(dev, y, rope, x, slots, pos)
    z = x.double().reshape(n, 2, hk, d)
    z[:, 0] = exactly(rope, z[:, 0], pos)[0]
    y.ref.append(z, slots)
    y.check()


def test_angles_backwards_are_those_of_positions_backwards(dev):
    rope, back = planned(64, 0, "forwards"), planned(64, 0, "backwards")
    x = rows_of(84, 300, 64, 0, torch.bfloat16, dev)[:300].to(dev)
    pos = (torch.arange(300, device=dev) * 987654321) ** 2 % (1 << 45)
    out = [torch.empty_like(x) for _ in range(2)]
    shape = shape_of(0, 1, 1, 64, 16, 1, 1, "bf16")
    for r, p, o in ((rope, -pos, out[0]), (back, pos, out[1])):
        hs.hs_rope_apply(shape, r, x, None, 0, p, 300, o, 0, None, 0)
    assert torch.equal(out[0], out[1])


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("amplitude,size", [(1.0, 3e38), (2.0 ** 20, 2.0 ** 107 * 1.5)])
def test_turned_keys_beyond_float32_count_as_not_finite(dev, layout, amplitude, size):
    """One pair of equal elements at an eighth of a turn: one turned value is sqrt 2 of its size, and the other, which is near 0,
    rounding alone."""
    rope = hs.hs_rope_plan(64, layout, 10000.0, amplitude=amplitude)
    n, pair = 40, 5
    rope.theta[pair] = math.pi / 4
    at = [(pair, pair + 32), (2 * pair, 2 * pair + 1)][layout]
    y = Layer(dev, 1, 64, 16, "bf16", 3)
    x = rows_of(85, n, 128, 0, torch.bfloat16, dev)[:n]
    x[3, list(at)] = x[20, list(at)] = size
    pos = [0] * n
    pos[3] = pos[20] = 1
    append_keys(dev, y, rope, x, list(range(n)), pos)
    z = x.double().reshape(n, 2, 1, 64)
    z[:, 0] = exactly(rope, z[:, 0], pos)[0]
    assert size * amplitude < torch.finfo(torch.float32).max < z[3, 0, 0, at[1]] == z[20, 0, 0, at[1]]
    z[3, 0, 0, list(at)] = z[20, 0, 0, list(at)] = math.nan
    y.ref.append(z, list(range(n)))
    y.check()
