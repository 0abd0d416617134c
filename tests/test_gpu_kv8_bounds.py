"""The decode step over the 8-bit cache within bounds that follow its documented roundings one by one
(tests/kv8_tight.py)."""
import math

import pytest
import torch

from tests.gpu_helpers import device
from tests.kv8_helpers import DT, filled, keys_of
from tests.kv8_tight import bounded, one_element_rows
from tests.test_gpu_kv8 import DECODE, decoded, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def scale_of(c, table, b, n):
    """The largest scale of a request's values, by KV head."""
    pages = table[b, :-(-n // c.page)].long()
    x = c.scales[pages, :, 1].permute(1, 0, 2).flatten(1)[:, :-(-n // 16)]
    return x.amax(dim=1)


def excess(c, table, q, heads, dtype, b, n, o, z, scale):
    """How far one request's outputs are beyond their bounds: the largest quotient, of o and of lse."""
    k, v = keys_of(c, table, b, n)
    x = q[b, :heads * c.d].double().reshape(c.kv_heads, heads // c.kv_heads, c.d)
    want, want_z, bound, bound_z = bounded(x, k, v, scale_of(c, table, b, n), scale, dtype)
    return (((o[b].double().reshape(want.shape) - want).abs() / bound).max().item(),
            ((z[b].double().reshape(want_z.shape) - want_z).abs() / bound_z).max().item())


SHAPES = [(8, 2, 128, 16, "bf16"), (16, 1, 128, 32, "bf16"), (12, 2, 64, 16, "bf16"), (32, 1, 64, 16, "bf16"),
          (8, 2, 128, 16, "fp16"), (16, 1, 64, 32, "fp16")]


@pytest.mark.parametrize("unsplit", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,page,dtype", SHAPES)
def test_weights_keep_more_bits_than_the_outputs(dev, heads, kv_heads, d, page, dtype, unsplit):
    """Outputs whose keys' shares cancel show what the weights lost."""
    lens = [2, 3, 5, 9, 17, 40, 100, 333, 1000, 1]
    c, table = filled(60, lens, kv_heads, page, d)
    q = one_element_rows(61, len(lens), heads, d, DT[dtype])
    o, z, err = decoded(dev, c, table, q, heads, dtype, lens, max(lens), scale=0.25, unsplit=unsplit)
    assert err == 0
    for b, n in enumerate(lens):
        over, over_z = excess(c, table, q, heads, dtype, b, n, o, z, 0.25)
        assert over <= 1 and over_z <= 1, (b, n, over, over_z)


@pytest.mark.parametrize("heads,kv_heads,d,page", [(4, 2, 128, 16), (12, 1, 128, 32), (3, 1, 64, 16), (20, 2, 64, 16)])
@pytest.mark.parametrize("e", [119, 112, 96])
def test_sums_of_large_values_stay_in_range(dev, heads, kv_heads, d, page, e):
    """Averages far below bf16's largest number whose sums are beyond float32, of either sign, however a row's keys
    are shared out."""
    lens = [3000, 1, 17, 250, 40]
    c, table = filled(62, lens, kv_heads, page, d, spread=0)
    c.bytes[:, :, 1] = torch.where(c.bytes[:, :, 1] % 128 > 56, c.bytes[:, :, 1] - 16, c.bytes[:, :, 1])   # 448 to 60
    c.scales[:, :, 1] *= 2.0 ** (e + 8)
    q = one_element_rows(63, len(lens), heads, d, torch.bfloat16, loud=4.0)
    for unsplit in (False, True):
        o, z, err = decoded(dev, c, table, q, heads, "bf16", lens, max(lens), scale=0.25, unsplit=unsplit)
        assert err == 0
        for b, n in enumerate(lens):
            over, over_z = excess(c, table, q, heads, "bf16", b, n, o, z, 0.25)
            assert over <= 1 and over_z <= 1, (unsplit, b, n, over, over_z)


@pytest.mark.parametrize("heads,kv_heads,d,page", [(8, 2, 128, 16), (16, 1, 128, 16), (6, 2, 64, 32), (12, 1, 64, 16)])
@pytest.mark.parametrize("e", [-126, -118, -101, -100, -90])
def test_smallest_scales_keep_the_weights_bits(dev, heads, kv_heads, d, page, e):
    """Values whose scales are all near the smallest one, alone and in front of larger ones."""
    lens = [600, 2, 40, 2000, 9]
    c, table = filled(64, lens, kv_heads, page, d, spread=0)
    c.scales[:, :, 1] *= 2.0 ** (e + 8)
    q = one_element_rows(65, len(lens), heads, d, torch.bfloat16)
    for late in (0, 30):
        if late:                     # the second half of each request's pages has larger scales
            for b, n in enumerate(lens):
                pages = table[b, :-(-n // page)].long()
                c.scales[pages[len(pages) // 2:], :, 1] *= 2.0 ** late
        for unsplit in (False, True):
            o, z, err = decoded(dev, c, table, q, heads, "bf16", lens, max(lens), scale=0.25, unsplit=unsplit)
            assert err == 0
            for b, n in enumerate(lens):
                over, over_z = excess(c, table, q, heads, "bf16", b, n, o, z, 0.25)
                assert over <= 1 and over_z <= 1, (late, unsplit, b, n, over, over_z)


@pytest.mark.parametrize("heads,kv_heads,d,dtype", [(8, 2, 128, "bf16"), (16, 1, 128, "fp16"), (12, 2, 64, "bf16"),
                                                    (4, 1, 64, "fp16")])
def test_unsplit_rows_know_nothing_of_their_groups_other_heads(dev, heads, kv_heads, d, dtype):
    """A row depends on its own query and its keys: not on what the other heads of its KV head ask."""
    lens = [900, 64, 2500]
    c, table = filled(66, lens, kv_heads, 16, d)
    q = one_element_rows(67, len(lens), heads, d, DT[dtype], loud=2.0)
    others = one_element_rows(68, len(lens), heads, d, DT[dtype], loud=40.0)
    group = heads // kv_heads
    kept = torch.arange(heads) % group == 1
    mixed = torch.where(kept.repeat_interleave(d), q, others)
    o, z, _ = decoded(dev, c, table, q, heads, dtype, lens, 2500, scale=0.25, unsplit=True)
    o1, z1, _ = decoded(dev, c, table, mixed, heads, dtype, lens, 2500, scale=0.25, unsplit=True)
    assert not torch.equal(o1, o)
    assert torch.equal(o1.unflatten(1, (heads, d))[:, kept], o.unflatten(1, (heads, d))[:, kept])
    assert torch.equal(z1[:, kept], z[:, kept])


# ---- keys that are lost do not meet the bounds ---------------------------------------------


def without(c, table, q, heads, dtype, b, n, scale, first, last):
    """The quotients of the exact outputs of a request without its keys [first, last)."""
    k, v = keys_of(c, table, b, n)
    x = q[b, :heads * c.d].double().reshape(c.kv_heads, heads // c.kv_heads, c.d)
    want, want_z, bound, bound_z = bounded(x, k, v, scale_of(c, table, b, n), scale, dtype)
    keep = (torch.arange(n) < first) | (torch.arange(n) >= last)
    s = (torch.einsum("agd,and->agn", x, k) * scale)[:, :, keep]
    z = torch.logsumexp(s, dim=2)
    o = torch.einsum("agn,and->agd", (s - z[..., None]).exp(), v[:, keep]).to(DT[dtype]).double()
    return ((o - want).abs() / bound).max().item(), ((z - want_z).abs() / bound_z).max().item()


def mark_tiles(seed, c, table, lens):
    """Values of 1 or -1 in one column of each tile of 16 keys, 0 elsewhere, and flat scales: a lost tile, or what is left of
    the last, changes a column by several of its bounds."""
    g = torch.Generator().manual_seed(seed)
    c.scales[:, :, 1] = 2.0 ** -3
    c.bytes[:, :, 1] = 0
    for b, n in enumerate(lens):
        t = torch.arange(-(-n // 16))
        column = (t * 7 + 3) % c.d
        sign = torch.randint(0, 2, t.shape, generator=g)
        at = t[:, None] * 16 + torch.arange(16)
        c.bytes[table[b].long()[at // c.page], :, 1, at % c.page, column[:, None]] = (56 + 128 * sign)[:, None, None]


LONG = [(2, 1, 64, 256, "bf16"), (1, 1, 128, 256, "fp16"), (16, 1, 128, 256, "bf16"), (12, 1, 64, 256, "fp16"),
        (4, 1, 128, 16, "bf16")]
LONG_LENS = [200_003, 30_000, 4_608, 1_000, 33]


def long_case(heads, kv_heads, d, page, dtype):
    c, table = filled(69, LONG_LENS, kv_heads, page, d)
    mark_tiles(71, c, table, LONG_LENS)
    return c, table, one_element_rows(70, len(LONG_LENS), heads, d, DT[dtype])


def lost(n):
    """First and last tiles, one inside, and a block's share of the keys, were the request a call's only one."""
    inside = n // 2 // 16 * 16
    return (0, 16), (inside, inside + 16), ((n - 1) // 16 * 16, n), (n // 3, n // 3 + max(-(-n // 152), 16))


@pytest.mark.parametrize("heads,kv_heads,d,page,dtype", LONG)
def test_every_tile_of_a_context_counts(dev, heads, kv_heads, d, page, dtype):
    """At every length the outputs meet bounds that those without one tile of 16 keys, or one block's share of them, do
    not meet."""
    c, table, q = long_case(heads, kv_heads, d, page, dtype)
    scale = 2.0 ** -6
    both = [decoded(dev, c, table, q, heads, dtype, LONG_LENS, max(LONG_LENS), scale=scale, unsplit=u) for u in (False, True)]
    for b, n in enumerate(LONG_LENS):
        for o, z, err in both:
            over, over_z = excess(c, table, q, heads, dtype, b, n, o, z, scale)
            assert err == 0 and over <= 1 and over_z <= 1, (b, n, over, over_z)
        for first, last in lost(n):
            over, _ = without(c, table, q, heads, dtype, b, n, scale, first, last)
            assert over > 1, (n, first, last, over)


@pytest.mark.parametrize("unsplit", [False, True])
@pytest.mark.parametrize("heads,kv_heads,d,page,dtype,lens", DECODE)
def test_decode_of_dense_queries(dev, heads, kv_heads, d, page, dtype, lens, unsplit):
    """Every head, page size and length of tests/test_gpu_kv8.py, within the bounds of single roundings."""
    c, table = filled(72, lens, kv_heads, page, d)
    q = rows_of(73, len(lens), heads * d, 8, DT[dtype], dev, loud=0.5)
    o, z, err = decoded(dev, c, table, q, heads, dtype, lens, max(lens), unsplit=unsplit)
    assert err == 0
    for b, n in list(enumerate(lens))[:40]:
        if n == 0:
            assert (o[b] == 0).all() and (z[b] == -math.inf).all()
            continue
        over, over_z = excess(c, table, q, heads, dtype, b, n, o, z, d ** -0.5)
        assert over <= 1 and over_z <= 1, (b, n, over, over_z)
