"""Appends of groups with skipped rows among their rows: every byte."""
import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.gpu_helpers import device
from tests.kv8_helpers import DT, G, turned
from tests.test_gpu_kv8 import Layer, append_keys, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def thinned(seed, page, blocks, lengths, share, gaps):
    """Slots of requests in the order of their tokens, `share` of them skipped, runs of skipped rows between requests."""
    g = torch.Generator().manual_seed(seed)
    order, slots = torch.randperm(blocks, generator=g).tolist(), []
    for n in lengths:
        first = int(torch.randint(0, page, (1,), generator=g))
        pages = [order.pop() for _ in range(-(-(first + n) // page))]
        one = [b * page + i for b in pages for i in range(page)][first:first + n]
        drop = (torch.rand(n, generator=g) < share).tolist()
        slots += [-1 - int(torch.randint(0, 5, (1,), generator=g)) if d else s for s, d in zip(one, drop)]
        slots += [-1] * gaps[int(torch.randint(0, len(gaps), (1,), generator=g))]
    return slots


CASES = [(2, 64, 16, "bf16"), (8, 128, 32, "fp16"), (3, 128, 64, "bf16"), (1, 64, 256, "fp16")]


@pytest.mark.parametrize("share", [0.05, 0.5, 0.9])
@pytest.mark.parametrize("kv_heads,d,page,dtype", CASES)
def test_skipped_rows_inside_groups(dev, kv_heads, d, page, dtype, share):
    lengths = [1, 2, 40, 1, 17, 100, 16, 33, 300, 3, 1, 1, 5, 64]
    blocks = sum(-(-n // page) + 1 for n in lengths)
    slots = thinned(90, page, blocks, lengths, share, [0, 1, 7, 15, 31, 33, 100])
    n, w = len(slots), kv_heads * d
    y = Layer(dev, kv_heads, d, page, dtype, blocks)
    y.append(91, list(range(0, blocks * page, G)), loud=0.25)          # every group is begun
    y.append(92, slots, loud=2.0)
    y.check()
    rope = hs.hs_rope_plan(d, 0, 10000.0)
    x, pos = rows_of(93, n, 2 * w, 0, DT[dtype], dev, loud=5.0)[:n], list(range(n))
    append_keys(dev, y, rope, x, slots, pos)
    z = x.double().reshape(n, 2, kv_heads, d)
    z[:, 0] = turned(rope, z[:, 0], pos)[0]
    y.ref.append(z, slots)
    y.check()


@pytest.mark.parametrize("before", [0, 1, 14, 15, 16, 31, 32, 47])
def test_a_groups_ends_alone(dev, before):
    """The first and the last token of a group 15 rows apart, at every place of a window of rows."""
    y = Layer(dev, 2, 128, 16, "bf16", 8)
    y.append(94, list(range(0, 8 * 16, G)), loud=0.25)
    y.append(95, [-1] * before + [33] + [-1] * 13 + [46, 50] + [-1] * 14 + [63, 64], loud=4.0)
    y.check()


def test_slots_out_of_range_inside_a_group(dev):
    y = Layer(dev, 1, 64, 16, "bf16", 3)
    y.append(96, list(range(0, 48, G)), loud=0.25)
    y.append(97, [3, 48, 4, 1 << 40, -5, 9, 20], loud=4.0)
    y.check(hs.HS_DEVERR_BLOCK_OOB)
