"""Long contexts: more keys than the other tests, and a call that one CTA works on for longer than a second."""
import math

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.gpu_helpers import device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch", [1, 33])      # without and behind a shared prefix, whose items have two tiles of rows
def test_one_cta_works_longer_than_a_second(batch):
    """320 million keys unsplit, all but seven in the same few pages: 2.5 million tiles, one after another.  The
    warps that make values at masked places finite (and with two tiles of rows one of the groups) wait for all
    of it.  The last seven keys have scores of 0, the others of -30 in units of log2 and values of 1 and -1 in
    turn, whose products cancel."""
    dev = device()
    n, d, page, dt = 320_000_007, 64, 256, torch.bfloat16
    pages = -(-n // page)
    assert n % page == 7
    cache = torch.zeros(4, 2, page, 1, d, dtype=dt, device=dev)
    cache[:3, 0, ..., 0] = -30
    cache[:3, 1, 0::2], cache[:3, 1, 1::2] = 1, -1
    cache[3] = math.nan
    cache[3, 0, :7] = 0
    cache[3, 1, :7] = torch.arange(1, 8, device=dev)[:, None, None].to(dt)
    table = torch.zeros(batch, pages, dtype=torch.int32, device=dev)
    table[0] = torch.arange(pages, dtype=torch.int32, device=dev) % 3
    table[0, -1] = 3
    lens = torch.arange(batch, dtype=torch.int32, device=dev) % 5
    lens[0] = n
    q = torch.zeros(batch, 4, d, dtype=dt, device=dev)
    q[..., 0] = 1
    o, lse = torch.full_like(q, math.nan), torch.zeros(batch, 4, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    shape = hs.make_attn_shape(batch, 4, 1, d, page, 4, pages, scale=math.log(2), unsplit=True)
    prefix = 100 if batch > 1 else 0
    pre = torch.ones(1, dtype=torch.int32, device=dev)
    size = hs.hs_attn_decode_shared_workspace_bytes(shape, prefix, n)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device=dev)
    hs.hs_attn_decode_shared(shape, q, cache, pre, prefix, table, lens, n, o, lse, ws, size, err)
    torch.cuda.synchronize()
    assert err.item() == 0
    for b in range(batch):
        keys = lens[b].item() + prefix
        total = keys * 2.0 ** -30 if b else 7 + (keys - 7) * 2.0 ** -30
        want = (lens[b].item() % 2) / keys if b else 28 / total
        # weights of 2^0 are exact: the output's rounding is left, and float32 ones of the sums
        assert (o[b].double() - want).abs().max().item() <= 2.0 ** -8 * want + 2.0 ** -16
        # of 21: the scale's two roundings, the maximum's, the logarithm's and the result's, 2^-24 each
        assert (lse[b].double() - math.log(total)).abs().max().item() <= 2.0 ** -16
