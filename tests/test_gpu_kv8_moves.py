"""Blocks of the 8-bit cache, whose scales lie in them, through the calls that move pages: a request restored with its
states, and one rank's heads."""
import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.gpu_helpers import device
from tests.kv8_helpers import filled, shape_of
from tests.test_gpu_kv8 import decoded, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


@pytest.mark.parametrize("heads,kv_heads,d,page", [(16, 4, 128, 16), (14, 2, 64, 32)])
def test_a_request_restored_with_its_states(dev, heads, kv_heads, d, page):
    """Two layers' blocks and three states in one call, into other blocks: the answers are the same bits."""
    n = 9 * page
    layers = [filled(100 + i, [n], kv_heads, page, d) for i in range(2)]
    size = layers[0][0].size()
    blocks = layers[0][0].blocks
    staging = [c.image()[table[0].long()].to(dev) for c, table in layers]
    caches = [torch.full((blocks, size), 0xEE, dtype=torch.uint8, device=dev) for _ in layers]
    states = torch.randn(3, 2, 64, 64, device=dev)
    live = torch.zeros_like(states)
    other = torch.randperm(blocks, generator=torch.Generator().manual_seed(1))[:9].int()
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    hs.hs_restore_request(hs.ptr_array(staging, dev), hs.ptr_array(caches, dev), 2, other.to(dev), 9, size, blocks,
                          hs.ptr_array(list(states), dev), hs.ptr_array(list(live), dev), 3, 2 * 64 * 64, err)
    torch.cuda.synchronize()
    assert err.item() == 0 and torch.equal(live, states)
    q = rows_of(102, 1, heads * d, 0, torch.bfloat16, dev)
    for (c, table), cache in zip(layers, caches):
        got = cache.cpu()
        assert torch.equal(got[other.long()], c.image()[table[0].long()])
        left = torch.ones(blocks, dtype=torch.bool)
        left[other.long()] = False
        assert (got[left] == 0xEE).all()
        want = decoded(dev, c, table, q, heads, "bf16", [n], n)[0]
        shape = shape_of(1, heads, kv_heads, d, page, blocks, 9, "bf16")
        need = hs.hs_kv8_decode_workspace_bytes(shape, n)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
        o = torch.empty(1, heads * d, dtype=torch.bfloat16, device=dev)
        hs.hs_kv8_decode(shape, q.to(dev), cache, other.reshape(1, 9).to(dev), torch.tensor([n], dtype=torch.int32, device=dev),
                         n, o, None, ws, need, err)
        torch.cuda.synchronize()
        assert err.item() == 0 and torch.equal(o.cpu(), want)


@pytest.mark.parametrize("kv_heads,d,page,first,count", [(4, 128, 32, 1, 1), (4, 128, 16, 2, 2), (3, 64, 64, 2, 1),
                                                         (8, 64, 16, 0, 2)])
def test_one_ranks_heads(dev, kv_heads, d, page, first, count):
    """A rank's values and scales saved and restored as two slices: its heads arrive, the others' bytes stay."""
    c, table = filled(103, [7 * page], kv_heads, page, d)
    image, size, ids = c.image(), c.size(), table[0].to(dev)
    B, S = 2 * page * d, page // 2
    source, cache = image.to(dev), torch.full_like(image, 0xEE, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    owned = torch.zeros(size, dtype=torch.bool)
    for off, n in ((first * B, count * B), (kv_heads * B + first * S, count * S)):
        owned[off:off + n] = True
        staging = torch.zeros(7, n, dtype=torch.uint8, device=dev)
        hs.hs_save_kv_page_slices(hs.ptr_array([source], dev), hs.ptr_array([staging], dev), 1, ids, 7, size, 1, off, n,
                                  c.blocks, err)
        hs.hs_restore_kv_page_slices(hs.ptr_array([staging], dev), hs.ptr_array([cache], dev), 1, ids, 7, size, 1, off, n,
                                     c.blocks, err)
    torch.cuda.synchronize()
    assert err.item() == 0
    got = cache.cpu()
    here = torch.zeros(c.blocks, dtype=torch.bool)
    here[table[0].long()] = True
    assert torch.equal(got[here][:, owned], image[here][:, owned])
    assert (got[~here] == 0xEE).all() and (got[here][:, ~owned] == 0xEE).all()
