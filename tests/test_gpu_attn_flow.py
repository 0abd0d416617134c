"""The full-attention calls together with the restore path, as an engine runs one layer: recompute,
save, restore, append the tail, resume, decode, and decode behind a shared prefix."""
import math

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.attn_helpers import DT, HSDT, workspace
from tests.gpu_helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


class Layer:
    """One full-attention layer: a cache, and a step of it for new tokens."""

    def __init__(self, dev, heads, kv_heads, d, page, blocks, dtype):
        self.dev, self.heads, self.kv_heads, self.d, self.page = dev, heads, kv_heads, d, page
        self.blocks, self.dtype, self.dt = blocks, dtype, DT[dtype]
        self.cache = torch.full((blocks, 2, page, kv_heads, d), math.nan, dtype=self.dt, device=dev)
        self.err = torch.zeros(1, dtype=torch.int32, device=dev)
        self.page_bytes = 2 * page * kv_heads * d * 2

    def shape(self, batch, width, **kw):
        row = (self.heads + 2 * self.kv_heads) * self.d
        return hs.make_attn_shape(batch, self.heads, self.kv_heads, self.d, self.page, self.blocks, width,
                                  HSDT[self.dtype], q_stride=row, **kw)

    def append(self, qkv, table, pos):
        """qkv: rows of a fused projection; the tokens of one request from position pos on."""
        h, hk, d = self.heads, self.kv_heads, self.d
        n = qkv.shape[0]
        at = torch.arange(pos, pos + n, device=self.dev)
        slots = table[at // self.page].long() * self.page + at % self.page
        base = qkv.data_ptr()
        hs.hs_kv_append(self.shape(0, 0), base + h * d * 2, base + (h + hk) * d * 2, qkv.shape[1], slots, n,
                        self.cache, self.err)
        return slots

    def prefill(self, qkv, table, pos, **kw):
        n = qkv.shape[0]
        shape = self.shape(1, table.numel(), **kw)
        size = hs.hs_attn_prefill_workspace_bytes(shape, [pos], [n])
        ws = workspace(size, self.dev)
        o = torch.full((n, self.heads, self.d), math.nan, dtype=self.dt, device=self.dev)
        hs.hs_attn_prefill(shape, qkv, self.cache, table, o, None, [pos], [n], [0, n], ws, size, self.err)
        return o

    def exact(self, qkv, rows):
        """float64 outputs of the listed rows of the whole prompt's projection."""
        h, hk, d = self.heads, self.kv_heads, self.d
        x = qkv.double().cpu().reshape(qkv.shape[0], h + 2 * hk, d)
        out = []
        for t in rows:
            q = x[t, :h].reshape(hk, h // hk, d)
            k, v = x[:t + 1, h:h + hk], x[:t + 1, h + hk:]
            w = torch.softmax(torch.einsum("agd,nad->agn", q, k) / math.sqrt(d), dim=2)
            out.append(torch.einsum("agn,nad->agd", w, v).reshape(h, d))
        return torch.stack(out)


def close(got, want, dtype):
    # two roundings of half a step (weights, output) relative to sums of |w v|, at most the largest
    # |v| of about 5: eps * 5 bounds both
    assert (got.double().cpu() - want).abs().max().item() <= 5 * torch.finfo(DT[dtype]).eps


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,d,page,N,c", [(8, 2, 64, 16, 256, 192), (16, 4, 128, 16, 700, 512),
                                                      (6, 2, 128, 32, 400, 0)])
def test_resume_equals_recompute_and_decodes_on(dev, dtype, heads, kv_heads, d, page, N, c):
    g = torch.Generator().manual_seed(N)
    steps, width = 5, -(-(N + 5) // page)
    qkv = torch.randn(N + steps, (heads + 2 * kv_heads) * d, generator=g).to(DT[dtype]).to(dev)
    blocks = 2 * width + 3
    ids = torch.randperm(blocks, generator=g).int().to(dev)
    cold = Layer(dev, heads, kv_heads, d, page, blocks, dtype)
    table = ids[:width].contiguous()
    cold.append(qkv[:N], table, 0)
    full = cold.prefill(qkv[:N], table, 0, unsplit=True)
    # save the pages of [0, c), restore them elsewhere in another cache with a linear layer's state
    n_pages = c // page
    staging = torch.zeros(max(n_pages, 1) * cold.page_bytes, dtype=torch.uint8, device=dev)
    hs.hs_save_kv_pages(hs.ptr_array([cold.cache], dev), hs.ptr_array([staging], dev), 1, table, n_pages,
                        cold.page_bytes, blocks, cold.err)
    warm = Layer(dev, heads, kv_heads, d, page, blocks, dtype)
    other = ids[width:2 * width].contiguous()
    slot, live = torch.randn(64, device=dev), torch.zeros(64, device=dev)
    hs.hs_restore_request(hs.ptr_array([staging], dev), hs.ptr_array([warm.cache], dev), 1, other, n_pages,
                          warm.page_bytes, blocks, hs.ptr_array([slot], dev), hs.ptr_array([live], dev), 1, 64,
                          warm.err)
    warm.append(qkv[c:N], other, c)
    tail = warm.prefill(qkv[c:N], other, c, unsplit=True)
    assert torch.equal(tail.view(torch.int16), full[c:].view(torch.int16))
    split = warm.prefill(qkv[c:N], other, c)
    rows = sorted({c, (c + N) // 2, N - 1})
    want = cold.exact(qkv[:N], rows)
    close(full[rows], want, dtype)
    close(split[[t - c for t in rows]], want, dtype)
    # decode on from the resumed cache, one token a step
    shape = warm.shape(1, width)
    size = hs.hs_attn_decode_workspace_bytes(shape, width * page)
    ws = workspace(size, dev)
    for t in range(N, N + steps):
        warm.append(qkv[t:t + 1], other, t)
        o = torch.full((1, heads, d), math.nan, dtype=DT[dtype], device=dev)
        hs.hs_attn_decode(shape, qkv[t], warm.cache, other, torch.tensor([t + 1], dtype=torch.int32, device=dev),
                          width * page, o, None, ws, size, warm.err)
        torch.cuda.synchronize()
        close(o, warm.exact(qkv, [t]), dtype)
    assert torch.equal(slot, live)
    assert cold.err.item() == 0 and warm.err.item() == 0


def test_a_captured_step_appends_and_decodes(dev):
    """One graph of append and decode, replayed for every token: slots, lengths and rows change in place."""
    heads, kv_heads, d, page, N, steps = 8, 2, 128, 16, 150, 40
    g = torch.Generator().manual_seed(3)
    layer = Layer(dev, heads, kv_heads, d, page, 40, "bf16")
    qkv = torch.randn(2, N + steps, (heads + 2 * kv_heads) * d, generator=g).bfloat16().to(dev)
    width = -(-(N + steps) // page)
    table = torch.randperm(40, generator=g)[:2 * width].int().reshape(2, width).to(dev)
    for b in range(2):
        layer.append(qkv[b, :N], table[b], 0)
    now = torch.zeros(2, qkv.shape[2], dtype=torch.bfloat16, device=dev)
    slots, lens = torch.zeros(2, dtype=torch.int64, device=dev), torch.zeros(2, dtype=torch.int32, device=dev)
    o = torch.zeros(2, heads, d, dtype=torch.bfloat16, device=dev)
    shape = layer.shape(2, width)
    size = hs.hs_attn_decode_workspace_bytes(shape, N + steps)
    ws = workspace(size, dev)

    def step(stream):
        base = now.data_ptr()
        hs.hs_kv_append(layer.shape(0, 0), base + heads * d * 2, base + (heads + kv_heads) * d * 2, now.shape[1],
                        slots, 2, layer.cache, layer.err, stream)
        hs.hs_attn_decode(shape, now, layer.cache, table, lens, N + steps, o, None, ws, size, layer.err, stream)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for t in range(N, N + steps):
        now.copy_(qkv[:, t])
        slots.copy_(table[:, t // page].long() * page + t % page)
        lens.fill_(t + 1)
        graph.replay()
        if t % 13 == 0 or t == N + steps - 1:
            torch.cuda.synchronize()
            for b in range(2):
                close(o[b:b + 1], layer.exact(qkv[b], [t]), "bf16")
    assert layer.err.item() == 0


def test_decode_behind_a_shared_prefix_equals_decode_over_whole_tables(dev):
    heads, kv_heads, d, page, prefix, batch = 16, 4, 128, 16, 1040, 11
    g = torch.Generator().manual_seed(4)
    own = [int(x) for x in torch.randint(1, 90, (batch,), generator=g)]
    width, shared = -(-max(own) // page), prefix // page
    layer = Layer(dev, heads, kv_heads, d, page, shared + batch * width + 1, "bf16")
    ids = torch.randperm(layer.blocks, generator=g).int().to(dev)
    pre, table = ids[:shared].contiguous(), ids[shared:shared + batch * width].reshape(batch, width).contiguous()
    first = torch.randn(prefix, (heads + 2 * kv_heads) * d, generator=g).bfloat16().to(dev)
    layer.append(first, pre, 0)
    rest = []
    for b in range(batch):
        rest.append(torch.randn(own[b], first.shape[1], generator=g).bfloat16().to(dev))
        layer.append(rest[b], table[b], 0)
    q = torch.stack([x[-1] for x in rest])
    lens = torch.tensor(own, dtype=torch.int32, device=dev)
    o, lse = (torch.zeros(batch, heads, *x, dtype=t, device=dev)
              for x, t in (((d,), torch.bfloat16), ((), torch.float32)))
    shape = layer.shape(batch, width)
    size = hs.hs_attn_decode_shared_workspace_bytes(shape, prefix, width * page)
    hs.hs_attn_decode_shared(shape, q, layer.cache, pre, prefix, table, lens, width * page, o, lse,
                             workspace(size, dev), size, layer.err)
    whole = torch.cat((pre.expand(batch, -1), table), dim=1).contiguous()
    o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
    shape = layer.shape(batch, whole.shape[1])
    size = hs.hs_attn_decode_workspace_bytes(shape, prefix + width * page)
    hs.hs_attn_decode(shape, q, layer.cache, whole, lens + prefix, prefix + width * page, o2, lse2,
                      workspace(size, dev), size, layer.err)
    torch.cuda.synchronize()
    assert layer.err.item() == 0
    for b in (0, batch - 1):
        want = layer.exact(torch.cat((first, rest[b])), [prefix + own[b] - 1])
        close(o[b:b + 1], want, "bf16")
        close(o2[b:b + 1], want, "bf16")
    assert (o.float() - o2.float()).abs().max().item() <= 10 * torch.finfo(torch.bfloat16).eps
    # float32 on both sides: scores of d products, sums of some thousand terms
    assert (lse - lse2).abs().max().item() <= 1e-4


def test_blocks_beyond_4_gib_of_a_cache(dev):
    """Pages at the far end of a 9.2 GB cache: byte offsets beyond 32 bits in every call."""
    heads, kv_heads, d, page, blocks, n = 8, 8, 128, 16, 140_000, 77
    layer = Layer.__new__(Layer)
    layer.dev, layer.heads, layer.kv_heads, layer.d, layer.page = dev, heads, kv_heads, d, page
    layer.blocks, layer.dtype, layer.dt = blocks, "bf16", torch.bfloat16
    layer.err = torch.zeros(1, dtype=torch.int32, device=dev)
    layer.cache = torch.empty(blocks, 2, page, kv_heads, d, dtype=torch.bfloat16, device=dev)
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn(n, (heads + 2 * kv_heads) * d, generator=g).bfloat16().to(dev)
    table = torch.tensor([blocks - 1, 70_000, 3, blocks - 2, 32_768], dtype=torch.int32, device=dev)
    layer.append(qkv, table, 0)
    rows = [0, 40, n - 1]
    o = layer.prefill(qkv, table, 0)
    shape = layer.shape(1, 5)
    size = hs.hs_attn_decode_workspace_bytes(shape, n)
    one = torch.zeros(1, heads, d, dtype=torch.bfloat16, device=dev)
    hs.hs_attn_decode(shape, qkv[n - 1], layer.cache, table, torch.tensor([n], dtype=torch.int32, device=dev), n,
                      one, None, workspace(size, dev), size, layer.err)
    torch.cuda.synchronize()
    assert layer.err.item() == 0
    want = layer.exact(qkv, rows)
    close(o[rows], want, "bf16")
    close(one, want[2:], "bf16")


def test_workspaces_that_are_too_small_are_refused(dev):
    # 240 items of many keys: shared out over CTAs, whose sums go through the workspace
    B = 30
    shape = hs.make_attn_shape(B, 32, 8, 128, 16, 1000, 400)
    lens, cu = ([4000] * B, [40] * B), [40 * b for b in range(B + 1)]
    for size, call in (
            (hs.hs_attn_prefill_workspace_bytes(shape, *lens),
             lambda ws, n: hs.hs_attn_prefill(shape, 1 << 20, 1 << 20, 1 << 20, 1 << 20, None, *lens, cu, ws, n)),
            (hs.hs_attn_decode_workspace_bytes(shape, 6000),
             lambda ws, n: hs.hs_attn_decode(shape, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 6000, 1 << 20, None,
                                             ws, n)),
            (hs.hs_attn_decode_shared_workspace_bytes(shape, 100, 10),
             lambda ws, n: hs.hs_attn_decode_shared(shape, 1 << 20, 1 << 20, 1 << 20, 100, 1 << 20, 1 << 20, 10,
                                                    1 << 20, None, ws, n))):
        assert size > 0 and size % 16 == 0
        for ws, n in ((1 << 20, size - 1), (None, size), (None, 0)):
            with pytest.raises(hs.HsError) as e:      # refused on the host: the addresses are never read
                call(ws, n)
            assert e.value.status == hs.HS_ERR_INVALID_ARG
