"""The full-attention calls against float64 at the bounds that include/hs_attn.h documents, in forms that the other
tests do not reach: many split items, long contexts, more than 2^22 units of work, every request of a step
behind a shared prefix."""
import math

import pytest
import torch

import paper_2609_15030_gb300 as hs
from tests.attn_cases import MANY_SPLIT
from tests.attn_helpers import DT, Problem, cu_of, run_decode, run_prefill, workspace
from tests.gpu_helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


def exact(q, k, v, group, scale, dtype):
    """(o, lse, bounds) of one query row [heads][d] over keys and values [n][kv heads][d], float64 wherever
    the inputs lie.  Weights and output: half a step of the element type each, of fp16 weights half a step of
    2^-32 of the row's largest where that is more; scores: d products and the scaling, one step of float32 each, on
    the sum of magnitudes; the sums: 2^-26 of them a key (the tensor core drops what lies below)."""
    n, hk, d = k.shape
    q = q.double().reshape(hk, group, d)
    kd, vd = k.double(), v.double()
    s = torch.einsum("agd,nad->agn", q, kd) * scale
    lse = torch.logsumexp(s, dim=2)
    w = (s - lse[..., None]).exp()
    o = torch.einsum("agn,nad->agd", w, vd)
    mag = torch.einsum("agn,nad->agd", w, vd.abs())
    size = torch.einsum("agd,nad->agn", q.abs(), kd.abs()) * scale
    ds = ((d + 4) * 2.0 ** -23 * size).amax(dim=2) + 2.0 ** -20 * (1 + s.abs().amax(dim=2))
    u = torch.finfo(dtype).eps / 2
    off = (u + 2 * ds[..., None] + n * 2.0 ** -26) * mag + u * o.abs()
    if dtype == torch.float16:
        off = off + 2.0 ** -33 * w.amax(dim=2)[..., None] * vd.abs().sum(dim=0)[:, None]
        off = off + 2.0 ** -25                      # half a step of the smallest outputs
    h = hk * group
    return o.reshape(h, d), lse.reshape(h), (off * (1 + 2 * u)).reshape(h, d), (ds + n * 2.0 ** -24).reshape(h)


class Tight(Problem):
    def row(self, r, k, v):
        if k.shape[0] == 0:
            return super().row(r, k, v)
        q = self.q[r, :self.heads * self.d]
        scale = torch.tensor(self.scale, dtype=torch.float32).item()
        return exact(q, k, v, self.group, scale, DT[self.dtype])

    def some_rows(self, pos0, n_tokens, cu, rows):
        """rows(n): the tokens of a request of n that are looked at."""
        for b, (p, n) in enumerate(zip(pos0, n_tokens)):
            for t in rows(n):
                yield (cu[b] + t, *self.row(cu[b] + t, self.K[b][:p + t + 1], self.V[b][:p + t + 1]))


def check_rows(out, rows):
    torch.cuda.synchronize()
    assert out.err.item() == 0
    p, o, lse = out.p, out.o.cpu(), out.lse.cpu()
    for r, want, want_lse, bound, bound_lse in rows:
        off = (o[r, :p.heads * p.d].double().reshape(p.heads, p.d) - want).abs()
        assert (off <= bound).all(), (r, (off / bound).max().item())
        assert ((lse[r].double() - want_lse).abs() <= bound_lse).all(), r


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("which", range(len(MANY_SPLIT)))
def test_prefill_with_many_split_items(dev, which, dtype, d):
    heads, kv_heads, pos0, n = MANY_SPLIT[which]
    p = Tight(61, heads, kv_heads, d, 16, dtype, [a + b for a, b in zip(pos0, n)], sum(n))
    assert hs.hs_attn_prefill_workspace_bytes(p.shape(len(n)), pos0, n) > 0
    out = run_prefill(p, pos0, n, dev)
    check_rows(out, p.some_rows(pos0, n, cu_of(n), lambda m: sorted({0, 31, m // 2, m - 2, m - 1})))
    again = run_prefill(p, pos0, n, dev)
    assert torch.equal(out.o.view(torch.int16), again.o.view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("sharp", [1.0, 4.0])
def test_small_weights_at_the_documented_step(dev, dtype, sharp):
    """Keys far below the largest, whose weights are small: what is allowed for these is 2^-33 of the largest."""
    pos0, n = [700, 3000, 0], [40, 3, 70]
    p = Tight(62, 6, 2, 64, 32, dtype, [a + b for a, b in zip(pos0, n)], sum(n), sharp=sharp)
    for unsplit in (False, True):
        out = run_prefill(p, pos0, n, dev, unsplit=unsplit)
        out.check(p.prefill_rows(pos0, n, cu_of(n)))
    kv_len = [3000, 17, 70]
    q = Tight(63, 6, 2, 128, 16, dtype, kv_len, 3, prefix_len=500, sharp=sharp)
    run_decode(q, kv_len, 3000, dev).check(q.decode_rows(kv_len))


@pytest.mark.parametrize("heads,kv_heads,d,dtype", [(4, 1, 128, "bf16"), (2, 2, 64, "fp16")])
def test_contexts_of_100k_keys(dev, heads, kv_heads, d, dtype):
    pos0, n = [100_000, 131_000], [37, 72]
    p = Tight(64, heads, kv_heads, d, 32, dtype, [a + b for a, b in zip(pos0, n)], sum(n), prefix_len=70_001)
    check_rows(run_prefill(p, pos0, n, dev), p.some_rows(pos0, n, cu_of(n), lambda m: [0, m // 2, m - 1]))
    kv_len = [100_037, 131_072]
    run_decode(p, kv_len, 131_072, dev, shared=True).check(p.decode_rows(kv_len))
    run_decode(p, kv_len, 131_072, dev, shared=False).check(
        (b, *p.row(b, p.K[b][:m], p.V[b][:m])) for b, m in enumerate(kv_len))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,d,prefix,batch", [(16, 4, 128, 1040, 11), (8, 8, 64, 320, 40)])
def test_every_request_behind_a_shared_prefix_and_over_whole_tables(dev, heads, kv_heads, d, prefix, batch, dtype):
    """The same keys through the prefix's table and through tables of their own that begin with its pages."""
    kv_len = [1 + (29 * b) % 90 for b in range(batch)]
    p = Tight(65, heads, kv_heads, d, 16, dtype, kv_len, batch, prefix_len=prefix)
    run_decode(p, kv_len, 90, dev).check(p.decode_rows(kv_len))
    whole = Tight(65, heads, kv_heads, d, 16, dtype, kv_len, batch, prefix_len=prefix)
    whole.table = torch.cat((p.prefix_table.expand(batch, -1), p.table), dim=1).contiguous()
    run_decode(whole, [prefix + x for x in kv_len], prefix + 90, dev, shared=False).check(p.decode_rows(kv_len))


# ---- more than 2^22 units of work: counts of units times CTAs pass 32 bits ----------------------------------


def cache_of(dev, blocks, page, kv_heads, d, dt, seed):
    g = torch.Generator(device=dev).manual_seed(seed)
    cache = torch.empty(blocks, 2, page, kv_heads, d, dtype=dt, device=dev)
    return cache.normal_(generator=g), g


def test_prefill_of_131072_tokens(dev):
    heads, kv_heads, d, page, n, dt = 32, 8, 64, 64, 131_072, torch.bfloat16
    cache, g = cache_of(dev, n // page, page, kv_heads, d, dt, 66)
    table = torch.randperm(n // page, device=dev, generator=g).int()[None].contiguous()
    q = torch.empty(n, heads, d, dtype=dt, device=dev).normal_(generator=g)
    o, lse = torch.full_like(q, math.nan), torch.full((n, heads), math.nan, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    shape = hs.make_attn_shape(1, heads, kv_heads, d, page, n // page, n // page)
    size = hs.hs_attn_prefill_workspace_bytes(shape, [0], [n])
    hs.hs_attn_prefill(shape, q, cache, table, o, lse, [0], [n], [0, n], workspace(size, dev), size, err)
    torch.cuda.synchronize()
    assert err.item() == 0
    k, v = (cache[table[0].long(), i].reshape(n, kv_heads, d) for i in (0, 1))
    for r in [0, 1, 63, 64, 127, 128, 16_383, 50_001, 65_535, 65_536, 92_682, 100_003, 120_000, n - 2, n - 1]:
        want, want_lse, bound, bound_lse = exact(q[r], k[:r + 1], v[:r + 1], heads // kv_heads, shape.scale, dt)
        assert ((o[r].double() - want).abs() <= bound).all(), r
        assert ((lse[r].double() - want_lse).abs() <= bound_lse).all(), r
    assert torch.isfinite(lse).all() and torch.isfinite(o).all()


def test_decode_of_384_requests_at_180224_keys(dev):
    """All requests' tables list the same pages, each from another place on."""
    batch, kv_heads, d, page, n, dt = 384, 8, 64, 64, 180_224, torch.float16
    pages = n // page
    cache, g = cache_of(dev, pages, page, kv_heads, d, dt, 67)
    table = ((torch.arange(pages, device=dev)[None] + 7 * torch.arange(batch, device=dev)[:, None]) % pages).int()
    lens = (n - 1000 * (torch.arange(batch, device=dev) % 3)).int()
    q = torch.empty(batch, kv_heads, d, dtype=dt, device=dev).normal_(generator=g)
    o, lse = torch.full_like(q, math.nan), torch.full((batch, kv_heads), math.nan, device=dev)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    shape = hs.make_attn_shape(batch, kv_heads, kv_heads, d, page, pages, pages, hs.HS_FP16)
    size = hs.hs_attn_decode_workspace_bytes(shape, n)
    assert size > 0
    hs.hs_attn_decode(shape, q, cache, table, lens, n, o, lse, workspace(size, dev), size, err)
    torch.cuda.synchronize()
    assert err.item() == 0
    for b in [0, 1, 2, 100, 191, 256, 382, 383]:
        k, v = (cache[table[b].long(), i].reshape(n, kv_heads, d)[:lens[b]] for i in (0, 1))
        want, want_lse, bound, bound_lse = exact(q[b], k, v, 1, shape.scale, dt)
        assert ((o[b].double() - want).abs() <= bound).all(), b
        assert ((lse[b].double() - want_lse).abs() <= bound_lse).all(), b
    assert torch.isfinite(lse).all() and torch.isfinite(o).all()
