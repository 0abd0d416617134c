"""Seeded problems for the full-attention calls and their float64 results.

Everything a call must not use is NaN: blocks of nobody, the rows behind a request's last key in its
last page, the rows of q, k and v behind the listed ones, the gaps of strided rows.
"""
import math

import torch

import paper_2609_15030_gb300 as hs

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
HSDT = {"bf16": hs.HS_BF16, "fp16": hs.HS_FP16}


class Problem:
    """keys[b] random keys and values of request b (and prefix_len shared ones), in pages at random
    blocks of a cache; q: a row per token, `pad` elements between rows."""

    def __init__(self, seed, heads, kv_heads, d, page, dtype, keys, rows, prefix_len=0, pad=0,
                 sharp=1.0, slope=0.0):
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        self.heads, self.kv_heads, self.d, self.page, self.dtype = heads, kv_heads, d, page, dtype
        self.group, self.scale = heads // kv_heads, 1.0 / math.sqrt(d)
        self.rows, self.pad = rows, pad

        def normal(*shape):
            return torch.randn(shape, generator=g).to(dt)
        self.K, self.V = [], []
        for n in [prefix_len] + list(keys):
            k = torch.randn(n, kv_heads, d, generator=g) * sharp
            # a drift along one direction shared with q: scores grow (or fall) along the keys
            k += slope * torch.arange(n)[:, None, None] * torch.ones(d) / max(n, 1)
            self.K.append(k.to(dt))
            self.V.append(normal(n, kv_heads, d))
        need = [-(-x.shape[0] // page) for x in self.K]
        self.blocks = sum(need) + 3
        order = torch.randperm(self.blocks, generator=g).int()
        self.cache = torch.full((self.blocks, 2, page, kv_heads, d), math.nan, dtype=dt)
        width = max(need[1:] + [1])
        self.table = torch.full((len(keys), width), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            ids = order[at:at + n]
            at += n
            if b == 0:
                self.prefix_table = ids.clone()
            else:
                self.table[b - 1, :n] = ids
            for i, x in enumerate((self.K[b], self.V[b])):
                flat = torch.full((n * page, kv_heads, d), math.nan, dtype=dt)
                flat[:x.shape[0]] = x
                self.cache[ids.long(), i] = flat.reshape(n, page, kv_heads, d)
        self.kp, self.vp = self.K.pop(0), self.V.pop(0)
        q = torch.full((rows + 1, heads * d + pad), math.nan, dtype=dt)
        q[:rows, :heads * d] = normal(rows, heads * d) + (0.2 if slope else 0.0)
        self.q = q

    def shape(self, batch, **kw):
        a = dict(dtype=HSDT[self.dtype], q_stride=self.heads * self.d + self.pad,
                 o_stride=self.heads * self.d + self.pad)
        a.update(kw)
        return hs.make_attn_shape(batch, self.heads, self.kv_heads, self.d, self.page, self.blocks,
                                  self.table.shape[1], **a)

    def row(self, r, k, v):
        """(o, lse, bound of |o - its float64 value|, bound for lse) of query row r over the keys."""
        h, hk, d, g = self.heads, self.kv_heads, self.d, self.group
        n = k.shape[0]
        if n == 0:
            z = torch.zeros(h, d, dtype=torch.float64)
            return z, torch.full((h,), -math.inf, dtype=torch.float64), z, torch.zeros(h)
        q = self.q[r, :h * d].double().reshape(hk, g, d)
        kd, vd = k.double(), v.double()
        s = torch.einsum("agd,nad->agn", q, kd) * self.scale
        lse = torch.logsumexp(s, dim=2)
        w = (s - lse[..., None]).exp()
        o = torch.einsum("agn,nad->agd", w, vd)
        # the error of a score: d products and the scaling, one step of float32 each, on the sum of
        # magnitudes; a weight is off by that, by its exponential and by the rescalings
        size = torch.einsum("agd,nad->agn", q.abs(), kd.abs()) * self.scale
        ds = ((d + 4) * 2.0 ** -23 * size).amax(dim=2) + 2.0 ** -20 * (1 + s.abs().amax(dim=2))
        u = torch.finfo(DT[self.dtype]).eps / 2
        tiny = torch.finfo(DT[self.dtype]).smallest_normal * u * 2       # half a step of a subnormal
        mag = torch.einsum("agn,nad->agd", w, vd.abs())
        total = n * 2.0 ** -23
        do = (u + 2 * ds[..., None] + 2 * total) * mag + u * o.abs()
        # fp16 weights below 2^-14 are rounded to steps of 2^-24, relative to a largest weight of 1
        do = do * (1 + 2 * u) + tiny * (1 + vd.abs().amax(dim=0)[:, None] * n)
        return (o.reshape(h, d), lse.reshape(h), do.reshape(h, d), (ds + total).reshape(h))

    def prefill_rows(self, pos0, n_tokens, cu):
        for b, (p, n) in enumerate(zip(pos0, n_tokens)):
            for t in range(n):
                yield (cu[b] + t, *self.row(cu[b] + t, self.K[b][:p + t + 1], self.V[b][:p + t + 1]))

    def decode_rows(self, kv_len):
        for b, n in enumerate(kv_len):
            k, v = (torch.cat((x, y[b][:n])) for x, y in ((self.kp, self.K), (self.vp, self.V)))
            yield (b, *self.row(b, k, v))


class Outputs:
    """NaN-filled o and lse on the device, one row more than the call has."""

    def __init__(self, p, dev):
        self.p = p
        self.o = torch.full(p.q.shape, math.nan, dtype=p.q.dtype, device=dev)
        self.lse = torch.full((p.rows + 1, p.heads), math.nan, device=dev)
        self.err = torch.zeros(1, dtype=torch.int32, device=dev)

    def check(self, rows, written=None):
        p = self.p
        torch.cuda.synchronize()
        assert self.err.item() == 0
        o, lse = self.o.cpu(), self.lse.cpu()
        seen = torch.zeros(p.rows + 1, dtype=torch.bool)
        for r, want, want_lse, bound, bound_lse in rows:
            seen[r] = True
            got = o[r, :p.heads * p.d].double().reshape(p.heads, p.d)
            off = (got - want).abs()
            assert (off <= bound).all(), (r, (off / bound.clamp(min=1e-30)).max().item())
            fine = want_lse > -math.inf
            off = (lse[r].double() - want_lse)[fine].abs()
            assert (off <= bound_lse[fine]).all(), (r, off.max().item())
            assert (lse[r][~fine] == -math.inf).all()
        assert torch.isnan(o[~seen]).all() and torch.isnan(lse[~seen]).all()
        assert torch.isnan(o[:, p.heads * p.d:]).all()


def workspace(n, dev):
    """Exactly n bytes of NaN, and guard bytes behind them."""
    x = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device=dev)
    return x


def guarded(x, n):
    return bool((x[n:] == 0xFF).all().item())


def cu_of(n):
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    return cu


def run_prefill(p, pos0, n_tokens, dev, cu=None, stream=None, **kw):
    cu = cu or cu_of(n_tokens)
    out = Outputs(p, dev)
    shape = p.shape(len(n_tokens), **kw)
    size = hs.hs_attn_prefill_workspace_bytes(shape, pos0, n_tokens)
    ws = workspace(size, dev)
    out.keep = (p.q.to(dev), p.cache.to(dev), p.table.to(dev), ws)
    q, cache, table, _ = out.keep
    hs.hs_attn_prefill(shape, q, cache, table, out.o, out.lse, pos0, n_tokens, cu, ws, size, out.err,
                       stream)
    torch.cuda.synchronize()
    assert guarded(ws, size)
    return out


def run_decode(p, kv_len, bound, dev, shared=True, **kw):
    out = Outputs(p, dev)
    batch = len(kv_len)
    shape = p.shape(batch, **kw)
    prefix = p.kp.shape[0]
    lens = torch.tensor(kv_len, dtype=torch.int32, device=dev)
    q, cache, table, pre = p.q.to(dev), p.cache.to(dev), p.table.to(dev), p.prefix_table.to(dev)
    if shared:
        size = hs.hs_attn_decode_shared_workspace_bytes(shape, prefix, bound)
        ws = workspace(size, dev)
        hs.hs_attn_decode_shared(shape, q, cache, pre if prefix else None, prefix, table, lens, bound,
                                 out.o, out.lse, ws, size, out.err)
    else:
        size = hs.hs_attn_decode_workspace_bytes(shape, bound)
        ws = workspace(size, dev)
        hs.hs_attn_decode(shape, q, cache, table, lens, bound, out.o, out.lse, ws, size, out.err)
    torch.cuda.synchronize()
    assert guarded(ws, size)
    out.keep = (q, cache, table, pre, lens, ws)
    return out
