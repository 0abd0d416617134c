"""Attention with scores far from zero, where a step of float32 is larger than the room that the softmax
weights have.

Queries and keys have one element that is not zero, so that scores are exact products, and different
ones lie 2^9 and more apart in units of log2: the softmax is the mean over the places of the largest.
"""
import math

import pytest
import torch

from tests.attn_helpers import DT, Problem, run_decode, run_prefill
from tests.gpu_helpers import device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return device()


class Far(Problem):
    """Keys +- size in one element, the largest and the smallest several times."""

    def __init__(self, size, seed, heads, kv_heads, d, page, dtype, keys, rows, prefix_len=0):
        super().__init__(seed, heads, kv_heads, d, page, dtype, keys, rows, prefix_len)
        g = torch.Generator().manual_seed(seed + 1)
        dt = DT[dtype]
        for x in [self.kp] + self.K:
            n = x.shape[0]
            x.zero_()
            x[..., 0] = ((torch.rand(n, kv_heads, generator=g) * 2 - 1) * size).to(dt)
            for part in range(0, n, 300):        # ties within a tile and between tiles
                at = torch.randint(part, min(n, part + 300), (4,), generator=g)
                x[at[:2], :, 0] = size
                x[at[2:], :, 0] = -size
        sign = torch.randint(0, 2, (rows, heads), generator=g) * 2 - 1
        q = torch.zeros(rows, heads, d)
        q[..., 0] = sign * (0.5 + torch.rand(rows, heads, generator=g) / 2) * size
        self.q[:rows, :heads * d] = q.reshape(rows, -1).to(dt)
        for b, x in enumerate([self.kp] + self.K):
            ids = self.prefix_table if b == 0 else self.table[b - 1, :-(-x.shape[0] // page)]
            flat = torch.full((ids.numel() * page, kv_heads, d), math.nan, dtype=dt)
            flat[:x.shape[0]] = x
            self.cache[ids.long(), 0] = flat.reshape(-1, page, kv_heads, d)

    def row(self, r, k, v):
        h, hk, d, g = self.heads, self.kv_heads, self.d, self.group
        q = self.q[r, :h * d].double().reshape(hk, g, d)
        s = torch.einsum("agd,nad->agn", q, k.double()) * self.scale
        lse = torch.logsumexp(s, dim=2)
        w = torch.softmax(s, dim=2)
        o = torch.einsum("agn,nad->agd", w, v.double())
        mag = torch.einsum("agn,nad->agd", w, v.double().abs())
        # half a step of the element type for the (equal) weights and for the output, some of float32
        u = torch.finfo(DT[self.dtype]).eps / 2
        bound = (u + 2.0 ** -20) * mag + u * (1 + u) * o.abs()
        # the scale's two roundings, the score's, the maximum's and the result's two, 2^-24 each
        return (o.reshape(h, d), lse.reshape(h), bound.reshape(h, d), (lse.abs() * 2.0 ** -21 + 2.0 ** -20).reshape(h))


SIZES = [("fp16", 4096.0), ("fp16", 5000.0), ("fp16", 8000.0), ("fp16", 12000.0), ("fp16", 30000.0),
         ("fp16", 60000.0), ("bf16", 4096.0), ("bf16", 3e4), ("bf16", 5e4), ("bf16", 1e5), ("bf16", 3e5),
         ("bf16", 5e7), ("bf16", 1e15)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,size", SIZES)
@pytest.mark.parametrize("unsplit", [False, True])
def test_prefill_of_scores_far_from_zero(dev, unsplit, dtype, size, d):
    for heads, kv_heads, pos0, n in ((2, 1, [1500], [60]), (4, 2, [0, 700], [300, 9])):
        p = Far(size, 41, heads, kv_heads, d, 16, dtype, [a + b for a, b in zip(pos0, n)], sum(n))
        cu = [0, n[0], sum(n)][:len(n) + 1]
        run_prefill(p, pos0, n, dev, unsplit=unsplit).check(p.prefill_rows(pos0, n, cu))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,size", SIZES)
def test_decode_of_scores_far_from_zero(dev, dtype, size, d):
    kv_len = [3000, 1, 0, 129]
    p = Far(size, 42, 8, 2, d, 32, dtype, kv_len, 4)
    run_decode(p, kv_len, 3000, dev, shared=False).check(p.decode_rows(kv_len))


@pytest.mark.parametrize("batch", [4, 40])      # one and two tiles of rows to an item of the prefix
@pytest.mark.parametrize("dtype,size", SIZES)
def test_decode_shared_of_scores_far_from_zero(dev, dtype, size, batch):
    kv_len = [(37 * b) % 300 for b in range(batch)]
    p = Far(size, 43, 8, 2, 128, 16, dtype, kv_len, batch, prefix_len=2000)
    run_decode(p, kv_len, max(kv_len), dev).check(p.decode_rows(kv_len))


def test_a_row_far_from_zero_leaves_its_neighbours_their_bits(dev):
    """Rows of a tile with and without such scores: each row's result is its own."""
    p = Problem(44, 4, 1, 128, 16, "fp16", [900], 60, sharp=100.0)
    clean = run_prefill(p, [840], [60], dev, unsplit=True)
    p.q[11, 128:256] *= 10000.0        # scores of some 10^6
    out = run_prefill(p, [840], [60], dev, unsplit=True)
    o, ref = (x.o[:60, :512].reshape(60, 4, 128).cpu().view(torch.int16) for x in (out, clean))
    keep = torch.ones(60, 4, dtype=torch.bool)
    keep[11, 1] = False
    assert torch.equal(o[keep], ref[keep])
    assert torch.equal(out.lse[:60].cpu()[keep], clean.lse[:60].cpu()[keep])
    assert torch.isfinite(out.o[11, 128:256].float()).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("call", ["prefill", "unsplit", "decode", "shared"])
def test_averages_of_the_largest_values_are_finite(dev, call, d):
    """Columns of 65504, of -65504 and of both: averages lie between them, and what the weights' rounding (2^-11)
    puts above rounds to the largest number, not to infinity.  Infinities in the values stay."""
    kv_len = [900, 333, 1, 260]
    p = Problem(45, 16, 2, d, 16, "fp16", kv_len, 60 if call in ("prefill", "unsplit") else 4,
                prefix_len=500 if call == "shared" else 0)
    p.scale = 1.0
    g = torch.Generator().manual_seed(46)
    q = torch.zeros(p.rows, 16, d)
    q[..., 0] = 0.5 + torch.rand(p.rows, 16, generator=g) / 2
    p.q[:p.rows, :16 * d] = q.reshape(p.rows, -1).half()
    sign = torch.ones(d)
    sign[1::3] = -1
    for b, (k, v) in enumerate(zip([p.kp] + p.K, [p.vp] + p.V)):
        # one key of 0, a later tile's of up to 6.5 (log2): a weight that is no power of two; the others below 2^-70
        k.zero_()
        k[..., 0] = -100
        k[10:11, :, 0], k[200:201, :, 0] = 0, 4.5
        v[:] = (65504.0 * sign).half()
        v[::2, :, 5::7] *= -1
        ids = p.prefix_table if b == 0 else p.table[b - 1, :-(-k.shape[0] // 16)]
        for plane, x in enumerate((k, v)):
            flat = torch.full((ids.numel() * 16, 2, d), math.nan, dtype=x.dtype)
            flat[:x.shape[0]] = x
            p.cache[ids.long(), plane] = flat.reshape(-1, 16, 2, d)
    if call in ("prefill", "unsplit"):
        pos0, n, cu = [858, 0, 0, 245], [42, 2, 1, 15], [0, 42, 44, 45, 60]
        out = run_prefill(p, pos0, n, dev, unsplit=call == "unsplit", scale=1.0)
        rows = list(p.prefill_rows(pos0, n, cu))
    else:
        out = run_decode(p, kv_len, 900, dev, shared=call == "shared", scale=1.0)
        rows = list(p.decode_rows(kv_len))
    assert torch.isfinite(out.o[:p.rows, :16 * d].float()).all()
    out.check(rows)
    p.cache[p.table[0, 2].long(), 1, 4, :, 9] = math.inf       # key 36 of the first request
    out = run_prefill(p, pos0, n, dev, scale=1.0) if call in ("prefill", "unsplit") else \
        run_decode(p, kv_len, 900, dev, shared=call == "shared", scale=1.0)
    o = out.o[0, :16 * d].reshape(16, d).float()
    assert not torch.isfinite(o[:, 9]).any() and torch.isfinite(o[:, :9]).all()
