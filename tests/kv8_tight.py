"""Bounds of a decode step's outputs that lost keys, lost parts and coarser weights do not meet (float64).

With s_j the scores, w_j the softmax weights (their sum is 1), v_j the values, and an error d_j of each weight relative to
itself, o = sum w_j v_j is off by at most  sum w_j |v_j| d_j + |o| sum w_j d_j  (the second from the weights' sum).
"""
import math

import torch

from tests.kv8_helpers import G, TINY, U


def one_element_rows(seed, n, heads, d, dt, pad=0, loud=1.0):
    """Queries with one element that is not 0: their scores are single products, so that nothing hides in sums.  A row of
    NaN behind the last."""
    g = torch.Generator().manual_seed(seed)
    x = torch.zeros(n + 1, heads, d)
    at = torch.randint(0, d, (n + 1, heads, 1), generator=g)
    x.scatter_(2, at, torch.randn(n + 1, heads, 1, generator=g) * loud)
    y = torch.full((n + 1, heads * d + pad), math.nan, dtype=dt)
    y[:n, :heads * d] = x[:n].flatten(1).to(dt)
    return y


def bounded(q, k, v, v_scale, scale, dtype):
    """q float64 [kv head][group][d] over k, v [kv head][token][d]; v_scale [kv head]: the largest scale of its values.
    (o, lse, bound of o's error, bound of lse's)."""
    n = k.shape[1]
    s = torch.einsum("agd,and->agn", q, k) * scale
    lse = torch.logsumexp(s, dim=2)
    w = (s - lse[..., None]).exp()
    o = torch.einsum("agn,and->agd", w, v)
    mag = torch.einsum("agn,and->agd", w, v.abs())
    # A score: as many products as q has elements, each of their float32 sums off by a step of 2^-23 of the magnitudes
    # (nothing where q has one), eight roundings of factors.  A weight: its exponential and those of two joins, 2^-22
    # each, the difference in front of it (at most 8 where the maximum lags, half a step of 2^-21; beyond that 2^-24 of it).
    some = (q != 0).sum(dim=2)[..., None]
    size = torch.einsum("agd,and->agn", q.abs(), k.abs()) * scale
    lost = q.abs().amax(dim=2)[..., None] * k.abs().sum(dim=2)[:, None] * scale * 2.0 ** -39 * (some > 1)
    off = (some + 8) * 2.0 ** -23 * size + lost + 2.0 ** -20 + 2.0 ** -23 * (s.amax(dim=2, keepdim=True) - s)
    do = torch.einsum("agn,and->agd", w * off, v.abs()) + o.abs() * (w * off).sum(dim=2, keepdim=True)
    # The weight in front of the product: two binary16 numbers, the second to half a step of 2^-24 where the row's largest
    # weight, at the largest scale, is 2^7 or more: 2^-32 of it.
    floor = 2.0 ** -32 * w.amax(dim=2) * v_scale[:, None] * 448.0 * n
    do = do + 2.0 ** -22 * mag + floor[..., None]
    # Sums of a tile's products are cut to float32 behind at most four passes, 2^-24 each of the running sum and of the
    # tile's magnitudes; a running sum is the difference of two of the sums from the first key on.  200 more for joins.
    tiles = -(-n // G)
    each = torch.zeros(*w.shape[:2], tiles * G, v.shape[2], dtype=torch.float64)
    each[:, :, :n] = w[..., None] * v[:, None]
    run = each.unflatten(2, (tiles, G)).sum(dim=3).cumsum(dim=2)
    zero = torch.zeros_like(o)
    span = torch.maximum(run.amax(dim=2), zero) - torch.minimum(run.amin(dim=2), zero)
    do = do + 2.0 ** -22 * mag + (tiles + 200) * 2.0 ** -22 * span
    # the weights' sum: a lane adds two of a tile's, 64 more for shuffles and joins; the output's factors and rounding
    total = (n / 8 + 64) * 2.0 ** -24
    do = do + (total + 2.0 ** -21) * o.abs() + U[dtype] * o.abs() * (1 + 2.0 ** -7) + TINY[dtype]
    dz = off.amax(dim=2) + total + 2.0 ** -21 * (1 + lse.abs() + s.abs().amax(dim=2))
    return o, lse, do, dz
