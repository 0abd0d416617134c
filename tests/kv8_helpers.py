"""The 8-bit cache and rotary positions from their definitions, in float64 and integers."""
import math

import numpy as np
import torch

import paper_2609_15030_gb300 as hs

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
HSDT = {"bf16": hs.HS_BF16, "fp16": hs.HS_FP16}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}            # half a step, relative
TINY = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25}       # half a step of the subnormals
G = hs.HS_KV8_GROUP


def e4m3_values():
    """The values of the 256 bytes, float64 (NaN for 0x7f and 0xff)."""
    out = []
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        if b & 127 == 127:
            x = math.nan
        out.append(-x if b & 128 else x)
    return torch.tensor(out, dtype=torch.float64)


VALUES = e4m3_values()


def to_e4m3(x):
    """The bytes of the nearest values of |x| <= 448, ties to even; NaN: 0x7f (float64 in, int64 out)."""
    mag = x.abs().clamp(max=448.0)
    e = torch.frexp(mag).exponent.clamp(min=-5) - 1            # 2^e <= mag, -6 at least
    q = torch.round(torch.ldexp(mag, 3 - e)).long()            # 8 to 16, or less for subnormals
    b = torch.where(q >= 8, ((e + 7) << 3) + (q - 8), q)       # 16 carries into the exponent
    b = b + torch.signbit(x).long() * 128
    return torch.where(torch.isnan(x), torch.full_like(b, 127), b)


def need_of(top):
    """The smallest 2^e >= top / 448, e >= -126, of float64 magnitudes."""
    f = torch.frexp(top)
    e = f.exponent - 9 + (f.mantissa > 0.875).int()
    e = torch.where(top > 0, e, torch.full_like(e, -126)).clamp(min=-126)
    return torch.ldexp(torch.ones_like(top), e)


class Cache:
    """A cache on the CPU: bytes int64 [block][kv head][2][P][d], scales float64 [block][kv head][2][P / 16]."""

    def __init__(self, blocks, kv_heads, page, d):
        self.blocks, self.kv_heads, self.page, self.d = blocks, kv_heads, page, d
        self.bytes = torch.full((blocks, kv_heads, 2, page, d), 127)
        self.scales = torch.full((blocks, kv_heads, 2, page // G), math.nan, dtype=torch.float64)

    def size(self):
        n = self.kv_heads * 2
        return -(-(n * self.page * self.d + n * self.page // G * 4) // 128) * 128

    def image(self):
        """The blocks as the library has them, uint8 [block][bytes]; what pads them is 0xee."""
        out = torch.full((self.blocks, self.size()), 0xEE, dtype=torch.uint8)
        n = self.kv_heads * 2 * self.page * self.d
        out[:, :n] = self.bytes.reshape(self.blocks, -1).to(torch.uint8)
        s = self.scales.to(torch.float32).reshape(self.blocks, -1).contiguous().view(torch.uint8)
        out[:, n:n + s.shape[1]] = s
        return out

    def values(self):
        """float64 [block][kv head][2][P][d]"""
        return VALUES[self.bytes] * self.scales.repeat_interleave(G, dim=3)[..., None]

    def append(self, x, slots):
        """x float64 [row][2][kv head][d] (NaN for what is not finite); the rows of a group as one."""
        groups = {}
        for r, slot in enumerate(slots):
            if 0 <= slot < self.blocks * self.page:
                groups.setdefault(slot // G, []).append(r)
        for g, rows in groups.items():
            at = [slots[r] % G for r in rows]
            blk, part = g * G // self.page, g % (self.page // G)
            y = x[rows].permute(2, 1, 0, 3)                              # [kv head][2][row][d]
            need = need_of(y.abs().nan_to_num(0.0).amax(dim=(2, 3)))
            span = slice(part * G, part * G + G)
            if 0 not in at:
                old = self.scales[blk, :, :, part]
                new = torch.maximum(old, need)
                held = VALUES[self.bytes[blk, :, :, span]] * (old / new)[..., None, None]
                grown = (new > old)[..., None, None].expand(held.shape)
                self.bytes[blk, :, :, span] = torch.where(grown, to_e4m3(held), self.bytes[blk, :, :, span])
                need = new
            self.scales[blk, :, :, part] = need
            z = to_e4m3(y / need[..., None, None])
            for i, token in enumerate(at):
                self.bytes[blk, :, :, part * G + token] = z[:, :, i]


def shape_of(batch, heads, kv_heads, d, page, blocks, width, dtype, **kw):
    return hs.make_attn_shape(batch, heads, kv_heads, d, page, blocks, width, HSDT[dtype], **kw)


def angles(rope, pos):
    """cos and sin of every row's pairs, float64 [row][pair], and how far an angle may be off (radians)."""
    turn = np.longdouble("6.283185307179586476925286766559005768")
    n = rope.dims // 2
    theta = np.array(rope.theta[:n], dtype=np.longdouble)
    a = np.fmod(np.asarray(pos, dtype=np.longdouble)[:, None] * theta, turn).astype(np.float64)
    # theta in turns is rounded twice; its product's upper 32 bits become a float of a half turn
    off = np.abs(np.asarray(pos, dtype=np.float64)[:, None] * theta.astype(np.float64)) * 2.0 ** -52 + \
        math.pi * 2.0 ** -24 + 2.0 ** -29
    return torch.from_numpy(np.cos(a)), torch.from_numpy(np.sin(a)), torch.from_numpy(off)


def turned(rope, x, pos):
    """x float64 [row][head][d] turned, and a bound of the float32 result's error."""
    n, amp = rope.dims // 2, rope.amplitude
    c, s, off = (t[:, None] for t in angles(rope, pos))
    y = x[..., :rope.dims]
    a, b = (y[..., :n], y[..., n:]) if rope.layout == hs.HS_ROPE_HALF else (y[..., 0::2], y[..., 1::2])
    p, q = amp * (a * c - b * s), amp * (b * c + a * s)
    # the angle; sine and cosine to 2 units, times the amplitude; two products and their sum
    err = amp * (a.abs() + b.abs()) * (off + 2.0 ** -22 + 2.0 ** -24 + 3 * 2.0 ** -24) + 2.0 ** -140
    if rope.layout == hs.HS_ROPE_HALF:
        z, e = torch.cat((p, q), dim=2), torch.cat((err, err), dim=2)
    else:
        z, e = (torch.stack(t, dim=3).flatten(2) for t in ((p, q), (err, err)))
    return (torch.cat((z, x[..., rope.dims:]), dim=2),
            torch.cat((e, torch.zeros_like(x[..., rope.dims:])), dim=2))


def filled(seed, keys, kv_heads, page, d, extra=3, spread=4, width=None):
    """A cache with keys[b] tokens of each request in random pages, and its table.  Everything else is NaN: blocks of
    nobody, tokens behind the last, scales of groups without a token."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in keys]
    c = Cache(sum(need) + extra, kv_heads, page, d)
    order = torch.randperm(c.blocks, generator=g)
    table = torch.full((len(keys), width or max(need + [1])), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(keys):
        ids = order[at:at + need[b]]
        at += need[b]
        table[b, :need[b]] = ids.int()
        full = need[b] * page
        code = torch.randint(0, 127, (full, kv_heads, 2, d), generator=g)
        code = torch.where(code > 119, code - 60, code) + 128 * torch.randint(0, 2, code.shape, generator=g)
        code[n:] = 127
        scale = torch.exp2(torch.randint(-8 - spread, -8 + spread + 1, (full // G, kv_heads, 2), generator=g).double())
        scale[-(-n // G):] = math.nan
        c.bytes[ids] = code.reshape(need[b], page, kv_heads, 2, d).permute(0, 2, 3, 1, 4)
        c.scales[ids] = scale.reshape(need[b], page // G, kv_heads, 2).permute(0, 2, 3, 1)
    return c, table


def keys_of(c, table, b, n):
    """float64 K and V [kv head][token][d] of a request's first n tokens."""
    pages = table[b, :-(-n // c.page)].long()
    x = c.values()[pages] if n else c.values()[:0]
    x = x.permute(2, 1, 0, 3, 4).flatten(2, 3)[:, :, :n]
    return x[0], x[1]


def attended(q, k, v, scale, dtype):
    """q float64 [kv head][group][d] over k, v [kv head][token][d]: (o, lse, bound of o's error, of lse's)."""
    hk, g, d = q.shape
    n = k.shape[1]
    if n == 0:
        z = torch.zeros(hk, g, d, dtype=torch.float64)
        return z, torch.full((hk, g), -math.inf, dtype=torch.float64), z, torch.zeros(hk, g)
    s = torch.einsum("agd,and->agn", q, k) * scale
    lse = torch.logsumexp(s, dim=2)
    w = (s - lse[..., None]).exp()
    o = torch.einsum("agn,and->agd", w, v)
    # a score: d products summed in float32, two factors; q's smallest elements in binary16 (2^-39 of the largest)
    size = torch.einsum("agd,and->agn", q.abs(), k.abs()) * scale
    lost = q.abs().amax(dim=2)[..., None] * k.abs().sum(dim=2)[:, None] * scale * 2.0 ** -39
    ds = ((d + 6) * 2.0 ** -23 * size + lost).amax(dim=2) + 2.0 ** -20 * (1 + s.abs().amax(dim=2))
    total = n * 2.0 ** -23
    # a weight is one binary16 number (2^-11 of it), for fp16 two (2^-22 of it, and a step of the sum), or 2^-32 of the
    # largest off, times the largest scale (a value is at most 448 of its own, and 1 / l is at most the largest weight's share)
    weight = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -21
    mag = torch.einsum("agn,and->agd", w, v.abs())
    small = 2.0 ** -32 * n * 448.0 * v.abs().amax(dim=(1, 2))[:, None, None]
    do = (weight + 2 * ds[..., None] + 2 * total) * mag + U[dtype] * o.abs() * (1 + 2.0 ** -7) + small + TINY[dtype]
    return o, lse, do, ds + total
