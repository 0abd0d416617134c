"""The 8-bit cache of the full-attention layers and the rotary positions in front of it, as one pass each.

A full-attention layer's keys are rotated by their positions, its cache may be held in 8 bits (E4M3 with
one power-of-two scale for each KV head and 16 tokens), and a decode step answers from that cache:

  rope     the rows of q and k turned by their positions: pair i of a head by the angle pos theta_i
  append   the new tokens' K and V rows quantised into their pages (a group of 16 tokens whose largest
           value grows takes a larger scale, and what it held is rounded to it); with "rope" the same
           call turns q and k on the way
  read     the first tokens of each request read back into the pages of a 16-bit cache, where a prefill
           finds them
  decode   one decode step: attention of one token of each request over its own length of 8-bit keys

Sizes follow the repository's stacks: hybrid (16 heads over 4 KV heads of 128, pages of 16), long-context
(32 heads over 8 KV heads of 128, pages of 32) and tiny (2 KV heads of 64, pages of 16).

A block of the cache: [kv head][2][token][head dim] E4M3, then [kv head][2][token / 16] float32 scales,
padded to a multiple of 128 bytes.
"""
import math
import random

import torch

DEV = "cuda:0"
GROUP = 16              # tokens that share a scale

own = False


# ---- the cases ---------------------------------------------------------------------------


def _case(name, op, batch, heads, kv_heads, d, page, dtype="bf16", tokens=(1, 1), kv=(0, 0), rot=0,
          layout="half", scaling="plain", factor=1.0, lse=False):
    """tokens: (lowest, highest) new tokens of a request; kv: of the tokens before them (rope, append),
    of all its tokens (read, decode).  rot: rotated dims of a head, 0: none."""
    return {"name": name, "op": op, "batch": batch, "heads": heads, "kv_heads": kv_heads, "d": d,
            "page": page, "dtype": dtype, "tokens_lo": tokens[0], "tokens_hi": tokens[1],
            "kv_lo": kv[0], "kv_hi": kv[1], "rot": rot, "layout": layout, "scaling": scaling,
            "factor": factor, "lse": lse, "lens": 1}


def listed():
    return [
        # q and k of one decode step of a serving batch
        _case("rope_step", "rope", 32, 16, 4, 128, 16, kv=(1, 8000), rot=128),
        # the recomputed tokens of four prompts of the long-context stack, far into their contexts
        _case("rope_prompts", "rope", 4, 32, 8, 128, 32, "fp16", tokens=(4096, 16384), kv=(0, 131072),
              rot=128, layout="interleaved", scaling="turns", factor=8.0),
        # one decode step of a serving batch: a token of each of 32 requests into its page
        _case("append_step", "append", 32, 16, 4, 128, 16, kv=(1, 8000)),
        # the same with positions, half of each head rotated: q, k and v in one call
        _case("append_rope_step", "append", 64, 32, 8, 128, 32, kv=(1, 32000), rot=64,
              scaling="linear", factor=4.0),
        # the tokens of four prompts of the long-context stack, rotated before
        _case("append_prompts", "append", 4, 32, 8, 128, 32, "fp16", tokens=(4096, 16384), kv=(0, 1000)),
        # the tails of nine requests of the hybrid stack, rotated and appended in one call
        _case("append_rope_tails", "append", 9, 16, 4, 128, 16, tokens=(65, 4096), kv=(0, 4096), rot=128,
              scaling="index", factor=4.0),
        # one hybrid-stack request's prefix of 4,608 tokens in front of a prefill
        _case("read_prefix", "read", 1, 16, 4, 128, 16, kv=(4608, 4608)),
        # the prefixes of four long-context requests (the largest)
        _case("read_long", "read", 4, 32, 8, 128, 32, kv=(98304, 131072)),
        # one decode step of one request of the hybrid stack
        _case("decode_one", "decode", 1, 16, 4, 128, 16, kv=(4608, 4700)),
        # one decode step of many short requests, heads of 64 in groups of 7
        _case("decode_short", "decode", 128, 14, 2, 64, 16, kv=(0, 300), lse=True),
        # one decode step of a serving batch: 32 requests at different positions
        _case("decode_batch", "decode", 32, 16, 4, 128, 16, "fp16", kv=(1, 8000), lse=True),
        # one decode step of four requests far into their contexts
        _case("decode_long", "decode", 4, 32, 8, 128, 32, kv=(98304, 131072)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "rope", "append", "append", "append", "read", "read", "decode", "decode",
                     "decode"])
    d = rng.choice([64, 128, 128, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 4, 8, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 12, 16])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    kv, tokens = (0, 0), (1, 1)
    if op in ("rope", "append"):
        batch = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, max(1, 40000 // batch))
        tokens, kv = (max(1, hi // 4), hi), (0, _log_int(rng, 1, 1000000 if op == "rope" else 8192))
    else:
        batch = _log_int(rng, 1, 128)
        hi = _log_int(rng, 1, max(1, min(131072, 400000 // batch)))
        kv = (rng.choice([0, 1, hi // 2]), hi)
    rot = 0
    if op == "rope" or (op == "append" and rng.random() < 0.6):
        rot = rng.choice([d, d, d, d // 2, d // 4, 3 * d // 4])
    case = _case("", op, batch, heads, kv_heads, d, page, dtype, tokens, kv, rot,
                 rng.choice(["half", "half", "interleaved"]),
                 rng.choice(["plain", "plain", "linear", "base", "turns", "index"]),
                 rng.choice([2.0, 4.0, 8.0, 32.0]), op == "decode" and rng.random() < 0.4)
    del case["name"]
    case["lens"] = rng.randint(1, 1 << 20)
    return case


# ---- sizes -------------------------------------------------------------------------------


def _lens(case):
    """Of each request: its new tokens, and the tokens before them (rope, append) or all (read, decode)."""
    r = random.Random(case["lens"])
    n, kv = [], []
    for _ in range(case["batch"]):
        n.append(r.randint(case["tokens_lo"], case["tokens_hi"]))
        kv.append(r.randint(case["kv_lo"], case["kv_hi"]))
    return n, kv


def _keys(case):
    """Tokens of each request that lie in its pages."""
    n, kv = _lens(case)
    return [a + b for a, b in zip(n, kv)] if case["op"] == "append" else kv


def _block_bytes(case):
    P, hk, d = case["page"], case["kv_heads"], case["d"]
    return -(-(hk * 2 * P * d + hk * 2 * (P // GROUP) * 4) // 128) * 128


def work(case):
    n, kv = _lens(case)
    h, hk, d, rows = case["heads"], case["kv_heads"], case["d"], sum(n)
    if case["op"] == "rope":
        return {"bytes": rows * ((h + hk) * d * 4 + 8), "flops": 6 * rows * (h + hk) * case["rot"] // 2}
    if case["op"] == "append":
        # K and V rows in, their bytes out, one scale a group; with positions q in and out
        groups = sum(-(-(a + b) // GROUP) - b // GROUP for a, b in zip(n, kv))
        size = rows * (2 * hk * d * 3 + 8) + groups * hk * 8
        if case["rot"]:
            size += rows * (h * d * 4 + 8)
        return {"bytes": size, "flops": 4 * rows * hk * d}
    groups = sum(-(-x // GROUP) for x in kv)
    size = sum(kv) * 2 * hk * d + groups * hk * 8
    if case["op"] == "read":
        return {"bytes": size + sum(kv) * 2 * hk * d * 2, "flops": sum(kv) * 2 * hk * d}
    return {"bytes": size + rows * h * (4 * d + 4 * case["lse"]), "flops": sum(kv) * h * 4 * d}


# ---- positions ---------------------------------------------------------------------------

BASE = 500000.0         # of the frequencies
CONTEXT = 8192          # tokens that the unscaled positions were made for
LOW, HIGH = 1.0, 32.0   # turns over CONTEXT: frequencies below LOW are divided by the factor, above HIGH kept


def _theta(case):
    """The angle of pair i for each position, float64, and the factor of the rotated values."""
    rot, kind, f = case["rot"], case["scaling"], case["factor"]
    i = torch.arange(rot // 2, dtype=torch.float64)
    base = BASE * f ** (rot / (rot - 2)) if kind == "base" else BASE
    theta = base ** (-2.0 * i / rot)
    if kind in ("plain", "base"):
        return theta, 1.0
    if kind == "linear":
        return theta / f, 1.0
    if kind == "turns":         # the kept share rises with the turns that a pair makes over CONTEXT
        keep = ((CONTEXT * theta / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        return theta / f * (1 - keep) + theta * keep, 1.0

    def place(turns):           # the index of the pair that makes so many turns
        return rot * math.log(CONTEXT / (turns * 2 * math.pi)) / (2 * math.log(base))
    lo, hi = max(math.floor(place(HIGH)), 0), min(math.ceil(place(LOW)), rot - 1)
    keep = 1.0 - ((i - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
    return theta / f * (1 - keep) + theta * keep, 0.1 * math.log(f) + 1.0


def _turned(case, x, cos, sin):
    """x: [row][head][d]; cos, sin: [row][1][rot / 2]."""
    rot = case["rot"]
    y = x[..., :rot]
    if case["layout"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        z = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=2)
    else:
        a, b = y[..., 0::2], y[..., 1::2]
        z = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=3).reshape(y.shape)
    return torch.cat((z, x[..., rot:]), dim=2)


# ---- one pass ----------------------------------------------------------------------------


def _views(case, cache):
    """The values [block][kv head][2][token][d] and scales [block][kv head][2][token / 16] of a cache."""
    P, hk, d = case["page"], case["kv_heads"], case["d"]
    size, groups = hk * 2 * P * d, P // GROUP
    values = cache[:, :size].view(torch.float8_e4m3fn).unflatten(1, (hk, 2, P, d))
    scales = cache[:, size:size + hk * 2 * groups * 4].view(torch.float32).unflatten(1, (hk, 2, groups))
    return values, scales


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n, kv = _lens(case)
    h, hk, d, P, rows = case["heads"], case["kv_heads"], case["d"], case["page"], sum(n)
    dt = torch.float16 if case["dtype"] == "fp16" else torch.bfloat16
    s = {"case": case, "n": n, "kv": kv}
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    first = torch.tensor(cu[:-1], device=DEV)
    b = torch.repeat_interleave(torch.arange(case["batch"], device=DEV), torch.tensor(n, device=DEV))
    pos = torch.arange(rows, device=DEV) - first[b] + torch.tensor(kv, device=DEV)[b]
    # a few wide channels in each head of the keys, and values whose size differs by head
    wide = torch.ones(hk, d, device=DEV)
    wide[torch.arange(hk, device=DEV)[:, None], torch.randint(d, (hk, 4), device=DEV, generator=g)] = 8.0
    loud = torch.exp2(torch.randn(hk, 1, device=DEV, generator=g))
    if case["op"] in ("rope", "append", "decode"):
        # the fused projection's output: [q | k | v] of each row
        qkv = torch.empty(rows, (h + 2 * hk) * d, dtype=dt, device=DEV).normal_(generator=g)
        s["qkv"] = qkv
        s["q"], s["k"], s["v"] = qkv[:, :h * d], qkv[:, h * d:(h + hk) * d], qkv[:, (h + hk) * d:]
        s["k"].mul_(wide.reshape(-1).to(dt))
        s["v"].mul_(loud.expand(hk, d).reshape(-1).to(dt))
    s["pos"] = pos
    if case["op"] == "rope":
        s["q_out"] = torch.zeros(rows, h * d, dtype=dt, device=DEV)
        s["k_out"] = torch.zeros(rows, hk * d, dtype=dt, device=DEV)
        return s
    # every request's pages, somewhere in a cache that holds other requests' pages too
    keys = _keys(case)
    pages = [-(-x // P) for x in keys]
    blocks = sum(pages) * 9 // 8 + 8
    width = max(max(pages), 1)

    def table():
        order = torch.randperm(blocks, device=DEV, generator=g).int()
        t = torch.full((case["batch"], width), -1, dtype=torch.int32, device=DEV)
        t[torch.arange(width, device=DEV) < torch.tensor(pages, device=DEV)[:, None]] = order[:sum(pages)]
        return t
    s["table"], s["blocks"] = table(), blocks
    s["cache"] = torch.zeros(blocks, _block_bytes(case), dtype=torch.uint8, device=DEV)
    values, scales = _views(case, s["cache"])
    for plane, size in ((0, wide), (1, loud)):
        for b0 in range(0, blocks, 4096):       # some blocks at a time: the cache is large
            x = torch.empty(min(4096, blocks - b0), hk, P, d, device=DEV).normal_(generator=g)
            x = (x * size[:, None]).unflatten(2, (P // GROUP, GROUP))
            top = torch.frexp(x.abs().amax(dim=(3, 4)) / 448.0)
            e = top.exponent - (top.mantissa == 0.5).int()
            scale = torch.ldexp(torch.ones_like(top.mantissa), e)
            values[b0:b0 + 4096, :, plane] = (x / scale[..., None, None]).flatten(2, 3).to(values.dtype)
            scales[b0:b0 + 4096, :, plane] = scale
    if case["op"] == "append":
        s["slots"] = s["table"][b, pos // P].long() * P + pos % P
        s["q_out"] = torch.zeros(rows, h * d, dtype=dt, device=DEV)
        return s
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=DEV)
    if case["op"] == "read":
        s["out_table"] = table()
        s["out"] = torch.zeros(blocks, 2, P, hk, d, dtype=dt, device=DEV)
        return s
    s["o"] = torch.zeros((rows, h, d), dtype=dt, device=DEV)
    s["lse"] = torch.zeros((rows, h), device=DEV) if case["lse"] else None
    return s


def _plan(s):
    """The shape, the frequencies and the workspace that a user's program keeps beside its cache."""
    import paper_2609_15030_gb300 as hs
    case = s["case"]
    h, hk, d = case["heads"], case["kv_heads"], case["d"]
    width = s["table"].shape[1] if "table" in s else 1
    shape = hs.make_attn_shape(case["batch"], h, hk, d, case["page"], s.get("blocks", 1), width,
                               hs.HS_FP16 if case["dtype"] == "fp16" else hs.HS_BF16,
                               q_stride=(h + 2 * hk) * d)
    rope = None
    if case["rot"]:
        layout = hs.HS_ROPE_HALF if case["layout"] == "half" else hs.HS_ROPE_INTERLEAVED
        kind = {"plain": hs.HS_ROPE_PLAIN, "linear": hs.HS_ROPE_LINEAR, "base": hs.HS_ROPE_BASE,
                "turns": hs.HS_ROPE_TURNS, "index": hs.HS_ROPE_INDEX}[case["scaling"]]
        amplitude = 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "index" else 1.0
        rope = hs.hs_rope_plan(case["rot"], layout, BASE, kind, case["factor"], CONTEXT, LOW, HIGH, amplitude)
    size, bound = 0, width * case["page"]       # the most tokens that the table can list
    if case["op"] == "decode":
        size = hs.hs_kv8_decode_workspace_bytes(shape, bound)
    s["plan"] = (hs, shape, rope, torch.empty(max(size, 16), dtype=torch.uint8, device=DEV), size, bound)
    return s["plan"]


def _answers(s):
    case = s["case"]
    if case["op"] == "rope":
        return {"q": s["q_out"], "k": s["k_out"]}
    if case["op"] == "append":
        values, scales = _views(case, s["cache"])
        out = {"values": values, "scales": scales}
        return {**out, "q": s["q_out"]} if case["rot"] else out
    if case["op"] == "read":
        return {"cache": s["out"]}
    return {"o": s["o"], "lse": s["lse"]} if s["lse"] is not None else {"o": s["o"]}


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        hs, shape, rope, ws, size, bound = s.get("plan") or _plan(s)
        rows, stride = s["pos"].shape[0], (case["heads"] + 2 * case["kv_heads"]) * case["d"]
        if op == "rope":
            hs.hs_rope_apply(shape, rope, s["q"], s["k"], stride, s["pos"], rows, s["q_out"], 0,
                             s["k_out"], 0)
        elif op == "append" and rope is not None:
            hs.hs_kv8_append_rope(shape, rope, s["q"], s["k"], s["v"], stride, s["pos"], s["slots"], rows,
                                  s["q_out"], 0, s["cache"])
        elif op == "append":
            hs.hs_kv8_append(shape, s["k"], s["v"], stride, s["slots"], rows, s["cache"])
        elif op == "read":
            hs.hs_kv8_read(shape, s["cache"], s["table"], s["kv_len"], bound, s["out"], s["blocks"],
                           s["out_table"])
        else:
            hs.hs_kv8_decode(shape, s["q"], s["cache"], s["table"], s["kv_len"], bound, s["o"], s["lse"],
                             ws, size)
        return _answers(s)
    if op == "rope":
        return _plain_rope(s)
    if op == "append":
        return _plain_append(s)
    if op == "read":
        return _plain_read(s)
    return _plain_decode(s)


def _angles(s):
    theta, amplitude = _theta(s["case"])
    angle = s["pos"].double()[:, None, None] * theta.to(DEV)
    return angle.cos() * amplitude, angle.sin() * amplitude


def _plain_rope(s):
    d, (cos, sin) = s["case"]["d"], (t.float() for t in _angles(s))
    for x, out in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
        out.copy_(_turned(s["case"], x.unflatten(1, (-1, d)).float(), cos, sin).flatten(1))
    return _answers(s)


def _plain_append(s):
    case = s["case"]
    hk, d, P = case["kv_heads"], case["d"], case["page"]
    k, v = s["k"].unflatten(1, (hk, d)).float(), s["v"].unflatten(1, (hk, d)).float()
    if case["rot"]:
        cos, sin = _angles(s)
        q = s["q"].unflatten(1, (-1, d)).float()
        s["q_out"].copy_(_turned(case, q, cos.float(), sin.float()).flatten(1))
        k, v = _turned(case, k.double(), cos, sin), v.double()      # the scale goes by a border
    x = torch.stack((k, v), dim=2)                                  # [row][kv head][2][d]
    values, scales = _views(case, s["cache"])
    # the groups that get rows, and each row's place among them
    ids, which = torch.unique(s["slots"] // GROUP, return_inverse=True)
    block, part = ids // (P // GROUP), ids % (P // GROUP)
    anew = torch.zeros(len(ids), device=DEV).index_reduce_(0, which, (s["slots"] % GROUP == 0).float(), "amax") > 0
    top = x.new_zeros(len(ids), hk, 2).index_reduce_(0, which, x.abs().amax(dim=3), "amax")
    # the smallest power of two that brings the largest value to 448 or less
    old, half = scales[block, :, :, part], torch.frexp(top)
    e = half.exponent - 9 + (half.mantissa > 0.875).int()
    need = torch.ldexp(torch.ones_like(old), e.clamp(min=-126)).masked_fill(top == 0, 2.0 ** -126)
    new = torch.where(anew[:, None, None], need, torch.maximum(old, need))
    # what a group held is rounded to its new scale
    token = part[:, None] * GROUP + torch.arange(GROUP, device=DEV)
    # bytes as integers: indexed writes know no 8-bit floats
    raw = values.view(torch.uint8)
    held = raw[block[:, None], :, :, token].view(torch.float8_e4m3fn).float()    # [group][16][kv head][2][d]
    shrunk = held * torch.where(anew[:, None, None], 1.0, old / new)[:, None, :, :, None]
    raw[block[:, None], :, :, token] = shrunk.to(torch.float8_e4m3fn).view(torch.uint8)
    scales[block, :, :, part] = new
    y = (x.float() / new[which][..., None]).to(torch.float8_e4m3fn)
    raw[s["slots"] // P, :, :, s["slots"] % P] = y.view(torch.uint8)
    return _answers(s)


def _gathered(s, length):
    """K and V of the first `length` tokens of each request, float32 [2][batch][kv head][token][d]."""
    values, scales = _views(s["case"], s["cache"])
    at = s["table"].clamp(min=0).long()
    x = values.view(torch.uint8)[at].view(torch.float8_e4m3fn).float()      # [batch][page][kv head][2][P][d]
    x = x.unflatten(4, (-1, GROUP)) * scales[at][..., None, None]
    x = x.flatten(4, 5).permute(3, 0, 2, 1, 4, 5)                           # [2][batch][kv head][page][P][d]
    return x.flatten(3, 4)[:, :, :, :length]


def _plain_read(s):
    P, kv = s["case"]["page"], s["kv_len"]
    width = s["table"].shape[1]
    x = _gathered(s, width * P).to(s["out"].dtype)
    seen = torch.arange(width * P, device=DEV) < kv[:, None]
    b, t = seen.nonzero(as_tuple=True)
    at = s["out_table"][b, t // P].long()
    s["out"][at, 0, t % P] = x[0][b, :, t]
    s["out"][at, 1, t % P] = x[1][b, :, t]
    return _answers(s)


def _plain_decode(s):
    case = s["case"]
    B, h, hk, d = case["batch"], case["heads"], case["kv_heads"], case["d"]
    longest = max(s["kv"])
    k, v = _gathered(s, longest)
    q = s["q"].float().reshape(B, hk, h // hk, d)
    x = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    unseen = torch.arange(longest, device=DEV) >= s["kv_len"][:, None, None, None]
    x = x.masked_fill(unseen, -math.inf)
    top = x.amax(dim=3, keepdim=True) if longest else x.new_full((*x.shape[:3], 1), -math.inf)
    top = top.masked_fill(top == -math.inf, 0.0)                            # rows that see no key
    x = (x - top).exp()
    total = x.sum(dim=3, keepdim=True)
    s["o"].copy_((torch.matmul(x, v) / total.masked_fill(total == 0, 1.0)).reshape(B, h, d))
    if s["lse"] is not None:
        s["lse"].copy_((top + total.log()).reshape(B, h))
    return _answers(s)


# ---- what is right -----------------------------------------------------------------------


def _spun(case, x, pos):
    """The rows of one request as complex numbers, turned: x float64 [token][head][d], pos its positions."""
    rot = case["rot"]
    if not rot:
        return x
    i = torch.arange(0, rot, 2, dtype=torch.float64, device=DEV)
    kind, f = case["scaling"], case["factor"]
    log_base = math.log(BASE) + (math.log(f) * rot / (rot - 2) if kind == "base" else 0.0)
    theta = torch.exp(-log_base * i / rot)
    amplitude = 1.0
    if kind == "linear":
        theta = theta / f
    elif kind == "turns":
        share = (theta * CONTEXT / math.tau - LOW) / (HIGH - LOW)
        share = torch.minimum(torch.maximum(share, torch.zeros_like(share)), torch.ones_like(share))
        theta = theta * (share + (1 - share) / f)
    elif kind == "index":
        def index_of(turns):
            return rot / 2 * math.log(CONTEXT / math.tau / turns) / log_base
        lo, hi = max(0, math.floor(index_of(HIGH))), min(rot - 1, math.ceil(index_of(LOW)))
        slow = torch.clamp((i / 2 - lo) / (hi - lo if hi > lo else 1e-3), 0, 1)
        theta = theta * (1 - slow + slow / f)
        amplitude = 1.0 + 0.1 * math.log(f)
    spin = torch.polar(torch.full_like(theta, amplitude).expand(len(pos), -1), pos.double()[:, None] * theta)
    if case["layout"] == "half":
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * spin[:, None]
        return torch.cat((z.real, z.imag, x[..., rot:]), dim=2)
    z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:2], rot // 2, 2).contiguous()) * spin[:, None]
    return torch.cat((torch.view_as_real(z).flatten(2), x[..., rot:]), dim=2)


def _to_e4m3(x):
    """The nearest value of 4 significant bits, down to steps of 2^-9, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    """Request by request in float64, straight from the definitions."""
    s = prepare(case, seed)
    h, hk, d, P = case["heads"], case["kv_heads"], case["d"], case["page"]
    row = [0]
    for x in s["n"]:
        row.append(row[-1] + x)
    if case["op"] == "rope" or case["op"] == "append" and case["rot"]:
        turned = {"q": torch.zeros(row[-1], h * d, dtype=torch.float64, device=DEV)}
        if case["op"] == "rope":
            turned["k"] = torch.zeros(row[-1], hk * d, dtype=torch.float64, device=DEV)
        for name, out in turned.items():
            for r0 in range(0, row[-1], 4096):
                x = s[name][r0:r0 + 4096].double()
                out[r0:r0 + 4096] = _spun(case, x.reshape(len(x), -1, d), s["pos"][r0:r0 + 4096]).flatten(1)
        if case["op"] == "rope":
            return turned
    values, scales = _views(case, s["cache"])
    if case["op"] == "append":
        values, scales = values.double(), scales.double()
        for b, (n, ahead) in enumerate(zip(s["n"], s["kv"])):
            r = slice(row[b], row[b] + n)
            k = _spun(case, s["k"][r].double().reshape(n, hk, d), s["pos"][r])
            new = torch.stack((k, s["v"][r].double().reshape(n, hk, d)), dim=1)        # [token][2][kv head][d]
            # the request's tokens from its first touched group on, the older ones as they are held
            begin = ahead // GROUP * GROUP
            pages = s["table"][b].long()
            at = torch.arange(begin, ahead, device=DEV)
            held = values[pages[at // P], :, :, at % P].transpose(1, 2)
            stop = -(-(ahead + n) // GROUP) * GROUP
            x = torch.zeros(stop - begin, 2, hk, d, dtype=torch.float64, device=DEV)
            x[ahead - begin:ahead - begin + n] = new
            x = x.reshape(-1, GROUP, 2, hk, d)
            top = x.abs().amax(dim=(1, 4))                                                # [group][2][kv head]
            scale = torch.exp2(torch.ceil(torch.log2(top / 448)))
            scale = torch.where(top <= 224 * scale, scale / 2, scale).clamp(min=2.0 ** -126)  # 448 itself needs 1
            group = begin // GROUP + torch.arange(len(x), device=DEV)
            page, part = pages[group // (P // GROUP)], group % (P // GROUP)
            if ahead > begin:       # the first group goes on: its scale never falls
                old = scales[page[0], :, :, part[0]].T
                scale[0] = torch.maximum(scale[0], old)
                held = _to_e4m3(held * (old / scale[0])[None, :, :, None])
                values[pages[at // P], :, :, at % P] = held.transpose(1, 2)
            # rows of the last group that the request does not have keep the bytes they held, though
            # a group that goes on was rounded to its scale as a whole
            if ahead > begin:
                rest = torch.arange(min(ahead + n, begin + GROUP), begin + GROUP, device=DEV)
                old_rest = values[page[:1], :, :, rest % P].transpose(1, 2)
                values[page[:1], :, :, rest % P] = _to_e4m3(old_rest * (old / scale[0])[None, :, :, None]).transpose(1, 2)
            y = _to_e4m3(x / scale[:, None, :, :, None]).reshape(-1, 2, hk, d)[ahead - begin:ahead - begin + n]
            at = torch.arange(ahead, ahead + n, device=DEV)
            values[pages[at // P], :, :, at % P] = y.transpose(1, 2)
            scales[page, :, :, part] = scale.transpose(1, 2)
        out = {"values": values, "scales": scales}
        return {**out, "q": turned["q"]} if case["rot"] else out
    if case["op"] == "read":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    else:
        o = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV)
        lse = torch.full(s["o"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for b, length in enumerate(s["kv"]):
        pages = s["table"][b, :-(-length // P)].long()
        for head in range(hk if length else 0):
            x = values[:, head].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double()   # [page][2][P][d]
            x *= scales[pages, head].double().repeat_interleave(GROUP, dim=2)[..., None]
            if case["op"] == "read":
                to, rest = s["out_table"][b, :len(pages)].long(), length % P or P
                out[to[:-1], :, :, head] = x[:-1]
                out[to[-1], :, :rest, head] = x[-1, :, :rest]
                continue
            k, v = x.transpose(0, 1).reshape(2, -1, d)[:, :length]
            g = h // hk
            q = s["q"][b].reshape(h, d)[head * g:(head + 1) * g].double()
            score = q @ k.T / math.sqrt(d)
            z = torch.logsumexp(score, dim=1)
            o[b, head * g:(head + 1) * g] = (score - z[:, None]).exp() @ v
            lse[b, head * g:(head + 1) * g] = z
    if case["op"] == "read":
        return {"cache": out}
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}
