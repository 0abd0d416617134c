"""The full-attention operators of the restore-and-resume library, as one pass each.

A hybrid stack has full-attention layers beside its linear ones.  Their keys and values live in
the paged cache that the restore calls fill; these operators write a layer's new tokens into it
and answer queries from it:

  append   the new tokens' K and V rows into their pages
  prefill  causal attention of the tails of a batch of prompts, packed, grouped heads:
               o_t = sum_{j <= p} softmax_j(scale q_t . k_j) v_j,   p = pos0 + t
  decode   the same for one token of each request over its own length
  shared   the decode step of requests whose prompts share a long cached prefix: each query
           attends to [prefix, own suffix], the prefix lying in the cache once

Sizes follow the repository's stacks: tiny (2 KV heads of 64, pages of 16), hybrid (16 heads over 4
KV heads of 128, pages of 16) and long-context (32 heads over 8 KV heads of 128, pages of 32).
"""
import math
import random

import torch

DEV = "cuda:0"

own = False


# ---- the cases ---------------------------------------------------------------------------


def _case(name, op, batch, heads, kv_heads, d, page, dtype="bf16", tokens=(1, 1), kv=(0, 0), grid=1,
          prefix=0, lse=False):
    """tokens: (lowest, highest) new tokens of a request; kv: of the keys before them (prefill), of
    all its keys (decode), of those behind the shared prefix (shared)."""
    return {"name": name, "op": op, "batch": batch, "heads": heads, "kv_heads": kv_heads, "d": d,
            "page": page, "dtype": dtype, "tokens_lo": tokens[0], "tokens_hi": tokens[1],
            "kv_lo": kv[0], "kv_hi": kv[1], "grid": grid, "prefix": prefix, "lse": lse, "lens": 1}


def listed():
    return [
        # one decode step of a serving batch: a token of each of 32 requests into its page
        _case("append_step", "append", 32, 16, 4, 128, 16, tokens=(1, 1), kv=(1, 8000)),
        # the recomputed tokens of four prompts of the long-context stack
        _case("append_prompts", "append", 4, 32, 8, 128, 32, tokens=(4096, 16384), kv=(0, 0)),
        # the tiny stack resumed at 192 of 256 tokens
        _case("prefill_tiny", "prefill", 1, 2, 2, 64, 16, tokens=(64, 64), kv=(192, 192), grid=64),
        # draft tokens to verify (or short suffixes after a full hit), ragged
        _case("prefill_drafts", "prefill", 8, 16, 4, 128, 16, tokens=(2, 8), kv=(200, 5000), lse=True),
        # the resumed 256-token tail of one hybrid-stack request of 4,608 tokens
        _case("prefill_tail", "prefill", 1, 16, 4, 128, 16, tokens=(256, 256), kv=(4352, 4352), grid=256),
        # one engine batch of nine requests' tails, unpadded
        _case("prefill_packed", "prefill", 9, 16, 4, 128, 16, "fp16", tokens=(65, 512), kv=(0, 4096),
              grid=256),
        # the largest: recomputation of two 16k-token prompts, one long-context layer
        _case("prefill_long", "prefill", 2, 32, 8, 128, 32, tokens=(16384, 16384), kv=(0, 0)),
        # one decode step of one request of the hybrid stack
        _case("decode_one", "decode", 1, 16, 4, 128, 16, kv=(4608, 4700)),
        # one decode step of a serving batch: 32 requests at different positions
        _case("decode_batch", "decode", 32, 16, 4, 128, 16, "fp16", kv=(1, 8000), lse=True),
        # one decode step of four requests far into their contexts
        _case("decode_long", "decode", 4, 32, 8, 128, 32, kv=(98304, 131072)),
        # eight answers to one prompt of the hybrid stack, a few tokens in
        _case("shared_samples", "shared", 8, 16, 4, 128, 16, kv=(1, 64), prefix=4608),
        # 64 requests behind one long document
        _case("shared_document", "shared", 64, 32, 8, 128, 32, kv=(1, 1024), prefix=32768, lse=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "prefill", "prefill", "prefill", "decode", "decode", "shared", "shared"])
    d = rng.choice([64, 128, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 4, 8, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
    page = rng.choice([16, 16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    kv, tokens, prefix, grid = (0, 0), (1, 1), 0, 1
    if op == "append":
        batch = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, max(1, 65536 // batch))
        tokens, kv = (max(1, hi // 4), hi), (0, _log_int(rng, 1, 8192))
    elif op == "prefill":
        batch = _log_int(rng, 1, 16)
        ahead = rng.choice([0, _log_int(rng, 1, 32768)])
        hi = _log_int(rng, 1, 16384)
        # no more work than two 16k-token prompts of 32 heads
        while batch * heads * hi * (ahead + hi // 2) > 8_000_000_000 or batch * (ahead + hi) > 200_000:
            batch, hi, ahead = max(1, batch // 2), max(1, hi // 2), ahead // 2
        tokens, kv = (max(1, hi // 8), hi), (ahead // 4, ahead)
        grid = rng.choice([1, 64])
    elif op == "decode":
        batch = _log_int(rng, 1, 128)
        hi = _log_int(rng, 1, max(1, min(131072, 524288 // batch)))
        kv = (rng.choice([0, 1, hi // 2]), hi)
    else:
        batch = _log_int(rng, 2, 128)
        prefix = _log_int(rng, 64, 65536)
        hi = _log_int(rng, 1, max(1, min(4096, 262144 // batch)))
        kv = (rng.choice([0, 1, hi // 2]), hi)
    case = _case("", op, batch, heads, kv_heads, d, page, dtype, tokens, kv, grid, prefix,
                 op != "append" and rng.random() < 0.4)
    del case["name"]
    case["lens"] = rng.randint(1, 1 << 20)
    return case


# ---- sizes -------------------------------------------------------------------------------


def _lens(case):
    """Of each request: its new tokens, and the keys before them (prefill, append), all its keys
    (decode), or those behind the prefix (shared)."""
    r = random.Random(case["lens"])
    g = case["grid"]
    n, kv = [], []
    for _ in range(case["batch"]):
        n.append(r.randint(case["tokens_lo"], case["tokens_hi"]))
        kv.append(r.randint(case["kv_lo"], case["kv_hi"]) // g * g)
    return n, kv


def _keys(case):
    """Keys of each request that lie in its own pages."""
    n, kv = _lens(case)
    return [a + b for a, b in zip(n, kv)] if case["op"] in ("append", "prefill") else kv


def work(case):
    n, kv = _lens(case)
    h, hk, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "append":
        return {"bytes": sum(n) * (2 * 2 * hk * d * 2 + 8), "flops": 0}
    # K and V of every key once (a shared prefix once for all), q in, o out, one lse a row
    rows = sum(n)
    size = (sum(_keys(case)) + case["prefix"]) * hk * d * 4 + rows * h * (4 * d + 4 * case["lse"])
    if case["op"] == "prefill":
        pairs = sum(t * p + t * (t + 1) // 2 for t, p in zip(n, kv))
    else:
        pairs = sum(kv) + rows * case["prefix"]
    return {"bytes": size, "flops": pairs * h * 4 * d}


# ---- one pass ----------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n, kv = _lens(case)
    keys = _keys(case)
    h, hk, d, P = case["heads"], case["kv_heads"], case["d"], case["page"]
    dt = torch.float16 if case["dtype"] == "fp16" else torch.bfloat16

    def normal(*shape):
        x = torch.empty(shape, dtype=dt, device=DEV)
        return x.normal_(generator=g)
    # every request's pages, somewhere in a cache that holds other requests' pages too
    pages = [-(-x // P) for x in keys]
    shared = -(-case["prefix"] // P)
    width = max(pages) if max(pages) else 1
    blocks = (sum(pages) + shared) * 5 // 4 + 8
    order = torch.randperm(blocks, device=DEV, generator=g).int()
    prefix_table, rest = order[:shared].contiguous(), order[shared:]
    count = torch.tensor(pages, device=DEV)
    listed_page = torch.arange(width, device=DEV) < count[:, None]
    table = torch.full((case["batch"], width), -1, dtype=torch.int32, device=DEV)
    table[listed_page] = rest[:sum(pages)]
    s = {"case": case, "n": n, "kv": kv, "table": table, "blocks": blocks,
         "prefix_table": prefix_table, "cache": normal(blocks, 2, P, hk, d)}
    rows = sum(n)
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    s["cu"] = cu
    if case["op"] == "append":
        s["k"], s["v"] = normal(rows, hk, d), normal(rows, hk, d)
        first = torch.tensor(cu[:-1], device=DEV)
        b = torch.repeat_interleave(torch.arange(case["batch"], device=DEV), torch.tensor(n, device=DEV))
        pos = torch.arange(rows, device=DEV) - first[b] + torch.tensor(kv, device=DEV)[b]
        s["slots"] = table[b, pos // P].long() * P + pos % P
        return s
    s["q"] = normal(rows, h, d)
    s["o"] = torch.zeros((rows, h, d), dtype=dt, device=DEV)
    s["lse"] = torch.zeros((rows, h), device=DEV) if case["lse"] else None
    # of each request: its first row, new tokens and keys, on the device
    s["first"] = torch.tensor(cu[:-1], device=DEV)
    s["n_dev"] = torch.tensor(n, device=DEV)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=DEV)
    return s


def _plan(s):
    """The shape and the workspace that a user's program keeps beside its cache."""
    import paper_2609_15030_gb300 as hs
    case = s["case"]
    shape = hs.make_attn_shape(case["batch"], case["heads"], case["kv_heads"], case["d"], case["page"],
                               s["blocks"], s["table"].shape[1],
                               hs.HS_FP16 if case["dtype"] == "fp16" else hs.HS_BF16)
    size, bound = 0, s["table"].shape[1] * case["page"]     # the most keys that the table can list
    if case["op"] == "prefill":
        size = hs.hs_attn_prefill_workspace_bytes(shape, s["kv"], s["n"])
    elif case["op"] == "decode":
        size = hs.hs_attn_decode_workspace_bytes(shape, bound)
    elif case["op"] == "shared":
        size = hs.hs_attn_decode_shared_workspace_bytes(shape, case["prefix"], bound)
    s["plan"] = (hs, shape, torch.empty(max(size, 16), dtype=torch.uint8, device=DEV), size, bound)
    return s["plan"]


def _answers(s):
    return {"o": s["o"], "lse": s["lse"]} if s["lse"] is not None else {"o": s["o"]}


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        hs, shape, ws, size, bound = s.get("plan") or _plan(s)
        if op == "append":
            hs.hs_kv_append(shape, s["k"], s["v"], 0, s["slots"], s["cu"][-1], s["cache"])
            return {"cache": s["cache"]}
        if op == "prefill":
            hs.hs_attn_prefill(shape, s["q"], s["cache"], s["table"], s["o"], s["lse"], s["kv"], s["n"],
                               s["cu"], ws, size)
        elif op == "decode":
            hs.hs_attn_decode(shape, s["q"], s["cache"], s["table"], s["kv_len"], bound, s["o"], s["lse"],
                              ws, size)
        else:
            hs.hs_attn_decode_shared(shape, s["q"], s["cache"], s["prefix_table"], case["prefix"],
                                     s["table"], s["kv_len"], bound, s["o"], s["lse"], ws, size)
        return _answers(s)
    if op == "append":
        P = case["page"]
        s["cache"][s["slots"] // P, 0, s["slots"] % P] = s["k"]
        s["cache"][s["slots"] // P, 1, s["slots"] % P] = s["v"]
        return {"cache": s["cache"]}
    if op == "prefill":
        return _plain(s, s["kv_len"] + s["n_dev"], s["kv_len"], max(s["n"]))
    return _plain(s, s["kv_len"], None, 1)


def _gathered(s, table, length):
    """K and V of the first `length` keys of each request, float32 [batch][kv head][key][d]."""
    x = s["cache"][table.clamp(min=0).long()].float()        # [batch][page][2][P][kv head][d]
    b, pages, _, P, hk, d = x.shape
    k, v = (x[:, :, i].reshape(b, pages * P, hk, d)[:, :length].transpose(1, 2) for i in (0, 1))
    return k, v


def _plain(s, kv_len, pos0, most):
    """Masked softmax attention of padded requests in float32, some query tokens at a time where the
    scores of all would not fit."""
    case = s["case"]
    B, h, hk, d = case["batch"], case["heads"], case["kv_heads"], case["d"]
    g = h // hk
    longest = max(_keys(case))
    k, v = _gathered(s, s["table"], longest)
    if case["prefix"]:
        kp, vp = _gathered(s, s["prefix_table"][None], case["prefix"])
    step = max(1, min(most, (1 << 31) // (B * h * max(1, longest + case["prefix"]))))
    for t0 in range(0, most, step):
        t = torch.arange(t0, min(most, t0 + step), device=DEV)
        inside = t[None] < s["n_dev"][:, None]                               # [batch][token]
        rows = (s["first"][:, None] + t)[inside]
        q = torch.zeros((B, len(t), h, d), device=DEV)
        q[inside] = s["q"][rows].float()
        q = q.reshape(B, len(t), hk, g, d).permute(0, 2, 1, 3, 4).reshape(B, hk, len(t) * g, d)
        keys = longest if pos0 is None else min(longest, case["kv_hi"] + t0 + len(t))
        j = torch.arange(keys, device=DEV)
        seen = (j < kv_len[:, None, None]).expand(B, len(t), keys)
        if pos0 is not None:
            seen = seen & (j <= (pos0[:, None] + t)[:, :, None])
        seen = seen[:, None, :, None].expand(B, 1, len(t), g, keys).reshape(B, 1, len(t) * g, keys)
        x = torch.matmul(q, k[:, :, :keys].transpose(2, 3)).mul_(1.0 / math.sqrt(d))
        x = x.masked_fill_(~seen, -math.inf)
        if case["prefix"]:      # one product for all requests: the prefix's keys are the same
            rows_of = q.transpose(0, 1).reshape(hk, B * len(t) * g, d)
            y = torch.matmul(rows_of, kp[0].transpose(1, 2)).mul_(1.0 / math.sqrt(d))
            y = y.reshape(hk, B, len(t) * g, case["prefix"]).transpose(0, 1)
            x = torch.cat((y, x), dim=3)
        top = x.amax(dim=3, keepdim=True) if x.shape[3] else x.new_full((*x.shape[:3], 1), -math.inf)
        top = top.masked_fill(top == -math.inf, 0.0)                         # rows that see no key
        x = x.sub_(top).exp_()
        total = x.sum(dim=3, keepdim=True)
        if case["prefix"]:
            y, x = x[..., :case["prefix"]], x[..., case["prefix"]:]
            y = y.transpose(0, 1).reshape(hk, B * len(t) * g, case["prefix"])
            o = torch.matmul(y, vp[0]).reshape(hk, B, len(t) * g, d).transpose(0, 1)
            o = o + torch.matmul(x, v[:, :, :keys])
        else:
            o = torch.matmul(x, v[:, :, :keys])
        o = o / total.masked_fill(total == 0, 1.0)

        def by_row(y):
            y = y.reshape(B, hk, len(t), g, -1).permute(0, 2, 1, 3, 4).reshape(B, len(t), h, -1)
            return y[inside]
        s["o"][rows] = by_row(o).to(s["o"].dtype)
        if s["lse"] is not None:
            s["lse"][rows] = by_row(top + total.log())[..., 0]
    return _answers(s)


# ---- what is right -----------------------------------------------------------------------


def exact(case, seed):
    """Request by request and KV head by KV head in float64, straight from the definition."""
    s = prepare(case, seed)
    if case["op"] == "append":          # copies: the cache's own values, moved
        P = case["page"]
        flat = s["cache"].double().transpose(1, 2).reshape(s["blocks"] * P, 2, case["kv_heads"], case["d"])
        flat[s["slots"]] = torch.stack((s["k"], s["v"]), dim=1).double()
        flat = flat.reshape(s["blocks"], P, 2, case["kv_heads"], case["d"])
        return {"cache": flat.transpose(1, 2).contiguous()}
    h, hk, d, P = case["heads"], case["kv_heads"], case["d"], case["page"]
    g = h // hk
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["o"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for b, (n, ahead, total) in enumerate(zip(s["n"], s["kv"], _keys(case))):
        pages = s["table"][b, :-(-total // P)].long()
        at = [(pages, total)]
        if case["prefix"]:
            at.insert(0, (s["prefix_table"].long(), case["prefix"]))
        if not sum(x for _, x in at):
            continue
        K, V = (torch.cat([s["cache"][p, i].reshape(-1, hk, d)[:x] for p, x in at]) for i in (0, 1))
        for head in range(hk):
            kd, vd = K[:, head].double(), V[:, head].double()
            for t0 in range(0, n, 2048):
                m = min(2048, n - t0)
                row = s["cu"][b] + t0
                q = s["q"][row:row + m, head * g:(head + 1) * g].double().reshape(m * g, d)
                end = ahead + t0 + m if case["op"] == "prefill" else len(kd)
                x = q @ kd[:end].T / math.sqrt(d)
                if case["op"] == "prefill":
                    last = ahead + t0 + torch.arange(m, device=DEV).repeat_interleave(g)
                    x.masked_fill_(torch.arange(end, device=DEV) > last[:, None], -math.inf)
                z = torch.logsumexp(x, dim=1)
                o[row:row + m, head * g:(head + 1) * g] = ((x - z[:, None]).exp() @ vd[:end]).reshape(m, g, d)
                lse[row:row + m, head * g:(head + 1) * g] = z.reshape(m, g)
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}
