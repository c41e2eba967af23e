"""Measured cases of the serving operators: the 4-bit cache (store, append, attention) and the attention with a sliding
window and sinks.

Plain forms are elementary torch operations; with ``own`` the same passes go through the package's public calls.

The 4-bit cache holds each K and V row (128 channels, bf16) as 64 bytes of codes plus four (scale, zero) pairs in bf16,
one per group of 32 channels.  For a group with least value lo and greatest value hi:
    scale = bf16((hi - lo) / 15),  zero = lo,  code = rint((x - zero) / scale) in 0 .. 15 (0 where scale = 0),
and the row stands for scale * code + zero.  Inside the 64 bytes
    K: channel 32 g + 8 t + u sits in nibble u of 32-bit word  4 t + g   (t < 4, g < 4, u < 8),
    V: channel 32 g + 4 t + u sits in nibble u of 16-bit word  4 t + g   (t < 8, g < 4, u < 4).
"""
import math

import torch

own = False

DEV = "cuda"
D = 128
SCALE = 1.0 / math.sqrt(D)


# ---------------------------------------------------------------- cases

def listed():
    return [
        # the smallest selection of the repository: 128 of 1024 tokens, 8 heads
        {"name": "store_cfg1", "op": "store", "batch": 1, "heads": 8, "n": 1024, "keep": 128, "packed": False},
        # prompt compression of a 32-layer model, 20 % of 8192 tokens + window 64, layers folded into the batch
        {"name": "store_cfg2", "op": "store", "batch": 32, "heads": 8, "n": 8192, "keep": 1702, "packed": False},
        # one generated token joins the cache of one sequence: latency
        {"name": "append_token", "op": "append", "batch": 1, "heads": 8, "rows": 1, "held": 1702, "ragged": False},
        # blocks of accepted tokens of different lengths join a batch of 16
        {"name": "append_ragged16", "op": "append", "batch": 16, "heads": 8, "rows": 64, "held": 2048, "ragged": True},
        # one token against the smallest compressed cache, no query groups
        {"name": "attend_cfg1", "op": "attend", "batch": 1, "heads": 8, "q_rows": 1, "n": 128, "ragged": False, "packed": False},
        # one token of one sequence against its compressed prompt, four query heads a KV head
        {"name": "attend_cfg2", "op": "attend", "batch": 1, "heads": 8, "q_rows": 4, "n": 1702, "ragged": False, "packed": False},
        # a decoding batch of 16 sequences of different lengths, heads packed one behind the other
        {"name": "attend_ragged16", "op": "attend", "batch": 16, "heads": 8, "q_rows": 4, "n": 16384, "ragged": True, "packed": True},
        # the longest context, nothing evicted, 8 sequences
        {"name": "attend_long", "op": "attend", "batch": 8, "heads": 8, "q_rows": 4, "n": 131072, "ragged": False, "packed": False},
        # one token of one long sequence that keeps 4 sinks and the last 128 tokens: latency
        {"name": "window_token", "op": "window", "batch": 1, "heads": 8, "group": 4, "n": 131072, "t": 1, "sink": 4, "window": 128, "ragged": False},
        # one token of each of 16 sequences of different lengths, window 4096
        {"name": "window_token_ragged16", "op": "window", "batch": 16, "heads": 8, "group": 4, "n": 16384, "t": 1, "sink": 4, "window": 4096, "ragged": True},
        # a padded batch of prompts of odd lengths
        {"name": "window_prompt_ragged4", "op": "window", "batch": 4, "heads": 8, "group": 4, "n": 2000, "t": 2000, "sink": 4, "window": 512, "ragged": True},
        # a whole prompt of 8192 tokens
        {"name": "window_prompt_8k", "op": "window", "batch": 1, "heads": 8, "group": 4, "n": 8192, "t": 8192, "sink": 4, "window": 1024, "ragged": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["store", "append", "attend", "attend", "window", "window"])
    heads = rng.choice([1, 2, 4, 8])
    if op == "store":
        n = _log(rng, 64, 131072)
        batch = _log(rng, 1, max(1, min(32, 32 * 8 * 8192 // (heads * n))))
        return {"op": op, "batch": batch, "heads": heads, "n": n, "keep": min(_log(rng, 16, n), max(16, 435712 // (batch * heads))),
                "packed": rng.random() < 0.5}
    if op == "append":
        return {"op": op, "batch": _log(rng, 1, 32), "heads": heads, "rows": _log(rng, 1, 256), "held": _log(rng, 1, 8192) - 1,
                "ragged": rng.random() < 0.5}
    if op == "attend":
        n = _log(rng, 1, 131072)
        batch = _log(rng, 1, max(1, min(32, 64 * 131072 // (heads * n))))
        return {"op": op, "batch": batch, "heads": heads, "q_rows": rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]), "n": n,
                "ragged": rng.random() < 0.5, "packed": rng.random() < 0.5}
    group = rng.choice([1, 2, 3, 4, 8])
    n = _log(rng, 1, 131072)
    room = 32 * 8192 * 8192 // (heads * group * n)
    t = min(n, _log(rng, 1, 8192) if rng.random() < 0.6 else rng.randint(1, 4), room)
    batch = _log(rng, 1, max(1, min(16, room // t)))
    # the cost of the largest listed prompt bounds the window
    window = min(_log(rng, 1, n), max(1, 32 * 8192 * 1024 // (batch * heads * group * t)))
    return {"op": op, "batch": batch, "heads": heads, "group": group, "n": n, "t": t, "sink": rng.choice([0, 1, 4, 16, 100]),
            "window": window, "ragged": rng.random() < 0.5}


def _spread(count, lo, hi, ragged):
    """`count` lengths spread over lo .. hi by a fixed irrational step; all hi where not ragged."""
    if not ragged:
        return [hi] * count
    return [lo + int((hi - lo + 1) * math.modf(0.5 + 0.6180339887498949 * i)[0]) for i in range(count)]


def _counts(case):
    """Rows held by each (sequence, head): of a selection with per-head budgets, or of sequences of different lengths."""
    b, h = case["batch"], case["heads"]
    if case["op"] == "store":
        return _spread(b * h, max(1, case["keep"] // 2), case["keep"], case["packed"])
    if case["op"] == "append":
        return [case["held"]] * (b * h)
    lens = _spread(b, max(1, case["n"] // 8), case["n"], case["ragged"])
    return [x for x in lens for _ in range(h)]


def _lens(case):
    return _spread(case["batch"], max(1, case["n"] // 8), case["n"], case["ragged"])


def work(case):
    row = 64 + 16                                   # bytes of one 4-bit row of K or V
    if case["op"] == "store":                       # read, quantise and write the kept rows; read them back as bf16
        kept = sum(_counts(case))
        return {"bytes": kept * 2 * (256 + 2 * row + 256) + kept * 4, "flops": kept * 2 * D * 6}
    if case["op"] == "append":
        rows = sum(_spread(case["batch"], 1, case["rows"], case["ragged"])) * case["heads"]
        return {"bytes": rows * 2 * (256 + 2 * row + 256), "flops": rows * 2 * D * 6}
    if case["op"] == "attend":
        held, q = sum(_counts(case)), case["q_rows"]
        return {"bytes": held * 2 * row + case["batch"] * case["heads"] * q * 2 * 2 * D, "flops": 4 * D * held * q}
    seen, touched, rows, s, w = 0, 0, 0, case["sink"], case["window"]
    for n in _lens(case):
        t = min(case["t"], n)
        p = torch.arange(n - t, n, dtype=torch.int64)
        seen += int((torch.clamp(p + 1, max=w) + torch.clamp(p - w + 1, min=0, max=s)).sum())
        first = max(0, n - t - w + 1)
        touched += n - first + min(s, first)
        rows += t
    hq = case["heads"] * case["group"]
    return {"bytes": touched * case["heads"] * 2 * 2 * D + rows * hq * 2 * 2 * D, "flops": 4 * D * hq * seen}


# ---------------------------------------------------------------- inputs

def _cache_like(gen, shape):
    """K with four strong channels a head, V with log-normal row norms, as cached rows are."""
    k = torch.randn(shape, generator=gen, device=DEV)
    strong = torch.rand(shape[:2] + (1, D), generator=gen, device=DEV).argsort(-1) < 4
    k = torch.where(strong, 10.0 * k, k).to(torch.bfloat16)
    v = torch.randn(shape, generator=gen, device=DEV)
    v = v * torch.exp(0.5 * torch.randn(shape[:3] + (1,), generator=gen, device=DEV))
    return k, v.to(torch.bfloat16)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    b, h = case["batch"], case["heads"]
    s = {"case": case}
    if case["op"] == "store":
        n, keep = case["n"], case["keep"]
        s["K"], s["V"] = _cache_like(gen, (b, h, n, D))
        counts = _counts(case)
        order = torch.rand((b * h, n), generator=gen, device=DEV).argsort(-1)[:, :keep]
        alive = torch.arange(keep, device=DEV) < _ints(counts)[:, None]
        order = torch.where(alive, order, n).sort(-1).values
        offsets = [0]
        for c in counts:
            offsets.append(offsets[-1] + c)
        s["counts"], s["offsets"] = _ints(counts).view(b, h), _ints(offsets)
        s["idx"] = (order[alive] if case["packed"] else torch.where(alive, order, -1).view(b, h, keep)).to(torch.int32)
        rows = (offsets[-1],) if case["packed"] else (b, h, keep)
        s["K_out"], s["V_out"] = (torch.zeros(rows + (D,), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    elif case["op"] == "append":
        t, held = case["rows"], case["held"]
        s["K"], s["V"] = _cache_like(gen, (b, h, t, D))
        s["held"] = _ints([held] * (b * h))
        new = _spread(b, 1, t, case["ragged"])
        s["t_new"] = _ints(new)
        fresh = torch.arange(t, device=DEV) < s["t_new"][:, None, None]
        s["slots"] = torch.where(fresh, held + torch.arange(t, device=DEV), -1).expand(b, h, t).to(torch.int32).contiguous()
        s["capacity"] = held + t
        s["K_out"], s["V_out"] = (torch.zeros((b, h, t, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    elif case["op"] == "attend":
        counts, n = _counts(case), case["n"]
        offsets = [0]
        for c in counts:
            offsets.append(offsets[-1] + c)
        s["counts"], s["offsets"] = _ints(counts), _ints(offsets)
        rows = offsets[-1] if case["packed"] else b * h * n
        s["K_codes"], s["V_codes"] = (torch.randint(0, 256, (rows, 64), generator=gen, device=DEV, dtype=torch.uint8) for _ in range(2))
        # ranges of 32 channels of cached rows: about 4 standard deviations wide, now and then ten times that for K
        wide = 1.0 + 9.0 * (torch.rand((rows, 4), generator=gen, device=DEV) < 0.5)
        s["K_meta"] = _meta(gen, rows, wide)
        s["V_meta"] = _meta(gen, rows, torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device=DEV)))
        s["Q"] = torch.randn((b, h, case["q_rows"], D), generator=gen, device=DEV).to(torch.bfloat16)
        s["O"] = torch.zeros_like(s["Q"])
        if not case["packed"]:
            s["K_codes"], s["V_codes"] = (s[x].view(b, h, n, 64) for x in ("K_codes", "V_codes"))
            s["K_meta"], s["V_meta"] = (s[x].view(b, h, n, 4, 2) for x in ("K_meta", "V_meta"))
    else:
        n, t = case["n"], case["t"]
        s["K"], s["V"] = _cache_like(gen, (b, h, n, D))
        s["Q"] = torch.randn((b, h * case["group"], t, D), generator=gen, device=DEV).to(torch.bfloat16)
        lens = _lens(case)
        s["lens"], s["q_lens"] = _ints(lens), _ints([min(t, x) for x in lens])
        s["O"] = torch.zeros_like(s["Q"])
    return s


def _meta(gen, rows, wide):
    width = wide * (3.0 + 2.0 * torch.rand((rows, 4), generator=gen, device=DEV))
    lo = -width * (0.4 + 0.2 * torch.rand((rows, 4), generator=gen, device=DEV))
    return torch.stack([(width / 15).to(torch.bfloat16), lo.to(torch.bfloat16)], dim=-1).contiguous()


# ---------------------------------------------------------------- plain forms

def _round_trip(x):
    """What bf16 rows [..., 128] stand for once they are held in 4 bits.  The codes are formed in 64 bits: a value next to a
    border between two codes has to fall on the right side of it."""
    g = x.float().unflatten(-1, (4, 32))
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    scale = ((hi - lo) / 15).to(torch.bfloat16).float()
    code = torch.round((g.double() - lo.double()) / scale.double()).clamp(0, 15).float()
    code = torch.where(scale > 0, code, 0.0)
    return (scale * code + lo).flatten(-2).to(torch.bfloat16)


def _rows_of_codes(codes, meta, lanes):
    """fp32 rows [..., 128] of 4-bit rows: codes uint8 [..., 64], meta bf16 [..., 4, 2]; `lanes` = 4 for K, 8 for V."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).float()
    c = c.unflatten(-1, (lanes, 4, 32 // lanes)).transpose(-3, -2).flatten(-2)          # [..., group, channel of the group]
    m = meta.float()
    return (c * m[..., :1] + m[..., 1:]).flatten(-2)


def _softmax_rows(s, seen):
    """exp(s - max) over the last axis where `seen`, and its sums; a row that sees nothing gives zeros."""
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
    return p, p.sum(-1, keepdim=True).clamp_min(1e-30)


def _plain_store(s):
    case = s["case"]
    b, h, n, keep = case["batch"], case["heads"], case["n"], case["keep"]
    if case["packed"]:
        head = torch.repeat_interleave(torch.arange(b * h, device=DEV), s["counts"].view(-1).long(), output_size=s["idx"].numel())
        at = head * n + s["idx"].long()
        return [_round_trip(s[x].view(-1, D)[at]) for x in ("K", "V")]
    at = s["idx"].long()
    out = [_round_trip(torch.gather(s[x], 2, at.clamp_min(0)[..., None].expand(b, h, keep, D))) for x in ("K", "V")]
    return [torch.where((at >= 0)[..., None], o, 0.0) for o in out]


def _plain_append(s):
    b, h = s["case"]["batch"], s["case"]["heads"]
    out = [torch.where((s["slots"] >= 0)[..., None], _round_trip(s[x]), 0.0) for x in ("K", "V")]
    return out + [(s["held"].view(b, h) + s["t_new"][:, None]).view(-1).to(torch.int32)]


def _plain_attend(s):
    case = s["case"]
    k, v = _rows_of_codes(s["K_codes"], s["K_meta"], 4), _rows_of_codes(s["V_codes"], s["V_meta"], 8)
    b, h, n = case["batch"], case["heads"], case["n"]
    q = s["Q"].float().view(b * h, case["q_rows"], D)
    seen = torch.arange(n, device=DEV) < s["counts"][:, None]                           # [heads, n]
    if case["packed"]:
        at = (s["offsets"][:-1, None] + torch.arange(n, device=DEV)).clamp_max(k.shape[0] - 1)
        k, v = (torch.where(seen[..., None], x[at], 0.0) for x in (k, v))
    else:
        k, v = (torch.where(seen[..., None], x.view(b * h, n, D), 0.0) for x in (k, v))
    p, total = _softmax_rows(q @ k.transpose(1, 2) * SCALE, seen[:, None])
    return (p @ v / total).to(torch.bfloat16).view(b, h, case["q_rows"], D)


def _plain_window(s):
    case = s["case"]
    b, h, g, n, t = (case[x] for x in ("batch", "heads", "group", "n", "t"))
    q = s["Q"].float().view(b, h, g * t, D)
    i, j = torch.arange(t, device=DEV), torch.arange(n, device=DEV)
    pos = (s["lens"] - s["q_lens"])[:, None] + i                                        # [b, t]
    ahead = pos[..., None] - j                                                          # [b, t, n]
    seen = (ahead >= 0) & ((ahead < case["window"]) | (j < case["sink"]))
    live = (j < s["lens"][:, None])[:, None, :, None]
    k, v = (torch.where(live, s[x].float(), 0.0) for x in ("K", "V"))
    p, total = _softmax_rows((q @ k.transpose(2, 3) * SCALE).view(b, h, g, t, n), seen[:, None, None])
    o = (p.view(b, h, g * t, n) @ v).view(b, h, g, t, D) / total
    o = torch.where((i < s["q_lens"][:, None])[:, None, None, :, None], o, 0.0)
    return o.to(torch.bfloat16).view(b, h * g, t, D)


# ---------------------------------------------------------------- the package's calls

def _handles(s):
    """What a program keeps beside its tensors: the cache object, descriptors and workspaces."""
    from paper_2509_15038_b200 import binding as cur

    case, out = s["case"], {"cur": cur}
    b, h = case["batch"], case["heads"]
    if case["op"] == "store":
        if case["packed"]:
            out["cache"] = cur.QuantCache(b, h, int(s["idx"].numel()), row_start=s["offsets"], device=DEV)
        else:
            out["cache"] = cur.QuantCache(b, h, case["keep"], device=DEV)
        out["desc"] = cur.make_desc(s["K"], s["V"], 1)
    elif case["op"] == "append":
        out["cache"] = cur.QuantCache(b, h, s["capacity"], device=DEV)
    elif case["op"] == "attend":
        out["cache"] = cur.QuantCache.of(s["K_codes"], s["V_codes"], s["K_meta"], s["V_meta"], s["counts"], b, h,
                                         row_start=s["offsets"] if case["packed"] else None)
        out["ws"] = cur.qcache_attention_workspace(out["cache"], case["q_rows"])
    else:
        out["desc"] = cur.make_desc(s["K"], s["V"], 1, q_heads=h * case["group"], seqlens=s["lens"])
        out["ws"] = cur.attention_window_workspace(out["desc"], case["t"], device=DEV)
    return out


def _own(s):
    if "handles" not in s:
        s["handles"] = _handles(s)
    case, x = s["case"], s["handles"]
    cur = x["cur"]
    if case["op"] == "store":
        cur.curdkv_qcache_store(x["cache"], s["K"], s["V"], x["desc"], s["idx"], s["counts"], s["offsets"], packed=case["packed"])
        cur.curdkv_qcache_read(x["cache"], K_out=s["K_out"], V_out=s["V_out"])
        return [s["K_out"], s["V_out"]]
    if case["op"] == "append":
        x["cache"].count.copy_(s["held"])
        cur.curdkv_qcache_append(x["cache"], s["K"], s["V"], t_new=s["t_new"])
        cur.curdkv_qcache_read(x["cache"], s["slots"], K_out=s["K_out"], V_out=s["V_out"])
        return [s["K_out"], s["V_out"], x["cache"].count]
    if case["op"] == "attend":
        return cur.curdkv_qcache_attention(s["Q"], x["cache"], scale=SCALE, O=s["O"], workspace=x["ws"])[0]
    return cur.curdkv_attention_window(s["Q"], s["K"], s["V"], x["desc"], case["window"], num_sink=case["sink"], scale=SCALE,
                                       q_lens=s["q_lens"], O=s["O"], workspace=x["ws"])[0]


def run(state):
    if own:
        return _own(state)
    return {"store": _plain_store, "append": _plain_append, "attend": _plain_attend, "window": _plain_window}[state["case"]["op"]](state)


# ---------------------------------------------------------------- 64 bits

def _exact_quantised(x):
    """Float64 values of bf16 rows [rows, 128] held in 4 bits, group by group."""
    x = x.double()
    out = torch.empty_like(x)
    for g in range(4):
        part = x[:, 32 * g: 32 * g + 32]
        lo, hi = part.min(1, keepdim=True).values, part.max(1, keepdim=True).values
        scale = ((hi - lo) / 15.0).float().bfloat16().double()
        ratio = torch.where(scale > 0, (part - lo) / torch.where(scale > 0, scale, 1.0), 0.0)
        code = ratio.floor()
        rest = ratio - code
        code = code + ((rest > 0.5) | ((rest == 0.5) & (code % 2 == 1))).double()
        out[:, 32 * g: 32 * g + 32] = lo + scale * code.clamp(max=15.0)
    return out


def _exact_attention(q, k, v, seen):
    """softmax(q k^T / sqrt(128)) v of one head in float64; `seen` [rows, keys] or None."""
    s = (q @ k.T) / math.sqrt(D)
    if seen is not None:
        s = s.masked_fill(~seen, -math.inf)
    return torch.exp(s - torch.logsumexp(s, -1, keepdim=True)) @ v


def exact(case, seed):
    s = prepare(case, seed)
    b, h = case["batch"], case["heads"]
    if case["op"] == "store":
        out = []
        for x in ("K", "V"):
            o = torch.zeros(s["K_out"].shape, dtype=torch.float64, device=DEV)
            at = 0
            for p, c in enumerate(_counts(case)):
                if case["packed"]:
                    o[at: at + c] = _exact_quantised(s[x].view(b * h, -1, D)[p][s["idx"][at: at + c].long()])
                    at += c
                else:
                    o[p // h, p % h, :c] = _exact_quantised(s[x][p // h, p % h][s["idx"][p // h, p % h, :c].long()])
            out.append(o)
        return out
    if case["op"] == "append":
        new = _spread(b, 1, case["rows"], case["ragged"])
        out = []
        for x in ("K", "V"):
            o = torch.zeros(s["K_out"].shape, dtype=torch.float64, device=DEV)
            for i, t in enumerate(new):
                for j in range(h):
                    o[i, j, :t] = _exact_quantised(s[x][i, j, :t])
            out.append(o)
        return out + [_ints([case["held"] + t for t in new for _ in range(h)])]
    if case["op"] == "attend":
        c = torch.arange(D, device=DEV)
        k_at = 8 * (4 * (c % 32 // 8) + c // 32) + c % 8                                # nibble of channel c in a K row
        v_at = 4 * (4 * (c % 32 // 4) + c // 32) + c % 4                                # and in a V row
        o = torch.zeros(s["O"].shape, dtype=torch.float64, device=DEV)
        begin = 0
        for p, count in enumerate(_counts(case)):
            if not case["packed"]:
                begin = p * case["n"]
            rows = slice(begin, begin + count)
            kv = []
            for codes, meta, at in (("K_codes", "K_meta", k_at), ("V_codes", "V_meta", v_at)):
                byte = s[codes].view(-1, 64)[rows][:, at // 2].int()
                code = (byte >> (4 * (at % 2))) & 15
                m = s[meta].view(-1, 4, 2)[rows].double()[:, c // 32]
                kv.append(m[..., 0] * code.double() + m[..., 1])
            o[p // h, p % h] = _exact_attention(s["Q"][p // h, p % h].double(), kv[0], kv[1], None)
            begin += count
        return o
    o = torch.zeros(s["O"].shape, dtype=torch.float64, device=DEV)
    for i, n in enumerate(_lens(case)):
        t = min(case["t"], n)
        pos = torch.arange(n - t, n, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)[None]
        seen = (j <= pos) & ((j > pos - case["window"]) | (j < case["sink"]))
        for m in range(h * case["group"]):
            o[i, m, :t] = _exact_attention(s["Q"][i, m, :t].double(), s["K"][i, m // case["group"], :n].double(),
                                           s["V"][i, m // case["group"], :n].double(), seen)
    return o
