"""Measured cases of the operators around accumulated attention weights and shared prefixes.

    scores  the weight that each cached row of a prompt receives, summed over the queries of its KV head (all tokens of the
            prompt, or the last few): what a selection may rank rows by
    step    one generation step over a cache of bounded size: new rows join it, the rows of least accumulated weight leave it
            (sinks and the most recent rows stay), and the new tokens attend over it and add their weights to the rows'
    prefix  attention of a decoding batch whose sequences share a long prefix

Plain forms are elementary torch operations; with ``own`` the same passes go through the package's public calls.
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
        # the smallest prompt of the repository, ranked by what its last 32 tokens look at: latency
        {"name": "scores_last32_cfg1", "op": "scores", "batch": 1, "heads": 8, "group": 4, "n": 1024, "t": 32, "lse": False, "ragged": False},
        # four long prompts, ranked by their last 64 tokens
        {"name": "scores_last64_32k", "op": "scores", "batch": 4, "heads": 8, "group": 4, "n": 32768, "t": 64, "lse": False, "ragged": False},
        # a padded batch of prompts of odd lengths, weights of all tokens
        {"name": "scores_ragged4", "op": "scores", "batch": 4, "heads": 8, "group": 4, "n": 2000, "t": 2000, "lse": False, "ragged": True},
        # a whole prompt of 8192 tokens behind its attention, which has left the log sums
        {"name": "scores_8k_lse", "op": "scores", "batch": 1, "heads": 8, "group": 4, "n": 8192, "t": 8192, "lse": True, "ragged": False},
        # one token of one sequence, 20 % of an 8192-token prompt held: latency
        {"name": "step_cfg2", "op": "step", "batch": 1, "heads": 8, "group": 4, "budget": 1702, "t": 1, "ragged": False},
        # a decoding batch of 16, some of whose sequences have not filled their budget yet
        {"name": "step_ragged16", "op": "step", "batch": 16, "heads": 8, "group": 4, "budget": 2048, "t": 1, "ragged": True},
        # 16 sequences in 8 layers at once
        {"name": "step_layers", "op": "step", "batch": 128, "heads": 8, "group": 4, "budget": 2048, "t": 1, "ragged": False},
        # blocks of accepted tokens join large caches, two query heads a KV head
        {"name": "step_long_block", "op": "step", "batch": 8, "heads": 8, "group": 2, "budget": 65536, "t": 4, "ragged": False},
        # four samples of one short prompt: latency
        {"name": "prefix_small", "op": "prefix", "prefixes": 1, "share": 4, "heads": 8, "group": 4, "n": 1024, "own": 32, "t": 1, "ragged": True},
        # 64 requests behind one long system prompt, own parts of different lengths
        {"name": "prefix_64x32k", "op": "prefix", "prefixes": 1, "share": 64, "heads": 8, "group": 4, "n": 32768, "own": 512, "t": 1, "ragged": True},
        # 8 samples of a prompt in 16 layers at once
        {"name": "prefix_layers", "op": "prefix", "prefixes": 16, "share": 8, "heads": 8, "group": 4, "n": 8192, "own": 200, "t": 1, "ragged": False},
        # the longest context, 16 sequences that verify four tokens each
        {"name": "prefix_long_block", "op": "prefix", "prefixes": 1, "share": 16, "heads": 8, "group": 4, "n": 131072, "own": 1000, "t": 4, "ragged": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["scores", "step", "prefix"])
    heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8])
    if op == "scores":
        n = _log(rng, 2, 32768)
        room = 32 * 8192 * 8192 // (heads * group * n)
        t = min(n, room, n if rng.random() < 0.5 else _log(rng, 1, 128))
        return {"op": op, "batch": _log(rng, 1, max(1, min(16, room // t))), "heads": heads, "group": group, "n": n, "t": t,
                "lse": rng.random() < 0.4, "ragged": rng.random() < 0.5}
    if op == "step":
        budget = _log(rng, 1, 65536)
        return {"op": op, "batch": _log(rng, 1, max(1, min(128, 64 * 65536 // (heads * budget)))), "heads": heads, "group": group,
                "budget": budget, "t": rng.choice([1, 1, 1, 2, 3, 5, 8]), "ragged": rng.random() < 0.5}
    n, t = _log(rng, 1, 131072), rng.choice([1, 1, 1, 2, 4])
    prefixes = _log(rng, 1, max(1, min(16, 8 * 131072 // (heads * n))))
    # the cost of the largest listed case bounds the query rows
    share = _log(rng, 1, max(1, min(64, 256 * 8 * 131072 // (prefixes * heads * group * t * n))))
    own_rows = _log(rng, 1, max(1, min(4096, 16 * 8 * 1000 * 4 // (prefixes * share * heads)))) - 1
    return {"op": op, "prefixes": prefixes, "share": share, "heads": heads, "group": group, "n": n, "own": own_rows, "t": t,
            "ragged": rng.random() < 0.5}


def _spread(count, lo, hi, ragged):
    """`count` lengths spread over lo .. hi by a fixed irrational step; all hi where not ragged."""
    if not ragged:
        return [hi] * count
    return [lo + int((hi - lo + 1) * math.modf(0.5 + 0.6180339887498949 * i)[0]) for i in range(count)]


def _lens(case):
    """Rows of each sequence of a prompt batch; rows held by each sequence of a cache; own rows behind a prefix."""
    if case["op"] == "scores":
        return _spread(case["batch"], max(1, case["n"] // 8), case["n"], case["ragged"])
    if case["op"] == "step":
        return _spread(case["batch"], max(1, case["budget"] // 2), case["budget"], case["ragged"])
    return _spread(case["prefixes"] * case["share"], case["own"] // 4, case["own"], case["ragged"])


def _prefix_lens(case):
    return _spread(case["prefixes"], max(1, case["n"] // 2), case["n"], case["ragged"] and case["prefixes"] > 1)


def _kept(case):
    """(sinks, most recent rows) that a cache of this budget always keeps."""
    return min(4, case["budget"] // 4), min(64, case["budget"] // 2)


def work(case):
    h, g, t = case["heads"], case["group"], case["t"]
    row = 2 * D                                     # bytes of a row of K, V, Q or O
    if case["op"] == "scores":
        rows = seen = queries = 0
        for n in _lens(case):
            q = min(t, n)
            rows, queries, seen = rows + n, queries + q, seen + q * n - q * (q - 1) // 2
        return {"bytes": h * (rows * (row + 4) + queries * g * (row + (4 if case["lse"] else 0))), "flops": 2 * D * h * g * seen}
    if case["op"] == "step":
        held = sum(min(x + t, case["budget"]) for x in _lens(case))
        new = case["batch"] * t
        # the rows once for attention, their weights read and written, their positions read; new rows read and written
        return {"bytes": h * (held * (2 * row + 12) + new * (4 * row + 2 * g * row)), "flops": 4 * D * h * g * t * held}
    own_rows, shared = sum(_lens(case)), sum(_prefix_lens(case))
    queries = case["prefixes"] * case["share"] * t * g
    return {"bytes": h * ((own_rows + shared) * 2 * row + queries * 2 * row),
            "flops": 4 * D * h * g * t * (shared * case["share"] + own_rows)}


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


def _queries(gen, *shape):
    return torch.randn(shape + (D,), generator=gen, device=DEV).to(torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    h, g, t = case["heads"], case["group"], case["t"]
    s = {"case": case, "lens": _ints(_lens(case))}
    if case["op"] == "scores":
        b, n = case["batch"], case["n"]
        s["K"], s["V"] = _cache_like(gen, (b, h, n, D))
        s["Q"] = _queries(gen, b, h * g, t)
        s["q_lens"] = _ints([min(t, x) for x in _lens(case)])
        if case["lse"]:                             # as the prompt's attention leaves them
            s["lse"] = _log_sums(s)
        s["scores"] = torch.zeros((b, h, n), dtype=torch.float32, device=DEV)
    elif case["op"] == "step":
        b, cap = case["batch"], case["budget"] + t
        s["K"], s["V"] = _cache_like(gen, (b, h, cap, D))
        s["K_new"], s["V_new"] = _cache_like(gen, (b, h, t, D))
        s["Q"] = _queries(gen, b, h * g, t)
        s["O"] = torch.zeros_like(s["Q"])
        # the cache has seen four times as many tokens as it holds: sinks, the most recent, and others between, in any order
        held, (sinks, recent) = s["lens"].view(b, 1, 1), _kept(case)
        slot = torch.arange(cap, device=DEV).expand(b, h, cap)
        gap = torch.rand((b, h, cap), generator=gen, device=DEV) * 4
        pos = torch.where(slot >= sinks, sinks + ((slot - sinks) * 4 + gap).long(), slot)
        pos = torch.where(slot >= held - recent, 4 * held - (held - slot), pos)
        order = torch.where(slot < held, torch.rand((b, h, cap), generator=gen, device=DEV), 2.0).argsort(-1)
        pos = torch.where(slot < held, pos.gather(-1, order), -1)
        raw = torch.exp(1.5 * torch.randn((b, h, cap), generator=gen, device=DEV))
        raw = torch.where(slot < held, raw, 0.0)
        # weights, positions, rows held and tokens seen lie in one buffer, so that a pass can begin from the same ones
        s["state0"] = torch.cat([raw.view(torch.int32).flatten(), pos.to(torch.int32).flatten(), s["lens"], 4 * s["lens"]])
        s["state"] = s["state0"].clone()
    else:
        p, b = case["prefixes"], case["prefixes"] * case["share"]
        s["K_prefix"], s["V_prefix"] = _cache_like(gen, (p, h, case["n"], D))
        s["K"], s["V"] = _cache_like(gen, (b, h, case["own"], D))
        s["Q"] = _queries(gen, b, h * g, t)
        s["O"] = torch.zeros_like(s["Q"])
        s["prefix_lens"] = _ints(_prefix_lens(case))
    return s


def _views(case, flat):
    """Weights, positions, counts and totals inside a step's buffer."""
    b, h, cap = case["batch"], case["heads"], case["budget"] + case["t"]
    m = b * h * cap
    return (flat[:m].view(torch.float32).view(b, h, cap), flat[m: 2 * m].view(b, h, cap), flat[2 * m: 2 * m + b],
            flat[2 * m + b: 2 * m + 2 * b])


# ---------------------------------------------------------------- plain forms

def _causal(s):
    """Keys [batch, 1, t, n] that each query token sees."""
    case = s["case"]
    first = (s["lens"] - s["q_lens"]).long().view(-1, 1, 1, 1)
    tok, key = torch.arange(case["t"], device=DEV)[:, None], torch.arange(case["n"], device=DEV)[None]
    return (key <= first + tok) & (tok < s["q_lens"].view(-1, 1, 1, 1))


def _logits(s):
    """Scaled products [batch, kv heads, group * t, n] of a prompt batch."""
    return s["Q"].float().unflatten(1, (-1, s["case"]["group"])).flatten(2, 3) @ s["K"].float().transpose(2, 3) * SCALE


def _log_sums(s):
    """Log sums of the exponentials of each query row of a prompt batch, -inf for rows that do not exist."""
    case = s["case"]
    x = _logits(s).view(case["batch"], -1, case["t"], case["n"]).masked_fill_(~_causal(s), -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    return torch.log(x.sub_(top).exp_().sum(-1)) + top[..., 0]


def _plain_scores(s):
    case = s["case"]
    b, h, g, t, n = (case[x] for x in ("batch", "heads", "group", "t", "n"))
    x = torch.where(_causal(s), _logits(s).view(b, h * g, t, n), -math.inf)
    if case["lse"]:
        ref = s["lse"][..., None]
        w = torch.exp(x - torch.where(ref > -math.inf, ref, 0.0))
    else:
        top = x.amax(-1, keepdim=True)
        w = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
        w = w / w.sum(-1, keepdim=True).clamp_min(1e-30)
    return w.sum(2).view(b, h, g, n).sum(2) / (s["q_lens"] * g)[:, None, None]


def _attend(q, k, v, seen):
    """exp(scale q k^T - top), its row sums and tops, and its product with v; a row that sees nothing gives zeros."""
    x = torch.where(seen, q @ k.transpose(-1, -2) * SCALE, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    return p, p.sum(-1, keepdim=True), top, p @ v


def _push(s):
    """New rows join, rows of least weight leave: the kept rows stay where they are, but for those behind the new count,
    which take the freed places in order.  Returns weights, positions, counts, totals; K and V are changed in place."""
    case = s["case"]
    b, h, t = case["batch"], case["heads"], case["t"]
    cap, (sinks, recent) = case["budget"] + t, _kept(case)
    raw, pos, held, total = _views(case, s["state0"])
    slot, held = torch.arange(cap, device=DEV).expand(b, h, cap), held.view(b, 1, 1).long()
    new = slot - held                                                  # number of the new row that slot would take
    fresh, total = (new >= 0) & (new < t), total.view(b, 1, 1)
    now_raw, now_pos = torch.where(fresh, 0.0, raw), torch.where(fresh, total + new, pos.long())
    forced = (now_pos < sinks) | (now_pos >= total + t - recent)
    key = torch.where(forced, math.inf, now_raw)
    key = torch.where(slot < held + t, key, -1.0)
    rank = key.sort(dim=-1, descending=True, stable=True).indices.argsort(-1)
    count = (held + t).clamp_max(case["budget"])
    keep = rank < count
    # the i-th kept row at or behind `count` takes the i-th place below it that was given up
    hole, mover = ~keep & (slot < count), keep & (slot >= count)
    holes = torch.where(hole, slot, cap).sort(-1).values[..., :t]
    movers = torch.where(mover, slot, cap).sort(-1).values[..., :t]
    live = movers < cap
    src = torch.where(live, movers, 0)
    # places: freed slots for moved rows, and the new rows that stay at their own slot
    own_slot = keep & fresh & (slot < count)
    first = torch.where(own_slot, slot, cap).sort(-1).values[..., :t]
    dst_all = torch.cat([torch.where(live, holes, cap), first], -1)    # [b, h, 2 t], cap where there is none
    src_all = torch.cat([torch.where(live, src, cap), first], -1)
    ok = dst_all < cap
    bi, hi, wi = ok.nonzero(as_tuple=True)
    to, frm = dst_all[bi, hi, wi], src_all[bi, hi, wi]
    number = frm - held.view(b)[bi]                                    # of the new row; rows that move are new ones here
    for x in ("K", "V"):
        s[x][bi, hi, to] = s[x + "_new"][bi, hi, number]
    out_raw, out_pos = raw.clone(), pos.clone()
    out_raw[bi, hi, to] = 0.0
    out_pos[bi, hi, to] = (total.view(b)[bi] + number).to(torch.int32)
    return out_raw, out_pos, count.view(b).to(torch.int32), (total.view(b) + t).to(torch.int32)


def _plain_step(s):
    case = s["case"]
    b, h, g, t = (case[x] for x in ("batch", "heads", "group", "t"))
    raw, pos, count, total = _push(s)
    at = (total - t)[:, None] + torch.arange(t, device=DEV).repeat(g)                  # position of each query row
    live = torch.arange(raw.shape[-1], device=DEV) < count[:, None]
    seen = live[:, None, None] & (pos[:, :, None] <= at[:, None, :, None])
    p, total_p, _, o = _attend(s["Q"].float().view(b, h, g * t, D), s["K"].float(), s["V"].float(), seen)
    total_p = total_p.clamp_min(1e-30)
    s["O"].copy_((o / total_p).view(b, h * g, t, D))
    return [s["O"], raw + (p / total_p).sum(2), pos, count, total, s["K"], s["V"]]


def _plain_prefix(s):
    case = s["case"]
    p, share, h, g, t = (case[x] for x in ("prefixes", "share", "heads", "group", "t"))
    q = s["Q"].float().view(p, share, h, g * t, D)
    seen = torch.arange(case["n"], device=DEV) < s["prefix_lens"].view(p, 1, 1, 1)
    _, total, top, o = _attend(q.transpose(1, 2).reshape(p, h, share * g * t, D), s["K_prefix"].float(), s["V_prefix"].float(), seen)
    o, total, top = (x.view(p, h, share, g * t, -1).transpose(1, 2) for x in (o, total, top))
    if case["own"] > 0:
        at = (s["lens"] - t).view(-1, 1, 1, 1) + torch.arange(t, device=DEV).repeat(g)[:, None]
        seen = torch.arange(case["own"], device=DEV) <= at
        k, v = (s[x].float().view(p, share, h, -1, D) for x in ("K", "V"))
        _, total1, top1, o1 = _attend(q, k, v, seen.view(p, share, 1, g * t, -1))
        most = torch.maximum(top, top1)
        f0, f1 = torch.exp(top - most), torch.exp(top1 - most)
        o, total = o * f0 + o1 * f1, total * f0 + total1 * f1
    s["O"].copy_((o / total).reshape(p * share, h * g, t, D))
    return s["O"]


# ---------------------------------------------------------------- the package's calls

def _handles(s):
    """What a program keeps beside its tensors: the cache object, descriptors and workspaces."""
    from paper_2509_15038_b200 import binding as cur

    case, x = s["case"], {"cur": cur}
    h, g, t = case["heads"], case["group"], case["t"]
    if case["op"] == "scores":
        x["desc"] = cur.make_desc(s["K"], s["V"], 1, q_heads=h * g, seqlens=s["lens"])
        x["ws"] = cur.attention_scores_workspace(x["desc"], t, device=DEV)
    elif case["op"] == "step":
        x["cache"] = cur.DeviceCache.of(s["K"], s["V"], *_views(case, s["state"]))
        x["ws_push"] = cur.cache_workspace(case["batch"], h, t, case["budget"] + t, case["budget"], device=DEV)
        x["ws"] = cur.cache_attention_workspace(x["cache"], h * g, t)
    else:
        x["desc_prefix"] = cur.make_desc(s["K_prefix"], s["V_prefix"], 1, seqlens=s["prefix_lens"])
        x["desc"] = cur.make_desc(s["K"], s["V"], 1, q_heads=h * g, seqlens=s["lens"])
        x["ws"] = cur.attention_prefix_workspace(x["desc_prefix"], x["desc"], t, device=DEV)
    return x


def _own(s):
    if "handles" not in s:
        s["handles"] = _handles(s)
    case, x = s["case"], s["handles"]
    cur = x["cur"]
    if case["op"] == "scores":
        return cur.curdkv_attention_scores(s["Q"], s["K"], x["desc"], scale=SCALE, q_lens=s["q_lens"], lse=s.get("lse"),
                                           lse_given=case["lse"], scores=s["scores"], workspace=x["ws"])[0]
    if case["op"] == "step":
        cache, (sinks, recent) = x["cache"], _kept(case)
        s["state"].copy_(s["state0"])
        cur.curdkv_cache_push(cache, s["K_new"], s["V_new"], case["budget"], x["ws_push"], num_sink=sinks, window=recent)
        cur.curdkv_cache_attention(s["Q"], cache, scale=SCALE, weights=cache.raw, O=s["O"], workspace=x["ws"])
        return [s["O"], cache.raw, cache.pos, cache.count, cache.total, s["K"], s["V"]]
    return cur.curdkv_attention_prefix(s["Q"], s["K_prefix"], s["V_prefix"], x["desc_prefix"], s["K"], s["V"], x["desc"],
                                       scale=SCALE, O=s["O"], workspace=x["ws"])[0]


def run(state):
    if own:
        return _own(state)
    return {"scores": _plain_scores, "step": _plain_step, "prefix": _plain_prefix}[state["case"]["op"]](state)


# ---------------------------------------------------------------- 64 bits

def _softmax64(q, k, seen):
    x = ((q.double() @ k.double().T) / math.sqrt(D)).masked_fill(~seen, -math.inf)
    return torch.exp(x - torch.logsumexp(x, -1, keepdim=True)).nan_to_num(0.0)


def _exact_scores(s):
    case = s["case"]
    g = case["group"]
    out = torch.zeros((case["batch"], case["heads"], case["n"]), dtype=torch.float64, device=DEV)
    for i, n in enumerate(_lens(case)):
        t = min(case["t"], n)
        seen = torch.ones((t, n), dtype=torch.bool, device=DEV).tril(n - t)
        for j in range(case["heads"]):
            for q in range(j * g, (j + 1) * g):
                if case["lse"]:
                    x = (s["Q"][i, q, :t].double() @ s["K"][i, j, :n].double().T) / math.sqrt(D)
                    w = torch.exp(x - s["lse"][i, q, :t, None].double()).masked_fill(~seen, 0.0)
                else:
                    w = _softmax64(s["Q"][i, q, :t], s["K"][i, j, :n], seen)
                out[i, j, :n] += w.sum(0)
            out[i, j] /= t * g
    return out


def _exact_step(s):
    case = s["case"]
    h, g, t, budget = (case[x] for x in ("heads", "group", "t", "budget"))
    sinks, recent = _kept(case)
    raw0, pos0, _, _ = _views(case, s["state0"])
    raw, pos = raw0.double(), pos0.clone()
    o = torch.zeros(s["O"].shape, dtype=torch.float64, device=DEV)
    counts, totals = [], []
    for i, held in enumerate(_lens(case)):
        n, seen_before = held + t, 4 * held
        kept, total = min(n, budget), 4 * held + t
        counts.append(kept)
        totals.append(total)
        for j in range(h):
            k, v = (torch.cat([s[x][i, j, :held], s[x + "_new"][i, j]]) for x in ("K", "V"))
            p = torch.cat([pos0[i, j, :held].long(), torch.arange(seen_before, total, device=DEV)])
            w = torch.cat([raw0[i, j, :held].double(), torch.zeros(t, dtype=torch.float64, device=DEV)])
            free = ((p >= sinks) & (p < total - recent)).nonzero()[:, 0]
            # leave: least weight first, of equal ones the highest slot
            leave = free.flip(0)[w[free.flip(0)].sort(dim=0, stable=True).indices[: n - kept]]
            alive = torch.ones(n, dtype=torch.bool, device=DEV)
            alive[leave] = False
            at = torch.arange(n, device=DEV)                        # which row each slot holds afterwards
            tail = alive[kept:].nonzero()[:, 0] + kept
            at[(~alive[:kept]).nonzero()[:, 0]] = tail
            at = at[:kept]
            raw[i, j, :kept], pos[i, j, :kept] = w[at], p[at].to(torch.int32)
            for q in range(g):
                m = _softmax64(s["Q"][i, j * g + q], k[at], p[at][None] <= torch.arange(seen_before, total, device=DEV)[:, None])
                o[i, j * g + q] = m @ v[at].double()
                raw[i, j, :kept] += m.sum(0)
    return [o, raw, pos, _ints(counts), _ints(totals), None, None]


def _exact_prefix(s):
    case = s["case"]
    g, t = case["group"], case["t"]
    o = torch.zeros(s["O"].shape, dtype=torch.float64, device=DEV)
    shared, lens = _prefix_lens(case), _lens(case)
    for i, n in enumerate(lens):
        i0 = i // case["share"]
        n0 = shared[i0]
        at = torch.arange(n - t, n, device=DEV)[:, None] + n0
        key = torch.arange(n0 + n, device=DEV)[None]
        seen = (key < n0) | (key <= at)
        for j in range(case["heads"]):
            k, v = (torch.cat([s[x + "_prefix"][i0, j, :n0], s[x][i, j, :n]]) for x in ("K", "V"))
            w = _softmax64(s["Q"][i, j * g: (j + 1) * g].flatten(0, 1), k, seen.repeat(g, 1))
            o[i, j * g: (j + 1) * g] = (w @ v.double()).view(g, t, D)
    return o


def exact(case, seed):
    s = prepare(case, seed)
    return {"scores": _exact_scores, "step": _exact_step, "prefix": _exact_prefix}[case["op"]](s)
