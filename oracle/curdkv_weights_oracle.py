"""Oracle of the calls around accumulated attention weights and shared prefixes, in numpy float64 on the host, shared with
nothing on the GPU side.  Attention itself is curdkv_serving_oracle.attend."""
import numpy as np

from oracle.curdkv_serving_oracle import attend, window_mask


def push(raw, pos, total, new_raw, budget, num_sink, window, offered=None):
    """Which rows a head holds after new ones have come and those beyond the budget have left.

    raw, pos: of the rows held, by slot; new_raw: of the rows that join (those that found room), whose positions follow
    `total`; offered: tokens of the sequence this step, joined or not.  Returns (from, raw, pos): per slot the row it
    holds (its slot had nothing left: held rows first, then the new ones), its weight and its position."""
    raw = np.concatenate([np.asarray(raw, np.float32), np.asarray(new_raw, np.float32)])
    held, t = len(pos), len(new_raw)
    pos = np.concatenate([np.asarray(pos, np.int64), total + np.arange(t)])
    now = total + (t if offered is None else offered)
    forced = (pos < num_sink) | (pos >= now - window)
    with np.errstate(invalid="ignore"):
        key = np.where(raw > 0, raw, np.float32(0)).astype(np.float64)       # NaN and what is not above 0 rank as 0
    key = np.where(forced, np.inf, key)
    n, kept = held + t, min(budget, held + t)
    order = sorted(range(n), key=lambda j: (-key[j], j))
    keep = set(order[:kept])
    at = list(range(kept))
    holes = [j for j in range(kept) if j not in keep]
    movers = [j for j in range(kept, n) if j in keep]
    assert len(holes) == len(movers)
    for h, m in zip(holes, movers):
        at[h] = m
    return np.array(at, dtype=np.int64), raw[at], pos[at]


def cache_attention(q, k, v, pos, total, scale):
    """One KV head of a cache: q [group, t, d], rows k, v [held, d] at positions `pos`; returns (o [group, t, d], lse [group, t],
    weights [group, t, held])."""
    group, t, d = q.shape
    seen = np.asarray(pos)[None] <= (total - t + np.arange(t))[:, None] if t > 1 else np.ones((t, len(pos)), bool)
    out = [attend(q[g], k, v, seen, scale) for g in range(group)]
    return tuple(np.stack([x[i] for x in out]) for i in range(3))


def scores(q, k, scale, normalised=True, lse=None):
    """Weights that the rows k [n, d] of one KV head get from the queries q [group, t, d] at the last t positions, summed;
    normalised: over the number of query rows that see something.  With `lse` [group, t] those stand for the log sums."""
    group, t, d = q.shape
    n = k.shape[0]
    seen = window_mask(n, t, n + t, 0)
    total, alive = np.zeros(n), 0
    for g in range(group):
        if lse is None:
            w = attend(q[g], k, np.zeros((n, 1)), seen, scale)[2]
        else:
            s = np.where(seen, scale * (q[g] @ k.T), -np.inf)
            dead = np.isneginf(lse[g])
            w = np.where(dead[:, None], 0.0, np.exp(s - np.where(dead, 0.0, lse[g])[:, None]))
        total += w.sum(0)
        alive += int(seen.any(-1).sum())
    return total / alive if normalised and alive else total


def prefix_attention(q, k0, v0, k, v, scale):
    """q [t, d] behind the shared rows k0, v0 and n own rows, the last t of which are the queries' own."""
    n0, n, t = k0.shape[0], k.shape[0], q.shape[0]
    own = np.arange(n)[None] <= (n - t + np.arange(t))[:, None]
    seen = np.concatenate([np.ones((t, n0), bool), own], axis=1)
    return attend(q, np.concatenate([k0, k]), np.concatenate([v0, v]), seen, scale)
