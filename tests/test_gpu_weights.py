"""Generation over a cache whose rows are ranked by the attention weights they receive (push, attention), on the GPU against
the float64 oracle.  Needs a B200."""
import numpy as np
import pytest
import torch

from oracle import curdkv_weights_oracle as orc
from paper_2509_15038_b200 import binding as cur
from paper_2509_15038_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = float(np.float32(128 ** -0.5))


def _rand(shape, seed, gain=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * gain).to(torch.bfloat16)


def _f64(t):
    return synth.u16_to_f64(synth.to_u16(t))


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _cache(B, H, cap, held, seed, d=128, weights=None):
    """A cache of rows at random positions (the last one is the latest token), in no order."""
    rng = np.random.default_rng(seed)
    c = cur.DeviceCache(B, H, cap, d)
    c.K.copy_(_rand(c.K.shape, seed))
    c.V.copy_(_rand(c.V.shape, seed + 1))
    raw = rng.exponential(size=(B, H, cap)).astype(np.float32) if weights is None else weights(rng, (B, H, cap))
    pos = np.full((B, H, cap), -1, np.int32)
    total = []
    for b in range(B):
        total.append(3 * held[b] + (1 if held[b] else 0))
        for h in range(H):
            if held[b]:
                p = rng.choice(total[b] - 1, held[b] - 1, replace=False)
                pos[b, h, : held[b]] = rng.permutation(np.append(p, total[b] - 1))
    c.raw.copy_(torch.from_numpy(raw))
    c.pos.copy_(torch.from_numpy(pos))
    c.count.copy_(_ints(held))
    c.total.copy_(_ints(total))
    return c


def _state(c):
    return {x: getattr(c, x).clone() for x in ("K", "V", "raw", "pos", "count", "total")}


def _check_push(c, old, K_new, V_new, new_raw, t_new, budget, sink, window):
    """Everything is copied or counted: equal bit for bit, slots behind the new count included where the cache is at most 8
    rows above its budget."""
    B, H, cap = old["raw"].shape
    for b in range(B):
        held, total = int(old["count"][b]), int(old["total"][b])
        offered = min(max(t_new[b], 0), K_new.shape[2])
        t = min(offered, cap - held)
        kept = min(held + t, budget)
        assert int(c.count[b]) == kept and int(c.total[b]) == total + offered
        for h in range(H):
            nr = new_raw[b, h, :t].cpu().numpy() if new_raw is not None else np.zeros(t, np.float32)
            at, raw, pos = orc.push(old["raw"][b, h, :held].cpu().numpy(), old["pos"][b, h, :held].cpu().numpy(), total, nr, budget,
                                    sink, window, offered)
            assert np.array_equal(c.pos[b, h, :kept].cpu().numpy(), pos), (b, h)
            assert np.array_equal(c.raw[b, h, :kept].cpu().numpy().view(np.int32), raw.view(np.int32))
            at = torch.from_numpy(at).to(DEV)
            for x, new in (("K", K_new), ("V", V_new)):
                want = torch.cat([old[x][b, h, :held], new[b, h, :t]])[at]
                assert torch.equal(getattr(c, x)[b, h, :kept], want)
            if cap - budget <= 8:
                for x in ("K", "V", "raw", "pos"):
                    bits = torch.int16 if x in "KV" else torch.int32
                    assert torch.equal(getattr(c, x)[b, h, kept:].view(bits), old[x][b, h, kept:].view(bits)), x


@pytest.mark.parametrize("H", [1, 3, 8, 9, 16])
@pytest.mark.parametrize("t,over", [(1, 1), (1, 0), (2, 3), (8, 8), (5, 2), (3, 40), (20, 40)])
def test_push(H, t, over):
    """Caches that are full, have room, are empty, or have none; rows dropped for want of slots; more rows over the budget than
    a handful."""
    budget, B = 100, 6
    cap = budget + over
    held = [cap, budget, budget - 1, 0, 37, max(0, cap - t)]
    for sink, window in ((4, 16), (0, 0), (0, 100), (60, 40)):
        c = _cache(B, H, cap, held, 7 * t + over)
        old = _state(c)
        K_new, V_new = (_rand((B, H, t, 128), 90 + i) for i in range(2))
        new_raw = torch.rand((B, H, t), device=DEV) if sink else None
        t_new = [t, t, t, t - 1, 0, t]
        ws = cur.cache_workspace(B, H, t, cap, budget)
        cur.curdkv_cache_push(c, K_new, V_new, budget, ws, num_sink=sink, window=window, scores_new=new_raw, t_new=_ints(t_new))
        dropped = any(min(max(x, 0), t) > cap - n for x, n in zip(t_new, held))
        assert cur.curdkv_device_status(ws) == (cur.DEV_CACHE_FULL if dropped else 0)
        _check_push(c, old, K_new, V_new, new_raw, t_new, budget, sink, window)


@pytest.mark.parametrize("budget,t", [(1, 1), (7, 8), (255, 1), (4089, 7), (5000, 3), (70001, 2)])
def test_push_sizes(budget, t):
    c = _cache(2, 2, budget + t, [budget, max(1, budget // 2)], budget)
    old = _state(c)
    K_new, V_new = (_rand((2, 2, t, 128), 5 + i) for i in range(2))
    ws = cur.cache_workspace(2, 2, t, budget + t, budget)
    sink, window = min(4, budget // 3), min(64, budget // 3)
    cur.curdkv_cache_push(c, K_new, V_new, budget, ws, num_sink=sink, window=window)
    assert cur.curdkv_device_status(ws) == 0
    _check_push(c, old, K_new, V_new, None, [t, t], budget, sink, window)


def test_push_equal_and_odd_weights():
    """Many equal weights, zeros, negative ones, NaN and infinities: the rule of the selection (not above 0 ranks as 0, of equal
    ones the lower slot stays)."""
    def odd(rng, shape):
        return rng.choice(np.array([0.0, -1.0, np.nan, 0.5, 0.5, 2.0, np.inf, 1e-42], np.float32), shape)
    for t in (1, 6):
        for window in (0, 20):
            c = _cache(3, 4, 64 + t, [64, 64 + t, 30], 11 + t, weights=odd)
            old = _state(c)
            K_new, V_new = (_rand((3, 4, t, 128), 15 + i) for i in range(2))
            new_raw = torch.from_numpy(odd(np.random.default_rng(3), (3, 4, t))).to(DEV)
            ws = cur.cache_workspace(3, 4, t, 64 + t, 64)
            cur.curdkv_cache_push(c, K_new, V_new, 64, ws, num_sink=3, window=window, scores_new=new_raw)
            _check_push(c, old, K_new, V_new, new_raw, [t] * 3, 64, 3, window)


def test_push_other_channels_and_strides():
    for d in (8, 64, 256):
        c = _cache(2, 2, 33, [32, 32], 60, d=d)
        old = _state(c)
        K_new = _rand((2, 1, 2, d), 61).transpose(1, 2)                      # tokens before heads
        V_new = _rand((2, 2, 3, d), 62)[:, :, 1:2]
        ws = cur.cache_workspace(2, 2, 1, 33, 32)
        cur.curdkv_cache_push(c, K_new, V_new, 32, ws, num_sink=1, window=2)
        _check_push(c, old, K_new, V_new, None, [1, 1], 32, 1, 2)


def test_push_is_append_and_compression():
    """The same cache as the older calls leave, whose scores come from G."""
    B, H, budget, t = 3, 8, 200, 4
    G = torch.randn((128, 32), device=DEV) / 32 ** 0.5
    a, b = _cache(B, H, budget + t, [budget, 150, 198], 70), _cache(B, H, budget + t, [budget, 150, 198], 70)
    K_new, V_new = (_rand((B, H, t, 128), 71 + i) for i in range(2))
    ws = cur.cache_workspace(B, H, t, budget + t, budget)
    desc = cur.make_desc(K_new, V_new, 32, raw_scores=1)
    scores = cur.curdkv_score(K_new, V_new, G, desc, cur.alloc_workspace(desc))[0]
    cur.curdkv_cache_step(a, K_new, V_new, G, budget, ws, num_sink=4, window=32)
    cur.curdkv_cache_push(b, K_new, V_new, budget, ws, num_sink=4, window=32, scores_new=scores)
    for x in ("count", "total"):
        assert torch.equal(getattr(a, x), getattr(b, x))
    for i, n in enumerate(a.count.tolist()):
        for x in ("K", "V", "raw", "pos"):
            assert torch.equal(getattr(a, x)[i, :, :n], getattr(b, x)[i, :, :n])


def _check_attention(O, lse, w, w0, c, Q, q_lens, scale, before, what=""):
    """Error budget.  O: weights rounded to bf16 (2^-8 of each), logits with fp32 sums of 128 exact products (2^-20 of the
    sum of magnitudes, in numerator and denominator) and their scaling (2^-23 of the logit), 2^-18 for exponentials and fp32
    sums, O rounded once (2^-8).  A weight of a row: twice the logits' error and 2^-18 of it, and its additions in
    fp32, 2^-24 of the result each."""
    got, Qf, Kf, Vf = _f64(O), _f64(Q), _f64(c.K), _f64(c.V)
    B, Hq, t = Q.shape[:3]
    H = c.kv_heads
    group = Hq // H
    for b in range(B):
        n, tb, total = int(c.count[b]), min(max(q_lens[b], 0), t), int(c.total[b])
        for h in range(H):
            pos = c.pos[b, h, :n].cpu().numpy() if t > 1 else np.zeros(n, np.int64)
            q, k, v = Qf[b, h * group: (h + 1) * group, :tb], Kf[b, h, :n], Vf[b, h, :n]
            want, want_lse, wt = orc.cache_attention(q, k, v, pos, total if t > 1 else 1, scale)
            d = (2.0 ** -20 + 2.0 ** -23) * scale * (np.abs(q) @ np.abs(k).T).max(-1, initial=0.0)             # [group, tb]
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * d + 2.0 ** -18)[..., None] * (wt @ np.abs(v)) * (1 + 2.0 ** -7) + 1e-38
            err = np.abs(got[b, h * group: (h + 1) * group, :tb] - want)
            assert np.all(err <= tol), f"{what} b={b} h={h}: {np.nanmax(err / tol):.3g} of the tolerance"
            assert np.array_equal(got[b, h * group: (h + 1) * group, tb:], before[b, h * group: (h + 1) * group, tb:])
            if lse is not None:
                g = lse[b, h * group: (h + 1) * group, :tb].cpu().numpy()
                dead = np.isneginf(want_lse)
                assert np.all(np.isneginf(g[dead])) and not got[b, h * group: (h + 1) * group, :tb][dead].any()
                ok = np.abs(g - np.where(dead, 0, want_lse)) <= d + 2.0 ** -20 * (1 + np.abs(np.where(dead, 0, want_lse))) + 2.0 ** -18
                assert np.all(ok | dead)
            if w is not None:
                w0h, wh = (x[b, h].cpu().numpy().astype(np.float64) for x in (w0, w))
                assert np.array_equal(wh[n:], w0h[n:])
                add = wt.sum((0, 1)) if n else np.zeros(0)
                tol = ((2 * d + 2.0 ** -18)[..., None] * wt).sum((0, 1)) + 2.0 ** -24 * (group * tb + 1) * (np.abs(w0h[:n]) + add) + 1e-37
                assert np.all(np.abs(wh[:n] - (w0h[:n] + add)) <= tol), f"{what} b={b} h={h}: weights"


def _attend(B, H, group, t, cap, held, q_lens=None, scale=SCALE, seed=0, c=None, Q=None, what=""):
    c = _cache(B, H, cap, held, seed) if c is None else c
    Q = _rand((B, H * group, t, 128), seed + 5) if Q is None else Q
    O = _rand(Q.shape, seed + 6)
    before, w0 = _f64(O), c.raw.clone()
    lse = torch.zeros(Q.shape[:3], device=DEV)
    _, ws = cur.curdkv_cache_attention(Q, c, scale=scale, weights=c.raw, q_lens=None if q_lens is None else _ints(q_lens), O=O, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    _check_attention(O, lse, c.raw, w0, c, Q, q_lens or [t] * B, scale, before, what)
    plain = cur.curdkv_cache_attention(Q, c, scale=scale, q_lens=None if q_lens is None else _ints(q_lens), O=_rand(Q.shape, seed + 6))[0]
    assert torch.equal(plain, O)
    return c, Q, O, ws


@pytest.mark.parametrize("group", [1, 2, 3, 4, 7, 8, 9, 16, 17])
@pytest.mark.parametrize("cap,held", [(1, [1, 0]), (40, [40, 17]), (128, [127, 128]), (700, [700, 513]), (2100, [1, 2049])])
def test_one_token(group, cap, held):
    _attend(2, 2, group, 1, cap, held, seed=100)


@pytest.mark.parametrize("t,group", [(2, 4), (3, 1), (5, 3), (16, 1), (16, 8), (64, 16)])
@pytest.mark.parametrize("cap,held", [(3, [3, 1, 0, 2, 3]), (300, [300, 129, 64, 1, 255])])
def test_several_tokens(t, group, cap, held):
    """Every token its own view of the positions; sequences with fewer tokens, or none."""
    _attend(5, 2, group, t, cap, held, q_lens=[t, t - 1, 0, t, 1], seed=200)


@pytest.mark.parametrize("B,H", [(1, 1), (1, 8), (40, 8), (300, 2)])
def test_many_heads_and_few(B, H):
    """Parts for the whole device from one head; several rounds of CTAs."""
    n = 5000 if B * H <= 8 else 600
    _attend(B, H, 4, 1, n + 3, [max(0, n - 7 * b) for b in range(B)], seed=300)


def test_large_weights_and_flat_ones():
    for gain, scale in ((8.0, SCALE), (1.0, 0.0), (0.01, SCALE)):
        c = _cache(2, 2, 500, [500, 333], 400)
        c.K.mul_(gain)
        _attend(2, 2, 4, 1, 500, [500, 333], scale=scale, c=c, seed=401)


def test_slots_behind_the_count_hold_anything():
    for t in (1, 4):
        c = _cache(2, 2, 300, [200, 131], 500)
        for b, n in enumerate((200, 131)):
            c.K[b, :, n:] = float("nan")
            c.V[b, :, n:] = float("inf")
            c.pos[b, :, n:] = -7
        _attend(2, 2, 4, t, 300, [200, 131], c=c, seed=501)


def test_odd_queries_stay_in_their_row():
    """A NaN in one query row reaches that row's output and its head's weights, and no others."""
    c = _cache(2, 2, 300, [300, 200], 600)
    Q = _rand((2, 8, 1, 128), 601)
    want = cur.curdkv_cache_attention(Q, c, scale=SCALE)[0]
    Q[0, 1, 0, 5] = float("nan")
    w = torch.zeros_like(c.raw)
    got = cur.curdkv_cache_attention(Q, c, scale=SCALE, weights=w)[0]
    assert got[0, 1].isnan().all()
    got[0, 1] = want[0, 1]
    assert torch.equal(got, want)
    assert w[0, 0].isnan().all() and not w[0, 1].isnan().any() and not w[1].isnan().any()


def test_dead_tokens_may_hold_nan():
    c = _cache(2, 2, 200, [200, 150], 650)
    Q = _rand((2, 8, 3, 128), 651)
    Q[0, :, 2], Q[1] = float("nan"), float("inf")
    _attend(2, 2, 4, 3, 200, [200, 150], q_lens=[2, 0], c=c, Q=Q, seed=652)


def test_queries_and_outputs_in_other_orders():
    c = _cache(2, 2, 300, [300, 200], 700)
    Q = _rand((2, 3, 8, 128), 701).transpose(1, 2)
    buf = torch.full((2, 3, 8, 136), 5.0, dtype=torch.bfloat16, device=DEV)
    O, w0 = buf[..., :128].transpose(1, 2), c.raw.clone()
    cur.curdkv_cache_attention(Q, c, scale=SCALE, weights=c.raw, O=O)
    _check_attention(O, None, c.raw, w0, c, Q, [3, 3], SCALE, _f64(O))
    assert torch.all(buf[..., 128:] == 5.0)


def test_counts_out_of_range_are_cut_and_noted():
    c = _cache(2, 1, 64, [64, 10], 800)
    c.count.copy_(_ints([1000, -5]))
    O, ws = cur.curdkv_cache_attention(_rand((2, 4, 1, 128), 801), c, scale=SCALE, weights=c.raw)
    assert cur.curdkv_device_status(ws) == cur.DEV_BAD_INDEX
    assert not O[1].any()
    c.count.copy_(_ints([64, 10]))
    _attend(2, 1, 4, 1, 64, [64, 10], c=c, seed=802)


def test_same_results_every_time_and_in_a_graph():
    """Equal bit for bit: again, on another stream, captured and replayed, and two calls side by side with a workspace each."""
    B, H = 2, 8
    caches = [_cache(B, H, 1703, [1702, 901], 900 + i) for i in range(2)]
    Q = [_rand((B, 4 * H, 1, 128), 910 + i) for i in range(2)]
    new = [[_rand((B, H, 1, 128), 920 + 2 * i + j) for j in range(2)] for i in range(2)]
    wsp = [cur.cache_workspace(B, H, 1, 1703, 1702) for _ in range(2)]
    wsa = [cur.cache_attention_workspace(c, 4 * H, 1) for c in caches]
    O = [torch.zeros_like(q) for q in Q]
    start = [_state(c) for c in caches]

    def restore():
        for c, s in zip(caches, start):
            for x, v in s.items():
                getattr(c, x).copy_(v)

    def step(i):
        cur.curdkv_cache_push(caches[i], *new[i], 1702, wsp[i], num_sink=4, window=64)
        cur.curdkv_cache_attention(Q[i], caches[i], scale=SCALE, weights=caches[i].raw, O=O[i], workspace=wsa[i])

    def run():
        for i in range(2):
            for _ in range(3):
                step(i)
    run()
    want = [(_state(c), o.clone()) for c, o in zip(caches, O)]

    def same():
        torch.cuda.synchronize()
        for c, o, (s, wo) in zip(caches, O, want):
            assert torch.equal(o, wo)
            for x, v in s.items():
                assert torch.equal(getattr(c, x), v), x
    restore()
    run()
    same()
    restore()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                step(i)
    same()
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in range(2):
            step(i)
    restore()
    for _ in range(3):
        graph.replay()
    same()


@pytest.mark.parametrize("B,H,group,t,cap", [(1, 2, 4, 1, 40), (1, 8, 4, 1, 1702), (1, 2, 4, 1, 40000), (40, 8, 4, 1, 2049), (2, 2, 4, 4, 900), (1, 1, 8, 5, 700)])
def test_weights_keep_their_bits_before_the_values(B, H, group, t, cap):
    """Every form of the call.  Error budget of O: two bf16 parts of a weight leave 2^-16 of it; logits (in numerator and
    denominator), exponentials and sums as above; O rounded once."""
    c, Q = _cache(B, H, cap, [cap] * B, 900 + cap), _rand((B, H * group, t, 128), 901 + cap)
    for weights in (None, torch.zeros_like(c.raw)):
        O = _f64(cur.curdkv_cache_attention(Q, c, scale=SCALE, weights=weights)[0])
        for b, h in {(0, 0), (B - 1, H - 1)}:
            q, k, v = _f64(Q[b, h * group: (h + 1) * group]), _f64(c.K[b, h]), _f64(c.V[b, h])
            pos = c.pos[b, h].cpu().numpy() if t > 1 else np.zeros(cap, np.int64)
            want, _, w = orc.cache_attention(q, k, v, pos, int(c.total[b]) if t > 1 else 1, SCALE)
            d = (2.0 ** -20 + 2.0 ** -23) * SCALE * (np.abs(q) @ np.abs(k).T).max(-1)
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -16 + 2 * d + 2.0 ** -18)[..., None] * (w @ np.abs(v)) * (1 + 2.0 ** -7)
            err = np.abs(O[b, h * group: (h + 1) * group] - want)
            assert np.all(err <= tol), f"{(err / tol).max():.3g} of the tolerance"
