"""Scores of a prompt's rows by the attention weights they receive, on the GPU against the float64 oracle, and the way from
them through selection, generation and eviction.  Needs a B200."""
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


def _check(scores, lse, Q, K, lens, q_lens, scale, normalised, given=None, heads=None, what=""):
    """Error budget of a score: every weight is off by the logits' fp32 sums of 128 exact products (2^-20 of the sum of magnitudes,
    in numerator and denominator; 2^-24 of a given log sum, twice) and 2^-18 for exponentials and the fp32 sum that it is
    divided by; the weights are added in fp32, at most a quarter of the query rows behind one another."""
    got, Qf, Kf = scores.cpu().numpy().astype(np.float64), _f64(Q), _f64(K)
    B, Hq, t = Q.shape[:3]
    H, n_max = K.shape[1], K.shape[2]
    group = Hq // H
    for b in range(B):
        n, tb = lens[b], min(max(q_lens[b], 0), t)
        for h in range(H) if heads is None else heads:
            q, k = Qf[b, h * group: (h + 1) * group, :tb], Kf[b, h, :n]
            g = None if given is None else given[b, h * group: (h + 1) * group, :tb].cpu().numpy().astype(np.float64)
            want = orc.scores(q, k, scale, normalised, g)
            mags = [scale * (np.abs(x) @ np.abs(k).T).max(initial=0.0) if tb and n else 0.0 for x in q]
            d = 2.0 ** -20 * max(mags, default=0.0)
            top = 0.0 if given is None or tb == 0 else 2.0 ** -22 * np.abs(np.where(np.isinf(g), 0, g)).max(initial=0.0)
            tol = (2 * d + top + 2.0 ** -18 + 2.0 ** -24 * (group * tb / 4 + 16)) * want + 1e-37
            err = np.abs(got[b, h, :n] - want)
            assert np.all(err <= tol), f"{what} b={b} h={h}: {np.nanmax(err / tol):.3g} of the tolerance at {np.argmax(err / tol)}"
            assert not got[b, h, n:].any()
            if lse is not None:
                for x in range(group):
                    seen = orc.window_mask(n, tb, n + tb, 0)
                    ref = orc.attend(q[x], k, np.zeros((n, 1)), seen, scale)[1]
                    have = lse[b, h * group + x, :tb].cpu().numpy()
                    dead = np.isneginf(ref)
                    assert np.array_equal(np.isneginf(have), dead)
                    ref = np.where(dead, 0, ref)
                    assert np.all(dead | (np.abs(have - ref) <= d + 2.0 ** -20 * (1 + np.abs(ref)) + 2.0 ** -18))


def _run(B, H, group, n, t, lens=None, q_lens=None, scale=SCALE, seed=0, K=None, Q=None, normalised=True, heads=None):
    K = _rand((B, H, n, 128), seed) if K is None else K
    Q = _rand((B, H * group, t, 128), seed + 1) if Q is None else Q
    desc = cur.make_desc(K, K, 1, q_heads=H * group, seqlens=None if lens is None else _ints(lens), raw_scores=int(not normalised))
    ql = None if q_lens is None else _ints(q_lens)
    lens, q_lens = lens or [n] * B, q_lens or [t] * B
    scores = torch.full((B, H, n), 7.0, device=DEV)
    lse = torch.full(Q.shape[:3], 7.0, device=DEV)
    what = f"{(B, H, group, n, t)}"
    _, ws = cur.curdkv_attention_scores(Q, K, desc, scale=scale, q_lens=ql, scores=scores, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    _check(scores, lse, Q, K, lens, q_lens, scale, normalised, heads=heads, what=what)
    for b in range(B):
        assert torch.all(lse[b, :, min(max(q_lens[b], 0), t):] == 7.0)
    again = cur.curdkv_attention_scores(Q, K, desc, scale=scale, q_lens=ql, workspace=ws)[0]
    assert torch.equal(again, scores)
    given = cur.curdkv_attention_scores(Q, K, desc, scale=scale, q_lens=ql, lse=lse, lse_given=True, workspace=ws)[0]
    assert cur.curdkv_device_status(ws) == 0
    _check(given, None, Q, K, lens, q_lens, scale, normalised, given=lse, heads=heads, what=what + " given")
    return scores, lse, Q, K, desc


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 8, 17, 65, 100, 128])
@pytest.mark.parametrize("n,t", [(1, 1), (130, 1), (300, 5)])
def test_groups(group, n, t):
    _run(2, 2, group, n, t, seed=10)


@pytest.mark.parametrize("n,t", [(2, 2), (127, 127), (128, 128), (129, 129), (257, 256), (600, 31), (600, 32), (600, 33), (1000, 64), (1000, 1000)])
@pytest.mark.parametrize("group", [1, 3, 4])
def test_lengths(group, n, t):
    _run(1, 2, group, n, t, seed=20)


@pytest.mark.parametrize("t", [1, 40, 300])
def test_ragged(t):
    """Sequences with fewer queries than the block, with none, with more queries than rows, and without rows."""
    for group in (2, 3):
        _run(6, 2, group, 300, t, lens=[300, 299, 150, 1, 0, 20], q_lens=[t, max(t - 3, 0), 0, t, t, t], seed=30)


def test_sums_without_normalisation_and_one_head():
    _run(1, 1, 4, 700, 700, normalised=False, seed=40)
    _run(1, 1, 1, 3000, 16, normalised=False, seed=41)


def test_many_heads_and_long_rows():
    _run(40, 8, 4, 260, 32, seed=50, heads=[0, 7])
    _run(1, 1, 4, 30000, 32, seed=51)
    _run(2, 2, 4, 2500, 2500, lens=[2500, 1700], q_lens=[2500, 1700], seed=52, heads=[1])


def test_large_and_flat_logits():
    K = _rand((1, 2, 500, 128), 60, 8.0)
    _run(1, 2, 4, 500, 100, K=K, seed=61)
    _run(1, 2, 4, 500, 100, scale=0.0, seed=62)
    ramp = torch.linspace(0, 40, 900, device=DEV)
    for x in (ramp, ramp.flip(0)):
        K = _rand((1, 1, 900, 128), 63, 0.2).float()
        K[..., 0] = x
        Q = _rand((1, 2, 200, 128), 64, 0.2)
        Q[..., 0] += 3
        _run(1, 1, 2, 900, 200, K=K.to(torch.bfloat16), Q=Q, seed=65)


def test_rows_that_do_not_exist_hold_anything():
    for group in (4, 3):
        K, Q = _rand((2, 2, 400, 128), 70), _rand((2, 2 * group, 90, 128), 71)
        lens, q_lens = [333, 129], [90, 41]
        for b in range(2):
            K[b, :, lens[b]:] = float("nan")
            Q[b, :, q_lens[b]:] = float("inf") if b else float("nan")
        _run(2, 2, group, 400, 90, lens=lens, q_lens=q_lens, K=K, Q=Q, seed=72)


def test_strides_and_views():
    """Tokens before heads."""
    B, H, group, n, t = 2, 2, 4, 300, 70
    K, Q = _rand((B, n, H, 128), 80).transpose(1, 2), _rand((B, t, H * group, 128), 81).transpose(1, 2)
    _run(B, H, group, n, t, K=K, Q=Q)
    wide = _rand((B, H, n, 256), 82)[..., 64:192]
    _run(B, H, group, n, t, K=wide, Q=_rand((B, H * group, 2 * t, 128), 83)[:, :, ::2])


def test_log_sums_of_the_window_attention_serve():
    B, H, group, n = 2, 2, 4, 520
    K, V, Q = _rand((B, H, n, 128), 90), _rand((B, H, n, 128), 91), _rand((B, H * group, n, 128), 92)
    lens = [520, 301]
    desc = cur.make_desc(K, V, 1, q_heads=H * group, seqlens=_ints(lens))
    lse = torch.zeros((B, H * group, n), device=DEV)
    cur.curdkv_attention_window(Q, K, V, desc, n, scale=SCALE, q_lens=_ints(lens), lse=lse)
    scores = cur.curdkv_attention_scores(Q, K, desc, scale=SCALE, q_lens=_ints(lens), lse=lse, lse_given=True)[0]
    _check(scores, None, Q, K, lens, lens, SCALE, True, given=lse)
    free = cur.curdkv_attention_scores(Q, K, desc, scale=SCALE, q_lens=_ints(lens))[0]
    assert torch.allclose(scores, free, rtol=2e-4, atol=1e-9)
    assert torch.allclose(scores.sum(-1), torch.ones((B, H), device=DEV), rtol=1e-4)


def test_same_results_every_time_and_in_a_graph():
    K, Q = _rand((2, 4, 1500, 128), 100), _rand((2, 16, 400, 128), 101)
    desc = cur.make_desc(K, K, 1, q_heads=16)
    want, _ = cur.curdkv_attention_scores(Q, K, desc, scale=SCALE)
    outs = [torch.zeros_like(want) for _ in range(2)]
    wss = [cur.attention_scores_workspace(desc, 400) for _ in range(2)]
    torch.cuda.synchronize()
    for i, st in enumerate([torch.cuda.Stream() for _ in range(2)]):
        with torch.cuda.stream(st):
            for _ in range(4):
                cur.curdkv_attention_scores(Q, K, desc, scale=SCALE, scores=outs[i], workspace=wss[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cur.curdkv_attention_scores(Q, K, desc, scale=SCALE, scores=outs[0], workspace=wss[0])
    outs[0].zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want)


def test_prompt_to_generation():
    """The calls together: a prompt ranked by what its last tokens look at, its best rows held, then tokens generated, each
    step evicting the least looked-at row; every step against the oracle on the cache as it stands, which tokens stay
    exactly."""
    B, H, group, n, budget, sink, window, steps = 2, 2, 4, 400, 60, 4, 16, 6
    K, V, Q = _rand((B, H, n, 128), 110), _rand((B, H, n, 128), 111), _rand((B, H * group, 32, 128), 112)
    lens = [400, 333]
    desc = cur.make_desc(K, V, 1, q_heads=H * group, seqlens=_ints(lens), raw_scores=1)
    scores, ws = cur.curdkv_attention_scores(Q, K, desc, scale=SCALE)
    _check(scores, None, Q, K, lens, [32] * B, SCALE, False)
    idx, counts, offsets = cur.curdkv_select(scores, desc, budget, num_sink=sink, window=window)
    cache = cur.DeviceCache(B, H, budget + 1, 128)
    K_c, V_c = cur.curdkv_compact(K, V, desc, idx, counts, offsets)
    cache.K[:, :, :budget], cache.V[:, :, :budget] = K_c, V_c
    cache.raw[:, :, :budget], cache.pos[:, :, :budget] = scores.gather(-1, idx.long()), idx
    cache.count.fill_(budget)
    cache.total.copy_(_ints(lens))
    wsp, wsa = cur.cache_workspace(B, H, 1, budget + 1, budget), cur.cache_attention_workspace(cache, H * group, 1)
    for s in range(steps):
        kn, vn, q = _rand((B, H, 1, 128), 120 + s), _rand((B, H, 1, 128), 140 + s), _rand((B, H * group, 1, 128), 160 + s)
        raw, pos = cache.raw.cpu().numpy(), cache.pos.cpu().numpy()
        old = {x: getattr(cache, x).clone() for x in "KV"}
        cur.curdkv_cache_push(cache, kn, vn, budget, wsp, num_sink=sink, window=window)
        mid = cache.raw.clone()
        for b in range(B):
            for h in range(H):
                at, r, p = orc.push(raw[b, h, :budget], pos[b, h, :budget], lens[b] + s, [0.0], budget, sink, window)
                assert np.array_equal(cache.pos[b, h, :budget].cpu().numpy(), p)
                assert np.array_equal(mid[b, h, :budget].cpu().numpy(), r)
                for x, new in (("K", kn), ("V", vn)):
                    assert torch.equal(getattr(cache, x)[b, h, :budget], torch.cat([old[x][b, h, :budget], new[b, h]])[torch.from_numpy(at).to(DEV)])
        O, _ = cur.curdkv_cache_attention(q, cache, scale=SCALE, weights=cache.raw, workspace=wsa)
        Kf, Vf, qf, got = _f64(cache.K), _f64(cache.V), _f64(q), _f64(O)
        for b in range(B):
            for h in range(H):
                want, _, w = orc.cache_attention(qf[b, h * group: (h + 1) * group], Kf[b, h, :budget], Vf[b, h, :budget],
                                                 np.zeros(budget), 1, SCALE)
                tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * 1.01 * (w @ np.abs(Vf[b, h, :budget])) + 1e-38
                assert np.all(np.abs(got[b, h * group: (h + 1) * group] - want) <= tol)
                grown = cache.raw[b, h, :budget].cpu().numpy() - mid[b, h, :budget].cpu().numpy().astype(np.float64)
                assert np.all(np.abs(grown - w.sum((0, 1))) <= 1e-4 * w.sum((0, 1)) + 2.0 ** -22 * (1 + mid[b, h, :budget].cpu().numpy()))
    assert cur.curdkv_device_status(wsp) == 0 and cur.curdkv_device_status(wsa) == 0 and cur.curdkv_device_status(ws) == 0


@pytest.mark.parametrize("t,lse", [(300, False), (300, True), (40, False), (40, True)])
def test_a_nan_reaches_every_row_that_it_should(t, lse):
    """Wherever it stands in a tile: one in a query makes the scores of all rows that it sees NaN and leaves the others as they are,
    one in a key the log sums of the tokens that see it, and the scores of the rows that these see."""
    n = 300
    K, Q = _rand((1, 1, n, 128), 300), _rand((1, 4, t, 128), 301)

    def call(Q, K):
        out = torch.zeros((1, 4, t), device=DEV) if lse else None
        return cur.curdkv_attention_scores(Q, K, cur.make_desc(K, K, 1, q_heads=4, raw_scores=1), scale=SCALE, lse=out)[0], out

    clean, clean_lse = call(Q, K)
    assert clean.isfinite().all()
    for i in [*range(9), 16, 31, t - 1]:                     # rows 4 i + head of a tile: each of 16 columns, and further tiles
        for head in range(4):
            q = Q.clone()
            q[0, head, i, 5] = float("nan")
            got, sums = call(q, K)
            sees = n - t + i + 1
            assert got[0, 0, :sees].isnan().all() and torch.equal(got[0, 0, sees:], clean[0, 0, sees:]), (i, head)
            if lse:
                assert sums[0, head, i].isnan()
                sums[0, head, i] = clean_lse[0, head, i]
                assert torch.equal(sums, clean_lse)
    for j in [*range(18), 64, 65, 66, 255, n - 1]:
        k = K.clone()
        k[0, 0, j, 77] = float("nan")
        got, sums = call(Q, k)
        assert got.isnan().all(), j                          # (the last token sees every row)
        if lse:
            first = max(0, j - (n - t))
            assert sums[0, :, first:].isnan().all() and torch.equal(sums[0, :, :first], clean_lse[0, :, :first]), j


@pytest.mark.parametrize("n,t", [(300, 300), (300, 40)])
def test_a_log_sum_far_too_low_gives_nothing_finite(n, t):
    """Weights of some 2^144 in one query row, wherever it stands in a tile: infinite scores (or NaN) of all rows that it sees, no
    numbers of either sign; the other rows' scores as they are."""
    K, Q = _rand((1, 1, n, 128), 310), _rand((1, 4, t, 128), 311)
    desc, lse = cur.make_desc(K, K, 1, q_heads=4), torch.zeros((1, 4, t), device=DEV)
    cur.curdkv_attention_scores(Q, K, desc, scale=SCALE, lse=lse)
    clean = cur.curdkv_attention_scores(Q, K, desc, scale=SCALE, lse=lse, lse_given=True)[0]
    for i in (0, 1, 2, 3, 4, 17, t - 1):
        for head in range(4):
            low = lse.clone()
            low[0, head, i] = -100.0
            got = cur.curdkv_attention_scores(Q, K, desc, scale=SCALE, lse=low, lse_given=True)[0]
            sees = n - t + i + 1
            assert not got[0, 0, :sees].isfinite().any() and torch.equal(got[0, 0, sees:], clean[0, 0, sees:]), (i, head)


@pytest.mark.parametrize("seed", [320, 330, 340])
@pytest.mark.parametrize("scale", [SCALE, 0.1, 0.0625])
def test_log_sums_in_full_precision(seed, scale):
    """Logits up to some 12 with log sums from elsewhere, exact but for their fp32.  Error budget of the 2-norm of the scores: the
    tensor cores cut a sum by 0.8e-7 to 1.5e-7 of it on average, of which all but 0.3e-7 is given back at the logits that carry
    weight (12 of it: 3.6e-7), and what is random (the rest of it, and half a step of a log sum, 2^-21) averages over a hundred rows
    and more to a tenth (0.4e-7); exponentials and sums 1e-7."""
    n, group = 1024, 4
    K = _rand((1, 2, n, 128), seed).float()
    strong = torch.rand((1, 2, 1, 128), generator=torch.Generator(device=DEV).manual_seed(seed + 1), device=DEV).argsort(-1) < 4
    K = torch.where(strong, 10.0 * K, K).to(torch.bfloat16)
    Q = _rand((1, 2 * group, n, 128), seed + 2)
    x = (Q.double() @ K.double().repeat_interleave(group, 1).transpose(2, 3)) * float(np.float32(scale))
    x = x.masked_fill(torch.ones((n, n), dtype=torch.bool, device=DEV).triu(1), float("-inf"))
    lse = torch.logsumexp(x, -1).float()
    want = torch.exp(x - lse.double()[..., None]).sum(2).unflatten(1, (2, group)).sum(2)
    got = cur.curdkv_attention_scores(Q, K, cur.make_desc(K, K, 1, q_heads=2 * group, raw_scores=1), scale=scale, lse=lse, lse_given=True)[0]
    off = float((got.double() - want).norm() / want.norm())
    assert off <= 5e-7, off
