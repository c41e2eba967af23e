"""Attention of a batch that shares a prefix, on the GPU against the float64 oracle.  Needs a B200."""
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


def _check(O, lse, Q, K0, V0, lens0, K, V, lens, q_lens, scale, before, heads=None, seqs=None, what=""):
    """Error budget: weights rounded to bf16 (2^-8 of each), logits with fp32 sums of 128 exact products (2^-20 of the sum of
    magnitudes, in numerator and denominator), 2^-18 for exponentials, fp32 sums and the joining of parts, O rounded
    once (2^-8)."""
    got, Qf, K0f, V0f, Kf, Vf = (_f64(x) for x in (O, Q, K0, V0, K, V))
    B, Hq, t = Q.shape[:3]
    group, share = Hq // K.shape[1], B // K0.shape[0]
    for b in range(B) if seqs is None else seqs:
        p, n0, n, tb = b // share, lens0[b // share], lens[b], min(max(q_lens[b], 0), t)
        for hq in range(Hq) if heads is None else heads:
            h = hq // group
            k0, v0, k, v, q = K0f[p, h, :n0], V0f[p, h, :n0], Kf[b, h, :n], Vf[b, h, :n], Qf[b, hq, :tb]
            want, want_lse, w = orc.prefix_attention(q, k0, v0, k, v, scale)
            keys, vals = np.concatenate([k0, k]), np.concatenate([v0, v])
            d = 2.0 ** -20 * scale * (np.abs(q) @ np.abs(keys).T).max(-1, initial=0.0)
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * d + 2.0 ** -18)[:, None] * (w @ np.abs(vals)) * (1 + 2.0 ** -7) + 1e-38
            err = np.abs(got[b, hq, :tb] - want)
            assert np.all(err <= tol), f"{what} b={b} head={hq}: {np.nanmax(err / tol):.3g} of the tolerance"
            dead = np.isneginf(want_lse)
            assert not got[b, hq, :tb][dead].any()
            assert np.array_equal(got[b, hq, tb:], before[b, hq, tb:])
            if lse is not None:
                g, ref = lse[b, hq, :tb].cpu().numpy(), np.where(dead, 0.0, want_lse)
                assert np.all(np.isneginf(g[dead]))
                assert np.all(dead | (np.abs(g - ref) <= d + 2.0 ** -20 * (1 + np.abs(ref)) + 2.0 ** -18))


def _run(Bp, share, H, group, n0, n, t, lens0=None, lens=None, q_lens=None, scale=SCALE, seed=0, K0=None, V0=None, K=None, V=None,
         Q=None, **kw):
    B = Bp * share
    K0 = _rand((Bp, H, n0, 128), seed) if K0 is None else K0
    V0 = _rand((Bp, H, n0, 128), seed + 1) if V0 is None else V0
    K = _rand((B, H, n, 128), seed + 2) if K is None else K
    V = _rand((B, H, n, 128), seed + 3) if V is None else V
    Q = _rand((B, H * group, t, 128), seed + 4) if Q is None else Q
    d0 = cur.make_desc(K0, V0, 1, seqlens=None if lens0 is None else _ints(lens0))
    d = cur.make_desc(K, V, 1, q_heads=H * group, seqlens=None if lens is None else _ints(lens))
    O = _rand(Q.shape, seed + 5)
    before = _f64(O)
    lse = torch.zeros(Q.shape[:3], device=DEV)
    _, ws = cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=scale, q_lens=None if q_lens is None else _ints(q_lens), O=O, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    _check(O, lse, Q, K0, V0, lens0 or [n0] * Bp, K, V, lens or [n] * B, q_lens or [t] * B, scale, before,
           what=f"{(Bp, share, H, group, n0, n, t)}", **kw)
    return O


@pytest.mark.parametrize("share,group", [(1, 1), (1, 4), (2, 4), (3, 3), (5, 4), (16, 1), (16, 8), (33, 4), (7, 5), (130, 1), (3, 64), (2, 100), (1, 200)])
@pytest.mark.parametrize("n0,n", [(1, 1), (127, 20), (128, 0), (700, 65), (0, 30), (129, 300)])
def test_one_token(share, group, n0, n):
    _run(1, share, 2, group, n0, n, 1, seed=10)


@pytest.mark.parametrize("t,share,group", [(2, 3, 4), (4, 16, 4), (3, 2, 3), (7, 5, 8), (32, 4, 4), (33, 3, 4), (100, 2, 4), (130, 2, 1)])
@pytest.mark.parametrize("n0,n", [(500, 140), (64, 0), (0, 131)])
def test_several_tokens(t, share, group, n0, n):
    """Own rows seen causally; tokens that have no own rows see the prefix only."""
    _run(1, share, 2, group, n0, n, t, seed=20)


@pytest.mark.parametrize("t", [1, 3])
def test_lengths(t):
    """Prefixes of different lengths, one of them empty; own lengths and query counts of every kind."""
    lens = [40, 1, 0, 39, 2, 17, 40, 0, 5, 33, 40, 8]
    q_lens = [t, 1, t, 0, t, t, 1, t, t, t, 0, 1]
    _run(3, 4, 3, 4, 300, 40, t, lens0=[300, 0, 131], lens=lens, q_lens=q_lens, seed=30)
    _run(3, 4, 3, 12, 300, 40, t, lens0=[1, 256, 0], lens=lens, q_lens=q_lens, seed=40)


def test_folded_layers_and_one_sequence_a_prefix():
    _run(8, 4, 2, 4, 400, 30, 1, lens0=[400, 1, 399, 128, 129, 255, 256, 257], seed=50)
    _run(6, 1, 2, 4, 200, 30, 1, seed=60)


def test_long_prefixes():
    """Split over many CTAs, joined."""
    _run(1, 2, 1, 4, 40000, 100, 1, seed=70)
    _run(1, 40, 1, 4, 20000, 3000, 1, seed=71, seqs=[0, 17, 39])
    _run(2, 20, 2, 4, 9000, 70, 2, lens0=[9000, 4097], seed=72, seqs=[0, 19, 20, 39])


def test_rows_behind_the_lengths_hold_anything():
    for share, t in ((2, 1), (12, 1), (12, 3)):
        K0, V0, K, V = (_rand((2 if i < 2 else 2 * share, 2, 300, 128), 80 + i) for i in range(4))
        lens0, lens = [170, 300], [(37 * i) % 290 for i in range(2 * share)]
        for x, ls in ((K0, lens0), (V0, lens0), (K, lens), (V, lens)):
            for b, n in enumerate(ls):
                x[b, :, n:] = float("nan") if x is K0 or x is K else float("inf")
        _run(2, share, 2, 4, 300, 300, t, lens0=lens0, lens=lens, K0=K0, V0=V0, K=K, V=V, seed=90)


def test_odd_queries_stay_in_their_row():
    for share in (2, 20):
        K0, V0, K, V = (_rand((1 if i < 2 else share, 2, 200, 128), 100 + i) for i in range(4))
        d0, d = cur.make_desc(K0, V0, 1), cur.make_desc(K, V, 1, q_heads=8)
        Q = _rand((share, 8, 1, 128), 105)
        want = cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=SCALE)[0]
        Q[1, 3, 0, 7], Q[0, 2, 0, 100] = float("nan"), float("inf")
        got = cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=SCALE)[0]
        assert got[1, 3].isnan().all() and got[0, 2].isnan().all()
        for b, h in ((1, 3), (0, 2)):
            got[b, h] = want[b, h]
        assert torch.equal(got, want)


@pytest.mark.parametrize("share", [2, 20])
def test_logits_that_grow_and_large_values(share):
    n0, n = 900, 200
    for sign in (1.0, -1.0):
        K0 = _rand((1, 1, n0, 128), 110, 0.2).float()
        K0[..., 0] = 40 * (torch.linspace(0, 1, n0, device=DEV) if sign > 0 else torch.linspace(1, 0, n0, device=DEV))
        K0 = K0.to(torch.bfloat16)
        Q = _rand((share, 4, 1, 128), 111, 0.2)
        Q[..., 0] += 3
        _run(1, share, 1, 4, n0, n, 1, K0=K0, Q=Q, seed=112)
    _run(1, share, 1, 4, n0, n, 1, K0=_rand((1, 1, n0, 128), 115, 30.0), V0=_rand((1, 1, n0, 128), 116, 1e30), seed=117)
    _run(1, share, 1, 4, n0, n, 1, scale=0.0, seed=118)


@pytest.mark.parametrize("share,t", [(2, 1), (20, 1), (20, 3)])
def test_strides_and_views(share, t):
    """Tokens before heads everywhere; a prefix that is one cache's expanded view; a longer output row."""
    H, group, n0, n = 2, 4, 260, 50
    K0, V0 = (_rand((1, n0, H, 128), 120 + i).transpose(1, 2) for i in range(2))
    K, V = (_rand((share, n, H, 128), 122 + i).transpose(1, 2) for i in range(2))
    Q = _rand((share, t, H * group, 128), 124).transpose(1, 2)
    d0, d = cur.make_desc(K0, V0, 1), cur.make_desc(K, V, 1, q_heads=H * group)
    buf = torch.full((share, t, H * group, 136), 5.0, dtype=torch.bfloat16, device=DEV)
    O = buf[..., :128].transpose(1, 2)
    cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=0.1, O=O)
    _check(O, None, Q, K0, V0, [n0], K, V, [n] * share, [t] * share, float(np.float32(0.1)), _f64(O))
    assert torch.all(buf[..., 128:] == 5.0)
    K0, V0 = (x.expand(2, H, n0, 128) for x in (K0, V0))                     # both prefixes the same rows
    Qe = Q[:1].expand(2 * share, H * group, t, 128)
    K, V = (torch.cat([x, x]) for x in (K, V))
    d0, d = cur.make_desc(K0, V0, 1), cur.make_desc(K, V, 1, q_heads=H * group)
    O = cur.curdkv_attention_prefix(Qe, K0, V0, d0, K, V, d, scale=0.1)[0]
    _check(O, None, Qe, K0, V0, [n0] * 2, K, V, [n] * 2 * share, [t] * 2 * share, float(np.float32(0.1)), _f64(O), seqs=[0, share + 1])


def test_lengths_out_of_range_are_cut_and_noted():
    K0, V0, K, V = (_rand((1 if i < 2 else 2, 1, 64, 128), 130 + i) for i in range(4))
    Q = _rand((2, 4, 1, 128), 134)
    for lens0, lens in (([100], [3, 5]), ([64], [70, -1])):
        d0, d = cur.make_desc(K0, V0, 1, seqlens=_ints(lens0)), cur.make_desc(K, V, 1, q_heads=4, seqlens=_ints(lens))
        O, ws = cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=SCALE)
        assert cur.curdkv_device_status(ws) == cur.DEV_BAD_INDEX
        cut = [min(max(x, 0), 64) for x in lens]
        _check(O, None, Q, K0, V0, [64], K, V, cut, [1, 1], SCALE, _f64(O))


@pytest.mark.parametrize("share", [3, 24])
def test_same_results_every_time_and_in_a_graph(share):
    """Equal bit for bit: again, on two streams at once with a workspace each, captured and replayed."""
    K0, V0, K, V = (_rand((1 if i < 2 else share, 4, 3000 if i < 2 else 90, 128), 140 + i) for i in range(4))
    Q = _rand((share, 16, 1, 128), 145)
    d0, d = cur.make_desc(K0, V0, 1), cur.make_desc(K, V, 1, q_heads=16)
    want, ws = cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=SCALE)
    outs = [torch.zeros_like(want) for _ in range(2)]
    wss = [cur.attention_prefix_workspace(d0, d, 1) for _ in range(2)]
    torch.cuda.synchronize()
    for i, st in enumerate([torch.cuda.Stream() for _ in range(2)]):
        with torch.cuda.stream(st):
            for _ in range(5):
                cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=SCALE, O=outs[i], workspace=wss[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=SCALE, O=outs[0], workspace=wss[0])
    outs[0].zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want)


@pytest.mark.parametrize("share,t,n0,n", [(1, 1, 40, 30), (4, 1, 700, 65), (2, 2, 300, 200), (3, 1, 0, 500), (40, 1, 0, 300), (1, 1, 9000, 0)])
def test_weights_keep_their_bits_before_the_values(share, t, n0, n):
    """Own rows, and prefixes behind few query rows (those that are read in tiles round weights to bf16).  Error budget: two bf16
    parts of a weight leave 2^-16 of it; logits (in numerator and denominator), exponentials and sums as above; O rounded once."""
    H, group = 2, 4
    K0, V0, K, V = (_rand((1 if i < 2 else share, H, n0 if i < 2 else n, 128), 150 + i) for i in range(4))
    Q = _rand((share, H * group, t, 128), 155)
    d0, d = cur.make_desc(K0, V0, 1), cur.make_desc(K, V, 1, q_heads=H * group)
    O = _f64(cur.curdkv_attention_prefix(Q, K0, V0, d0, K, V, d, scale=SCALE)[0])
    for b in {0, share - 1}:
        for hq in range(H * group):
            h, q = hq // group, _f64(Q[b, hq])
            k0, v0, k, v = _f64(K0[0, h]), _f64(V0[0, h]), _f64(K[b, h]), _f64(V[b, h])
            want, _, w = orc.prefix_attention(q, k0, v0, k, v, SCALE)
            e = 2.0 ** -20 * SCALE * (np.abs(q) @ np.abs(np.concatenate([k0, k])).T).max(-1)
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -16 + 2 * e + 2.0 ** -18)[:, None] * (w @ np.abs(np.concatenate([v0, v]))) * (1 + 2.0 ** -7)
            err = np.abs(O[b, hq] - want)
            assert np.all(err <= tol), f"{(err / tol).max():.3g} of the tolerance"
