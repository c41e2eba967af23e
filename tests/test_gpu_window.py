"""Attention with a sliding window and sinks on the GPU against the float64 oracle.  Needs a B200."""
import numpy as np
import pytest
import torch

from oracle import curdkv_serving_oracle as orc
from paper_2509_15038_b200 import binding as cur
from paper_2509_15038_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rand(shape, seed, gain=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * gain).to(torch.bfloat16)


def _f64(t):
    return synth.u16_to_f64(synth.to_u16(t))


def _check(O, lse, Q, K, V, lens, q_lens, window, sink, scale, before=None, heads=None, what=""):
    """Error budget per output: the weights are rounded to bf16 (half a step: 2^-8 of each), logits carry fp32 sums of 128
    exact products (2^-20 of the sum of magnitudes, in numerator and denominator), 2^-18 for the exponential and the fp32
    sums; O is rounded to bf16 once (2^-8)."""
    got = _f64(O)
    Qf, Kf, Vf = _f64(Q), _f64(K), _f64(V)
    B, Hq, t = Q.shape[:3]
    group = Hq // K.shape[1]
    for b in range(B):
        n, tb = int(lens[b]), int(q_lens[b])
        mask = orc.window_mask(n, tb, window, sink)
        for hq in (range(Hq) if heads is None else heads):
            k, v, q = Kf[b, hq // group, :n], Vf[b, hq // group, :n], Qf[b, hq, :tb]
            want, want_lse, w = orc.attend(q, k, v, mask, scale)
            d = 2.0 ** -20 * scale * (np.abs(q) @ np.abs(k).T).max(-1, initial=0.0)
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * d + 2.0 ** -18)[:, None] * (w @ np.abs(v)) * (1 + 2.0 ** -7) + 1e-38
            err = np.abs(got[b, hq, :tb] - want)
            assert np.all(err <= tol), f"{what} b={b} head={hq}: {np.nanmax(err / tol):.3g} of the tolerance, row {np.argmax((err / tol).max(-1))}"
            dead = ~mask.any(-1)
            assert not got[b, hq, :tb][dead].any()
            if lse is not None:
                g = lse[b, hq, :tb].cpu().numpy()
                assert np.all(np.isneginf(g[dead]))
                assert np.all(np.abs(g[~dead] - want_lse[~dead]) <= (d + 2.0 ** -20 * (1 + np.abs(np.where(dead, 0, want_lse))) + 2.0 ** -18)[~dead])
            if before is not None:
                assert np.array_equal(got[b, hq, tb:], before[b, hq, tb:])       # rows behind the last query


def _run(B, H, group, n, t, window, sink, lens=None, q_lens=None, scale=128 ** -0.5, seed=0, K=None, V=None, **kw):
    K = _rand((B, H, n, 128), seed) if K is None else K
    V = _rand((B, H, n, 128), seed + 1) if V is None else V
    Q = _rand((B, H * group, t, 128), seed + 2)
    lens_t = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    ql_t = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device=DEV)
    desc = cur.make_desc(K, V, 1, q_heads=H * group, seqlens=lens_t)
    O = _rand(Q.shape, seed + 3)
    before = _f64(O)
    lse = torch.zeros(Q.shape[:3], device=DEV)
    _, ws = cur.curdkv_attention_window(Q, K, V, desc, window, num_sink=sink, scale=scale, q_lens=ql_t, O=O, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    lens = [n] * B if lens is None else lens
    q_lens = [t] * B if q_lens is None else [min(max(x, 0), t) for x in q_lens]
    _check(O, lse, Q, K, V, lens, q_lens, window, sink, float(np.float32(scale)), before, what=f"{(B, H, group, n, t, window, sink)}", **kw)
    return Q, K, V, desc, O


@pytest.mark.parametrize("group", [1, 3, 4, 8, 9])
@pytest.mark.parametrize("window,sink", [(1, 0), (16, 4), (17, 0), (128, 4), (1000, 4), (5000, 0), (0, 5), (0, 0), (100, 300)])
def test_single_token(group, window, sink):
    _run(3, 2, group, 1000, 1, window, sink, lens=[1000, 1, 417], seed=10)


@pytest.mark.parametrize("t", [2, 3, 7, 16])
@pytest.mark.parametrize("window,sink", [(1, 0), (16, 4), (200, 33), (5000, 0), (0, 5)])
def test_few_tokens(t, window, sink):
    """Drafted tokens: every query its own window; a sequence with fewer queries than the block, one without any, one with
    more queries than rows."""
    _run(5, 2, 4, 600, t, window, sink, lens=[600, 333, 50, 1, 0], q_lens=[t, t - 1, 0, t, t], seed=20)


@pytest.mark.parametrize("t", [100, 128, 129, 300, 700])
@pytest.mark.parametrize("window,sink", [(1, 0), (64, 4), (128, 0), (129, 130), (333, 1), (5000, 0), (0, 3), (0, 0)])
def test_prompts(t, window, sink):
    _run(3, 2, 2, 700, t, window, sink, lens=[700, 650, 90], q_lens=[t, t - 37, 90], seed=30)


@pytest.mark.parametrize("group,n,t", [(1, 300, 300), (3, 260, 260), (8, 129, 129), (4, 1500, 200), (2, 64, 64), (4, 127, 90)])
def test_prompt_shapes(group, n, t):
    _run(2, 2, group, n, t, 100, 4, lens=[n, max(1, n - 41)], q_lens=[t, max(1, min(t, n - 41))], seed=40)


def test_rows_behind_the_sequence_hold_anything():
    for t in (1, 5, 200):
        K, V = _rand((2, 2, 512, 128), 50), _rand((2, 2, 512, 128), 51)
        lens = [300, 257]
        for b, n in enumerate(lens):
            K[b, :, n:] = float("nan")
            V[b, :, n:] = float("inf")
        _run(2, 2, 2, 512, t, 100, 4, lens=lens, K=K, V=V, seed=52)


def test_strides_and_views():
    """Tokens before heads, as a model's projections leave them, for Q, K, V and O."""
    for t in (1, 4, 150):
        B, H, group, n = 2, 2, 4, 400
        K, V = (_rand((B, n, H, 128), 60 + i).transpose(1, 2) for i in range(2))
        Q = _rand((B, t, H * group, 128), 62).transpose(1, 2)
        desc = cur.make_desc(K, V, 1, q_heads=H * group)
        buf = torch.full((B, t, H * group, 136), 5.0, dtype=torch.bfloat16, device=DEV)
        O = buf[..., :128].transpose(1, 2)
        lse = torch.zeros((B, H * group, t), device=DEV)
        cur.curdkv_attention_window(Q, K, V, desc, 90, num_sink=4, scale=0.1, O=O, lse=lse)
        _check(O, lse, Q, K, V, [n] * B, [t] * B, 90, 4, float(np.float32(0.1)), what=f"t={t}")
        assert torch.all(buf[..., 128:] == 5.0)


@pytest.mark.parametrize("t", [1, 6, 300])
def test_logits_that_grow_or_shrink(t):
    n = 1200
    ramp = torch.linspace(0, 1, n, device=DEV)
    for sign in (1.0, -1.0):
        K = _rand((1, 1, n, 128), 70, 0.2).float()
        K[..., 0] = 40 * (ramp if sign > 0 else 1 - ramp)
        K = K.to(torch.bfloat16)
        V = _rand((1, 1, n, 128), 71)
        Q = _rand((1, 2, t, 128), 72, 0.2).float()
        Q[..., 0] += 3
        Q = Q.to(torch.bfloat16)
        desc = cur.make_desc(K, V, 1, q_heads=2)
        lse = torch.zeros((1, 2, t), device=DEV)
        for scale, window in ((1.0, 5000), (1.0, 700), (0.0, 700)):
            O, ws = cur.curdkv_attention_window(Q, K, V, desc, window, num_sink=3, scale=scale, lse=lse)
            assert cur.curdkv_device_status(ws) == 0
            _check(O, lse, Q, K, V, [n], [t], window, 3, scale, what=f"{sign} {scale} {window}")


def test_window_of_everything_is_causal_attention_and_agrees_with_the_evaluator():
    """With a window beyond the sequence the last query sees every row: what curdkv_attention_out computes for it."""
    B, H, n = 2, 2, 640
    Q, K, V, desc, O = _run(B, H, 1, n, 200, n, 0, seed=80)
    full, _ = cur.curdkv_attention_out(Q[:, :, -1:].contiguous(), K, V, desc, scale=128 ** -0.5)
    d = (O[:, :, -1:].float() - full).abs().max().item()
    # both within their own budget of the exact value: 2^-8 for the output's rounding, 2^-8 for the weights'
    assert d <= 2.0 ** -7 * full.abs().max().item()


@pytest.mark.parametrize("t", [1, 4, 260])
def test_graph_other_stream_and_repeat(t):
    B, H, group, n, window, sink = 2, 2, 4, 1500, 300, 4
    K, V = _rand((B, H, n, 128), 90), _rand((B, H, n, 128), 91)
    lens = torch.tensor([1400, 900], dtype=torch.int32, device=DEV)
    desc = cur.make_desc(K, V, 1, q_heads=H * group, seqlens=lens)
    Q = _rand((B, H * group, t, 128), 92)
    O, lse = torch.zeros_like(Q), torch.zeros(Q.shape[:3], device=DEV)
    ws = cur.attention_window_workspace(desc, t)
    call = lambda: cur.curdkv_attention_window(Q, K, V, desc, window, num_sink=sink, scale=0.1, O=O, lse=lse, workspace=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    _check(O, lse, Q, K, V, [1400, 900], [t, t], window, sink, float(np.float32(0.1)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):                                     # new rows and lengths under the same graph
        K.copy_(_rand(K.shape, 100 + i))
        Q.copy_(_rand(Q.shape, 110 + i))
        now = [1400 + i, 900 - 300 * i]
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        _check(O, lse, Q, K, V, now, [t, t], window, sink, float(np.float32(0.1)))
    first = O.clone()
    graph.replay()
    assert torch.equal(first, O)
    assert cur.curdkv_device_status(ws) == 0


def test_parts_join_by_their_log_sums():
    """A sequence attended in two parts -- its old rows held in 4 bits, the recent ones in bf16 through the window call --
    joins by lse to the attention over both (within the two parts' own budgets)."""
    H, n_old, n_new = 2, 500, 60
    K, V = _rand((1, H, n_old + n_new, 128), 120), _rand((1, H, n_old + n_new, 128), 121)
    Q = _rand((1, H, 1, 128), 122)
    cache = cur.QuantCache(1, H, n_old)
    cur.curdkv_qcache_store(cache, K[:, :, :n_old], V[:, :, :n_old], cur.make_desc(K[:, :, :n_old], V[:, :, :n_old], 1))
    l0, l1 = torch.zeros((1, H, 1), device=DEV), torch.zeros((1, H, 1), device=DEV)
    o0, _ = cur.curdkv_qcache_attention(Q, cache, scale=0.1, lse=l0)
    new = (K[:, :, n_old:], V[:, :, n_old:])
    o1, _ = cur.curdkv_attention_window(Q, *new, cur.make_desc(*new, 1), n_new, scale=0.1, lse=l1)
    w = torch.sigmoid(l0.double() - l1.double())[..., None]
    joined = (w * o0.double() + (1 - w) * o1.double()).cpu().numpy()
    bits = lambda m: m.view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
    for h in range(H):
        k, _ = orc.unpack(cache.K_codes[0, h].cpu().numpy(), bits(cache.K_meta[0, h].view(-1, 8)), "K")
        v, vp = orc.unpack(cache.V_codes[0, h].cpu().numpy(), bits(cache.V_meta[0, h].view(-1, 8)), "V")
        k, v = np.concatenate([k, _f64(K)[0, h, n_old:]]), np.concatenate([v, _f64(V)[0, h, n_old:]])
        vp = np.concatenate([vp, np.abs(_f64(V)[0, h, n_old:])])
        want, _, wt = orc.attend(_f64(Q)[0, h], k, v, np.ones((1, k.shape[0]), bool), float(np.float32(0.1)))
        assert np.all(np.abs(joined[0, h] - want) <= (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -12) * (wt @ vp) * (1 + 2.0 ** -7))


# Prompts over enough heads that the tensor-core form for prompts is taken (few heads and short windows
# take the form for few query rows, which the tests above cover).
HEADS = [0, 13, 31]                                        # query heads that are compared


@pytest.mark.parametrize("t", [129, 300, 700])
@pytest.mark.parametrize("window,sink", [(64, 4), (128, 0), (129, 130), (333, 1), (5000, 0), (0, 300)])
def test_prompts_over_many_heads(t, window, sink):
    _run(3, 8, 4, 700, t, window, sink, lens=[700, 650, 90], q_lens=[t, t - 37, 90], seed=130, heads=HEADS)


@pytest.mark.parametrize("window,sink", [(1, 0), (2, 1), (0, 3), (0, 0)])
def test_long_prompts_that_see_little(window, sink):
    _run(3, 16, 4, 1200, 1200, window, sink, lens=[1200, 0, 1], q_lens=[1200, 1200, 1200], seed=135, heads=[0, 63])


@pytest.mark.parametrize("B,H,group,n,t", [(30, 9, 1, 300, 300), (12, 8, 3, 260, 260), (3, 8, 8, 129, 129), (64, 8, 1, 200, 200),
                                          (8, 8, 4, 64, 64), (8, 8, 4, 127, 90), (3, 16, 4, 1500, 200), (40, 8, 16, 40, 20)])
def test_prompt_shapes_over_many_heads(B, H, group, n, t):
    lens = [max(1, n - 41) if b % 2 else n for b in range(B)]
    _run(B, H, group, n, t, 100, 4, lens=lens, q_lens=[max(1, min(t, x)) for x in lens], seed=140, heads=[0, H * group - 1])


def test_prompts_with_rows_behind_the_sequence_that_hold_anything():
    K, V = _rand((3, 8, 512, 128), 150), _rand((3, 8, 512, 128), 151)
    lens = [300, 257, 512]
    for b, n in enumerate(lens):
        K[b, :, n:] = float("nan")
        V[b, :, n:] = float("inf")
    _run(3, 8, 4, 512, 250, 100, 4, lens=lens, K=K, V=V, seed=152, heads=HEADS)


def test_prompts_with_strides_and_views():
    B, H, group, n, t = 3, 8, 4, 400, 300
    K, V = (_rand((B, n, H, 128), 160 + i).transpose(1, 2) for i in range(2))
    Q = _rand((B, t, H * group, 128), 162).transpose(1, 2)
    desc = cur.make_desc(K, V, 1, q_heads=H * group)
    buf = torch.full((B, t, H * group, 136), 5.0, dtype=torch.bfloat16, device=DEV)
    O = buf[..., :128].transpose(1, 2)
    lse = torch.zeros((B, H * group, t), device=DEV)
    cur.curdkv_attention_window(Q, K, V, desc, 90, num_sink=4, scale=0.1, O=O, lse=lse)
    _check(O, lse, Q, K, V, [n] * B, [t] * B, 90, 4, float(np.float32(0.1)), heads=HEADS)
    assert torch.all(buf[..., 128:] == 5.0)


@pytest.mark.parametrize("sign", [1, -1])
def test_prompts_with_logits_that_grow_or_shrink(sign):
    H, n, t = 8, 1200, 700
    ramp = torch.linspace(0, 1, n, device=DEV)
    K = _rand((2, H, n, 128), 170, 0.2).float()
    K[..., 0] = 40 * (ramp if sign > 0 else 1 - ramp)
    K = K.to(torch.bfloat16)
    V = _rand((2, H, n, 128), 171)
    Q = _rand((2, 4 * H, t, 128), 172, 0.2).float()
    Q[..., 0] += 3
    Q = Q.to(torch.bfloat16)
    desc = cur.make_desc(K, V, 1, q_heads=4 * H)
    lse = torch.zeros((2, 4 * H, t), device=DEV)
    for scale, window in ((1.0, 5000), (1.0, 700), (0.0, 700)):
        O, ws = cur.curdkv_attention_window(Q, K, V, desc, window, num_sink=3, scale=scale, lse=lse)
        assert cur.curdkv_device_status(ws) == 0
        _check(O, lse, Q, K, V, [n, n], [t, t], window, 3, scale, heads=[0, 31], what=f"{sign} {scale} {window}")


@pytest.mark.parametrize("t", [1, 300])
def test_heads_and_sequences_that_share_their_rows(t):
    """K and V broadcast over sequences and KV heads (strides of zero), as beams over one prompt have them."""
    B, H, group, n = 3, 8, 4, 400
    K, V = (_rand((1, 1, n, 128), 180 + i).expand(B, H, n, 128) for i in range(2))
    _run(B, H, group, n, t, 150, 4, K=K, V=V, seed=182, heads=HEADS)


def test_prompts_replayed_and_beside_another_call():
    """A captured call replayed with other rows and lengths, while another prompt runs on a second stream with a workspace of
    its own."""
    B, H, group, n, t, window, sink = 3, 8, 4, 1500, 300, 300, 4
    K, V = _rand((B, H, n, 128), 190), _rand((B, H, n, 128), 191)
    lens = torch.tensor([1400, 900, 10], dtype=torch.int32, device=DEV)
    desc = cur.make_desc(K, V, 1, q_heads=H * group, seqlens=lens)
    Q = _rand((B, H * group, t, 128), 192)
    O, lse = torch.zeros_like(Q), torch.zeros(Q.shape[:3], device=DEV)
    ws = cur.attention_window_workspace(desc, t)
    call = lambda: cur.curdkv_attention_window(Q, K, V, desc, window, num_sink=sink, scale=0.1, O=O, lse=lse, workspace=ws)  # noqa: E731
    call()
    other = (_rand((2, H, 800, 128), 193), _rand((2, H, 800, 128), 194))
    od = cur.make_desc(*other, 1, q_heads=H * group)
    oq = _rand((2, H * group, 700, 128), 195)
    oo, ows = torch.zeros_like(oq), cur.attention_window_workspace(od, 700)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side = torch.cuda.Stream()
    for i in range(3):
        K.copy_(_rand(K.shape, 200 + i))
        Q.copy_(_rand(Q.shape, 210 + i))
        now = [1400 + i, 900 - 300 * i, 10 + i]
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        oo.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            cur.curdkv_attention_window(oq, *other, od, 100, scale=0.1, O=oo, workspace=ows)
        graph.replay()
        torch.cuda.current_stream().wait_stream(side)
        _check(O, lse, Q, K, V, now, [t] * B, window, sink, float(np.float32(0.1)), heads=[0, 31])
        _check(oo, None, oq, *other, [800, 800], [700, 700], 100, 0, float(np.float32(0.1)), heads=[5])
    assert cur.curdkv_device_status(ws) == 0 and cur.curdkv_device_status(ows) == 0


@pytest.mark.parametrize("B,H,group,t", [(2, 2, 2, 1), (2, 2, 2, 7), (3, 8, 4, 250)])
@pytest.mark.parametrize("window,sink", [(100, 4), (0, 5), (0, 0), (33, 130), (300, 0)])
def test_rows_that_no_query_sees_hold_anything(B, H, group, t, window, sink):
    """Old rows that have left the first query's window, as a cache that drops them leaves them."""
    n = 700
    K, V = _rand((B, H, n, 128), 220), _rand((B, H, n, 128), 221)
    lens = [700, 555, 600][:B]
    for b, m in enumerate(lens):
        unseen = torch.from_numpy(~orc.window_mask(m, t, window, sink).any(0)).to(DEV)
        K[b, :, :m][:, unseen] = float("nan")
        V[b, :, :m][:, unseen] = float("inf")
        K[b, :, m:] = float("inf")
        V[b, :, m:] = float("nan")
    Q = _rand((B, H * group, t, 128), 222)
    desc = cur.make_desc(K, V, 1, q_heads=H * group, seqlens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    lse = torch.zeros(Q.shape[:3], device=DEV)
    O, ws = cur.curdkv_attention_window(Q, K, V, desc, window, num_sink=sink, scale=0.1, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    K, V = (torch.nan_to_num(x, 0.0, 0.0, 0.0) for x in (K, V))          # (rows the oracle gives no weight)
    _check(O, lse, Q, K, V, lens, [t] * B, window, sink, float(np.float32(0.1)), heads=[0, H * group - 1])


def test_prompts_without_queries_in_some_sequences():
    _run(4, 8, 4, 400, 300, 90, 4, lens=[400, 400, 0, 1], q_lens=[0, 300, 300, 0], seed=230, heads=HEADS)
    _run(3, 8, 4, 400, 300, 90, 4, lens=[400, 400, 300], q_lens=[0, -5, 0], seed=231, heads=HEADS)


@pytest.mark.parametrize("t", [1, 3])
@pytest.mark.parametrize("B,H,n,window", [(1, 1, 9000, 8900), (1, 2, 3001, 2900), (9, 8, 1200, 1000), (18, 8, 700, 500), (40, 8, 300, 90)])
def test_few_tokens_however_the_keys_are_shared_out(B, H, n, window, t):
    """Equal runs over all heads, clusters of eight, four and two CTAs per head, one CTA per head."""
    lens = [n - 7 * b if b % 5 else n for b in range(B)]
    lens[-1] = n if B == 1 else 1
    _run(B, H, 4, n, t, window, 4, lens=lens, q_lens=[min(t, x) for x in lens], seed=240, heads=[0, 4 * H - 1])


@pytest.mark.parametrize("t", [1, 6])
def test_few_tokens_over_equal_runs_replayed_and_beside_another_call(t):
    """One long head, which equal runs and a joining launch take: captured, replayed with other rows and lengths, while another
    such call runs on a second stream with a workspace of its own."""
    n, window, sink = 12000, 11000, 4
    K, V = _rand((1, 1, n, 128), 300), _rand((1, 1, n, 128), 301)
    lens = torch.tensor([n], dtype=torch.int32, device=DEV)
    desc = cur.make_desc(K, V, 1, q_heads=2, seqlens=lens)
    Q = _rand((1, 2, t, 128), 302)
    O, lse = torch.zeros_like(Q), torch.zeros(Q.shape[:3], device=DEV)
    size = cur.attention_window_workspace(desc, t).numel()
    buf = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    buf[:256] = 0
    call = lambda: cur.curdkv_attention_window(Q, K, V, desc, window, num_sink=sink, scale=0.1, O=O, lse=lse, workspace=buf[:size])  # noqa: E731
    before = cur.launch_count()
    call()
    assert cur.launch_count() - before == 2
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side, oq, oo = torch.cuda.Stream(), _rand(Q.shape, 303), torch.zeros_like(Q)
    ows = cur.attention_window_workspace(desc, t)
    for now in (n, 9001, 17, n - 1):
        K.copy_(_rand(K.shape, 310 + now))
        Q.copy_(_rand(Q.shape, 320 + now))
        lens.fill_(now)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            cur.curdkv_attention_window(oq, K, V, desc, n, scale=0.1, O=oo, workspace=ows)
        graph.replay()
        torch.cuda.current_stream().wait_stream(side)
        _check(O, lse, Q, K, V, [now], [t], window, sink, float(np.float32(0.1)), what=f"{now}")
        _check(oo, None, oq, K, V, [now], [t], n, 0, float(np.float32(0.1)), what=f"{now} beside")
    assert torch.all(buf[size:] == 0xA5) and cur.curdkv_device_status(buf) == 0 and cur.curdkv_device_status(ows) == 0


@pytest.mark.parametrize("n", [1, 100, 5000, 40000])
@pytest.mark.parametrize("q_rows", [1, 5, 64, 200])
def test_the_stated_workspace_is_enough_for_every_window(n, q_rows):
    """The size call knows no window: what it says serves any, plans for the window's keys included."""
    K = _rand((2, 2, n, 128), 330)
    desc = cur.make_desc(K, K, 1, q_heads=4)
    size = cur.attention_window_workspace(desc, q_rows).numel()
    Q = _rand((2, 4, q_rows, 128), 331)
    buf = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    buf[:256] = 0
    for window, sink in ((0, 0), (1, 0), (0, 4), (17, 4), (1000, 4), (4096, 0), (n, 0), (2 ** 31 - 1, 2 ** 31 - 1)):
        lse = torch.zeros(Q.shape[:3], device=DEV)
        O, _ = cur.curdkv_attention_window(Q, K, K, desc, window, num_sink=sink, scale=0.1, lse=lse, workspace=buf[:size])
        assert torch.all(buf[size:] == 0xA5) and cur.curdkv_device_status(buf) == 0
        t = min(q_rows, n)                                   # queries before the first row see nothing
        assert not O[:, :, :q_rows - t].any()
        _check(O[:, :, q_rows - t:], lse[:, :, q_rows - t:], Q[:, :, q_rows - t:], K, K, [n, n], [t, t], window, sink,
               float(np.float32(0.1)), heads=[0, 3], what=f"{window} {sink}")
        with pytest.raises(cur.CurdkvError, match="status 3"):
            cur.curdkv_attention_window(Q, K, K, desc, window, num_sink=sink, scale=0.1, workspace=buf[: size - 1])


@pytest.mark.parametrize("t", [1, 3])
def test_few_tokens_over_more_heads_than_a_line_holds(t):
    B = 1100
    lens = [(37 * b) % 61 for b in range(B)]
    Q, K, V, desc, O = _run(B, 8, 1, 60, t, 20, 4, lens=lens, q_lens=[min(t, x) for x in lens], seed=340, heads=[0, 7])
    assert cur.attention_window_workspace(desc, t).numel() == 256


@pytest.mark.parametrize("B,H,t", [(1, 2, 1), (1, 2, 5), (3, 8, 250)])
@pytest.mark.parametrize("scale", [0.0, 1e-32, 1e-36])
def test_tiny_scales_with_large_products(B, H, t, scale):
    """A scale of 0 averages whatever the products are (1e32 here), and tiny ones are not taken for larger ones."""
    K, Q = _rand((B, H, 400, 128), 350, 1e16), _rand((B, 2 * H, t, 128), 351, 1e15)
    V = _rand((B, H, 400, 128), 352)
    desc = cur.make_desc(K, V, 1, q_heads=2 * H)
    lse = torch.zeros(Q.shape[:3], device=DEV)
    O, ws = cur.curdkv_attention_window(Q, K, V, desc, 300, num_sink=4, scale=scale, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    _check(O, lse, Q, K, V, [400] * B, [t] * B, 300, 4, float(np.float32(scale)), heads=[0, 2 * H - 1])


@pytest.mark.parametrize("B,H,group,t", [(1, 2, 4, 1), (2, 2, 4, 5), (3, 8, 4, 250)])
def test_non_finite_queries_stay_in_their_row(B, H, group, t):
    Q, K, V, desc, O = _run(B, H, group, 700, t, 300, 4, seed=360, heads=[0, H * group - 1])
    bad = Q.clone()
    bad[0, 0, t // 2, 5], bad[B - 1, H * group - 1, 0, 77] = float("nan"), float("nan")
    got, ws = cur.curdkv_attention_window(bad, K, V, desc, 300, num_sink=4, scale=128 ** -0.5)
    assert cur.curdkv_device_status(ws) == 0
    rest = torch.ones(Q.shape[:3], dtype=torch.bool, device=DEV)
    rest[0, 0, t // 2] = rest[B - 1, H * group - 1, 0] = False
    assert torch.isnan(got[~rest]).all()
    _check(torch.where(rest[..., None], got, O), None, Q, K, V, [700] * B, [t] * B, 300, 4, float(np.float32(128 ** -0.5)),
           heads=[0, 1, H * group - 1])


@pytest.mark.parametrize("B,H,t", [(1, 2, 1), (1, 2, 5), (3, 8, 250)])
def test_a_cache_without_rows(B, H, t):
    K, Q = torch.zeros((B, H, 0, 128), dtype=torch.bfloat16, device=DEV), _rand((B, 2 * H, t, 128), 370)
    lse = torch.zeros(Q.shape[:3], device=DEV)
    O, ws = cur.curdkv_attention_window(Q, K, K, cur.make_desc(K, K, 1, q_heads=2 * H), 100, num_sink=4, scale=0.1, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    assert not O.any() and torch.all(lse == -float("inf"))
