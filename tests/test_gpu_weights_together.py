"""Attention-weight calls beside one another, on the GPU: forms that only many heads reach, one workspace in several captured
graphs, calls of different sizes in turn over one workspace.  Needs a B200."""
import pytest
import torch

from paper_2509_15038_b200 import binding as cur
from tests import test_gpu_scores as scores
from tests import test_gpu_weights as weights

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = weights.SCALE


@pytest.mark.parametrize("B,H,cap,t", [(37, 16, 500, 1), (25, 16, 500, 1), (37, 8, 2600, 1), (9, 8, 4400, 2), (75, 16, 130, 4)])
def test_rounds_of_clusters(B, H, cap, t):
    """More heads than the device holds at a time: whole rounds, a part of one, clusters of several CTAs."""
    held = [max(0, cap - (b * 37) % (cap + 5)) for b in range(B)]
    weights._attend(B, H, 4, t, cap, held, seed=1000 + cap)


@pytest.mark.parametrize("lens_step,n", [(1, 130), (7, 260)])
def test_scores_of_very_many_short_prompts(lens_step, n):
    """More units of work than are taken one at a time, many of them empty."""
    B = 1250
    lens = [(b * lens_step) % (n + 1) for b in range(B)]
    scores._run(B, 8, 1, n, 2, lens=lens, q_lens=[b % 3 for b in range(B)], seed=1100, heads=[0, 7])


def _graph(f):
    f()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f()
    return g


def test_graphs_share_a_workspace():
    """Graphs of different sizes captured over one workspace, replayed in turn: every time the results of a call alone."""
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device=DEV)
    calls = []
    for i, (B, H, group, n, t) in enumerate([(2, 2, 4, 900, 32), (300, 1, 1, 200, 1), (1, 8, 4, 1500, 700)]):
        K, Q = weights._rand((B, H, n, 128), 1200 + i), weights._rand((B, H * group, t, 128), 1210 + i)
        desc, out = cur.make_desc(K, K, 1, q_heads=H * group), torch.zeros((B, H, n), device=DEV)
        calls.append((out, lambda Q=Q, K=K, desc=desc, out=out, w=None: cur.curdkv_attention_scores(Q, K, desc, scale=SCALE, scores=out, workspace=w)))
    for i, (B, H, group, n, t) in enumerate([(1, 8, 4, 1700, 1), (1, 2, 4, 40000, 1), (60, 8, 4, 600, 1), (2, 2, 4, 700, 9)]):
        c, Q = weights._cache(B, H, n, [n] * B, 1220 + i), weights._rand((B, H * group, t, 128), 1230 + i)
        O = torch.zeros_like(Q)
        calls.append((O, lambda Q=Q, c=c, O=O, w=None: cur.curdkv_cache_attention(Q, c, scale=SCALE, O=O, weights=torch.zeros_like(c.raw), workspace=w)))
    for i, (Bp, share, n0, n) in enumerate([(1, 2, 500, 30), (2, 40, 700, 90)]):
        K0, K = weights._rand((Bp, 2, n0, 128), 1240 + i), weights._rand((Bp * share, 2, n, 128), 1250 + i)
        Q = weights._rand((Bp * share, 8, 1, 128), 1260 + i)
        d0, d, O = cur.make_desc(K0, K0, 1, q_heads=8), cur.make_desc(K, K, 1, q_heads=8), torch.zeros_like(Q)
        calls.append((O, lambda Q=Q, K0=K0, K=K, d0=d0, d=d, O=O, w=None: cur.curdkv_attention_prefix(Q, K0, K0, d0, K, K, d, scale=SCALE, O=O, workspace=w)))
    want = []
    for out, f in calls:
        f()
        want.append(out.clone())
    graphs = [_graph(lambda f=f: f(w=ws)) for _, f in calls]
    for order in (range(len(calls)), reversed(range(len(calls))), [0, 0, 3, 1, 5, 1, 4, 2, 8, 3, 7, 6, 2]):
        for out, _ in calls:
            out.fill_(9.0)
        used = set()
        for i in order:
            graphs[i].replay()
            used.add(i)
        torch.cuda.synchronize()
        for i in used:
            assert torch.equal(calls[i][0], want[i]), i
    assert cur.curdkv_device_status(ws) == 0


def test_streams_side_by_side():
    """The three attentions at once on three streams, a workspace each, again and again: the results of each alone."""
    c = weights._cache(3, 8, 1700, [1700, 900, 3], 1300)
    Q = weights._rand((3, 32, 1, 128), 1301)
    K, Qs = weights._rand((3, 8, 1000, 128), 1302), weights._rand((3, 32, 64, 128), 1303)
    desc = cur.make_desc(K, K, 1, q_heads=32)
    K0, Kp, Qp = weights._rand((1, 8, 3000, 128), 1304), weights._rand((24, 8, 100, 128), 1305), weights._rand((24, 32, 1, 128), 1306)
    d0, d = cur.make_desc(K0, K0, 1, q_heads=32), cur.make_desc(Kp, Kp, 1, q_heads=32)

    def calls(ws):
        w = torch.zeros_like(c.raw)
        return [lambda: (cur.curdkv_cache_attention(Q, c, scale=SCALE, weights=w.zero_(), workspace=ws[0]), w)[0][0],
                lambda: cur.curdkv_attention_scores(Qs, K, desc, scale=SCALE, workspace=ws[1])[0],
                lambda: cur.curdkv_attention_prefix(Qp, K0, K0, d0, Kp, Kp, d, scale=SCALE, workspace=ws[2])[0]]

    want = [f() for f in calls([None] * 3)]
    ws = [torch.zeros(16 << 20, dtype=torch.uint8, device=DEV) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    fs = calls(ws)
    torch.cuda.synchronize()
    got = [[] for _ in fs]
    for _ in range(20):
        for s, f, g in zip(streams, fs, got):
            with torch.cuda.stream(s):
                g.append(f())
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, w) for x in g)
    assert all(cur.curdkv_device_status(x) == 0 for x in ws)


def test_one_workspace_for_all_shorter_calls():
    """A workspace of the size for the longest rows, in calls of shorter ones that are cut into more parts: the results of calls with
    one of their own."""
    rows = [1, 127, 129, 2305, 2368, 4736, 4737, 9000]
    K, Q = weights._rand((1, 2, 9000, 128), 1400), weights._rand((1, 8, 32, 128), 1401)
    full = cur.make_desc(K, K, 1, q_heads=8)
    ws_s = cur.attention_scores_workspace(full, 32)
    d0, ws_p = cur.make_desc(K[:, :, :300], K[:, :, :300], 1), None
    for n in reversed(rows):
        x = K[:, :, :n]
        d = cur.make_desc(x, x, 1, q_heads=8)
        want = cur.curdkv_attention_scores(Q, x, d, scale=SCALE)[0]
        assert torch.equal(cur.curdkv_attention_scores(Q, x, d, scale=SCALE, workspace=ws_s)[0], want)
        for t in (1, 3):
            q = Q[:, :, :t]
            if ws_p is None:
                ws_p = cur.attention_prefix_workspace(d0, d, 3)
                ws_0 = cur.attention_prefix_workspace(cur.make_desc(x, x, 1), cur.make_desc(x, x, 1, q_heads=8), 3)
            want = cur.curdkv_attention_prefix(q, K[:, :, :300], K[:, :, :300], d0, x, x, d, scale=SCALE)[0]
            assert torch.equal(cur.curdkv_attention_prefix(q, K[:, :, :300], K[:, :, :300], d0, x, x, d, scale=SCALE, workspace=ws_p)[0], want)
            want = cur.curdkv_attention_prefix(q, x, x, cur.make_desc(x, x, 1), x, x, d, scale=SCALE)[0]
            assert torch.equal(cur.curdkv_attention_prefix(q, x, x, cur.make_desc(x, x, 1), x, x, d, scale=SCALE, workspace=ws_0)[0], want)
    c = weights._cache(1, 2, 9000, [9000], 1402)
    ws_c = cur.cache_attention_workspace(c, 8, 3)
    for n in rows:
        short = cur.DeviceCache.of(*(x[:, :, :n].contiguous() for x in (c.K, c.V, c.raw, c.pos)), torch.full_like(c.count, n), c.total)
        for t in (1, 3):
            w, v = torch.zeros_like(short.raw), torch.zeros_like(short.raw)
            want = cur.curdkv_cache_attention(Q[:, :, :t], short, scale=SCALE, weights=w)[0]
            assert torch.equal(cur.curdkv_cache_attention(Q[:, :, :t], short, scale=SCALE, weights=v, workspace=ws_c)[0], want)
            assert torch.equal(v, w)
    for ws in (ws_s, ws_p, ws_0, ws_c):
        assert cur.curdkv_device_status(ws) == 0


@pytest.mark.parametrize("B,H,group,cap,t", [(1, 2, 4, 300, 1), (1, 8, 4, 1703, 1), (40, 8, 4, 2049, 1), (1, 2, 4, 40001, 1), (2, 2, 8, 700, 5)])
def test_a_workspace_of_what_one_call_uses(B, H, group, cap, t):
    """With weights and without: the same results, and not a byte behind it touched."""
    c, Q = weights._cache(B, H, cap, [cap - b % 3 for b in range(B)], 1500), weights._rand((B, H * group, t, 128), 1501)
    for ask in (True, False):
        w = torch.zeros_like(c.raw) if ask else None
        want = cur.curdkv_cache_attention(Q, c, scale=SCALE, weights=w)[0]
        size = cur.cache_attention_workspace(c, H * group, t, weights=ask).numel()
        assert size <= cur.cache_attention_workspace(c, H * group, t).numel()
        buf = torch.full((size + 4096,), 7, dtype=torch.uint8, device=DEV)
        buf[:256] = 0
        v = torch.zeros_like(c.raw) if ask else None
        got = cur.curdkv_cache_attention(Q, c, scale=SCALE, weights=v, workspace=buf[:size])[0]
        assert torch.equal(got, want) and torch.all(buf[size:] == 7) and cur.curdkv_device_status(buf) == 0
        assert not ask or torch.equal(v, w)


def test_batches_of_none():
    """No sequences: every call answers, with outputs of none."""
    none = cur.DeviceCache(0, 2, 65, 128)
    for t in (1, 8):
        new, Q = torch.zeros((0, 2, t, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((0, 8, t, 128), dtype=torch.bfloat16, device=DEV)
        cur.curdkv_cache_push(none, new, new, 64, cur.cache_workspace(0, 2, t, 65, 64), num_sink=4, window=8)
        assert cur.curdkv_cache_attention(Q, none, scale=SCALE, weights=none.raw)[0].shape == Q.shape
        K = torch.zeros((0, 2, 50, 128), dtype=torch.bfloat16, device=DEV)
        desc = cur.make_desc(K, K, 1, q_heads=8)
        assert cur.curdkv_attention_scores(Q, K, desc, scale=SCALE)[0].shape == (0, 2, 50)
        for K0 in (K, weights._rand((1, 2, 50, 128), 1600)):
            assert cur.curdkv_attention_prefix(Q, K0, K0, cur.make_desc(K0, K0, 1), K, K, desc, scale=SCALE)[0].shape == Q.shape
