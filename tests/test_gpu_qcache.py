"""The 4-bit cache on the GPU (store, append, read, attention) against the float64 oracle.  Needs a B200."""
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
    x = torch.randn(shape, generator=g, device=DEV) * gain
    x[..., 3] *= 10.0
    return x.to(torch.bfloat16)


def _f64(t):
    return synth.u16_to_f64(synth.to_u16(t))


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def _check_rows(cache, p_rows, wants):
    """Codes and metas of cache rows p_rows (flat indices) bit for bit those of the rows `wants` = (K, V) float64."""
    for which, codes, meta, want in (("K", cache.K_codes, cache.K_meta, wants[0]), ("V", cache.V_codes, cache.V_meta, wants[1])):
        c, _, _, m = orc.quantise(want)
        got_c = codes.reshape(-1, 64).cpu().numpy()[p_rows]
        got_m = _bits(meta.reshape(-1, 8)).reshape(-1, 4, 2)[p_rows]
        # -0.0 and 0.0 are the same zero point
        gm, wm = got_m.copy(), m.copy()
        gm[gm == 0x8000] = 0
        wm[wm == 0x8000] = 0
        assert np.array_equal(gm, wm), which
        assert np.array_equal(got_c, orc.pack(c, which)), which


@pytest.mark.parametrize("B,H,n", [(1, 1, 1), (2, 3, 37), (1, 2, 1000), (3, 8, 130)])
@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_store_all_rows_bit_exact(B, H, n, layout):
    if layout == "bhnd":
        K, V = _rand((B, H, n, 128), 1), _rand((B, H, n, 128), 2, 0.01)
    else:                                            # heads inside the token axis: strided rows
        K, V = (_rand((B, n, H, 128), s).transpose(1, 2) for s in (3, 4))
    cache = cur.QuantCache(B, H, n + 5)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1), workspace=ws)
    assert cur.curdkv_device_status(ws) == 0
    assert cache.count.tolist() == [n] * (B * H)
    rows = np.concatenate([np.arange(n) + p * (n + 5) for p in range(B * H)])
    _check_rows(cache, rows, (_f64(K).reshape(-1, 128), _f64(V).reshape(-1, 128)))
    # the rows behind are as they were
    rest = np.setdiff1d(np.arange(B * H * (n + 5)), rows)
    assert not cache.K_codes.view(-1, 64).cpu().numpy()[rest].any()
    # and back: the value rounded to bf16 once (fma in fp32, then bf16: at most a half step of bf16 and 2^-24 of its parts)
    Ko, Vo = cur.curdkv_qcache_read(cache)
    for out, codes, meta, which in ((Ko, cache.K_codes, cache.K_meta, "K"), (Vo, cache.V_codes, cache.V_meta, "V")):
        val, part = orc.unpack(codes.cpu().numpy().reshape(-1, 64)[rows], _bits(meta.reshape(-1, 8))[rows], which)
        got = _f64(out).reshape(-1, 128)[rows]
        assert np.all(np.abs(got - val) <= 2.0 ** -8 * np.abs(val) + 2.0 ** -23 * part)


def test_store_hard_groups_bit_exact():
    """Ties, constant groups, tiny and huge ranges, a tiny value beside a large zero point, signed zeros."""
    rows = []
    base = np.zeros(128)
    rows.append(base.copy())                                             # all zero: scale 0
    rows.append(np.full(128, -2.5))                                      # constant: scale 0, zero -2.5
    r = base.copy(); r[0::32] = -1.40625; r[1::32] = 1.40625             # scale 0.1875 exactly; zeros fall on the tie 7.5
    rows.append(r)
    r = r.copy(); r[2::32] = 1e-10; r[3::32] = -1e-10                    # beside that tie on either side
    rows.append(r)
    r = np.tile(np.arange(32) * 0.5, 4); rows.append(r)                  # many ties: steps of half a code
    r = np.tile(np.arange(32) * 2.0 ** -130, 4); rows.append(r)          # subnormal scale
    r = np.tile(np.arange(32) * 2.0 ** 120, 4); rows.append(r)           # huge
    r = base.copy(); r[5] = 2.0 ** -133; rows.append(r)                  # smallest subnormal bf16
    r = base.copy(); r[7] = -0.0; r[40] = 1.0; rows.append(r)
    x = np.stack(rows)
    t = torch.tensor(x, dtype=torch.float64).to(torch.bfloat16)
    t = torch.cat([t, (torch.randn(300, 128, generator=torch.Generator().manual_seed(0)) + 100).to(torch.bfloat16)])
    K = t.view(1, 1, -1, 128).to(DEV)
    V = -K
    cache = cur.QuantCache(1, 1, K.shape[2])
    cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1))
    _check_rows(cache, np.arange(K.shape[2]), (_f64(K)[0, 0], _f64(V)[0, 0]))


def test_store_nonfinite_group_stays_inside_its_group():
    K = _rand((1, 1, 8, 128), 5)
    K[0, 0, 1, 5] = float("nan")
    K[0, 0, 2, 40] = float("inf")
    K[0, 0, 3, 100] = -float("inf")
    K[0, 0, 4, 70], K[0, 0, 4, 71] = 3e38, -3e38                         # a range beyond fp32
    cache = cur.QuantCache(1, 1, 8)
    cur.curdkv_qcache_store(cache, K, K, cur.make_desc(K, K, 1))
    _check_rows(cache, np.arange(8), (_f64(K)[0, 0], _f64(K)[0, 0]))
    for out in cur.curdkv_qcache_read(cache):
        got = torch.isnan(out[0, 0]).view(8, 4, 32).cpu()
        want = torch.zeros(8, 4, 32, dtype=torch.bool)
        want[1, 0] = want[2, 1] = want[3, 3] = want[4, 2] = True
        assert torch.equal(got, want)


@pytest.mark.parametrize("adaptive", [False, True])
def test_store_of_a_selection(adaptive):
    """The rows curdkv_select names, fixed and packed, equal the gathered rows quantised."""
    B, H, n, k = 2, 4, 700, 90
    w = synth.shrink(synth.CONFIGS["cfg2"], layers=1, batch=B, n_max=n, kv_heads=H, q_heads=H)
    K, V, _ = synth.make_kv(w, DEV)
    lens = torch.tensor([700, 50], dtype=torch.int32, device=DEV)        # the second keeps all its 50 rows
    desc = cur.make_desc(K, V, 32, seqlens=lens)
    ws = cur.alloc_workspace(desc, k, adaptive)
    G = torch.as_tensor(synth.make_G(128, 32, seed=0), device=DEV)
    scores, _ = cur.curdkv_score(K, V, G, desc, ws)
    idx, cnt, off = cur.curdkv_select(scores, desc, k, num_sink=4, window=16, adaptive=adaptive, workspace=ws)
    if adaptive:
        cache = cur.QuantCache(B, H, idx.numel(), row_start=off)
    else:
        cache = cur.QuantCache(B, H, k + 3)
    cur.curdkv_qcache_store(cache, K, V, desc, idx, cnt, off, packed=adaptive, workspace=ws)
    assert cur.curdkv_device_status(ws) == 0
    assert torch.equal(cache.count, cnt.view(-1))
    gi, gc, go = idx.cpu().numpy().reshape(-1) if adaptive else idx.cpu().numpy(), cnt.cpu().numpy(), off.cpu().numpy()
    rows, wants = [], [[], []]
    Kf, Vf = _f64(K), _f64(V)
    for p in range(B * H):
        b, h = divmod(p, H)
        c = gc[b, h]
        kept = gi[go[p]: go[p] + c] if adaptive else gi[b, h, :c]
        rows.append((go[p] if adaptive else p * (k + 3)) + np.arange(c))
        wants[0].append(Kf[b, h][kept])
        wants[1].append(Vf[b, h][kept])
    _check_rows(cache, np.concatenate(rows), [np.concatenate(x) for x in wants])


def test_store_flags_bad_indices_and_overflow():
    K, V = _rand((1, 2, 64, 128), 6), _rand((1, 2, 64, 128), 7)
    desc = cur.make_desc(K, V, 1, seqlens=torch.tensor([40], dtype=torch.int32, device=DEV))
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    idx = torch.tensor([[0, 39, 40, -1], [1, 2, 1 << 30, 5]], dtype=torch.int32, device=DEV).view(1, 2, 4)
    cnt = torch.tensor([4, 4], dtype=torch.int32, device=DEV)
    cache = cur.QuantCache(1, 2, 4)
    cache.K_codes.fill_(0xEE)
    cur.curdkv_qcache_store(cache, K, V, desc, idx, cnt, workspace=ws)
    assert cur.curdkv_device_status(ws) == cur.DEV_BAD_INDEX
    Ko, _ = cur.curdkv_qcache_read(cache)
    assert not Ko[0, 0, 2:].any() and not Ko[0, 1, 2].any()              # rows of zeros, not stale ones
    assert cache.count.tolist() == [4, 4]
    # a head with less room than its list: cut and flagged, the neighbour's rows untouched
    ws.zero_()
    small = cur.QuantCache(1, 2, 3)
    cur.curdkv_qcache_store(small, K, V, desc, idx.clamp(0, 39), cnt, workspace=ws)
    assert cur.curdkv_device_status(ws) == cur.DEV_CACHE_FULL
    assert small.count.tolist() == [3, 3]
    _check_rows(small, np.arange(6), (np.concatenate([_f64(K)[0, 0][[0, 39, 39]], _f64(K)[0, 1][[1, 2, 39]]]),
                                      np.concatenate([_f64(V)[0, 0][[0, 39, 39]], _f64(V)[0, 1][[1, 2, 39]]])))
    # a count beyond its list
    ws.zero_()
    cur.curdkv_qcache_store(cache, K, V, desc, idx.clamp(0, 39), cnt + 3, workspace=ws)
    assert cur.curdkv_device_status(ws) & cur.DEV_BAD_INDEX and cache.count.tolist() == [4, 4]


@pytest.mark.parametrize("steps", [[1] * 5, [64, 65, 1], [200]])
@pytest.mark.parametrize("packed", [False, True])
def test_append_equals_store(steps, packed):
    B, H, total = 2, 3, sum(steps)
    K, V = _rand((B, H, total, 128), 8), _rand((B, H, total, 128), 9)
    start = torch.arange(B * H + 1, dtype=torch.int32, device=DEV) * total if packed else None
    mk = lambda: cur.QuantCache(B, H, B * H * total if packed else total, row_start=start)  # noqa: E731
    whole, grown = mk(), mk()
    cur.curdkv_qcache_store(whole, K, V, cur.make_desc(K, V, 1))
    at = 0
    for t in steps:
        cur.curdkv_qcache_append(grown, K[:, :, at:at + t], V[:, :, at:at + t])
        at += t
        assert grown.count.tolist() == [at] * (B * H)
    for x in ("K_codes", "V_codes"):
        assert torch.equal(getattr(whole, x), getattr(grown, x))
    for x in ("K_meta", "V_meta"):
        assert torch.equal(getattr(whole, x).view(torch.int16), getattr(grown, x).view(torch.int16))


@pytest.mark.parametrize("t", [5, 70])
def test_append_ragged_and_full(t):
    B, H, cap = 3, 2, 80
    K, V = _rand((B, H, t, 128), 10), _rand((B, H, t, 128), 11)
    cache = cur.QuantCache(B, H, cap)
    cache.count.copy_(torch.tensor([0, 0, 40, 40, 78, 78], dtype=torch.int32))
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    cur.curdkv_qcache_append(cache, K, V, t_new=torch.tensor([0, t - 1, t], dtype=torch.int32, device=DEV), workspace=ws)
    fit = [0, min(t - 1, 40), 2]
    full = cur.DEV_CACHE_FULL
    assert cur.curdkv_device_status(ws) == full
    assert cache.count.tolist() == [0, 0, 40 + fit[1], 40 + fit[1], 80, 80]
    rows = [p * cap + h0 + np.arange(f) for p, (h0, f) in enumerate([(0, 0), (0, 0), (40, fit[1]), (40, fit[1]), (78, 2), (78, 2)])]
    pick = lambda X: np.concatenate([_f64(X)[p // H, p % H][: len(r)] for p, r in enumerate(rows)])  # noqa: E731
    _check_rows(cache, np.concatenate(rows), (pick(K), pick(V)))
    live = np.zeros(B * H * cap, dtype=bool)
    live[np.concatenate(rows)] = True
    assert not cache.V_codes.view(-1, 64).cpu().numpy()[~live].any()


def test_read_named_slots():
    K, V = _rand((2, 2, 30, 128), 12), _rand((2, 2, 30, 128), 13)
    cache = cur.QuantCache(2, 2, 32)
    cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1))
    idx = torch.tensor([[0, 29, -1], [5, 5, 30], [1, 2, 3], [-1, -1, 7]], dtype=torch.int32, device=DEV).view(2, 2, 3)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    full_k, full_v = cur.curdkv_qcache_read(cache)
    out = torch.full((2, 2, 3, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    Ko, Vo = cur.curdkv_qcache_read(cache, idx, K_out=out.clone(), V_out=out.clone(), workspace=ws)
    assert cur.curdkv_device_status(ws) == cur.DEV_BAD_INDEX             # slot 30 of a head that holds 30
    for got, full in ((Ko, full_k), (Vo, full_v)):
        for p, row in enumerate(idx.view(4, 3).tolist()):
            for i, j in enumerate(row):
                want = full.view(4, 32, 128)[p, j] if 0 <= j < 30 else out[0, 0, 0]
                assert torch.equal(got.view(4, 3, 128)[p, i], want)


def _check_attention(O, lse, Q, cache, counts, starts, scale, what=""):
    """Against the oracle on the rows the codes stand for.  Error budget per output: the weights are rounded to fp16 twice
    (half a step is 2^-11 each: once alone, once times the scale), the zero points meet only the first; logits carry fp32
    sums of 128 products (and the zero points' part rounded to 24 bits), say 2^-20 of the sum of magnitudes, which enters
    every weight twice (numerator and denominator); 2^-21 for the exponential and the fp32 sums over the keys per
    addition chain; O is rounded to bf16 once (2^-8)."""
    got, Qf = _f64(O), _f64(Q)
    kc, vc = cache.K_codes.cpu().numpy().reshape(-1, 64), cache.V_codes.cpu().numpy().reshape(-1, 64)
    km, vm = _bits(cache.K_meta.reshape(-1, 8)), _bits(cache.V_meta.reshape(-1, 8))
    B, H = Q.shape[:2]
    for p, c in enumerate(counts):
        b, h = divmod(p, H)
        rows = slice(starts[p], starts[p] + c)
        k, kp = orc.unpack(kc[rows], km[rows], "K")
        v, vp = orc.unpack(vc[rows], vm[rows], "V")
        q = Qf[b, h]
        want, want_lse, w = orc.attend(q, k, v, np.ones((q.shape[0], c), dtype=bool), scale)
        if c == 0:
            assert not got[b, h].any() and np.all(np.isneginf(lse[b, h].cpu().numpy()))
            continue
        d = 2.0 ** -20 * scale * (np.abs(q) @ kp.T).max(-1)              # logit error, natural units
        rel = 2.0 ** -10 + 2 * d + 2.0 ** -18
        tol = 2.0 ** -8 * np.abs(want) + rel[:, None] * (w @ vp) * (1 + 2.0 ** -7) + 1e-38
        err = np.abs(got[b, h] - want)
        assert np.all(err <= tol), f"{what} p={p} count={c}: {np.max(err / tol):.3g} of the tolerance"
        assert np.all(np.abs(lse[b, h].cpu().numpy() - want_lse) <= d + 2.0 ** -20 * (1 + np.abs(want_lse)) + 2.0 ** -18)


def _random_cache(B, H, cap, counts, seed, packed=False, k_gain=1.0, v_gain=1.0, v_shift=0.0):
    n = max(max(counts), 1)
    K = _rand((B, H, n, 128), seed, k_gain)
    V = (_rand((B, H, n, 128), seed + 1, v_gain).float() + v_shift).to(torch.bfloat16)
    if packed:
        starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        cache = cur.QuantCache(B, H, max(int(starts[-1]), 1), row_start=torch.as_tensor(starts, device=DEV))
    else:
        starts = np.arange(B * H) * cap
        cache = cur.QuantCache(B, H, cap)
    idx = torch.arange(n, dtype=torch.int32, device=DEV).expand(B, H, n).contiguous()
    cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1), idx,
                            torch.tensor(counts, dtype=torch.int32, device=DEV))
    return cache, starts


COUNTS = [0, 1, 15, 16, 17, 31, 32, 33, 255, 256, 257, 300, 700, 1000, 1023, 2049]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("q_rows", [1, 4, 8, 9, 16, 37])
def test_attention_matches_oracle(packed, q_rows):
    B, H = 2, 8
    cache, starts = _random_cache(B, H, 2100, COUNTS, 20, packed)
    Q = _rand((B, H, q_rows, 128), 30)
    lse = torch.zeros((B, H, q_rows), device=DEV)
    scale = 128 ** -0.5
    O, ws = cur.curdkv_qcache_attention(Q, cache, scale=scale, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    _check_attention(O, lse, Q, cache, COUNTS, starts, scale, f"packed={packed} q_rows={q_rows}")
    again, _ = cur.curdkv_qcache_attention(Q, cache, scale=scale, workspace=ws)
    assert torch.equal(O, again)                                         # no order of arrival decides anything


@pytest.mark.parametrize("k_gain,v_gain,v_shift,q_gain", [
    (1.0, 1e4, 0.0, 1.0), (1.0, 1e-6, 0.0, 1.0), (1e3, 1.0, 0.0, 1e-3), (1e-4, 1.0, 50.0, 1e4), (1.0, 1e30, 0.0, 1.0),
    (1e-20, 1e-30, 0.0, 1e20), (5.0, 1.0, 0.0, 3.0)])
def test_attention_over_the_range_of_bf16(k_gain, v_gain, v_shift, q_gain):
    """Values far from 1 on every side, values that sit on an offset, and logits of hundreds."""
    counts = [500, 3]
    cache, starts = _random_cache(1, 2, 512, counts, 40, k_gain=k_gain, v_gain=v_gain, v_shift=v_shift)
    Q = _rand((1, 2, 5, 128), 41, q_gain)
    lse = torch.zeros((1, 2, 5), device=DEV)
    O, _ = cur.curdkv_qcache_attention(Q, cache, scale=0.0884, lse=lse)
    _check_attention(O, lse, Q, cache, counts, starts, float(np.float32(0.0884)), f"{k_gain} {v_gain} {v_shift} {q_gain}")


def test_attention_values_that_grow_along_the_cache():
    """Value rows whose scale grows by 2^40 along the sequence, and logits that grow with them: both running references move
    many times."""
    n = 900
    ramp = torch.linspace(0, 1, n, device=DEV)[:, None]
    K = _rand((1, 1, n, 128), 50, 0.2).float()
    K[0, 0, :, 0] = 40 * ramp[:, 0]
    V = _rand((1, 1, n, 128), 51).float() * torch.exp2(40 * (ramp - 0.5))
    K, V = K.to(torch.bfloat16), V.to(torch.bfloat16)
    cache = cur.QuantCache(1, 1, n)
    cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1))
    Q = _rand((1, 1, 4, 128), 52, 0.2)
    Q[..., 0] = torch.tensor([1.0, -1.0, 0.0, 2.0], device=DEV)
    lse = torch.zeros((1, 1, 4), device=DEV)
    O, _ = cur.curdkv_qcache_attention(Q, cache, scale=1.0, lse=lse)
    _check_attention(O, lse, Q, cache, [n], [0], 1.0)


def test_attention_scale_zero_strides_and_stale_rows():
    """Scale 0 averages the rows; strided Q and O; whatever lies behind the held rows (NaN metas) has no part."""
    cache, starts = _random_cache(2, 2, 64, [40, 1, 64, 0], 60)
    cache.K_meta.view(4, 64, 4, 2)[0, 40:] = float("nan")
    cache.V_meta.view(4, 64, 4, 2)[0, 40:] = float("nan")
    cache.V_meta.view(4, 64, 4, 2)[3] = float("inf")
    wide = _rand((2, 6, 2, 192), 61)
    Q = wide[..., :128].transpose(1, 2)                                  # [2, 2, 6, 128] with rows 384 apart
    buf = torch.full((2, 6, 2, 136), 9.0, dtype=torch.bfloat16, device=DEV)
    O = buf[..., 8:].transpose(1, 2)
    lse = torch.zeros((2, 2, 6), device=DEV)
    for scale in (0.0, 0.1):
        cur.curdkv_qcache_attention(Q, cache, scale=scale, O=O, lse=lse)
        _check_attention(O, lse, Q, cache, [40, 1, 64, 0], starts, float(np.float32(scale)))
    assert torch.all(buf[..., :8] == 9.0)


def test_attention_flags_a_count_out_of_range():
    cache, starts = _random_cache(1, 2, 32, [32, 32], 70)
    cache.count.copy_(torch.tensor([40, -3], dtype=torch.int32))
    Q = _rand((1, 2, 1, 128), 71)
    lse = torch.zeros((1, 2, 1), device=DEV)
    O, ws = cur.curdkv_qcache_attention(Q, cache, scale=0.1, lse=lse)
    assert cur.curdkv_device_status(ws) == cur.DEV_BAD_INDEX
    _check_attention(O, lse, Q, cache, [32, 0], starts, float(np.float32(0.1)))


def test_generation_together_in_a_graph():
    """Prompt compressed into a packed 4-bit cache with slack, then generation steps (append, attend) captured once and
    replayed with fresh rows; the cache and every output as the oracle has them."""
    B, H, group, n, k, steps = 2, 4, 4, 600, 100, 5
    w = synth.shrink(synth.CONFIGS["cfg2"], layers=1, batch=B, n_max=n, kv_heads=H, q_heads=H * group)
    K, V, _ = synth.make_kv(w, DEV)
    G = torch.as_tensor(synth.make_G(128, 32, seed=0), device=DEV)
    desc = cur.make_desc(K, V, 32, q_heads=H * group)
    ws = cur.alloc_workspace(desc, k, True)
    _, _, idx, cnt, off, _, _ = cur.curdkv_compress(K, V, G, desc, k, ws, num_sink=4, window=16, adaptive=True)
    start = off + 8 * torch.arange(B * H + 1, dtype=torch.int32, device=DEV)
    cache = cur.QuantCache(B, H, int(start[-1].item()), row_start=start)
    cur.curdkv_qcache_store(cache, K, V, desc, idx, cnt, off, packed=True, workspace=ws)
    k1, v1 = (torch.zeros((B, H, 1, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q1 = torch.zeros((B, H, group, 128), dtype=torch.bfloat16, device=DEV)
    lse, O = torch.zeros((B, H, group), device=DEV), torch.zeros_like(q1)
    aws = cur.qcache_attention_workspace(cache, group)
    held = cache.count.clone()

    def step():
        cur.curdkv_qcache_append(cache, k1, v1, workspace=aws)
        cur.curdkv_qcache_attention(q1, cache, scale=0.0884, O=O, lse=lse, workspace=aws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    cache.count.copy_(held)
    for i in range(steps):
        k1.copy_(_rand((B, H, 1, 128), 100 + i))
        v1.copy_(_rand((B, H, 1, 128), 200 + i))
        q1.copy_(_rand((B, H, group, 128), 300 + i))
        graph.replay()
        counts = (held + i + 1).tolist()
        assert cache.count.tolist() == counts
        rows = np.asarray([start[p].item() + counts[p] - 1 for p in range(B * H)])
        _check_rows(cache, rows, (_f64(k1).reshape(-1, 128), _f64(v1).reshape(-1, 128)))
        _check_attention(O, lse, q1, cache, counts, start.tolist(), float(np.float32(0.0884)), f"step {i}")
    assert cur.curdkv_device_status(aws) == 0


def test_long_cache_offsets_pass_32_bits():
    """A cache whose codes lie beyond 4 GB: the last head's rows are its own."""
    H, cap = 9, 1 << 23                                                  # 9 * 2^23 rows * 64 B = 4.8 GB a tensor
    cache = cur.QuantCache(1, H, cap)
    K, V = _rand((1, H, 50, 128), 80), _rand((1, H, 50, 128), 81)
    cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1))
    rows = np.arange(50) + 8 * cap
    small = cur.QuantCache(1, 1, 50)
    small.K_codes.copy_(cache.K_codes[:, 8:, :50])
    small.V_codes.copy_(cache.V_codes[:, 8:, :50])
    small.K_meta.copy_(cache.K_meta[:, 8:, :50])
    small.V_meta.copy_(cache.V_meta[:, 8:, :50])
    small.count.fill_(50)
    _check_rows(small, np.arange(50), (_f64(K)[0, 8], _f64(V)[0, 8]))
    assert rows[-1] * 64 > 1 << 32
    Q = _rand((1, H, 2, 128), 82)
    lse = torch.zeros((1, H, 2), device=DEV)
    O, _ = cur.curdkv_qcache_attention(Q, cache, scale=0.1, lse=lse)
    lse_s = torch.zeros((1, 1, 2), device=DEV)
    cur.curdkv_qcache_attention(Q[:, 8:], small, scale=0.1, lse=lse_s)
    _check_attention(O[:, 8:], lse[:, 8:], Q[:, 8:], small, [50], [0], float(np.float32(0.1)))


def test_store_and_read_the_same_index_more_than_once():
    B, H, n = 2, 2, 90
    K, V = _rand((B, H, n, 128), 400), _rand((B, H, n, 128), 401)
    rng = np.random.default_rng(5)
    idx = torch.from_numpy(np.concatenate([rng.integers(0, n, (B, H, 50)), np.full((B, H, 20), 7)], -1).astype(np.int32)).to(DEV)
    cache = cur.QuantCache(B, H, 80)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    counts = torch.full((B * H,), 70, dtype=torch.int32, device=DEV)
    cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1), idx, counts, workspace=ws)
    take = lambda x: np.take_along_axis(_f64(x), idx.cpu().numpy()[..., None].astype(np.int64), 2).reshape(-1, 128)  # noqa: E731
    _check_rows(cache, np.concatenate([np.arange(70) + 80 * p for p in range(B * H)]), (take(K), take(V)))
    again = torch.tensor([69, 0, 69, -1, 69], dtype=torch.int32, device=DEV).expand(B, H, 5).contiguous()
    k, v = cur.curdkv_qcache_read(cache, again, workspace=ws)
    assert cur.curdkv_device_status(ws) == 0
    assert torch.equal(k[:, :, 0], k[:, :, 2]) and torch.equal(v[:, :, 0], v[:, :, 4]) and not k[:, :, 3].any()


def test_attention_calls_side_by_side():
    """Two streams, two caches, a workspace each: the same results as one after the other; and a call that follows an
    append on its own stream sees the new row."""
    sets = []
    for i in range(2):
        B, H, n = 3, 8, 3000 + 500 * i
        K, V = _rand((B, H, n, 128), 410 + 2 * i), _rand((B, H, n, 128), 411 + 2 * i)
        cache = cur.QuantCache(B, H, n + 40)
        cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1))
        Q = _rand((B, H, 4, 128), 420 + i, 0.3)
        sets.append((cache, Q, torch.empty_like(Q), cur.qcache_attention_workspace(cache, 4), torch.cuda.Stream()))
    run = lambda s: cur.curdkv_qcache_attention(s[1], s[0], scale=0.1, O=s[2], workspace=s[3])  # noqa: E731
    alone = []
    for s in sets:
        run(s)
        alone.append(s[2].clone())
    torch.cuda.synchronize()
    for _ in range(10):
        for s in sets:
            with torch.cuda.stream(s[4]):
                run(s)
    torch.cuda.synchronize()
    for s, want in zip(sets, alone):
        assert torch.equal(s[2], want)
        assert cur.curdkv_device_status(s[3]) == 0
    cache, Q, O, ws, stream = sets[0]
    with torch.cuda.stream(stream):
        big = torch.zeros((3, 8, 1, 128), device=DEV)
        big += 20 * torch.sign(Q[:, :, :1].float())
        big[..., 3] = 0
        new = big.to(torch.bfloat16)
        cur.curdkv_qcache_append(cache, new, torch.full_like(new, 5.0))
        run(sets[0])
    torch.cuda.synchronize()
    # a key of 20 sign(q) has logits of 2 sum |q|, some 60 above every other: its value, 5, is the answer of query 0 to
    # within the weight of the others (exp(-20) each at most) and the roundings to fp16 and bf16
    assert torch.all((O[:, :, 0].float() - 5.0).abs() <= 5.0 * (2.0 ** -8 + 2.0 ** -10))


@pytest.mark.parametrize("q_rows", [1, 5, 16])
@pytest.mark.parametrize("B,H,cap", [(1, 1, 20000), (3, 2, 12000), (1, 2, 3001), (10, 8, 1500), (25, 8, 600), (60, 8, 100)])
def test_attention_however_the_keys_are_shared_out(B, H, cap, q_rows):
    """Equal runs over all heads, clusters of eight, four and two CTAs per head, one CTA per head; heads without rows, with one,
    with one more than a tile."""
    rng = np.random.default_rng(B)
    counts = rng.integers(0, cap + 1, B * H).tolist()
    for p, c in enumerate([cap, 0, 1, 33, cap - 1]):
        if p < B * H:
            counts[p] = c
    cache, starts = _random_cache(B, H, cap, counts, 430)
    Q = _rand((B, H, q_rows, 128), 431)
    lse = torch.zeros((B, H, q_rows), device=DEV)
    O, ws = cur.curdkv_qcache_attention(Q, cache, scale=0.0884, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    _check_attention(O, lse, Q, cache, counts, starts, float(np.float32(0.0884)), f"{(B, H, cap, q_rows)}")
    for _ in range(3):
        again, _ = cur.curdkv_qcache_attention(Q, cache, scale=0.0884, workspace=ws)
        assert torch.equal(O, again)


@pytest.mark.parametrize("cap", [32, 500, 3000])
def test_attention_flags_counts_and_attends_to_the_rest(cap):
    cache, starts = _random_cache(2, 2, cap, [cap] * 4, 440)
    cache.count.copy_(torch.tensor([cap + 1, -3, cap, 5], dtype=torch.int32))
    Q = _rand((2, 2, 3, 128), 441)
    lse = torch.zeros((2, 2, 3), device=DEV)
    O, ws = cur.curdkv_qcache_attention(Q, cache, scale=0.1, lse=lse)
    assert cur.curdkv_device_status(ws) == cur.DEV_BAD_INDEX
    _check_attention(O, lse, Q, cache, [cap, 0, cap, 5], starts, float(np.float32(0.1)))


def _launches(call):
    before = cur.launch_count()
    call()
    return cur.launch_count() - before


@pytest.mark.parametrize("B,H,cap,launches", [(1, 2, 20000, 2), (3, 2, 12000, 2), (1, 8, 1700, 1), (2, 2, 300, 1), (4, 8, 60, 1)])
@pytest.mark.parametrize("bad", ["counts", "row_start"])
def test_attention_flags_bad_heads_in_every_form(B, H, cap, launches, bad):
    """Counts out of range, and row_start that runs backwards or beyond the cache, over equal runs (two launches), clusters
    and single CTAs: flagged, the head bounded or empty, every other head as the oracle has it."""
    P = B * H
    counts = [max(cap - 3 * p, 0) for p in range(P)]
    cache, starts = _random_cache(B, H, cap, counts, 450, packed=bad == "row_start")
    held = list(counts)
    if bad == "counts":
        held[0], held[P - 1] = cap, 0
        cache.count.copy_(torch.tensor([cap + 7] + counts[1:-1] + [-1], dtype=torch.int32))
    else:                                            # the first head ends before it begins, the last one behind the cache
        held[0], held[P - 1] = 0, 0
        cache.row_start[0] = cache.row_start[1] + 1
        cache.row_start[P] = cache.capacity + 1
    Q = _rand((B, H, 4, 128), 451)
    lse = torch.zeros((B, H, 4), device=DEV)
    ws = cur.qcache_attention_workspace(cache, 4)
    call = lambda: cur.curdkv_qcache_attention(Q, cache, scale=0.0884, O=O, lse=lse, workspace=ws)  # noqa: E731
    for _ in range(3):
        O = torch.full_like(Q, 3.0)
        ws[:256].zero_()
        n = _launches(call)
        assert n == launches or bad == "row_start"
        assert cur.curdkv_device_status(ws) == cur.DEV_BAD_INDEX
        _check_attention(O, lse, Q, cache, held, starts, float(np.float32(0.0884)), f"{(B, H, cap, bad)}")


def _check_wild(O, lse, Q, cache, counts, starts, scale, what=""):
    """_check_attention's budget for values of any size, NaN among them: a channel is NaN where the oracle's is and nowhere
    else, and every other channel is held to the budget by its own channel's values.  Below it, what is less than 2^-90 of
    the head's largest value counts as nothing."""
    got, Qf = _f64(O), _f64(Q)
    kc, vc = cache.K_codes.cpu().numpy().reshape(-1, 64), cache.V_codes.cpu().numpy().reshape(-1, 64)
    km, vm = _bits(cache.K_meta.reshape(-1, 8)), _bits(cache.V_meta.reshape(-1, 8))
    H = Q.shape[1]
    for p, c in enumerate(counts):
        b, h = divmod(p, H)
        rows = slice(starts[p], starts[p] + c)
        k, kp = orc.unpack(kc[rows], km[rows], "K")
        v, vp = orc.unpack(vc[rows], vm[rows], "V")
        q = Qf[b, h]
        want, want_lse, w = orc.attend(q, k, v, np.ones((q.shape[0], c), dtype=bool), scale)
        d = 2.0 ** -20 * scale * (np.abs(q) @ kp.T).max(-1)
        rel = 2.0 ** -10 + 2 * d + 2.0 ** -18
        least = 2.0 ** -90 * np.abs(v[np.isfinite(v)]).max(initial=0.0)
        tol = 2.0 ** -8 * np.abs(want) + rel[:, None] * (w @ vp) * (1 + 2.0 ** -7) + least + 1e-38
        nan = np.isnan(want)
        assert np.array_equal(np.isnan(got[b, h]), nan), f"{what} p={p}: NaN in other channels"
        err = np.abs(got[b, h] - want)
        assert np.all((err <= tol)[~nan]), f"{what} p={p} count={c}: {np.max((err / tol)[~nan]):.3g} of the tolerance"
        assert np.all(np.abs(lse[b, h].cpu().numpy() - want_lse) <= d + 2.0 ** -20 * (1 + np.abs(want_lse)) + 2.0 ** -18), what


def _attend_wild(V, seed, q_rows=4, K=None, scale=0.0884, Q=None, what=""):
    H, n = V.shape[1:3]
    K = _rand((1, H, n, 128), seed) if K is None else K
    cache = cur.QuantCache(1, H, n)
    cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1))
    Q = _rand((1, H, q_rows, 128), seed + 1) if Q is None else Q
    lse = torch.zeros((1, H, Q.shape[2]), device=DEV)
    O, ws = cur.curdkv_qcache_attention(Q, cache, scale=scale, lse=lse)
    assert cur.curdkv_device_status(ws) == 0
    _check_wild(O, lse, Q, cache, [n] * H, [h * n for h in range(H)], float(np.float32(scale)), what)


@pytest.mark.parametrize("n", [20, 128, 700, 20000])
@pytest.mark.parametrize("power", [10, 13, 16, 20, 40, 90, -10, -20, -40, -90])
def test_attention_one_group_of_one_row_far_from_the_rest(n, power):
    """One group of one V row 2^power times as large as everything else: the other 96 channels, and the other rows, keep
    their precision.  The row stands at the start, in the middle and at the end of a head."""
    V = _rand((1, 3, n, 128), 500).float()
    for h, row in enumerate((0, n // 2, n - 1)):
        V[0, h, row, 32 * h + 32: 32 * h + 64] *= 2.0 ** power
    _attend_wild(V.to(torch.bfloat16), 501, q_rows=4 if n > 700 else 16, what=f"{n} 2^{power}")


@pytest.mark.parametrize("n", [20, 128, 700, 20000])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_attention_non_finite_values_stay_in_their_group(n, value):
    V = _rand((1, 3, n, 128), 510)
    for h, row in enumerate((0, n // 2, n - 1)):
        V[0, h, row, 32 * h + 5] = value
    _attend_wild(V, 511, what=f"{n} {value}")
    V[0, 0, :, 127] = value                                  # and a whole group of a head
    _attend_wild(V, 512, q_rows=9, what=f"{n} {value}")


@pytest.mark.parametrize("n", [33, 700, 20000])
@pytest.mark.parametrize("kind", ["rows", "groups", "channels", "tiles", "single", "offsets", "sparse"])
def test_attention_values_of_every_size_side_by_side(n, kind):
    """Magnitudes between 2^-40 and 2^40 that differ from row to row, from group to group, from channel to channel, from tile to
    tile; rows of a single channel; groups on a large offset; rows that are mostly zero."""
    g = torch.Generator(device=DEV).manual_seed(520)
    V = torch.randn((1, 2, n, 128), generator=g, device=DEV)
    rand = lambda *shape: 80 * torch.rand(shape, generator=g, device=DEV) - 40  # noqa: E731
    if kind == "rows":
        V = V * torch.exp2(rand(1, 2, n, 1))
    elif kind == "groups":
        V = V * torch.exp2(rand(1, 2, n, 4)).repeat_interleave(32, -1)
    elif kind == "channels":
        V = V * torch.exp2(rand(1, 2, n, 128))
    elif kind == "tiles":
        V = V * torch.exp2(rand(1, 2, (n + 31) // 32, 1)).repeat_interleave(32, 2)[:, :, :n]
    elif kind == "single":
        V = V * 2.0 ** 30 * (torch.rand(V.shape, generator=g, device=DEV) < 0.01)
        V[:, :, 1::2] = torch.randn((1, 2, n // 2, 128), generator=g, device=DEV).abs()
    elif kind == "offsets":
        V = V + torch.exp2(rand(1, 2, n, 4) / 3).repeat_interleave(32, -1)
    else:
        V = torch.where(torch.rand((1, 2, n, 4), generator=g, device=DEV) < 0.2, torch.exp2(rand(1, 2, n, 4)), 0.0).repeat_interleave(32, -1) * V
    _attend_wild(V.to(torch.bfloat16), 521, q_rows=4 if n > 700 else 11, what=f"{n} {kind}")


@pytest.mark.parametrize("n", [96, 700, 20000])
@pytest.mark.parametrize("slope", [30.0, -30.0, 90.0, -90.0])
def test_attention_values_against_the_logits(n, slope):
    """Values that grow or fall by 2^slope along the head while the logits fall or grow by some 2^40: what matters for the
    output is not what matters for the row sum."""
    ramp = torch.linspace(0, 1, n, device=DEV)
    V = _rand((1, 2, n, 128), 530).float() * torch.exp2(slope * (ramp - 0.5))[:, None]
    K = _rand((1, 2, n, 128), 531, 0.2).float()
    K[..., 0] = 28 * ramp
    Q = _rand((1, 2, 4, 128), 532, 0.2)
    Q[..., 0] = torch.tensor([-1.0, 1.0, -0.3, 0.0], device=DEV)
    _attend_wild(V.to(torch.bfloat16), 533, K=K.to(torch.bfloat16), Q=Q, scale=1.0, what=f"{n} {slope}")


@pytest.mark.parametrize("big", [1e6, 1e12, 1e20, 1e30])
@pytest.mark.parametrize("n", [64, 128, 2048, 24000])
def test_attention_rows_of_zeros_beside_large_ones(n, big):
    """Equal weights: the mean of the rows, and log n, whatever half of them is zero or 2^-100 of the others."""
    for small in (0.0, 1e-6):
        V = torch.full((1, 2, n, 128), small, device=DEV)
        V[0, 0, n // 2:] = big
        V[0, 1, : n // 2] = big
        V = V.to(torch.bfloat16)
        cache = cur.QuantCache(1, 2, n)
        K = _rand((1, 2, n, 128), 540)
        cur.curdkv_qcache_store(cache, K, V, cur.make_desc(K, V, 1))
        lse = torch.zeros((1, 2, 3), device=DEV)
        O, _ = cur.curdkv_qcache_attention(_rand((1, 2, 3, 128), 541), cache, scale=0.0, lse=lse)
        want = 0.5 * V[0, 0, -1, 0].double() + 0.5 * V[0, 0, 0, 0].double()
        # weights, and their products with a scale of 0: exact; the fp32 sums of n equal terms and O's rounding remain
        assert torch.all((O.double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -18)), (big, small)
        assert torch.all((lse.double() - np.log(n)).abs() <= 2.0 ** -18 + 2.0 ** -20 * np.log(n))


def test_store_scales_whose_quotient_lies_between_two_numbers():
    """Groups with hi - lo = 15 m, m midway between two bf16 numbers: the scale is the written rule's, bf16 of the fp32 product
    with fp32(1/15), which is one of the two numbers nearest to the quotient: half a step off, and the product's own 2^-24."""
    los = -(128 + np.arange(128)) * 2.0 ** -13                           # 8-bit numbers of [2^-6, 2^-5)
    rows = [(8.5625, -0.021484375)]
    for lo in los:                                                       # 12-bit differences: hi has to be a bf16 number too
        for odd in range(257, 512, 2):                                   # m = odd / 2^9 ... times a power of two
            for e in range(-8, 8):
                hi = 15 * odd * 2.0 ** (e - 9) + lo
                if hi > 0 and hi == float(orc.bf16_value(orc.bf16_bits(hi))):
                    rows.append((hi, lo))
    rows = rows[: 4 * (len(rows) // 4)]
    assert len(rows) >= 4
    x = np.zeros((len(rows), 32))
    x[:, 0], x[:, 1] = np.asarray(rows).T
    x = x.reshape(-1, 128)
    K = torch.tensor(x, dtype=torch.float64).to(torch.bfloat16).view(1, 1, -1, 128).to(DEV)
    assert np.array_equal(_f64(K)[0, 0], x)
    cache = cur.QuantCache(1, 1, x.shape[0])
    cur.curdkv_qcache_store(cache, K, K, cur.make_desc(K, K, 1))
    d = np.asarray(rows)[:, 0] - np.asarray(rows)[:, 1]
    for meta in (cache.K_meta, cache.V_meta):
        s = _f64(meta)[0, 0, :, :, 0].reshape(-1)
        assert np.array_equal(s, orc.bf16_value(orc.bf16_bits(d.astype(np.float32) * np.float32(1 / 15))))
        step = 2.0 ** (np.floor(np.log2(s)) - 7)
        assert np.all(np.abs(s - d / 15) <= 0.5 * step + 2.0 ** -23 * s)
        assert s[0] == 0.57421875
    # and as PyTorch has it
    t = ((K.float().unflatten(-1, (4, 32)).amax(-1) - K.float().unflatten(-1, (4, 32)).amin(-1)) / 15).to(torch.bfloat16)
    assert torch.equal(t[0, 0], cache.K_meta[0, 0, :, :, 0])


def _line_case(seed, packed):
    """Few long heads, which equal runs over all of them and a joining launch take."""
    counts = [20000, 0, 1, 7777, 33, 12000]
    cache, starts = _random_cache(3, 2, 20000, counts, seed, packed)
    return cache, starts, counts


@pytest.mark.parametrize("packed", [False, True])
def test_attention_over_equal_runs_captured_and_replayed(packed):
    """Replayed with other rows, counts and queries, and after another call on the same workspace."""
    cache, starts, counts = _line_case(600, packed)
    Q, lse = _rand((3, 2, 4, 128), 601), torch.zeros((3, 2, 4), device=DEV)
    O, ws = torch.zeros_like(Q), cur.qcache_attention_workspace(cache, 4)
    call = lambda: cur.curdkv_qcache_attention(Q, cache, scale=0.0884, O=O, lse=lse, workspace=ws)  # noqa: E731
    assert _launches(call) == 2
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        Q.copy_(_rand(Q.shape, 610 + i))
        cache.V_codes.bitwise_xor_(0x5A)
        now = [counts[0] - 100 * i, 0, 1, counts[3] - 5000 * (i % 2), 33 - i, 4000 * i]
        cache.count.copy_(torch.tensor(now, dtype=torch.int32))
        if i == 2:
            cache.count.zero_()                              # nothing at all: one replay of zeros
            now = [0] * 6
        graph.replay()
        _check_attention(O, lse, Q, cache, now, starts, float(np.float32(0.0884)), f"{packed} {i}")
        first = O.clone()
        graph.replay()
        assert torch.equal(first, O)
    assert cur.curdkv_device_status(ws) == 0


def test_attention_over_equal_runs_side_by_side():
    """Two streams, a workspace each, both with their joining launch; one of them packed."""
    sets = []
    for i in range(2):
        cache, starts, counts = _line_case(620 + 10 * i, bool(i))
        Q = _rand((3, 2, 3, 128), 640 + i)
        sets.append((cache, starts, counts, Q, torch.zeros_like(Q), torch.zeros((3, 2, 3), device=DEV),
                     cur.qcache_attention_workspace(cache, 3), torch.cuda.Stream()))
    torch.cuda.synchronize()
    before = cur.launch_count()
    for _ in range(20):
        for s in sets:
            with torch.cuda.stream(s[7]):
                cur.curdkv_qcache_attention(s[3], s[0], scale=0.1, O=s[4], lse=s[5], workspace=s[6])
    torch.cuda.synchronize()
    assert cur.launch_count() - before == 80
    for s in sets:
        _check_attention(s[4], s[5], s[3], s[0], s[2], s[1], float(np.float32(0.1)))
        assert cur.curdkv_device_status(s[6]) == 0


@pytest.mark.parametrize("q_rows", [1, 8, 9, 40])
def test_attention_over_equal_runs_stale_rows_and_untouched_memory(q_rows):
    """NaN behind the held rows, and a workspace of exactly the stated size: nothing behind it is written."""
    cache, starts, counts = _line_case(650, False)
    for p, c in enumerate(counts):
        cache.K_meta.view(6, 20000, 4, 2)[p, c:] = float("nan")
        cache.V_meta.view(6, 20000, 4, 2)[p, c:] = float("nan")
    Q, lse = _rand((3, 2, q_rows, 128), 651), torch.zeros((3, 2, q_rows), device=DEV)
    size = cur.qcache_attention_workspace(cache, q_rows).numel()
    buf = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    buf[:256] = 0
    call = lambda: cur.curdkv_qcache_attention(Q, cache, scale=0.1, lse=lse, workspace=buf[:size])  # noqa: E731
    O, _ = call()
    assert _launches(call) == 2
    assert torch.all(buf[size:] == 0xA5) and cur.curdkv_device_status(buf) == 0
    _check_attention(O, lse, Q, cache, counts, starts, float(np.float32(0.1)))
    with pytest.raises(cur.CurdkvError, match="status 3"):
        cur.curdkv_qcache_attention(Q, cache, scale=0.1, workspace=buf[: size - 1])


@pytest.mark.parametrize("q_rows", [1, 20])
def test_attention_over_more_heads_than_a_line_holds(q_rows):
    """More than 8192 heads (or blocks of rows): one CTA each, a workspace without parts."""
    B, H, cap = 1100, 8, 40
    rng = np.random.default_rng(3)
    counts = rng.integers(0, cap + 1, B * H)
    cache, starts = _random_cache(B, H, cap, counts.tolist(), 660)
    Q, lse = _rand((B, H, q_rows, 128), 661), torch.zeros((B, H, q_rows), device=DEV)
    ws = cur.qcache_attention_workspace(cache, q_rows)
    assert ws.numel() == 256
    assert _launches(lambda: cur.curdkv_qcache_attention(Q, cache, scale=0.1, lse=lse, workspace=ws)) == 1
    O, _ = cur.curdkv_qcache_attention(Q, cache, scale=0.1, lse=lse, workspace=ws)
    assert cur.curdkv_device_status(ws) == 0
    kc, vc = (x.view(B * H, cap, 64) for x in (cache.K_codes, cache.V_codes))
    km, vm = (x.view(B * H, cap, 4, 2) for x in (cache.K_meta, cache.V_meta))
    for p in [0, 1, 8191, 8192, B * H - 1] + rng.integers(0, B * H, 20).tolist():
        one = cur.QuantCache.of(*(x[p][None, None].contiguous() for x in (kc, vc, km, vm)), cache.count[p:p + 1].clone(), 1, 1)
        b, h = divmod(p, H)
        _check_attention(O[b:b + 1, h:h + 1], lse[b:b + 1, h:h + 1], Q[b:b + 1, h:h + 1], one, [int(counts[p])], [0],
                         float(np.float32(0.1)), f"head {p}")


@pytest.mark.parametrize("scale", [0.0, 1e-32, 1e-36])
def test_attention_tiny_scales_with_large_products(scale):
    counts = [500, 3]
    cache, starts = _random_cache(1, 2, 512, counts, 670, k_gain=1e16)
    Q, lse = _rand((1, 2, 4, 128), 671, 1e15), torch.zeros((1, 2, 4), device=DEV)
    O, _ = cur.curdkv_qcache_attention(Q, cache, scale=scale, lse=lse)
    _check_attention(O, lse, Q, cache, counts, starts, float(np.float32(scale)))


def test_store_lists_that_run_beyond_their_index():
    """A packed index shorter than its offsets say (those of another selection): lists are cut at its end and flagged, nothing
    behind it is read."""
    K, V = _rand((1, 3, 64, 128), 680), _rand((1, 3, 64, 128), 681)
    desc = cur.make_desc(K, V, 1)
    store = torch.full((64,), 1 << 20, dtype=torch.int32, device=DEV)    # what lies behind the index would be out of range
    store[:24] = torch.arange(24, dtype=torch.int32, device=DEV)
    counts = torch.tensor([10, 10, 10], dtype=torch.int32, device=DEV)
    for entries, off, held in ((24, [0, 10, 20, 30], [10, 10, 4]), (10, [0, 10, 20, 30], [10, 0, 0]), (24, [0, 10, 40, 50], [10, 10, 0])):
        cache, ws = cur.QuantCache(1, 3, 12), torch.zeros(256, dtype=torch.uint8, device=DEV)
        cur.curdkv_qcache_store(cache, K, V, desc, store[:entries], counts, torch.tensor(off, dtype=torch.int32, device=DEV), packed=True,
                                workspace=ws)
        assert cur.curdkv_device_status(ws) == cur.DEV_BAD_INDEX
        assert cache.count.tolist() == held
        rows = np.concatenate([np.arange(c) + 12 * p for p, c in enumerate(held)])
        pick = lambda x: np.concatenate([_f64(x)[0, p][off[p]: off[p] + c] for p, c in enumerate(held)])  # noqa: E731
        _check_rows(cache, rows, (pick(K), pick(V)))
    # offsets that fit: as ever
    cache, ws = cur.QuantCache(1, 3, 12), torch.zeros(256, dtype=torch.uint8, device=DEV)
    cur.curdkv_qcache_store(cache, K, V, desc, store[:24], torch.tensor([10, 10, 4], dtype=torch.int32, device=DEV),
                            torch.tensor([0, 10, 20, 24], dtype=torch.int32, device=DEV), packed=True, workspace=ws)
    assert cur.curdkv_device_status(ws) == 0 and cache.count.tolist() == [10, 10, 4]


@pytest.mark.parametrize("n", [40, 700, 20000])
@pytest.mark.parametrize("q_rows", [4, 16])
def test_attention_non_finite_queries_stay_in_their_row(n, q_rows):
    cache, starts = _random_cache(1, 2, n, [n, n // 2], 690)
    Q = _rand((1, 2, q_rows, 128), 691)
    lse = torch.zeros((1, 2, q_rows), device=DEV)
    want, _ = cur.curdkv_qcache_attention(Q, cache, scale=0.0884, lse=lse)
    _check_attention(want, lse, Q, cache, [n, n // 2], starts, float(np.float32(0.0884)))
    bad = Q.clone()
    bad[0, 0, 1, 5], bad[0, 1, 2, 77] = float("nan"), float("inf")
    got, _ = cur.curdkv_qcache_attention(bad, cache, scale=0.0884)
    rest = torch.ones(Q.shape[:3], dtype=torch.bool, device=DEV)
    rest[0, 0, 1] = rest[0, 1, 2] = False
    assert torch.isnan(got[~rest]).all()
    # another row's weights do not enter, but where its logits move the shared vote a weight may be rounded elsewhere
    lse2 = torch.where(rest, lse, 0.0)
    O = torch.where(rest[..., None], got, want)
    _check_attention(O, torch.where(rest, lse2, lse), Q, cache, [n, n // 2], starts, float(np.float32(0.0884)))


def test_store_append_and_read_of_nothing():
    """No rows, an empty selection (fixed and packed), no new tokens, no slots asked for: counts say so, nothing else moves."""
    K, none = _rand((1, 2, 8, 128), 700), torch.zeros((1, 2, 0, 128), dtype=torch.bfloat16, device=DEV)
    zeros = torch.zeros(3, dtype=torch.int32, device=DEV)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    for case in ("rows", "fixed", "packed"):
        cache = cur.QuantCache(1, 2, 4)
        cache.K_codes.fill_(0xEE)
        cache.count.fill_(3)
        if case == "rows":
            cur.curdkv_qcache_store(cache, none, none, cur.make_desc(none, none, 1), workspace=ws)
        else:
            idx = torch.zeros((1, 2, 0) if case == "fixed" else (0,), dtype=torch.int32, device=DEV)
            cur.curdkv_qcache_store(cache, K, K, cur.make_desc(K, K, 1), idx, zeros[:2], zeros if case == "packed" else None,
                                    packed=case == "packed", workspace=ws)
        assert cache.count.tolist() == [0, 0] and torch.all(cache.K_codes == 0xEE), case
    bad = torch.zeros(256, dtype=torch.uint8, device=DEV)                # offsets and counts that an empty index does not have
    cur.curdkv_qcache_store(cache, K, K, cur.make_desc(K, K, 1), idx, zeros[:2] + 4, 4 * torch.arange(3, dtype=torch.int32, device=DEV),
                            packed=True, workspace=bad)
    assert cur.curdkv_device_status(bad) == cur.DEV_BAD_INDEX
    assert cache.count.tolist() == [0, 0] and torch.all(cache.K_codes == 0xEE)
    cur.curdkv_qcache_append(cache, none, none, workspace=ws)
    cur.curdkv_qcache_append(cache, K[:, :, :3], K[:, :, :3], t_new=torch.zeros(1, dtype=torch.int32, device=DEV), workspace=ws)
    assert cache.count.tolist() == [0, 0] and torch.all(cache.K_codes == 0xEE)
    out = cur.curdkv_qcache_read(cache, torch.zeros((1, 2, 0), dtype=torch.int32, device=DEV), workspace=ws)
    assert [tuple(x.shape) for x in out] == [(1, 2, 0, 128)] * 2
    assert not cur.curdkv_qcache_read(cache, workspace=ws)[0].any()
    assert cur.curdkv_device_status(ws) == 0
