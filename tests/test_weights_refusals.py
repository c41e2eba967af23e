"""The calls around attention weights and shared prefixes refuse, on the host and before anything is launched, what they do not
take; and their oracle does what its words say.  Runs without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import curdkv_weights_oracle as orc
from paper_2509_15038_b200 import binding as cur

ANY = 0x7000_0000_1000                                       # an aligned address that is never followed
BIG = 1 << 40


def _cache(**kw):
    f = dict(K=ANY, V=ANY, raw=ANY, pos=ANY, count=ANY, total=ANY, capacity=64)
    f.update(kw)
    return cur.Cache(*[f[n] for n, _ in cur.Cache._fields_])


def _desc(**kw):
    d = cur.Desc(2, 2, 8, 100, 128, 1, 25600, 12800, 128, 25600, 12800, 128, None, 0, 1)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _push(c=None, d=None, K=ANY, V=ANY, scores=None, budget=60, sink=4, window=16, ws=ANY, nbytes=BIG):
    return cur.load().curdkv_cache_push(ctypes.byref(c or _cache()), K, V, scores, ctypes.byref(d or _desc()), budget, sink, window,
                                        ws, nbytes, None)


def _attend(c=None, d=None, Q=ANY, rows=1, qs=(1024, 128, 128), scale=0.1, O=ANY + 8192, os=(1024, 128, 128), lse=None, weights=None,
            ws=ANY, nbytes=BIG):
    return cur.load().curdkv_cache_attention(Q, rows, *qs, None, ctypes.byref(c or _cache()), ctypes.byref(d or _desc()), scale, O, *os,
                                             lse, weights, ws, nbytes, None)


def _prefix(d0=None, d=None, Q=ANY, rows=1, qs=(1024, 128, 128), K0=ANY, V0=ANY, K=ANY, V=ANY, scale=0.1, O=ANY + 8192,
            os=(1024, 128, 128), ws=ANY, nbytes=BIG):
    return cur.load().curdkv_attention_prefix(Q, rows, *qs, None, K0, V0, ctypes.byref(d0 or _desc(batch=1)), K, V,
                                              ctypes.byref(d or _desc()), scale, O, *os, None, ws, nbytes, None)


def _scores(d=None, Q=ANY, rows=4, qs=(4096, 512, 128), K=ANY, scale=0.1, lse=None, given=0, scores=ANY, ws=ANY, nbytes=BIG):
    return cur.load().curdkv_attention_scores(Q, rows, *qs, None, K, ctypes.byref(d or _desc()), scale, lse, given, scores, ws, nbytes, None)


@pytest.mark.parametrize("call,kw,code", [(*x, 1)[:3] for x in [
    (_push, dict(c=_cache(K=None)), 1), (_push, dict(c=_cache(total=None)), 1), (_push, dict(c=_cache(capacity=0)), 1),
    (_push, dict(c=_cache(V=ANY + 8)), 1), (_push, dict(budget=0)), (_push, dict(sink=-1)), (_push, dict(window=-1)),
    (_push, dict(sink=40, window=40)), (_push, dict(K=None)), (_push, dict(V=ANY + 2)), (_push, dict(ws=None)), (_push, dict(ws=ANY + 8)),
    (_push, dict(nbytes=256), 3), (_push, dict(d=_desc(d=12)), 2), (_push, dict(d=_desc(n_max=-1))), (_push, dict(d=_desc(kv_heads=0))),
    (_push, dict(c=_cache(capacity=300 * 1024), budget=100), 2),
    (_attend, dict(c=_cache(pos=None))), (_attend, dict(d=_desc(d=64)), 2), (_attend, dict(d=_desc(q_heads=7))),
    (_attend, dict(d=_desc(kv_heads=0))), (_attend, dict(Q=None)), (_attend, dict(Q=ANY + 2)), (_attend, dict(O=ANY)), (_attend, dict(O=None)),
    (_attend, dict(rows=0)), (_attend, dict(scale=-0.5)), (_attend, dict(scale=float("nan"))), (_attend, dict(scale=float("inf"))),
    (_attend, dict(qs=(1024, 130, 128))), (_attend, dict(qs=(1024, 128, 64), rows=2)), (_attend, dict(os=(0, 128, 128))),
    (_attend, dict(os=(1024, 64, 128))), (_attend, dict(ws=None)), (_attend, dict(ws=ANY + 16)), (_attend, dict(nbytes=0), 3),
    (_attend, dict(rows=300, qs=(307200, 38400, 128), os=(307200, 38400, 128)), 2), (_attend, dict(c=_cache(K=ANY + 8))),
    (_prefix, dict(d0=_desc(batch=1, kv_heads=1, q_heads=1))), (_prefix, dict(d=_desc(batch=3), d0=_desc(batch=2))),
    (_prefix, dict(d0=_desc(batch=0))), (_prefix, dict(d0=_desc(batch=1, d=64)), 2), (_prefix, dict(K0=None)), (_prefix, dict(V0=ANY + 4)),
    (_prefix, dict(K=None)), (_prefix, dict(Q=None)), (_prefix, dict(O=ANY)), (_prefix, dict(rows=0)), (_prefix, dict(scale=-1.0)),
    (_prefix, dict(scale=float("nan"))), (_prefix, dict(os=(1024, 0, 128))), (_prefix, dict(ws=None)), (_prefix, dict(ws=ANY + 64)),
    (_prefix, dict(nbytes=300), 3), (_prefix, dict(d=_desc(q_heads=9))), (_prefix, dict(d=_desc(k_stride_n=100))),
    (_scores, dict(Q=None)), (_scores, dict(K=None)), (_scores, dict(K=ANY + 8)), (_scores, dict(scores=None)), (_scores, dict(given=1)),
    (_scores, dict(rows=0)), (_scores, dict(scale=float("inf"))), (_scores, dict(scale=-1e-3)), (_scores, dict(d=_desc(d=256))), (_scores, dict(d=_desc(d=64)), 2),
    (_scores, dict(d=_desc(q_heads=7))), (_scores, dict(d=_desc(k_stride_n=4))), (_scores, dict(d=_desc(q_heads=2 * 129)), 2),
    (_scores, dict(d=_desc(k_stride_b=0)), 2), (_scores, dict(qs=(0, 512, 128)), 2), (_scores, dict(qs=(4096, 512, 100))),
    (_scores, dict(ws=None)), (_scores, dict(ws=ANY + 32)), (_scores, dict(nbytes=512), 3),
]])
def test_refused_before_any_launch(call, kw, code):
    before = cur.launch_count()
    assert call(**kw) == code
    assert cur.launch_count() == before


def test_workspace_sizes():
    lib = cur.load()
    c, d = _cache(), _desc()
    r = ctypes.byref
    small = lib.curdkv_cache_attention_workspace_bytes(r(c), r(d), 1)
    assert small >= 256 and small % 256 == 0
    assert lib.curdkv_cache_attention_workspace_bytes(r(_cache(capacity=4096)), r(d), 1) > small
    assert lib.curdkv_cache_attention_workspace_bytes(r(c), r(d), 0) == 0
    assert lib.curdkv_cache_attention_workspace_bytes(r(c), r(d), 257) == 0                       # more than 1024 rows a KV head
    assert lib.curdkv_cache_attention_workspace_bytes(None, r(d), 1) == 0
    one = lib.curdkv_attention_scores_workspace_bytes(r(d), 4)
    assert one >= 512 and one % 256 == 0
    assert lib.curdkv_attention_scores_workspace_bytes(r(d), 4000) > one
    assert lib.curdkv_attention_scores_workspace_bytes(r(_desc(q_heads=7)), 4) == 0
    p = lib.curdkv_attention_prefix_workspace_bytes(r(_desc(batch=1)), r(d), 1)
    assert p >= 256 and p % 256 == 0
    assert lib.curdkv_attention_prefix_workspace_bytes(r(_desc(batch=2)), r(_desc(batch=3)), 1) == 0
    assert lib.curdkv_attention_prefix_workspace_bytes(r(_desc(batch=1)), r(d), 0) == 0


@pytest.mark.parametrize("share,group,t", [(1, 1, 1), (5, 4, 1), (64, 4, 1), (16, 4, 4), (200, 3, 1)])
def test_a_prefix_workspace_for_long_own_rows_serves_short_ones(share, group, t):
    size = lambda n0, n: cur.load().curdkv_attention_prefix_workspace_bytes(
        ctypes.byref(_desc(batch=1, n_max=n0)), ctypes.byref(_desc(batch=share, q_heads=2 * group, n_max=n)), t)
    for n0 in (0, 100, 5000, 100000):
        sizes = [size(n0, n) for n in (0, 1, 100, 1000, 20000)]
        assert all(a <= sizes[-1] for a in sizes), sizes


def _lengths(most):
    return [*range(min(most, 300)), *range(300, most, 61), *(x for e in range(5, 18) for x in (2 ** e - 1, 2 ** e, 2 ** e + 1) if x < most), most]


@pytest.mark.parametrize("heads,group,share", [(8, 4, 1), (1, 1, 1), (8, 4, 8), (2, 8, 64), (16, 1, 16), (1, 128, 3), (4, 200, 2)])
def test_a_workspace_for_the_largest_sizes_serves_all_smaller_ones(heads, group, share):
    """Along every axis, densely, from several places: no call asks for more than one that is no smaller in anything."""
    lib, r = cur.load(), ctypes.byref

    def desc(batch, n):
        return _desc(batch=batch, kv_heads=heads, q_heads=heads * group, n_max=n)

    def prefix(prefixes=1, seqs=share, n0=1000, n=100, t=1):
        return lib.curdkv_attention_prefix_workspace_bytes(r(desc(prefixes, n0)), r(desc(prefixes * seqs, n)), t)

    def cache(batch=1, capacity=2049, t=1):
        return lib.curdkv_cache_attention_workspace_bytes(r(_cache(capacity=capacity)), r(desc(batch, 0)), t)

    def scores(batch=1, n=2000, t=32):
        return lib.curdkv_attention_scores_workspace_bytes(r(desc(batch, n)), t)

    def grows(size, axis, values, **at):
        values = sorted(set(values))
        sizes = [size(**{axis: x}, **at) for x in values]
        assert min(sizes) >= 256
        for a, b, x in zip(sizes, sizes[1:], values[1:]):
            assert a <= b, (axis, x, at, a, b)

    long, counts = _lengths(40000), range(1, 300)
    for t in (1, 5):
        grows(prefix, "n", long, t=t)
        grows(prefix, "n", long, t=t, n0=0)
        grows(prefix, "n0", long, t=t)
        grows(prefix, "n0", long, t=t, n=5000)
    grows(prefix, "t", counts, n0=20000)
    grows(prefix, "t", counts, n0=100, n=3000)
    grows(prefix, "seqs", counts)
    grows(prefix, "seqs", counts, n0=30000, n=700)
    grows(prefix, "prefixes", counts, n0=3000)
    grows(cache, "capacity", long[1:])
    grows(cache, "capacity", long[1:], t=3)
    grows(cache, "batch", counts)
    grows(cache, "t", range(1, 1024 // group + 1))
    if group <= 128:
        grows(scores, "n", long)
        grows(scores, "n", long, t=2000)
        grows(scores, "t", long[1:])
        grows(scores, "t", long[1:], n=30000)
        grows(scores, "batch", counts)
        if (heads, group) == (8, 4):
            grows(lambda n: scores(n=n, t=max(n, 1)), "n", long)


@pytest.mark.parametrize("batch,group,capacity,t", [(1, 4, 64, 1), (64, 4, 2049, 1), (20, 4, 2049, 1), (4, 2, 65540, 4), (1, 64, 3000, 1), (1, 4, 900, 256)])
def test_a_cache_attention_asks_for_what_it_uses(batch, group, capacity, t):
    """Logits have room only where weights are asked for and memory has to hold them, the status word is all that one launch
    needs, and a call takes just that."""
    lib, r = cur.load(), ctypes.byref
    c, d = _cache(capacity=capacity), _desc(batch=batch, q_heads=2 * group)
    whole = lib.curdkv_cache_attention_workspace_bytes(r(c), r(d), t)
    with_weights, without = (lib.curdkv_cache_attention_call_workspace_bytes(r(c), r(d), t, w) for w in (1, 0))
    logits = 4 * 2 * batch * capacity * max(2, -(-group * t // 4) * 4)
    assert 256 <= without <= with_weights <= whole and whole >= logits
    assert with_weights == whole if without > 256 else with_weights == 256
    assert without <= whole - logits
    strides = (group * 2 * t * 128, t * 128, 128)
    for weights, need in ((ANY, with_weights), (None, without)):
        assert _attend(c=c, d=d, rows=t, qs=strides, os=strides, weights=weights, nbytes=need - 1) == 3
    assert lib.curdkv_cache_attention_call_workspace_bytes(r(c), r(_desc(q_heads=7)), t, 1) == 0


def test_calls_on_nothing():
    """A batch of none is an answer, not an error."""
    assert _push(d=_desc(batch=0)) == 0
    assert _attend(d=_desc(batch=0)) == 0
    assert _prefix(d=_desc(batch=0), d0=_desc(batch=0)) == 0
    assert _scores(d=_desc(batch=0)) == 0


@pytest.mark.parametrize("rows,q_heads", [(1, 8), (5, 8), (8, 8), (2, 64), (1, 34), (300, 8)])
def test_calls_on_nothing_with_many_query_rows(rows, q_heads):
    """The same with more than 16 query rows a KV head, where a prefix would be read in tiles: no sequences, and no prefixes or
    some, have a workspace and an answer."""
    lib, none = cur.load(), _desc(batch=0, q_heads=q_heads)
    strides = (q_heads * rows * 128, rows * 128, 128)
    for prefixes in (0, 1):
        prefix = _desc(batch=prefixes)
        assert lib.curdkv_attention_prefix_workspace_bytes(ctypes.byref(prefix), ctypes.byref(none), rows) >= 256
        assert _prefix(d=none, d0=prefix, rows=rows, qs=strides, os=strides) == 0
    assert lib.curdkv_attention_scores_workspace_bytes(ctypes.byref(none), rows) >= 256
    assert _scores(d=none, rows=rows, qs=strides) == 0
    if rows * q_heads // 2 <= 1024:
        assert lib.curdkv_cache_attention_workspace_bytes(ctypes.byref(_cache()), ctypes.byref(none), rows) >= 256
        assert _attend(d=none, rows=rows, qs=strides, os=strides) == 0


def test_scores_of_absurd_sizes_are_refused():
    """Sizes that no memory holds: units of more tiles than an int counts, and counts beyond 64 bits."""
    for batch, kv_heads, n, rows in ((4736, 8, 1 << 24, 1 << 29), (16, 8, 1 << 24, 1 << 29), (1 << 20, 16, 1 << 29, 1 << 29)):
        d = _desc(batch=batch, kv_heads=kv_heads, q_heads=kv_heads * 128, n_max=n)
        assert cur.load().curdkv_attention_scores_workspace_bytes(ctypes.byref(d), rows) == 0
    d = _desc(batch=1, kv_heads=1, q_heads=128, n_max=1 << 29)
    assert cur.load().curdkv_attention_scores_workspace_bytes(ctypes.byref(d), 1 << 29) > 1 << 40


def test_binding_checks_without_a_device():
    K = torch.zeros((1, 2, 8, 128), dtype=torch.bfloat16)
    raw, pos = torch.zeros((1, 2, 8)), torch.zeros((1, 2, 8), dtype=torch.int32)
    n = torch.zeros((1,), dtype=torch.int32)
    c = cur.DeviceCache.of(K, K.clone(), raw, pos, n, n.clone())
    assert (c.batch, c.kv_heads, c.capacity, c.d) == (1, 2, 8, 128)
    for bad in ((K.float(), K, raw, pos, n, n), (K, K[:, :1], raw, pos, n, n), (K, K, raw.double(), pos, n, n), (K, K, raw, pos.long(), n, n),
                (K, K, raw, pos, n.long(), n), (K.transpose(1, 2), K, raw, pos, n, n), (K[0], K[0], raw, pos, n, n),
                (K, K, raw[..., :7], pos, n, n)):
        with pytest.raises(ValueError):
            cur.DeviceCache.of(*bad)
    Q = torch.zeros((1, 4, 1, 128), dtype=torch.bfloat16)
    desc = cur.make_desc(K, K, 1, q_heads=4)
    with pytest.raises(ValueError):
        cur.curdkv_cache_attention(Q.float(), c, scale=1.0)
    with pytest.raises(ValueError):
        cur.curdkv_cache_attention(torch.zeros((1, 3, 1, 128), dtype=torch.bfloat16), c, scale=1.0)
    with pytest.raises(ValueError):
        cur.curdkv_cache_attention(Q, c, scale=1.0, weights=raw[..., :7])
    with pytest.raises(ValueError):
        cur.curdkv_cache_attention(Q, c, scale=1.0)                                              # not on a CUDA device
    with pytest.raises(ValueError):
        cur.curdkv_cache_push(c, K[:, :, :1], K[:, :, :1], 8, torch.zeros(4096, dtype=torch.uint8))
    with pytest.raises(ValueError):
        cur.curdkv_attention_scores(Q, K, desc, scale=1.0, lse_given=True)
    with pytest.raises(ValueError):
        cur.curdkv_attention_scores(Q, K, desc, scale=1.0, scores=torch.zeros((1, 2, 9)))
    with pytest.raises(ValueError):
        cur.curdkv_attention_prefix(Q, K, K, desc, K, K, cur.make_desc(K, K, 1, q_heads=2), scale=1.0)


# ---- the oracle itself --------------------------------------------------------------------------

def test_oracle_push_by_hand():
    """Five rows, budget four, one new: the least free row (slot 1) goes, the new row takes its place; then equal weights, where
    the higher slot goes; then a new row that is not in the window and weighs least itself."""
    at, raw, pos = orc.push([5.0, 1.0, 3.0, 2.0], [0, 7, 3, 9], 10, [0.0], 4, 1, 2)
    assert at.tolist() == [0, 4, 2, 3] and pos.tolist() == [0, 10, 3, 9] and raw.tolist() == [5.0, 0.0, 3.0, 2.0]
    at, _, _ = orc.push([1.0, 1.0, 1.0, 1.0], [0, 1, 2, 3], 4, [0.0], 4, 0, 1)
    assert at.tolist() == [0, 1, 2, 4]
    at, _, pos = orc.push([1.0, 2.0, 3.0], [0, 1, 2], 3, [0.5], 3, 0, 0)
    assert at.tolist() == [0, 1, 2] and pos.tolist() == [0, 1, 2]


def test_oracle_scores_by_hand():
    """Two keys, one query row at each position, zero logits: the first key gets 1 + 1/2, the second 1/2."""
    q, k = np.zeros((1, 2, 4)), np.ones((2, 4))
    assert np.allclose(orc.scores(q, k, 1.0, normalised=False), [1.5, 0.5])
    assert np.allclose(orc.scores(q, k, 1.0), [0.75, 0.25])
    assert np.allclose(orc.scores(q, k, 1.0, False, lse=np.array([[0.0, np.log(4.0)]])), [1.25, 0.25])
    assert np.allclose(orc.scores(np.zeros((1, 3, 4)), k, 1.0), [0.75, 0.25])                     # a query before the first row


def test_oracle_prefix_is_attention_over_both():
    rng = np.random.default_rng(0)
    q, k0, v0, k, v = (rng.standard_normal((n, 8)) for n in (2, 5, 5, 3, 3))
    o, lse, w = orc.prefix_attention(q, k0, v0, k, v, 0.3)
    for i, sees in enumerate((7, 8)):
        s = 0.3 * q[i] @ np.concatenate([k0, k])[:sees].T
        e = np.exp(s)
        assert np.allclose(o[i], e @ np.concatenate([v0, v])[:sees] / e.sum()) and np.isclose(lse[i], np.log(e.sum()))
        assert np.all(w[i, sees:] == 0)
