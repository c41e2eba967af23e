"""The serving calls refuse, on the host and before anything is launched, what they do not take.  Runs without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import curdkv_serving_oracle as orc
from paper_2509_15038_b200 import binding as cur

ANY = 0x7000_0000_1000                                       # an aligned address that is never followed


def _cache(**kw):
    f = dict(K_codes=ANY, V_codes=ANY, K_meta=ANY, V_meta=ANY, count=ANY, row_start=None, capacity=64, batch=1, kv_heads=2)
    f.update(kw)
    return cur.QCache(*[f[n] for n, _ in cur.QCache._fields_])


def _desc(**kw):
    d = cur.Desc(1, 2, 8, 100, 128, 1, 25600, 12800, 128, 25600, 12800, 128, None, 0, 1)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _store(c=None, d=None, K=ANY, V=ANY, idx=None, stride=0, counts=None, offs=None, ws=None):
    return cur.load().curdkv_qcache_store(ctypes.byref(c or _cache()), K, V, ctypes.byref(d or _desc()), idx, stride, counts,
                                          offs, ws, None)


def _attend(c=None, Q=ANY, rows=4, qs=(1024, 512, 128), scale=0.1, O=ANY + 4096, os=(1024, 512, 128), ws=ANY, nbytes=1 << 30):
    return cur.load().curdkv_qcache_attention(Q, rows, *qs, ctypes.byref(c or _cache()), scale, O, *os, None, ws, nbytes, None)


def _window(d=None, Q=ANY, rows=4, qs=(4096, 512, 128), K=ANY, V=ANY, sink=4, window=16, scale=0.1, O=ANY + 4096,
            os=(4096, 512, 128), ws=ANY, nbytes=1 << 30):
    return cur.load().curdkv_attention_window(Q, rows, *qs, None, K, V, ctypes.byref(d or _desc()), sink, window, scale, O, *os,
                                              None, ws, nbytes, None)


@pytest.mark.parametrize("call,kw,code", [
    (_store, dict(c=_cache(K_codes=None)), 1), (_store, dict(c=_cache(V_meta=ANY + 8)), 1), (_store, dict(c=_cache(capacity=0)), 1),
    (_store, dict(c=_cache(capacity=1 << 31)), 2), (_store, dict(c=_cache(batch=2)), 1), (_store, dict(c=_cache(kv_heads=0)), 1),
    (_store, dict(c=_cache(count=None)), 1), (_store, dict(K=None), 1), (_store, dict(V=ANY + 2), 1), (_store, dict(d=_desc(d=64)), 2),
    (_store, dict(d=_desc(k_stride_n=64)), 1), (_store, dict(d=_desc(v_stride_h=12801)), 1), (_store, dict(d=_desc(n_max=-1)), 1),
    (_store, dict(idx=ANY, stride=4), 1), (_store, dict(idx=ANY, counts=ANY, stride=-1), 1), (_store, dict(counts=ANY), 1),
    (_store, dict(ws=ANY + 16), 1),
    (_attend, dict(Q=None), 1), (_attend, dict(O=ANY), 1), (_attend, dict(rows=0), 1), (_attend, dict(scale=float("nan")), 1),
    (_attend, dict(scale=-1.0), 1), (_attend, dict(scale=float("inf")), 1), (_attend, dict(qs=(1024, 512, 64)), 1),
    (_attend, dict(os=(1024, 500, 128)), 1), (_attend, dict(ws=None), 1), (_attend, dict(ws=ANY + 128), 1),
    (_attend, dict(nbytes=128), 3), (_attend, dict(Q=ANY + 2), 1), (_attend, dict(c=_cache(K_meta=None)), 1),
    (_window, dict(Q=None), 1), (_window, dict(O=ANY), 1), (_window, dict(rows=0), 1), (_window, dict(sink=-1), 1),
    (_window, dict(window=-1), 1), (_window, dict(scale=float("nan")), 1), (_window, dict(scale=-0.5), 1), (_window, dict(d=_desc(d=64)), 2),
    (_window, dict(d=_desc(q_heads=7)), 1), (_window, dict(K=None), 1), (_window, dict(V=ANY + 8), 1), (_window, dict(ws=None), 1),
    (_window, dict(nbytes=0), 3), (_window, dict(qs=(4096, 512, 130)), 1), (_window, dict(os=(-8, 512, 128)), 1),
])
def test_refused_before_any_launch(call, kw, code):
    before = cur.launch_count()
    assert call(**kw) == code
    assert cur.launch_count() == before


def test_read_and_append_refusals():
    lib, before = cur.load(), cur.launch_count()
    c = ctypes.byref(_cache())
    assert lib.curdkv_qcache_read(c, None, -1, ANY, ANY, None, None) == 1
    assert lib.curdkv_qcache_read(c, ANY, 0, ANY, ANY, None, None) == 1
    assert lib.curdkv_qcache_read(c, None, 4, None, ANY, None, None) == 1
    assert lib.curdkv_qcache_read(c, None, 4, ANY, ANY + 4, None, None) == 1
    assert lib.curdkv_qcache_append(c, None, ANY, ctypes.byref(_desc()), None, None) == 1
    assert lib.curdkv_qcache_append(c, ANY, ANY, ctypes.byref(_desc(batch=3)), None, None) == 1
    assert cur.launch_count() == before


def test_workspace_sizes():
    lib = cur.load()
    small = lib.curdkv_qcache_attention_workspace_bytes(ctypes.byref(_cache()), 4)
    assert small >= 256 and small % 256 == 0
    assert lib.curdkv_qcache_attention_workspace_bytes(ctypes.byref(_cache(kv_heads=64)), 4) >= small
    assert lib.curdkv_qcache_attention_workspace_bytes(ctypes.byref(_cache()), 0) == 0
    assert lib.curdkv_qcache_attention_workspace_bytes(None, 4) == 0
    # what a window call needs never exceeds what the size call says, whatever its window
    for n in (1, 100, 5000, 131072):
        d = _desc(n_max=n)
        room = lib.curdkv_attention_window_workspace_bytes(ctypes.byref(d), 1)
        assert 256 <= room
    assert lib.curdkv_attention_window_workspace_bytes(ctypes.byref(_desc()), 0) == 0
    assert lib.curdkv_attention_window_workspace_bytes(ctypes.byref(_desc(q_heads=3)), 1) == 0


def test_binding_refuses_wrong_tensors():
    Q = torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16)
    K = torch.zeros((1, 2, 8, 128), dtype=torch.bfloat16)
    desc = cur.make_desc(K, K, 1)
    with pytest.raises(ValueError, match="CUDA device"):
        cur.curdkv_attention_window(Q, K, K, desc, 4, scale=0.1, workspace=torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError, match="Q must be"):
        cur.curdkv_attention_window(Q.float(), K, K, desc, 4, scale=0.1)
    with pytest.raises(ValueError, match="O must be"):
        cur.curdkv_attention_window(Q, K, K, desc, 4, scale=0.1, O=Q.float())
    with pytest.raises(ValueError, match="differ"):
        cur.curdkv_attention_window(torch.zeros((1, 3, 4, 128), dtype=torch.bfloat16), K, K, desc, 4, scale=0.1)
    cache = cur.QuantCache(1, 2, 8, device="cpu")
    with pytest.raises(ValueError, match="CUDA device"):
        cur.curdkv_qcache_store(cache, K, K, desc)
    with pytest.raises(ValueError, match="contiguous"):
        cur.QuantCache.of(cache.K_codes, cache.V_codes, cache.K_meta.float(), cache.V_meta, cache.count, 1, 2)
    with pytest.raises(ValueError, match="int32"):
        cur.QuantCache(1, 2, 8, row_start=torch.zeros(2, dtype=torch.int32), device="cpu")
    with pytest.raises(ValueError, match="lse"):
        cur.curdkv_qcache_attention(Q, cache, scale=0.1, lse=torch.zeros(3))


def test_oracle_of_the_format():
    """The oracle's own rules on values worked out by hand."""
    x = np.zeros((1, 128))
    x[0, :32] = np.arange(32) * 0.5                          # range 15.5: scale bf16(15.5 / 15) = 1.03125
    codes, s, z, meta = orc.quantise(x)
    assert s[0, 0] == 1.03125 and z[0, 0] == 0.0 and s[0, 1] == 0.0
    assert codes[0, 0, 31] == 15 and codes[0, 0, 1] == 0 and codes[0, 0, 2] == 1   # 0.5 / 1.03125 < 0.5 < 1 / 1.03125
    assert (codes[0, 1:] == 0).all()
    p = orc.pack(codes, "K")
    assert (p[0, 4] >> 4, p[0, 0] & 15) == (0, 0)
    for which in "KV":
        assert sorted(orc.PLACES[which]) == list(range(128))
        val, _ = orc.unpack(orc.pack(codes, which), meta, which)
        assert np.array_equal(val.reshape(4, 32), s[0][:, None] * codes[0] + z[0][:, None])
    assert orc.PLACES["K"][32 * 2 + 8 * 3 + 5] == 8 * (4 * 3 + 2) + 5
    assert orc.PLACES["V"][32 * 1 + 4 * 6 + 3] == 4 * (4 * 6 + 1) + 3
    m = orc.window_mask(6, 2, 2, 1)
    assert m.tolist() == [[True, False, False, True, True, False], [True, False, False, False, True, True]]


def _elsewhere(monkeypatch):
    """Has the binding take CPU tensors for tensors of device 0, and fail where a call would reach the library."""
    monkeypatch.setattr(cur, "_on_device", lambda what, first, *rest: 0)

    def reached():
        raise AssertionError("the call was not refused")
    monkeypatch.setattr(cur, "load", reached)


def test_rows_that_the_descriptor_does_not_describe(monkeypatch):
    """K and V shorter, of another type or laid out otherwise than their descriptor says, and lengths on another device, are
    refused: the kernels go by the descriptor and would read beyond the tensors."""
    K = torch.zeros((1, 2, 16, 128), dtype=torch.bfloat16)
    desc = cur.make_desc(K, K, 1)
    cache = cur.QuantCache(1, 2, 16, device="cpu")
    Q = torch.zeros((1, 2, 1, 128), dtype=torch.bfloat16)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    assert (cur.Desc.n_max.offset, cur.Desc.k_stride_b.offset, cur.Desc.v_stride_n.offset) == (12, 24, 64)   # as they are read
    _elsewhere(monkeypatch)
    calls = (lambda k, v, d: cur.curdkv_qcache_store(cache, k, v, d),
             lambda k, v, d: cur.curdkv_attention_window(Q, k, v, d, 4, scale=0.1, workspace=ws))
    turned = torch.zeros((1, 16, 2, 128), dtype=torch.bfloat16).transpose(1, 2)
    for call in calls:
        for k, v in ((K[:, :, :8], K), (K, K[:, :, :8]), (K[:, :1], K[:, :1]), (K[:, :, :8], K[:, :, :8])):
            with pytest.raises(ValueError, match="descriptor"):
                call(k, v, desc)
        for k, v in ((turned, K), (K, turned)):
            with pytest.raises(ValueError, match="strides"):
                call(k, v, desc)
        for k, v in ((K.half(), K), (K, K.float())):
            with pytest.raises(TypeError, match="bf16"):
                call(k, v, desc)
        away = cur.make_desc(K, K, 1, seqlens=torch.full((1,), 16, dtype=torch.int32))       # on the host
        with pytest.raises(ValueError, match="seqlens"):
            call(K, K, away)
        with pytest.raises(AssertionError, match="not refused"):     # and what is described passes
            call(K, K, desc)
        odd = torch.zeros(5000, dtype=torch.bfloat16).as_strided((1, 2, 16, 128), (8, 2048, 128, 1))   # an axis of one
        with pytest.raises(AssertionError, match="not refused"):
            call(odd, K, desc)


@pytest.mark.parametrize("big", [2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63, 10 ** 30])
def test_numbers_beyond_int32_are_not_cut(monkeypatch, big):
    """A window, or sinks, of more rows than int32 counts reach the library as the largest number, negative ones as one that
    it refuses."""
    K = torch.zeros((1, 2, 16, 128), dtype=torch.bfloat16)
    Q, ws = torch.zeros((1, 2, 1, 128), dtype=torch.bfloat16), torch.zeros(1 << 20, dtype=torch.uint8)
    got = []

    class Library:
        @staticmethod
        def curdkv_attention_window(*args):
            got.append(args[9:11])
            return 0
    monkeypatch.setattr(cur, "_on_device", lambda what, first, *rest: 0)
    monkeypatch.setattr(cur, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(cur, "load", lambda: Library)
    call = lambda window, sink: cur.curdkv_attention_window(Q, K, K, cur.make_desc(K, K, 1), window, num_sink=sink, scale=0.1, workspace=ws)  # noqa: E731
    call(big, 4)
    call(4, big)
    call(-big, 0)
    call(0, -big)
    call(np.int64(7), 0)
    assert got == [(4, 2 ** 31 - 1), (2 ** 31 - 1, 4), (0, -1), (-1, 0), (0, 7)]
    with pytest.raises(TypeError):
        call(1.5, 0)


@pytest.mark.parametrize("call,os,kw", [
    (_attend, (1024, 0, 128), {}), (_attend, (1024, 384, 128), {}), (_attend, (1024, 128, 128), {}), (_attend, (1024, 128, 136), {}),
    (_attend, (0, 512, 128), dict(c=_cache(batch=2))), (_attend, (1016, 512, 128), dict(c=_cache(batch=2))),
    (_window, (4096, 0, 128), {}), (_window, (4096, 504, 128), {}), (_window, (4096, 128, 1016), {}),
    (_window, (128, 512, 128), dict(d=_desc(batch=2))), (_window, (0, 512, 128), dict(d=_desc(batch=2))),
])
def test_output_rows_that_share_memory(call, os, kw):
    """Rows of O that lie over one another, as those of an expanded tensor, would be written by several at once."""
    before = cur.launch_count()
    assert call(os=os, **kw) == 1
    assert cur.launch_count() == before


def test_read_into_one_buffer_twice():
    lib, before = cur.load(), cur.launch_count()
    rows = 2 * 4 * 256                                       # bytes of 2 heads of 4 rows
    for k, v in ((ANY, ANY), (ANY, ANY + rows - 16), (ANY + rows - 16, ANY)):
        assert lib.curdkv_qcache_read(ctypes.byref(_cache()), None, 4, k, v, None, None) == 1
        assert lib.curdkv_qcache_read(ctypes.byref(_cache()), ANY, 4, k, v, None, None) == 1
        assert lib.curdkv_qcache_read(ctypes.byref(_cache(capacity=4)), None, 0, k, v, None, None) == 1
        assert lib.curdkv_qcache_read(ctypes.byref(_cache(capacity=8, row_start=ANY)), None, 0, k, v, None, None) == 1
    assert cur.launch_count() == before


def test_workspaces_that_are_smaller_than_they_look(monkeypatch):
    """A workspace is counted by its elements: one that is expanded, or strided, does not hold as many bytes side by side."""
    K, Q = torch.zeros((1, 2, 16, 128), dtype=torch.bfloat16), torch.zeros((1, 2, 1, 128), dtype=torch.bfloat16)
    cache, desc = cur.QuantCache(1, 2, 16, device="cpu"), cur.make_desc(K, K, 1)
    _elsewhere(monkeypatch)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 20, dtype=torch.uint8)[::2],
               torch.zeros((256, 64), dtype=torch.uint8).t()):
        for call in (lambda: cur.curdkv_qcache_attention(Q, cache, scale=0.1, workspace=ws),
                     lambda: cur.curdkv_attention_window(Q, K, K, desc, 4, scale=0.1, workspace=ws),
                     lambda: cur.curdkv_qcache_store(cache, K, K, desc, workspace=ws),
                     lambda: cur.curdkv_qcache_append(cache, K, K, workspace=ws),
                     lambda: cur.curdkv_qcache_read(cache, workspace=ws)):
            with pytest.raises(ValueError, match="workspace must be contiguous"):
                call()
