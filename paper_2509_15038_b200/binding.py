"""Thin ctypes binding of ``libcurdkv.so`` (declared in ``include/curdkv.h``).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  torch supplies device memory and the current stream.  There is no
CPU or eager fallback: if the library is missing or a call fails, an exception
is raised.
"""
from __future__ import annotations

import ctypes
import struct
from operator import index
from pathlib import Path
from typing import Optional

import torch

_LIB_PATH = Path(__file__).resolve().parent / "libcurdkv.so"
_lib = None

STATUS_OK = 0
DEV_TIMEOUT = 0x1
DEV_BAD_INDEX = 0x2
DEV_CACHE_FULL = 0x4
DEV_NOT_SPD = 0x8

EXPORTS = (
    "curdkv_workspace_bytes", "curdkv_score", "curdkv_select", "curdkv_compact",
    "curdkv_gqa_map", "curdkv_device_status", "curdkv_launch_count", "curdkv_status_string",
    "curdkv_score_static", "curdkv_host_arena_bytes", "curdkv_compress_host",
    "curdkv_profile_next_score", "curdkv_cache_workspace_bytes", "curdkv_cache_append",
    "curdkv_cache_compress", "curdkv_attention_workspace_bytes", "curdkv_attention_out",
    "curdkv_eviction_loss", "curdkv_gqa_expand", "curdkv_cache_compress_inplace",
    "curdkv_selftest_bounded_wait", "curdkv_selftest_gather_wait", "curdkv_compress", "curdkv_cache_step",
    "curdkv_qcache_store", "curdkv_qcache_append", "curdkv_qcache_read",
    "curdkv_qcache_attention_workspace_bytes", "curdkv_qcache_attention",
    "curdkv_attention_window_workspace_bytes", "curdkv_attention_window",
    "curdkv_cache_push", "curdkv_cache_attention_workspace_bytes", "curdkv_cache_attention_call_workspace_bytes",
    "curdkv_cache_attention",
    "curdkv_attention_prefix_workspace_bytes", "curdkv_attention_prefix",
    "curdkv_attention_scores_workspace_bytes", "curdkv_attention_scores",
)


class CurdkvError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {status_string(code)} (status {code})")
        self.code = code


class Desc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("q_heads", ctypes.c_int32),
        ("n_max", ctypes.c_int32), ("d", ctypes.c_int32), ("r", ctypes.c_int32),
        ("k_stride_b", ctypes.c_int64), ("k_stride_h", ctypes.c_int64), ("k_stride_n", ctypes.c_int64),
        ("v_stride_b", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("v_stride_n", ctypes.c_int64),
        ("seqlens", ctypes.c_void_p),
        ("score_mode", ctypes.c_int32), ("use_projection", ctypes.c_int32),
        ("raw_scores", ctypes.c_int32), ("whiten", ctypes.c_int32), ("ridge", ctypes.c_double),
    ]


class Cache(ctypes.Structure):
    """``curdkv_cache``: device pointers of one layer's generation-phase cache."""

    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("raw", ctypes.c_void_p),
        ("pos", ctypes.c_void_p), ("count", ctypes.c_void_p), ("total", ctypes.c_void_p),
        ("capacity", ctypes.c_int32),
    ]


class QCache(ctypes.Structure):
    """``curdkv_qcache``: device pointers of one 4-bit cache."""

    _fields_ = [
        ("K_codes", ctypes.c_void_p), ("V_codes", ctypes.c_void_p), ("K_meta", ctypes.c_void_p),
        ("V_meta", ctypes.c_void_p), ("count", ctypes.c_void_p), ("row_start", ctypes.c_void_p),
        ("capacity", ctypes.c_int64), ("batch", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
    ]


def load():
    """Load the CUDA library, compiling it first with nvcc if it is missing or older than its
    sources (a fresh checkout has no binary).  There is no other implementation to fall back to:
    if the build fails, this raises."""
    global _lib
    if _lib is not None:
        return _lib
    from . import build as _build

    try:
        _build.build_library()
    except Exception as exc:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is missing and could not be built: {exc} "
                               "(there is no fallback path)") from exc
    lib = ctypes.CDLL(str(_LIB_PATH))
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    dp = ctypes.POINTER(Desc)
    lib.curdkv_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_workspace_bytes.argtypes = [dp, i32, i32]
    lib.curdkv_score.restype = ctypes.c_int
    lib.curdkv_score.argtypes = [vp, vp, vp, i32, dp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.curdkv_score_static.restype = ctypes.c_int
    lib.curdkv_score_static.argtypes = [vp, vp, vp, i32, dp, vp, vp, vp, vp]
    lib.curdkv_select.restype = ctypes.c_int
    lib.curdkv_select.argtypes = [vp, dp, i32, vp, i32, i32, i32, ctypes.c_double, vp, vp, vp, vp,
                                  ctypes.c_size_t, vp]
    lib.curdkv_compact.restype = ctypes.c_int
    lib.curdkv_compact.argtypes = [vp, vp, dp, vp, i64, vp, vp, vp, vp, i64, vp, vp]
    lib.curdkv_compress.restype = ctypes.c_int
    lib.curdkv_compress.argtypes = [vp, vp, vp, i32, dp, i32, vp, i32, i32, i32, ctypes.c_double,
                                    vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.curdkv_host_arena_bytes.restype = ctypes.c_size_t
    lib.curdkv_host_arena_bytes.argtypes = [dp, i32, i32, i32]
    lib.curdkv_compress_host.restype = ctypes.c_int
    lib.curdkv_compress_host.argtypes = [vp, vp, vp, i32, dp, i32, i32, i32, i32, ctypes.c_double,
                                         vp, vp, vp, vp, vp, vp, ctypes.c_size_t, i32,
                                         ctypes.POINTER(ctypes.c_uint32)]
    lib.curdkv_gqa_map.restype = ctypes.c_int
    lib.curdkv_gqa_map.argtypes = [dp, vp, vp]
    lib.curdkv_gqa_expand.restype = ctypes.c_int
    lib.curdkv_gqa_expand.argtypes = [dp, vp, vp, i32, vp, vp, vp]
    lib.curdkv_device_status.restype = ctypes.c_int
    lib.curdkv_device_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32), vp]
    cp = ctypes.POINTER(Cache)
    lib.curdkv_cache_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_cache_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.curdkv_cache_append.restype = ctypes.c_int
    lib.curdkv_cache_append.argtypes = [cp, vp, vp, vp, i32, dp, vp, ctypes.c_size_t, vp]
    lib.curdkv_cache_compress.restype = ctypes.c_int
    lib.curdkv_cache_compress.argtypes = [cp, cp, dp, i32, i32, i32, vp, ctypes.c_size_t, vp]
    lib.curdkv_cache_compress_inplace.restype = ctypes.c_int
    lib.curdkv_cache_compress_inplace.argtypes = [cp, dp, i32, i32, i32, vp, ctypes.c_size_t, vp]
    lib.curdkv_cache_step.restype = ctypes.c_int
    lib.curdkv_cache_step.argtypes = [cp, vp, vp, vp, i32, dp, i32, i32, i32, vp, ctypes.c_size_t, vp]
    lib.curdkv_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_attention_workspace_bytes.argtypes = [dp]
    lib.curdkv_attention_out.restype = ctypes.c_int
    lib.curdkv_attention_out.argtypes = [vp, i32, i64, i64, i64, vp, vp, dp, vp, vp, i64, vp,
                                         ctypes.c_float, i32, vp, vp, ctypes.c_size_t, vp]
    lib.curdkv_eviction_loss.restype = ctypes.c_int
    lib.curdkv_eviction_loss.argtypes = [vp, vp, i32, i64, vp, vp, vp]
    qp, f32 = ctypes.POINTER(QCache), ctypes.c_float
    lib.curdkv_qcache_store.restype = ctypes.c_int
    lib.curdkv_qcache_store.argtypes = [qp, vp, vp, dp, vp, i64, vp, vp, vp, vp]
    lib.curdkv_qcache_append.restype = ctypes.c_int
    lib.curdkv_qcache_append.argtypes = [qp, vp, vp, dp, vp, vp]
    lib.curdkv_qcache_read.restype = ctypes.c_int
    lib.curdkv_qcache_read.argtypes = [qp, vp, i64, vp, vp, vp, vp]
    lib.curdkv_qcache_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_qcache_attention_workspace_bytes.argtypes = [qp, i32]
    lib.curdkv_qcache_attention.restype = ctypes.c_int
    lib.curdkv_qcache_attention.argtypes = [vp, i32, i64, i64, i64, qp, f32, vp, i64, i64, i64, vp, vp,
                                            ctypes.c_size_t, vp]
    lib.curdkv_attention_window_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_attention_window_workspace_bytes.argtypes = [dp, i32]
    lib.curdkv_attention_window.restype = ctypes.c_int
    lib.curdkv_attention_window.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, dp, i32, i32, f32, vp, i64, i64,
                                            i64, vp, vp, ctypes.c_size_t, vp]
    lib.curdkv_cache_push.restype = ctypes.c_int
    lib.curdkv_cache_push.argtypes = [cp, vp, vp, vp, dp, i32, i32, i32, vp, ctypes.c_size_t, vp]
    lib.curdkv_cache_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_cache_attention_workspace_bytes.argtypes = [cp, dp, i32]
    lib.curdkv_cache_attention_call_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_cache_attention_call_workspace_bytes.argtypes = [cp, dp, i32, i32]
    lib.curdkv_cache_attention.restype = ctypes.c_int
    lib.curdkv_cache_attention.argtypes = [vp, i32, i64, i64, i64, vp, cp, dp, f32, vp, i64, i64, i64, vp, vp, vp,
                                           ctypes.c_size_t, vp]
    lib.curdkv_attention_prefix_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_attention_prefix_workspace_bytes.argtypes = [dp, dp, i32]
    lib.curdkv_attention_prefix.restype = ctypes.c_int
    lib.curdkv_attention_prefix.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, dp, vp, vp, dp, f32, vp, i64, i64, i64, vp, vp,
                                            ctypes.c_size_t, vp]
    lib.curdkv_attention_scores_workspace_bytes.restype = ctypes.c_size_t
    lib.curdkv_attention_scores_workspace_bytes.argtypes = [dp, i32]
    lib.curdkv_attention_scores.restype = ctypes.c_int
    lib.curdkv_attention_scores.argtypes = [vp, i32, i64, i64, i64, vp, vp, dp, f32, vp, i32, vp, vp, ctypes.c_size_t, vp]
    lib.curdkv_selftest_bounded_wait.restype = ctypes.c_int
    lib.curdkv_selftest_bounded_wait.argtypes = [ctypes.c_uint64, vp, vp]
    lib.curdkv_selftest_gather_wait.restype = ctypes.c_int
    lib.curdkv_selftest_gather_wait.argtypes = [ctypes.c_uint64, vp, vp]
    lib.curdkv_profile_next_score.restype = ctypes.c_int
    lib.curdkv_profile_next_score.argtypes = [vp, vp]
    lib.curdkv_launch_count.restype = ctypes.c_uint64
    lib.curdkv_launch_count.argtypes = []
    lib.curdkv_status_string.restype = ctypes.c_char_p
    lib.curdkv_status_string.argtypes = [ctypes.c_int]
    _lib = lib
    return lib


def status_string(code: int) -> str:
    return load().curdkv_status_string(int(code)).decode()


def launch_count() -> int:
    return int(load().curdkv_launch_count())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    # an empty view of a live allocation still has a valid base address
    return ctypes.c_void_p(t.data_ptr() if t.numel() else t.untyped_storage().data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(code: int, what: str):
    if code != STATUS_OK:
        raise CurdkvError(code, what)


def make_desc(K: torch.Tensor, V: torch.Tensor, r: int, *, q_heads: Optional[int] = None,
              seqlens: Optional[torch.Tensor] = None, score_mode: int = 0,
              use_projection: int = 1, raw_scores: int = 0, whiten: int = 0,
              ridge: float = 0.0) -> Desc:
    """Descriptor of bf16 K, V ``[B, Hkv, n_max, d]`` (any strides with d contiguous)."""
    if K.dtype is not torch.bfloat16 or V.dtype is not torch.bfloat16:
        raise TypeError("K and V must be bf16")
    shape, k, v = K.shape, K.stride(), V.stride()
    if len(shape) != 4 or shape != V.shape or k[3] != 1 or v[3] != 1:
        raise ValueError("K and V must be [B, Hkv, n, d] with a contiguous last axis")
    B, H, n, d = shape
    if seqlens is None:
        lens = None
    elif seqlens.dtype is not torch.int32 or seqlens.numel() != B or not seqlens.is_contiguous():
        raise ValueError("seqlens must be a contiguous int32 tensor of length B")
    else:
        lens = seqlens.data_ptr()
    desc = Desc(B, H, q_heads or H, n, d, int(r), k[0], k[1], k[2], v[0], v[1], v[2], lens,
                int(score_mode), int(use_projection), int(raw_scores), int(whiten), float(ridge))
    desc.seqlens_tensor = seqlens        # the lengths live as long as the descriptor that points at them
    return desc


def workspace_bytes(desc: Desc, max_budget: int = 0, adaptive: bool = False) -> int:
    return int(load().curdkv_workspace_bytes(ctypes.byref(desc), int(max_budget), int(adaptive)))


def alloc_workspace(desc: Desc, max_budget: int = 1, adaptive: bool = False, device=None) -> torch.Tensor:
    nbytes = workspace_bytes(desc, max_budget, adaptive)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device or "cuda")


def curdkv_score(K, V, G, desc: Desc, workspace: torch.Tensor, scores=None, head_sums=None):
    """Alg. 1 (scoring steps).  G: fp32 device tensor [d, r] or [Hkv, d, r].  Returns (scores, head_sums)."""
    dev = K.device
    if scores is None:
        scores = torch.empty((desc.batch, desc.kv_heads, desc.n_max), dtype=torch.float32, device=dev)
    if head_sums is None:
        head_sums = torch.empty((desc.batch, desc.kv_heads), dtype=torch.float32, device=dev)
    g_per_head = int(G is not None and G.dim() == 3)
    if G is not None and (G.dtype != torch.float32 or not G.is_contiguous()):
        raise TypeError("G must be a contiguous fp32 tensor")
    code = load().curdkv_score(_ptr(K), _ptr(V), _ptr(G), g_per_head, ctypes.byref(desc),
                               _ptr(scores), _ptr(head_sums), _ptr(workspace),
                               workspace.numel(), _stream())
    _check(code, "curdkv_score")
    return scores, head_sums


def curdkv_score_static(K, V, G, desc: Desc, scores=None, head_sums=None, status_flags=None):
    """curdkv_score for callers that may not allocate device memory: the library's built-in
    scratch array stands in for the workspace (see the header for its limit and sharing rules).
    Output tensors are still the caller's; pass them in to keep this call allocation-free."""
    dev = K.device
    if scores is None:
        scores = torch.empty((desc.batch, desc.kv_heads, desc.n_max), dtype=torch.float32, device=dev)
    if head_sums is None:
        head_sums = torch.empty((desc.batch, desc.kv_heads), dtype=torch.float32, device=dev)
    g_per_head = int(G is not None and G.dim() == 3)
    code = load().curdkv_score_static(_ptr(K), _ptr(V), _ptr(G), g_per_head, ctypes.byref(desc),
                                      _ptr(scores), _ptr(head_sums), _ptr(status_flags), _stream())
    _check(code, "curdkv_score_static")
    return scores, head_sums


def curdkv_select(scores, desc: Desc, budget: int, *, num_sink: int = 0, window: int = 0,
                  head_budgets=None, adaptive: bool = False, alpha: float = 0.2,
                  workspace: Optional[torch.Tensor] = None, idx=None, head_counts=None,
                  head_offsets=None):
    """Alg. 1 (sinks, top-k, union) / AdaCurDKV.  Returns (idx, head_counts, head_offsets)."""
    dev = scores.device
    P = desc.batch * desc.kv_heads
    if idx is None:
        if adaptive:
            idx = torch.empty((P * max(min(budget, desc.n_max), 0) + 1,), dtype=torch.int32, device=dev)[:-1]
        else:
            idx = torch.empty((P * max(budget, 0) + 1,), dtype=torch.int32, device=dev)
            idx = idx[: P * max(budget, 0)].view(desc.batch, desc.kv_heads, max(budget, 0))
    if head_counts is None:
        head_counts = torch.empty((desc.batch, desc.kv_heads), dtype=torch.int32, device=dev)
    if head_offsets is None:
        head_offsets = torch.empty((P + 1,), dtype=torch.int32, device=dev)
    code = load().curdkv_select(_ptr(scores), ctypes.byref(desc), int(budget), _ptr(head_budgets),
                                int(num_sink), int(window), int(adaptive), float(alpha),
                                _ptr(idx), _ptr(head_counts), _ptr(head_offsets), _ptr(workspace),
                                0 if workspace is None else workspace.numel(), _stream())
    _check(code, "curdkv_select")
    return idx, head_counts, head_offsets


def curdkv_compact(K, V, desc: Desc, idx, head_counts, head_offsets=None, *, packed: bool = False,
                   K_out=None, V_out=None, workspace: Optional[torch.Tensor] = None):
    """Alg. 1 (gather step).  Fixed layout -> [B, Hkv, budget, d]; packed -> [capacity, d]."""
    dev = K.device
    if packed:
        rows = idx.numel()
        shape, out_stride_h, idx_stride = (rows, desc.d), 0, 0
    else:
        budget = idx.shape[-1]
        shape, out_stride_h, idx_stride = (desc.batch, desc.kv_heads, budget, desc.d), budget, budget
    if K_out is None:
        K_out = torch.zeros(shape, dtype=torch.bfloat16, device=dev)
    if V_out is None:
        V_out = torch.zeros(shape, dtype=torch.bfloat16, device=dev)
    if not packed and out_stride_h == 0:
        return K_out, V_out
    code = load().curdkv_compact(_ptr(K), _ptr(V), ctypes.byref(desc), _ptr(idx), idx_stride,
                                 _ptr(head_counts), _ptr(head_offsets), _ptr(K_out), _ptr(V_out),
                                 out_stride_h, _ptr(workspace), _stream())
    _check(code, "curdkv_compact")
    return K_out, V_out


def curdkv_compress(K, V, G, desc: Desc, budget: int, workspace: torch.Tensor, *, num_sink: int = 0,
                    window: int = 0, head_budgets=None, adaptive: bool = False, alpha: float = 0.2,
                    scores=None, head_sums=None, idx=None, head_counts=None, head_offsets=None,
                    K_out=None, V_out=None):
    """Alg. 1 (all steps) (or AdaCurDKV) in one call; the workspace must come from
    ``alloc_workspace(desc, budget, adaptive)``.  Returns (scores, head_sums, idx, head_counts,
    head_offsets, K_out, V_out) with the layouts of the three separate calls."""
    dev = K.device
    P, b = desc.batch * desc.kv_heads, max(budget, 0)
    if scores is None:
        scores = torch.empty((desc.batch, desc.kv_heads, desc.n_max), dtype=torch.float32, device=dev)
    if head_sums is None:
        head_sums = torch.empty((desc.batch, desc.kv_heads), dtype=torch.float32, device=dev)
    rows = P * (min(b, desc.n_max) if adaptive else b)
    if idx is None:
        idx = torch.empty((rows + 1,), dtype=torch.int32, device=dev)[:rows]
        if not adaptive:
            idx = idx.view(desc.batch, desc.kv_heads, b)
    if head_counts is None:
        head_counts = torch.empty((desc.batch, desc.kv_heads), dtype=torch.int32, device=dev)
    if head_offsets is None:
        head_offsets = torch.empty((P + 1,), dtype=torch.int32, device=dev)
    shape = (rows, desc.d) if adaptive else (desc.batch, desc.kv_heads, b, desc.d)
    if K_out is None:
        K_out = torch.zeros(shape, dtype=torch.bfloat16, device=dev)
    if V_out is None:
        V_out = torch.zeros(shape, dtype=torch.bfloat16, device=dev)
    g_per_head = int(G is not None and G.dim() == 3)
    code = load().curdkv_compress(_ptr(K), _ptr(V), _ptr(G), g_per_head, ctypes.byref(desc), int(budget),
                                  _ptr(head_budgets), int(num_sink), int(window), int(adaptive), float(alpha),
                                  _ptr(scores), _ptr(head_sums), _ptr(idx), _ptr(head_counts),
                                  _ptr(head_offsets), _ptr(K_out), _ptr(V_out), _ptr(workspace),
                                  workspace.numel(), _stream())
    _check(code, "curdkv_compress")
    return scores, head_sums, idx, head_counts, head_offsets, K_out, V_out


class HostBuffers:
    """Pinned host outputs and the device arena of :func:`curdkv_compress_host`."""

    def __init__(self, desc: Desc, budget: int, adaptive: bool, chunk_batch: int, device="cuda"):
        P = desc.batch * desc.kv_heads
        rows = P * (min(budget, desc.n_max) if adaptive else budget)
        pin = dict(pin_memory=True)
        self.idx = torch.empty((max(rows, 1),), dtype=torch.int32, **pin)[:rows]
        self.K_out = torch.empty((max(rows, 1), desc.d), dtype=torch.bfloat16, **pin)[:rows]
        self.V_out = torch.empty((max(rows, 1), desc.d), dtype=torch.bfloat16, **pin)[:rows]
        self.counts = torch.empty((desc.batch, desc.kv_heads), dtype=torch.int32, **pin)
        self.offsets = torch.empty((P + 1,), dtype=torch.int32, **pin)
        nbytes = int(load().curdkv_host_arena_bytes(ctypes.byref(desc), int(budget), int(adaptive),
                                                    int(chunk_batch)))
        if nbytes == 0:
            raise ValueError("invalid shape for curdkv_compress_host")
        self.arena = torch.empty((nbytes,), dtype=torch.uint8, device=device)
        self.chunk_batch = int(chunk_batch)
        if not adaptive:
            self.idx = self.idx.view(desc.batch, desc.kv_heads, budget)
            self.K_out = self.K_out.view(desc.batch, desc.kv_heads, budget, desc.d)
            self.V_out = self.V_out.view(desc.batch, desc.kv_heads, budget, desc.d)


def curdkv_compress_host(K_host, V_host, G_host, desc: Desc, budget: int, buffers: HostBuffers, *,
                         num_sink: int = 0, window: int = 0, adaptive: bool = False,
                         alpha: float = 0.2) -> int:
    """Whole path on host-resident K, V (CPU tensors, ideally pinned); ``desc`` must describe the
    host tensors (``desc.seqlens`` = address of a host int32 array or None).  Results land in
    ``buffers``; returns the device status flags."""
    for t in (K_host, V_host):
        if t.device.type != "cpu" or not t.is_contiguous():
            raise ValueError("host tensors must be contiguous CPU tensors")
    flags = ctypes.c_uint32(0)
    g_per_head = int(G_host is not None and G_host.dim() == 3)
    code = load().curdkv_compress_host(
        _ptr(K_host), _ptr(V_host), _ptr(G_host), g_per_head, ctypes.byref(desc), int(budget),
        int(num_sink), int(window), int(adaptive), float(alpha), _ptr(buffers.K_out),
        _ptr(buffers.V_out), _ptr(buffers.idx), _ptr(buffers.counts), _ptr(buffers.offsets),
        _ptr(buffers.arena), buffers.arena.numel(), buffers.chunk_batch, ctypes.byref(flags))
    _check(code, "curdkv_compress_host")
    return int(flags.value)


class DeviceCache:
    """Torch-owned buffers of one generation-phase cache plus the ``curdkv_cache`` view of them."""

    def __init__(self, batch: int, kv_heads: int, capacity: int, d: int, device="cuda"):
        K = torch.zeros((batch, kv_heads, capacity, d), dtype=torch.bfloat16, device=device)
        raw = torch.zeros((batch, kv_heads, capacity), dtype=torch.float32, device=device)
        pos = torch.full((batch, kv_heads, capacity), -1, dtype=torch.int32, device=device)
        count = torch.zeros((batch,), dtype=torch.int32, device=device)
        self._set(K, torch.zeros_like(K), raw, pos, count, torch.zeros_like(count))

    @classmethod
    def of(cls, K, V, raw, pos, count, total) -> "DeviceCache":
        """A cache over buffers that exist already: K, V bf16 ``[B, Hkv, capacity, d]``, raw fp32 and pos int32 of
        ``[B, Hkv, capacity]``, count and total int32 ``[B]``, contiguous, on one device."""
        self = cls.__new__(cls)
        if K.dim() != 4:
            raise ValueError("K of a DeviceCache must be [batch, kv_heads, capacity, d]")
        for t, shape, dtype in ((K, K.shape, torch.bfloat16), (V, K.shape, torch.bfloat16), (raw, K.shape[:3], torch.float32),
                                (pos, K.shape[:3], torch.int32), (count, K.shape[:1], torch.int32),
                                (total, K.shape[:1], torch.int32)):
            if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
                raise ValueError(f"a buffer of a DeviceCache must be contiguous {dtype} {tuple(shape)}")
            if t.device != K.device:
                raise ValueError("the buffers of a DeviceCache must lie on one device")
        self._set(K, V, raw, pos, count, total)
        return self

    def _set(self, K, V, raw, pos, count, total):
        self.batch, self.kv_heads, self.capacity, self.d = K.shape
        self.K, self.V, self.raw, self.pos, self.count, self.total = K, V, raw, pos, count, total
        self.c = Cache(K.data_ptr(), V.data_ptr(), raw.data_ptr(), pos.data_ptr(), count.data_ptr(), total.data_ptr(),
                       self.capacity)
        self._ref = ctypes.byref(self.c)
        self._descs = {}


def cache_workspace(batch: int, kv_heads: int, t_max: int, capacity: int, budget: int,
                    device="cuda") -> torch.Tensor:
    nbytes = int(load().curdkv_cache_workspace_bytes(batch, kv_heads, t_max, capacity, budget))
    if nbytes == 0:
        raise ValueError("invalid shape for the generation-phase cache")
    return torch.zeros((nbytes,), dtype=torch.uint8, device=device)


def curdkv_cache_append(cache: DeviceCache, K_new, V_new, G, workspace: torch.Tensor, *,
                        t_new: Optional[torch.Tensor] = None) -> None:
    """Sec. 3.2, generation phase: score K_new, V_new ``[B, Hkv, t, d]`` and append them."""
    desc = make_desc(K_new, V_new, G.shape[-1], seqlens=t_new)
    code = load().curdkv_cache_append(ctypes.byref(cache.c), _ptr(K_new), _ptr(V_new), _ptr(G),
                                      int(G.dim() == 3), ctypes.byref(desc), _ptr(workspace),
                                      workspace.numel(), _stream())
    _check(code, "curdkv_cache_append")


def curdkv_cache_compress(src: DeviceCache, dst: DeviceCache, budget: int, workspace: torch.Tensor, *,
                          num_sink: int = 0, window: int = 0) -> None:
    """Alg. 1 (normalisation, selection, gather) on the rows held in ``src``; survivors go to ``dst``."""
    desc = Desc(src.batch, src.kv_heads, src.kv_heads, src.capacity, src.d, 1)
    desc.use_projection = 1
    code = load().curdkv_cache_compress(ctypes.byref(src.c), ctypes.byref(dst.c), ctypes.byref(desc),
                                        int(budget), int(num_sink), int(window), _ptr(workspace),
                                        workspace.numel(), _stream())
    _check(code, "curdkv_cache_compress")


def curdkv_cache_compress_inplace(cache: DeviceCache, budget: int, workspace: torch.Tensor, *,
                                  num_sink: int = 0, window: int = 0) -> None:
    """Alg. 1 (normalisation, selection, gather) on the rows held in ``cache``, in place (the row order is given up)."""
    desc = Desc(cache.batch, cache.kv_heads, cache.kv_heads, cache.capacity, cache.d, 1)
    desc.use_projection = 1
    code = load().curdkv_cache_compress_inplace(ctypes.byref(cache.c), ctypes.byref(desc), int(budget),
                                                int(num_sink), int(window), _ptr(workspace),
                                                workspace.numel(), _stream())
    _check(code, "curdkv_cache_compress_inplace")


def curdkv_cache_step(cache: DeviceCache, K_new, V_new, G, budget: int, workspace: torch.Tensor, *,
                      num_sink: int = 0, window: int = 0, t_new: Optional[torch.Tensor] = None) -> None:
    """One generation step: append K_new, V_new ``[B, Hkv, t, d]`` and compress in place to ``budget``."""
    desc = make_desc(K_new, V_new, G.shape[-1], seqlens=t_new)
    code = load().curdkv_cache_step(ctypes.byref(cache.c), _ptr(K_new), _ptr(V_new), _ptr(G), int(G.dim() == 3),
                                    ctypes.byref(desc), int(budget), int(num_sink), int(window),
                                    _ptr(workspace), workspace.numel(), _stream())
    _check(code, "curdkv_cache_step")


def curdkv_attention_out(Q, K, V, desc: Desc, *, scale: float = 1.0, head_rows=None, head_offsets=None,
                         extra_zero_keys=None, O=None, workspace: Optional[torch.Tensor] = None,
                         weight_split: bool = True):
    """O = softmax(scale Q K^T) V per (b, h).  Q bf16 ``[B, Hkv, m, 128]``; K, V as described by
    ``desc``, or packed ``[rows, 128]`` arrays when ``head_offsets`` is given."""
    if Q.dtype != torch.bfloat16 or Q.dim() != 4 or Q.stride(3) != 1:
        raise ValueError("Q must be bf16 [B, Hkv, m, d] with a contiguous last axis")
    B, H, m, d = Q.shape
    if O is None:
        O = torch.empty((B, H, m, d), dtype=torch.float32, device=Q.device)
    if workspace is None:
        nbytes = int(load().curdkv_attention_workspace_bytes(ctypes.byref(desc)))
        workspace = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=Q.device)
    packed_rows = K.shape[0] if head_offsets is not None else 0
    code = load().curdkv_attention_out(_ptr(Q), m, Q.stride(0), Q.stride(1), Q.stride(2), _ptr(K), _ptr(V),
                                       ctypes.byref(desc), _ptr(head_rows), _ptr(head_offsets),
                                       packed_rows, _ptr(extra_zero_keys), float(scale), int(weight_split),
                                       _ptr(O), _ptr(workspace), workspace.numel(), _stream())
    _check(code, "curdkv_attention_out")
    return O, workspace


def curdkv_eviction_loss(O_full, O_comp):
    """(||O - O'||_F, ||O||_F) per (b, h) for fp32 ``[B, Hkv, m, d]`` outputs."""
    B, H = O_full.shape[:2]
    loss = torch.empty((B, H), dtype=torch.float32, device=O_full.device)
    ref = torch.empty_like(loss)
    code = load().curdkv_eviction_loss(_ptr(O_full), _ptr(O_comp), B * H, O_full[0, 0].numel(), _ptr(loss),
                                       _ptr(ref), _stream())
    _check(code, "curdkv_eviction_loss")
    return loss, ref


# ---- serving: the 4-bit cache and the attention with a sliding window ---------------------------

def _on_device(what: str, first: torch.Tensor, *rest: Optional[torch.Tensor]) -> int:
    """Index of the device that every given tensor lies on, which has to be the current one (the
    calls launch on its current stream)."""
    dev = first.get_device()
    if dev < 0:
        raise ValueError(f"{what}: tensors must be on a CUDA device")
    for t in rest:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{what}: tensors are on {first.device} and {t.device}")
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"{what}: tensors are on {first.device}, which is not the current device")
    return dev


# batch, kv_heads, q_heads, n_max, d, r and the strides of K and V
_DESC_ROWS = struct.Struct("=6i6q").unpack_from
_DESC = struct.Struct("=6i6qQ4id").pack                    # a whole descriptor, lengths' address and flags behind those


def _described(what: str, K: torch.Tensor, V: torch.Tensor, desc: Desc, dev: int) -> None:
    """K and V have to be what the descriptor says, whose shape and strides the kernels go by, and its lengths have to
    lie where they run."""
    shape = K.shape
    B, H, _, n, d, _, kb, kh, kn, vb, vh, vn = _DESC_ROWS(desc)          # (its fields at once: half a microsecond less)
    if K.dtype is not torch.bfloat16 or V.dtype is not torch.bfloat16:
        raise TypeError(f"{what}: K and V must be bf16")
    if shape != (B, H, n, d) or shape != V.shape:
        raise ValueError(f"{what}: K is {tuple(shape)}, V {tuple(V.shape)}, the descriptor says {(B, H, n, d)}")
    k, v = K.stride(), V.stride()
    if k != (kb, kh, kn, 1) or v != (vb, vh, vn, 1):       # (an axis of one is never stepped along)
        if any(n > 1 and (a, b) != (c, d) for n, a, b, c, d in zip(shape, k, v, (kb, kh, kn, 1), (vb, vh, vn, 1))):
            raise ValueError(f"{what}: K or V has other strides than the descriptor")
    lens = getattr(desc, "seqlens_tensor", None)
    if lens is not None and lens.get_device() != dev:
        raise ValueError(f"{what}: the descriptor's seqlens are on {lens.device}")


def _described_keys(what: str, K: torch.Tensor, desc: Desc, dev: int) -> None:
    """The same where only K is read."""
    B, H, _, n, d, _, kb, kh, kn, _, _, _ = _DESC_ROWS(desc)
    shape, k = K.shape, K.stride()
    if K.dtype is not torch.bfloat16:
        raise TypeError(f"{what}: K must be bf16")
    if shape != (B, H, n, d):
        raise ValueError(f"{what}: K is {tuple(shape)}, the descriptor says {(B, H, n, d)}")
    if k != (kb, kh, kn, 1) and any(n > 1 and a != c for n, a, c in zip(shape, k, (kb, kh, kn, 1))):
        raise ValueError(f"{what}: K has other strides than the descriptor")
    lens = getattr(desc, "seqlens_tensor", None)
    if lens is not None and lens.get_device() != dev:
        raise ValueError(f"{what}: the descriptor's seqlens are on {lens.device}")


def _int32(what: str, t: Optional[torch.Tensor], numel: Optional[int] = None) -> None:
    if t is not None and (t.dtype is not torch.int32 or not t.is_contiguous() or (numel is not None and t.numel() != numel)):
        raise ValueError(f"{what} must be a contiguous int32 tensor" + (f" of {numel} entries" if numel is not None else ""))


def _count(x: int) -> int:
    """A number of rows for an int32 argument: what no cache holds is as good as the largest (ctypes would drop the upper
    bits), what is negative is left to the call to refuse."""
    if x.__class__ is int and -1 <= x <= 0x7FFFFFFF:
        return x
    return min(max(index(x), -1), 0x7FFFFFFF)


def _status_buffer(what: str, t: Optional[torch.Tensor]) -> None:
    if t is not None and (not t.is_contiguous() or t.numel() * t.element_size() < 256):
        raise ValueError(f"{what}: workspace must be contiguous and hold at least 256 bytes")


def _raw_stream(index: int) -> int:
    return torch._C._cuda_getCurrentRawStream(index)


def _addr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _base(t: torch.Tensor, other: torch.Tensor) -> int:
    """Address of `t`; of `other` where an empty tensor has none (its rows are none: it is not followed)."""
    return t.data_ptr() or other.data_ptr()


class QuantCache:
    """Torch-owned buffers of one 4-bit cache plus the ``curdkv_qcache`` view of them.

    ``QuantCache(batch, kv_heads, capacity)`` gives every head ``capacity`` rows.  With ``row_start``
    (int32 ``[batch * kv_heads + 1]``, ascending) the heads lie one behind the other, ``capacity`` rows in
    all.  Rows are 128 channels: codes uint8 ``[..., 64]`` and meta bf16 ``[..., 4, 2]`` (scale, zero)."""

    def __init__(self, batch: int, kv_heads: int, capacity: int, *, row_start: Optional[torch.Tensor] = None,
                 device="cuda"):
        rows = (capacity,) if row_start is not None else (batch, kv_heads, capacity)
        codes = [torch.zeros(rows + (64,), dtype=torch.uint8, device=device) for _ in range(2)]
        meta = [torch.zeros(rows + (4, 2), dtype=torch.bfloat16, device=device) for _ in range(2)]
        count = torch.zeros((batch * kv_heads,), dtype=torch.int32, device=device)
        self._set(*codes, *meta, count, batch, kv_heads, capacity, row_start)

    @classmethod
    def of(cls, K_codes, V_codes, K_meta, V_meta, count, batch: int, kv_heads: int, *,
           row_start: Optional[torch.Tensor] = None) -> "QuantCache":
        """A cache over buffers that exist already (contiguous, laid out as above)."""
        self = cls.__new__(cls)
        self._set(K_codes, V_codes, K_meta, V_meta, count, batch, kv_heads,
                  K_codes.shape[0] if row_start is not None else K_codes.shape[2], row_start)
        return self

    def _set(self, K_codes, V_codes, K_meta, V_meta, count, batch, kv_heads, capacity, row_start):
        rows = (capacity,) if row_start is not None else (batch, kv_heads, capacity)
        for t, tail, dtype in ((K_codes, (64,), torch.uint8), (V_codes, (64,), torch.uint8),
                               (K_meta, (4, 2), torch.bfloat16), (V_meta, (4, 2), torch.bfloat16)):
            if tuple(t.shape) != rows + tail or t.dtype != dtype or not t.is_contiguous():
                raise ValueError(f"a buffer of a QuantCache must be contiguous {dtype} {rows + tail}")
        _int32("count", count, batch * kv_heads)
        _int32("row_start", row_start, batch * kv_heads + 1)
        self.K_codes, self.V_codes, self.K_meta, self.V_meta = K_codes, V_codes, K_meta, V_meta
        self.count, self.row_start = count, row_start
        self.batch, self.kv_heads, self.capacity, self.device = batch, kv_heads, capacity, K_codes.device
        for t in (V_codes, K_meta, V_meta, count, row_start):
            if t is not None and t.device != self.device:
                raise ValueError("the buffers of a QuantCache must lie on one device")
        self.c = QCache(K_codes.data_ptr(), V_codes.data_ptr(), K_meta.data_ptr(), V_meta.data_ptr(),
                        count.data_ptr(), None if row_start is None else row_start.data_ptr(),
                        capacity, batch, kv_heads)
        self._ref = ctypes.byref(self.c)


def curdkv_qcache_store(cache: QuantCache, K, V, desc: Desc, idx=None, head_counts=None, head_offsets=None, *,
                        packed: bool = False, workspace: Optional[torch.Tensor] = None) -> None:
    """Rows of K, V (all, or those a selection names, laid out as :func:`curdkv_select` returns them; ``packed``
    for an adaptive one) quantised into ``cache`` from slot 0; sets ``cache.count``."""
    dev = _on_device("curdkv_qcache_store", cache.K_codes, K, V, idx, head_counts, head_offsets, workspace)
    _described("curdkv_qcache_store", K, V, desc, dev)
    P = cache.batch * cache.kv_heads
    _int32("idx", idx)
    _int32("head_counts", head_counts, P)
    _status_buffer("curdkv_qcache_store", workspace)
    stride = 0
    if idx is not None and packed:
        if head_offsets is None:
            raise ValueError("a packed idx needs head_offsets")
        _int32("head_offsets", head_offsets, P + 1)
        stride = idx.numel()
        packed = stride > 0                  # (an empty index holds lists of nothing, whatever the offsets say)
    elif idx is not None:
        if P > 0 and idx.numel() % P != 0:
            raise ValueError("idx must be [batch, kv_heads, budget]")
        stride = idx.numel() // max(P, 1)
    if P == 0:
        return
    code = load().curdkv_qcache_store(cache._ref, _base(K, cache.K_codes), _base(V, cache.K_codes), ctypes.byref(desc),
                                      None if idx is None else _base(idx, cache.K_codes), stride,
                                      _addr(head_counts) if idx is not None else None,
                                      _addr(head_offsets) if idx is not None and packed else None,
                                      _addr(workspace), _raw_stream(dev))
    _check(code, "curdkv_qcache_store")


def curdkv_qcache_append(cache: QuantCache, K_new, V_new, *, t_new: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None) -> None:
    """K_new, V_new ``[B, Hkv, t, 128]`` quantised behind the held rows (``t_new`` int32 ``[B]``: real rows)."""
    dev = _on_device("curdkv_qcache_append", cache.K_codes, K_new, V_new, t_new, workspace)
    _status_buffer("curdkv_qcache_append", workspace)
    desc = make_desc(K_new, V_new, 1, seqlens=t_new)
    if K_new.numel() == 0:
        return
    code = load().curdkv_qcache_append(cache._ref, K_new.data_ptr(), V_new.data_ptr(), ctypes.byref(desc),
                                       _addr(workspace), _raw_stream(dev))
    _check(code, "curdkv_qcache_append")


def curdkv_qcache_read(cache: QuantCache, idx: Optional[torch.Tensor] = None, *, K_out=None, V_out=None,
                       workspace: Optional[torch.Tensor] = None):
    """Held rows as bf16: laid out as the cache's rows are, or the slots ``idx`` (int32 ``[B, Hkv, rows]``, negative
    entries passed over) names.  Rows without a slot keep what the outputs hold (zeros where this call makes them)."""
    dev = _on_device("curdkv_qcache_read", cache.K_codes, idx, K_out, V_out, workspace)
    _status_buffer("curdkv_qcache_read", workspace)
    _int32("idx", idx)
    P = cache.batch * cache.kv_heads
    if idx is not None:
        if P > 0 and idx.numel() % P != 0:
            raise ValueError("idx must be [batch, kv_heads, rows]")
        rows = idx.numel() // max(P, 1)
        shape = (cache.batch, cache.kv_heads, rows, 128)
    elif cache.row_start is not None:
        rows, shape = 0, (cache.capacity, 128)
    else:
        rows, shape = cache.capacity, (cache.batch, cache.kv_heads, cache.capacity, 128)
    out = []
    for t in (K_out, V_out):
        if t is None:
            t = torch.zeros(shape, dtype=torch.bfloat16, device=cache.device)
        elif t.dtype is not torch.bfloat16 or not t.is_contiguous() or t.shape != shape:
            raise ValueError(f"outputs must be contiguous bf16 {shape}")
        out.append(t)
    if out[0].numel() == 0:
        return out[0], out[1]
    code = load().curdkv_qcache_read(cache._ref, _addr(idx), rows, out[0].data_ptr(), out[1].data_ptr(), _addr(workspace),
                                     _raw_stream(dev))
    _check(code, "curdkv_qcache_read")
    return out[0], out[1]


def qcache_attention_workspace(cache: QuantCache, q_rows: int) -> torch.Tensor:
    nbytes = int(load().curdkv_qcache_attention_workspace_bytes(cache._ref, int(q_rows)))
    if nbytes == 0:
        raise ValueError("invalid shape for curdkv_qcache_attention")
    return torch.zeros((nbytes,), dtype=torch.uint8, device=cache.device)


def attention_window_workspace(desc: Desc, q_rows: int, device="cuda") -> torch.Tensor:
    nbytes = int(load().curdkv_attention_window_workspace_bytes(ctypes.byref(desc), int(q_rows)))
    if nbytes == 0:
        raise ValueError("invalid shape for curdkv_attention_window")
    return torch.zeros((nbytes,), dtype=torch.uint8, device=device)


def _queries(what, Q, O, lse):
    """Checks Q, O and lse; returns O (made where not given), Q's shape, and both tensors' strides."""
    shape, q = Q.shape, Q.stride()
    if Q.dtype is not torch.bfloat16 or len(shape) != 4 or q[3] != 1 or shape[3] != 128:
        raise ValueError(f"{what}: Q must be bf16 [B, H, rows, 128] with a contiguous last axis")
    if O is None:
        O = torch.empty(shape, dtype=torch.bfloat16, device=Q.device)
    o = O.stride()
    if O.dtype is not torch.bfloat16 or O.shape != shape or o[3] != 1:
        raise ValueError(f"{what}: O must be bf16 of Q's shape with a contiguous last axis")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != shape[:3] or not lse.is_contiguous()):
        raise ValueError(f"{what}: lse must be contiguous fp32 [B, H, rows]")
    return O, shape, q, o


def curdkv_qcache_attention(Q, cache: QuantCache, *, scale: float, O=None, lse=None,
                            workspace: Optional[torch.Tensor] = None):
    """O = softmax(scale Q K^T) V over the held rows.  Q bf16 ``[B, Hkv, q_rows, 128]``, the queries of a GQA group
    stacked along q_rows; ``lse`` fp32 ``[B, Hkv, q_rows]`` receives the log sums where given.  Returns (O, workspace)."""
    O, (B, H, m, _), q, o = _queries("curdkv_qcache_attention", Q, O, lse)
    if B != cache.batch or H != cache.kv_heads:
        raise ValueError("curdkv_qcache_attention: Q and the cache differ in batch or heads")
    if workspace is None:
        workspace = qcache_attention_workspace(cache, m)
    elif not workspace.is_contiguous():
        raise ValueError("curdkv_qcache_attention: workspace must be contiguous")
    dev = _on_device("curdkv_qcache_attention", cache.K_codes, Q, O, lse, workspace)
    if B == 0:
        return O, workspace
    code = load().curdkv_qcache_attention(Q.data_ptr(), m, q[0], q[1], q[2], cache._ref, scale, O.data_ptr(), o[0], o[1],
                                          o[2], _addr(lse), workspace.data_ptr(), workspace.numel(), _raw_stream(dev))
    if code:
        _check(code, "curdkv_qcache_attention")
    return O, workspace


def curdkv_attention_window(Q, K, V, desc: Desc, window: int, *, num_sink: int = 0, scale: float,
                            q_lens: Optional[torch.Tensor] = None, O=None, lse=None,
                            workspace: Optional[torch.Tensor] = None):
    """Causal attention over the last ``window`` rows and the first ``num_sink``.  Q bf16 ``[B, Hq, t, 128]``: the last
    ``q_lens`` (int32 ``[B]``, default t) positions of each sequence of ``desc``; query rows beyond leave O untouched.
    Returns (O, workspace)."""
    O, (B, H, t, _), q, o = _queries("curdkv_attention_window", Q, O, lse)
    if B != desc.batch or H != desc.q_heads:
        raise ValueError("curdkv_attention_window: Q and the descriptor differ in batch or query heads")
    _int32("q_lens", q_lens, B)
    if workspace is None:
        workspace = attention_window_workspace(desc, t, device=Q.device)
    elif not workspace.is_contiguous():
        raise ValueError("curdkv_attention_window: workspace must be contiguous")
    dev = _on_device("curdkv_attention_window", Q, K, V, O, lse, q_lens, workspace)
    _described("curdkv_attention_window", K, V, desc, dev)
    if B == 0:
        return O, workspace
    code = load().curdkv_attention_window(Q.data_ptr(), t, q[0], q[1], q[2], _addr(q_lens), K.data_ptr() or Q.data_ptr(),
                                          V.data_ptr() or Q.data_ptr(), ctypes.byref(desc), _count(num_sink), _count(window), scale, O.data_ptr(), o[0],
                                          o[1], o[2], _addr(lse), workspace.data_ptr(), workspace.numel(), _raw_stream(dev))
    if code:
        _check(code, "curdkv_attention_window")
    return O, workspace


# ---- generation over a cache whose rows are ranked by the attention weights they receive --------

def attention_scores_workspace(desc: Desc, q_rows: int, device="cuda") -> torch.Tensor:
    nbytes = int(load().curdkv_attention_scores_workspace_bytes(ctypes.byref(desc), int(q_rows)))
    if nbytes == 0:
        raise ValueError("invalid shape for curdkv_attention_scores")
    return torch.zeros((nbytes,), dtype=torch.uint8, device=device)


def curdkv_attention_scores(Q, K, desc: Desc, *, scale: float, q_lens: Optional[torch.Tensor] = None,
                            lse: Optional[torch.Tensor] = None, lse_given: bool = False,
                            scores: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """Scores fp32 ``[B, Hkv, n_max]`` of the rows of K: the causal softmax weights they receive from Q bf16 ``[B, Hq, t, 128]``,
    the last ``q_lens`` (default t) tokens of each sequence of ``desc``, summed over query heads and tokens (normalised
    unless ``desc.raw_scores``).  ``lse`` fp32 ``[B, Hq, t]`` receives the log sums, or with ``lse_given`` brings them.
    Returns (scores, workspace)."""
    what = "curdkv_attention_scores"
    shape, q = Q.shape, Q.stride()
    if Q.dtype is not torch.bfloat16 or len(shape) != 4 or q[3] != 1 or shape[3] != 128:
        raise ValueError(f"{what}: Q must be bf16 [B, H, rows, 128] with a contiguous last axis")
    B, H, t, _ = shape
    if B != desc.batch or H != desc.q_heads:
        raise ValueError(f"{what}: Q and the descriptor differ in batch or query heads")
    _int32("q_lens", q_lens, B)
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != shape[:3] or not lse.is_contiguous()):
        raise ValueError(f"{what}: lse must be contiguous fp32 [B, H, rows]")
    if lse_given and lse is None:
        raise ValueError(f"{what}: lse_given without lse")
    out = (B, desc.kv_heads, desc.n_max)
    if scores is None:
        scores = torch.empty(out, dtype=torch.float32, device=Q.device)
    elif scores.dtype is not torch.float32 or scores.shape != out or not scores.is_contiguous():
        raise ValueError(f"{what}: scores must be contiguous fp32 {out}")
    if workspace is None:
        workspace = attention_scores_workspace(desc, t, device=Q.device)
    elif not workspace.is_contiguous():
        raise ValueError(f"{what}: workspace must be contiguous")
    dev = _on_device(what, Q, K, q_lens, lse, scores, workspace)
    _described_keys(what, K, desc, dev)
    if B == 0:
        return scores, workspace
    code = load().curdkv_attention_scores(Q.data_ptr(), t, q[0], q[1], q[2], _addr(q_lens), _base(K, Q), ctypes.byref(desc), scale,
                                          _addr(lse), int(bool(lse_given)), _base(scores, Q), workspace.data_ptr(),
                                          workspace.nbytes, _raw_stream(dev))
    if code:
        _check(code, what)
    return scores, workspace


def curdkv_cache_push(cache: DeviceCache, K_new, V_new, budget: int, workspace: torch.Tensor, *, num_sink: int = 0,
                      window: int = 0, scores_new: Optional[torch.Tensor] = None,
                      t_new: Optional[torch.Tensor] = None) -> None:
    """K_new, V_new ``[B, Hkv, t, d]`` join ``cache`` with the scores ``scores_new`` (fp32 ``[B, Hkv, t]``; 0 each where not
    given), then rows beyond ``budget`` leave: the least of ``cache.raw`` but for sinks and the ``window`` most recent.
    The workspace is :func:`cache_workspace`'s."""
    what = "curdkv_cache_push"
    dev = _on_device(what, cache.K, K_new, V_new, scores_new, t_new, workspace)
    if not workspace.is_contiguous():
        raise ValueError(f"{what}: workspace must be contiguous")
    if K_new.dtype is not torch.bfloat16 or V_new.dtype is not torch.bfloat16:
        raise TypeError(f"{what}: K_new and V_new must be bf16")
    shape, k, v = K_new.shape, K_new.stride(), V_new.stride()
    if len(shape) != 4 or shape != V_new.shape or k[3] != 1 or v[3] != 1:
        raise ValueError(f"{what}: K_new and V_new must be [B, Hkv, t, d] with a contiguous last axis")
    B, H, t, d = shape
    if B != cache.batch or H != cache.kv_heads or d != cache.d:
        raise ValueError(f"{what}: new rows are {tuple(shape)}, the cache {(cache.batch, cache.kv_heads, cache.capacity, cache.d)}")
    if t_new is not None:
        _int32("t_new", t_new, B)
    if scores_new is not None and (scores_new.dtype is not torch.float32 or scores_new.shape != shape[:3]
                                   or not scores_new.is_contiguous()):
        raise ValueError(f"{what}: scores_new must be contiguous fp32 {tuple(shape[:3])}")
    if B == 0:
        return
    desc = Desc.from_buffer_copy(_DESC(B, H, H, t, d, 1, k[0], k[1], k[2], v[0], v[1], v[2], 0 if t_new is None else t_new.data_ptr(), 0, 1, 0, 0, 0.0))
    code = load().curdkv_cache_push(cache._ref, K_new.data_ptr() or cache.K.data_ptr(), V_new.data_ptr() or cache.K.data_ptr(), _addr(scores_new),
                                    ctypes.byref(desc), index(budget), _count(num_sink), _count(window), workspace.data_ptr(),
                                    workspace.nbytes, _raw_stream(dev))
    if code:
        _check(code, what)


def _cache_desc(cache: DeviceCache, q_heads: int):
    """Reference to a descriptor of the cache's shape for this number of query heads (shapes only: kept on the cache)."""
    ref = cache._descs.get(q_heads)
    if ref is None:
        ref = cache._descs[q_heads] = ctypes.byref(Desc(cache.batch, cache.kv_heads, q_heads, cache.capacity, cache.d, 1))
    return ref


def cache_attention_workspace(cache: DeviceCache, q_heads: int, q_rows: int, *,
                              weights: Optional[bool] = None) -> torch.Tensor:
    """For every call of no more tokens on caches that are no larger; with ``weights`` True or False only for calls of
    exactly these sizes that ask for weights or do not (much less where logits need no room)."""
    args = cache._ref, _cache_desc(cache, int(q_heads)), int(q_rows)
    if weights is None:
        nbytes = int(load().curdkv_cache_attention_workspace_bytes(*args))
    else:
        nbytes = int(load().curdkv_cache_attention_call_workspace_bytes(*args, int(bool(weights))))
    if nbytes == 0:
        raise ValueError("invalid shape for curdkv_cache_attention")
    ws = torch.empty((nbytes,), dtype=torch.uint8, device=cache.K.device)
    ws[:256].zero_()                                         # (the rest is written before it is read)
    return ws


def curdkv_cache_attention(Q, cache: DeviceCache, *, scale: float, weights: Optional[torch.Tensor] = None,
                           q_lens: Optional[torch.Tensor] = None, O=None, lse=None,
                           workspace: Optional[torch.Tensor] = None):
    """O = softmax(scale Q K^T) V over the held rows, Q bf16 ``[B, Hq, t, 128]`` the last ``q_lens`` (default t) tokens of each
    sequence; ``weights`` (fp32 ``[B, Hkv, capacity]``, ``cache.raw`` for instance) grows by the softmax weights of each
    row, summed over its query heads and tokens.  Returns (O, workspace)."""
    what = "curdkv_cache_attention"
    O, (B, H, t, _), q, o = _queries(what, Q, O, lse)
    if B != cache.batch or H % cache.kv_heads or H == 0:
        raise ValueError(f"{what}: Q and the cache differ in batch or heads")
    _int32("q_lens", q_lens, B)
    if weights is not None and (weights.dtype is not torch.float32 or weights.shape != cache.raw.shape
                                or not weights.is_contiguous()):
        raise ValueError(f"{what}: weights must be contiguous fp32 {tuple(cache.raw.shape)}")
    if workspace is None:
        workspace = cache_attention_workspace(cache, H, t)
    elif not workspace.is_contiguous():
        raise ValueError(f"{what}: workspace must be contiguous")
    dev = _on_device(what, cache.K, Q, O, lse, q_lens, weights, workspace)
    if B == 0:
        return O, workspace
    code = load().curdkv_cache_attention(Q.data_ptr(), t, q[0], q[1], q[2], _addr(q_lens), cache._ref, _cache_desc(cache, H), scale,
                                         O.data_ptr(), o[0], o[1], o[2], _addr(lse), _addr(weights), workspace.data_ptr(),
                                         workspace.nbytes, _raw_stream(dev))
    if code:
        _check(code, what)
    return O, workspace


# ---- attention of a batch that shares a prefix -----------------------------------------------

def attention_prefix_workspace(desc_prefix: Desc, desc: Desc, q_rows: int, device="cuda") -> torch.Tensor:
    nbytes = int(load().curdkv_attention_prefix_workspace_bytes(ctypes.byref(desc_prefix), ctypes.byref(desc), int(q_rows)))
    if nbytes == 0:
        raise ValueError("invalid shape for curdkv_attention_prefix")
    return torch.zeros((nbytes,), dtype=torch.uint8, device=device)


def curdkv_attention_prefix(Q, K_prefix, V_prefix, desc_prefix: Desc, K, V, desc: Desc, *, scale: float,
                            q_lens: Optional[torch.Tensor] = None, O=None, lse=None,
                            workspace: Optional[torch.Tensor] = None):
    """Attention over shared rows ``[Bp, Hkv, n0, 128]`` and each sequence's own ``[B, Hkv, n, 128]`` behind them; sequences
    ``i * B / Bp`` onwards share prefix i.  Q bf16 ``[B, Hq, t, 128]``: the last ``q_lens`` (int32 ``[B]``, default t)
    positions of each sequence, which see the whole prefix; query rows beyond leave O untouched.  Returns (O, workspace)."""
    what = "curdkv_attention_prefix"
    O, (B, H, t, _), q, o = _queries(what, Q, O, lse)
    if B != desc.batch or H != desc.q_heads:
        raise ValueError(f"{what}: Q and the descriptor differ in batch or query heads")
    _int32("q_lens", q_lens, B)
    if workspace is None:
        workspace = attention_prefix_workspace(desc_prefix, desc, t, device=Q.device)
    elif not workspace.is_contiguous():
        raise ValueError(f"{what}: workspace must be contiguous")
    dev = _on_device(what, Q, K_prefix, V_prefix, K, V, O, lse, q_lens, workspace)
    _described(what, K_prefix, V_prefix, desc_prefix, dev)
    _described(what, K, V, desc, dev)
    if B == 0:
        return O, workspace
    code = load().curdkv_attention_prefix(Q.data_ptr(), t, q[0], q[1], q[2], _addr(q_lens), _base(K_prefix, Q), _base(V_prefix, Q),
                                          ctypes.byref(desc_prefix), _base(K, Q), _base(V, Q), ctypes.byref(desc), scale,
                                          O.data_ptr(), o[0], o[1], o[2], _addr(lse), workspace.data_ptr(),
                                          workspace.nbytes, _raw_stream(dev))
    if code:
        _check(code, what)
    return O, workspace


def curdkv_profile_next_score(start: torch.cuda.Event, stop: torch.cuda.Event) -> None:
    """Have the next curdkv_score call of this thread record ``start`` / ``stop`` (timing events
    that have been recorded at least once, so that their handles exist) around its sketch kernel."""
    _check(load().curdkv_profile_next_score(ctypes.c_void_p(start.cuda_event),
                                            ctypes.c_void_p(stop.cuda_event)),
           "curdkv_profile_next_score")


def curdkv_selftest_bounded_wait(limit_ns: int, workspace: torch.Tensor) -> None:
    """Runs the kernels' bounded wait on a barrier nobody completes; leaves DEV_TIMEOUT in the status word."""
    _check(load().curdkv_selftest_bounded_wait(int(limit_ns), _ptr(workspace), _stream()),
           "curdkv_selftest_bounded_wait")


def curdkv_selftest_gather_wait(limit_ns: int, workspace: torch.Tensor) -> None:
    """Runs the gather's bounded wait for a head that is never announced; leaves DEV_TIMEOUT in the status word."""
    _check(load().curdkv_selftest_gather_wait(int(limit_ns), _ptr(workspace), _stream()),
           "curdkv_selftest_gather_wait")


def curdkv_gqa_map(desc: Desc, device="cuda") -> torch.Tensor:
    out = torch.empty((desc.q_heads,), dtype=torch.int32, device=device)
    _check(load().curdkv_gqa_map(ctypes.byref(desc), _ptr(out), _stream()), "curdkv_gqa_map")
    return out


def curdkv_gqa_expand(desc: Desc, idx: torch.Tensor, head_counts: torch.Tensor):
    """Per-query-head copies of a fixed-layout selection: (idx_q [B, Hq, budget], counts_q [B, Hq])."""
    budget = idx.shape[-1]
    idx_q = torch.empty((desc.batch, desc.q_heads, budget), dtype=torch.int32, device=idx.device)
    counts_q = torch.empty((desc.batch, desc.q_heads), dtype=torch.int32, device=idx.device)
    _check(load().curdkv_gqa_expand(ctypes.byref(desc), _ptr(idx), _ptr(head_counts), budget, _ptr(idx_q),
                                    _ptr(counts_q), _stream()), "curdkv_gqa_expand")
    return idx_q, counts_q


def curdkv_device_status(workspace: torch.Tensor, with_code: bool = False):
    """Synchronises the current stream and returns the device status flags (with_code: the pair
    (return code, flags); the code is 5, CURDKV_ERR_TIMEOUT, when the timeout bit is set)."""
    flags = ctypes.c_uint32(0)
    code = load().curdkv_device_status(_ptr(workspace), ctypes.byref(flags), _stream())
    if code not in (STATUS_OK, 5):
        raise CurdkvError(code, "curdkv_device_status")
    return (int(code), int(flags.value)) if with_code else int(flags.value)
