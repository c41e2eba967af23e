"""Oracle of the serving calls: 4-bit rows and attention over them, and the attention with a sliding window and sinks, in
numpy float64 on the host, shared with nothing on the GPU side.

A group of 32 channels with least value lo and greatest hi is held as scale = bf16(fp32(hi - lo) * fp32(1/15)), zero = lo and
codes rint((x - zero) / scale) in 0 .. 15; channel 32 g + 8 t + u of K sits in nibble u of 32-bit word 4 t + g of its
row's 64 bytes, channel 32 g + 4 t + u of V in nibble u of 16-bit word 4 t + g.
"""
import numpy as np


def bf16_bits(x):
    """fp32 array -> bf16 bits, ties to even; NaN -> 0x7fc0."""
    x = np.asarray(x, dtype=np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def bf16_value(bits):
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32)


def quantise(x):
    """bf16 values (float64 [rows, 128]) -> (codes uint8 [rows, 4, 32], scale, zero float64 [rows, 4], meta bits [rows, 4, 2])."""
    x = np.asarray(x, dtype=np.float64).reshape(-1, 4, 32)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1), x.max(-1)
        s32 = ((hi.astype(np.float32) - lo.astype(np.float32)) * np.float32(1 / 15)).astype(np.float32)
        bits = bf16_bits(s32)
        s = bf16_value(bits).astype(np.float64)
        bad = ~np.isfinite(s) | ~np.isfinite(x).all(-1)
        ratio = np.where((s > 0)[..., None], (x - lo[..., None]) / np.where(s > 0, s, 1.0)[..., None], 0.0)
        codes = np.clip(np.rint(np.where(bad[..., None], 0.0, ratio)), 0, 15).astype(np.uint8)
    zero = np.where(bad, 0.0, lo)
    bits = np.where(bad, np.uint16(0x7FC0), bits)
    meta = np.stack([bits, bf16_bits(zero)], axis=-1)
    return codes, np.where(bad, np.nan, s), zero, meta


def _places(lanes):
    """Nibble of each channel inside a row's 128."""
    c = np.arange(128)
    g, rest, per = c // 32, c % 32, 32 // lanes
    return per * (4 * (rest // per) + g) + rest % per


PLACES = {"K": _places(4), "V": _places(8)}


def pack(codes, which):
    """codes uint8 [rows, 4, 32] -> bytes uint8 [rows, 64]."""
    nib = np.zeros((codes.shape[0], 128), dtype=np.uint8)
    nib[:, PLACES[which]] = codes.reshape(-1, 128)
    return nib[:, 0::2] | (nib[:, 1::2] << 4)


def unpack(packed, meta_bits, which):
    """(values, parts) float64 [rows, 128]: what the rows stand for, and |scale code| + |zero| (for error bounds)."""
    packed = np.asarray(packed, dtype=np.uint8).reshape(-1, 64)
    nib = np.empty((packed.shape[0], 128), dtype=np.uint8)
    nib[:, 0::2], nib[:, 1::2] = packed & 15, packed >> 4
    code = nib[:, PLACES[which]].astype(np.float64).reshape(-1, 4, 32)
    m = bf16_value(np.asarray(meta_bits, dtype=np.uint16)).astype(np.float64).reshape(-1, 4, 2)
    with np.errstate(invalid="ignore"):
        step = m[..., :1] * code
    return (step + m[..., 1:]).reshape(-1, 128), (np.abs(step) + np.abs(m[..., 1:])).reshape(-1, 128)


def attend(q, k, v, seen, scale):
    """One head: (o [rows, d], lse [rows], weights [rows, keys]) of softmax(scale q k^T) v over the keys `seen` [rows, keys]
    marks; a row that sees nothing gives 0 and -inf."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    s = np.where(seen, scale * (q @ k.T), -np.inf) if k.shape[0] else np.full((q.shape[0], 0), -np.inf)
    top = s.max(-1, initial=-np.inf)
    e = np.exp(s - np.where(np.isfinite(top), top, 0.0)[:, None])
    total = e.sum(-1)
    w = e / np.where(total > 0, total, 1.0)[:, None]
    with np.errstate(divide="ignore"):
        lse = np.where(total > 0, top + np.log(np.where(total > 0, total, 1.0)), -np.inf)
    o = w @ v if k.shape[0] else np.zeros((q.shape[0], v.shape[1] if v.ndim == 2 else 128))
    return o, lse, w


def window_mask(n, t, window, num_sink):
    """Keys [n] that each of the t queries at the last t positions sees."""
    pos = np.arange(n - t, n)[:, None]
    j = np.arange(n)[None]
    return (j <= pos) & ((j > pos - window) | (j < num_sink))
