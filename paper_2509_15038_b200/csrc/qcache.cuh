// The 4-bit cache: rows of 128 bf16 channels held as 64 bytes of codes and four (scale, zero)
// pairs.  Quantising store (with or without a selection), append, and the way back to bf16.
//
// A group of 32 channels with least value lo and greatest hi is held as
//   s = bf16((hi - lo) / 15),  z = lo,  code = rint((x - z) / s)  (ties to even, 0 .. 15)
// and stands for s * code + z.  The zero needs no rounding (lo is a bf16 value), and the
// rounding of the scale costs nothing either: the codes are formed with the rounded scale, and
// at the top of the range (hi - lo) / s <= 15 (1 + 2^-8) still rounds to 15.
//
// Where the codes sit (chosen for the attention kernel, which wants the operands of its matrix
// instructions without any exchange between lanes):
//   K row: channel 32 g + 8 t + u in nibble u of 32-bit word 4 t + g  (t, g < 4, u < 8)
//   V row: channel 32 g + 4 t + u in nibble u of 16-bit word 4 t + g  (t < 8, g, u < 4)
#pragma once
#include "common.cuh"

namespace curdkv {
namespace qcache {

constexpr int kRowBytes = 64;        // codes of one row of K or V
constexpr int kMetaBytes = 16;       // its four (scale, zero) pairs, bf16 each

struct View {
  uint8_t* K_codes;
  uint8_t* V_codes;
  uint32_t* K_meta;                  // [rows][4]: scale in the low half, zero in the high half
  uint32_t* V_meta;
  int32_t* count;                    // [batch * heads]
  const int32_t* row_start;          // [batch * heads + 1] or nullptr
  int64_t capacity;                  // rows per head, or all rows when row_start is given
};

// First row and number of rows of head p.  Offsets that run backwards or beyond the cache give a
// head without rows (the caller of this function flags it).
__device__ __forceinline__ bool rows_of(const View& c, int64_t p, int64_t& first, int& room) {
  if (c.row_start == nullptr) {
    first = p * c.capacity;
    room = (int)c.capacity;
    return true;
  }
  const int64_t lo = c.row_start[p], hi = c.row_start[p + 1];
  const bool ok = lo >= 0 && hi >= lo && hi <= c.capacity;
  first = ok ? lo : 0;
  room = ok ? (int)(hi - lo) : 0;
  return ok;
}

// rint((x - z) / s) in 64 bits: the definition, for values that the 32-bit path finds next to a
// border between two codes (about one in 10^5).
__device__ __noinline__ float code_exact(float x, float z, float s) {
  const double q = rint(((double)x - (double)z) / (double)s);
  return (float)fmin(fmax(q, 0.0), 15.0);
}

// The eight channels 8 * l16 .. 8 * l16 + 7 of one row: their codes, four bits each from the
// lowest, and the (scale, zero) word of their group, which four neighbouring lanes share.  All 32
// lanes of the warp call this together.
__device__ __forceinline__ uint32_t quantise8(const uint4& v, uint32_t& meta) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  // greatest x and greatest -x side by side; a NaN anywhere in the group wins both
  __nv_bfloat162 top = *reinterpret_cast<const __nv_bfloat162*>(&w[0]), low = top;
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
    top = __hmax2_nan(top, x);
    low = __hmin2_nan(low, x);
  }
  __nv_bfloat162 ext = __halves2bfloat162(__hmax_nan(__low2bfloat16(top), __high2bfloat16(top)),
                                          __hneg(__hmin_nan(__low2bfloat16(low), __high2bfloat16(low))));
#pragma unroll
  for (int o = 1; o <= 2; o <<= 1) {
    uint32_t mine = *reinterpret_cast<const uint32_t*>(&ext);
    const uint32_t other = __shfl_xor_sync(0xffffffffu, mine, o);
    ext = __hmax2_nan(ext, *reinterpret_cast<const __nv_bfloat162*>(&other));
  }
  const float hi = __low2float(ext), lo = -__high2float(ext);
  const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.f));
  const float s = __bfloat162float(sb);
  if (!(s < INFINITY)) {             // a NaN, an infinity or a range beyond fp32: the group is NaN
    meta = 0x7fc0u;
    return 0u;
  }
  meta = (uint32_t)__bfloat16_as_ushort(sb) | (__float_as_uint(lo) & 0xffff0000u);
  const float inv = s > 0.f ? __frcp_rn(s) : 0.f;
  float x[8], r[8];
  unpack_bf16x8(v, x);
  // t carries at most ~3e-6 of absolute error (two roundings of a value below 15.1 and that of
  // 1/s), so a t farther than 2e-5 from every border rounds as the exact ratio does -- where 1/s is a
  // normal number
  bool near = s < 0x1p-120f || s > 0x1p120f;
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const float t = fminf((x[u] - lo) * inv, 15.f);
    r[u] = rintf(t);
    const float e = fabsf(t - r[u]);
    near = near || e > 0.49998f;
  }
  if (near && s > 0.f) {
#pragma unroll 1
    for (int u = 0; u < 8; ++u) r[u] = code_exact(x[u], lo, s);
  }
  // codes are small integers: gather them as digits of two base-16 numbers below 2^16
  const float a = fmaf(r[3], 4096.f, fmaf(r[2], 256.f, fmaf(r[1], 16.f, r[0])));
  const float b = fmaf(r[7], 4096.f, fmaf(r[6], 256.f, fmaf(r[5], 16.f, r[4])));
  return (uint32_t)a | ((uint32_t)b << 16);
}

// Writes one row's codes and metas from the 16 lanes that quantised it (l16 = lane & 15, K rows in
// lanes 0-15, V rows in lanes 16-31).  Called by all 32 lanes; `put` = this lane's row exists.
__device__ __forceinline__ void put_row(const View& c, int64_t row, int half, int l16, uint32_t codes,
                                        uint32_t meta, bool put) {
  const int g = l16 >> 2, t = l16 & 3;
  // V: the two 16-bit words 4 (2t) + g and 4 (2t + 1) + g; lanes of groups g and g ^ 1 exchange
  // one each, and every lane then holds a whole 32-bit word
  const uint32_t give = (g & 1) ? (codes & 0xffffu) : (codes >> 16);
  const uint32_t got = __shfl_xor_sync(0xffffffffu, give, 4);
  const uint32_t v_word = (g & 1) ? (got | (codes & 0xffff0000u)) : ((codes & 0xffffu) | (got << 16));
  const int v_at = 4 * t + 2 * (g & 1) + (g >> 1);
  if (!put) return;
  uint8_t* base = half ? c.V_codes : c.K_codes;
  reinterpret_cast<uint32_t*>(base + row * kRowBytes)[half ? v_at : 4 * t + g] = half ? v_word : codes;
  if (t == 0) (half ? c.V_meta : c.K_meta)[row * 4 + g] = meta;
}

constexpr int kStoreWarps = 8;
constexpr int kStoreRowsPerWarp = 4;                       // rows of K and of V a warp has in flight
constexpr int kStoreRowsPerCta = kStoreWarps * kStoreRowsPerWarp;

struct StoreArgs {
  View cache;
  KvView K, V;
  const int32_t* seqlens;            // or nullptr
  const int32_t* idx;                // or nullptr: every row
  const int32_t* head_counts;        // with idx
  const int32_t* head_offsets;       // packed idx, or nullptr
  int64_t idx_stride;                // fixed idx
  int heads, n_max, ctas_per_head;
  uint32_t* status;                  // or nullptr
};

// Gathers the selected rows and holds them in 4 bits, slot 0 upwards; sets count.
// grid = batch * heads * ctas_per_head, block = 256.
__global__ void __launch_bounds__(kStoreWarps * 32) store_kernel(const StoreArgs a) {
  const int p = blockIdx.x / a.ctas_per_head, part = blockIdx.x % a.ctas_per_head;
  const int b = p / a.heads, h = p % a.heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
  const int n = seq_len_of(a.seqlens, b, a.n_max);
  int64_t first;
  int room;
  bool ok = rows_of(a.cache, p, first, room);
  int64_t offered = n;
  const int32_t* ix = nullptr;
  if (a.idx != nullptr) {
    offered = a.head_counts[p];
    int64_t listed = a.idx_stride, at = (int64_t)p * a.idx_stride;
    if (a.head_offsets != nullptr) {
      at = a.head_offsets[p];
      listed = (int64_t)a.head_offsets[p + 1] - at;
    }
    if (at < 0 || offered < 0 || offered > listed) {       // a count beyond the index row: corrupted
      ok = false;
      offered = at < 0 || offered < 0 || listed < 0 ? 0 : listed;
    }
    ix = a.idx + (at < 0 ? 0 : at);
  }
  const bool lead = part == 0 && threadIdx.x == 0;
  if (lead && !ok) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
  if (lead && offered > room) flag_status(a.status, CURDKV_DEV_CACHE_FULL);
  const int count = (int)(offered < room ? offered : room);
  if (lead) a.cache.count[p] = count;
  const KvView& T = half ? a.V : a.K;
  const __nv_bfloat16* src = T.base + b * T.stride_b + h * T.stride_h;

  for (int t0 = (part * kStoreWarps + warp) * kStoreRowsPerWarp; t0 < count;
       t0 += a.ctas_per_head * kStoreRowsPerCta) {
    int mine = -1;
    if (lane < kStoreRowsPerWarp && t0 + lane < count) {
      mine = ix != nullptr ? __ldg(ix + t0 + lane) : t0 + lane;
      if (mine < 0 || mine >= n) {
        flag_status(a.status, CURDKV_DEV_BAD_INDEX);
        mine = -1;
      }
    }
    uint4 v[kStoreRowsPerWarp];
#pragma unroll
    for (int i = 0; i < kStoreRowsPerWarp; ++i) {
      const int j = __shfl_sync(0xffffffffu, mine, i);
      v[i] = make_uint4(0u, 0u, 0u, 0u);                   // an index outside the sequence: a row of zeros
      if (j >= 0) v[i] = __ldg(reinterpret_cast<const uint4*>(src + (int64_t)j * T.stride_n) + l16);
    }
#pragma unroll
    for (int i = 0; i < kStoreRowsPerWarp; ++i) {
      uint32_t meta;
      const uint32_t codes = quantise8(v[i], meta);
      put_row(a.cache, first + t0 + i, half, l16, codes, meta, t0 + i < count);
    }
  }
}

struct AppendArgs {
  View cache;
  KvView K, V;
  const int32_t* t_new;              // [batch] or nullptr
  int heads, t, chunks;              // chunks of kAppendRows rows per head
  uint32_t* status;
};

constexpr int kAppendRows = 64;      // rows of a head one CTA takes

__device__ __forceinline__ int rows_to_append(const AppendArgs& a, int p, int held, int room, bool& full) {
  int tb = a.t_new != nullptr ? a.t_new[p / a.heads] : a.t;
  tb = tb < 0 ? 0 : (tb > a.t ? a.t : tb);
  full = tb > room - held;
  return full ? room - held : tb;
}

// Holds new rows behind the held ones.  Up to kAppendRows rows per head a head is one CTA's, which
// also moves the counter (one launch); longer blocks take several CTAs, and advance_kernel follows.
// grid = batch * heads * chunks, block = 256.
__global__ void __launch_bounds__(kStoreWarps * 32) append_kernel(const AppendArgs a) {
  const int p = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int b = p / a.heads, h = p % a.heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
  int64_t first;
  int room;
  const bool ok = rows_of(a.cache, p, first, room);
  const int was = a.cache.count[p];
  const int held = was < 0 ? 0 : (was > room ? room : was);
  bool full;
  const int tb = rows_to_append(a, p, held, room, full);
  if (chunk == 0 && threadIdx.x == 0) {
    if (!ok || was != held) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
    if (full) flag_status(a.status, CURDKV_DEV_CACHE_FULL);
  }
  const KvView& T = half ? a.V : a.K;
  const __nv_bfloat16* src = T.base + b * T.stride_b + h * T.stride_h;
  const int end = min(tb, (chunk + 1) * kAppendRows);
  for (int t0 = chunk * kAppendRows + warp; t0 < end; t0 += 2 * kStoreWarps) {
    uint4 v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = t0 + i * kStoreWarps;
      v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (j < end) v[i] = __ldg(reinterpret_cast<const uint4*>(src + (int64_t)j * T.stride_n) + l16);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = t0 + i * kStoreWarps;
      uint32_t meta;
      const uint32_t codes = quantise8(v[i], meta);
      put_row(a.cache, first + held + j, half, l16, codes, meta, j < end);
    }
  }
  if (a.chunks == 1) {
    __syncthreads();                                       // every thread has read the counter
    if (threadIdx.x == 0) a.cache.count[p] = held + tb;
  }
}

// grid = ceil(batch * heads / 256), block = 256.
__global__ void advance_kernel(const AppendArgs a, int problems) {
  const int p = blockIdx.x * blockDim.x + threadIdx.x;
  if (p >= problems) return;
  int64_t first;
  int room;
  rows_of(a.cache, p, first, room);
  const int was = a.cache.count[p], held = was < 0 ? 0 : (was > room ? room : was);
  bool full;
  a.cache.count[p] = held + rows_to_append(a, p, held, room, full);
}

struct ReadArgs {
  View cache;
  const int32_t* idx;                // [batch * heads][rows] or nullptr (slot t)
  __nv_bfloat16* K_out;              // idx or no row_start: [batch * heads][rows][128]; else [all rows][128]
  __nv_bfloat16* V_out;
  int heads, ctas_per_head;
  int64_t rows;                      // output rows per head; 0: packed like the cache
  uint32_t* status;
};

// Eight channels of a row from their codes: bf16(s * code + z), one rounding (fma).
__device__ __forceinline__ uint4 dequantise8(uint32_t codes, uint32_t meta) {
  const float s = __uint_as_float(meta << 16), z = __uint_as_float(meta & 0xffff0000u);
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x0 = fmaf(s, (float)((codes >> (8 * i)) & 15u), z), x1 = fmaf(s, (float)((codes >> (8 * i + 4)) & 15u), z);
    const __nv_bfloat162 x = __floats2bfloat162_rn(x0, x1);
    o[i] = *reinterpret_cast<const uint32_t*>(&x);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Held rows as bf16.  Rows beyond count, and entries of idx that are negative, leave the output as
// it is.  grid = batch * heads * ctas_per_head, block = 256.
__global__ void __launch_bounds__(kStoreWarps * 32) read_kernel(const ReadArgs a) {
  const int p = blockIdx.x / a.ctas_per_head, part = blockIdx.x % a.ctas_per_head;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
  const int g = l16 >> 2, t = l16 & 3;
  int64_t first;
  int room;
  const bool ok = rows_of(a.cache, p, first, room);
  const int was = a.cache.count[p], held = was < 0 ? 0 : (was > room ? room : was);
  if (part == 0 && threadIdx.x == 0 && (!ok || was != held)) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
  const int64_t want = a.idx != nullptr ? a.rows : (a.rows > 0 && a.rows < held ? a.rows : held);
  const int64_t out0 = a.rows > 0 ? (int64_t)p * a.rows : first;
  const uint8_t* codes = half ? a.cache.V_codes : a.cache.K_codes;
  const uint32_t* metas = half ? a.cache.V_meta : a.cache.K_meta;
  __nv_bfloat16* out = half ? a.V_out : a.K_out;
  for (int64_t t0 = (int64_t)(part * kStoreWarps + warp) * kStoreRowsPerWarp; t0 < want;
       t0 += (int64_t)a.ctas_per_head * kStoreRowsPerCta) {
    uint32_t c[kStoreRowsPerWarp], m[kStoreRowsPerWarp];
    int64_t row[kStoreRowsPerWarp];
#pragma unroll
    for (int i = 0; i < kStoreRowsPerWarp; ++i) {
      row[i] = -1;
      if (t0 + i < want) {
        const int64_t j = a.idx != nullptr ? (int64_t)__ldg(a.idx + (int64_t)p * a.rows + t0 + i) : t0 + i;
        if (j >= held && l16 == 0) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
        if (j >= 0 && j < held) row[i] = first + j;
      }
      if (row[i] >= 0) {
        const uint8_t* r = codes + row[i] * kRowBytes;
        if (half) {
          const uint16_t* hw = reinterpret_cast<const uint16_t*>(r);
          c[i] = (uint32_t)hw[8 * t + g] | ((uint32_t)hw[8 * t + 4 + g] << 16);
        } else {
          c[i] = reinterpret_cast<const uint32_t*>(r)[4 * t + g];
        }
        m[i] = metas[row[i] * 4 + g];
      }
    }
#pragma unroll
    for (int i = 0; i < kStoreRowsPerWarp; ++i)
      if (row[i] >= 0)
        __stcs(reinterpret_cast<uint4*>(out + (out0 + t0 + i) * 128) + l16, dequantise8(c[i], m[i]));
  }
}

}  // namespace qcache
}  // namespace curdkv
