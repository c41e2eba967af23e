// The 4-bit cache: rows of 128 bf16 channels held as 64 bytes of codes and four (scale, zero)
// pairs.  Quantising store (with or without a selection), append, and the way back to bf16.
//
// A group of 32 channels with least value lo and greatest hi is held as
//   s = bf16((hi - lo) * fp32(1/15)),  z = lo,  code = rint((x - z) / s)  (ties to even, 0 .. 15)
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

// ---- asynchronous copies, 16 bytes a thread
__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
// 16 bytes global -> shared, zeros when `live` is false (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

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

// The exact code of each of eight values, given one that is off by at most one.  With r that code,
// e = (x - z) - r s is formed without error (the difference by TwoSum, r s by the fused multiply-add)
// and compared with s / 2; ties go to the even code.
__device__ __noinline__ void codes_exact(const float (&x)[8], float z, float s, float (&r)[8]) {
  const float h = 0.5f * s;
#pragma unroll 1
  for (int u = 0; u < 8; ++u) {
    if (s < 0x1p-100f || s > 0x1p100f) {                   // products below may leave fp32's range
      r[u] = (float)fmin(fmax(rint(((double)x[u] - (double)z) / (double)s), 0.0), 15.0);
      continue;
    }
    const float d = __fsub_rn(x[u], z), back = __fsub_rn(d, x[u]);
    float low = __fadd_rn(__fsub_rn(x[u], __fsub_rn(d, back)), __fsub_rn(-z, back));   // x - z = d + low
    if (fabsf(low) < 0x1p-50f * s) low = 0.f;              // beyond 64-bit arithmetic's sight
    const float e = __fmaf_rn(-r[u], s, d), over = (fabsf(e) - h) + copysignf(1.f, e) * low;
    const bool odd = (int)r[u] & 1;
    if (over > 0.f || (over == 0.f && odd)) r[u] += copysignf(1.f, e);
    r[u] = fminf(fmaxf(r[u], 0.f), 15.f);
  }
}

// Pairs of fp32 values in one instruction.
__device__ __forceinline__ uint64_t f2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unf2(uint64_t r, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul_f2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma_f2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t sub_f2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Eight channels of one group: their codes, four bits each from the lowest, and the (scale, zero)
// word of the group, which four neighbouring lanes share.  All 32 lanes of the warp call this together.
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
  const uint32_t tu = *reinterpret_cast<const uint32_t*>(&top), lu = *reinterpret_cast<const uint32_t*>(&low) ^ 0x80008000u;
  const uint32_t one = __byte_perm(tu, lu, 0x5410), two = __byte_perm(tu, lu, 0x7632);
  __nv_bfloat162 ext = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&one), *reinterpret_cast<const __nv_bfloat162*>(&two));
#pragma unroll
  for (int o = 1; o <= 2; o <<= 1) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<const uint32_t*>(&ext), o);
    ext = __hmax2_nan(ext, *reinterpret_cast<const __nv_bfloat162*>(&other));
  }
  const uint32_t eu = *reinterpret_cast<const uint32_t*>(&ext);
  const float hi = __uint_as_float(eu << 16), lo = -__uint_as_float(eu & 0xffff0000u);
  const __nv_bfloat16 sb = __float2bfloat16_rn(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f));
  const float s = __bfloat162float(sb);
  if (!(s < INFINITY)) {             // a NaN, an infinity or a range beyond fp32: the group is NaN
    meta = 0x7fc0u;
    return 0u;
  }
  meta = (uint32_t)__bfloat16_as_ushort(sb) | (__float_as_uint(lo) & 0xffff0000u);
  // The ratio (x - lo) / s by the approximate reciprocal and one correction with the exact residual
  // (Markstein): where the ratio is a representable number, as every tie between two codes is, that
  // number exactly.  Ties are common (x - lo and s are both short numbers: one value in 300 of cached rows).
  // A ratio that is no tie can only round to one, or x - lo to fewer bits than it has, where |x| or |lo| is
  // below 2^-12 s; such rows, and scales whose reciprocal is no normal number, are decided exactly.
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  uint32_t least = w[0] & 0x7fff7fffu;
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    const uint32_t x = w[i] & 0x7fff7fffu;
    const __nv_bfloat162 m = __hmin2(*reinterpret_cast<const __nv_bfloat162*>(&least), *reinterpret_cast<const __nv_bfloat162*>(&x));
    least = *reinterpret_cast<const uint32_t*>(&m);
  }
  const float tiny = fminf(fminf(__uint_as_float(least << 16), __uint_as_float(least & 0xffff0000u)), fabsf(lo));
  const bool hard = s < 0x1p-100f || s > 0x1p100f;
  if (hard) inv = 0.f;
  const uint64_t lo2 = f2(lo, lo), inv2 = f2(inv, inv), ns2 = f2(-s, -s), magic = f2(12582912.f, 12582912.f);   // 1.5 * 2^23
  uint64_t r2[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t d2 = sub_f2(f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), lo2);
    const uint64_t q2 = mul_f2(d2, inv2), t2 = fma_f2(fma_f2(ns2, q2, d2), inv2, q2);
    r2[i] = sub_f2(add_f2(t2, magic), magic);              // rounded to an integer, ties to even
  }
  if ((hard || tiny < 0x1p-12f * s) && s > 0.f) {
    float x[8], r[8];
    unpack_bf16x8(v, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) unf2(r2[i], r[2 * i], r[2 * i + 1]);
    codes_exact(x, lo, s, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) r2[i] = f2(r[2 * i], r[2 * i + 1]);
  }
  // codes are small integers: gather them as digits (even and odd ones apart, then together), and
  // take the sums' bits from above 2^23
  const uint64_t by256 = f2(256.f, 256.f);
  float e01, o01, e23, o23;
  unf2(fma_f2(r2[1], by256, r2[0]), e01, o01);
  unf2(fma_f2(r2[3], by256, r2[2]), e23, o23);
  return __byte_perm(__float_as_uint(fmaf(o01, 16.f, e01) + 8388608.f), __float_as_uint(fmaf(o23, 16.f, e23) + 8388608.f), 0x5410);
}

// How a warp takes rows: lanes 0-15 four rows of K, lanes 16-31 the same four rows of V; the four lanes
// t of a row take channels 32 g + 8 t .. + 7 of every group g.  That is a 64-byte run of the row for each
// g, and the codes of a lane are 16 bytes of the cache's row, whichever tensor.
struct RowLane {
  int half, row, t;
  __device__ __forceinline__ RowLane() {
    const int lane = threadIdx.x & 31;
    half = lane >> 4;
    row = (lane >> 2) & 3;
    t = lane & 3;
  }
};
// 16-bit words g of two 8-channel runs <-> the 16-bit words of a V row's 16 bytes (runs 2 t and
// 2 t + 1 of four channels, groups ascending in each)
__device__ __forceinline__ uint4 to_v_order(const uint32_t (&w)[4]) {
  return make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410),
                    __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
}
__device__ __forceinline__ void from_v_order(const uint4& v, uint32_t (&w)[4]) {
  w[0] = __byte_perm(v.x, v.z, 0x5410);
  w[1] = __byte_perm(v.x, v.z, 0x7632);
  w[2] = __byte_perm(v.y, v.w, 0x5410);
  w[3] = __byte_perm(v.y, v.w, 0x7632);
}
// Quantises this lane's 32 channels and writes them to cache row `row` when `put`.  Called by all 32
// lanes.
__device__ __forceinline__ void put_row(const View& c, int64_t row, const RowLane& l, const uint4 (&v)[4], bool put) {
  uint32_t w[4], m[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) w[g] = quantise8(v[g], m[g]);
  if (!put) return;
  const uint4 codes = l.half ? to_v_order(w) : make_uint4(w[0], w[1], w[2], w[3]);
  reinterpret_cast<uint4*>(l.half ? c.V_codes : c.K_codes)[row * 4 + l.t] = codes;
  if (l.t == 0) reinterpret_cast<uint4*>(l.half ? c.V_meta : c.K_meta)[row] = make_uint4(m[0], m[1], m[2], m[3]);
}
__device__ __forceinline__ void get_row(const __nv_bfloat16* src, const RowLane& l, bool live, uint4 (&v)[4]) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    v[g] = make_uint4(0u, 0u, 0u, 0u);
    if (live) v[g] = __ldg(reinterpret_cast<const uint4*>(src) + 4 * g + l.t);
  }
}

constexpr int kStoreWarps = 8;
constexpr int kStoreTurns = 2;                             // runs of four rows a warp has in flight
constexpr int kStoreRowsPerWarp = 4 * kStoreTurns;
constexpr int kStoreRowsPerCta = kStoreWarps * kStoreRowsPerWarp;

struct StoreArgs {
  View cache;
  KvView K, V;
  const int32_t* seqlens;            // or nullptr
  const int32_t* idx;                // or nullptr: every row
  const int32_t* head_counts;        // with idx
  const int32_t* head_offsets;       // packed idx, or nullptr
  int64_t idx_stride;                // fixed idx; packed: entries of idx, or 0
  int heads, n_max, ctas_per_head;
  uint32_t* status;                  // or nullptr
};

// Gathers the selected rows and holds them in 4 bits, slot 0 upwards; sets count.
// 435712 rows of 256 heads (223 MB read, 70 MB written): 81 us, 3.6 TB/s.  What bounds it is the quantiser's
// instructions, some 125 per 8 x 32 channels (72 % of the issue slots, 55 % of the integer pipe).  With the next
// turn's rows in registers instead of shared memory 94 us (80 registers: three CTAs an SM where this runs
// four, and one turn ahead); with half as many CTAs 5 us more, since the last ones run alone.
// grid = batch * heads * ctas_per_head, block = 256.
__global__ void __launch_bounds__(kStoreWarps * 32, 4) store_kernel(const StoreArgs a) {
  __shared__ uint4 ring[kStoreWarps][3][4][32];            // [warp][turn][group][lane]
  const int p = blockIdx.x / a.ctas_per_head, part = blockIdx.x % a.ctas_per_head;
  const int b = p / a.heads, h = p % a.heads;
  const int warp = threadIdx.x >> 5;
  const RowLane l;
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
      if (a.idx_stride > 0) listed = min(listed, a.idx_stride - at);       // nothing behind idx is read
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
  const KvView& T = l.half ? a.V : a.K;
  const __nv_bfloat16* src = T.base + b * T.stride_b + h * T.stride_h;

  // A turn of the warp is four rows of K and of V.  The rows of the next two turns are in flight while this
  // one's are quantised, as asynchronous copies into shared memory (every lane reads back what it copied
  // itself: no barrier), and the index of the third: a turn's chain of two loads (index, row) would
  // otherwise be waited for.
  const int stride = a.ctas_per_head * kStoreWarps * 4;
  const uint32_t mine = smem_addr(&ring[warp][0][0][threadIdx.x & 31]);
  bool bad = false;
  auto index_of = [&](int slot) { return slot >= count ? -1 : (ix != nullptr ? __ldg(ix + slot) : slot); };
  auto fetch = [&](int stage, int j, int slot) {           // (the index is looked at here, a turn after its load)
    const bool live = j >= 0 && j < n;
    bad = bad || (!live && slot < count);                  // outside the sequence: a row of zeros
    const __nv_bfloat16* row = src + (live ? (int64_t)j * T.stride_n : 0) + 8 * l.t;
#pragma unroll
    for (int g = 0; g < 4; ++g) copy16(mine + (uint32_t)(stage * 4 + g) * 512u, row + 32 * g, live);
    copy_commit();
  };
  int slot = (part * kStoreWarps + warp) * 4 + l.row, stage = 0;
  fetch(0, index_of(slot), slot);
  fetch(1, index_of(slot + stride), slot + stride);
  int next = index_of(slot + 2 * stride);
  for (; slot - l.row < count; slot += stride) {
    fetch(stage == 0 ? 2 : stage - 1, next, slot + 2 * stride);
    next = index_of(slot + 3 * stride);
    copy_wait<2>();
    uint4 v[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) v[g] = ring[warp][stage][g][threadIdx.x & 31];
    put_row(a.cache, first + slot, l, v, slot < count);
    stage = stage == 2 ? 0 : stage + 1;
  }
  copy_wait<0>();
  if (bad) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
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
// also moves the counter (one launch); longer blocks take several CTAs, and advance_kernel follows.  One
// row of 8 heads: the launch and one pass over dependent loads (counter, row), some 3 us.
// grid = batch * heads * chunks, block = 256.
__global__ void __launch_bounds__(kStoreWarps * 32) append_kernel(const AppendArgs a) {
  const int p = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int b = p / a.heads, h = p % a.heads;
  const int warp = threadIdx.x >> 5;
  const RowLane l;
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
  const KvView& T = l.half ? a.V : a.K;
  const __nv_bfloat16* src = T.base + b * T.stride_b + h * T.stride_h;
  const int end = min(tb, (chunk + 1) * kAppendRows);
  for (int t0 = chunk * kAppendRows + 4 * warp; t0 < end; t0 += 4 * kStoreWarps) {
    const int j = t0 + l.row;
    uint4 v[4];
    get_row(src + (int64_t)j * T.stride_n, l, j < end, v);
    put_row(a.cache, first + held + j, l, v, j < end);
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

// Eight channels of a row from their codes: bf16(s * code + z), fp32 inside.
__device__ __forceinline__ uint4 dequantise8(uint32_t codes, uint32_t meta) {
  const float s = __uint_as_float(meta << 16), z = __uint_as_float(meta & 0xffff0000u);
  const uint64_t s2 = f2(s, s), z2 = f2(z, z), base = f2(8388608.f, 8388608.f);
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // the code as a float: its bits under the exponent of 2^23, minus 2^23
    const uint64_t c2 = sub_f2(f2(__uint_as_float(((codes >> (8 * i)) & 15u) | 0x4b000000u),
                                  __uint_as_float(((codes >> (8 * i + 4)) & 15u) | 0x4b000000u)), base);
    float x0, x1;
    unf2(fma_f2(s2, c2, z2), x0, x1);
    const __nv_bfloat162 x = __floats2bfloat162_rn(x0, x1);
    o[i] = *reinterpret_cast<const uint32_t*>(&x);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Held rows as bf16.  Rows beyond count, and entries of idx that are negative, leave the output as
// it is.  What bounds it are the bytes: 435712 rows, 70 MB read and 223 MB written, 50 us, 5.9 TB/s.
// grid = batch * heads * ctas_per_head, block = 256.
__global__ void __launch_bounds__(kStoreWarps * 32) read_kernel(const ReadArgs a) {
  const int p = blockIdx.x / a.ctas_per_head, part = blockIdx.x % a.ctas_per_head;
  const int warp = threadIdx.x >> 5;
  const RowLane l;
  int64_t first;
  int room;
  const bool ok = rows_of(a.cache, p, first, room);
  const int was = a.cache.count[p], held = was < 0 ? 0 : (was > room ? room : was);
  if (part == 0 && threadIdx.x == 0 && (!ok || was != held)) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
  const int64_t want = a.idx != nullptr ? a.rows : (a.rows > 0 && a.rows < held ? a.rows : held);
  const int64_t out0 = a.rows > 0 ? (int64_t)p * a.rows : first;
  const uint4* codes = reinterpret_cast<const uint4*>(l.half ? a.cache.V_codes : a.cache.K_codes);
  const uint4* metas = reinterpret_cast<const uint4*>(l.half ? a.cache.V_meta : a.cache.K_meta);
  __nv_bfloat16* out = l.half ? a.V_out : a.K_out;
  for (int64_t t0 = (int64_t)(part * kStoreWarps + warp) * kStoreRowsPerWarp; t0 < want;
       t0 += (int64_t)a.ctas_per_head * kStoreRowsPerCta) {
    uint4 c[kStoreTurns], m[kStoreTurns];
    bool live[kStoreTurns];
#pragma unroll
    for (int i = 0; i < kStoreTurns; ++i) {
      const int64_t slot = t0 + 4 * i + l.row;
      int64_t j = -1;
      if (slot < want) {
        j = a.idx != nullptr ? (int64_t)__ldg(a.idx + (int64_t)p * a.rows + slot) : slot;
        if (j >= held) {
          flag_status(a.status, CURDKV_DEV_BAD_INDEX);
          j = -1;
        }
      }
      live[i] = j >= 0;
      if (live[i]) {
        c[i] = __ldg(codes + (first + j) * 4 + l.t);
        m[i] = __ldg(metas + first + j);
      }
    }
#pragma unroll
    for (int i = 0; i < kStoreTurns; ++i) {
      if (!live[i]) continue;
      uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
      if (l.half) from_v_order(c[i], w);
      const uint32_t mw[4] = {m[i].x, m[i].y, m[i].z, m[i].w};
      uint4* dst = reinterpret_cast<uint4*>(out + (out0 + t0 + 4 * i + l.row) * 128) + l.t;
#pragma unroll
      for (int g = 0; g < 4; ++g) __stcs(dst + 4 * g, dequantise8(w[g], mw[g]));
    }
  }
}

}  // namespace qcache
}  // namespace curdkv
