// Attention of a few query rows per KV head over a long cache: the generation step.  Two caches,
// one kernel: rows held in 4 bits (curdkv_qcache_attention) and bf16 rows of which a sliding window
// and the first tokens are visible (curdkv_attention_window with few queries).
//
// What has to be moved are the cache's bytes, each once.  4-bit rows are bound by the instructions that
// unpack and weigh them instead (some 281 per 16 keys of a warp, integer pipe 59 % busy): 64 heads of 131072
// rows and 4 queries 235 us, 5.7 TB/s (273 when the device's power limit holds its clock down); a copy that
// only loads takes 196.  bf16 rows are bound by their loads: 128 heads with a window of 4096 46 us, 5.8 TB/s.
// The tiles of all items -- an item is a head and a block of query rows -- form one line, and every CTA takes
// an equal run of it, whatever the items' lengths: whole items are finished where they are, the partial
// results of an item that several CTAs share are joined by a second kernel.  (128 heads of 2048 to 16384 rows:
// 51 us; with a CTA per item, as long as the longest, it was 70 where equal runs took 49.)  Where that gains
// little an item has a CTA or a cluster of two, four or eight to itself, whose parts are joined through
// distributed shared memory in the same launch: 8 heads of 1702 rows 7.4 us, 12.7 with equal runs and the second
// kernel; 128 windows of 4096 46 us against 53.  A CTA's warps take its tiles in turn, each warp with its own ring of
// tiles in shared memory, filled by 16-byte asynchronous copies (rows that do not exist are filled with
// zeros, so nothing behind a head's last row is ever read).  No barrier stands in the key loop.  Per 16
// keys a warp forms
//   S^T [16 keys x 8 queries] = K Q^T        m16n8k16, keys as the M side: with the few queries of
//   O^T [128 x 8 queries]    += V^T P^T      a KV head as N = 8 half the instructions that a layout
//                                            with 16 padded queries as M would need
// and between the two the online softmax: a warp's reference moves only when some logit exceeds it by more
// than 2^slack (one vote per tile), and since S^T and O^T hold a query in the same lanes the rescale needs
// no exchange.  P^T reaches the second product's operand layout by two 8x8 transposes (movmatrix).  Sums,
// references and accumulators are fp32; the weights enter the second product as fp16 (4-bit rows) or bf16
// (bf16 rows), at most 2^-11 / 2^-8 of each weight off; the row sum is taken over the unrounded weights.
//
// 4-bit rows cost five integer instructions per eight values and no conversion: a code left in the
// low bits of a half is the fp16 subnormal code * 2^-24 (or code * 2^-20 one nibble up), which the
// tensor cores multiply exactly.  The scales are applied outside: on the K side to the products of
// each group of 32 channels (S = sum_g s_g (codes_g . q_g) + sum_g z_g sum(q_g), the second sum one
// more matrix instruction whose A operand is the zeros), on the V side to the weights (one set per
// group, P_g = p * s_g), with the zeros as a further instruction.
//
// The values' magnitude is kept out of the weights' 16 bits.  A warp holds one power of two 2^E for V: scales
// and zeros relative to it are exact in fp16, and have bits enough, as long as every scale of a tile lies below
// 2^E but not more than 2^8 to 2^14 below (the fewer keys, the more), and every zero in [2^(E-17), 2^(E+14)), or
// is 0 (a vote per tile).  E follows the tiles: one that lies elsewhere but fits by itself brings its own.  A tile
// that fits nowhere -- groups or rows further apart than that, or a NaN or an infinity, which may meet its own
// group's channels only -- takes its products in bf16 instead, weights times scale split into two pieces: 16 bits,
// at fp32's range.  So does one that lies far below what went before: fp16 weights in the accumulators' unit
// would lose their bits.
// O^T is held in units of 2^(T + E - lift) and the row sum in units of 2^(R - lift), R the reference of the
// logits alone: what a row's values are like has no part in the sum.  T, E and R are whole numbers, so that
// every rescale is a power of two.  What contributes less than 2^-90 of the largest value held may be lost.
#pragma once
#include "qcache.cuh"

namespace curdkv {
namespace token {

constexpr int kStages = 3;
// Log2 units a logit may exceed the running maximum; fp16 weights are 2^(x - m + kLift): at most 2^15.
template <bool Q4>
__host__ __device__ constexpr float slack() { return Q4 ? 4.f : 6.f; }
constexpr float kLift = 11.f;
// A tile's products are taken in fp16 when its scales lie in [2^(E - span), 2^E) and its zeros in
// [2^(E - kZeroDown), 2^(E + kZeroUp)), where both are exact.  Weight times scale then loses bits below 2^-14, by at
// most 2^-25 a key, of 2^(kLift - 1 - span - kFall) that the key of the largest logit has: 2^-10 of the sum of magnitudes
// for 2^n keys, were all errors alike, with a span of 24 - n.
constexpr int kZeroUp = 14, kZeroDown = 17;
constexpr int kLeastSpan = 8, kMostSpan = 14;
__device__ __forceinline__ int span_of(int keys) { return min(max(__clz(max(keys - 1, 1)) - 8, kLeastSpan), kMostSpan); }
constexpr int kLeastE = -126, kMostE = 112;                // 2^-E is a normal number, and an infinite zero is outside
constexpr int kMostAbove = 60;       // how far values may lie above 2^E
constexpr int kFall = 1;             // how far E may fall while the accumulators' unit stays: T - R at most

struct Args {
  const __nv_bfloat16* Q;            // [batch][q_heads][q_n][128], strides in elements
  int64_t q_sb, q_sh, q_sn;
  __nv_bfloat16* O;
  int64_t o_sb, o_sh, o_sn;
  float* lse;                        // [batch][q_heads][q_n] or nullptr
  int heads, group, q_n;             // query heads per KV head; query tokens
  int rows, blocks;                  // rows = group * q_n, row r = token r / group, head r % group
  int items;                         // batch * heads * blocks
  int ctas;                          // runs the tiles are cut into; 0: a cluster of 2^split CTAs per item
  int split;
  float scale_log2;                  // scale * log2(e)
  // 4-bit rows
  qcache::View cache;
  // bf16 rows
  KvView K, V;
  const int32_t* seqlens;
  const int32_t* q_lens;
  int n_max, num_sink, window;
  // partial results, two per CTA (of the item its run begins in, of the one it ends in): [8 NT] references,
  // sums and units (Part), [8 NT][128] sums of values; and where each item begins on the line, [items + 1]
  float* part_ml;
  float* part_o;
  int64_t* begins;
  uint32_t* status;
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// A cluster's barrier, and shared memory of its CTA `rank`.  The barrier, like the matrix instructions, is of the
// aligned kind: a warp has to come to it with all its lanes together, whatever one of them did alone before.
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 peer_float4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// 2^(e - 127) for 1 <= e <= 253, and 0 below
__device__ __forceinline__ float pow2_biased(int e) { return __int_as_float(e > 0 ? e << 23 : 0); }
// 2^d for whole d < 127, 0 below 2^-126, and back: whole numbers pass through the low bits of 1.5 * 2^23 + d
// (the conversion instructions take several times as long)
__device__ __forceinline__ float pow2_whole(float d) {
  return __int_as_float(__float_as_int(fmaxf(d, -127.f) + (12582912.f + 127.f)) << 23);
}
__device__ __forceinline__ int exponent_of(float pow2) { return (__float_as_int(pow2) >> 23) - 127; }
__device__ __forceinline__ float whole_of(float pow2) {
  return __int_as_float((__float_as_int(pow2) >> 23) + 0x4b400000) - (12582912.f + 127.f);
}

// What a warp, or several, have of one query: sum = sum of 2^(x - ref), and sums of values in units of
// 2^(ref + unit), where the unit says how large the values are (0 for bf16 rows).
struct Part {
  float ref, sum, unit;
};
// Joining parts: `all` is the largest reference, `unit` the largest of unit + (ref - all).  A part's sum
// counts 2^(ref - all), its values 2^(unit + (ref - all) - that unit).
__device__ __forceinline__ float above(const Part& p, float all) { return p.unit + (p.ref - all); }
__device__ __forceinline__ float share(float d, float all) { return all == -INFINITY ? 1.f : exp2_approx(d); }   // (all -inf: zeros, or NaN)

template <bool Q4>
struct Tile {                                              // one warp's stage
  static constexpr int kKeys = Q4 ? 32 : 16;
  static constexpr int kK = 0;
  static constexpr int kV = kKeys * (Q4 ? qcache::kRowBytes : 256);
  static constexpr int kKMeta = 2 * kV;
  static constexpr int kVMeta = kKMeta + (Q4 ? kKeys * qcache::kMetaBytes : 0);
  static constexpr int kBytes = kVMeta + (Q4 ? kKeys * qcache::kMetaBytes : 0);
  // V's scales and zeros in fp16, pairs of keys side by side: [key pair][group] each
  static constexpr int kScaled = Q4 ? kKeys * 8 * 2 : 0;
  static constexpr int kWarpBytes = kStages * kBytes + kScaled;
};
// Four warps a CTA, one on each of the SM's schedulers (six a CTA, two CTAs, left two schedulers with
// twice the warps of the others), and as many CTAs as registers and shared memory hold: one streams
// while another begins or ends an item.
constexpr int kWarps = 4, kThreads = kWarps * 32;
template <bool Q4, int NT>
__host__ __device__ constexpr int ctas_per_sm() {
  return Q4 && NT == 1 ? 3 : 2;
}
template <bool Q4, int NT>
constexpr int smem_bytes() {
  constexpr int ring = kWarps * Tile<Q4>::kWarpBytes;
  constexpr int merge = kWarps * 8 * NT * 132 * 4;         // the warps' sums meet in the ring's space
  return ring > merge ? ring : merge;
}

// Keys a block of query rows sees, as a run of `total` positions u: row u for u < sinks, row
// first + (u - sinks) above.
struct Seen {
  int sinks, first, total;
  __device__ __forceinline__ int row(int u) const { return u < sinks ? u : first + (u - sinks); }
};

// One item: its head, its query rows [r0, r1), and the keys these see.
template <bool Q4, int NT>
struct Item {
  int b, h, p, blk, r0, r1;
  Seen seen;
  int64_t first_row;                                       // 4-bit rows: of the head
  int pos0, q_live;                                        // position of query token 0; tokens that exist
  bool ok;                                                 // counters in range
  int tiles;
  __device__ __forceinline__ Item(const Args& a, int item) {
    p = item / a.blocks;
    blk = item % a.blocks;
    b = p / a.heads;
    h = p % a.heads;
    r0 = blk * 8 * NT;
    r1 = min(a.rows, r0 + 8 * NT);
    pos0 = 0;
    q_live = a.q_n;
    first_row = 0;
    ok = true;
    if (Q4) {
      int room;
      ok = qcache::rows_of(a.cache, p, first_row, room);
      const int was = a.cache.count[p], held = was < 0 ? 0 : (was > room ? room : was);
      ok = ok && was == held;
      seen.sinks = 0;
      seen.first = 0;
      seen.total = held;
    } else {
      const int n = seq_len_of(a.seqlens, b, a.n_max);
      if (a.q_lens != nullptr) q_live = min(max(a.q_lens[b], 0), a.q_n);
      pos0 = n - q_live;
      const int i0 = r0 / a.group, i1 = min((r1 - 1) / a.group, q_live - 1);   // tokens of the block
      const int hi = i1 >= i0 ? max(pos0 + i1 + 1, 0) : 0; // keys [0, hi) may be seen
      const int lo = a.window > 0 ? (int)min((int64_t)hi, max((int64_t)0, (int64_t)pos0 + i0 + 1 - a.window)) : hi;
      seen.sinks = min(a.num_sink, lo);
      seen.first = lo;
      seen.total = seen.sinks + hi - lo;
    }
    tiles = (seen.total + Tile<Q4>::kKeys - 1) / Tile<Q4>::kKeys;
  }
};

// CTA whose run holds tile x of a line of `total` tiles cut into `runs` runs [i total / runs, ...).
__device__ __forceinline__ int cta_of(int64_t x, int64_t total, int64_t runs) { return (int)(((x + 1) * runs - 1) / total); }

// V's 16-bit words number g of four-bit rows `key` and `key` + 1 of a stage side by side, one register a group.
__device__ __forceinline__ void v_words(const unsigned char* st, int key, int g, uint32_t (&y)[4]) {
  uint2 v[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = (key + k) * 4 + (g >> 1), line = c >> 3;
    v[k] = *reinterpret_cast<const uint2*>(st + Tile<true>::kV + line * 128 + (((c & 7) ^ (2 * (line & 3))) * 16) + 8 * (g & 1));
  }
  y[0] = __byte_perm(v[0].x, v[1].x, 0x5410);
  y[1] = __byte_perm(v[0].x, v[1].x, 0x7632);
  y[2] = __byte_perm(v[0].y, v[1].y, 0x5410);
  y[3] = __byte_perm(v[0].y, v[1].y, 0x7632);
}

// O^T += V^T P^T of a tile whose scales and zeros fp16 does not hold: in bf16, weights (times scale) in two pieces; codes as
// numbers, those one nibble up times 16 as in the other form, and 2^-24 with the scales, so that the units are the same.
// (Some 1.8 times the other form's time: 64 heads of 131072 rows, every tile so, 425 us against 235.  As a
// function called with copies of the accumulators four times.)
template <int NT>
__device__ __forceinline__ void wide_products(float (&acc)[NT][8][4], float (&accz)[NT][4], const float (&weights)[NT][2][4],
                                              const unsigned char* st, float inv) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  auto pieces = [&](float a, float b, uint32_t& most, uint32_t& rest) {
    const uint32_t top2 = pack_bf16(a, b);
    most = transpose8x8(top2);
    rest = transpose8x8(pack_bf16(a - __uint_as_float(top2 << 16), b - __uint_as_float(top2 & 0xffff0000u)));
  };
  auto number = [](uint32_t code) {                        // 0 .. 15 in each half -> bf16
    const uint32_t up = code | 0x43004300u, base = 0x43004300u;                // 128 + code, 128
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&up), *reinterpret_cast<const __nv_bfloat162*>(&base));
    return *reinterpret_cast<const uint32_t*>(&d);
  };
  auto times16 = [](uint32_t v) {
    const __nv_bfloat162 d = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&v), __float2bfloat162_rn(16.f));
    return *reinterpret_cast<const uint32_t*>(&d);
  };
#pragma unroll
  for (int kb16 = 0; kb16 < 2; ++kb16) {
    const uint32_t* meta = reinterpret_cast<const uint32_t*>(st + Tile<true>::kVMeta) + kb16 * 64;
    uint32_t y[2][4], z[2] = {0u, 0u};
    v_words(st, kb16 * 16 + 2 * t, g, y[0]);
    v_words(st, kb16 * 16 + 8 + 2 * t, g, y[1]);
    if (g < 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        z[i] = pack_bf16(__uint_as_float(meta[(8 * i + 2 * t) * 4 + g] & 0xffff0000u) * inv,
                         __uint_as_float(meta[(8 * i + 2 * t + 1) * 4 + g] & 0xffff0000u) * inv);
    }
    __syncwarp();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float(&w)[4] = weights[nt][kb16];
      uint32_t most[2], rest[2];
      pieces(w[0], w[1], most[0], rest[0]);
      pieces(w[2], w[3], most[1], rest[1]);
      mma_bf16(accz[nt], z[0], 0u, z[1], 0u, most[0], most[1]);
      mma_bf16(accz[nt], z[0], 0u, z[1], 0u, rest[0], rest[1]);
    }
#pragma unroll
    for (int gr = 0; gr < 4; ++gr) {
      uint32_t v[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[i][k] = number((y[i][gr] >> (4 * k)) & 0x000f000fu);
          if (k & 1) v[i][k] = times16(v[i][k]);
        }
      const float sa = __uint_as_float(meta[g * 4 + gr] << 16) * inv * 0x1p-24f;
      const float sb = __uint_as_float(meta[(8 + g) * 4 + gr] << 16) * inv * 0x1p-24f;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float(&w)[4] = weights[nt][kb16];
        uint32_t most[2], rest[2];
        pieces(w[0] * sa, w[1] * sa, most[0], rest[0]);
        pieces(w[2] * sb, w[3] * sb, most[1], rest[1]);
        mma_bf16(acc[nt][2 * gr], v[0][0], v[0][1], v[1][0], v[1][1], most[0], most[1]);
        mma_bf16(acc[nt][2 * gr], v[0][0], v[0][1], v[1][0], v[1][1], rest[0], rest[1]);
        mma_bf16(acc[nt][2 * gr + 1], v[0][2], v[0][3], v[1][2], v[1][3], most[0], most[1]);
        mma_bf16(acc[nt][2 * gr + 1], v[0][2], v[0][3], v[1][2], v[1][3], rest[0], rest[1]);
      }
    }
  }
}

constexpr int kMostSplit = 3;                              // log2 of the CTAs of a cluster
constexpr int kMostItems = 8192;                           // items that are put on one line

template <bool Q4, int NT>
__global__ void __launch_bounds__(kThreads, (ctas_per_sm<Q4, NT>())) attend_kernel(const Args a) {
  using T = Tile<Q4>;
  constexpr int KB = T::kKeys / 16;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ Part s_part[kWarps][8 * NT];
  __shared__ float4 s_ml[8 * NT];                          // the CTA's references, sums and units
  __shared__ int64_t s_sum[kWarps], s_at;
  __shared__ int s_item;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // the joining kernel waits for this one's end

  // ------------------------------------------------------------ this CTA's run of tiles
  const int rank = blockIdx.x & ((1 << a.split) - 1);     // (split is 0 where the line is cut)
  int item_no = blockIdx.x >> a.split;
  int64_t off = 0, left_over = 1;                          // first tile inside the item; tiles of the run
  if (a.ctas > 0) {
    // every CTA sums up the items' tiles: a run of items per thread, then over the threads
    const int each = (a.items + kThreads - 1) / kThreads, e0 = min(tid * each, a.items), e1 = min(e0 + each, a.items);
    int64_t mine = 0;
    int tiles0 = 0;                                        // of the thread's first item
    for (int e = e0; e < e1; ++e) {
      const Item<Q4, NT> it(a, e);
      mine += it.tiles;
      if (e == e0) tiles0 = it.tiles;
      if (e % a.ctas != (int)blockIdx.x) continue;
      if (!it.ok) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
      if (it.tiles == 0) {                                 // nothing to see: zeros, written here
        for (int r = it.r0; r < it.r1; ++r) {
          const int i = r / a.group, hq = it.h * a.group + r % a.group;
          if (i >= it.q_live) continue;
          uint4* o = reinterpret_cast<uint4*>(a.O + it.b * a.o_sb + (int64_t)hq * a.o_sh + (int64_t)i * a.o_sn);
          for (int c = 0; c < 16; ++c) o[c] = make_uint4(0u, 0u, 0u, 0u);
          if (a.lse != nullptr) a.lse[((int64_t)it.b * a.heads * a.group + hq) * a.q_n + i] = -INFINITY;
        }
      }
    }
    int64_t upto = mine;                                   // inclusive sum over the warp's threads
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) s_sum[warp] = upto;
    __syncthreads();
    int64_t before = upto - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += s_sum[w];
      total += s_sum[w];
    }
    const int64_t runs = min((int64_t)a.ctas, total);      // none of them empty
    const int64_t lo = blockIdx.x < runs ? blockIdx.x * total / runs : 0;
    const int64_t hi = blockIdx.x < runs ? (blockIdx.x + 1) * total / runs : 0;
    if (blockIdx.x == 0 || (before <= lo && lo < before + mine)) {
      int64_t x = before;
      for (int e = e0; e < e1; ++e) {
        if (blockIdx.x == 0) a.begins[e] = x;
        const int tiles = e == e0 ? tiles0 : Item<Q4, NT>(a, e).tiles;
        if (x <= lo && lo < x + tiles) {
          s_item = e;
          s_at = lo - x;
        }
        x += tiles;
      }
      if (blockIdx.x == 0 && e1 == a.items && e0 < e1) a.begins[e1] = x;
    }
    __syncthreads();
    __syncwarp();                                          // lanes above went different ways; matrix instructions follow
    left_over = hi - lo;
    if (left_over <= 0) return;
    item_no = s_item;
    off = s_at;
  }

  for (;; ++item_no, off = 0) {
  const Item<Q4, NT> it(a, item_no);
  const int p = it.p, b = it.b, h = it.h, r0 = it.r0, r1 = it.r1, pos0 = it.pos0, q_live = it.q_live;
  const Seen seen = it.seen;
  const int64_t first_row = it.first_row;
  if (a.ctas == 0) {
    off = (it.tiles * rank) >> a.split;                    // (at most 2^27 tiles)
    left_over = ((it.tiles * (rank + 1)) >> a.split) - off;
  } else if (it.tiles == 0) {
    continue;
  }
  const int t_lo = (int)off, t_hi = (int)min((int64_t)it.tiles, off + left_over);
  left_over -= t_hi - t_lo;

  // ------------------------------------------------------------ the ring of this warp
  unsigned char* ring = smem + warp * T::kWarpBytes;
  const uint32_t ring_u = smem_addr(ring);
  const __nv_bfloat16 *kb = nullptr, *vb = nullptr;
  if (!Q4) {
    kb = a.K.base + b * a.K.stride_b + h * a.K.stride_h;
    vb = a.V.base + b * a.V.stride_b + h * a.V.stride_h;
  }
  auto fetch = [&](int tile, int stage) {
    const uint32_t dst = ring_u + stage * T::kBytes;
    const int u0 = tile * T::kKeys;
    if (Q4) {
      // two 64-byte rows share a 128-byte line of shared memory; the line's eight 16-byte places are
      // permuted by the line number so that both products' reads are free of bank conflicts
      const int64_t row0 = first_row + u0;
      const uint8_t* ks = a.cache.K_codes + row0 * qcache::kRowBytes + lane * 16;
      const uint8_t* vs = a.cache.V_codes + row0 * qcache::kRowBytes + lane * 16;
      const uint32_t* km = a.cache.K_meta + (row0 + lane) * 4;
      const uint32_t* vm = a.cache.V_meta + (row0 + lane) * 4;
      // chunk c = 32 i + lane: line c / 8 = 4 i + lane / 8, so the permutation is the lane's alone
      const uint32_t at = dst + (uint32_t)((lane >> 3) * 128 + (((lane & 7) ^ (2 * (lane >> 3))) * 16));
      const int left = seen.total - u0;                    // rows of the tile that exist (or more)
      if (left >= T::kKeys) {
#pragma unroll
        for (int i = 0; i < T::kKeys * 4 / 32; ++i) {
          copy16(at + T::kK + 512u * i, ks + 512 * i);
          copy16(at + T::kV + 512u * i, vs + 512 * i);
        }
        copy16(dst + T::kKMeta + lane * 16, km);
        copy16(dst + T::kVMeta + lane * 16, vm);
      } else {
#pragma unroll
        for (int i = 0; i < T::kKeys * 4 / 32; ++i) {
          const bool live = 8 * i + (lane >> 2) < left;
          copy16(at + T::kK + 512u * i, live ? ks + 512 * i : a.cache.K_codes, live);
          copy16(at + T::kV + 512u * i, live ? vs + 512 * i : a.cache.V_codes, live);
        }
        const bool live = lane < left;
        copy16(dst + T::kKMeta + lane * 16, live ? km : a.cache.K_meta, live);
        copy16(dst + T::kVMeta + lane * 16, live ? vm : a.cache.V_meta, live);
      }
    } else {
#pragma unroll
      for (int i = 0; i < T::kKeys / 2; ++i) {
        const int key = 2 * i + (lane >> 4), c = lane & 15;
        const int u = u0 + key;
        const bool live = u < seen.total;
        const int64_t j = live ? seen.row(u) : 0;
        const uint32_t at = (uint32_t)(key * 256 + ((c ^ (key & 7)) * 16));
        copy16(dst + T::kK + at, live ? kb + j * a.K.stride_n + c * 8 : kb, live);
        copy16(dst + T::kV + at, live ? vb + j * a.V.stride_n + c * 8 : vb, live);
      }
    }
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    if (t_lo + warp + s * kWarps < t_hi) fetch(t_lo + warp + s * kWarps, s);
    copy_commit();
  }

  // ------------------------------------------------------------ the query rows of this block
  // B operand of S^T: this lane holds query g of each set of 8, for 4-bit rows the channels
  // 32 gr + 8 t + u of every group gr, for bf16 rows 16 s + 2 t + {0, 1, 8, 9} of every step s.
  uint32_t q[NT][16], qz[NT][2];
  float unit[NT][2];                                       // logit (log2 units) per unit of S, queries 2t, 2t + 1
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = r0 + 8 * nt + g;
    const bool live = r < r1;
    const __nv_bfloat16* src = a.Q + b * a.q_sb + (int64_t)(h * a.group + (live ? r % a.group : 0)) * a.q_sh +
                               (int64_t)(live ? r / a.group : 0) * a.q_sn;
    if (Q4) {
      // the row times a power of two that brings its largest entry to 2^12 .. 2^13, as fp16: exact
      // but for entries 2^26 times smaller than that
      float x[4][8];
#pragma unroll
      for (int gr = 0; gr < 4; ++gr) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (live) v = *reinterpret_cast<const uint4*>(src + 32 * gr + 8 * t);
        unpack_bf16x8(v, x[gr]);
      }
      float top = 0.f, sum[4];
#pragma unroll
      for (int gr = 0; gr < 4; ++gr) {
        sum[gr] = 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          top = fmaxf(top, fabsf(x[gr][u]));
          sum[gr] += x[gr][u];
        }
      }
#pragma unroll
      for (int o = 1; o <= 2; o <<= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) sum[gr] += __shfl_xor_sync(0xffffffffu, sum[gr], o);
      }
      // biased exponent of the largest entry, kept where both powers below are normal numbers
      const int e = min(max((__float_as_int(top) >> 23) & 255, 16), 240);
      const float up = pow2_biased(127 + 12 - (e - 127)), down = pow2_biased(127 - 12 + (e - 127));
#pragma unroll
      for (int gr = 0; gr < 4; ++gr) {
        // nibbles one place up stand for 16 times their code: their channels take q / 16
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float f = (u & 1) ? up * 0.0625f : up;
          q[nt][gr * 4 + u] = pack_f16(x[gr][u] * f, x[gr][u + 4] * f);
        }
      }
      // sum of the group t, in S's units (2^-24 up), as three bf16 pieces (24 bits)
      const float z = (t == 0 ? sum[0] : t == 1 ? sum[1] : t == 2 ? sum[2] : sum[3]) * up * 0x1p-24f;
      const float z0 = __bfloat162float(__float2bfloat16_rn(z));
      const float z1 = __bfloat162float(__float2bfloat16_rn(z - z0));
      qz[nt][0] = pack_bf16(z0, z1);
      qz[nt][1] = pack_bf16(z - z0 - z1, 0.f);
      // queries 2t and 2t + 1 live in lanes 8 t and 8 t + 4
      unit[nt][0] = __shfl_sync(0xffffffffu, down, 8 * t) * 0x1p24f * a.scale_log2;
      unit[nt][1] = __shfl_sync(0xffffffffu, down, 8 * t + 4) * 0x1p24f * a.scale_log2;
    } else {
#pragma unroll
      for (int s = 0; s < 8; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          q[nt][2 * s + i] = live ? *reinterpret_cast<const uint32_t*>(src + 16 * s + 8 * i + 2 * t) : 0u;
      unit[nt][0] = unit[nt][1] = a.scale_log2;
    }
  }
  // positions of queries 2t, 2t + 1 of each set (bf16 rows with several query tokens)
  int pos[NT][2];
  if (!Q4) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) pos[nt][i] = pos0 + (r0 + 8 * nt + 2 * t + i) / a.group;
  }
  const int pos_lo = pos0 + r0 / a.group, pos_hi = pos0 + (r1 - 1) / a.group;

  float acc[NT][8][4], accz[NT][4];                        // O^T: 128 channels x queries 2t, 2t + 1; zeros' part
  // m: reference of the weights (T for 4-bit rows); l: row sum; rise: 2^(T - R)
  float m[NT][2], l[NT][2], rise[NT][2];
  // (this warp's share of the run's keys)
  const int span = span_of(((t_hi - t_lo + kWarps - 1) / kWarps) * T::kKeys);
  int vexp;                                                // E
  uint32_t below_hi, from_lo;                              // what brings what lies too high, or high enough, to bit 15
  auto set_unit = [&](int e) {
    vexp = e;
    const int hi = 128 * (e + 127), lo = hi - 128 * span - 1, zero_lo = hi - 128 * kZeroDown - 1;
    below_hi = (uint32_t)(0x8000 - hi) | (uint32_t)(0x8000 - hi - 128 * kZeroUp) << 16;
    from_lo = (uint32_t)(0x8000 - max(lo, 0)) | (uint32_t)(0x8000 - max(zero_lo, 0)) << 16;
  };
  set_unit(kLeastE);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[nt][i][j] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) accz[nt][j] = 0.f;
    m[nt][0] = m[nt][1] = -INFINITY;
    l[nt][0] = l[nt][1] = 0.f;
    rise[nt][0] = rise[nt][1] = 1.f;
  }

  // ------------------------------------------------------------ the key loop
  int stage = 0;
  for (int tile = t_lo + warp; tile < t_hi; tile += kWarps) {
    {
      const int ahead = tile + (kStages - 1) * kWarps;
      const int into = stage == 0 ? kStages - 1 : stage - 1;
      if (ahead < t_hi) fetch(ahead, into);
      copy_commit();
    }
    copy_wait<kStages - 1>();
    __syncwarp();
    const unsigned char* st = ring + stage * T::kBytes;
    const uint32_t st_u = ring_u + stage * T::kBytes;
    const int u0 = tile * T::kKeys;
    const int left = seen.total - u0;

    // ---- do V's scales and zeros lie where E has them?  (largest and least of the row's, bf16 bits side by side, 0 apart)
    auto v_meta = [&](uint32_t (&w)[4]) {
      const uint4 v = *reinterpret_cast<const uint4*>(st + T::kVMeta + lane * 16);
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    };
    auto extremes = [](const uint32_t (&w)[4], uint32_t& top, uint32_t& low) {
      top = w[0] & 0x7fff7fffu;
      low = top - 0x00010001u;                             // (0 becomes the largest)
#pragma unroll
      for (int gr = 1; gr < 4; ++gr) {
        const uint32_t x = w[gr] & 0x7fff7fffu;
        top = __vmaxu2(top, x);
        low = __vminu2(low, x - 0x00010001u);
      }
      low = __vminu2(low, 0x7fff7fffu);
    };
    bool elsewhere = false;
    if constexpr (Q4) {
      uint32_t w[4], top, low;
      v_meta(w);
      extremes(w, top, low);
      elsewhere = (((top + below_hi) | ~(low + from_lo)) & 0x80008000u) != 0u;
    }
    // ---- S^T
    float s[NT][KB][4];
#pragma unroll
    for (int kb16 = 0; kb16 < KB; ++kb16) {
      if constexpr (Q4) {
        uint32_t w[2][4];                                  // codes of rows g and g + 8: word = group
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int c = (kb16 * 16 + 8 * i + g) * 4 + t, line = c >> 3;
          const uint4 v = *reinterpret_cast<const uint4*>(st + T::kK + line * 128 + (((c & 7) ^ (2 * (line & 3))) * 16));
          w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
        }
        const uint32_t* meta = reinterpret_cast<const uint32_t*>(st + T::kKMeta) + (kb16 * 16 + g) * 4;
        const uint32_t za = __byte_perm(meta[t], 0u, 0x3232), zb = __byte_perm(meta[32 + t], 0u, 0x3232);
        const uint4 ma = *reinterpret_cast<const uint4*>(meta), mb = *reinterpret_cast<const uint4*>(meta + 32);
        const uint32_t sa[4] = {ma.x, ma.y, ma.z, ma.w}, sb[4] = {mb.x, mb.y, mb.z, mb.w};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int j = 0; j < 4; ++j) s[nt][kb16][j] = 0.f;
          mma_bf16(s[nt][kb16], za, zb, za, zb, qz[nt][0], qz[nt][1]);
        }
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
          uint32_t x[2][4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t hi = w[i][gr] >> 8;
            x[i][0] = w[i][gr] & 0x000f000fu;
            x[i][1] = w[i][gr] & 0x00f000f0u;
            x[i][2] = hi & 0x000f000fu;
            x[i][3] = hi & 0x00f000f0u;
          }
          const float fa = __uint_as_float(sa[gr] << 16), fb = __uint_as_float(sb[gr] << 16);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float d[4] = {0.f, 0.f, 0.f, 0.f};
            mma_f16(d, x[0][0], x[1][0], x[0][1], x[1][1], q[nt][4 * gr], q[nt][4 * gr + 1]);
            mma_f16(d, x[0][2], x[1][2], x[0][3], x[1][3], q[nt][4 * gr + 2], q[nt][4 * gr + 3]);
            s[nt][kb16][0] = fmaf(d[0], fa, s[nt][kb16][0]);
            s[nt][kb16][1] = fmaf(d[1], fa, s[nt][kb16][1]);
            s[nt][kb16][2] = fmaf(d[2], fb, s[nt][kb16][2]);
            s[nt][kb16][3] = fmaf(d[3], fb, s[nt][kb16][3]);
          }
        }
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[nt][kb16][j] = 0.f;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          uint32_t x[4];
          const int key = kb16 * 16 + (lane & 15), c = 2 * ks + (lane >> 4);
          ldmatrix4(x, st_u + T::kK + key * 256 + ((c ^ (key & 7)) * 16));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            mma_bf16(s[nt][kb16], x[0], x[1], x[2], x[3], q[nt][2 * ks], q[nt][2 * ks + 1]);
        }
      }
    }
    // ---- logits in log2 units; what a query does not see becomes -inf
#pragma unroll
    for (int kb16 = 0; kb16 < KB; ++kb16)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[nt][kb16][j] *= unit[nt][j & 1];
    bool masked = left < T::kKeys;
    if (!Q4) {
      // a tile that every query of the block sees whole needs no comparison
      const int j_lo = seen.row(u0), j_hi = seen.row(min(u0 + T::kKeys, seen.total) - 1);
      masked = masked || j_hi > pos_lo || (j_hi >= a.num_sink && (int64_t)j_lo <= (int64_t)pos_hi - a.window &&
                                           pos_hi != pos_lo);
    }
    if (masked) {
#pragma unroll
      for (int kb16 = 0; kb16 < KB; ++kb16)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int u = u0 + kb16 * 16 + 8 * i + g;
          const int j = Q4 ? u : seen.row(u);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              bool see = u < seen.total;
              if (!Q4) see = see && j <= pos[nt][c] && (j < a.num_sink || (int64_t)j > (int64_t)pos[nt][c] - a.window);
              if (!see) s[nt][kb16][2 * i + c] = -INFINITY;
            }
        }
    }
    // ---- running maximum
    bool move = elsewhere;
    float top[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x = fmaxf(s[nt][0][c], s[nt][0][2 + c]);
#pragma unroll
        for (int kb16 = 1; kb16 < KB; ++kb16) x = fmaxf(x, fmaxf(s[nt][kb16][c], s[nt][kb16][2 + c]));
        top[nt][c] = x;
        move = move || x > m[nt][c] + slack<Q4>();
      }
    bool wide = false;                                     // fp16 is not enough for this tile
    if (__any_sync(0xffffffffu, move)) {
      int shift = 0;                                       // by how much this tile moves E
      if (Q4 && __any_sync(0xffffffffu, elsewhere)) {
        uint32_t w[4], top, low;
        v_meta(w);
        extremes(w, top, low);
        const int hi = max((int)(top & 0xffffu), (int)(top >> 16) - 128 * kZeroUp);
        const int lo = min((int)(low & 0xffffu), (int)(low >> 16) + 128 * (kZeroDown - span));
        auto outside = [&](int h, int l, int e) { return h >= 128 * (e + 127) || l < 128 * (e + 127 - span) - 1; };
        int th = (int)__reduce_max_sync(0xffffffffu, (unsigned)max(hi, 0));
        const int tl = (int)__reduce_min_sync(0xffffffffu, (unsigned)lo);
        const bool huge = th >= 128 * (kMostE + 127);      // a NaN or an infinity among them, perhaps
        if (huge) {
          int h = 0;                                       // the largest of the others
#pragma unroll
          for (int gr = 0; gr < 4; ++gr) {
            const int sc = (int)(w[gr] & 0x7fffu), ze = (int)((w[gr] >> 16) & 0x7fffu);
            h = max(h, max(sc >= 0x7f80 ? 0 : sc, ze >= 0x7f80 ? 0 : ze - 128 * kZeroUp));
          }
          th = (int)__reduce_max_sync(0xffffffffu, (unsigned)h);
        }
        const int own = (th >> 7) - 126;                   // every scale is below 2^own
        // A tile that fits by itself brings its E, but not one so low that fp16 weights would lose their bits against
        // the accumulators' unit: later tiles would then all pay for this one.  One that does not keeps E, unless its
        // values lie too far above (then E is such that rows like its smaller ones fit next).
        int to = vexp;
        wide = huge || outside(th, tl, own);
        if (!wide) {
          to = own;
          if (own < vexp) {
            int up = 0;                                    // of the accumulators' unit over 2^E
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) up = max(up, max(exponent_of(rise[nt][0]), exponent_of(rise[nt][1])));
            wide = __any_sync(0xffffffffu, vexp - own + up > kFall);
            if (wide) to = vexp;
          }
        } else if (own > vexp + kMostAbove) {
          to = min(kMostE, max(own - kMostAbove, min(own, (tl >> 7) - 127 + span / 2)));
        }
        shift = to - vexp;
        set_unit(to);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float x = top[nt][c];
#pragma unroll
          for (int o = 4; o <= 16; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
          float f;                                         // 0 on the first rows
          if (Q4) {
            // T + E of the accumulators stays where it is or rises; R rises with the logits alone
            const float r = m[nt][c] - whole_of(rise[nt][c]), was = m[nt][c] - (float)shift;
            x = ceilf(x);
            const float r_now = fmaxf(r, x), now = fmaxf(fmaxf(was, x), r_now - 100.f);
            f = now == -INFINITY ? 1.f : pow2_whole(was - now);
            l[nt][c] *= now == -INFINITY ? 1.f : pow2_whole(r - r_now);
            rise[nt][c] = now == -INFINITY ? 1.f : pow2_whole(now - r_now);
            m[nt][c] = now;
          } else {
            const float now = fmaxf(m[nt][c], x);
            f = now == -INFINITY ? 1.f : exp2_approx(m[nt][c] - now);
            m[nt][c] = now;
            l[nt][c] *= f;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            acc[nt][i][c] *= f;
            acc[nt][i][2 + c] *= f;
          }
          accz[nt][c] *= f;
        }
    }
    // ---- weights and O^T
    float nref[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) nref[nt][c] = (Q4 ? kLift : 0.f) - (m[nt][c] == -INFINITY ? 0.f : m[nt][c]);
    // the weights take the logits' place
    auto weigh = [&](float (&w)[4], int nt) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = exp2_approx(w[j] + nref[nt][j & 1]);
      if (Q4) {
        l[nt][0] = fmaf(w[2], rise[nt][0], fmaf(w[0], rise[nt][0], l[nt][0]));
        l[nt][1] = fmaf(w[3], rise[nt][1], fmaf(w[1], rise[nt][1], l[nt][1]));
      } else {
        l[nt][0] = w[2] + (w[0] + l[nt][0]);
        l[nt][1] = w[3] + (w[1] + l[nt][1]);
      }
    };
    if (!Q4 || __builtin_expect(!wide, 1)) {
    if constexpr (Q4) {
      // V's scales and zeros in fp16: lanes 2 i and 2 i + 1 hold a pair of keys; the even one takes the pair's groups 0 and
      // 1, the odd one 2 and 3
      const float inv = pow2_biased(127 - vexp);
      uint32_t w[4], sz[2][2];                             // [scale, zero][groups 0-1, 2-3] of this key
      v_meta(w);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sz[0][i] = pack_f16(__uint_as_float(w[2 * i] << 16) * inv, __uint_as_float(w[2 * i + 1] << 16) * inv);
        sz[1][i] = pack_f16(__uint_as_float(w[2 * i] & 0xffff0000u) * inv, __uint_as_float(w[2 * i + 1] & 0xffff0000u) * inv);
      }
      const bool odd = lane & 1;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? sz[k][0] : sz[k][1], 1);
        const uint32_t keep = odd ? sz[k][1] : sz[k][0];
        const uint32_t ev = odd ? got : keep, od = odd ? keep : got;                 // key 2 i, key 2 i + 1
        *reinterpret_cast<uint2*>(ring + kStages * T::kBytes + k * (T::kKeys * 8) + lane * 8) =
            make_uint2(__byte_perm(ev, od, 0x5410), __byte_perm(ev, od, 0x7632));
      }
      __syncwarp();
    }
#pragma unroll
    for (int kb16 = 0; kb16 < KB; ++kb16) {
      uint32_t pt[NT][2];                                  // P^T as B operand: keys 2t, 2t + 1 / 2t + 8, 2t + 9 of query g
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float(&w)[4] = s[nt][kb16];
        weigh(w, nt);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          pt[nt][i] = transpose8x8(Q4 ? pack_f16(w[2 * i], w[2 * i + 1]) : pack_bf16(w[2 * i], w[2 * i + 1]));
      }
      if constexpr (Q4) {
        const __half* scaled = reinterpret_cast<const __half*>(ring + kStages * T::kBytes);
        uint32_t x[2][4][4], sc[2][4], z[2];               // [keys 2t.. / 2t + 8..][group][nibble]
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int pair = (kb16 * 16 + 8 * i + 2 * t) >> 1;
          uint32_t y[4];
          v_words(st, kb16 * 16 + 8 * i + 2 * t, g, y);
#pragma unroll
          for (int gr = 0; gr < 4; ++gr) {
            const uint32_t hi = y[gr] >> 8;
            x[i][gr][0] = y[gr] & 0x000f000fu;
            x[i][gr][1] = y[gr] & 0x00f000f0u;
            x[i][gr][2] = hi & 0x000f000fu;
            x[i][gr][3] = hi & 0x00f000f0u;
          }
          const uint4 f = *reinterpret_cast<const uint4*>(scaled + pair * 8);
          sc[i][0] = f.x; sc[i][1] = f.y; sc[i][2] = f.z; sc[i][3] = f.w;
          z[i] = g < 4 ? *reinterpret_cast<const uint32_t*>(scaled + T::kKeys * 4 + pair * 8 + 2 * g) : 0u;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma_f16(accz[nt], z[0], 0u, z[1], 0u, pt[nt][0], pt[nt][1]);
#pragma unroll
          for (int gr = 0; gr < 4; ++gr) {
            const uint32_t b0 = hmul2(pt[nt][0], sc[0][gr]), b1 = hmul2(pt[nt][1], sc[1][gr]);
            mma_f16(acc[nt][2 * gr], x[0][gr][0], x[0][gr][1], x[1][gr][0], x[1][gr][1], b0, b1);
            mma_f16(acc[nt][2 * gr + 1], x[0][gr][2], x[0][gr][3], x[1][gr][2], x[1][gr][3], b0, b1);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t x[4];                                   // V^T: channels 16 i .. + 15 of the 16 keys
          const int key = kb16 * 16 + (lane & 7) + ((lane >> 4) & 1) * 8, c = 2 * i + ((lane >> 3) & 1);
          ldmatrix4_trans(x, st_u + T::kV + key * 256 + ((c ^ (key & 7)) * 16));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma_bf16(acc[nt][i], x[0], x[1], x[2], x[3], pt[nt][0], pt[nt][1]);
        }
      }
    }
    } else if constexpr (Q4) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int kb16 = 0; kb16 < KB; ++kb16) weigh(s[nt][kb16], nt);
      wide_products<NT>(acc, accz, s, st, pow2_biased(127 - vexp));
    }
    __syncwarp();                                          // the stage may be filled again
    stage = stage == kStages - 1 ? 0 : stage + 1;
  }
  copy_wait<0>();

  // ------------------------------------------------------------ the warps' results meet
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int o = 4; o <= 16; o <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], o);
      if (g == 0) {
        Part own = {m[nt][c], l[nt][c], 0.f};
        if (Q4) {
          const int up = exponent_of(rise[nt][c]);
          own.ref -= (float)up;
          own.unit = (float)(vexp + up);
        }
        s_part[warp][8 * nt + 2 * t + c] = own;
      }
    }
  __syncthreads();                                         // also: every warp is done with its ring
  float* meet = reinterpret_cast<float*>(smem);            // [warp][8 NT][132]
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int qi = 8 * nt + 2 * t + c;
      float all = -INFINITY, unit = Q4 ? -INFINITY : 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) all = fmaxf(all, s_part[w][qi].ref);
      if (Q4) {
#pragma unroll
        for (int w = 0; w < kWarps; ++w) unit = fmaxf(unit, above(s_part[w][qi], all));
      }
      if (warp == 0) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) sum = fmaf(s_part[w][qi].sum, share(s_part[w][qi].ref - all, all), sum);
        if (g == 0) s_ml[qi] = make_float4(Q4 ? all - kLift : all, sum, unit, 0.f);
        __syncwarp();
      }
      const float f = share(Q4 ? above(s_part[warp][qi], all) - unit : m[nt][c] - all, all);
      float* dst = meet + ((size_t)warp * 8 * NT + qi) * 132;
      if (Q4) {
#pragma unroll
        for (int gr = 0; gr < 4; ++gr) {
          const float z = __shfl_sync(0xffffffffu, accz[nt][c], gr * 4 + t);
          float4 o;
          o.x = (acc[nt][2 * gr][c] * 0x1p24f + z) * f;
          o.y = (acc[nt][2 * gr][2 + c] * 0x1p20f + z) * f;
          o.z = (acc[nt][2 * gr + 1][c] * 0x1p24f + z) * f;
          o.w = (acc[nt][2 * gr + 1][2 + c] * 0x1p20f + z) * f;
          *reinterpret_cast<float4*>(dst + 32 * gr + 4 * g) = o;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dst[16 * i + g] = acc[nt][i][c] * f;
          dst[16 * i + 8 + g] = acc[nt][i][2 + c] * f;
        }
      }
    }
  __syncthreads();
  // one row's four channels: O = sums / sum in units of 2^unit, and its log sum
  auto finish = [&](int qi, int c4, const float4& o, float top, float sum, float unit) {
    const int r = r0 + qi, i = r / a.group, hq = h * a.group + r % a.group;
    if (i >= q_live) return;                               // rows behind the last query stay as they are
    const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);     // a NaN sum stays one
    const float up = Q4 ? exp2_approx(unit) : 1.f;         // (apart from the sum's: either may be far from 1)
    uint2 v;
    v.x = pack_bf16(o.x * inv * up, o.y * inv * up);
    v.y = pack_bf16(o.z * inv * up, o.w * inv * up);
    *reinterpret_cast<uint2*>(a.O + b * a.o_sb + (int64_t)hq * a.o_sh + (int64_t)i * a.o_sn + c4) = v;
    if (c4 == 0 && a.lse != nullptr)
      a.lse[((int64_t)b * a.heads * a.group + hq) * a.q_n + i] =
          sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
  };
  for (int e = tid; e < (r1 - r0) * 32; e += kThreads) {
    const int qi = e >> 5, c4 = (e & 31) * 4;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(meet + ((size_t)w * 8 * NT + qi) * 132 + c4);
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    if (a.split > 0) {                                     // (only this thread reads these four places)
      *reinterpret_cast<float4*>(meet + (size_t)qi * 132 + c4) = o;
    } else if (t_hi - t_lo < it.tiles) {                   // a part: of the item this run begins or ends in
      const size_t at = ((size_t)blockIdx.x * 2 + (t_lo == 0 ? 1 : 0)) * 8 * NT + qi;
      *reinterpret_cast<float4*>(a.part_o + at * 128 + c4) = o;
      if (c4 == 0) reinterpret_cast<float4*>(a.part_ml)[at] = s_ml[qi];
    } else {
      const float4 ml = s_ml[qi];
      finish(qi, c4, o, ml.x, ml.y, ml.z);
    }
  }
  if (a.ctas == 0) {
    // (one lane's work: behind all matrix instructions and barriers, to which a warp has to come together)
    auto flag = [&]() {
      if (!it.ok && rank == 0 && tid == 0) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
    };
    if (a.split == 0) {
      flag();
      return;
    }
    // the CTAs of a cluster join their parts, in the order of their ranks, a share of the rows each
    cluster_sync();
    for (int e = rank * kThreads + tid; e < (r1 - r0) * 32; e += kThreads << a.split) {
      const int qi = e >> 5, c4 = (e & 31) * 4;
      const uint32_t ml = smem_addr(&s_ml[qi]), at = smem_addr(meet + (size_t)qi * 132 + c4);
      Part part[1 << kMostSplit];
      float4 x[1 << kMostSplit];
      float all = -INFINITY, sum = 0.f, unit = -INFINITY;
#pragma unroll
      for (int c = 0; c < (1 << kMostSplit); ++c) {
        if (c >> a.split) break;
        const float4 y = peer_float4(peer_addr(ml, c));
        part[c] = Part{y.x, y.y, y.z};
        x[c] = peer_float4(peer_addr(at, c));
        all = fmaxf(all, part[c].ref);
      }
#pragma unroll
      for (int c = 0; c < (1 << kMostSplit); ++c) {
        if (c >> a.split) break;
        unit = fmaxf(unit, above(part[c], all));
      }
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int c = 0; c < (1 << kMostSplit); ++c) {
        if (c >> a.split) break;
        const float f = share(above(part[c], all) - unit, all);
        sum = fmaf(share(part[c].ref - all, all), part[c].sum, sum);
        o.x = fmaf(f, x[c].x, o.x); o.y = fmaf(f, x[c].y, o.y); o.z = fmaf(f, x[c].z, o.z); o.w = fmaf(f, x[c].w, o.w);
      }
      finish(qi, c4, o, all, sum, unit);
    }
    cluster_sync();                                        // nobody leaves while its parts are read
    flag();
    return;
  }
  if (left_over <= 0) return;
  __syncthreads();                                         // the ring is the next item's
  __syncwarp();
  }
}

// Joins the parts of items that several CTAs share (Part), in the order of the CTAs.  grid = items * block_rows, block = 32 (four channels a lane).
__global__ void __launch_bounds__(32) join_kernel(const Args a, int block_rows) {
  asm volatile("griddepcontrol.wait;" ::: "memory");       // behind the last CTA of attend_kernel
  const int item = blockIdx.x / block_rows, qi = blockIdx.x % block_rows;
  const int64_t from = a.begins[item], to = a.begins[item + 1], total = a.begins[a.items];
  if (to <= from) return;
  const int64_t runs = min((int64_t)a.ctas, total);
  const int c0 = cta_of(from, total, runs), c1 = cta_of(to - 1, total, runs);
  const int p = item / a.blocks, r = (item % a.blocks) * block_rows + qi;
  if (c0 == c1 || r >= a.rows) return;
  const int b = p / a.heads, h = p % a.heads, i = r / a.group, hq = h * a.group + r % a.group;
  const int lane = threadIdx.x;
  if (a.q_lens != nullptr && i >= min(max(a.q_lens[b], 0), a.q_n)) return;
  // the item begins in c0 (its second part) and goes on in the others (their first)
  auto part = [&](int c) { return ((size_t)c * 2 + (c == c0 ? 1 : 0)) * block_rows + qi; };
  // maxima and sums: a lane per part; sums of values: four parts in flight
  auto at = [&](int c) { return part(min(c, c1)); };
  auto head = [&](int c) {
    const float4 y = reinterpret_cast<const float4*>(a.part_ml)[at(c)];
    return Part{y.x, y.y, y.z};
  };
  auto values = [&](int c) { return *reinterpret_cast<const float4*>(a.part_o + at(c) * 128 + lane * 4); };
  const Part first = head(c0 + lane);
  float4 x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = values(c0 + k);
  auto most = [](float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  };
  float all = first.ref;
  for (int c = c0 + 32 + lane; c <= c1; c += 32) all = fmaxf(all, head(c).ref);
  all = most(all);
  float unit = above(first, all);
  for (int c = c0 + 32 + lane; c <= c1; c += 32) unit = fmaxf(unit, above(head(c), all));
  unit = most(fmaxf(unit, -INFINITY));                     // (not a NaN, where all is -inf)
  float sum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int cb = c0; cb <= c1; cb += 32) {
    const Part e = cb == c0 ? first : head(cb + lane);
    const bool live = cb + lane <= c1;
    const float f = live ? share(above(e, all) - unit, all) : 0.f;
    float l = live ? share(e.ref - all, all) * e.sum : 0.f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    sum += l;
    for (int c = cb; c < cb + 32 && c <= c1; c += 4) {
      float4 now[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        now[k] = x[k];
        if (c + 4 <= c1) x[k] = values(c + 4 + k);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float fk = __shfl_sync(0xffffffffu, f, c - cb + k);
        if (c + k > c1) continue;
        o.x = fmaf(fk, now[k].x, o.x); o.y = fmaf(fk, now[k].y, o.y); o.z = fmaf(fk, now[k].z, o.z); o.w = fmaf(fk, now[k].w, o.w);
      }
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
  const float up = exp2_approx(unit);                      // 1 for bf16 rows
  uint2 v;
  v.x = pack_bf16(o.x * inv * up, o.y * inv * up);
  v.y = pack_bf16(o.z * inv * up, o.w * inv * up);
  *reinterpret_cast<uint2*>(a.O + b * a.o_sb + (int64_t)hq * a.o_sh + (int64_t)i * a.o_sn + lane * 4) = v;
  if (lane == 0 && a.lse != nullptr)
    a.lse[((int64_t)b * a.heads * a.group + hq) * a.q_n + i] =
        sum == 0.f ? -INFINITY : (all + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace token
}  // namespace curdkv
