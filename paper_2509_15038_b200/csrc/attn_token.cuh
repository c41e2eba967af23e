// Attention of a few query rows per KV head over a long cache: the generation step.  Two caches,
// one kernel: rows held in 4 bits (curdkv_qcache_attention) and bf16 rows of which a sliding window
// and the first tokens are visible (curdkv_attention_window with few queries).
//
// What has to be moved are the cache's bytes, each once.  4-bit rows are bound by the instructions that
// unpack and weigh them instead (some 285 per 16 keys of a warp, integer pipe 57 % busy): 64 heads of 131072
// rows and 4 queries 236 us, 5.7 TB/s (280 when the device's power limit holds its clock down); a copy that
// only loads takes 196.  bf16 rows are bound by their loads: 128 heads with a window of 4096 46 us, 5.7 TB/s.
// The tiles of all items -- an item is a head and a block of query rows -- form one line, and every CTA takes
// an equal run of it, whatever the items' lengths: whole items are finished where they are, the partial
// results of an item that several CTAs share are joined by a second kernel.  (128 heads of 2048 to 16384 rows:
// 70 us with a CTA per item, as long as the longest, 49 with equal runs.)  Where that gains little an item has
// a CTA or a cluster of two, four or eight to itself, whose parts are joined through distributed shared
// memory in the same launch: 8 heads of 1702 rows 6.4 us, 10.7 with equal runs and the second kernel; 128
// windows of 4096 46 us against 53.  A CTA's warps take its tiles in turn, each warp with its own ring of
// tiles in shared memory, filled by 16-byte asynchronous copies (rows that do not exist are filled with
// zeros, so nothing behind a head's last row is ever read).  No barrier stands in the key loop.  Per 16
// keys a warp forms
//   S^T [16 keys x 8 queries] = K Q^T        m16n8k16, keys as the M side: with the few queries of
//   O^T [128 x 8 queries]    += V^T P^T      a KV head as N = 8 half the instructions that a layout
//                                            with 16 padded queries as M would need
// and between the two the online softmax: a warp's running maximum moves only when some logit
// exceeds it by more than 2^kSlack (one vote per tile), and since S^T and O^T hold a query in the
// same lanes the rescale needs no exchange.  P^T reaches the second product's operand layout by two
// 8x8 transposes (movmatrix).  Sums, maxima and accumulators are fp32; the weights enter the second
// product as fp16 (4-bit rows) or bf16 (bf16 rows), at most 2^-11 / 2^-8 of each weight off by
// half a step; the row sum is taken over the unrounded weights.
//
// 4-bit rows cost five integer instructions per eight values and no conversion: a code left in the
// low bits of a half is the fp16 subnormal code * 2^-24 (or code * 2^-20 one nibble up), which the
// tensor cores multiply exactly.  The scales are applied outside: on the K side to the products of
// each group of 32 channels (S = sum_g s_g (codes_g . q_g) + sum_g z_g sum(q_g), the second sum one
// more matrix instruction whose A operand is the zeros), on the V side to the weights (one set per
// group, P_g = p * s_g), with the zeros as a further instruction.  Every V row brings its own power of
// two 2^e that covers its values: its scales and zeros relative to it fit fp16, and 2^e goes into the
// exponent of its weight, so that the running maximum follows logit + e -- what a row adds to the
// output -- and rows of any bf16 magnitude share a cache; the row sum takes the 2^e out again.
#pragma once
#include "qcache.cuh"

namespace curdkv {
namespace token {

constexpr int kStages = 3;
constexpr float kSlack = 6.f;        // log2 units a logit may exceed the running maximum
constexpr float kLift = 8.f;         // fp16 weights are 2^(x - m + kLift): at most 2^14, and exact
                                     // to 11 bits down to 2^-22 of the largest

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
  // partial results, two per CTA (of the item its run begins in, of the one it ends in): [8 NT] maxima
  // and sums, [8 NT][128] sums of values; and where each item begins on the line, [items + 1]
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
__device__ __forceinline__ float2 peer_float2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float4 peer_float4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// 2^(e - 127) for 1 <= e <= 253, and 0 below
__device__ __forceinline__ float pow2_biased(int e) { return __int_as_float(e > 0 ? e << 23 : 0); }

template <bool Q4>
struct Tile {                                              // one warp's stage
  static constexpr int kKeys = Q4 ? 32 : 16;
  static constexpr int kK = 0;
  static constexpr int kV = kKeys * (Q4 ? qcache::kRowBytes : 256);
  static constexpr int kKMeta = 2 * kV;
  static constexpr int kVMeta = kKMeta + (Q4 ? kKeys * qcache::kMetaBytes : 0);
  static constexpr int kBytes = kVMeta + (Q4 ? kKeys * qcache::kMetaBytes : 0);
  // V's scales and zeros in fp16, pairs of keys side by side: [key pair][group] each; then e and 2^-e
  // of each key
  static constexpr int kScaled = Q4 ? kKeys * (8 * 2 + 8) : 0;
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

constexpr int kMostSplit = 3;                              // log2 of the CTAs of a cluster
constexpr int kMostItems = 8192;                           // items that are put on one line

template <bool Q4, int NT>
__global__ void __launch_bounds__(kThreads, (ctas_per_sm<Q4, NT>())) attend_kernel(const Args a) {
  using T = Tile<Q4>;
  constexpr int KB = T::kKeys / 16;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float s_m[kWarps][8 * NT], s_l[kWarps][8 * NT];
  __shared__ float2 s_ml[8 * NT];                          // the CTA's maxima and sums (clusters)
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
  float m[NT][2], l[NT][2];
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

    // ---- V's scales and zeros of this tile in fp16, each row's relative to a power of two of its own
    if constexpr (Q4) {
      const uint4 v = *reinterpret_cast<const uint4*>(st + T::kVMeta + lane * 16);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
      uint32_t top = w[0] & 0x7fff7fffu;                   // largest |zero| and largest scale, bf16 side by side
#pragma unroll
      for (int gr = 1; gr < 4; ++gr) top = __vmaxu2(top, w[gr] & 0x7fff7fffu);
      // bits of the larger of |zero| and 16 * scale (a scale of 0 gives 2^-123, which the limit below covers)
      const uint32_t big = max(top & 0x7fff0000u, (top << 16) + (4u << 23));
      // biased exponent above it; rows far below the tile's largest (rows of zeros among them) take one
      // near it, so that their weights stay numbers
      int e = min(max((int)(big >> 23) + 1, 37), 250);       // (sums of 2^20 weights times 2^-e stay numbers)
      e = max(e, __reduce_max_sync(0xffffffffu, e) - 30);
      const float inv = pow2_biased(254 - e);
      *reinterpret_cast<float2*>(ring + kStages * T::kBytes + T::kKeys * 16 + lane * 8) = make_float2((float)(e - 127), inv);
      // lanes 2 i and 2 i + 1 hold a pair of keys: the even one takes the pair's groups 0 and 1, the odd
      // one 2 and 3
      uint32_t sz[2][2];                                   // [scale, zero][groups 0-1, 2-3] of this key
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
    // ---- logits in log2 units (4-bit rows: plus the row's e); what a query does not see becomes -inf
    float took[KB][2];                                     // 2^-e of keys g, g + 8
#pragma unroll
    for (int kb16 = 0; kb16 < KB; ++kb16)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float2 f = make_float2(0.f, 1.f);
        if (Q4) f = *reinterpret_cast<const float2*>(ring + kStages * T::kBytes + T::kKeys * 16 + (kb16 * 16 + 8 * i + g) * 8);
        took[kb16][i] = f.y;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c)
            s[nt][kb16][2 * i + c] = Q4 ? fmaf(s[nt][kb16][2 * i + c], unit[nt][c], f.x) : s[nt][kb16][2 * i + c] * unit[nt][c];
      }
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
    bool move = false;
    float top[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x = fmaxf(s[nt][0][c], s[nt][0][2 + c]);
#pragma unroll
        for (int kb16 = 1; kb16 < KB; ++kb16) x = fmaxf(x, fmaxf(s[nt][kb16][c], s[nt][kb16][2 + c]));
        top[nt][c] = x;
        move = move || x > m[nt][c] + kSlack;
      }
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float x = top[nt][c];
#pragma unroll
          for (int o = 4; o <= 16; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
          const float now = fmaxf(m[nt][c], x);
          const float f = now == -INFINITY ? 1.f : exp2_approx(m[nt][c] - now);   // 0 on the first rows
          m[nt][c] = now;
          l[nt][c] *= f;
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
#pragma unroll
    for (int kb16 = 0; kb16 < KB; ++kb16) {
      uint32_t pt[NT][2];                                  // P^T as B operand: keys 2t, 2t + 1 / 2t + 8, 2t + 9 of query g
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j] = exp2_approx(s[nt][kb16][j] + nref[nt][j & 1]);
        }
        l[nt][0] = fmaf(w[2], took[kb16][1], fmaf(w[0], took[kb16][0], l[nt][0]));
        l[nt][1] = fmaf(w[3], took[kb16][1], fmaf(w[1], took[kb16][0], l[nt][1]));
#pragma unroll
        for (int i = 0; i < 2; ++i)
          pt[nt][i] = transpose8x8(Q4 ? pack_f16(w[2 * i], w[2 * i + 1]) : pack_bf16(w[2 * i], w[2 * i + 1]));
      }
      if constexpr (Q4) {
        const __half* scaled = reinterpret_cast<const __half*>(ring + kStages * T::kBytes);
        uint32_t x[2][4][4], sc[2][4], z[2];               // [keys 2t.. / 2t + 8..][group][nibble]
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int key = kb16 * 16 + 8 * i + 2 * t, pair = key >> 1;
          uint2 v[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int c = (key + k) * 4 + (g >> 1), line = c >> 3;
            v[k] = *reinterpret_cast<const uint2*>(st + T::kV + line * 128 + (((c & 7) ^ (2 * (line & 3))) * 16) + 8 * (g & 1));
          }
          // 16-bit words of the two keys side by side, one register a group
          const uint32_t y[4] = {__byte_perm(v[0].x, v[1].x, 0x5410), __byte_perm(v[0].x, v[1].x, 0x7632),
                                 __byte_perm(v[0].y, v[1].y, 0x5410), __byte_perm(v[0].y, v[1].y, 0x7632)};
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
        s_m[warp][8 * nt + 2 * t + c] = m[nt][c];
        s_l[warp][8 * nt + 2 * t + c] = l[nt][c];
      }
    }
  __syncthreads();                                         // also: every warp is done with its ring
  float* meet = reinterpret_cast<float*>(smem);            // [warp][8 NT][132]
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int qi = 8 * nt + 2 * t + c;
      float all = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) all = fmaxf(all, s_m[w][qi]);
      const float f = m[nt][c] == -INFINITY ? 0.f : exp2_approx(m[nt][c] - all);
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
  // one row's four channels: O = sums / sum, and its log sum
  auto finish = [&](int qi, int c4, const float4& o, float top, float sum) {
    const int r = r0 + qi, i = r / a.group, hq = h * a.group + r % a.group;
    if (i >= q_live) return;                               // rows behind the last query stay as they are
    const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);     // a NaN sum stays one
    uint2 v;
    v.x = pack_bf16(o.x * inv, o.y * inv);
    v.y = pack_bf16(o.z * inv, o.w * inv);
    *reinterpret_cast<uint2*>(a.O + b * a.o_sb + (int64_t)hq * a.o_sh + (int64_t)i * a.o_sn + c4) = v;
    if (c4 == 0 && a.lse != nullptr)
      a.lse[((int64_t)b * a.heads * a.group + hq) * a.q_n + i] =
          sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
  };
  for (int e = tid; e < (r1 - r0) * 32; e += kThreads) {
    const int qi = e >> 5, c4 = (e & 31) * 4;
    float all = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all = fmaxf(all, s_m[w][qi]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += all == -INFINITY ? 0.f : s_l[w][qi] * exp2_approx(s_m[w][qi] - all);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(meet + ((size_t)w * 8 * NT + qi) * 132 + c4);
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    if (Q4) all -= kLift;
    if (a.split > 0) {                                     // (only this thread reads these four places)
      *reinterpret_cast<float4*>(meet + (size_t)qi * 132 + c4) = o;
      if (c4 == 0) s_ml[qi] = make_float2(all, sum);
    } else if (t_hi - t_lo < it.tiles) {                   // a part: of the item this run begins or ends in
      const size_t at = ((size_t)blockIdx.x * 2 + (t_lo == 0 ? 1 : 0)) * 8 * NT + qi;
      *reinterpret_cast<float4*>(a.part_o + at * 128 + c4) = o;
      if (c4 == 0) {
        a.part_ml[at * 2] = all;
        a.part_ml[at * 2 + 1] = sum;
      }
    } else {
      finish(qi, c4, o, all, sum);
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
      float2 part[1 << kMostSplit];
      float4 x[1 << kMostSplit];
      float all = -INFINITY, sum = 0.f;
#pragma unroll
      for (int c = 0; c < (1 << kMostSplit); ++c) {
        if (c >> a.split) break;
        part[c] = peer_float2(peer_addr(ml, c));
        x[c] = peer_float4(peer_addr(at, c));
        all = fmaxf(all, part[c].x);
      }
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int c = 0; c < (1 << kMostSplit); ++c) {
        if (c >> a.split) break;
        const float f = all == -INFINITY ? 1.f : exp2_approx(part[c].x - all);                 // (all -inf: zeros, or NaN)
        sum = fmaf(f, part[c].y, sum);
        o.x = fmaf(f, x[c].x, o.x); o.y = fmaf(f, x[c].y, o.y); o.z = fmaf(f, x[c].z, o.z); o.w = fmaf(f, x[c].w, o.w);
      }
      finish(qi, c4, o, all, sum);
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

// Joins the parts of items that several CTAs share: O = sum_c 2^(m_c - m) O_c / sum_c 2^(m_c - m) l_c,
// in the order of the CTAs.  grid = items * block_rows, block = 32 (four channels a lane).
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
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml);
  auto at = [&](int c) { return part(min(c, c1)); };
  auto values = [&](int c) { return *reinterpret_cast<const float4*>(a.part_o + at(c) * 128 + lane * 4); };
  const float2 first = ml[at(c0 + lane)];
  float4 x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = values(c0 + k);
  float all = first.x;
  for (int c = c0 + 32 + lane; c <= c1; c += 32) all = fmaxf(all, ml[part(c)].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
  float sum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int cb = c0; cb <= c1; cb += 32) {
    const float2 e = cb == c0 ? first : ml[at(cb + lane)];
    const float f = cb + lane > c1 ? 0.f : (all == -INFINITY ? 1.f : exp2_approx(e.x - all));      // (all -inf: zeros, or NaN)
    float l = f * e.y;
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
  uint2 v;
  v.x = pack_bf16(o.x * inv, o.y * inv);
  v.y = pack_bf16(o.z * inv, o.w * inv);
  *reinterpret_cast<uint2*>(a.O + b * a.o_sb + (int64_t)hq * a.o_sh + (int64_t)i * a.o_sn + lane * 4) = v;
  if (lane == 0 && a.lse != nullptr)
    a.lse[((int64_t)b * a.heads * a.group + hq) * a.q_n + i] =
        sum == 0.f ? -INFINITY : (all + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace token
}  // namespace curdkv
