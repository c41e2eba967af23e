// Attention of a few query rows per KV head over bf16 rows, in parts that a second kernel joins: the generation step over a
// cache whose rows collect the weights they receive (curdkv_cache_attention), and the own rows, and short prefixes, of
// a batch that shares a prefix (curdkv_attention_prefix).
//
// A part is a run of `chunk` keys of one item (a KV head and a block of 8 or 16 query rows), a CTA each: it leaves its
// reference m (log2 units), sum l = sum 2^(x - m) and sums of values o = sum 2^(x - m) v in fp32.  With M the largest m,
//   O = (sum 2^(m - M) o) / L,  L = sum 2^(m - M) l,  and a key's weight is 2^(x - M) / L,
// for which the parts also leave the logits x where weights are asked for: M and L are there only when all keys have been
// seen, and 4 bytes a key and query row are less than its 256 bytes of K read again.  Where a cluster's shared memory holds a
// head's logits the parts are its CTAs, and one launch does all of it.
//
// As in attn_token.cuh a warp takes 16 keys at a time from a ring that asynchronous copies fill, forms S^T = K Q^T and
// O^T += V^T P^T with keys as the M side of m16n8k16, and moves its reference only when a logit exceeds it by more than
// 2^slack.  Weights multiply the values as two bf16 parts each (2^-16 of each is lost), so that O's own rounding is all that is
// left of its error; rounded to one they added a fifth to it, and the second product costs 0 to 5 % (8 heads of 1702 rows 7.9 ->
// 8.2 us, 1024 of 2048 177.9 -> 179.1, 64 of 65540 with 8 query rows 464 -> 470 for a step).
//
// What bounds it: bytes.  1024 heads of 2048 rows (1.07 GB) 158 us without weights, 6.8 TB/s, and 177 with (the logits'
// 33 MB written and read, 16 MB of weights); 64 heads of 65540 rows, 8 query rows, 315 and 424 us (134 MB of logits).  8
// heads of 1702 rows 8.2 us: a launch, one dependent chain of loads in a cluster of eight, the join.  Beyond 16 query rows
// keys and values are read once for every 16 of them, and logits outgrow them: 64 heads of 65540 rows with 32 rows 610 and
// 853 us, with 256 4250 and 5830.
// Measured and dropped (with one product a weight): streaming hints on the logits' stores (no change); rings of three with 14 KB of logits a CTA, so
// clusters of two for 1024 heads (211 us); a warp per row for the join of many parts (53 us where four warps a row with
// their loads ahead take 14, cold).
#pragma once
#include "warp_ptx.cuh"

namespace curdkv {
namespace rows {

constexpr int kKeys = 16;                                  // of a warp's step
constexpr int kStages = 2;                                 // (three leave room for two CTAs an SM: 128 heads of 2048 rows 29.0 us, so 23.3)
constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStageBytes = 2 * kKeys * 256;
constexpr float kSlack = 6.f;
constexpr float kLn2 = 0.6931471805599453f;

// Query rows: a set of `share` sequences, t tokens each, and the `group` query heads of one KV head.  Row r is head r % group
// of token (r / group) % t of sequence r / (group t) of the set.
struct Queries {
  const __nv_bfloat16* Q;            // [sets * share][heads * group][t][128], strides in elements
  int64_t q_sb, q_sh, q_sn;
  int heads, group, t, share;
  int rows;                          // share * t * group
};

struct Args {
  Queries q;
  const int32_t* q_lens;             // [sets * share] live tokens, or nullptr
  KvView K, V;                       // rows of each set and head
  const int32_t* lens;               // [sets] rows that exist, or nullptr
  int n_max;
  const int32_t* pos;                // [sets][heads][n_max] positions of the rows, nullptr: row j is at j
  const int32_t* total;              // [sets] tokens so far (with pos): token i is at total - q_len + i
  int causal;                        // 0: every query sees every row; 1: rows at or before its position
  int blocks;                        // of query rows per KV head
  int chunk, chunks;                 // keys a part takes, parts per item
  float scale_log2;
  float2* part_ml;                   // [items][chunks][8 NT]: m, l
  float* part_o;                     // [items][chunks][8 NT][128]
  float* logits;                     // [sets * heads][blocks][n_max][pitch], or nullptr
  int stages;                        // of a warp's ring: kStages, or 1 with chunk <= 64
  int late;                          // 1: runs beside the kernel before it
  int pitch;                         // 2 or a multiple of 4, at least the rows of a block
  uint32_t* status;
};

// Rows of a set that exist; a count out of range is cut and noted.
__device__ __forceinline__ int rows_held(const int32_t* lens, int set, int n_max, bool& ok) {
  if (lens == nullptr) return n_max;
  const int n = lens[set], cut = min(max(n, 0), n_max);
  ok = n == cut;
  return cut;
}

// Shared memory of a CTA with rings of `stages`: two, or one where a part is a single step of its warps.
template <int NT>
__host__ __device__ constexpr int smem_bytes(int stages = kStages) {
  const int ring = kWarps * stages * kStageBytes, meet = kWarps * 8 * NT * 132 * 4;
  return ring > meet ? ring : meet;
}

// Where results go.
struct Outputs {
  __nv_bfloat16* O;                  // [batch][heads * group][t][128], strides in elements
  int64_t o_sb, o_sh, o_sn;
  float* lse;                        // [batch][heads * group][t] or nullptr
  float* weights;                    // [batch][heads][n_max] or nullptr
};

__device__ __forceinline__ float inverse(float sum) { return sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum); }   // a NaN sum stays one
__device__ __forceinline__ float share(float m, float top) { return top == -INFINITY ? 1.f : token::exp2_approx(m - top); }   // (top -inf: zeros, or NaN)

// FUSED: the parts of an item are the CTAs of a cluster, which join them through distributed shared memory; logits (where
// weights are asked for) stay in shared memory until reference and sum are known, and the call is one launch.
constexpr int kMostSplit = 3;                              // log2 of the CTAs of a cluster
constexpr int kLogitBytes = 35 * 1024;                     // of a CTA; two an SM fit beside their rings

template <int NT, bool LOGITS, bool FUSED>
__global__ void __launch_bounds__(kThreads, 2) part_kernel(const __grid_constant__ Args before, const __grid_constant__ Args behind,
                                                           const int first_ctas, const Outputs out) {
  using namespace token;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float2 s_ml[kWarps][8 * NT];
  __shared__ float2 s_cta[8 * NT];                         // FUSED: this CTA's references and sums
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // the joining kernel waits for this one's end

  // two sets of parts may share a launch (the prefix's and the own rows'): the first CTAs take the first
  const bool second = (int)blockIdx.x >= first_ctas;
  const Args& a = second ? behind : before;
  const int cta = (int)blockIdx.x - (second ? first_ctas : 0);
  const int item = cta / a.chunks, chunk = cta % a.chunks;             // (FUSED: chunk = rank in the cluster)
  if (!a.late) asm volatile("griddepcontrol.wait;" ::: "memory");
  const int p = item / a.blocks, blk = item % a.blocks, set = p / a.q.heads, h = p % a.q.heads;
  bool held_ok = true;
  const int held = rows_held(a.lens, set, a.n_max, held_ok);
  if (!held_ok && chunk == 0 && tid == 0) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
  // (chunks * chunk stays below 2^31; the CTAs of a cluster share what is there evenly)
  const int each = FUSED ? ((held + a.chunks - 1) / a.chunks + kKeys - 1) / kKeys * kKeys : a.chunk;
  const int k0 = chunk * each, k1 = min(held, k0 + each);
  // With `late` the kernel before this one has begun and nothing of it is needed here, but the joining kernel, which waits for
  // the end of this one only, needs both: the first CTA stays until that one has ended, the others make room.
  auto wait_late = [&]() {
    if (a.late && blockIdx.x == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
  };
  if (!FUSED && k0 >= k1) {
    wait_late();
    return;
  }
  const int r0 = blk * 8 * NT, r1 = min(a.q.rows, r0 + 8 * NT);

  // ------------------------------------------------------------ the ring of this warp
  const int stages = FUSED ? kStages : a.stages;
  const uint32_t ring = smem_addr(smem) + warp * stages * kStageBytes;
  const __nv_bfloat16* kb = a.K.base + set * a.K.stride_b + h * a.K.stride_h + (lane & 15) * 8;
  const __nv_bfloat16* vb = a.V.base + set * a.V.stride_b + h * a.V.stride_h + (lane & 15) * 8;
  // rows that one block of queries reads once leave the L2 to the logits and parts (1024 heads of 2048 rows 189 -> 182 us)
  uint64_t pol;
  if (a.blocks > 1) asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pol));
  else asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
  auto fetch = [&](int u0, int stage) {
    const uint32_t dst = ring + stage * kStageBytes;
#pragma unroll
    for (int i = 0; i < kKeys / 2; ++i) {
      const int key = 2 * i + (lane >> 4);
      const bool live = u0 + key < k1;
      const int64_t j = live ? u0 + key : k0;
      const uint32_t at = (uint32_t)(key * 256 + (((lane & 15) ^ (key & 7)) * 16));
      copy16(dst + at, kb + j * a.K.stride_n, live, pol);
      copy16(dst + kKeys * 256 + at, vb + j * a.V.stride_n, live, pol);
    }
  };
  constexpr int kStep = kWarps * kKeys;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    const int u = k0 + warp * kKeys + s * kStep;
    if (s < stages && u < k1) fetch(u, s);                 // (a ring of one: the only step)
    copy_commit();
  }

  // ------------------------------------------------------------ query rows: B operand of S^T, and their positions
  uint32_t q[NT][16];
  int at[NT][2];                                           // of queries 2t, 2t + 1
  const int per = a.q.group * a.q.t;
  auto place = [&](int r, int& i) {                        // sequence of row r, its token
    i = (r / a.q.group) % a.q.t;
    return set * a.q.share + r / per;
  };
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = r0 + 8 * nt + g;
    const bool live = r < r1;
    int i = 0;
    const int b = place(live ? r : 0, i);
    const __nv_bfloat16* src = a.q.Q + b * a.q.q_sb + (int64_t)(h * a.q.group + (live ? r % a.q.group : 0)) * a.q.q_sh + i * a.q.q_sn;
#pragma unroll
    for (int s = 0; s < 8; ++s)
#pragma unroll
      for (int e = 0; e < 2; ++e) q[nt][2 * s + e] = live ? *reinterpret_cast<const uint32_t*>(src + 16 * s + 8 * e + 2 * t) : 0u;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int rr = r0 + 8 * nt + 2 * t + c;
      at[nt][c] = 0x7fffffff;                              // sees every row
      if (rr >= r1) {
        at[nt][c] = (int)0x80000000;
      } else if (a.causal || a.q_lens != nullptr) {
        int ti;
        const int bb = place(rr, ti);
        const int live_t = a.q_lens != nullptr ? min(max(a.q_lens[bb], 0), a.q.t) : a.q.t;
        if (ti >= live_t) at[nt][c] = (int)0x80000000;     // no query
        else if (a.causal) at[nt][c] = (a.pos != nullptr ? a.total[set] : held) - live_t + ti;
      }
    }
  }
  // every query of the block sees every row up to:
  int sees_to = 0x7fffffff;
  if (a.causal || a.q_lens != nullptr) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (r0 + 8 * nt + 2 * t + c < r1) sees_to = min(sees_to, at[nt][c]);
    sees_to = __reduce_min_sync(0xffffffffu, sees_to);
  }
  const int32_t* pos = a.pos != nullptr ? a.pos + (int64_t)p * a.n_max : nullptr;
  float* logits = nullptr;                                 // of key k0 onwards
  if (LOGITS) {
    if (FUSED) logits = reinterpret_cast<float*>(smem + smem_bytes<NT>());
    else logits = a.logits + (((int64_t)p * a.blocks + blk) * a.n_max + k0) * a.pitch;
  }

  float acc[NT][8][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[nt][i][j] = 0.f;
    m[nt][0] = m[nt][1] = -INFINITY;
    l[nt][0] = l[nt][1] = 0.f;
  }

  // ------------------------------------------------------------ the key loop
  int stage = 0;
  for (int u0 = k0 + warp * kKeys; u0 < k1; u0 += kStep) {
    {
      const int ahead = u0 + (kStages - 1) * kStep;        // (k1 + 3 kStep stays below 2^31)
      if (ahead < k1) fetch(ahead, stage == 0 ? kStages - 1 : stage - 1);            // (never with a ring of one)
      copy_commit();
    }
    int key_at[2];                                         // positions of keys g, g + 8
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int u = u0 + 8 * i + g;
      key_at[i] = u < k1 ? (pos != nullptr ? pos[u] : u) : 0x7fffffff;
    }
    copy_wait<kStages - 1>();
    __syncwarp();
    const uint32_t st = ring + stage * kStageBytes;
    float s[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[nt][j] = 0.f;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      uint32_t x[4];
      const int key = lane & 15, c = 2 * ks + (lane >> 4);
      ldmatrix4(x, st + key * 256 + ((c ^ (key & 7)) * 16));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_bf16(s[nt], x[0], x[1], x[2], x[3], q[nt][2 * ks], q[nt][2 * ks + 1]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[nt][j] *= a.scale_log2;
    // (a key that does not exist stands at the greatest position, which only queries that see everything reach)
    if (u0 + kKeys > k1 || pos != nullptr || sees_to < u0 + kKeys - 1) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (key_at[j >> 1] > at[nt][j & 1] || u0 + 8 * (j >> 1) + g >= k1) s[nt][j] = -INFINITY;
    }
    if (LOGITS) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (8 * nt + 2 * t < a.pitch && u0 + 8 * i + g < k1)
            *reinterpret_cast<float2*>(logits + (int64_t)(u0 - k0 + 8 * i + g) * a.pitch + 8 * nt + 2 * t) =
                make_float2(s[nt][2 * i], s[nt][2 * i + 1]);
    }
    bool move = false;
    float top[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        top[nt][c] = fmaxf(s[nt][c], s[nt][2 + c]);
        move = move || top[nt][c] > m[nt][c] + kSlack;
      }
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float x = top[nt][c];
#pragma unroll
          for (int o = 4; o <= 16; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
          const float now = fmaxf(m[nt][c], x), f = now == -INFINITY ? 1.f : exp2_approx(m[nt][c] - now);
          m[nt][c] = now;
          l[nt][c] *= f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            acc[nt][i][c] *= f;
            acc[nt][i][2 + c] *= f;
          }
        }
    }
    uint32_t hi[NT][2], lo[NT][2];                         // P^T as B operand, in two parts
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < 4; ++j) s[nt][j] = exp2_approx(s[nt][j] - (m[nt][j & 1] == -INFINITY ? 0.f : m[nt][j & 1]));
      l[nt][0] += s[nt][0] + s[nt][2];
      l[nt][1] += s[nt][1] + s[nt][3];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t a0, a1;
        split_bf16(s[nt][2 * i], s[nt][2 * i + 1], a0, a1);
        hi[nt][i] = transpose8x8(a0);
        lo[nt][i] = transpose8x8(a1);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t x[4];                                       // V^T: channels 16 i .. + 15 of the 16 keys
      const int key = (lane & 7) + ((lane >> 4) & 1) * 8, c = 2 * i + ((lane >> 3) & 1);
      ldmatrix4_trans(x, st + kKeys * 256 + key * 256 + ((c ^ (key & 7)) * 16));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma_bf16(acc[nt][i], x[0], x[1], x[2], x[3], hi[nt][0], hi[nt][1]);
        mma_bf16(acc[nt][i], x[0], x[1], x[2], x[3], lo[nt][0], lo[nt][1]);
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
      if (g == 0) s_ml[warp][8 * nt + 2 * t + c] = make_float2(m[nt][c], l[nt][c]);
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
      for (int w = 0; w < kWarps; ++w) all = fmaxf(all, s_ml[w][qi].x);
      const float f = all == -INFINITY ? 1.f : exp2_approx(m[nt][c] - all);        // (all -inf: zeros, or NaN)
      float* dst = meet + ((size_t)warp * 8 * NT + qi) * 132;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dst[16 * i + g] = acc[nt][i][c] * f;
        dst[16 * i + 8 + g] = acc[nt][i][2 + c] * f;
      }
    }
  __syncthreads();
  const size_t part = (size_t)cta * 8 * NT;
  for (int e = tid; e < (r1 - r0) * 32; e += kThreads) {
    const int qi = e >> 5, c4 = (e & 31) * 4;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(meet + ((size_t)w * 8 * NT + qi) * 132 + c4);
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    float2 ml = make_float2(-INFINITY, 0.f);
    if (c4 == 0) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) ml.x = fmaxf(ml.x, s_ml[w][qi].x);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) ml.y += s_ml[w][qi].y * share(s_ml[w][qi].x, ml.x);
    }
    if (FUSED) {                                           // (only this thread reads these four places)
      *reinterpret_cast<float4*>(meet + (size_t)qi * 132 + c4) = o;
      if (c4 == 0) s_cta[qi] = ml;
    } else {
      *reinterpret_cast<float4*>(a.part_o + (part + qi) * 128 + c4) = o;
      if (c4 == 0) a.part_ml[part + qi] = ml;
    }
  }
  if constexpr (FUSED) {
    // ---------------------------------------------------------- the cluster joins its parts, in the order of their ranks
    __shared__ float2 s_norm[8 * NT];                      // reference, 1 / sum
    __shared__ float2 s_all[1 << kMostSplit][8 * NT];
    // (the old weights are asked for before the wait for the others)
    float* weights = LOGITS ? out.weights + (int64_t)p * a.n_max + k0 : nullptr;
    constexpr int kAhead = 5;                              // (18: 1024 heads of 500 rows 56.5 -> 58.9 us, for the code's length)
    float was[kAhead];
    auto ask = [&](int from, float (&x)[kAhead]) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (from + tid + k * kThreads < k1 - k0) x[k] = weights[from + tid + k * kThreads];
    };
    if (LOGITS) ask(0, was);
    if (a.chunks > 1) cluster_sync(); else __syncthreads();
    for (int e = tid; e < a.chunks * 8 * NT; e += kThreads) {
      const int c = e / (8 * NT), qi = e % (8 * NT);
      if (a.chunks == 1) {
        s_all[c][qi] = s_cta[qi];
      } else {
        float2 v;
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(peer_addr(smem_addr(&s_cta[qi]), c)) : "memory");
        s_all[c][qi] = v;
      }
    }
    __syncthreads();
    if (LOGITS && tid < 8 * NT) {
      float top = -INFINITY, sum = 0.f;
      int i = 0;
      const bool there = tid < r1 - r0;
      const int bb = place(there ? r0 + tid : 0, i);
      const bool live = there && i < (a.q_lens != nullptr ? min(max(a.q_lens[bb], 0), a.q.t) : a.q.t);
      for (int c = 0; c < a.chunks; ++c) top = fmaxf(top, s_all[c][tid].x);
      for (int c = 0; c < a.chunks; ++c) sum = fmaf(share(s_all[c][tid].x, top), s_all[c][tid].y, sum);
      // (a row that does not exist weighs nothing)
      s_norm[tid] = live ? make_float2(top == -INFINITY ? 0.f : top, inverse(sum)) : make_float2(0.f, 0.f);
    }
    const int rows = r1 - r0;
    for (int e = chunk * kThreads + tid; e < rows * 32; e += a.chunks * kThreads) {
      const int qi = e >> 5, c4 = (e & 31) * 4;
      float2 ml[1 << kMostSplit];
      float4 x[1 << kMostSplit];
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int c = 0; c < (1 << kMostSplit); ++c) {
        if (c >= a.chunks) break;
        ml[c] = s_all[c][qi];
        const float* at_c4 = meet + (size_t)qi * 132 + c4;
        x[c] = a.chunks == 1 ? *reinterpret_cast<const float4*>(at_c4) : peer_float4(peer_addr(smem_addr(at_c4), c));
        top = fmaxf(top, ml[c].x);
      }
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int c = 0; c < (1 << kMostSplit); ++c) {
        if (c >= a.chunks) break;
        const float f = share(ml[c].x, top);
        sum = fmaf(f, ml[c].y, sum);
        o.x = fmaf(f, x[c].x, o.x); o.y = fmaf(f, x[c].y, o.y); o.z = fmaf(f, x[c].z, o.z); o.w = fmaf(f, x[c].w, o.w);
      }
      int i;
      const int r = r0 + qi, bb = place(r, i), hq = h * a.q.group + r % a.q.group;
      const int live = a.q_lens != nullptr ? min(max(a.q_lens[bb], 0), a.q.t) : a.q.t;
      if (i >= live) continue;                             // rows behind the last query stay as they are
      const float inv = inverse(sum);
      *reinterpret_cast<uint2*>(out.O + bb * out.o_sb + hq * out.o_sh + i * out.o_sn + c4) =
          make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
      if (c4 == 0 && out.lse != nullptr)
        out.lse[((int64_t)bb * a.q.heads * a.q.group + hq) * a.q.t + i] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
    if (LOGITS) {
      __syncthreads();
      auto weight = [&](int j) {
        const float* x = logits + (size_t)j * a.pitch;
        float w = 0.f;
        for (int r = 0; r < a.pitch; r += 2) {
          const float2 v = *reinterpret_cast<const float2*>(x + r), n0 = s_norm[r], n1 = s_norm[r + 1];
          w = fmaf(exp2_approx(v.x - n0.x), n0.y, w);
          w = fmaf(exp2_approx(v.y - n1.x), n1.y, w);
        }
        return w;
      };
      for (int from = 0; from < k1 - k0; from += kAhead * kThreads) {
        float next[kAhead];
        ask(from + kAhead * kThreads, next);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int j = from + tid + k * kThreads;
          if (j < k1 - k0) weights[j] = was[k] + weight(j);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) was[k] = next[k];
      }
    }
    if (a.chunks > 1) cluster_sync();                      // nobody leaves while its parts are read
  }
  wait_late();
}

// ---- joining -----------------------------------------------------------------------------------

// The parts of a call: `chunks` per item at most, each of tile_rows query rows; an item is a problem (set, KV head) and a
// tile.  Tiles hold consecutive rows, or (seqs > 0) `tokens` tokens of `seqs` sequences each, `token_tiles` tiles a sequence.
struct Parts {
  const float2* ml;
  const float* o;
  const int32_t* lens;               // [sets] rows, or nullptr
  int n_max, chunk, chunks;
  int tile_rows, tiles;              // per problem
  int seqs, tokens, token_tiles;
  __device__ __forceinline__ int used(int set) const {                 // parts that have keys
    const int n = seq_len_of(lens, set, n_max);
    return (n + chunk - 1) / chunk;
  }
  // first part's entry of query row (sequence s of the set, token i, head g of the group) of a problem
  __device__ __forceinline__ size_t entry(int problem, int s, int i, int g, int t, int group) const {
    int tile, row;
    if (seqs > 0) {
      tile = (s / seqs) * token_tiles + i / tokens;
      row = ((s % seqs) * tokens + i % tokens) * group + g;
    } else {
      const int r = (s * t + i) * group + g;
      tile = r / tile_rows;
      row = r % tile_rows;
    }
    return ((size_t)problem * tiles + tile) * chunks * tile_rows + row;
  }
};

struct JoinArgs {
  Parts own, prefix;                 // prefix: only with PREFIX
  int heads, group, t, share;        // (set of the prefix: sequence / share)
  const int32_t* q_lens;
  Outputs out;
  int slices;                        // CTAs per problem
  int by_warp;                       // 1: a warp per query row (few parts, many rows)
  const float* logits;               // as in Args, with LOGITS
  int n_max, pitch, block_rows;
};

constexpr int kJoinWarps = 4;
constexpr int kMostRows = 1024;                            // query rows of a problem whose weights are kept

// The CTAs of a problem take its query rows in turn.  A row's parts are dealt to the four warps, which ask for four each
// before they know what these count (that, and not their bytes, is what takes time here), and their sums are added in order.
// With LOGITS the problem's CTAs then add the weights of their share of the keys, summed over the query rows in order.
// grid = sequences * heads * slices.
template <bool PREFIX, bool LOGITS>
__global__ void __launch_bounds__(kJoinWarps * 32) join_parts_kernel(const JoinArgs a) {
  __shared__ float2 s_norm[LOGITS ? kMostRows + 16 : 1];   // reference, 1 / sum
  __shared__ float4 s_part[2][kJoinWarps][32];
  const int p = blockIdx.x / a.slices, slice = blockIdx.x % a.slices, b = p / a.heads, h = p % a.heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rows = a.t * a.group, set = PREFIX ? b / a.share : 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int live = a.q_lens != nullptr ? min(max(a.q_lens[b], 0), a.t) : a.t;
  const int own = a.own.used(b), all_parts = own + (PREFIX ? a.prefix.used(set) : 0);
  struct Row {
    size_t own_at, pre_at;
  };
  auto row_of = [&](int r) {
    const int i = r / a.group, g = r % a.group;
    return Row{a.own.entry(p, 0, i, g, a.t, a.group), PREFIX ? a.prefix.entry(set * a.heads + h, b % a.share, i, g, a.t, a.group) : 0};
  };
  auto ml = [&](const Row& x, int c) {
    return PREFIX && c >= own ? a.prefix.ml[x.pre_at + (size_t)(c - own) * a.prefix.tile_rows] : a.own.ml[x.own_at + (size_t)c * a.own.tile_rows];
  };
  auto values = [&](const Row& x, int c) {
    const float* o = PREFIX && c >= own ? a.prefix.o + (x.pre_at + (size_t)(c - own) * a.prefix.tile_rows) * 128
                                        : a.own.o + (x.own_at + (size_t)c * a.own.tile_rows) * 128;
    return *reinterpret_cast<const float4*>(o + lane * 4);
  };
  auto most = [](float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  };
  auto total = [](float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  };
  // reference and sum of a row, a lane per part
  auto stats = [&](const Row& x, float& top, float& sum) {
    const float2 first = lane < all_parts ? ml(x, lane) : make_float2(-INFINITY, 0.f);
    top = first.x;
    for (int c = 32 + lane; c < all_parts; c += 32) top = fmaxf(top, ml(x, c).x);
    top = most(top);
    sum = lane < all_parts ? share(first.x, top) * first.y : 0.f;
    for (int c = 32 + lane; c < all_parts; c += 32) {
      const float2 e = ml(x, c);
      sum += share(e.x, top) * e.y;
    }
    sum = total(sum);
  };

  auto finish = [&](int i, int g, const float4& o, float top, float sum) {
    const float inv = inverse(sum);
    const int hq = h * a.group + g;
    *reinterpret_cast<uint2*>(a.out.O + b * a.out.o_sb + hq * a.out.o_sh + i * a.out.o_sn + lane * 4) =
        make_uint2(token::pack_bf16(o.x * inv, o.y * inv), token::pack_bf16(o.z * inv, o.w * inv));
    if (lane == 0 && a.out.lse != nullptr)
      a.out.lse[((int64_t)b * a.heads * a.group + hq) * a.t + i] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
  };
  if (!LOGITS && a.by_warp) {
    for (int r = slice * kJoinWarps + warp; r < rows; r += a.slices * kJoinWarps) {
      const int i = r / a.group, g = r % a.group;
      if (i >= live) continue;
      const Row x = row_of(r);
      float4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < all_parts) v[k] = values(x, k);
      float top, sum;
      stats(x, top, sum);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int c0 = 0; c0 < all_parts; c0 += 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (c0 + k >= all_parts) continue;
          const float4 y = c0 == 0 ? v[k] : values(x, c0 + k);
          const float f = share(ml(x, c0 + k).x, top);
          o.x = fmaf(f, y.x, o.x); o.y = fmaf(f, y.y, o.y); o.z = fmaf(f, y.z, o.z); o.w = fmaf(f, y.w, o.w);
        }
      }
      finish(i, g, o, top, sum);
    }
    return;
  }
  int turn = 0;
  for (int r = slice; r < rows; r += a.slices) {
    const int i = r / a.group, g = r % a.group;
    if (i >= live) continue;
    const Row x = row_of(r);
    float4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (warp + 4 * k < all_parts) v[k] = values(x, warp + 4 * k);
    float top, sum;
    stats(x, top, sum);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = warp; c0 < all_parts; c0 += 16) {
      float4 now[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        now[k] = v[k];
        if (c0 + 16 + 4 * k < all_parts) v[k] = values(x, c0 + 16 + 4 * k);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (c0 + 4 * k >= all_parts) continue;
        const float f = share(ml(x, c0 + 4 * k).x, top);
        o.x = fmaf(f, now[k].x, o.x); o.y = fmaf(f, now[k].y, o.y); o.z = fmaf(f, now[k].z, o.z); o.w = fmaf(f, now[k].w, o.w);
      }
    }
    s_part[turn][warp][lane] = o;
    __syncthreads();                                       // (the other buffer is free again behind the next one)
    if (warp == 0) {
#pragma unroll
      for (int w = 1; w < kJoinWarps; ++w) {
        const float4 y = s_part[turn][w][lane];
        o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
      }
      finish(i, g, o, top, sum);
    }
    turn ^= 1;
  }
  if (!LOGITS) return;
  const int blocks = (rows + a.block_rows - 1) / a.block_rows, padded = (blocks - 1) * a.block_rows + a.pitch;
  for (int r = warp; r < padded; r += kJoinWarps) {
    float top = 0.f, inv = 0.f;                            // (a row that does not exist weighs nothing)
    if (r < rows && r / a.group < live) {
      float sum;
      stats(row_of(r), top, sum);
      inv = inverse(sum);
      if (top == -INFINITY) top = 0.f;
    }
    if (lane == 0) {
      s_norm[r].x = top;
      s_norm[r].y = inv;
    }
  }
  __syncthreads();
  const int held = seq_len_of(a.own.lens, b, a.n_max);
  const int j0 = (int)((int64_t)held * slice / a.slices), j1 = (int)((int64_t)held * (slice + 1) / a.slices);
  const float* logits = a.logits + (int64_t)p * blocks * a.n_max * a.pitch;
  float* weights = a.out.weights + (int64_t)p * a.n_max;
  constexpr int kAtOnce = 4;                               // keys of a thread in flight
  for (int j = j0 + threadIdx.x; j < j1; j += kAtOnce * kJoinWarps * 32) {
    float w[kAtOnce], was[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int jk = j + k * kJoinWarps * 32;
      w[k] = 0.f;
      if (jk < j1) was[k] = weights[jk];
    }
    for (int blk = 0; blk < blocks; ++blk) {
      const float* x = logits + ((int64_t)blk * a.n_max + j) * a.pitch;
      const float2* norm = s_norm + blk * a.block_rows;
      if (a.pitch == 2) {
        float2 v[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
          if (j + k * kJoinWarps * 32 < j1) v[k] = *reinterpret_cast<const float2*>(x + k * kJoinWarps * 64);
        const float2 n0 = norm[0], n1 = norm[1];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
          w[k] = fmaf(token::exp2_approx(v[k].y - n1.x), n1.y, fmaf(token::exp2_approx(v[k].x - n0.x), n0.y, w[k]));
        continue;
      }
      for (int r = 0; r < a.pitch; r += 4) {
        float4 v[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
          if (j + k * kJoinWarps * 32 < j1) v[k] = *reinterpret_cast<const float4*>(x + (int64_t)k * kJoinWarps * 32 * a.pitch + r);
        const float2 n0 = norm[r], n1 = norm[r + 1], n2 = norm[r + 2], n3 = norm[r + 3];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          w[k] = fmaf(token::exp2_approx(v[k].x - n0.x), n0.y, w[k]);
          w[k] = fmaf(token::exp2_approx(v[k].y - n1.x), n1.y, w[k]);
          w[k] = fmaf(token::exp2_approx(v[k].z - n2.x), n2.y, w[k]);
          w[k] = fmaf(token::exp2_approx(v[k].w - n3.x), n3.y, w[k]);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (j + k * kJoinWarps * 32 < j1) weights[j + k * kJoinWarps * 32] = was[k] + w[k];
  }
}

}  // namespace rows
}  // namespace curdkv
