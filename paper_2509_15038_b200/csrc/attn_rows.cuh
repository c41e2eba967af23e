// Attention of a few query rows per KV head over bf16 rows, in parts that a second kernel joins: the generation step over a
// cache whose rows collect the weights they receive (curdkv_cache_attention), and the own rows, and short prefixes, of
// a batch that shares a prefix (curdkv_attention_prefix).
//
// A part is a run of `chunk` keys of one item (a KV head and a block of 8 or 16 query rows), a CTA each: it leaves its
// reference m (log2 units), sum l = sum 2^(x - m) and sums of values o = sum 2^(x - m) v in fp32.  With M the largest m,
//   O = (sum 2^(m - M) o) / L,  L = sum 2^(m - M) l,  and a key's weight is 2^(x - M) / L,
// for which the parts also leave the logits x where weights are asked for: they are known to be right only when all keys
// have been seen, and 4 bytes a key and query row are less than its 256 bytes of K read again.
//
// As in attn_token.cuh a warp takes 16 keys at a time from a ring that asynchronous copies fill, forms S^T = K Q^T and
// O^T += V^T P^T with keys as the M side of m16n8k16, and moves its reference only when a logit exceeds it by more than
// 2^slack.  Weights are rounded to bf16 before they multiply the values (2^-9 of each weight), the sums take them
// unrounded.
#pragma once
#include "warp_ptx.cuh"

namespace curdkv {
namespace rows {

constexpr int kKeys = 16;                                  // of a warp's step
constexpr int kStages = 3;
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
  int pitch;                         // even
  uint32_t* status;
};

// Rows of a set that exist; a count out of range is cut and noted.
__device__ __forceinline__ int rows_held(const int32_t* lens, int set, int n_max, bool& ok) {
  if (lens == nullptr) return n_max;
  const int n = lens[set], cut = min(max(n, 0), n_max);
  ok = n == cut;
  return cut;
}

template <int NT>
constexpr int smem_bytes() {
  constexpr int ring = kWarps * kStages * kStageBytes, meet = kWarps * 8 * NT * 132 * 4;
  return ring > meet ? ring : meet;
}

template <int NT, bool LOGITS>
__global__ void __launch_bounds__(kThreads, 2) part_kernel(const Args a) {
  using namespace token;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float2 s_ml[kWarps][8 * NT];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // the joining kernel waits for this one's end

  const int item = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int p = item / a.blocks, blk = item % a.blocks, set = p / a.q.heads, h = p % a.q.heads;
  bool held_ok = true;
  const int held = rows_held(a.lens, set, a.n_max, held_ok);
  if (!held_ok && chunk == 0 && tid == 0) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
  const int k0 = chunk * a.chunk, k1 = min(held, k0 + a.chunk);          // (chunks * chunk stays below 2^31)
  if (k0 >= k1) return;
  const int r0 = blk * 8 * NT, r1 = min(a.q.rows, r0 + 8 * NT);

  // ------------------------------------------------------------ the ring of this warp
  const uint32_t ring = smem_addr(smem) + warp * kStages * kStageBytes;
  const __nv_bfloat16* kb = a.K.base + set * a.K.stride_b + h * a.K.stride_h + (lane & 15) * 8;
  const __nv_bfloat16* vb = a.V.base + set * a.V.stride_b + h * a.V.stride_h + (lane & 15) * 8;
  auto fetch = [&](int u0, int stage) {
    const uint32_t dst = ring + stage * kStageBytes;
#pragma unroll
    for (int i = 0; i < kKeys / 2; ++i) {
      const int key = 2 * i + (lane >> 4);
      const bool live = u0 + key < k1;
      const int64_t j = live ? u0 + key : k0;
      const uint32_t at = (uint32_t)(key * 256 + (((lane & 15) ^ (key & 7)) * 16));
      copy16(dst + at, kb + j * a.K.stride_n, live);
      copy16(dst + kKeys * 256 + at, vb + j * a.V.stride_n, live);
    }
  };
  constexpr int kStep = kWarps * kKeys;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    const int u = k0 + warp * kKeys + s * kStep;
    if (u < k1) fetch(u, s);
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
  float* logits = LOGITS ? a.logits + ((int64_t)p * a.blocks + blk) * a.n_max * a.pitch : nullptr;

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
      if (ahead < k1) fetch(ahead, stage == 0 ? kStages - 1 : stage - 1);
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
            *reinterpret_cast<float2*>(logits + (int64_t)(u0 + 8 * i + g) * a.pitch + 8 * nt + 2 * t) =
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
    uint32_t pt[NT][2];                                    // P^T as B operand
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < 4; ++j) s[nt][j] = exp2_approx(s[nt][j] - (m[nt][j & 1] == -INFINITY ? 0.f : m[nt][j & 1]));
      l[nt][0] += s[nt][0] + s[nt][2];
      l[nt][1] += s[nt][1] + s[nt][3];
#pragma unroll
      for (int i = 0; i < 2; ++i) pt[nt][i] = transpose8x8(pack_bf16(s[nt][2 * i], s[nt][2 * i + 1]));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t x[4];                                       // V^T: channels 16 i .. + 15 of the 16 keys
      const int key = (lane & 7) + ((lane >> 4) & 1) * 8, c = 2 * i + ((lane >> 3) & 1);
      ldmatrix4_trans(x, st + kKeys * 256 + key * 256 + ((c ^ (key & 7)) * 16));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_bf16(acc[nt][i], x[0], x[1], x[2], x[3], pt[nt][0], pt[nt][1]);
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
  const size_t part = (size_t)blockIdx.x * 8 * NT;
  for (int e = tid; e < (r1 - r0) * 32; e += kThreads) {
    const int qi = e >> 5, c4 = (e & 31) * 4;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(meet + ((size_t)w * 8 * NT + qi) * 132 + c4);
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    *reinterpret_cast<float4*>(a.part_o + (part + qi) * 128 + c4) = o;
    if (c4 == 0) {
      float all = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) all = fmaxf(all, s_ml[w][qi].x);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += s_ml[w][qi].y * (all == -INFINITY ? 1.f : exp2_approx(s_ml[w][qi].x - all));
      a.part_ml[part + qi] = make_float2(all, sum);
    }
  }
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
  __nv_bfloat16* O;                  // [batch][heads * group][t][128], strides in elements
  int64_t o_sb, o_sh, o_sn;
  float* lse;
  int slices;                        // CTAs per problem
  const float* logits;               // as in Args, with LOGITS
  int n_max, pitch, block_rows;
  float* weights;                    // [batch][heads][n_max]
};

constexpr int kJoinWarps = 4;
constexpr int kMostRows = 1024;                            // query rows of a problem whose weights are kept

// A warp per query row joins its parts, in their order; with LOGITS the problem's CTAs then add the weights of their share
// of the keys, summed over the query rows in order.  grid = sequences * heads * slices.
template <bool PREFIX, bool LOGITS>
__global__ void __launch_bounds__(kJoinWarps * 32) join_parts_kernel(const JoinArgs a) {
  __shared__ float2 s_norm[LOGITS ? kMostRows : 1];        // reference, 1 / sum
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int p = blockIdx.x / a.slices, slice = blockIdx.x % a.slices, b = p / a.heads, h = p % a.heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rows = a.t * a.group, live = a.q_lens != nullptr ? min(max(a.q_lens[b], 0), a.t) : a.t;
  const int own = a.own.used(b), set = PREFIX ? b / a.share : 0, all_parts = own + (PREFIX ? a.prefix.used(set) : 0);
  for (int r = LOGITS ? warp : warp + slice * kJoinWarps; r < rows; r += LOGITS ? kJoinWarps : kJoinWarps * a.slices) {
    const int i = r / a.group, g = r % a.group;
    if (i >= live) {
      if (LOGITS && lane == 0) s_norm[r] = make_float2(0.f, 0.f);
      continue;
    }
    const size_t own_at = a.own.entry(p, 0, i, g, a.t, a.group);
    const size_t pre_at = PREFIX ? a.prefix.entry(set * a.heads + h, b % a.share, i, g, a.t, a.group) : 0;
    auto entry = [&](int c) {
      return PREFIX && c >= own ? pre_at + (size_t)(c - own) * a.prefix.tile_rows : own_at + (size_t)c * a.own.tile_rows;
    };
    auto ml = [&](int c) { return (PREFIX && c >= own ? a.prefix.ml : a.own.ml)[entry(c)]; };
    float top = -INFINITY;
    for (int c = lane; c < all_parts; c += 32) top = fmaxf(top, ml(c).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    auto share = [&](float m) { return top == -INFINITY ? 1.f : token::exp2_approx(m - top); };    // (top -inf: zeros, or NaN)
    const bool mine = !LOGITS || (r / kJoinWarps) % a.slices == slice;
    float sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = 0; c0 < all_parts; c0 += 32) {
      const float2 e = c0 + lane < all_parts ? ml(c0 + lane) : make_float2(-INFINITY, 0.f);
      const float f = c0 + lane < all_parts ? share(e.x) : 0.f;
      float l = f * e.y;
      if (c0 + lane >= all_parts) l = 0.f;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
      sum += l;
      if (!mine) continue;
      const int n = min(32, all_parts - c0);
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const int c = c0 + k;
        const float4 x = *reinterpret_cast<const float4*>((PREFIX && c >= own ? a.prefix.o : a.own.o) + entry(c) * 128 + lane * 4);
        const float fk = __shfl_sync(0xffffffffu, f, k);
        o.x = fmaf(fk, x.x, o.x); o.y = fmaf(fk, x.y, o.y); o.z = fmaf(fk, x.z, o.z); o.w = fmaf(fk, x.w, o.w);
      }
    }
    const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);        // a NaN sum stays one
    if (mine) {
      const int hq = h * a.group + g;
      *reinterpret_cast<uint2*>(a.O + b * a.o_sb + hq * a.o_sh + i * a.o_sn + lane * 4) =
          make_uint2(token::pack_bf16(o.x * inv, o.y * inv), token::pack_bf16(o.z * inv, o.w * inv));
      if (lane == 0 && a.lse != nullptr)
        a.lse[((int64_t)b * a.heads * a.group + hq) * a.t + i] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
    if (LOGITS && lane == 0) s_norm[r] = make_float2(top == -INFINITY ? 0.f : top, inv);
  }
  if (!LOGITS) return;
  __syncthreads();
  const int held = seq_len_of(a.own.lens, b, a.n_max);
  const int j0 = (int)((int64_t)held * slice / a.slices), j1 = (int)((int64_t)held * (slice + 1) / a.slices);
  const int blocks = (rows + a.block_rows - 1) / a.block_rows;
  for (int j = j0 + threadIdx.x; j < j1; j += kJoinWarps * 32) {
    float w = 0.f;
    for (int blk = 0; blk < blocks; ++blk) {
      const float* x = a.logits + (((int64_t)p * blocks + blk) * a.n_max + j) * a.pitch;
      const int n = min(a.block_rows, rows - blk * a.block_rows);
      for (int r = 0; r < n; r += 2) {
        const float2 v = *reinterpret_cast<const float2*>(x + r);
        const float2 s0 = s_norm[blk * a.block_rows + r];
        w = fmaf(token::exp2_approx(v.x - s0.x), s0.y, w);
        if (r + 1 < n) {
          const float2 s1 = s_norm[blk * a.block_rows + r + 1];
          w = fmaf(token::exp2_approx(v.y - s1.x), s1.y, w);
        }
      }
    }
    a.weights[(int64_t)p * a.n_max + j] += w;
  }
}

}  // namespace rows
}  // namespace curdkv
