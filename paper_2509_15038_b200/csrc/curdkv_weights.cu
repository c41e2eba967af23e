// Generation over a cache whose rows collect the attention weights they receive, and the attention of a
// batch that shares a prefix.  Argument checks and kernel launches.
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "attn_prefix.cuh"
#include "attn_rows.cuh"
#include "host.cuh"

namespace {

using namespace curdkv;
using namespace curdkv::host;

// How the keys of `problems` KV heads with `query_rows` query rows each are cut into parts.
struct RowsPlan {
  int nt, blocks, chunk, chunks;
  size_t entries, most;              // query rows of all parts; and at most, of any call of no larger sizes
};

// Parts at most of up to `items` items of up to `keys` keys.  What plan_rows makes of shorter or fewer ones can be more parts
// (one key fewer, a step less a part: 37 of 128 keys for 4736, 25 of 192 for 4737), so a size that is to serve them too has to come
// from bounds: `slots` parts, or four rounds of them for long caches, of at least 128 keys each; six rounds and a part an
// item, of at least 512 keys, for more items.  Each grows with items and keys.
int64_t most_parts(int64_t items, int64_t keys) {
  const int64_t slots = 2 * (int64_t)sms();
  if (items < 1) items = 1;
  auto of = [](int64_t n, int64_t each) { return n > 0 ? (n + each - 1) / each : 1; };
  auto few = [&](int64_t n) {
    const int64_t rounds = keys / (4 * slots / n) >= 2048 ? 4 * slots : slots, all = n * of(keys, 128);
    return all < rounds ? all : rounds;
  };
  if (items <= slots) return few(items);
  const int64_t rounds = 6 * slots + items, all = items * of(keys, 512), many = all < rounds ? all : rounds, less = few(slots);
  return many > less ? many : less;
}

// As many parts as fill the device (two CTAs an SM) when heads are few, so that a head's keys are read by many SMs, and four
// rounds of them while each has 2048 keys (64 heads of 65540 rows, 8 query rows: 421 us instead of 440, both with one product a weight); several
// rounds of parts when heads are many, so that the last round costs little and ragged heads even out.  A part has at least
// two steps of its four warps (128 keys).
RowsPlan plan_rows(int64_t problems, int64_t query_rows, int64_t keys, int nt = 0) {
  RowsPlan pl;
  pl.nt = nt > 0 ? nt : (query_rows <= 8 ? 1 : 2);
  pl.blocks = (int)((query_rows + 8 * pl.nt - 1) / (8 * pl.nt));
  const int64_t items = problems * pl.blocks > 0 ? problems * pl.blocks : 1, slots = 2 * (int64_t)sms();
  int64_t chunks = items <= slots ? slots / items : (6 * slots + items - 1) / items;
  if (items <= slots && keys / (4 * slots / items) >= 2048) chunks = 4 * slots / items;
  int64_t chunk = chunks > 0 ? (keys + chunks - 1) / chunks : keys;
  const int64_t least = items <= slots ? 128 : 512;
  if (chunk < least) chunk = least;
  if (chunk > keys) chunk = keys > 0 ? keys : 1;
  chunk = (chunk + 63) / 64 * 64;
  chunks = keys > 0 ? (keys + chunk - 1) / chunk : 1;
  pl.chunk = (int)chunk;
  pl.chunks = (int)chunks;
  pl.entries = (size_t)items * chunks * 8 * pl.nt;
  pl.most = (size_t)most_parts(items, keys) * 8 * pl.nt;
  return pl;
}

size_t parts_bytes(size_t entries) { return round256(entries * sizeof(float2)) + round256(entries * 128 * sizeof(float)); }

// Launched behind the kernel before it on the stream without waiting for its end: the kernels themselves wait.  `cluster` CTAs
// each, where above 1.
template <typename Kernel, typename... Args>
bool launch_behind(Kernel kernel, int64_t ctas, int threads, int smem, int cluster, cudaStream_t stream, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) return false;
  return launched();
}

template <int NT, bool LOGITS, bool FUSED>
bool launch_parts(const rows::Args& a, const rows::Outputs& out, int64_t ctas, cudaStream_t stream, const rows::Args* first = nullptr,
                  int64_t first_ctas = 0) {
  constexpr int most = rows::smem_bytes<NT>() + (FUSED && LOGITS ? rows::kLogitBytes : 0);
  static std::atomic<uint64_t> done{0};
  if (!allow_smem(rows::part_kernel<NT, LOGITS, FUSED>, most, done)) return false;
  rows::Args x = a, y = first_ctas > 0 ? *first : a;
  const int64_t longest = ctas == 0 || (first_ctas > 0 && first->chunk > a.chunk) ? y.chunk : x.chunk;
  x.stages = y.stages = longest <= rows::kWarps * rows::kKeys ? 1 : rows::kStages;
  const int smem = FUSED ? most : rows::smem_bytes<NT>(x.stages);
  return launch_behind(rows::part_kernel<NT, LOGITS, FUSED>, first_ctas + ctas, rows::kThreads, smem, FUSED ? a.chunks : 1, stream,
                       y, x, (int)first_ctas, out);
}

template <bool PREFIX, bool LOGITS>
bool launch_join(const rows::JoinArgs& a, int64_t ctas, cudaStream_t stream) {
  return launch_behind(rows::join_parts_kernel<PREFIX, LOGITS>, ctas, rows::kJoinWarps * 32, 0, 1, stream, a);
}

rows::Parts parts_of(const RowsPlan& pl, unsigned char* at, const int32_t* lens, int n_max) {
  rows::Parts x = {};
  x.ml = reinterpret_cast<const float2*>(at);
  x.o = reinterpret_cast<const float*>(at + round256(pl.entries * sizeof(float2)));
  x.lens = lens;
  x.n_max = n_max;
  x.chunk = pl.chunk;
  x.chunks = pl.chunks;
  x.tile_rows = 8 * pl.nt;
  x.tiles = pl.blocks;
  return x;
}

// CTAs that join a problem's parts: one for each query row, as long as a grid holds them.
int join_slices(int64_t problems, int64_t query_rows) {
  const int64_t most = 0x7fffffffLL / (problems > 0 ? problems : 1);
  return (int)(query_rows < most ? query_rows : most);
}

bool cache_ok(const curdkv_cache* c) {
  return c != nullptr && c->K != nullptr && c->V != nullptr && c->raw != nullptr && c->pos != nullptr &&
         c->count != nullptr && c->total != nullptr && c->capacity >= 1;
}

// ---- attention over a generation-phase cache ---------------------------------------------------
struct CachePlan {
  RowsPlan rows;
  int cluster;                       // CTAs of a KV head's cluster; 0: parts and a second kernel
  int pitch, slices;
  size_t parts_at, logits_at, bytes;
};

bool heads_ok(const curdkv_desc* d) {
  return d != nullptr && d->batch >= 0 && d->kv_heads >= 1 && d->q_heads >= d->kv_heads && d->q_heads % d->kv_heads == 0;
}

bool plan_cache(const curdkv_cache* c, const curdkv_desc* d, int32_t q_rows, CachePlan* pl) {
  if (c == nullptr || c->capacity < 1 || c->capacity > (1 << 30) || !heads_ok(d) || q_rows < 1) return false;
  const int64_t P = (int64_t)d->batch * d->kv_heads, rows = (int64_t)(d->q_heads / d->kv_heads) * q_rows;
  if (rows > rows::kMostRows || P > (1 << 24)) return false;
  pl->rows = plan_rows(P, rows, c->capacity);
  pl->pitch = (int)(rows <= 2 ? 2 : (rows < 8 * pl->rows.nt ? (rows + 3) / 4 * 4 : 8 * pl->rows.nt));
  // One launch where a KV head's query rows are one block and its logits fit into the shared memory of a cluster, with more
  // CTAs while all find room on the device and each keeps two steps of its warps.  Not where clusters fill their last round
  // badly, nor where clusters of eight leave half the places empty to long caches.  The rule does not ask for weights, so that
  // outputs are the same with them and without (32 heads of 1702 rows without: 7.9 | 8.1, 128 of 2048 23.2 | 21.6).
  // 4 query rows, with weights, us, clusters | parts and a second kernel:
  //   8 heads of 200 rows 6.3 | 8.9, of 1702 8.2 | 8.7, of 7000 15.8 | 12.6        32 of 1702 9.4 | 11.1        64 of 7000 41 | 42
  //   128 heads of 2048 26.0 | 27.0, of 4096 47 | 49       320 of 2048 81 | 70       480 of 2048 87 | 93       1024 of 500 56 | 64, of 2048 181 | 183
  pl->cluster = 0;
  if (pl->rows.blocks == 1) {
    const int64_t keys = c->capacity, slots = 2 * (int64_t)sms();
    int split = 0;
    auto fits = [&](int k) { return (((keys + (1 << k) - 1) >> k) + rows::kKeys) * pl->pitch * 4 <= rows::kLogitBytes; };
    while (split < rows::kMostSplit && !fits(split)) ++split;
    const bool fit = fits(split);
    while (split < rows::kMostSplit && (P << (split + 1)) <= slots && keys > (2 * rows::kWarps * rows::kKeys) << split) ++split;
    const int64_t ctas = P << split, rounds = (ctas + slots - 1) / slots;
    const bool full = ctas <= slots || 10 * rounds * slots <= 13 * ctas;
    const bool idle = 2 * ctas <= slots && (keys >> split) > 512;
    if (fit && full && !idle) pl->cluster = 1 << split;
  }
  // joining: about eight CTAs an SM, but 128 keys each at least
  int64_t slices = (8 * (int64_t)sms() + (P > 0 ? P : 1) - 1) / (P > 0 ? P : 1);
  const int64_t most = (c->capacity + 127) / 128;
  if (slices > most) slices = most;
  pl->slices = (int)slices;
  pl->parts_at = 256;
  pl->logits_at = pl->parts_at + parts_bytes(pl->rows.most);
  pl->bytes = pl->logits_at + round256((size_t)P * pl->rows.blocks * c->capacity * pl->pitch * sizeof(float));
  return true;
}

// Of a workspace, what one call uses: logits only where weights are asked for, and where a cluster keeps everything nothing but the
// status word.
size_t call_bytes(const CachePlan& pl, bool weights) { return pl.cluster > 0 ? 256 : (weights ? pl.bytes : pl.logits_at); }

// ---- attention behind a shared prefix ----------------------------------------------------------
struct PrefixPlan {
  RowsPlan pre, own;
  bool tiles;                        // the prefix in 128-row tiles on the tensor cores
  int seqs, tokens, token_tiles, row_tiles, chunk, chunks;
  size_t pre_at, own_at, bytes;
};

// The tile form of the prefix: CTAs (one an SM) per tile of query rows, or pair of them, so that the call ends soonest.  A
// round takes its run of key tiles, 1.75 us each for a pair and 1.15 us for a single tile, and 8 us for start, first and last
// tile and output.  SMs that it leaves free read the own rows meanwhile, up to 90 GB/s each; what is left of these then
// takes the whole device, 6 TB/s.  (64 sequences of up to 512 own rows behind 32768: 112 CTAs of
// 19 steps 58 us, 144 of 15 steps 64.)
void plan_tiles(int64_t problems, int share, int t, int group, int64_t keys, double own_bytes, PrefixPlan* pl) {
  const int most = kTileRows / group;                      // (sequence, token) pairs of a tile
  pl->tokens = t < most ? t : most;
  pl->seqs = most / pl->tokens < share ? most / pl->tokens : share;
  pl->token_tiles = (t + pl->tokens - 1) / pl->tokens;
  pl->row_tiles = (share + pl->seqs - 1) / pl->seqs * pl->token_tiles;
  const int64_t key_tiles = (keys + kTileRows - 1) / kTileRows, items = problems * ((pl->row_tiles + 1) / 2), places = sms();
  const double step = pl->row_tiles > 1 ? 1.75 : 1.15;
  double best = -1.;
  const int64_t upto = 2 * places / items + 2;             // (two rounds)
  for (int64_t c = 1; c <= key_tiles && c <= upto; ++c) {
    const int64_t each = (key_tiles + c - 1) / c, ctas = items * ((key_tiles + each - 1) / each);
    const double walk = (double)((ctas + places - 1) / places) * ((double)each * step + 8.);
    const double beside = ctas < places ? (double)(places - ctas) * 90e3 * walk : 0.;
    const double cost = walk + (own_bytes > beside ? (own_bytes - beside) / 6e6 : 0.);
    if (best < 0. || cost < best) {
      best = cost;
      pl->chunk = (int)each * kTileRows;
      pl->chunks = (int)((key_tiles + each - 1) / each);
    }
  }
}

bool plan_prefix(const curdkv_desc* dp, const curdkv_desc* d, int32_t q_rows, PrefixPlan* pl) {
  if (!heads_ok(dp) || !heads_ok(d) || q_rows < 1 || dp->n_max < 0 || d->n_max < 0 || dp->n_max > (1 << 30) || d->n_max > (1 << 30))
    return false;
  if (dp->kv_heads != d->kv_heads || (d->batch > 0 && (dp->batch < 1 || d->batch % dp->batch != 0))) return false;
  const int64_t P = (int64_t)d->batch * d->kv_heads, P0 = (int64_t)dp->batch * dp->kv_heads;
  const int group = d->q_heads / d->kv_heads;
  const int64_t rows = (int64_t)group * q_rows, share = d->batch > 0 ? d->batch / dp->batch : 1;
  if (P > (1 << 24) || rows > (1 << 24) || rows * share > (1 << 28)) return false;
  pl->pre = plan_rows(P0, rows * share, dp->n_max);
  pl->own = plan_rows(P, rows, d->n_max, pl->pre.nt);      // (both may be one launch)
  if (rows * share > 16) pl->own = plan_rows(P, rows, d->n_max);
  pl->tiles = P0 > 0 && rows * share > 16 && group <= kTileRows && dp->n_max > 0;
  size_t entries = pl->pre.most;
  if (pl->tiles) {
    plan_tiles(P0, (int)share, q_rows, group, dp->n_max, 512. * (double)P * d->n_max * ((rows + 15) / 16), pl);
    // as many parts as any own rows, and any fewer and shorter prefixes, could lead to (plan_tiles' runs of CTAs, a pair of
    // tiles or a single one each)
    const int64_t row_tiles = P0 * pl->row_tiles, key_tiles = ((int64_t)dp->n_max + kTileRows - 1) / kTileRows;
    const int64_t runs = (pl->row_tiles > 1 ? 4 : 2) * (int64_t)sms() + 2 * row_tiles, all = row_tiles * key_tiles;
    const size_t tiles = (size_t)(all < runs ? all : runs) * kTileRows;
    if (tiles > entries) entries = tiles;                  // (rows that the maps cannot hold take the other form)
  }
  pl->pre_at = 256;
  pl->own_at = pl->pre_at + parts_bytes(entries);
  // (blocks of 8 query rows turn into such of 16 and back as sequences join)
  pl->bytes = pl->own_at + parts_bytes((size_t)most_parts(P * ((rows + 15) / 16), d->n_max) * 16);
  return true;
}

}  // namespace

extern "C" {

size_t curdkv_cache_attention_workspace_bytes(const curdkv_cache* cache, const curdkv_desc* desc, int32_t q_rows) {
  CachePlan pl;
  return plan_cache(cache, desc, q_rows, &pl) ? pl.bytes : 0;
}

size_t curdkv_cache_attention_call_workspace_bytes(const curdkv_cache* cache, const curdkv_desc* desc, int32_t q_rows,
                                                   int32_t with_weights) {
  CachePlan pl;
  return plan_cache(cache, desc, q_rows, &pl) ? call_bytes(pl, with_weights != 0) : 0;
}

curdkv_status curdkv_cache_attention(const void* Q, int32_t q_rows, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_n,
                                     const int32_t* q_lens, const curdkv_cache* cache, const curdkv_desc* desc, float scale,
                                     void* O, int64_t o_stride_b, int64_t o_stride_h, int64_t o_stride_n, float* lse,
                                     float* weights, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!cache_ok(cache) || !heads_ok(desc) || q_rows < 1 || !(scale >= 0.f) || std::isinf(scale)) return CURDKV_ERR_INVALID_ARG;
  if (desc->d != 128) return CURDKV_ERR_UNSUPPORTED;
  if (!aligned16(cache->K) || !aligned16(cache->V)) return CURDKV_ERR_INVALID_ARG;
  if (!query_strides_ok(Q, q_stride_b, q_stride_h, q_stride_n) || !query_strides_ok(O, o_stride_b, o_stride_h, o_stride_n) ||
      Q == O || !rows_apart(desc->batch, desc->q_heads, q_rows, o_stride_b, o_stride_h, o_stride_n))
    return CURDKV_ERR_INVALID_ARG;
  if (workspace == nullptr || !status_ok(workspace)) return CURDKV_ERR_INVALID_ARG;
  CachePlan pl;
  if (!plan_cache(cache, desc, q_rows, &pl)) return CURDKV_ERR_UNSUPPORTED;
  if (workspace_bytes < call_bytes(pl, weights != nullptr)) return CURDKV_ERR_WORKSPACE;
  const int64_t P = (int64_t)desc->batch * desc->kv_heads;
  if (P == 0) return CURDKV_OK;
  const int64_t ctas = pl.cluster > 0 ? P * pl.cluster : P * pl.rows.blocks * pl.rows.chunks;
  if (ctas > 0x7fffffffLL || P * pl.slices > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  const int64_t row = 128, head = row * cache->capacity, seq = head * desc->kv_heads;
  rows::Args a = {};
  a.q = rows::Queries{static_cast<const __nv_bfloat16*>(Q), q_stride_b, q_stride_h, q_stride_n, desc->kv_heads,
                      desc->q_heads / desc->kv_heads, q_rows, 1, desc->q_heads / desc->kv_heads * q_rows};
  a.q_lens = q_lens;
  a.K = KvView{static_cast<const __nv_bfloat16*>(cache->K), seq, head, row};
  a.V = KvView{static_cast<const __nv_bfloat16*>(cache->V), seq, head, row};
  a.lens = cache->count;
  a.n_max = cache->capacity;
  if (q_rows > 1) {                                        // (one token sees every held row)
    a.pos = cache->pos;
    a.total = cache->total;
    a.causal = 1;
  }
  a.blocks = pl.rows.blocks;
  a.chunk = pl.rows.chunk;
  a.chunks = pl.rows.chunks;
  a.scale_log2 = scale * 1.4426950408889634f;
  const rows::Parts own = parts_of(pl.rows, ws + pl.parts_at, cache->count, cache->capacity);
  a.part_ml = const_cast<float2*>(own.ml);
  a.part_o = const_cast<float*>(own.o);
  a.status = reinterpret_cast<uint32_t*>(ws);
  a.pitch = pl.pitch;
  const rows::Outputs out = {static_cast<__nv_bfloat16*>(O), o_stride_b, o_stride_h, o_stride_n, lse, weights};
  const bool one = pl.rows.nt == 1;
  if (pl.cluster > 0) {
    a.chunks = pl.cluster;
    const bool done = weights != nullptr ? (one ? launch_parts<1, true, true>(a, out, ctas, stream) : launch_parts<2, true, true>(a, out, ctas, stream))
                                         : (one ? launch_parts<1, false, true>(a, out, ctas, stream) : launch_parts<2, false, true>(a, out, ctas, stream));
    return done ? CURDKV_OK : CURDKV_ERR_CUDA;
  }
  rows::JoinArgs j = {};
  j.own = own;
  j.heads = desc->kv_heads;
  j.group = a.q.group;
  j.t = q_rows;
  j.share = 1;
  j.q_lens = q_lens;
  j.out = out;
  if (weights == nullptr) {
    j.slices = join_slices(P, a.q.rows);
    if (!(one ? launch_parts<1, false, false>(a, out, ctas, stream) : launch_parts<2, false, false>(a, out, ctas, stream))) return CURDKV_ERR_CUDA;
    return launch_join<false, false>(j, P * j.slices, stream) ? CURDKV_OK : CURDKV_ERR_CUDA;
  }
  a.logits = reinterpret_cast<float*>(ws + pl.logits_at);
  j.slices = pl.slices;
  j.logits = a.logits;
  j.n_max = cache->capacity;
  j.pitch = pl.pitch;
  j.block_rows = 8 * pl.rows.nt;
  if (!(one ? launch_parts<1, true, false>(a, out, ctas, stream) : launch_parts<2, true, false>(a, out, ctas, stream))) return CURDKV_ERR_CUDA;
  return launch_join<false, true>(j, P * pl.slices, stream) ? CURDKV_OK : CURDKV_ERR_CUDA;
}

size_t curdkv_attention_prefix_workspace_bytes(const curdkv_desc* desc_prefix, const curdkv_desc* desc, int32_t q_rows) {
  PrefixPlan pl;
  return plan_prefix(desc_prefix, desc, q_rows, &pl) ? pl.bytes : 0;
}

curdkv_status curdkv_attention_prefix(const void* Q, int32_t q_rows, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_n,
                                      const int32_t* q_lens, const void* K_prefix, const void* V_prefix,
                                      const curdkv_desc* desc_prefix, const void* K, const void* V, const curdkv_desc* desc,
                                      float scale, void* O, int64_t o_stride_b, int64_t o_stride_h, int64_t o_stride_n, float* lse,
                                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
  curdkv_status st = check_call(K_prefix, V_prefix, desc_prefix);
  if (st != CURDKV_OK) return st;
  if ((st = check_call(K, V, desc)) != CURDKV_OK) return st;
  if (desc->d != 128 || desc_prefix->d != 128) return CURDKV_ERR_UNSUPPORTED;
  if (q_rows < 1 || !(scale >= 0.f) || std::isinf(scale)) return CURDKV_ERR_INVALID_ARG;
  if (desc_prefix->kv_heads != desc->kv_heads) return CURDKV_ERR_INVALID_ARG;
  if (desc->batch > 0 && (desc_prefix->batch < 1 || desc->batch % desc_prefix->batch != 0)) return CURDKV_ERR_INVALID_ARG;
  if (!query_strides_ok(Q, q_stride_b, q_stride_h, q_stride_n) || !query_strides_ok(O, o_stride_b, o_stride_h, o_stride_n) ||
      Q == O || !rows_apart(desc->batch, desc->q_heads, q_rows, o_stride_b, o_stride_h, o_stride_n))
    return CURDKV_ERR_INVALID_ARG;
  if (workspace == nullptr || !status_ok(workspace)) return CURDKV_ERR_INVALID_ARG;
  PrefixPlan pl;
  if (!plan_prefix(desc_prefix, desc, q_rows, &pl)) return CURDKV_ERR_UNSUPPORTED;
  if (workspace_bytes < pl.bytes) return CURDKV_ERR_WORKSPACE;
  const int64_t P = (int64_t)desc->batch * desc->kv_heads, P0 = (int64_t)desc_prefix->batch * desc->kv_heads;
  if (P == 0) return CURDKV_OK;
  const int64_t pre_ctas = P0 * pl.pre.blocks * pl.pre.chunks, own_ctas = P * pl.own.blocks * pl.own.chunks;
  if (own_ctas > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  const int group = desc->q_heads / desc->kv_heads, share = desc->batch / desc_prefix->batch;
  rows::JoinArgs j = {};
  j.prefix = parts_of(pl.pre, ws + pl.pre_at, desc_prefix->seqlens, desc_prefix->n_max);
  j.own = parts_of(pl.own, ws + pl.own_at, desc->seqlens, desc->n_max);
  rows::Args a = {};
  a.scale_log2 = scale * 1.4426950408889634f;
  a.q_lens = q_lens;
  a.status = reinterpret_cast<uint32_t*>(ws);
  auto cut = [&](const RowsPlan& r, const rows::Parts& parts) {
    a.blocks = r.blocks;
    a.chunk = r.chunk;
    a.chunks = r.chunks;
    a.part_ml = const_cast<float2*>(parts.ml);
    a.part_o = const_cast<float*>(parts.o);
  };
  rows::Args both = {};                                    // the prefix's parts, where the own rows' launch takes them along
  int64_t both_ctas = 0;
  const bool tiles = pl.tiles &&
      map_strides_ok(desc_prefix->batch, desc->kv_heads, desc_prefix->k_stride_b, desc_prefix->k_stride_h, desc_prefix->k_stride_n) &&
      map_strides_ok(desc_prefix->batch, desc->kv_heads, desc_prefix->v_stride_b, desc_prefix->v_stride_h, desc_prefix->v_stride_n) &&
      map_strides_ok(desc->batch, desc->q_heads, q_stride_b, q_stride_h, q_stride_n) &&
      map_strides_ok(1, desc->kv_heads, 0, (int64_t)group * q_stride_h, 128) && P0 * pl.row_tiles * pl.chunks <= 0x7fffffffLL;
  if (tiles) {
    j.prefix = rows::Parts{};
    const size_t entries = (size_t)P0 * pl.row_tiles * pl.chunks * kTileRows;
    j.prefix.ml = reinterpret_cast<const float2*>(ws + pl.pre_at);
    j.prefix.o = reinterpret_cast<const float*>(ws + pl.pre_at + round256(entries * sizeof(float2)));
    j.prefix.lens = desc_prefix->seqlens;
    j.prefix.n_max = desc_prefix->n_max;
    j.prefix.chunk = pl.chunk;
    j.prefix.chunks = pl.chunks;
    j.prefix.tile_rows = kTileRows;
    j.prefix.tiles = pl.row_tiles;
    j.prefix.seqs = pl.seqs;
    j.prefix.tokens = pl.tokens;
    j.prefix.token_tiles = pl.token_tiles;
    umma::PrefixArgs x = {};
    x.lens = desc_prefix->seqlens;
    x.n_max = desc_prefix->n_max;
    x.heads = desc->kv_heads;
    x.group = group;
    x.t = q_rows;
    x.share = share;
    x.seqs = pl.seqs;
    x.tokens = pl.tokens;
    x.token_tiles = pl.token_tiles;
    x.tiles = pl.row_tiles;
    x.chunk = pl.chunk;
    x.chunks = pl.chunks;
    // (products are masked before they are scaled, and -inf times 0 would be NaN)
    x.scale_log2 = a.scale_log2 > FLT_MIN ? a.scale_log2 : FLT_MIN;
    x.part_ml = const_cast<float2*>(j.prefix.ml);
    x.part_o = const_cast<float*>(j.prefix.o);
    x.status = a.status;
    CUtensorMap mq, mk, mv;
    const uint64_t sizes[5] = {128, (uint64_t)group, (uint64_t)q_rows, (uint64_t)desc->kv_heads, (uint64_t)desc->batch};
    const int64_t strides[5] = {1, q_stride_h, q_stride_n, (int64_t)group * q_stride_h, q_stride_b};
    const uint32_t box[5] = {64, (uint32_t)group, (uint32_t)pl.tokens, 1, (uint32_t)pl.seqs};
    if (!bf16_map(&mq, Q, 5, sizes, strides, box) ||
        !rows_map(&mk, K_prefix, desc_prefix->batch, desc->kv_heads, desc_prefix->n_max, desc_prefix->k_stride_b,
                  desc_prefix->k_stride_h, desc_prefix->k_stride_n) ||
        !rows_map(&mv, V_prefix, desc_prefix->batch, desc->kv_heads, desc_prefix->n_max, desc_prefix->v_stride_b,
                  desc_prefix->v_stride_h, desc_prefix->v_stride_n))
      return CURDKV_ERR_CUDA;
    static std::atomic<uint64_t> pair_done{0}, one_done{0};
    const unsigned grid = (unsigned)(P0 * ((pl.row_tiles + 1) / 2) * pl.chunks);
    if (pl.row_tiles > 1) {
      if (!allow_smem(umma::prefix_attention_kernel<true>, umma::kPrefixDynamic, pair_done)) return CURDKV_ERR_CUDA;
      umma::prefix_attention_kernel<true><<<grid, umma::kPrefixThreads, umma::kPrefixDynamic, stream>>>(mq, mk, mv, x);
    } else {
      if (!allow_smem(umma::prefix_attention_kernel<false>, umma::kPrefixDynamic, one_done)) return CURDKV_ERR_CUDA;
      umma::prefix_attention_kernel<false><<<grid, umma::kPrefixThreads, umma::kPrefixDynamic, stream>>>(mq, mk, mv, x);
    }
    if (!launched()) return CURDKV_ERR_CUDA;
  } else if (desc_prefix->n_max > 0) {
    if (pre_ctas > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
    a.q = rows::Queries{static_cast<const __nv_bfloat16*>(Q), q_stride_b, q_stride_h, q_stride_n, desc->kv_heads, group, q_rows,
                        share, share * q_rows * group};
    a.K = KvView{static_cast<const __nv_bfloat16*>(K_prefix), desc_prefix->k_stride_b, desc_prefix->k_stride_h, desc_prefix->k_stride_n};
    a.V = KvView{static_cast<const __nv_bfloat16*>(V_prefix), desc_prefix->v_stride_b, desc_prefix->v_stride_h, desc_prefix->v_stride_n};
    a.lens = desc_prefix->seqlens;
    a.n_max = desc_prefix->n_max;
    cut(pl.pre, j.prefix);
    both = a;
    both_ctas = pre_ctas;
  }
  if (desc->n_max > 0) {
    a.q = rows::Queries{static_cast<const __nv_bfloat16*>(Q), q_stride_b, q_stride_h, q_stride_n, desc->kv_heads, group, q_rows,
                        1, q_rows * group};
    a.K = KvView{static_cast<const __nv_bfloat16*>(K), desc->k_stride_b, desc->k_stride_h, desc->k_stride_n};
    a.V = KvView{static_cast<const __nv_bfloat16*>(V), desc->v_stride_b, desc->v_stride_h, desc->v_stride_n};
    a.lens = desc->seqlens;
    a.n_max = desc->n_max;
    a.causal = 1;
    a.late = tiles ? 1 : 0;                                // (that kernel is launched behind everything before it)
    cut(pl.own, j.own);
  }
  const int64_t ctas = desc->n_max > 0 ? own_ctas : 0;
  if (both_ctas > 0 && (pl.pre.nt != pl.own.nt || ctas + both_ctas > 0x7fffffffLL)) {
    if (!(pl.pre.nt == 1 ? launch_parts<1, false, false>(both, rows::Outputs{}, both_ctas, stream)
                         : launch_parts<2, false, false>(both, rows::Outputs{}, both_ctas, stream)))
      return CURDKV_ERR_CUDA;
    both_ctas = 0;
  }
  if (ctas + both_ctas > 0) {
    if (!(pl.own.nt == 1 ? launch_parts<1, false, false>(a, rows::Outputs{}, ctas, stream, &both, both_ctas)
                         : launch_parts<2, false, false>(a, rows::Outputs{}, ctas, stream, &both, both_ctas)))
      return CURDKV_ERR_CUDA;
  }
  j.heads = desc->kv_heads;
  j.group = group;
  j.t = q_rows;
  j.share = share;
  j.q_lens = q_lens;
  j.out = rows::Outputs{static_cast<__nv_bfloat16*>(O), o_stride_b, o_stride_h, o_stride_n, lse, nullptr};
  j.by_warp = (desc_prefix->n_max > 0 ? j.prefix.chunks : 0) + pl.own.chunks <= 8;
  j.slices = join_slices(P, j.by_warp ? ((int64_t)group * q_rows + rows::kJoinWarps - 1) / rows::kJoinWarps : (int64_t)group * q_rows);
  return launch_join<true, false>(j, P * j.slices, stream) ? CURDKV_OK : CURDKV_ERR_CUDA;
}

}  // extern "C"
