// Serving calls: the 4-bit cache (store, append, read, attention) and the attention with a sliding
// window and sinks.  Argument checks and kernel launches.
#include <atomic>
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "attn_token.cuh"
#include "attn_window.cuh"
#include "common.cuh"
#include "host.cuh"
#include "qcache.cuh"

namespace {

using namespace curdkv;
using namespace curdkv::host;

curdkv_status check_cache(const curdkv_qcache* c) {
  if (c == nullptr || c->K_codes == nullptr || c->V_codes == nullptr || c->K_meta == nullptr ||
      c->V_meta == nullptr || c->count == nullptr)
    return CURDKV_ERR_INVALID_ARG;
  if (c->batch < 0 || c->kv_heads < 1 || c->capacity < 1) return CURDKV_ERR_INVALID_ARG;
  if (!aligned16(c->K_codes) || !aligned16(c->V_codes) || !aligned16(c->K_meta) || !aligned16(c->V_meta))
    return CURDKV_ERR_INVALID_ARG;
  if ((int64_t)c->batch * c->kv_heads > (int64_t)1 << 24 || c->capacity > 0x7fffffffLL)
    return CURDKV_ERR_UNSUPPORTED;
  return CURDKV_OK;
}

qcache::View view_of(const curdkv_qcache* c) {
  return qcache::View{static_cast<uint8_t*>(c->K_codes), static_cast<uint8_t*>(c->V_codes),
                      static_cast<uint32_t*>(c->K_meta), static_cast<uint32_t*>(c->V_meta),
                      c->count, c->row_start, c->capacity};
}

// CTAs per head so that `problems` heads of up to `rows` rows fill the device a few times over.
int ctas_for(int64_t problems, int64_t rows, int rows_per_cta) {
  int64_t want = (16LL * sms() + problems - 1) / (problems > 0 ? problems : 1);
  const int64_t most = (rows + rows_per_cta - 1) / rows_per_cta;
  if (want > most) want = most;
  return (int)(want < 1 ? 1 : want);
}

curdkv_status check_rows(const curdkv_qcache* cache, const void* K, const void* V, const curdkv_desc* desc,
                         const void* workspace) {
  curdkv_status st = check_cache(cache);
  if (st != CURDKV_OK) return st;
  if ((st = check_call(K, V, desc)) != CURDKV_OK) return st;
  if (desc->d != 128) return CURDKV_ERR_UNSUPPORTED;
  if (desc->batch != cache->batch || desc->kv_heads != cache->kv_heads) return CURDKV_ERR_INVALID_ARG;
  if (!status_ok(workspace)) return CURDKV_ERR_INVALID_ARG;
  return CURDKV_OK;
}

// ---- attention of few query rows ---------------------------------------------------------------
struct Plan {
  int nt, blocks;                    // sets of 8 query rows a CTA takes, blocks of rows per head
  int ctas, split;                   // runs of the line; 0: a cluster of 2^split CTAs per item
  size_t begins_at, ml_at, o_at, bytes;                    // inside the workspace, and its size
};

// `keys`: what the longest head may hold or see in this call, `total`: all heads together.  An item has a cluster to itself -- the most CTAs, up to
// eight, that find room on the device at once with two rounds of tiles each -- unless one line of all tiles, cut
// into equal runs, needs so many rounds less that joining its parts pays.  Runs: as many as CTAs fit the
// device, but none shorter than two rounds unless there are more items.  In us, clusters | line, 4 query rows,
// heads full, calls in a graph over rows that are not in L2; the rule takes the faster one of each pair:
//    8 heads of 4 bits:    1702 rows 7.4 | 12.7     3340 rows 9.0 | 14.0     8192 rows 12.1 | 18.0
//   32 heads:              1702 rows 9.4 | 14.5     8192 rows 16.7 | 22.6    16384 rows 25.9 | 30.1
//  128 heads:              1702 rows 14.9 | 20.8    3340 rows 22.3 | 27.0    one head of 8192 rows 11.6 | 11.6
//  128 heads, bf16:        window 1024 15.8 | 20.7  window 4096 46.1 | 52.9
//  456 heads:              1702 rows 38.2 | 40.5    8192 rows 140 | 118      bf16, window 2048 78.7 | 84.9
// 1024 heads:              1702 rows 61.4 | 76.7    8192 rows 228 | 245      bf16, window 2048 160 | 179
//   16 query rows:         128 heads of 1702 rows 20.1 | 28.2    8 of 16384 24.2 | 23.6    64 of 131072 367 | 329
// What the host knows is the capacity, not what is held: a cache much larger than that may take the line where
// clusters are faster (8 heads of 1702 rows in a cache of 17020 7.2 | 15.2, of 131072 8.9 | 16.4; 128 heads of
// 1702 in one of 17020 15.0 | 20.3).
// (Four times as many runs, to even out SMs of different speed, was slower: 282 against 276 us for 64 heads of
// 131072 rows, 66 against 51 for 128 heads of 2048 to 16384.)  The workspace depends on neither.
Plan plan_token(int64_t problems, int64_t rows, int64_t keys, int64_t total, int tile_keys, int ctas_per_sm) {
  Plan pl;
  pl.nt = rows <= 8 ? 1 : 2;
  pl.blocks = (int)((rows + 8 * pl.nt - 1) / (8 * pl.nt));
  const int64_t items = problems * pl.blocks, slots = (int64_t)ctas_per_sm * sms();
  const int64_t tiles = (keys + tile_keys - 1) / tile_keys, all = (total / tile_keys + problems) * pl.blocks;
  pl.ctas = 0;
  pl.split = 0;
  while (pl.split < token::kMostSplit && (items << (pl.split + 1)) <= slots && tiles > (2 * token::kWarps) << pl.split)
    ++pl.split;
  const int64_t cluster = (int64_t)token::kWarps << pl.split;
  // Rounds of tiles when every item has its cluster: those of one item where all run at once; else as many
  // as the SMs need for all, the last, partly filled wave counted as a quarter at least (few CTAs on an SM are faster).
  const int64_t per = (tiles + cluster - 1) / cluster, n = items << pl.split, rest = n % slots;
  const int64_t last = rest == 0 ? 0 : (rest > slots / 4 ? rest : slots / 4);
  const int64_t alone = n <= slots ? per : (n - rest + last) * per / slots;
  const int64_t even = (all + token::kWarps * slots - 1) / (token::kWarps * slots);             // of equal runs
  // the line's own cost: the join, and the scan of its items
  const int64_t line = n <= slots ? 7 : 3 + items / 256;
  if (alone > even + line && items <= token::kMostItems) {
    pl.split = 0;
    int64_t ctas = all / (2 * token::kWarps);
    if (ctas < items) ctas = items;
    if (ctas > slots) ctas = slots;
    pl.ctas = (int)ctas;
  }
  const bool room = items <= token::kMostItems;
  const size_t parts = room ? 2 * (size_t)slots * 8 * pl.nt : 0;
  pl.begins_at = 256;
  pl.ml_at = pl.begins_at + round256(room ? (size_t)(items + 1) * sizeof(int64_t) : 0);
  pl.o_at = pl.ml_at + round256(parts * 4 * sizeof(float));
  pl.bytes = pl.o_at + round256(parts * 128 * sizeof(float));
  return pl;
}

Plan plan_qcache(const curdkv_qcache* c, int32_t q_rows) {
  // Packed heads share `capacity` rows unevenly: the longest is taken to hold four times its share.  (8 heads of
  // 1702 rows take 8.0 us so and 13.1 with equal runs, one of 12916 and seven of 100 15.8 and 17.3.)
  const int64_t P = (int64_t)c->batch * c->kv_heads, share = P > 0 ? 4 * ((c->capacity + P - 1) / P) : 0;
  const bool packed = c->row_start != nullptr;
  const int64_t longest = packed && share < c->capacity ? share : c->capacity;
  return plan_token(P, q_rows, longest, packed ? c->capacity : P * c->capacity, token::Tile<true>::kKeys,
                    q_rows <= 8 ? token::ctas_per_sm<true, 1>() : token::ctas_per_sm<true, 2>());
}

Plan plan_window(const curdkv_desc* d, int32_t q_rows, int64_t seen) {
  const int64_t P = (int64_t)d->batch * d->kv_heads;
  return plan_token(P, (int64_t)(d->q_heads / d->kv_heads) * q_rows, seen, P * seen, token::Tile<false>::kKeys,
                    token::ctas_per_sm<false, 1>());
}

template <bool Q4, int NT>
bool launch_attend(const token::Args& a, cudaStream_t stream) {
  constexpr int smem = token::smem_bytes<Q4, NT>();
  static std::atomic<uint64_t> done{0};
  if (!allow_smem(token::attend_kernel<Q4, NT>, smem, done)) return false;
  if (a.split > 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.items << a.split);
    cfg.blockDim = dim3(token::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 1u << a.split;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, token::attend_kernel<Q4, NT>, a) != cudaSuccess) return false;
    return launched();
  }
  const int grid = a.ctas > 0 ? a.ctas : a.items;
  token::attend_kernel<Q4, NT><<<(unsigned)grid, token::kThreads, smem, stream>>>(a);
  if (!launched()) return false;
  if (a.ctas == 0) return true;
  // launched behind attend_kernel without waiting for its end: the kernel itself waits
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.items * 8 * NT));
  cfg.blockDim = dim3(32);
  cfg.stream = stream;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, token::join_kernel, a, 8 * NT) != cudaSuccess) return false;
  return launched();
}

// Which form of the window attention a call takes: the one whose slowest SM is estimated to end first.
// Measured: the token form needs 9.8 ns per key for 16 query rows of a KV head on one SM, plus the time of 64
// keys, and spreads its work evenly; the prompt form 18 ns per key for a pair of 128-row tiles (14.7 for a
// single one), full or not, plus the time of some 320 keys (tiles partly outside the window, the start of an
// item), and takes whole rounds of a pair per SM.  In us, token | prompt, rows = query rows per KV head (group x
// tokens), at the sizes around the change from one to the other.  The token form's time goes by the rows alone, the
// prompt form's by group * ceil(tokens / 128) tiles: it stands for groups of 1 / 4 / 8.  The rule takes the faster
// one of each pair.
//   16 x 8 heads, 8192 keys, window 8192    32 rows  175 | 124 / 293 / 579      64 rows  272 | 126 / 293 / 576
//                                          128 rows  535 | 127 / 295 / 577
//   16 x 8 heads, 8192 keys, window 1024    32 rows   25 | 28 / 57 / 104        64 rows   46 | 28 / 57 / 105
//                                          128 rows   88 | 28 / 57 / 105
//   16 x 8 heads, 512 keys, window 256      64 rows   21 | 16 / 30 / 51        128 rows   39 | 17 / 30 / 52
//    4 x 8 heads, 8192 keys, window 8192    64 rows   76 | 121 / 148 / 148     128 rows  134 | 121 / 147 / 150
//                                          256 rows  270 | 148 / 149 / 152
//    1 x 8 heads, 8192 keys, window 8192   256 rows   72 | 143 / 143 / 145     (the pairs fill few SMs)
//   64 x 8 heads, 512 keys, window 256     128 rows  132 | 49 / 87 / 164       256 rows  258 | 60 / 88 / 164
bool prompt_form(int64_t problems, int64_t rows, int64_t tiles, int64_t window_keys, int64_t n_max) {
  const int64_t keys = window_keys < n_max ? window_keys : n_max, places = sms(), pairs = (tiles + 1) / 2;
  const double token = 9.8 * (double)(problems * ((rows + 15) / 16)) / (double)places * (double)(keys + 64);
  const double prompt =
      (tiles > 1 ? 18.0 : 14.7) * (double)((problems * pairs + places - 1) / places) * (double)(keys + 320);
  return prompt < token;
}

}  // namespace

extern "C" {

curdkv_status curdkv_qcache_store(const curdkv_qcache* cache, const void* K, const void* V,
                                  const curdkv_desc* desc, const int32_t* idx, int64_t idx_stride,
                                  const int32_t* head_counts, const int32_t* head_offsets,
                                  void* workspace, void* cuda_stream) {
  curdkv_status st = check_rows(cache, K, V, desc, workspace);
  if (st != CURDKV_OK) return st;
  if (idx != nullptr && (head_counts == nullptr || idx_stride < 0)) return CURDKV_ERR_INVALID_ARG;
  if (idx == nullptr && (head_counts != nullptr || head_offsets != nullptr)) return CURDKV_ERR_INVALID_ARG;
  const int64_t P = (int64_t)desc->batch * desc->kv_heads;
  if (P == 0) return CURDKV_OK;
  qcache::StoreArgs a;
  a.cache = view_of(cache);
  a.K = KvView{static_cast<const __nv_bfloat16*>(K), desc->k_stride_b, desc->k_stride_h, desc->k_stride_n};
  a.V = KvView{static_cast<const __nv_bfloat16*>(V), desc->v_stride_b, desc->v_stride_h, desc->v_stride_n};
  a.seqlens = desc->seqlens;
  a.idx = idx;
  a.head_counts = head_counts;
  a.head_offsets = head_offsets;
  a.idx_stride = idx_stride;
  a.heads = desc->kv_heads;
  a.n_max = desc->n_max;
  a.status = static_cast<uint32_t*>(workspace);
  int64_t rows = idx != nullptr && head_offsets == nullptr ? idx_stride : desc->n_max;
  if (cache->row_start == nullptr && rows > cache->capacity) rows = cache->capacity;
  a.ctas_per_head = ctas_for(P, rows, qcache::kStoreRowsPerCta);
  if (P * a.ctas_per_head > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
  qcache::store_kernel<<<(unsigned)(P * a.ctas_per_head), qcache::kStoreWarps * 32, 0,
                         static_cast<cudaStream_t>(cuda_stream)>>>(a);
  return launched() ? CURDKV_OK : CURDKV_ERR_CUDA;
}

curdkv_status curdkv_qcache_append(const curdkv_qcache* cache, const void* K_new, const void* V_new,
                                   const curdkv_desc* desc, void* workspace, void* cuda_stream) {
  curdkv_status st = check_rows(cache, K_new, V_new, desc, workspace);
  if (st != CURDKV_OK) return st;
  const int64_t P = (int64_t)desc->batch * desc->kv_heads;
  if (P == 0 || desc->n_max == 0) return CURDKV_OK;
  qcache::AppendArgs a;
  a.cache = view_of(cache);
  a.K = KvView{static_cast<const __nv_bfloat16*>(K_new), desc->k_stride_b, desc->k_stride_h, desc->k_stride_n};
  a.V = KvView{static_cast<const __nv_bfloat16*>(V_new), desc->v_stride_b, desc->v_stride_h, desc->v_stride_n};
  a.t_new = desc->seqlens;
  a.heads = desc->kv_heads;
  a.t = desc->n_max;
  a.chunks = (int)(((int64_t)desc->n_max + qcache::kAppendRows - 1) / qcache::kAppendRows);
  a.status = static_cast<uint32_t*>(workspace);
  if (P * a.chunks > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  qcache::append_kernel<<<(unsigned)(P * a.chunks), qcache::kStoreWarps * 32, 0, stream>>>(a);
  if (!launched()) return CURDKV_ERR_CUDA;
  if (a.chunks > 1) {
    qcache::advance_kernel<<<(unsigned)((P + 255) / 256), 256, 0, stream>>>(a, (int)P);
    if (!launched()) return CURDKV_ERR_CUDA;
  }
  return CURDKV_OK;
}

curdkv_status curdkv_qcache_read(const curdkv_qcache* cache, const int32_t* idx, int64_t rows, void* K_out,
                                 void* V_out, void* workspace, void* cuda_stream) {
  curdkv_status st = check_cache(cache);
  if (st != CURDKV_OK) return st;
  if (K_out == nullptr || V_out == nullptr || !aligned16(K_out) || !aligned16(V_out)) return CURDKV_ERR_INVALID_ARG;
  if (rows < 0 || (idx != nullptr && rows < 1) || rows > 0x7fffffffLL || !status_ok(workspace))
    return CURDKV_ERR_INVALID_ARG;
  const int64_t P = (int64_t)cache->batch * cache->kv_heads;
  const int64_t out_rows = rows > 0 ? rows : cache->capacity;                // of a head, or of all of a packed cache
  if (overlap(K_out, V_out, (__int128)(rows > 0 || cache->row_start == nullptr ? P : 1) * out_rows * 256))
    return CURDKV_ERR_INVALID_ARG;
  if (P == 0) return CURDKV_OK;
  qcache::ReadArgs a;
  a.cache = view_of(cache);
  a.idx = idx;
  a.K_out = static_cast<__nv_bfloat16*>(K_out);
  a.V_out = static_cast<__nv_bfloat16*>(V_out);
  a.heads = cache->kv_heads;
  a.rows = rows;
  a.status = static_cast<uint32_t*>(workspace);
  a.ctas_per_head = ctas_for(P, rows > 0 ? rows : cache->capacity, qcache::kStoreRowsPerCta);
  if (P * a.ctas_per_head > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
  qcache::read_kernel<<<(unsigned)(P * a.ctas_per_head), qcache::kStoreWarps * 32, 0,
                        static_cast<cudaStream_t>(cuda_stream)>>>(a);
  return launched() ? CURDKV_OK : CURDKV_ERR_CUDA;
}

size_t curdkv_qcache_attention_workspace_bytes(const curdkv_qcache* cache, int32_t q_rows) {
  if (cache == nullptr || cache->batch < 0 || cache->kv_heads < 1 || cache->capacity < 1 || q_rows < 1) return 0;
  return plan_qcache(cache, q_rows).bytes;
}

curdkv_status curdkv_qcache_attention(const void* Q, int32_t q_rows, int64_t q_stride_b, int64_t q_stride_h,
                                      int64_t q_stride_n, const curdkv_qcache* cache, float scale, void* O,
                                      int64_t o_stride_b, int64_t o_stride_h, int64_t o_stride_n, float* lse,
                                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
  curdkv_status st = check_cache(cache);
  if (st != CURDKV_OK) return st;
  if (q_rows < 1 || !(scale >= 0.f) || std::isinf(scale)) return CURDKV_ERR_INVALID_ARG;
  if (!query_strides_ok(Q, q_stride_b, q_stride_h, q_stride_n) ||
      !query_strides_ok(O, o_stride_b, o_stride_h, o_stride_n) || Q == O ||
      !rows_apart(cache->batch, cache->kv_heads, q_rows, o_stride_b, o_stride_h, o_stride_n))
    return CURDKV_ERR_INVALID_ARG;
  if (workspace == nullptr || !status_ok(workspace)) return CURDKV_ERR_INVALID_ARG;
  const Plan pl = plan_qcache(cache, q_rows);
  if (workspace_bytes < pl.bytes) return CURDKV_ERR_WORKSPACE;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int64_t P = (int64_t)cache->batch * cache->kv_heads;
  if (P == 0) return CURDKV_OK;
  if (P * pl.blocks > 0x7fffffffLL || P * q_rows > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
  token::Args a = {};
  a.Q = static_cast<const __nv_bfloat16*>(Q);
  a.q_sb = q_stride_b; a.q_sh = q_stride_h; a.q_sn = q_stride_n;
  a.O = static_cast<__nv_bfloat16*>(O);
  a.o_sb = o_stride_b; a.o_sh = o_stride_h; a.o_sn = o_stride_n;
  a.lse = lse;
  a.heads = cache->kv_heads;
  a.group = 1;
  a.q_n = a.rows = q_rows;
  a.blocks = pl.blocks;
  a.items = (int)(P * pl.blocks);
  a.ctas = pl.ctas;
  a.split = pl.split;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.cache = view_of(cache);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  a.begins = reinterpret_cast<int64_t*>(ws + pl.begins_at);
  a.part_ml = reinterpret_cast<float*>(ws + pl.ml_at);
  a.part_o = reinterpret_cast<float*>(ws + pl.o_at);
  a.status = reinterpret_cast<uint32_t*>(ws);
  return (pl.nt == 1 ? launch_attend<true, 1>(a, stream) : launch_attend<true, 2>(a, stream)) ? CURDKV_OK
                                                                                                  : CURDKV_ERR_CUDA;
}

size_t curdkv_attention_window_workspace_bytes(const curdkv_desc* desc, int32_t q_rows) {
  if (desc == nullptr || desc->batch < 0 || desc->kv_heads < 1 || desc->q_heads < desc->kv_heads ||
      desc->q_heads % desc->kv_heads != 0 || desc->n_max < 0 || q_rows < 1)
    return 0;
  return plan_window(desc, q_rows, desc->n_max).bytes;
}

curdkv_status curdkv_attention_window(const void* Q, int32_t q_rows, int64_t q_stride_b, int64_t q_stride_h,
                                      int64_t q_stride_n, const int32_t* q_lens, const void* K, const void* V,
                                      const curdkv_desc* desc, int32_t num_sink, int32_t window, float scale,
                                      void* O, int64_t o_stride_b, int64_t o_stride_h, int64_t o_stride_n,
                                      float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  curdkv_status st = check_call(K, V, desc);
  if (st != CURDKV_OK) return st;
  if (desc->d != 128) return CURDKV_ERR_UNSUPPORTED;
  if (q_rows < 1 || num_sink < 0 || window < 0 || !(scale >= 0.f) || std::isinf(scale)) return CURDKV_ERR_INVALID_ARG;
  if (!query_strides_ok(Q, q_stride_b, q_stride_h, q_stride_n) ||
      !query_strides_ok(O, o_stride_b, o_stride_h, o_stride_n) || Q == O ||
      !rows_apart(desc->batch, desc->q_heads, q_rows, o_stride_b, o_stride_h, o_stride_n))
    return CURDKV_ERR_INVALID_ARG;
  if (workspace == nullptr || !status_ok(workspace)) return CURDKV_ERR_INVALID_ARG;
  // the most rows a block of queries sees: its window, the tokens between, the sinks
  int64_t seen = (int64_t)window + num_sink + q_rows;
  if (seen > desc->n_max) seen = desc->n_max;
  Plan pl = plan_window(desc, q_rows, seen);
  if (workspace_bytes < pl.bytes) return CURDKV_ERR_WORKSPACE;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int64_t P = (int64_t)desc->batch * desc->kv_heads;
  if (P == 0) return CURDKV_OK;
  const int group = desc->q_heads / desc->kv_heads;
  const float scale_log2 = scale * 1.4426950408889634f;
  const int64_t tiles = ((int64_t)q_rows + kTileRows - 1) / kTileRows * group, pairs = (tiles + 1) / 2;
  if (desc->n_max > 0 && (int64_t)desc->n_max + q_rows < (1 << 30) && P * pairs <= 0x3fffffffLL &&
      prompt_form(P, (int64_t)group * q_rows, tiles, (int64_t)window + num_sink, desc->n_max) &&
      map_strides_ok(desc->batch, desc->kv_heads, desc->k_stride_b, desc->k_stride_h, desc->k_stride_n) &&
      map_strides_ok(desc->batch, desc->kv_heads, desc->v_stride_b, desc->v_stride_h, desc->v_stride_n) &&
      map_strides_ok(desc->batch, desc->q_heads, q_stride_b, q_stride_h, q_stride_n)) {
    CUtensorMap mq, mk, mv;
    if (!rows_map(&mq, Q, desc->batch, desc->q_heads, q_rows, q_stride_b, q_stride_h, q_stride_n) ||
        !rows_map(&mk, K, desc->batch, desc->kv_heads, desc->n_max, desc->k_stride_b, desc->k_stride_h, desc->k_stride_n) ||
        !rows_map(&mv, V, desc->batch, desc->kv_heads, desc->n_max, desc->v_stride_b, desc->v_stride_h, desc->v_stride_n))
      return CURDKV_ERR_CUDA;
    umma::WindowArgs wa = {};
    wa.seqlens = desc->seqlens;
    wa.q_lens = q_lens;
    wa.batch = desc->batch;
    wa.heads = desc->kv_heads;
    wa.group = group;
    wa.q_rows = q_rows;
    wa.n_max = desc->n_max;
    wa.num_sink = num_sink < desc->n_max ? num_sink : desc->n_max;
    wa.window = window < desc->n_max ? window : desc->n_max;
    // (this form masks products before it scales them, and -inf times 0 would be NaN)
    wa.scale_log2 = scale_log2 > FLT_MIN ? scale_log2 : FLT_MIN;
    wa.O = static_cast<__nv_bfloat16*>(O);
    wa.o_sb = o_stride_b; wa.o_sh = o_stride_h; wa.o_sn = o_stride_n;
    wa.lse = lse;
    wa.status = static_cast<uint32_t*>(workspace);
    wa.wait_ns = umma::kWaitLimitNs;
    wa.pairs = (int)pairs;
    wa.items = (int)(P * pairs);
    static std::atomic<uint64_t> done{0};
    if (!allow_smem(umma::window_umma_kernel, umma::kWinDynamic, done)) return CURDKV_ERR_CUDA;
    const int grid = wa.items < sms() ? wa.items : sms();
    umma::window_umma_kernel<<<(unsigned)grid, umma::kWinThreads, umma::kWinDynamic, stream>>>(mq, mk, mv, wa);
    return launched() ? CURDKV_OK : CURDKV_ERR_CUDA;
  }
  token::Args a = {};
  a.Q = static_cast<const __nv_bfloat16*>(Q);
  a.q_sb = q_stride_b; a.q_sh = q_stride_h; a.q_sn = q_stride_n;
  a.O = static_cast<__nv_bfloat16*>(O);
  a.o_sb = o_stride_b; a.o_sh = o_stride_h; a.o_sn = o_stride_n;
  a.lse = lse;
  a.heads = desc->kv_heads;
  a.group = group;
  a.q_n = q_rows;
  if ((int64_t)a.group * q_rows > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
  a.rows = a.group * q_rows;
  a.blocks = pl.blocks;
  a.items = (int)(P * pl.blocks);
  a.ctas = pl.ctas;
  a.split = pl.split;
  if (P * pl.blocks > 0x7fffffffLL || P * a.rows > 0x7fffffffLL) return CURDKV_ERR_UNSUPPORTED;
  a.scale_log2 = scale_log2;
  a.K = KvView{static_cast<const __nv_bfloat16*>(K), desc->k_stride_b, desc->k_stride_h, desc->k_stride_n};
  a.V = KvView{static_cast<const __nv_bfloat16*>(V), desc->v_stride_b, desc->v_stride_h, desc->v_stride_n};
  a.seqlens = desc->seqlens;
  a.q_lens = q_lens;
  a.n_max = desc->n_max;
  a.num_sink = num_sink;
  a.window = window;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  a.begins = reinterpret_cast<int64_t*>(ws + pl.begins_at);
  a.part_ml = reinterpret_cast<float*>(ws + pl.ml_at);
  a.part_o = reinterpret_cast<float*>(ws + pl.o_at);
  a.status = reinterpret_cast<uint32_t*>(ws);
  return (pl.nt == 1 ? launch_attend<false, 1>(a, stream) : launch_attend<false, 2>(a, stream)) ? CURDKV_OK
                                                                                                    : CURDKV_ERR_CUDA;
}

}  // extern "C"
