// Scores of a prompt's rows by the attention weights they receive: argument checks and launches.
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "attn_scores.cuh"
#include "host.cuh"

namespace {

using namespace curdkv;
using namespace curdkv::host;

struct ScoresPlan {
  int tokens, row_tiles, key_tiles;
  int row_seg, row_segs, key_seg, key_segs;                // of the rows pass and the columns pass
  size_t stats_at, logsum_at, parts_at, bytes;
};

// B tiles a unit takes: twelve units a CTA, so that they end together, but twelve tiles each (a unit costs about one beside
// them) while that leaves every SM one.
int unit_length(int64_t steps) {
  const int64_t n = sms();
  int64_t seg = (steps + 12 * n - 1) / (12 * n), each = (steps + n - 1) / n;
  const int64_t least = each < 12 ? each : 12;
  if (seg < least) seg = least;
  return (int)(seg < 1 ? 1 : (seg < (1 << 30) ? seg : 1 << 30));             // (no tensor has that many tiles)
}

bool plan_scores(const curdkv_desc* d, int32_t q_rows, ScoresPlan* pl) {
  if (d == nullptr || d->batch < 0 || d->kv_heads < 1 || d->q_heads < d->kv_heads || d->q_heads % d->kv_heads != 0 || d->n_max < 0 ||
      q_rows < 1)
    return false;
  const int group = d->q_heads / d->kv_heads;
  const int64_t P = (int64_t)d->batch * d->kv_heads;
  if (group > kTileRows || (int64_t)d->n_max + q_rows > (1 << 30) || P > (1 << 24)) return false;
  pl->tokens = kTileRows / group;
  pl->row_tiles = (q_rows + pl->tokens - 1) / pl->tokens;
  pl->key_tiles = d->n_max > 0 ? (d->n_max + kTileRows - 1) / kTileRows : 1;
  if (P * pl->row_tiles > 0x7fffffff) return false;        // (so that the counts below stay within 64 bits)
  // B tiles of all pairs, from what the first and the last pair see
  const int64_t row_pairs = (pl->row_tiles + 1) / 2, key_pairs = (pl->key_tiles + 1) / 2;
  const int64_t before = d->n_max > q_rows ? d->n_max - q_rows : 0;          // keys that every token sees
  pl->row_seg = unit_length(P * row_pairs * (before / kTileRows + pl->key_tiles + 1) / 2);
  pl->row_segs = (pl->key_tiles + pl->row_seg - 1) / pl->row_seg;
  const int64_t whole = before / (2 * kTileRows);                             // pairs of key tiles that every token sees
  pl->key_seg = unit_length(P * (whole * pl->row_tiles + (key_pairs - whole) * (pl->row_tiles + 1) / 2));
  pl->key_segs = (pl->row_tiles + pl->key_seg - 1) / pl->key_seg;
  // Room for the most that any call of no larger sizes leaves: shorter ones may be cut into more units (the last 32 of 2305 rows
  // into 19, of 2369 into 10).  With U = 12 n units aimed at on n SMs and S steps in all, a unit has at least S / U of them (S / n
  // below twelve), and the tiles of all pairs, row_tiles x key_tiles each, are at most 4 S: the rows pass leaves 4 U parts and one
  // for each row tile at most, 2 U and one of a single row tile.
  const int64_t n = sms(), row_all = P * pl->row_tiles, units = (pl->row_tiles > 1 ? 48 : 24) * n + row_all;
  const int64_t row_parts = row_all * pl->key_tiles < units ? row_all * pl->key_tiles : units;
  pl->stats_at = 512;                                      // (status word, and at 256 the two passes' counters)
  pl->logsum_at = pl->stats_at + round256((size_t)row_parts * kTileRows * 2 * sizeof(float2));
  pl->parts_at = pl->logsum_at + round256((size_t)row_all * kTileRows * sizeof(float));
  // The columns pass has pairs x row_tiles <= 2 S: at most 2 U parts and one a pair.  Twelve row tiles or fewer are one unit, and
  // so no part, but where S / n is below twelve: 4 n at most.
  int64_t key_parts = 0;
  if (pl->row_tiles > 1) {
    key_parts = P * key_pairs * pl->row_tiles;
    const int64_t most = pl->row_tiles <= 12 ? 4 * n : 24 * n + P * key_pairs;
    if (key_parts > most) key_parts = most;
  }
  pl->bytes = pl->parts_at + (size_t)key_parts * 2 * 2 * kTileRows * sizeof(float);
  return P * row_pairs * pl->row_segs <= 0x7fffffff && P * key_pairs * pl->key_segs <= 0x7fffffff && P * ((d->n_max + 255) / 256) <= 0x7fffffff;
}

// Launched behind the kernel before it without waiting for its end (`chained`): the kernel itself waits.
template <typename Kernel, typename... Args>
bool launch(Kernel kernel, int64_t grid, int block, int smem, bool chained, cudaStream_t stream, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = chained ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) return false;
  return launched();
}

}  // namespace

extern "C" {

size_t curdkv_attention_scores_workspace_bytes(const curdkv_desc* desc, int32_t q_rows) {
  ScoresPlan pl;
  return plan_scores(desc, q_rows, &pl) ? pl.bytes : 0;
}

curdkv_status curdkv_attention_scores(const void* Q, int32_t q_rows, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_n,
                                      const int32_t* q_lens, const void* K, const curdkv_desc* desc, float scale, float* lse,
                                      int32_t lse_given, float* scores, void* workspace, size_t workspace_bytes,
                                      void* cuda_stream) {
  if (desc == nullptr) return CURDKV_ERR_INVALID_ARG;
  curdkv_desc d = *desc;                                   // (V is not read)
  d.v_stride_b = d.k_stride_b; d.v_stride_h = d.k_stride_h; d.v_stride_n = d.k_stride_n;
  curdkv_status st = check_call(K, K, &d);
  if (st != CURDKV_OK) return st;
  if (d.d != 128) return CURDKV_ERR_UNSUPPORTED;
  if (q_rows < 1 || !(scale >= 0.f) || std::isinf(scale) || scores == nullptr || (lse_given && lse == nullptr)) return CURDKV_ERR_INVALID_ARG;
  if (!query_strides_ok(Q, q_stride_b, q_stride_h, q_stride_n)) return CURDKV_ERR_INVALID_ARG;
  if (workspace == nullptr || !status_ok(workspace)) return CURDKV_ERR_INVALID_ARG;
  ScoresPlan pl;
  if (!plan_scores(&d, q_rows, &pl) || !map_strides_ok(d.batch, d.kv_heads, d.k_stride_b, d.k_stride_h, d.k_stride_n) ||
      !map_strides_ok(d.batch, d.q_heads, q_stride_b, q_stride_h, q_stride_n) ||
      !map_strides_ok(1, d.kv_heads, 0, (int64_t)(d.q_heads / d.kv_heads) * q_stride_h, 128))
    return CURDKV_ERR_UNSUPPORTED;
  if (workspace_bytes < pl.bytes) return CURDKV_ERR_WORKSPACE;
  const int64_t P = (int64_t)d.batch * d.kv_heads;
  if (P == 0) return CURDKV_OK;
  const int group = d.q_heads / d.kv_heads;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  CUtensorMap mq, mk;
  const uint64_t sizes[5] = {128, (uint64_t)group, (uint64_t)q_rows, (uint64_t)d.kv_heads, (uint64_t)d.batch};
  const int64_t strides[5] = {1, q_stride_h, q_stride_n, (int64_t)group * q_stride_h, q_stride_b};
  const uint32_t box[5] = {64, (uint32_t)group, (uint32_t)pl.tokens, 1, 1};
  umma::ScoreArgs a = {};
  a.seqlens = d.seqlens;
  a.q_lens = q_lens;
  a.batch = d.batch;
  a.heads = d.kv_heads;
  a.group = group;
  a.q_rows = q_rows;
  a.n_max = d.n_max;
  a.tokens = pl.tokens;
  a.row_tiles = pl.row_tiles;
  a.key_tiles = pl.key_tiles;
  // (products are masked before they are scaled, and -inf times 0 would be NaN)
  // The tensor cores cut the sums of products towards zero: measured, 0.8e-7 (small ones) to 1.5e-7 of |S| on average, 1.4e-7
  // where the weights are.  The scale gives that back, and log sums carry the factor that S then really gets, rounded scale and
  // all: what is off in both cancels where a key weighs something.  (8192 tokens with log sums formed in full fp32: off by 0.7
  // to 1.0e-6 of a score without either, much of it a factor of log sums that had 24 bits.)
  constexpr double kLog2e = 1.4426950408889634, kCut = 1.4e-7;
  const float scale_log2 = (float)((double)scale * kLog2e * (1. + kCut));
  a.scale_log2 = scale_log2 > FLT_MIN ? scale_log2 : FLT_MIN;
  const double ratio = scale_log2 > FLT_MIN ? (double)scale_log2 / (scale * (1. + kCut)) : kLog2e;
  auto two = [](double x) { return make_float2((float)x, (float)(x - (float)x)); };
  a.log2_of_ln = two(ratio);
  a.ln_of_log2 = two(1. / ratio);
  a.stats = reinterpret_cast<float2*>(ws + pl.stats_at);
  a.status = reinterpret_cast<uint32_t*>(ws);
  float* logsum = reinterpret_cast<float*>(ws + pl.logsum_at);
  a.logsum = logsum;
  a.next_unit = reinterpret_cast<uint32_t*>(ws + 256);
  a.segs = pl.row_segs;
  a.seg = pl.row_seg;
  a.units = (int)(P * ((pl.row_tiles + 1) / 2) * pl.row_segs);
  const int logsum_threads = kTileRows * (lse_given ? 1 : umma::row_threads(pl.row_segs));
  if (d.n_max == 0) {                                      // no scores; a query that sees nothing has a log sum all the same
    if (lse == nullptr || lse_given) return CURDKV_OK;
    return launch(umma::score_logsum_kernel, P * pl.row_tiles, logsum_threads, 0, false, stream, a, (const float*)nullptr, logsum, lse,
                  scores, (int64_t)0, reinterpret_cast<uint32_t*>(ws + 256) + 1)
               ? CURDKV_OK : CURDKV_ERR_CUDA;
  }
  if (!bf16_map(&mq, Q, 5, sizes, strides, box) ||
      !rows_map(&mk, K, d.batch, d.kv_heads, d.n_max, d.k_stride_b, d.k_stride_h, d.k_stride_n))
    return CURDKV_ERR_CUDA;
  static std::atomic<uint64_t> rows_done{0}, cols_done{0}, join_done{0};
  const auto rows_pass = umma::score_attention_kernel<false, false>;
  const int64_t places = sms();
  // Short calls whose log sums nobody asks for go without the kernel between the passes: the columns' CTAs, a unit each, join the
  // parts that they need, as often as there are pairs of key tiles (us, so | with the kernel
  // between: 32 tokens over 8 heads of 1024 rows 11.1 | 14.9, of 4096 13.7 | 16.2; 64 over one head of 4000 15.4 | 16.8.)
  const int64_t key_units = P * ((pl.key_tiles + 1) / 2) * pl.key_segs;
  const bool direct = !lse_given && lse == nullptr && key_units <= places && pl.key_seg <= umma::ScoreSmem<true>::kRing && pl.row_segs <= 16;
  const auto cols_pass = direct ? umma::score_attention_kernel<true, true> : umma::score_attention_kernel<true, false>;
  if (!allow_smem(rows_pass, umma::kScoreDynamic, rows_done) || !allow_smem(cols_pass, umma::kScoreDynamic, direct ? join_done : cols_done))
    return CURDKV_ERR_CUDA;
  if (direct && pl.key_segs == 1) {
    a.clear = scores;
    a.clear_count = P * d.n_max;
  }
  if (!lse_given && a.units > places && cudaMemsetAsync(a.next_unit, 0, sizeof(uint32_t), stream) != cudaSuccess) return CURDKV_ERR_CUDA;
  if (!lse_given &&
      !launch(rows_pass, a.units < places ? a.units : places, umma::kScoreThreads, umma::kScoreDynamic, false,
              stream, mq, mk, a))
    return CURDKV_ERR_CUDA;
  if (!direct &&
      !launch(umma::score_logsum_kernel, P * pl.row_tiles, logsum_threads, 0, !lse_given, stream, a,
              (const float*)(lse_given ? lse : nullptr), logsum, lse_given ? (float*)nullptr : lse, scores,
              pl.key_segs > 1 ? (int64_t)0 : P * d.n_max, a.next_unit + 1))
    return CURDKV_ERR_CUDA;
  a.next_unit += 1;
  a.join_segs = direct ? pl.row_segs : 0;
  a.join_seg = pl.row_seg;
  a.segs = pl.key_segs;
  a.seg = pl.key_seg;
  a.units = (int)key_units;
  float* parts = reinterpret_cast<float*>(ws + pl.parts_at);
  const int normalise = d.raw_scores ? 0 : 1;
  a.out = pl.key_segs > 1 ? parts : scores;
  a.normalise = pl.key_segs > 1 ? 0 : normalise;
  if (!launch(cols_pass, a.units < places ? a.units : places, umma::kScoreThreads, umma::kScoreDynamic, true,
              stream, mq, mk, a))
    return CURDKV_ERR_CUDA;
  if (pl.key_segs > 1 && !launch(umma::score_sum_kernel, P * ((d.n_max + 255) / 256), 256, 0, true, stream, a, (const float*)parts, scores, normalise))
    return CURDKV_ERR_CUDA;
  return CURDKV_OK;
}

}  // extern "C"
