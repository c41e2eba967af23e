// Attention weights of a prompt summed per key: w_j = sum over query rows r of 2^(x_rj - L_r), x = scale log2(e) q_r . k_j over
// the keys that row sees, L_r = log2 of its sum of exponentials.  No values, no output rows: two streams of logits that
// stay on the SM.
//
//   rows     S = Q K^T, a thread per query row: running maximum and sum, L_r                    (skipped when L is given)
//   columns  S^T = K Q^T, a thread per key: w_j is a sum along the thread's own row of the accumulator
//
// Transposing the second product puts each sum into one thread (two, for the halves of a row): no exchange between lanes, a
// fixed order.  Both are one kernel: fixed operand tiles A (M side: a thread a row of them) against a stream of tiles B.  A
// CTA works on a pair of A tiles, eight epilogue warps each (two threads a row, 64 columns each), so that every B tile is used
// twice; the accumulators (128 x 128 fp32) are double-buffered per A tile and fill TMEM.  What a pair sees -- the key
// tiles up to its last position, the row tiles from its first one on -- is cut into units of at most `seg` B tiles, which
// persistent CTAs take one by one, longest first.
//
// Query rows of a KV head are tiled as tokens x heads of the group (a 5-D map), so a tile of 128 rows is 128 / group tokens:
// few tokens of many heads fill a tile, and little of a tile lies beyond the diagonal.
//
// What bounds it: the special function units, 16 exponentials a clock and SM, two tiles' 2 x 1024 cycles a step; they are busy
// 80 to 82 % of the time, the tensor pipe 42 to 46 %, and the clock falls to 1.65 GHz beside them.  In the rows pass one pair of
// exponentials in eight runs on the FMA pipe: issue slots are 53 % taken, and with two in eight what the units gain is lost
// there.  8192 tokens, 32 / 8 heads: 333 us with log sums at hand (825 TFLOP/s over the visible pairs), 635 without; 64
// tokens over 4 x 8 heads of 32768 rows 178 us, the keys read twice.
// Measured and dropped: A in TMEM, brought there by the epilogue warps (345 us where shared memory gave 350 at the time: the
// products were not the bound, and short units paid for the copies); four epilogue warps a tile (377); a fixed deal of units
// in alternating direction (SMs idle a tenth of the time); sums of thousands of terms in one fp32 chain (1.3e-6 off).
#pragma once
#include "umma_ptx.cuh"

namespace curdkv {
namespace umma {

struct ScoreArgs {
  const int32_t* seqlens;            // [batch] or nullptr
  const int32_t* q_lens;             // [batch] or nullptr
  int batch, heads, group, q_rows, n_max;
  int tokens;                        // of a row tile: 128 / group; tokens * group rows
  int row_tiles, key_tiles;          // per (sequence, KV head)
  int segs, seg;                     // units per pair, B tiles of a unit at most
  int units;                         // pairs * batch * heads * segs
  uint32_t* next_unit;               // counter, 0 before, from which the CTAs take their units behind the first
  float scale_log2;                  // scale log2(e)
  float2 log2_of_ln, ln_of_log2;     // from natural log sums to L and back, in two parts each
  float2* stats;                     // rows: [segs][2][batch * heads][row_tiles][128] maximum (log2 units), sum
  const float* logsum;               // columns: [batch * heads][row_tiles][128] -L, -inf for rows that do not count
  float* out;                        // columns: [segs][2][batch * heads][n_max]; [batch * heads][n_max], 0 before, where segs = 1
  int normalise;                     // columns: divide by the rows that count (segs = 1)
  int join_segs, join_seg;           // columns that join the rows pass's parts themselves: its `segs` and `seg`
  float* clear;                      // rows: cleared for the columns pass, clear_count of them
  int64_t clear_count;
  uint32_t* status;
  unsigned long long wait_ns = kWaitLimitNs;
};

constexpr int kScoreThreads = 576;                         // TMA, MMA, 2 x 8 epilogue warps
// Seven tiles of shared memory: where the stream B is the keys, out of device memory, it gets five (a pair of A tiles is there
// for many of them then), where B is the queries, two pairs of A tiles (keys, two steps a pair when only a prompt's last
// tokens ask).
template <bool COLS>
struct ScoreSmem {
  static constexpr int kPairs = COLS ? 2 : 1, kRing = 7 - 2 * kPairs;
  static constexpr int kA = 0, kB = 2 * kPairs * kSlotBytes;
};
constexpr int kScoreLog = 7 * kSlotBytes;                  // columns: -L of the row tile in each B slot
constexpr int kScoreBar = kScoreLog + 3 * 512;
constexpr int kScoreDynamic = kScoreBar + 512 + 1024;
constexpr int kScoreTmemCols = 512;                        // S of A tile g, buffer u at 128 (2 g + u)
constexpr int kScoreUnits = 3;                             // units told ahead
constexpr float kScoreSlack = 8.f;
// Of 8 pairs of exponentials in the rows pass, how many the FMA pipe takes.  None in the columns pass, where they gained nothing
// (8192 tokens 365 us without, 367 with one) and where a caller's log sums may leave x beyond what that form takes.
constexpr int kScorePoly = 1;

// The live query tokens of a sequence and where they stand.
struct ScoreSeq {
  int n, q, pos0;                                          // rows, tokens, position of token 0
  __device__ __forceinline__ ScoreSeq() {}
  __device__ __forceinline__ ScoreSeq(const ScoreArgs& a, int b) {
    n = seq_len_of(a.seqlens, b, a.n_max);
    q = a.q_lens != nullptr ? min(max(a.q_lens[b], 0), a.q_rows) : a.q_rows;
    pos0 = n - q;
  }
};

// Maximum and sum of a query row, from the parts that the rows pass left.
struct RowSum {
  float top = -INFINITY, sum = 0.f;
  __device__ __forceinline__ void join(float2 e) {
    const float now = fmaxf(top, e.x);
    sum = sum * (now == -INFINITY ? 1.f : fast_exp2(top - now)) + e.y * (now == -INFINITY ? 1.f : fast_exp2(e.x - now));
    top = now;
  }
  // Parts `sub`, `sub` + `subs`, ...; the pair of tiles that `tile` belongs to walked units of `seg` key tiles.
  __device__ __forceinline__ void join_parts(const ScoreArgs& a, const ScoreSeq& s, int p, int tile, int r, int sub, int subs, int seg) {
    const int end_tok = min((tile / 2 * 2 + min(2, a.row_tiles - tile / 2 * 2)) * a.tokens, s.q);
    const int used = 2 * ((((s.pos0 + end_tok) + kTileRows - 1) / kTileRows + seg - 1) / seg);
    const float2* stats = a.stats + ((int64_t)p * a.row_tiles + tile) * kTileRows + r;
    const int64_t next = (int64_t)a.batch * a.heads * a.row_tiles * kTileRows;
    for (int g = sub; g < used; g += 4 * subs) {
      float2 e[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = g + subs * k < used ? stats[(g + subs * k) * next] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) join(e[k]);
    }
  }
  __device__ __forceinline__ float log() const { return sum == 0.f ? INFINITY : top + log2f(sum); }      // (of no weights: every 2^-L is 0)
};
__host__ __device__ constexpr int row_threads(int segs) { return segs > 4 ? 4 : 1; }           // that join a row's parts in turn

// A unit: a pair of A tiles of one (sequence, KV head) and a run of B tiles.
template <bool COLS>
struct ScoreUnit {
  int p, b, h, seg, a0, count, first, steps;               // A tiles a0 .. a0 + count - 1; B tiles first .. first + steps - 1
  __device__ __forceinline__ ScoreUnit() {}
  __device__ __forceinline__ ScoreUnit(const ScoreArgs& a, int unit) {
    const int tiles = COLS ? a.key_tiles : a.row_tiles, P = a.batch * a.heads, pairs = (tiles + 1) / 2;
    seg = unit % a.segs;
    p = unit / a.segs % P;
    const int at = unit / a.segs / P;
    a0 = 2 * (COLS ? at : pairs - 1 - at);                 // longest first
    count = min(2, tiles - a0);
    b = p / a.heads;
    h = p % a.heads;
    const ScoreSeq s(a, b);
    int end;
    if (COLS) {                                            // row tiles whose last token stands at or behind the first key
      end = (s.q + a.tokens - 1) / a.tokens;
      first = max(0, a0 * kTileRows - s.pos0) / a.tokens;
      if (a0 * kTileRows >= s.n) end = 0;
    } else {                                               // key tiles up to the pair's last position
      const int tok = min((a0 + count) * a.tokens, s.q);   // tokens below this
      end = tok > a0 * a.tokens ? (max(s.pos0 + tok, 0) + kTileRows - 1) / kTileRows : 0;
      first = 0;
    }
    first += seg * a.seg;
    steps = min(max(end - first, 0), a.seg);
  }
};

// map_q: 5-D (channel, head of the group, token, KV head, sequence), boxes of 64 x group x tokens; map_k: tiles of 128 rows.
// JOIN: a columns pass whose CTAs have one unit each, of no more steps than B slots, and join the rows pass's parts themselves.
template <bool COLS, bool JOIN>
__global__ void __launch_bounds__(kScoreThreads, 1)
score_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const ScoreArgs a) {
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  constexpr int kRing = ScoreSmem<COLS>::kRing, kPairs = ScoreSmem<COLS>::kPairs;
  const uint32_t bar0 = base + kScoreBar;
  auto a_full = [&](uint32_t s) { return bar0 + 8u * s; };
  auto a_empty = [&](uint32_t s) { return bar0 + 16u + 8u * s; };
  auto s_full = [&](uint32_t g, uint32_t u) { return bar0 + 32u + 16u * g + 8u * u; };
  auto s_empty = [&](uint32_t g, uint32_t u) { return bar0 + 64u + 16u * g + 8u * u; };
  auto b_full = [&](uint32_t s) { return bar0 + 96u + 8u * s; };
  auto b_empty = [&](uint32_t s) { return bar0 + 96u + 8u * (kRing + s); };
  constexpr int kBars = 96 + 16 * kRing;
  const uint32_t drain_bar = bar0 + kBars;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(base_ptr + kScoreBar + kBars + 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  auto i_full = [&](uint32_t e) { return bar0 + kBars + 16u + 8u * e; };
  auto i_empty = [&](uint32_t e) { return bar0 + kBars + 16u + 8u * (kScoreUnits + e); };
  int4* unit_ring = reinterpret_cast<int4*>(base_ptr + kScoreBar + 256);         // [kScoreUnits][3]
  static_assert(kBars + 16 + 16 * kScoreUnits <= 256 && 48 * kScoreUnits <= 256, "barriers and units fit");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rows_used = a.tokens * a.group;                // of a row tile

  if (tid == 0) {
    for (int k = 0; k < kPairs; ++k) { mbar_init(a_full(k), 1); mbar_init(a_empty(k), 1); }
    // (columns: the sixteen epilogue warps read the row tile's L beside the product)
    for (int s = 0; s < kRing; ++s) { mbar_init(b_full(s), 1); mbar_init(b_empty(s), COLS ? 17 : 1); }
    for (int g = 0; g < 2; ++g)
      for (int k = 0; k < 2; ++k) { mbar_init(s_full(g, k), 1); mbar_init(s_empty(g, k), 8); }
    for (int e = 0; e < kScoreUnits; ++e) { mbar_init(i_full(e), 1); mbar_init(i_empty(e), 17); }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of a query tile that no copy ever fills: zeros
  if (rows_used < kTileRows) {
    const int slots = COLS ? kRing : 2 * kPairs, from = COLS ? ScoreSmem<COLS>::kB : ScoreSmem<COLS>::kA;
    const int dead = (kTileRows - rows_used) * 8;
    for (int x = tid; x < slots * 2 * dead; x += kScoreThreads) {
      const int half = x / dead, y = x % dead;             // half tiles lie kHalfBytes apart
      *reinterpret_cast<uint4*>(base_ptr + from + half * kHalfBytes + rows_used * 128 + y * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                 "r"((uint32_t)kScoreTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  constexpr uint32_t tmem_base = 0u;                       // all 512 columns are this CTA's: they begin at 0
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // The columns pass is launched behind the kernel that leaves L (or its parts), which began when everything before it had
  // ended: queries and keys are loaded at once, what comes from that kernel is waited for where it is needed.
  auto wait_before = [&]() { asm volatile("griddepcontrol.wait;" ::: "memory"); };
  if (!COLS) {
    wait_before();
    for (int64_t x = (int64_t)blockIdx.x * kScoreThreads + tid; x < a.clear_count; x += (int64_t)gridDim.x * kScoreThreads) a.clear[x] = 0.f;
  }

  // The producer takes units from the counter, longest first, and tells the others one ahead; one without steps: no more.  (Which CTA takes
  // which changes no result.)  A fixed deal in alternating direction left SMs idle a tenth of the time.
  uint32_t told = 0;                                       // units heard of
  auto next_unit = [&](ScoreUnit<COLS>& u, ScoreSeq& seq, bool& ok) {        // for the warps that listen
    const uint32_t e = told % kScoreUnits;
    ok = __all_sync(0xffffffffu, mbar_wait(i_full(e), (told / kScoreUnits) & 1u, abort_flag, a.status, a.wait_ns) && ok);
    if (!ok) return false;
    const int4 x = unit_ring[3 * e], y = unit_ring[3 * e + 1], z = unit_ring[3 * e + 2];
    __syncwarp();
    if (elect_one()) mbar_arrive(i_empty(e));
    ++told;
    u.p = x.x; u.b = x.y; u.h = x.z; u.seg = x.w;
    u.a0 = y.x; u.count = y.y; u.first = y.z; u.steps = y.w;
    seq.n = z.x; seq.q = z.y; seq.pos0 = z.z;
    return u.steps > 0;
  };
  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      uint64_t keep;
      asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(keep));
      const uint32_t q_bytes = (uint32_t)rows_used * 256u;
      bool ok = true;
      uint32_t it = 0, pairs = 0;
      auto wait = [&](uint32_t bar, uint32_t parity) { return ok = ok && mbar_wait(bar, parity, abort_flag, a.status, a.wait_ns); };
      auto load = [&](const ScoreUnit<COLS>& u, bool queries, uint32_t dst, uint32_t bar, int tile) {
        if (queries) {
          tma_load_5d(dst, &map_q, bar, 0, 0, tile * a.tokens, u.h, u.b);
          tma_load_5d(dst + kHalfBytes, &map_q, bar, 64, 0, tile * a.tokens, u.h, u.b);
        } else {
          tma_load_4d(dst, &map_k, bar, 0, tile * kTileRows, u.h, u.b, keep);
          tma_load_4d(dst + kHalfBytes, &map_k, bar, 64, tile * kTileRows, u.h, u.b, keep);
        }
      };
      // (of very many units, of which short sequences leave many without steps, several are taken at a time)
      const int64_t batch = min(max(a.units / (32 * (int)gridDim.x), 1), 16);
      int64_t at = blockIdx.x, last = at + 1;              // units taken
      bool waited = !COLS;
      auto behind = [&]() {
        if (!waited) wait_before();
        waited = true;
      };
      auto take = [&](ScoreUnit<COLS>& u) {                // the next unit that has steps, told to the others
        do {
          if (at == last) {
            if (a.units > (int)gridDim.x) behind();
            at = a.units > (int)gridDim.x ? (int64_t)gridDim.x + batch * atomicAdd(a.next_unit, 1u) : (int64_t)a.units;
            last = at + batch;
          }
          if (at >= a.units) {
            u.steps = 0;
            break;
          }
          u = ScoreUnit<COLS>(a, (int)at++);
        } while (u.steps == 0);
        const uint32_t e = told % kScoreUnits;
        if (wait(i_empty(e), ((told / kScoreUnits) & 1u) ^ 1u)) {
          const ScoreSeq seq(a, u.b);
          unit_ring[3 * e] = make_int4(u.p, u.b, u.h, u.seg);
          unit_ring[3 * e + 1] = make_int4(u.a0, u.count, u.first, u.steps);
          unit_ring[3 * e + 2] = make_int4(seq.n, seq.q, seq.pos0, 0);
          mbar_arrive(i_full(e));
        }
        ++told;
      };
      ScoreUnit<COLS> u(a, 0), then(a, 0);
      take(u);
      if (u.steps > 0) take(then);
      while (ok && u.steps > 0) {
        const uint32_t pair = pairs % kPairs;
        if (!wait(a_empty(pair), ((pairs / kPairs) & 1u) ^ 1u)) break;
        ++pairs;
        mbar_arrive_expect_tx(a_full(pair), (uint32_t)u.count * (COLS ? (uint32_t)kSlotBytes : q_bytes));
        for (int g = 0; g < u.count; ++g) load(u, !COLS, base + ScoreSmem<COLS>::kA + (2 * pair + g) * kSlotBytes, a_full(pair), u.a0 + g);
        for (int x = 0; ok && x < u.steps; ++x) {
          const uint32_t slot = it % kRing;
          if (!wait(b_empty(slot), ((it / kRing) & 1u) ^ 1u)) break;
          ++it;
          const int tile = u.first + x;
          mbar_arrive_expect_tx(b_full(slot), COLS ? q_bytes + (JOIN ? 0u : 512u) : (uint32_t)kSlotBytes);
          load(u, COLS, base + ScoreSmem<COLS>::kB + slot * kSlotBytes, b_full(slot), tile);
          if (COLS && !JOIN) {
            behind();
            bulk_load(base + kScoreLog + slot * 512, a.logsum + ((int64_t)u.p * a.row_tiles + tile) * kTileRows, 512u, b_full(slot));
          }
        }
        u = then;
        if (u.steps > 0) take(then);                       // (behind the last unit `then` stays as it is)
      }
      if (!ok) {                                           // let what was issued land before the CTA ends
        auto land = [&](uint32_t bar, uint32_t parity) {
          const unsigned long long t0 = global_ns();
          while (!mbar_try_wait(bar, parity) && global_ns() - t0 < a.wait_ns) {}
        };
        for (uint32_t x = it - min(it, (uint32_t)kRing); x < it; ++x) land(b_full(x % kRing), (x / kRing) & 1u);
        for (uint32_t x = pairs - min(pairs, (uint32_t)kPairs); x < pairs; ++x) land(a_full(x % kPairs), (x / kPairs) & 1u);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ products: the whole warp waits, one lane issues
    constexpr uint32_t idesc = instr_desc_bf16(kTileRows);
    if (COLS && !JOIN) wait_before();                      // (it would spin on L; joined calls are short)
    const uint64_t a_desc0 = smem_desc_sw128(base + ScoreSmem<COLS>::kA), b_desc0 = smem_desc_sw128(base + ScoreSmem<COLS>::kB);
    bool ok = true;
    uint32_t it = 0, pairs = 0, done[2] = {0, 0};          // B tiles, pairs of A tiles, products of each group
    auto wait = [&](uint32_t bar, uint32_t parity) { ok = mbar_wait(bar, parity, abort_flag, a.status, a.wait_ns) && ok; };
    ScoreUnit<COLS> u;
    ScoreSeq seq;
    while (next_unit(u, seq, ok)) {
      const uint32_t pair = pairs % kPairs;
      wait(a_full(pair), (pairs / kPairs) & 1u);
      ++pairs;
      for (int x = 0; ok && x < u.steps; ++x, ++it) {
        const uint32_t slot = it % kRing;
        wait(b_full(slot), (it / kRing) & 1u);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (g >= u.count || !ok) continue;
          const uint32_t buf = done[g] & 1u;
          wait(s_empty(g, buf), ((done[g] >> 1) & 1u) ^ 1u);
          ++done[g];
          if (!(ok = __all_sync(0xffffffffu, ok))) continue;
          tc_fence_after();
          const uint64_t ad = a_desc0 + (2 * pair + g) * (kSlotBytes >> 4), bd = b_desc0 + slot * (kSlotBytes >> 4);
          if (elect_one()) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t off = (uint32_t)(e >> 2) * (kHalfBytes >> 4) + (uint32_t)(e & 3) * 2u;
              tc_mma_bf16(tmem_base + 128u * (2 * g + buf), ad + off, bd + off, idesc, e > 0);
            }
            tc_commit(s_full(g, buf));
          }
          __syncwarp();
        }
        if (ok && elect_one()) tc_commit(b_empty(slot));
        __syncwarp();
      }
      if (ok && elect_one()) tc_commit(a_empty(pair));
      __syncwarp();
    }
    if (!ok) {
      if (elect_one()) tc_commit(drain_bar);
      __syncwarp();
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(drain_bar, 0) && global_ns() - t0 < a.wait_ns) {}
    }
  } else {
    // ------------------------------------------------------------ epilogue: row r of A tile g, columns 64 half onwards
    const int g = (warp - 2) >> 3, half = ((warp - 2) >> 2) & 1, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const float sc = a.scale_log2;
    const uint64_t sc2 = pack2(sc, sc);
    const int P = a.batch * a.heads;
    if (COLS) wait_before();
    if constexpr (JOIN) {
      // This CTA's only unit has a slot for each of its row tiles: -L goes to where a copy would bring it.  (The second pair of
      // A tiles is never used then.)
      const ScoreUnit<COLS> own(a, (int)blockIdx.x);
      const ScoreSeq s(a, own.b);
      float2* others = reinterpret_cast<float2*>(base_ptr + ScoreSmem<COLS>::kA + 2 * kSlotBytes);
      const int e = tid - 64, row = e % kTileRows, sub = e / kTileRows, subs = row_threads(a.join_segs);
      for (int x = 0; x < own.steps; ++x) {
        const int tok = (own.first + x) * a.tokens + row / a.group;
        const bool sees = row < rows_used && tok < s.q && s.pos0 + tok >= 0;
        RowSum all;
        if (sees && sub < subs) all.join_parts(a, s, own.p, own.first + x, row, sub, subs, a.join_seg);
        if (sub > 0) others[(sub - 1) * kTileRows + row] = make_float2(all.top, all.sum);
        asm volatile("bar.sync 1, 512;" ::: "memory");
        if (sub == 0) {
          for (int k = 0; k < subs - 1; ++k) all.join(others[k * kTileRows + row]);
          reinterpret_cast<float*>(base_ptr + kScoreLog + x * 512)[row] = sees ? -all.log() : -INFINITY;
        }
        asm volatile("bar.sync 1, 512;" ::: "memory");
      }
    }
    bool ok = true;
    uint32_t it = 0, done = 0;                             // B tiles, this group's products
    ScoreUnit<COLS> u;
    ScoreSeq seq;
    while (next_unit(u, seq, ok)) {
      const bool mine = g < u.count;
      float top = -INFINITY, sum = 0.f, lost = 0.f;
      const int key = (u.a0 + g) * kTileRows + r;          // columns
      const int tok = (u.a0 + g) * a.tokens + r / a.group; // rows
      const int pos = !COLS && r < rows_used && tok < seq.q ? seq.pos0 + tok : -1;           // keys up to here
      for (int x = 0; x < u.steps; ++x, ++it) {
        if (!COLS && !mine) break;
        // (columns: L lands with the tile, and a group without an A tile keeps pace, its arrivals count)
        const uint32_t slot = it % kRing, buf = done & 1u;
        if (COLS) ok = mbar_wait(b_full(slot), (it / kRing) & 1u, abort_flag, a.status, a.wait_ns);
        if (mine) {
          ok = ok && mbar_wait(s_full(g, buf), (done >> 1) & 1u, abort_flag, a.status, a.wait_ns);
          ++done;
        }
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        tc_fence_after();
        const uint32_t s_addr = lane_addr + 128u * (2 * g + buf) + 64u * half;
        if (COLS && mine) {
          const float4* L = reinterpret_cast<const float4*>(base_ptr + kScoreLog + slot * 512 + 256 * half);
          const int tok0 = (u.first + x) * a.tokens;
          // columns [c_lo, c_hi) count: tokens at or behind this key, and those that exist
          const int c_hi = min(seq.q - tok0, a.tokens) * a.group - 64 * half;
          const int ahead = key - (seq.pos0 + tok0), c_lo = (ahead > 0 ? min(ahead, a.tokens) * a.group : 0) - 64 * half;
          uint64_t part[4] = {0ull, 0ull, 0ull, 0ull};
          if (__all_sync(0xffffffffu, c_lo <= 0) && c_hi >= rows_used - 64 * half) {
            float v[2][32];
            tmem_ld32(s_addr, v[0]);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              tmem_ld_wait();
              if (c < 1) tmem_ld32(s_addr + 32, v[1]);
              const float(&w)[32] = v[c];
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const float4 l4 = L[8 * c + (e >> 2)];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                  const int j = (e >> 1) + i;
                  const uint64_t x2 = fma2(pack2(w[2 * j], w[2 * j + 1]), sc2, i == 0 ? pack2(l4.x, l4.y) : pack2(l4.z, l4.w));
                  part[j & 3] = add2(part[j & 3], exp2_pair(x2));
                }
              }
            }
          } else if (__any_sync(0xffffffffu, c_lo < 64) && c_hi > 0) {
#pragma unroll 1
            for (int c0 = 0; c0 < 64; c0 += 32) {
              float v[32];
              tmem_ld32(s_addr + c0, v);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                const float2 l2 = reinterpret_cast<const float2*>(L)[(c0 + e) >> 1];
                const int c = c0 + e;
                const float x0 = c < c_lo || c >= c_hi ? -INFINITY : fmaf(v[e], sc, l2.x);
                const float x1 = c + 1 < c_lo || c + 1 >= c_hi ? -INFINITY : fmaf(v[e + 1], sc, l2.y);
                part[(e >> 1) & 3] = add2(part[(e >> 1) & 3], pack2(fast_exp2(x0), fast_exp2(x1)));
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (elect_one()) mbar_arrive(s_empty(g, buf));
          float p0, p1;
          unpack2(add2(add2(part[0], part[1]), add2(part[2], part[3])), p0, p1);
          // the tiles' sums are added with what their additions lose (thousands of rows may follow one another)
          const float y = (p0 + p1) - lost, now = sum + y;
          lost = (now - sum) - y;
          sum = now;
        }
        if (COLS) {
          __syncwarp();
          if (elect_one()) mbar_arrive(b_empty(slot));
        }
        if (!COLS && mine) {
          float v[64];
          tmem_ld32(s_addr, *reinterpret_cast<float(*)[32]>(v));
          tmem_ld32(s_addr + 32, *reinterpret_cast<float(*)[32]>(v + 32));
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (elect_one()) mbar_arrive(s_empty(g, buf));   // S is in registers
          const int see = pos + 1 - (u.first + x) * kTileRows - 64 * half;         // columns below this
          if (!__any_sync(0xffffffffu, see > 0)) continue;
          if (__any_sync(0xffffffffu, see < 64)) {
#pragma unroll
            for (int e = 0; e < 64; ++e)
              if (e >= see) v[e] = -INFINITY;
          }
          float ext[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int e = 4; e < 60; e += 8)
#pragma unroll
            for (int j = 0; j < 4; ++j) ext[j] = max3(ext[j], v[e + 2 * j], v[e + 2 * j + 1]);
#pragma unroll
          for (int j = 0; j < 4; ++j) ext[j] = fmaxf(ext[j], v[60 + j]);
          const float tile_top = fmaxf(fmaxf(ext[0], ext[1]), fmaxf(ext[2], ext[3])) * sc;
          if (tile_top > top + kScoreSlack || top == -INFINITY) {
            const float now = fmaxf(top, tile_top);
            sum *= now == -INFINITY ? 1.f : fast_exp2(top - now);
            top = now;
          }
          const float ref = top == -INFINITY ? 0.f : top;
          const uint64_t nref2 = pack2(-ref, -ref);
          uint64_t part[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            const uint64_t x2 = fma2(pack2(v[e], v[e + 1]), sc2, nref2);
            part[(e >> 1) & 3] = add2(part[(e >> 1) & 3], (e >> 1) % 8 < kScorePoly ? exp2_pair_fma(x2) : exp2_pair(x2));
          }
          float p0, p1;
          unpack2(add2(add2(part[0], part[1]), add2(part[2], part[3])), p0, p1);
          sum += p0 + p1;
        }
      }
      if (!ok) break;
      if (COLS && mine && key < seq.n) {
        if (a.segs == 1)                                   // two halves are added to 0: either order gives the same
          atomicAdd(a.out + (int64_t)u.p * a.n_max + key, a.normalise ? sum * (1.f / (float)max(min(seq.q, seq.n) * a.group, 1)) : sum);
        else
          a.out[((int64_t)(2 * u.seg + half) * P + u.p) * a.n_max + key] = sum;
      }
      if (!COLS && mine)
        a.stats[(((int64_t)(2 * u.seg + half) * P + u.p) * a.row_tiles + (u.a0 + g)) * kTileRows + r] = make_float2(top, sum);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)kScoreTmemCols)
                 : "memory");
  }
}

// -L of every query row, from the parts of the rows pass or from log sums that the caller has; -inf where a row does not count.
// Clears `clear` floats of `scores` and the columns pass's counter beside it.  grid = batch * heads * row tiles, block = 128, or
// 512 for many parts: four threads a row take them in turn.
constexpr int kLogsumThreads = 4 * kTileRows;
__global__ void __launch_bounds__(kLogsumThreads) score_logsum_kernel(const ScoreArgs a, const float* given, float* logsum,
                                                                      float* lse_out, float* scores, int64_t clear,
                                                                      uint32_t* next_unit) {
  __shared__ float2 s_part[3][kTileRows];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int64_t x = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; x < clear; x += (int64_t)gridDim.x * blockDim.x) scores[x] = 0.f;
  if (blockIdx.x == 0 && threadIdx.x == 0) *next_unit = 0u;
  const int tile = blockIdx.x % a.row_tiles, p = blockIdx.x / a.row_tiles, b = p / a.heads, h = p % a.heads;
  const int r = threadIdx.x % kTileRows, sub = threadIdx.x / kTileRows, subs = blockDim.x / kTileRows;
  const ScoreSeq s(a, b);
  const int tok = tile * a.tokens + r / a.group;
  const bool live = r < a.tokens * a.group && tok < s.q, sees = live && s.pos0 + tok >= 0;
  RowSum all;
  if (given == nullptr) {
    if (sees) all.join_parts(a, s, p, tile, r, sub, subs, a.seg);
    if (sub > 0) s_part[sub - 1][r] = make_float2(all.top, all.sum);
    __syncthreads();
  }
  if (sub > 0) return;
  const int64_t at = ((int64_t)b * a.heads * a.group + h * a.group + r % a.group) * a.q_rows + tok;
  float L = INFINITY;
  if (sees) {
    if (given != nullptr) {
      const float g = given[at];
      L = g == -INFINITY ? INFINITY : fmaf(g, a.log2_of_ln.x, g * a.log2_of_ln.y);           // (-inf: a row that saw nothing)
    } else {
      for (int k = 0; k < subs - 1; ++k) all.join(s_part[k][r]);
      L = all.log();
    }
  }
  logsum[((int64_t)p * a.row_tiles + tile) * kTileRows + r] = -L;
  if (live && lse_out != nullptr) lse_out[at] = L == INFINITY ? -INFINITY : fmaf(L, a.ln_of_log2.x, L * a.ln_of_log2.y);
}

// Sums the units' parts of each key in order.  grid = batch * heads * ceil(n_max / 256), block = 256.
__global__ void __launch_bounds__(256) score_sum_kernel(const ScoreArgs a, const float* parts, float* scores, int normalise) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int each = (a.n_max + 255) / 256, p = blockIdx.x / each, key = blockIdx.x % each * 256 + threadIdx.x;
  if (key >= a.n_max) return;
  const ScoreSeq s(a, p / a.heads);
  float w = 0.f;
  if (key < s.n) {
    // what the key's pair of tiles sees, and so the units that had something to do
    const int first = max(0, key / (2 * kTileRows) * (2 * kTileRows) - s.pos0) / a.tokens, end = (s.q + a.tokens - 1) / a.tokens;
    const int used = end > first ? 2 * ((end - first + a.seg - 1) / a.seg) : 0;
    for (int g = 0; g < used; ++g) w += parts[((int64_t)g * a.batch * a.heads + p) * a.n_max + key];
    if (normalise) w *= 1.f / (float)max(min(s.q, s.n) * a.group, 1);
  }
  scores[(int64_t)p * a.n_max + key] = w;
}

}  // namespace umma
}  // namespace curdkv
