// Causal attention with a sliding window and sinks for prompts (many query rows per head):
// O = softmax(scale Q K^T) V over the keys j <= pos with j > pos - window or j < num_sink.
//
// Persistent CTAs, one per SM.  A work item is a pair of query tiles (128 rows of one query head each)
// of the same KV head, so that both read the same tiles of K and V: tiles are numbered row block
// major, query head of the group minor, and tiles 2 i and 2 i + 1 make a pair -- two heads at the
// same rows for even groups, neighbouring row blocks for a group of one.  Only the key tiles that some
// row of the pair sees are walked: those holding sinks, then those of the window.
//
// Ten warps.  Four softmax warps own each query tile, a thread per row: S = Q K^T arrives in TMEM,
// the thread takes its 128 logits into registers, and the weights go back over S as bf16, where they are
// the A operand of O += P V straight from TMEM.  One issuing warp alternates P V of a key tile with S of
// the next, tile by tile: while one query tile turns logits into weights the tensor pipe works for the
// other.  P is handed over in halves, so that P V starts on the first 64 keys.  The last warp walks
// the work: it feeds Q and the ring of K and V tiles by TMA and describes every step (one key tile of one
// item) to the others in a small ring of its own.  Items follow each other without a gap: the next pair's
// first S is issued right behind the last product of this one, and O is free again as soon as it is in
// registers.
//
// The issuing warp has to be quick between its batches of products, or the pipe runs dry: it works
// converged with one elected lane issuing (inside `if (lane == 0)` the compiler cannot use uniform
// registers, and a product beside busy softmax warps took 270 cycles to issue instead of 90), in one rolled
// loop with little code.  Measured and dropped: two threads per row (a tile's softmax 2650 cycles against
// 1700, the warps crowding each other out); an issuing warp per query tile (205 us where this takes 180: the
// tiles fall into step, and their exponentials with them; with turns for the exponentials 199); 64-key
// steps; every other pair of exponentials as a polynomial on the FMA pipe (no change).
//
// What bounds it: the chain of one query tile.  A step of 128 keys takes 3900 cycles: 2300 from logits to weights
// (500 for reading them and the maximum, 850 for each half of the exponentials and its hand-over), 256 for the
// second half of P V, 512 for the next S, and some 800 of waits and wake-ups between them.  S cannot be issued
// earlier, because the weights lie over it and two S and two O fill TMEM.  Of the 3900 cycles the two tiles keep
// the tensor pipe busy for 2048, and the special function units for as many.  A change of items costs
// 4000 cycles (the last product, O through registers, the first S of the next) every nine steps at window
// 1024.  8192 tokens, 32 / 8 heads, window 1024: 180 us, 718 TFLOP/s over the visible keys; 4 prompts of up
// to 2000 tokens, window 512: 72 us.
//
// The running maximum moves only when a tile exceeds it by more than 2^8 (as in attn_umma.cuh); the
// group then rescales its accumulator in TMEM, which after the first tiles is rare.  All waits are bounded.
#pragma once
#include "attn_token.cuh"
#include "umma_ptx.cuh"

namespace curdkv {

// Map of a bf16 tensor [batch][heads][rows][128] for tiles of 128 rows (defined beside the C ABI).
bool rows_map(CUtensorMap* map, const void* base, int32_t batch, int32_t heads, int32_t rows, int64_t stride_b,
              int64_t stride_h, int64_t stride_n);

namespace umma {

struct WindowArgs {
  const int32_t* seqlens;            // [batch] or nullptr
  const int32_t* q_lens;             // [batch] or nullptr
  int batch, heads, group, q_rows, n_max;
  int num_sink, window;
  float scale_log2;
  __nv_bfloat16* O;
  int64_t o_sb, o_sh, o_sn;
  float* lse;
  uint32_t* status;
  int pairs;                         // tile pairs per (sequence, KV head)
  int items;                         // batch * heads * pairs
                                     // (num_sink and window: at most n_max, and n_max + q_rows below 2^30)
  unsigned long long wait_ns = kWaitLimitNs;
};

constexpr int kWinThreads = 320;
constexpr int kWinSoftmaxWarps = 8;
constexpr int kWinRing = 4;
constexpr int kWinQ = 0;                                   // Q of the two tiles
constexpr int kWinSlot0 = 2 * kSlotBytes;
constexpr int kWinStage = kWinSlot0 + kWinRing * kSlotBytes;         // 4 KB per softmax warp for its output
constexpr int kWinBar = kWinStage + kWinSoftmaxWarps * 4096;
constexpr int kWinInfoRing = 8;                            // steps described ahead
constexpr int kWinDynamic = kWinBar + 1024 + 1024;
constexpr int kWinTmemCols = 512;                          // S_A, S_B, O_A, O_B
constexpr float kWinSlack = 8.f;

// A step: one key tile of one item.  Flag bits of query tile g are shifted by 4 g.
constexpr uint32_t kStepNeeds = 1u, kStepFirst = 2u, kStepLast = 4u;
constexpr uint32_t kStepZero = 8u;                         // the query tile has rows that see no key at all: O = 0
constexpr uint32_t kStepStop = 1u << 8;                    // no step: the work is done
constexpr uint32_t kStepEmpty = 1u << 9;                   // no key tile: only zeros to write
constexpr int kStepGroups = 12;                            // from this bit: groups of 16 keys that matter (1 .. 8)

struct alignas(16) StepInfo {
  uint32_t flags;
  int j0, n, b;                      // first key of the tile; rows of the sequence; sequence
  int head[2], row0[2];              // query heads; first query rows of the tiles
  int pos0[2], rows[2];              // position of that row; rows that exist
};
static_assert(sizeof(StepInfo) == 48, "written and read as three 16-byte words");

// One query tile of an item, and which key tiles it needs: [0, sink_tiles) and [lo, hi).
struct WinTile {
  int rows, sink_tiles, lo, hi;
  __device__ __forceinline__ bool needs(int kt) const { return kt < sink_tiles || (kt >= lo && kt < hi); }
  __device__ __forceinline__ bool any() const { return sink_tiles > 0 || hi > lo; }
  __device__ __forceinline__ int first() const { return sink_tiles > 0 ? 0 : lo; }
  __device__ __forceinline__ int last() const { return max(sink_tiles, hi > lo ? hi : 0) - 1; }
};

// A wait that a whole warp makes together: false for all lanes when it ran out for one.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t* status,
                                          unsigned long long limit) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, status, limit));
}

__global__ void __launch_bounds__(kWinThreads, 1)
window_umma_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, const WindowArgs a) {
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bar0 = base + kWinBar;
  auto full_bar = [&](uint32_t s) { return bar0 + 8u * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8u * (kWinRing + s); };
  const uint32_t gbar = bar0 + 8u * 2 * kWinRing;
  auto q_full = [&](int g) { return gbar + 8u * g; };
  auto q_empty = [&](int g) { return gbar + 16u + 8u * g; };
  auto s_full = [&](int g) { return gbar + 32u + 8u * g; };
  auto p_ready = [&](int g, int half) { return gbar + 48u + 16u * half + 8u * g; };
  auto o_full = [&](int g) { return gbar + 80u + 8u * g; };
  auto o_empty = [&](int g) { return gbar + 96u + 8u * g; };
  const uint32_t drain_bar = gbar + 112u;
  auto info_full = [&](uint32_t e) { return gbar + 144u + 8u * e; };
  auto info_empty = [&](uint32_t e) { return gbar + 144u + 8u * (kWinInfoRing + e); };
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(base_ptr + kWinBar + 480);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  uint4* info = reinterpret_cast<uint4*>(base_ptr + kWinBar + 512);           // [kWinInfoRing][3]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int s = 0; s < kWinRing; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int e = 0; e < kWinInfoRing; ++e) { mbar_init(info_full(e), 1); mbar_init(info_empty(e), kWinSoftmaxWarps + 1); }
    for (int g = 0; g < 2; ++g) {
      mbar_init(q_full(g), 1);
      mbar_init(q_empty(g), 1);
      mbar_init(s_full(g), 1);
      mbar_init(p_ready(g, 0), 128);
      mbar_init(p_ready(g, 1), 128);
      mbar_init(o_full(g), 1);
      mbar_init(o_empty(g), 128);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kWinSoftmaxWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                 "r"((uint32_t)kWinTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  constexpr uint32_t tmem_base = 0u;                       // all 512 columns are this CTA's: they begin at 0

  if (warp == kWinSoftmaxWarps + 1) {
    // ------------------------------------------------------------ the work, step by step, and its tiles
    // Ring order of an item: K_0, V_0, K_1, V_1, ...; its two Q tiles follow K_0.
    if (lane == 0) {
      uint64_t pol;
      asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
      uint32_t it = 0, step = 0, q_it[2] = {0, 0};
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) { return ok = ok && mbar_wait(bar, parity, abort_flag, a.status, a.wait_ns); };
      auto load = [&](const CUtensorMap* map, int j0, int h, int b) {
        const uint32_t slot = it % kWinRing;
        if (!wait(empty_bar(slot), ((it / kWinRing) & 1u) ^ 1u)) return;
        mbar_arrive_expect_tx(full_bar(slot), kSlotBytes);
        const uint32_t dst = base + kWinSlot0 + slot * kSlotBytes;
        tma_load_4d(dst, map, full_bar(slot), 0, j0, h, b, pol);
        tma_load_4d(dst + kHalfBytes, map, full_bar(slot), 64, j0, h, b, pol);
        ++it;
      };
      auto describe = [&](const StepInfo& i) {
        const uint32_t e = step % kWinInfoRing;
        if (!wait(info_empty(e), ((step / kWinInfoRing) & 1u) ^ 1u)) return;
        info[3 * e] = make_uint4(i.flags, (uint32_t)i.j0, (uint32_t)i.n, (uint32_t)i.b);
        info[3 * e + 1] = make_uint4((uint32_t)i.head[0], (uint32_t)i.head[1], (uint32_t)i.row0[0], (uint32_t)i.row0[1]);
        info[3 * e + 2] = make_uint4((uint32_t)i.pos0[0], (uint32_t)i.pos0[1], (uint32_t)i.rows[0], (uint32_t)i.rows[1]);
        mbar_arrive(info_full(e));
        ++step;
      };
      // Items: the row blocks fall from the last pair on (longest rows first); heads and sequences
      // vary fastest.
      const int per = a.batch * a.heads;
      const int skip_pairs = (int)gridDim.x / per, skip_p = (int)gridDim.x % per;
      int pair = a.pairs - 1 - (int)blockIdx.x / per, p = (int)blockIdx.x % per;
      while (ok && pair >= 0) {
        const int b = p / a.heads, h = p % a.heads;
        StepInfo i;
        i.b = b;
        i.n = seq_len_of(a.seqlens, b, a.n_max);
        const int q = a.q_lens != nullptr ? min(max(a.q_lens[b], 0), a.q_rows) : a.q_rows;
        WinTile t[2];
        int sinks = 0, lo = 0x7fffffff, hi = 0, rb = 2 * pair / a.group, head = 2 * pair % a.group;
        uint32_t zero = 0u;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          i.head[g] = h * a.group + head;
          i.row0[g] = rb * kTileRows;
          i.rows[g] = t[g].rows = min(max(q - rb * kTileRows, 0), kTileRows);
          i.pos0[g] = i.n - q + rb * kTileRows;
          t[g].sink_tiles = t[g].lo = t[g].hi = 0;
          const int end = t[g].rows > 0 ? max(i.pos0[g] + t[g].rows, 0) : 0;       // keys [0, end) may be seen
          if (end > 0) {
            t[g].sink_tiles = (min(a.num_sink, end) + kTileRows - 1) / kTileRows;
            if (a.window > 0) {
              t[g].lo = max(0, max(i.pos0[g], 0) + 1 - a.window) / kTileRows;
              t[g].hi = (end + kTileRows - 1) / kTileRows;
              lo = min(lo, t[g].lo);
              hi = max(hi, t[g].hi);
            }
            sinks = max(sinks, t[g].sink_tiles);
          }
          if (t[g].rows > 0 && !t[g].any()) zero |= kStepZero << (4 * g);
          if (++head == a.group) { head = 0; ++rb; }
        }
        const int win_lo = lo;                             // first key tile that holds keys of a window
        lo = max(hi > 0 ? lo : 0, sinks);                  // the pair's key tiles: [0, sinks), then [lo, hi)
        const int tiles = sinks + max(hi - lo, 0);
        if (tiles == 0 && zero != 0u) {
          i.flags = kStepEmpty | zero;
          i.j0 = 0;
          describe(i);
        }
        for (int u = 0; ok && u < tiles; ++u) {
          const int kt = u < sinks ? u : lo + (u - sinks);
          i.j0 = kt * kTileRows;
          // a tile below the window holds sinks only: the rest of its keys need no products
          const int keys = kt >= win_lo ? kTileRows : min(a.num_sink - i.j0, kTileRows);
          i.flags = (uint32_t)((keys + 15) >> 4) << kStepGroups | (u == 0 ? zero : 0u);
#pragma unroll
          for (int g = 0; g < 2; ++g)
            if (t[g].needs(kt))
              i.flags |= (kStepNeeds | (kt == t[g].first() ? kStepFirst : 0u) | (kt == t[g].last() ? kStepLast : 0u)) << (4 * g);
          describe(i);
          if (ok) load(&map_k, i.j0, h, b);
          if (u == 0) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              if (!t[g].any() || !wait(q_empty(g), (q_it[g] & 1u) ^ 1u)) continue;
              mbar_arrive_expect_tx(q_full(g), kSlotBytes);
              const uint32_t dst = base + kWinQ + g * kSlotBytes;
              tma_load_4d(dst, &map_q, q_full(g), 0, i.row0[g], i.head[g], b, pol);
              tma_load_4d(dst + kHalfBytes, &map_q, q_full(g), 64, i.row0[g], i.head[g], b, pol);
              ++q_it[g];
            }
          }
          if (ok) load(&map_v, i.j0, h, b);
        }
        pair -= skip_pairs;
        p += skip_p;
        if (p >= per) { p -= per; --pair; }
      }
      if (ok) {
        StepInfo i = {};
        i.flags = kStepStop;
        describe(i);
      }
      if (!ok) {                                           // let what was issued land before the CTA ends
        auto land = [&](uint32_t bar, uint32_t parity) {
          const unsigned long long t0 = global_ns();
          while (!mbar_try_wait(bar, parity) && global_ns() - t0 < a.wait_ns) {}
        };
        const uint32_t pending = it < (uint32_t)kWinRing ? it : (uint32_t)kWinRing;
        for (uint32_t k = it - pending; k < it; ++k) land(full_bar(k % kWinRing), (k / kWinRing) & 1u);
#pragma unroll
        for (int g = 0; g < 2; ++g)
          if (q_it[g] > 0) land(q_full(g), (q_it[g] - 1) & 1u);
      }
    }
  } else if (warp == kWinSoftmaxWarps) {
    // ------------------------------------------------------------ products
    // The whole warp walks the steps and waits; one elected lane issues.
    constexpr uint32_t idesc_pv = instr_desc_pv();
    constexpr uint32_t kSlotUnits = kSlotBytes >> 4;
    const uint64_t q_desc = smem_desc_sw128(base + kWinQ);
    const uint64_t k_desc0 = smem_desc_sw128(base + kWinSlot0), v_desc0 = smem_desc_mn_sw128(base + kWinSlot0);
    uint32_t step = 0;                                     // steps described
    uint32_t q_phase = 0, p_phase = 0, o_phase = 3;        // a bit per query tile
    uint32_t ring_phase = 0;                               // a bit per ring slot
    bool ok = true;                                        // the lanes agree on it at the end of each step
    auto wait = [&](uint32_t bar, uint32_t parity) { ok = mbar_wait(bar, parity, abort_flag, a.status, a.wait_ns) && ok; };
    auto next_step = [&]() {                               // the flags of the step after this one
      const uint32_t e = step % kWinInfoRing;
      wait(info_full(e), (step / kWinInfoRing) & 1u);
      const uint32_t f = info[3 * e].x;
      __syncwarp();
      if (elect_one()) mbar_arrive(info_empty(e));
      ++step;
      return f;
    };
    auto landed = [&](uint32_t slot) { wait(full_bar(slot), (ring_phase >> slot) & 1u); ring_phase ^= 1u << slot; };
    auto release = [&](uint32_t slot) {
      if (elect_one()) tc_commit(empty_bar(slot));
      __syncwarp();
    };
    auto real = [](uint32_t flags) { return !(flags & (kStepStop | kStepEmpty)); };
    // One copy of the code of either product, in a rolled loop: unrolled over tiles and slots it fell out of
    // the instruction cache, and a product took 100 cycles to issue instead of 64.
    // What the loop needs besides products -- the flags of the step after the next, tiles that have to have
    // landed -- is asked for between the batches of products, a little at a time: the pipe has work for
    // the next two or three hundred cycles then.
    uint32_t f = kStepEmpty, fn = next_step();             // this step's flags, the next one's
    uint32_t parity = 0;                                   // K and V of this step are in slots 2 parity, 2 parity + 1
#pragma unroll 1
    while ((ok = __all_sync(0xffffffffu, ok)) && !(f & kStepStop)) {
      const bool now = real(f), then = real(fn);
      const uint32_t v_slot = 2 * parity + 1, k_slot = now ? 2 - 2 * parity : 2 * parity;
      const uint64_t vd = v_desc0 + v_slot * kSlotUnits, kd = k_desc0 + k_slot * kSlotUnits;
      uint32_t f2 = fn;
#pragma unroll 1
      for (int g = 0; g < 2; ++g) {
        const uint32_t t = f >> (4 * g), tn = fn >> (4 * g);
        // O_g (+)= P_g V: 16 keys per product, 8 columns of P, 2048 bytes (128 units) of V
        if (now && (t & kStepNeeds)) {
          const int groups = (int)((f >> kStepGroups) & 15u);
          const uint32_t o_tmem = tmem_base + 256u + g * 128u, p_tmem = tmem_base + g * 128u;
          if (t & kStepFirst) {
            wait(o_empty(g), (o_phase >> g) & 1u);
            o_phase ^= 1u << g;
          }
          wait(p_ready(g, 0), (p_phase >> g) & 1u);
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (k < groups) tc_mma_bf16_ts(o_tmem, p_tmem + 8u * k, vd + 128u * k, idesc_pv, (k > 0 || !(t & kStepFirst)) ? 1u : 0u);
          }
          __syncwarp();
          wait(p_ready(g, 1), (p_phase >> g) & 1u);
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = 4; k < 8; ++k)
              if (k < groups) tc_mma_bf16_ts(o_tmem, p_tmem + 8u * k, vd + 128u * k, idesc_pv, 1u);
            if (t & kStepLast) tc_commit(o_full(g));
          }
          __syncwarp();
          p_phase ^= 1u << g;
        }
        if (now && g == 1) release(v_slot);
        if (then && g == 0) landed(k_slot);
        // S_g = Q_g K^T of the next step, over the keys that matter
        if (then && (tn & kStepNeeds)) {
          if (tn & kStepFirst) {
            wait(q_full(g), (q_phase >> g) & 1u);
            q_phase ^= 1u << g;
          }
          tc_fence_after();
          const uint64_t qd = q_desc + g * kSlotUnits;
          const uint32_t idesc = instr_desc_bf16(16 * (int)((fn >> kStepGroups) & 15u));
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const uint32_t off = (uint32_t)(k >> 2) * (kHalfBytes >> 4) + (uint32_t)(k & 3) * 2u;
              tc_mma_bf16(tmem_base + g * 128u, qd + off, kd + off, idesc, k > 0);
            }
            tc_commit(s_full(g));
            if (tn & kStepLast) tc_commit(q_empty(g));
          }
          __syncwarp();
        }
        if (g == 0 && !(fn & kStepStop)) f2 = next_step();
      }
      if (then) {
        release(k_slot);
        landed(k_slot + 1);
      }
      if (now) parity ^= 1u;
      f = fn;
      fn = f2;
    }
    if (!ok) {
      if (elect_one()) tc_commit(drain_bar);
      __syncwarp();
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(drain_bar, 0) && global_ns() - t0 < a.wait_ns) {}
    }
  } else {
    // ------------------------------------------------------------ softmax and output
    const int g = warp >> 2;                               // the query tile this warp works for
    const int quarter = warp & 3;
    const int r = quarter * 32 + lane;                     // query row of the tile = TMEM lane
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + g * 128u, o_addr = lane_addr + 256u + g * 128u;
    const float sc = a.scale_log2;
    const uint64_t sc2 = pack2(sc, sc);
    uint32_t step = 0, tiles = 0;                          // steps seen; key tiles passed
    uint32_t s_phase = 0, o_phase = 0;
    float top = -INFINITY, sum = 0.f;
    for (;; ++step) {
      const uint32_t e = step % kWinInfoRing;
      if (!warp_wait(info_full(e), (step / kWinInfoRing) & 1u, abort_flag, a.status, a.wait_ns)) break;
      const uint4 i0 = info[3 * e], i1 = info[3 * e + 1], i2 = info[3 * e + 2];
      __syncwarp();
      if (elect_one()) mbar_arrive(info_empty(e));
      const uint32_t flags = i0.x >> (4 * g);
      if (i0.x & kStepStop) break;
      const uint32_t v_at = 2 * tiles + 1;                 // ring entry of this tile's V
      if (!(i0.x & kStepEmpty)) ++tiles;
      if (!(flags & (kStepNeeds | kStepZero))) continue;
      const int j0 = (int)i0.y, n = (int)i0.z;
      const int pos0 = (int)(g == 0 ? i2.x : i2.y), rows = (int)(g == 0 ? i2.z : i2.w);
      const int pos = pos0 + r, pos_lo = pos0 + quarter * 32;              // this row; the warp's first
      if (flags & (kStepFirst | kStepZero)) {
        top = -INFINITY;
        sum = 0.f;
      }
      if (flags & kStepNeeds) {
        // Value rows that no query of the sequence sees -- behind its end, or older than its first query's
        // window and no sinks -- are cleared: a weight of zero would not stop a NaN.
        const int first_pos = pos0 - (int)(g == 0 ? i1.z : i1.w);
        const int old = a.window > 0 ? min(n, max(first_pos + 1 - a.window, 0)) : n;       // keys [num_sink, old)
        const int used = 16 * (int)((i0.x >> kStepGroups) & 15u);            // rows of the tile that are multiplied
        if (j0 + used > n || (j0 < old && j0 + used > a.num_sink)) {
          const uint32_t slot = v_at % kWinRing;
          if (!warp_wait(full_bar(slot), (v_at / kWinRing) & 1u, abort_flag, a.status, a.wait_ns)) break;
          unsigned char* v = base_ptr + kWinSlot0 + slot * kSlotBytes;
          for (int x = r; x < used * 16; x += kTileRows) {
            const int row = x >> 4, c = x & 15, key = j0 + row;
            if (key >= n || (key >= a.num_sink && key < old))
              *reinterpret_cast<uint4*>(v + (c >> 3) * kHalfBytes + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (!warp_wait(s_full(g), s_phase, abort_flag, a.status, a.wait_ns)) break;
        s_phase ^= 1u;
        tc_fence_after();
        // What the warp's 32 rows see of each 32 keys: all, none, or some.  Tiles seen whole (most) run
        // without a branch.
        auto all_seen = [&](int k, int keys) {
          return k + keys - 1 <= pos_lo && (k > pos_lo + 31 - a.window || k + keys <= a.num_sink);
        };
        auto none_seen = [&](int k) {
          return k > pos_lo + 31 || (k >= a.num_sink && k + 31 <= pos_lo - a.window);
        };
        const bool whole = all_seen(j0, kTileRows);
        float v[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + 32 * c, *reinterpret_cast<float(*)[32]>(v + 32 * c));
        tmem_ld_wait();
        if (!whole) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int k = j0 + 32 * c;
            if (all_seen(k, 32)) continue;
            // columns [lo, hi) are in the window, those below sk are sinks
            auto below = [](int x) { return x >= 32 ? 0xffffffffu : (x <= 0 ? 0u : (1u << x) - 1u); };
            const uint32_t see = below(pos + 1 - k) & (~below(pos + 1 - a.window - k) | below(a.num_sink - k));
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(see & (1u << e))) v[32 * c + e] = -INFINITY;
          }
        }
        float ext[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int e = 4; e < 124; e += 8)
#pragma unroll
          for (int j = 0; j < 4; ++j) ext[j] = max3(ext[j], v[e + 2 * j], v[e + 2 * j + 1]);
#pragma unroll
        for (int j = 0; j < 4; ++j) ext[j] = fmaxf(ext[j], v[124 + j]);
        const float mx = fmaxf(fmaxf(ext[0], ext[1]), fmaxf(ext[2], ext[3]));
        const float tile_top = mx * sc;
        const bool move = tile_top > top + kWinSlack || top == -INFINITY;
        if (__any_sync(0xffffffffu, move)) {
          const float new_top = move ? fmaxf(top, tile_top) : top;
          if (!(flags & kStepFirst)) {                     // rescale (the previous product has retired)
            const float alpha = !move || new_top == -INFINITY ? 1.f : fast_exp2(top - new_top);
            sum *= alpha;
#pragma unroll 1
            for (int c0 = 0; c0 < 128; c0 += 16) {
              uint32_t o[16];
              tmem_ld16(o_addr + c0, o);
              tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha);
              tmem_st16(o_addr + c0, o);
            }
            tmem_st_wait();
          }
          top = new_top;
        }
        const float ref = top == -INFINITY ? 0.f : top;
        const uint64_t nref2 = pack2(-ref, -ref);
        uint64_t part[2] = {0ull, 0ull};
        auto weights = [&](int c) {
          uint32_t h[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x0, x1;
            unpack2(fma2(pack2(v[32 * c + 2 * e], v[32 * c + 2 * e + 1]), sc2, nref2), x0, x1);
            const float w0 = fast_exp2(x0), w1 = fast_exp2(x1);
            part[e & 1] = add2(part[e & 1], pack2(w0, w1));
            h[e] = token::pack_bf16(w0, w1);
          }
          tmem_st16(s_addr + 16 * c, h);
        };
        auto hand_over = [&](int half) {                   // 64 keys' weights are in place
          tmem_st_wait();
          tc_fence_before();
          mbar_arrive(p_ready(g, half));
        };
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if (!whole && none_seen(j0 + 32 * c)) {
            uint32_t h[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) h[e] = 0u;
            tmem_st16(s_addr + 16 * c, h);
          } else {
            weights(c);
          }
          if (c & 1) hand_over(c >> 1);
        }
        float p0, p1;
        unpack2(add2(part[0], part[1]), p0, p1);
        sum += p0 + p1;
        if (!(flags & kStepLast)) continue;
        if (!warp_wait(o_full(g), o_phase, abort_flag, a.status, a.wait_ns)) break;
        o_phase ^= 1u;
        tc_fence_after();
      }
      // ---- output of this tile
      {
        const bool any = flags & kStepNeeds;
        const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);    // a NaN sum stays one
        const int b = (int)i0.w, hq = (int)(g == 0 ? i1.x : i1.y), row0 = (int)(g == 0 ? i1.z : i1.w);
        __nv_bfloat16* out = a.O + b * a.o_sb + hq * a.o_sh + (int64_t)(row0 + quarter * 32) * a.o_sn;
        unsigned char* stage = base_ptr + kWinStage + warp * 4096;           // 32 rows of 128 bytes
        const int live = rows - quarter * 32;
        float o[128];
        if (any) {
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32(o_addr + 32 * c, *reinterpret_cast<float(*)[32]>(o + 32 * c));
          tmem_ld_wait();
          tc_fence_before();
          mbar_arrive(o_empty(g));                         // the next item's products may begin
        } else {
#pragma unroll
          for (int c = 0; c < 128; ++c) o[c] = 0.f;
        }
        // Rows go through shared memory, so that eight lanes write 128 bytes of one row side by side
        // (16-byte stores to 32 different rows took 8000 cycles a tile); a row's eight places are permuted
        // against bank conflicts.
#pragma unroll
        for (int c0 = 0; c0 < 128; c0 += 64) {
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const float* x = o + c0 + 8 * c;
            *reinterpret_cast<uint4*>(stage + lane * 128 + (c ^ (lane & 7)) * 16) =
                make_uint4(token::pack_bf16(x[0] * inv, x[1] * inv), token::pack_bf16(x[2] * inv, x[3] * inv),
                           token::pack_bf16(x[4] * inv, x[5] * inv), token::pack_bf16(x[6] * inv, x[7] * inv));
          }
          __syncwarp();
          const int c = lane & 7;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int row = 4 * k + (lane >> 3);
            const uint4 x = *reinterpret_cast<const uint4*>(stage + row * 128 + (c ^ (row & 7)) * 16);
            if (row < live) *reinterpret_cast<uint4*>(out + (int64_t)row * a.o_sn + c0 + 8 * c) = x;
          }
          __syncwarp();
        }
        if (r < rows && a.lse != nullptr)
          a.lse[((int64_t)b * a.heads * a.group + hq) * a.q_rows + row0 + r] =
              sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kWinSoftmaxWarps) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)kWinTmemCols)
                 : "memory");
  }
}

}  // namespace umma
}  // namespace curdkv
