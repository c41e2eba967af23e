// Causal attention with a sliding window and sinks for prompts (many query rows per head):
// O = softmax(scale Q K^T) V over the keys j <= pos with j > pos - window or j < num_sink.
//
// Persistent CTAs, one per SM.  A work item is a pair of query tiles (128 rows of one query head each)
// of the same KV head, so that both read the same tiles of K and V: tiles are numbered row block
// major, query head of the group minor, and tiles 2 i and 2 i + 1 make a pair -- two heads at the
// same rows for even groups, neighbouring row blocks for a group of one.  Only the key tiles that some
// row of the pair sees are walked: those holding sinks, then those of the window.
//
// Ten warps.  Two groups of four softmax warps own one query tile each (a thread per row): S = Q K^T
// arrives in TMEM, the thread keeps its row of 128 logits in registers, the weights go back over S as
// bf16 and are the A operand of O += P V straight from TMEM.  One thread issues all products in the
// order  P_A V, S_A', P_B V, S_B'  (S' the next key tile's), so that while one group turns logits
// into weights the tensor pipe works for the other; P is handed over in halves, so that P V starts
// on the first 64 keys.  One thread feeds Q and the ring of K and V tiles by TMA.  Items follow each
// other without a gap: the next pair's first S is issued right behind the last product of this one,
// and a group writes its O while that runs.
//
// What bounds it: 128 x 128 keys cost the tensor pipe 1024 cycles (two products of 512) and the
// exponentials of the tile 1024 cycles of the special function units, so every kPolyEvery-th pair of
// weights is formed on the FMA pipe instead (a minimax polynomial of degree 4).
//
// The running maximum moves only when a tile exceeds it by more than 2^8 (as in attn_umma.cuh); the
// group then rescales its accumulator in TMEM, which after the first tiles is rare.  Value rows at or
// beyond the sequence's end are cleared in shared memory by the softmax threads (a zero weight would
// not stop a NaN).  All waits are bounded.
#pragma once
#include <type_traits>

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
  unsigned long long wait_ns = kWaitLimitNs;
};

constexpr int kWinThreads = 320;
constexpr int kWinRing = 5;
constexpr int kWinQ = 0;                                   // Q of the two tiles
constexpr int kWinSlot0 = 2 * kSlotBytes;
constexpr int kWinBar = kWinSlot0 + kWinRing * kSlotBytes;
constexpr int kWinDynamic = kWinBar + 256 + 1024;
constexpr int kWinTmemCols = 512;                          // S_A, S_B, O_A, O_B
constexpr float kWinSlack = 8.f;

// One query tile of an item: which rows, and which key tiles it needs.
struct WinTile {
  int rb, head;                      // row block, query head within the group
  int rows;                          // query rows that exist (0: none)
  int pos0;                          // position of its first row
  int sink_tiles, lo, hi;            // key tiles [0, sink_tiles) and [lo, hi)
  __device__ __forceinline__ bool needs(int kt) const { return kt < sink_tiles || (kt >= lo && kt < hi); }
  __device__ __forceinline__ bool any() const { return sink_tiles > 0 || hi > lo; }
  __device__ __forceinline__ int first() const { return sink_tiles > 0 ? 0 : lo; }
  __device__ __forceinline__ int last() const { return max(sink_tiles, hi > lo ? hi : 0) - 1; }
};

struct WinItem {
  int b, h, n, q;                    // sequence, KV head, cached rows, query tokens
  WinTile t[2];
  int sinks, lo, hi, tiles;          // key tiles of the pair: [0, sinks), then [lo, hi)
  __device__ __forceinline__ int key_tile(int u) const { return u < sinks ? u : lo + (u - sinks); }
};

__device__ __forceinline__ WinItem win_item(const WindowArgs& a, int item) {
  WinItem w;
  // longest rows first: the row block falls from the last pair on, heads and sequences vary fastest
  const int per = a.batch * a.heads;
  const int pair = a.pairs - 1 - item / per, p = item % per;
  w.b = p / a.heads;
  w.h = p % a.heads;
  w.n = seq_len_of(a.seqlens, w.b, a.n_max);
  w.q = a.q_lens != nullptr ? min(max(a.q_lens[w.b], 0), a.q_rows) : a.q_rows;
  w.sinks = 0;
  w.lo = 0x7fffffff;
  w.hi = 0;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    WinTile& t = w.t[g];
    const int tau = 2 * pair + g;
    t.rb = tau / a.group;
    t.head = tau % a.group;
    t.rows = min(max(w.q - t.rb * kTileRows, 0), kTileRows);
    t.pos0 = w.n - w.q + t.rb * kTileRows;
    t.sink_tiles = t.lo = t.hi = 0;
    const int end = t.rows > 0 ? max(t.pos0 + t.rows, 0) : 0;          // keys [0, end) may be seen
    if (end > 0) {
      const int first = (int)max((int64_t)0, (int64_t)max(t.pos0, 0) + 1 - a.window);   // window's first key
      t.sink_tiles = (min(a.num_sink, end) + kTileRows - 1) / kTileRows;
      if (a.window > 0) {
        t.lo = first / kTileRows;
        t.hi = (end + kTileRows - 1) / kTileRows;
        w.lo = min(w.lo, t.lo);
        w.hi = max(w.hi, t.hi);
      }
      w.sinks = max(w.sinks, t.sink_tiles);
    }
  }
  if (w.hi == 0) w.lo = 0;
  w.lo = max(w.lo, w.sinks);                               // the runs do not overlap
  w.hi = max(w.hi, w.lo);
  w.tiles = w.sinks + w.hi - w.lo;
  return w;
}

// 2^x for x <= 0 on the FMA pipe: x = i + f, |f| <= 1/2, 2^f by the polynomial of degree 4 with the
// least greatest relative error there (Remez exchange: 2.6e-6), and i added to the exponent.
__device__ __forceinline__ uint64_t exp2_poly2(uint64_t x2) {
  float x0, x1;
  unpack2(x2, x0, x1);
  const uint64_t x = pack2(fmaxf(x0, -126.f), fmaxf(x1, -126.f));
  const uint64_t magic = pack2(12582912.f, 12582912.f);   // 1.5 * 2^23: adding it rounds to an integer
  const uint64_t r = add2(x, magic);
  const uint64_t f = sub2(x, sub2(r, magic));
  uint64_t p = fma2(pack2(0x1.3997d6p-7f, 0x1.3997d6p-7f), f, pack2(0x1.ca1440p-5f, 0x1.ca1440p-5f));
  p = fma2(p, f, pack2(0x1.ec06dap-3f, 0x1.ec06dap-3f));
  p = fma2(p, f, pack2(0x1.62e0dcp-1f, 0x1.62e0dcp-1f));
  p = fma2(p, f, pack2(0x1.ffffe8p-1f, 0x1.ffffe8p-1f));
  float p0, p1, r0, r1;
  unpack2(p, p0, p1);
  unpack2(r, r0, r1);
  return pack2(__int_as_float(__float_as_int(p0) + (__float_as_int(r0) << 23)),
               __int_as_float(__float_as_int(p1) + (__float_as_int(r1) << 23)));
}

constexpr int kPolyEvery = 4;        // every 4th pair of weights by polynomial

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
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(base_ptr + kWinBar + 8 * (2 * kWinRing + 15));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int s = 0; s < kWinRing; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
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
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                 "r"((uint32_t)kWinTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_holder;

  if (warp == 9) {
    // ------------------------------------------------------------ TMA producer
    // Ring order of an item: K_0, V_0, K_1, V_1, ...; its two Q tiles follow K_0.
    if (lane == 0) {
      uint64_t pol;
      asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
      uint32_t it = 0, q_it[2] = {0, 0};
      bool ok = true;
      auto load = [&](const CUtensorMap* map, int kt, const WinItem& w) {
        const uint32_t slot = it % kWinRing;
        if (!(ok = mbar_wait(empty_bar(slot), ((it / kWinRing) & 1u) ^ 1u, abort_flag, a.status, a.wait_ns))) return;
        mbar_arrive_expect_tx(full_bar(slot), kSlotBytes);
        const uint32_t dst = base + kWinSlot0 + slot * kSlotBytes;
        tma_load_4d(dst, map, full_bar(slot), 0, kt * kTileRows, w.h, w.b, pol);
        tma_load_4d(dst + kHalfBytes, map, full_bar(slot), 64, kt * kTileRows, w.h, w.b, pol);
        ++it;
      };
      for (int item = blockIdx.x; ok && item < a.items; item += gridDim.x) {
        const WinItem w = win_item(a, item);
        for (int u = 0; ok && u < w.tiles; ++u) {
          load(&map_k, w.key_tile(u), w);
          if (u == 0) {
            for (int g = 0; ok && g < 2; ++g) {
              if (!w.t[g].any()) continue;           // nothing to multiply
              if (!(ok = mbar_wait(q_empty(g), (q_it[g] & 1u) ^ 1u, abort_flag, a.status, a.wait_ns))) break;
              mbar_arrive_expect_tx(q_full(g), kSlotBytes);
              const uint32_t dst = base + kWinQ + g * kSlotBytes;
              const int hq = w.h * a.group + w.t[g].head;
              tma_load_4d(dst, &map_q, q_full(g), 0, w.t[g].rb * kTileRows, hq, w.b, pol);
              tma_load_4d(dst + kHalfBytes, &map_q, q_full(g), 64, w.t[g].rb * kTileRows, hq, w.b, pol);
              ++q_it[g];
            }
          }
          if (ok) load(&map_v, w.key_tile(u), w);
        }
      }
      if (!ok) {                                           // let what was issued land before the CTA ends
        auto land = [&](uint32_t bar, uint32_t parity) {
          const unsigned long long t0 = global_ns();
          while (!mbar_try_wait(bar, parity) && global_ns() - t0 < a.wait_ns) {}
        };
        const uint32_t pending = it < (uint32_t)kWinRing ? it : (uint32_t)kWinRing;
        for (uint32_t q = it - pending; q < it; ++q) land(full_bar(q % kWinRing), (q / kWinRing) & 1u);
        for (int g = 0; g < 2; ++g)
          if (q_it[g] > 0) land(q_full(g), (q_it[g] - 1) & 1u);
      }
    }
  } else if (warp == 8) {
    // ------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      constexpr uint32_t idesc_s = instr_desc_bf16(128);
      constexpr uint32_t idesc_pv = instr_desc_pv();
      uint32_t q_it[2] = {0, 0}, p_it[2] = {0, 0}, o_it[2] = {0, 0};
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        ok = ok && mbar_wait(bar, parity, abort_flag, a.status, a.wait_ns);
        return ok;
      };
      // One step is one key tile of one item; steps follow each other across items.
      struct Step {
        WinItem w;
        int item, u;
        uint32_t it;                                       // ring position of this step's K tile (V follows)
      };
      auto settle = [&](Step& s) {                         // the first item from s.item on that has key tiles
        while (s.item < a.items) {
          s.w = win_item(a, s.item);
          if (s.w.tiles > 0) break;
          s.item += gridDim.x;
        }
        s.u = 0;
      };
      // S_g = Q_g K^T of a step, if the step is one of tile g's
      auto issue_s = [&](const Step& s, int g) {
        const WinTile& t = s.w.t[g];
        const int kt = s.w.key_tile(s.u);
        const uint32_t slot = s.it % kWinRing;
        if (!wait(full_bar(slot), (s.it / kWinRing) & 1u) || !t.needs(kt)) return;
        if (kt == t.first() && !wait(q_full(g), q_it[g]++ & 1u)) return;
        tc_fence_after();
        const uint64_t q_desc = smem_desc_sw128(base + kWinQ + g * kSlotBytes);
        const uint64_t k_desc = smem_desc_sw128(base + kWinSlot0 + slot * kSlotBytes);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t off = (uint32_t)(k >> 2) * (kHalfBytes >> 4) + (uint32_t)(k & 3) * 2u;
          tc_mma_bf16(tmem_base + g * 128u, q_desc + off, k_desc + off, idesc_s, k > 0);
        }
        tc_commit(s_full(g));
        if (kt == t.last()) tc_commit(q_empty(g));
      };
      // O_g (+)= P_g V of a step
      auto issue_pv = [&](const Step& s, int g) {
        const WinTile& t = s.w.t[g];
        const int kt = s.w.key_tile(s.u);
        const uint32_t at = s.it + 1, slot = at % kWinRing;
        const bool first = kt == t.first();
        if (!wait(full_bar(slot), (at / kWinRing) & 1u) || !t.needs(kt)) return;
        if (first && !wait(o_empty(g), (o_it[g]++ & 1u) ^ 1u)) return;
        const uint64_t v_desc = smem_desc_mn_sw128(base + kWinSlot0 + slot * kSlotBytes);
        const uint32_t o_tmem = tmem_base + 256u + g * 128u, p_tmem = tmem_base + g * 128u;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!wait(p_ready(g, half), p_it[g] & 1u)) return;
          tc_fence_after();
#pragma unroll
          for (int k = 4 * half; k < 4 * half + 4; ++k)    // 16 keys: 8 columns of P, 2048 bytes of V
            tc_mma_bf16_ts(o_tmem, p_tmem + 8u * k, v_desc + 128u * k, idesc_pv, (!first || k > 0) ? 1u : 0u);
        }
        ++p_it[g];
        if (kt == t.last()) tc_commit(o_full(g));
      };
      Step now, next;
      next.item = blockIdx.x;
      next.it = 0;
      settle(next);
      if (next.item < a.items) {
        issue_s(next, 0);
        if (ok) issue_s(next, 1);
        if (ok) tc_commit(empty_bar(next.it % kWinRing));
      }
      while (ok && next.item < a.items) {
        now = next;
        next.it += 2;
        if (++next.u == next.w.tiles) {
          next.item += gridDim.x;
          settle(next);
        }
        const bool more = next.item < a.items;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (ok) issue_pv(now, g);
          if (g == 1 && ok) tc_commit(empty_bar((now.it + 1) % kWinRing));       // V of this step
          if (ok && more) issue_s(next, g);
        }
        if (ok && more) tc_commit(empty_bar(next.it % kWinRing));                // K of the next
      }
      if (!ok) {
        tc_commit(drain_bar);
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(drain_bar, 0) && global_ns() - t0 < a.wait_ns) {}
      }
    }
  } else {
    // ------------------------------------------------------------ softmax and output
    const int g = warp >> 2;                               // the query tile this warp works for
    const int quarter = warp & 3;
    const int r = quarter * 32 + lane;                     // query row of the tile = TMEM lane
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + g * 128u, o_addr = lane_addr + 256u + g * 128u;
    const float sc = a.scale_log2;
    uint32_t it = 0, s_it = 0, o_it = 0;
    bool ok = true;
    for (int item = blockIdx.x; ok && item < a.items; item += gridDim.x) {
      const WinItem w = win_item(a, item);
      const WinTile t = g == 0 ? w.t[0] : w.t[1];
      const int pos = t.pos0 + r;
      float top = -INFINITY, sum = 0.f;
      for (int u = 0; ok && u < w.tiles; ++u) {
        const int kt = w.key_tile(u), j0 = kt * kTileRows;
        if (!t.needs(kt)) continue;
        if (j0 + kTileRows > w.n) {                        // value rows behind the sequence: cleared
          const uint32_t at = it + 2 * u + 1, slot = at % kWinRing;
          if (!(ok = warp_wait(full_bar(slot), (at / kWinRing) & 1u, abort_flag, a.status, a.wait_ns))) break;
          unsigned char* v = base_ptr + kWinSlot0 + slot * kSlotBytes;
          const int dead = kTileRows - max(w.n - j0, 0), from = kTileRows - dead;
          for (int e = r; e < dead * 16; e += kTileRows) {
            const int row = from + (e >> 4), c = e & 15;
            *reinterpret_cast<uint4*>(v + (c >> 3) * kHalfBytes + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (!(ok = warp_wait(s_full(g), s_it & 1u, abort_flag, a.status, a.wait_ns))) break;
        ++s_it;
        tc_fence_after();
        float v[128];
#pragma unroll
        for (int c0 = 0; c0 < 128; c0 += 32) tmem_ld32(s_addr + c0, *reinterpret_cast<float(*)[32]>(v + c0));
        tmem_ld_wait();
        // a tile that every row of the query tile sees whole needs no mask
        const bool whole = j0 + kTileRows - 1 <= t.pos0 &&
                           ((int64_t)j0 > (int64_t)t.pos0 + kTileRows - 1 - a.window || j0 + kTileRows <= a.num_sink);
        if (!whole) {
          // columns [lo, hi) are in the window, those below sk are sinks
          const int hi = min(max(pos + 1 - j0, 0), 128);
          const int lo = (int)min(max((int64_t)pos + 1 - a.window - j0, (int64_t)0), (int64_t)128);
          const int sk = min(max(a.num_sink - j0, 0), 128);
#pragma unroll
          for (int c0 = 0; c0 < 128; c0 += 32) {
            auto below = [&](int x) { return x >= c0 + 32 ? 0xffffffffu : (x <= c0 ? 0u : (1u << (x - c0)) - 1u); };
            const uint32_t see = below(hi) & (~below(lo) | below(sk));
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!((see >> c) & 1u)) v[c0 + c] = -INFINITY;
          }
        }
        float ext[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int c = 4; c < 124; c += 8)
#pragma unroll
          for (int j = 0; j < 4; ++j) ext[j] = max3(ext[j], v[c + 2 * j], v[c + 2 * j + 1]);
#pragma unroll
        for (int j = 0; j < 4; ++j) ext[j] = fmaxf(ext[j], v[124 + j]);
        const float tile_top = fmaxf(fmaxf(ext[0], ext[1]), fmaxf(ext[2], ext[3])) * sc;
        const bool move = tile_top > top + kWinSlack || top == -INFINITY;
        const float new_top = move ? fmaxf(top, tile_top) : top;
        if (kt != t.first() && __any_sync(0xffffffffu, move)) {      // (the previous product has retired)
          const float alpha = !move || new_top == -INFINITY ? 1.f : fast_exp2(top - new_top);
          sum *= alpha;
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 32) {
            float o[32];
            tmem_ld32(o_addr + c0, o);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] *= alpha;
            tmem_st32(o_addr + c0, o);
          }
          tmem_st_wait();
        }
        top = new_top;
        const float ref = top == -INFINITY ? 0.f : top;
        const uint64_t sc2 = pack2(sc, sc), nref2 = pack2(-ref, -ref);
        uint64_t part[4] = {0ull, 0ull, 0ull, 0ull};
        // (a masked logit has to give exactly 0, which the polynomial does not: special function units
        // alone for the few tiles with a mask)
        auto weights = [&](auto poly) {
#pragma unroll
          for (int c0 = 0; c0 < 128; c0 += 32) {
            uint32_t h[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint64_t x2 = fma2(pack2(v[c0 + 2 * e], v[c0 + 2 * e + 1]), sc2, nref2);
              uint64_t w2;
              if (poly.value && e % kPolyEvery == kPolyEvery - 1) {
                w2 = exp2_poly2(x2);
              } else {
                float x0, x1;
                unpack2(x2, x0, x1);
                w2 = pack2(fast_exp2(x0), fast_exp2(x1));
              }
              part[e & 3] = add2(part[e & 3], w2);
              float w0, w1;
              unpack2(w2, w0, w1);
              const __nv_bfloat162 b2 = __floats2bfloat162_rn(w0, w1);
              h[e] = *reinterpret_cast<const uint32_t*>(&b2);
            }
            tmem_st16(s_addr + (uint32_t)c0 / 2, h);
            if (c0 == 32 || c0 == 96) {                    // 64 keys' weights are in place
              tmem_st_wait();
              tc_fence_before();
              mbar_arrive(p_ready(g, c0 == 96));
            }
          }
        };
        if (whole) weights(std::true_type{});
        else weights(std::false_type{});
        float p0, p1;
        unpack2(add2(add2(part[0], part[1]), add2(part[2], part[3])), p0, p1);
        sum += p0 + p1;
      }
      it += 2 * w.tiles;
      // ---- output of this tile
      const bool any = t.any();
      if (any && ok) {
        ok = warp_wait(o_full(g), o_it & 1u, abort_flag, a.status, a.wait_ns);
        ++o_it;
        tc_fence_after();
      }
      if (ok) {
        const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);    // a NaN sum stays one
        const int hq = w.h * a.group + t.head;
        const int64_t row = (int64_t)t.rb * kTileRows + r;
        __nv_bfloat16* out = a.O + w.b * a.o_sb + hq * a.o_sh + row * a.o_sn;
#pragma unroll 1
        for (int c0 = 0; c0 < 128; c0 += 32) {
          float o[32];
          if (any) {
            tmem_ld32(o_addr + c0, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = 0.f;
          }
          if (r < t.rows) {
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
              uint4 x;
              x.x = token::pack_bf16(o[c] * inv, o[c + 1] * inv);
              x.y = token::pack_bf16(o[c + 2] * inv, o[c + 3] * inv);
              x.z = token::pack_bf16(o[c + 4] * inv, o[c + 5] * inv);
              x.w = token::pack_bf16(o[c + 6] * inv, o[c + 7] * inv);
              *reinterpret_cast<uint4*>(out + c0 + c) = x;
            }
          }
        }
        if (any) {
          tc_fence_before();
          mbar_arrive(o_empty(g));
        }
        if (r < t.rows && a.lse != nullptr)
          a.lse[((int64_t)w.b * a.heads * a.group + hq) * a.q_rows + row] =
              sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)kWinTmemCols)
                 : "memory");
  }
}

}  // namespace umma
}  // namespace curdkv
