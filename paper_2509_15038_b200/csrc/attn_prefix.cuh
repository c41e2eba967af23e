// Attention of many query rows over a prefix that their sequences share: the rows of all sequences, stacked, against the
// prefix's keys once.  One part (attn_rows.cuh) per CTA: a tile of up to 128 query rows against a run of keys; it leaves
// reference, sum and fp32 sums of values for the joining kernel.
//
// A tile is `seqs` sequences x `tokens` tokens x the heads of a KV head's group, brought in by one 5-D map, whatever the
// strides.  The walk over the keys is that of attn_umma.cuh and attn_window.cuh: S = Q K_t^T per 128-key tile, a thread per
// query row, the weights back over S in TMEM as bf16, where they are the A operand of O_g += P V_t (handed over in halves).
// Two groups of four softmax warps, each with its own running maximum (moved when a tile exceeds it by more than 2^8), sum and
// accumulator, take alternate key tiles of one tile of rows, or all key tiles of a tile of rows each: a pair then
// reads every tile of K and V once, where a CTA per tile drew twice the bytes through the L2 (193 us against 168 for 256 rows
// over 8 heads of 131072).  Weights are rounded to bf16 (half a step: 2^-8 of each), sums take them unrounded: O is then off by
// 0.18 to 0.21 % (2-norm), 0.16 to 0.18 of it its own rounding.  Two bf16 parts of a weight, as in attn_rows.cuh, leave only that, but the
// second product and the remainders lengthen the chain below: 64 sequences behind 32768 rows 66 -> 79 us, 16 x 8 behind 8192
// 122 -> 140, 64 x 4 query rows behind 131072 177 -> 225.
//
// What bounds it: a single tile of rows the keys' bytes (128 heads of 8192 rows, 32 query rows: 84 us, 6.4 TB/s); a pair the
// chain of a group, 3400 cycles a step: 1870 from logits to weights, then P V of the second half, the next S and the
// wake-ups between; tensor pipe and special function units are busy half of the time.
// Measured and dropped: a product warp per group (81 us against 73 for 64 sequences behind 32768 rows: they fall into step);
// one to three of eight pairs of exponentials on the FMA pipe (no gain); a pair's steps in halves of 64 keys, so that one half
// of S is formed while the group is at the other (156 us against 143 for 512 rows over 8 heads of 131072: products of 64
// columns); the weights handed over in 32 + 96 or 96 + 32 keys (143 to 145).
#pragma once
#include "umma_ptx.cuh"

namespace curdkv {
namespace umma {

struct PrefixArgs {
  const int32_t* lens;               // [sets] or nullptr
  int n_max, heads, group, t, share;
  int seqs, tokens, token_tiles, tiles;                    // of a set: tile = (sequences / seqs) * token_tiles + tokens / tokens
  int chunk, chunks;                 // keys a CTA takes (a multiple of 128), CTAs per tile at most
  float scale_log2;
  float2* part_ml;                   // [sets * heads][tiles][chunks][128]
  float* part_o;                     // [sets * heads][tiles][chunks][128][128]
  uint32_t* status;
  unsigned long long wait_ns = kWaitLimitNs;
};

constexpr int kPrefixThreads = 320;                        // TMA, products, two sets of four softmax warps
constexpr int kPrefixRing = 5;
constexpr int kPrefixQ = 0;                                // one or two tiles
constexpr int kPrefixSlot0 = 2 * kSlotBytes;
constexpr int kPrefixBar = kPrefixSlot0 + kPrefixRing * kSlotBytes;
constexpr int kPrefixDynamic = kPrefixBar + 256 + 1024;
constexpr int kPrefixTmemCols = 512;                       // S of group g at 128 g (its weights over it), O of group g at 256 + 128 g
constexpr float kPrefixSlack = 8.f;

// PAIR: two tiles of query rows, a group of softmax warps each, which share every tile of keys and values; else one tile, whose
// groups take every other tile of keys each and meet at the end.
// grid = sets * heads * chunks * (tiles or pairs of tiles), these innermost: CTAs that read the same keys run side by side.
template <bool PAIR>
__global__ void __launch_bounds__(kPrefixThreads, 1)
prefix_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v, const PrefixArgs a) {
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bar0 = base + kPrefixBar;
  auto full_bar = [&](uint32_t s) { return bar0 + 8u * s; };
  auto empty_bar = [&](uint32_t s) { return bar0 + 8u * (kPrefixRing + s); };
  const uint32_t gbar = bar0 + 16u * kPrefixRing;
  auto s_full_bar = [&](uint32_t g) { return gbar + 8u * g; };
  auto p_ready_bar = [&](uint32_t g, uint32_t half) { return gbar + 16u + 16u * g + 8u * half; };
  auto o_full_bar = [&](uint32_t g) { return gbar + 48u + 8u * g; };
  const uint32_t q_full_bar = gbar + 64u, drain_bar = gbar + 72u;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(base_ptr + kPrefixBar + 16 * kPrefixRing + 80);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const int sets_of_tiles = PAIR ? (a.tiles + 1) / 2 : a.tiles;
  const int tile0 = blockIdx.x % sets_of_tiles * (PAIR ? 2 : 1), chunk = blockIdx.x / sets_of_tiles % a.chunks;
  const int p = blockIdx.x / sets_of_tiles / a.chunks, set = p / a.heads, h = p % a.heads;
  const int count = PAIR ? min(2, a.tiles - tile0) : 1;    // tiles of query rows
  int n = a.n_max;
  if (a.lens != nullptr) {
    n = seq_len_of(a.lens, set, a.n_max);
    if (n != a.lens[set] && tid == 0 && chunk == 0 && tile0 == 0) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
  }
  const int k0 = chunk * a.chunk, keys = min(n - k0, a.chunk);
  if (keys <= 0) return;
  const int T = (keys + kTileRows - 1) / kTileRows;

  if (tid == 0) {
    for (int s = 0; s < kPrefixRing; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int g = 0; g < 2; ++g) {
      mbar_init(s_full_bar(g), 1);
      mbar_init(o_full_bar(g), 1);
      for (int half = 0; half < 2; ++half) mbar_init(p_ready_bar(g, half), 128);
    }
    mbar_init(q_full_bar, 1);
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)),
                 "r"((uint32_t)kPrefixTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  constexpr uint32_t tmem_base = 0u;                       // all 512 columns are this CTA's: they begin at 0

  // Ring order, that of the products: a pair K_0, V_0, K_1, V_1, ...; else K_0, K_1, V_0, K_2, V_1, ...  Every entry is waited
  // for in order by one warp (a barrier tells only two rounds apart).
  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      uint64_t pol;
      asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
      mbar_arrive_expect_tx(q_full_bar, (uint32_t)(count * a.seqs * a.tokens * a.group) * 256u);
      for (int g = 0; g < count; ++g) {
        const int tok0 = (tile0 + g) % a.token_tiles * a.tokens, seq = set * a.share + (tile0 + g) / a.token_tiles * a.seqs;
        const uint32_t dst = base + kPrefixQ + g * kSlotBytes;
        tma_load_5d(dst, &map_q, q_full_bar, 0, 0, tok0, h, seq);
        tma_load_5d(dst + kHalfBytes, &map_q, q_full_bar, 64, 0, tok0, h, seq);
      }
      uint32_t it = 0;
      bool ok = true;
      auto load = [&](const CUtensorMap* map, int t) {
        const uint32_t slot = it % kPrefixRing;
        if (!(ok = ok && mbar_wait(empty_bar(slot), ((it / kPrefixRing) & 1u) ^ 1u, abort_flag, a.status, a.wait_ns))) return;
        mbar_arrive_expect_tx(full_bar(slot), kSlotBytes);
        const uint32_t dst = base + kPrefixSlot0 + slot * kSlotBytes;
        tma_load_4d(dst, map, full_bar(slot), 0, k0 + t * kTileRows, h, set, pol);
        tma_load_4d(dst + kHalfBytes, map, full_bar(slot), 64, k0 + t * kTileRows, h, set, pol);
        ++it;
      };
      constexpr int kAhead = PAIR ? 1 : 2;
      for (int t = 0; t < kAhead && t < T; ++t) load(&map_k, t);
      for (int t = 0; ok && t < T; ++t) {
        load(&map_v, t);
        if (t + kAhead < T) load(&map_k, t + kAhead);
      }
      if (!ok) {                                           // let what was issued land before the CTA ends
        auto land = [&](uint32_t bar, uint32_t parity) {
          const unsigned long long t0 = global_ns();
          while (!mbar_try_wait(bar, parity) && global_ns() - t0 < a.wait_ns) {}
        };
        for (uint32_t q = it - min(it, (uint32_t)kPrefixRing); q < it; ++q) land(full_bar(q % kPrefixRing), (q / kPrefixRing) & 1u);
        land(q_full_bar, 0);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ products: the whole warp waits, one lane issues
    constexpr uint32_t idesc_s = instr_desc_bf16(128), idesc_pv = instr_desc_pv();
    const uint64_t q_desc = smem_desc_sw128(base + kPrefixQ);
    const uint64_t k_desc0 = smem_desc_sw128(base + kPrefixSlot0), v_desc0 = smem_desc_mn_sw128(base + kPrefixSlot0);
    uint32_t it = 0;                                       // entries of the ring that have landed
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, a.status, a.wait_ns) && ok);
      tc_fence_after();
    };
    auto next_slot = [&]() {
      const uint32_t slot = it % kPrefixRing;
      wait(full_bar(slot), (it / kPrefixRing) & 1u);
      ++it;
      return slot;
    };
    auto release = [&](uint32_t slot) {
      if (ok && elect_one()) tc_commit(empty_bar(slot));
      __syncwarp();
    };
    auto issue_s = [&](uint32_t g, uint32_t slot) {        // S_g = Q K^T
      if (ok && elect_one()) {
        const uint64_t qd = q_desc + (PAIR ? g * (kSlotBytes >> 4) : 0u), kd = k_desc0 + slot * (kSlotBytes >> 4);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t off = (uint32_t)(k >> 2) * (kHalfBytes >> 4) + (uint32_t)(k & 3) * 2u;
          tc_mma_bf16(tmem_base + 128u * g, qd + off, kd + off, idesc_s, k > 0);
        }
        tc_commit(s_full_bar(g));
      }
      __syncwarp();
    };
    // O_g += P_g V: 16 keys per product, 8 columns of P, 2048 bytes (128 units) of the V tile; the weights come in halves
    auto issue_pv = [&](uint32_t g, uint32_t slot, int groups, uint32_t parity, bool first) {
      const uint64_t vd = v_desc0 + slot * (kSlotBytes >> 4);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (ok) wait(p_ready_bar(g, half), parity);
        if (ok && elect_one()) {
#pragma unroll
          for (int k = 4 * half; k < 4 * half + 4; ++k)
            if (k < groups)
              tc_mma_bf16_ts(tmem_base + 256u + 128u * g, tmem_base + 128u * g + 8u * k, vd + 128u * k, idesc_pv, (!first || k > 0) ? 1u : 0u);
        }
        __syncwarp();
      }
    };
    auto finish = [&](uint32_t g) {
      if (ok && elect_one()) tc_commit(o_full_bar(g));
      __syncwarp();
    };
    auto clear_behind = [&](uint32_t slot, int rows) {     // value rows that do not exist: a weight of 0 would not stop a NaN
      const int upto = (rows + 15) / 16 * 16;
      if (rows >= upto) return;
      for (int x = lane; x < (upto - rows) * 16; x += 32)
        *reinterpret_cast<uint4*>(base_ptr + kPrefixSlot0 + slot * kSlotBytes + (x >> 3 & 1) * kHalfBytes + (rows + (x >> 4)) * 128 +
                                  (x & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
    };
    wait(q_full_bar, 0);
    // A group's S is taken over by its weights; its next S goes into it right behind P V (the tensor pipe runs one thread's
    // products in order, so the product has read P by then).
    if (PAIR) {
      uint32_t slot = ok ? next_slot() : 0u;
      for (int g = 0; g < count; ++g) issue_s((uint32_t)g, slot);
      release(slot);
      for (int t = 0; ok && t < T; ++t) {
        const int rows = min(kTileRows, keys - t * kTileRows);
        const uint32_t v_slot = next_slot();
        if (!ok) break;
        clear_behind(v_slot, rows);
        const bool more = t + 1 < T;
        const uint32_t k_slot = more ? next_slot() : 0u;
        for (int g = 0; ok && g < count; ++g) {
          issue_pv((uint32_t)g, v_slot, (rows + 15) >> 4, (uint32_t)t & 1u, t == 0);
          if (more) issue_s((uint32_t)g, k_slot); else finish((uint32_t)g);
        }
        release(v_slot);
        if (more) release(k_slot);
      }
    } else {
      for (uint32_t g = 0; g < 2u && (int)g < T && ok; ++g) {
        const uint32_t slot = next_slot();
        issue_s(g, slot);
        release(slot);
      }
      for (int t = 0; ok && t < T; ++t) {
        const uint32_t g = (uint32_t)t & 1u, v_slot = next_slot();
        if (!ok) break;
        const int rows = min(kTileRows, keys - t * kTileRows);
        clear_behind(v_slot, rows);
        issue_pv(g, v_slot, (rows + 15) >> 4, (uint32_t)(t >> 1) & 1u, t < 2);
        release(v_slot);
        if (ok && t + 2 < T) {
          const uint32_t slot = next_slot();
          issue_s(g, slot);
          release(slot);
        }
      }
      for (uint32_t g = 0; g < 2u; ++g) finish(g);
    }
    if (!ok) {
      if (elect_one()) tc_commit(drain_bar);
      __syncwarp();
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(drain_bar, 0) && global_ns() - t0 < a.wait_ns) {}
    }
  } else {
    // ------------------------------------------------------------ softmax: thread r of a tile of query rows
    const int group = (warp - 2) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + group * 128u, o_addr = lane_addr + 256u + group * 128u;
    const float sc = a.scale_log2;
    const uint64_t sc2 = pack2(sc, sc);
    float top = -INFINITY, sum = 0.f;
    bool has_o = false, ok = true;
    const int step = PAIR ? 1 : 2, end = PAIR && group >= count ? 0 : T;
    for (int t = PAIR ? 0 : group; ok && t < end; t += step) {
      ok = mbar_wait(s_full_bar(group), (uint32_t)(PAIR ? t : t >> 1) & 1u, abort_flag, a.status, a.wait_ns);
      if (!(ok = __all_sync(0xffffffffu, ok))) break;
      tc_fence_after();
      const int valid = keys - t * kTileRows;              // keys of this tile that exist
      float v[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + 32 * c, *reinterpret_cast<float(*)[32]>(v + 32 * c));
      tmem_ld_wait();
      if (valid < kTileRows) {
#pragma unroll
        for (int e = 0; e < 128; ++e)
          if (e >= valid) v[e] = -INFINITY;
      }
      float ext[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
      for (int e = 4; e < 124; e += 8)
#pragma unroll
        for (int j = 0; j < 4; ++j) ext[j] = max3(ext[j], v[e + 2 * j], v[e + 2 * j + 1]);
#pragma unroll
      for (int j = 0; j < 4; ++j) ext[j] = fmaxf(ext[j], v[124 + j]);
      const float tile_top = fmaxf(fmaxf(ext[0], ext[1]), fmaxf(ext[2], ext[3])) * sc;
      const bool move = tile_top > top + kPrefixSlack || top == -INFINITY;
      if (__any_sync(0xffffffffu, move)) {
        const float now = move ? fmaxf(top, tile_top) : top;
        if (has_o) {                                       // rescale O_group (its previous product retired before this S)
          const float f = !move || now == -INFINITY ? 1.f : fast_exp2(top - now);
          sum *= f;
#pragma unroll 1
          for (int c0 = 0; c0 < 128; c0 += 16) {
            uint32_t o[16];
            tmem_ld16(o_addr + c0, o);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
            tmem_st16(o_addr + c0, o);
          }
          tmem_st_wait();
        }
        top = now;
      }
      const float ref = top == -INFINITY ? 0.f : top;
      const uint64_t nref2 = pack2(-ref, -ref);
      uint64_t part[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
      for (int c = 0; c < 4; ++c) {                        // 32 keys -> 16 columns of P
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint64_t w2 = exp2_pair(fma2(pack2(v[32 * c + 2 * e], v[32 * c + 2 * e + 1]), sc2, nref2));
          part[e & 3] = add2(part[e & 3], w2);
          float w0, w1;
          unpack2(w2, w0, w1);
          const __nv_bfloat162 b = __floats2bfloat162_rn(w0, w1);
          w[e] = *reinterpret_cast<const uint32_t*>(&b);
        }
        tmem_st16(s_addr + 16 * c, w);
        if (c & 1) {                                       // 64 keys' weights are in place
          tmem_st_wait();
          tc_fence_before();
          mbar_arrive(p_ready_bar(group, c >> 1));
        }
      }
      float p0, p1;
      unpack2(add2(add2(part[0], part[1]), add2(part[2], part[3])), p0, p1);
      sum += p0 + p1;
      has_o = true;
    }
    // ------------------------------------------------------------ output
    // Rows go through shared memory, so that a warp writes 128 contiguous bytes of four rows at a time; a row's eight places
    // are permuted against bank conflicts.  The space: a row tile's own Q (for a single tile the one behind it), which no
    // product reads any more once all of the group are done.
    if (end > 0) ok = ok && mbar_wait(o_full_bar(group), 0, abort_flag, a.status, a.wait_ns);
    if (!PAIR) ok = ok && mbar_wait(o_full_bar(1 - group), 0, abort_flag, a.status, a.wait_ns);
    ok = __all_sync(0xffffffffu, ok);
    unsigned char* stage = base_ptr + kPrefixQ + (PAIR ? group * kSlotBytes : kSlotBytes) + (PAIR ? warp - 2 - 4 * group : warp - 2) * 4096;
    float f0 = 1.f, f1 = 0.f, m = top, l = sum;
    if (!PAIR) {                                           // the groups' halves meet (group 0 always has a tile of keys)
      float2* xchg = reinterpret_cast<float2*>(base_ptr + kPrefixQ);
      xchg[group * kTileRows + r] = make_float2(has_o ? top : -INFINITY, has_o ? sum : 0.f);
      asm volatile("bar.sync 1, 256;" ::: "memory");       // reached by all eight warps, aborted or not
      const float2 e0 = xchg[r], e1 = xchg[kTileRows + r];
      m = fmaxf(e0.x, e1.x);
      f0 = m == -INFINITY ? 1.f : fast_exp2(e0.x - m);
      f1 = T > 1 ? (m == -INFINITY ? 1.f : fast_exp2(e1.x - m)) : 0.f;
      l = f0 * e0.y + f1 * e1.y;
    }
    if (ok && end > 0) {
      tc_fence_after();
      const size_t part = (((size_t)p * a.tiles + tile0 + (PAIR ? group : 0)) * a.chunks + chunk) * kTileRows;
      const int used = a.seqs * a.tokens * a.group;
      if ((PAIR || group == 0) && r < used) a.part_ml[part + r] = make_float2(m, l);
      const bool both = !PAIR && T > 1;
      const int c_from = PAIR ? 0 : 64 * group, c_to = PAIR ? 128 : c_from + 64;
#pragma unroll 1
      for (int c0 = c_from; c0 < c_to; c0 += 32) {
        float v[32], w[32];
        tmem_ld32((PAIR ? o_addr : lane_addr + 256u) + c0, v);
        if (both) tmem_ld32(lane_addr + 384u + c0, w);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          float4 o = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
          if (!PAIR) { o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0; }
          if (both) {
            o.x = fmaf(w[4 * c], f1, o.x);
            o.y = fmaf(w[4 * c + 1], f1, o.y);
            o.z = fmaf(w[4 * c + 2], f1, o.z);
            o.w = fmaf(w[4 * c + 3], f1, o.w);
          }
          *reinterpret_cast<float4*>(stage + lane * 128 + ((c ^ (lane & 7)) * 16)) = o;
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int row = 4 * k + (lane >> 3), c = lane & 7;
          const float4 o = *reinterpret_cast<const float4*>(stage + row * 128 + ((c ^ (row & 7)) * 16));
          if (quarter * 32 + row < used) *reinterpret_cast<float4*>(a.part_o + (part + quarter * 32 + row) * 128 + c0 + 4 * c) = o;
        }
        __syncwarp();
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)kPrefixTmemCols)
                 : "memory");
  }
}

}  // namespace umma
}  // namespace curdkv
