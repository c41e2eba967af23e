// Attention of many query rows over a prefix that their sequences share: the rows of all sequences, stacked, against the
// prefix's keys once.  One part (attn_rows.cuh) per CTA: a tile of up to 128 query rows against a run of keys; it leaves
// reference, sum and fp32 sums of values for the joining kernel.
//
// A tile is `seqs` sequences x `tokens` tokens x the heads of a KV head's group, brought in by one 5-D map, whatever the
// strides.  The walk over the keys is that of attn_umma.cuh: S = Q K_t^T per 128-key tile, two groups of four softmax warps
// on alternate tiles, a thread per query row; the weights go back over S in TMEM as bf16 and are the A operand of
// O_g += P V_t; each group has its own running maximum (moved when a tile exceeds it by more than 2^8), sum and accumulator.
// Weights are rounded to bf16 (2^-9 of each), sums take them unrounded.
//
// What bounds it: with one tile of rows a KV head the keys' bytes (64 KB a tile of keys; the SM's share of the memory
// takes 1.5 us for it), with more the walk itself, 1900 cycles a tile of keys: the products 1550, the exponentials 1020.
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

constexpr int kPrefixThreads = 320;                        // TMA, MMA, 2 x 4 softmax warps
constexpr int kPrefixRing = 5;
constexpr int kPrefixQ = 0;
constexpr int kPrefixSlot0 = kSlotBytes;
constexpr int kPrefixBar = kPrefixSlot0 + kPrefixRing * kSlotBytes;
constexpr int kPrefixDynamic = kPrefixBar + 256 + 1024;
constexpr int kPrefixTmemCols = 512;                       // S of group g at 128 g (its weights over it), O of group g at 256 + 128 g
constexpr float kPrefixSlack = 8.f;

// grid = sets * heads * chunks * tiles, tiles innermost: CTAs that read the same keys run side by side.
__global__ void __launch_bounds__(kPrefixThreads, 1)
prefix_attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v, const PrefixArgs a) {
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bar0 = base + kPrefixBar;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kPrefixRing + s); };
  auto s_full_bar = [&](int s) { return bar0 + 8u * (2 * kPrefixRing + s); };
  auto p_ready_bar = [&](int s) { return bar0 + 8u * (2 * kPrefixRing + 2 + s); };
  const uint32_t q_full_bar = bar0 + 8u * (2 * kPrefixRing + 4);
  const uint32_t o_full_bar = bar0 + 8u * (2 * kPrefixRing + 5);
  const uint32_t drain_bar = bar0 + 8u * (2 * kPrefixRing + 6);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(base_ptr + kPrefixBar + 8 * (2 * kPrefixRing + 7));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  __shared__ float2 xchg[2][kTileRows];                    // each group's reference and sum
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const int tile = blockIdx.x % a.tiles, chunk = blockIdx.x / a.tiles % a.chunks, p = blockIdx.x / a.tiles / a.chunks;
  const int set = p / a.heads, h = p % a.heads;
  int n = a.n_max;
  if (a.lens != nullptr) {
    n = seq_len_of(a.lens, set, a.n_max);
    if (n != a.lens[set] && tid == 0 && chunk == 0 && tile == 0) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
  }
  const int k0 = chunk * a.chunk, keys = min(n - k0, a.chunk);
  if (keys <= 0) return;
  const int T = (keys + kTileRows - 1) / kTileRows;
  const int seq0 = tile / a.token_tiles * a.seqs, tok0 = tile % a.token_tiles * a.tokens;

  if (tid == 0) {
    for (int s = 0; s < kPrefixRing; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(s_full_bar(s), 1);
      mbar_init(p_ready_bar(s), 128);
    }
    mbar_init(q_full_bar, 1);
    mbar_init(o_full_bar, 1);
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

  // Tiles go through the ring in the order the products consume them: K_0, K_1, then for every t: V_t, K_{t+2} (if any).
  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      uint64_t pol;
      asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
      mbar_arrive_expect_tx(q_full_bar, (uint32_t)(a.seqs * a.tokens * a.group) * 256u);
      tma_load_5d(base + kPrefixQ, &map_q, q_full_bar, 0, 0, tok0, h, set * a.share + seq0);
      tma_load_5d(base + kPrefixQ + kHalfBytes, &map_q, q_full_bar, 64, 0, tok0, h, set * a.share + seq0);
      uint32_t it = 0;
      bool ok = true;
      auto load = [&](const CUtensorMap* map, int t) {
        const int slot = it % kPrefixRing;
        if (!(ok = mbar_wait(empty_bar(slot), ((it / kPrefixRing) & 1u) ^ 1u, abort_flag, a.status, a.wait_ns))) return;
        mbar_arrive_expect_tx(full_bar(slot), kSlotBytes);
        const uint32_t dst = base + kPrefixSlot0 + slot * kSlotBytes;
        tma_load_4d(dst, map, full_bar(slot), 0, k0 + t * kTileRows, h, set, pol);
        tma_load_4d(dst + kHalfBytes, map, full_bar(slot), 64, k0 + t * kTileRows, h, set, pol);
        ++it;
      };
      load(&map_k, 0);
      if (ok && T > 1) load(&map_k, 1);
      for (int t = 0; ok && t < T; ++t) {
        load(&map_v, t);
        if (ok && t + 2 < T) load(&map_k, t + 2);
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
    uint32_t it = 0;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) {
      ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, a.status, a.wait_ns) && ok);
      tc_fence_after();
    };
    wait(q_full_bar, 0);
    auto issue_s = [&](uint32_t buf) {                     // S[buf] = Q K^T for the next K tile of the ring
      const uint32_t slot = it % kPrefixRing;
      wait(full_bar(slot), (it / kPrefixRing) & 1u);
      ++it;
      if (!ok) return;
      const uint64_t kd = k_desc0 + slot * (kSlotBytes >> 4);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t off = (uint32_t)(k >> 2) * (kHalfBytes >> 4) + (uint32_t)(k & 3) * 2u;
          tc_mma_bf16(tmem_base + buf * 128u, q_desc + off, kd + off, idesc_s, k > 0);
        }
        tc_commit(empty_bar(slot));
        tc_commit(s_full_bar(buf));
      }
      __syncwarp();
    };
    // A group's S is taken over by its weights; S_{t+2} goes into it right behind P_t V_t (the tensor pipe runs one thread's
    // products in order, so the product has read P by then).
    if (ok) issue_s(0);
    if (ok && T > 1) issue_s(1);
    for (int t = 0; ok && t < T; ++t) {
      const uint32_t slot = it % kPrefixRing, buf = (uint32_t)t & 1u;
      wait(full_bar(slot), (it / kPrefixRing) & 1u);
      ++it;
      if (!ok) break;
      const int rows = min(kTileRows, keys - t * kTileRows), groups = (rows + 15) >> 4;
      if (rows < groups * 16) {                            // value rows that do not exist: a weight of 0 would not stop a NaN
        for (int x = lane; x < (groups * 16 - rows) * 16; x += 32)
          *reinterpret_cast<uint4*>(base_ptr + kPrefixSlot0 + slot * kSlotBytes + (x >> 3 & 1) * kHalfBytes + (rows + (x >> 4)) * 128 +
                                    (x & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }
      wait(p_ready_bar(buf), (uint32_t)(t >> 1) & 1u);
      if (!ok) break;
      const uint64_t vd = v_desc0 + slot * (kSlotBytes >> 4);
      const uint32_t o_tmem = tmem_base + 256u + buf * 128u, p_tmem = tmem_base + buf * 128u;
      if (elect_one()) {
        // 16 keys per product: 8 columns of P, 2048 bytes (128 units) of the V tile
#pragma unroll
        for (int g = 0; g < 8; ++g)
          if (g < groups) tc_mma_bf16_ts(o_tmem, p_tmem + 8u * g, vd + 128u * g, idesc_pv, (t > 1 || g > 0) ? 1u : 0u);
        tc_commit(empty_bar(slot));
      }
      __syncwarp();
      if (t + 2 < T) issue_s(buf);
    }
    if (ok && elect_one()) tc_commit(o_full_bar);
    __syncwarp();
    if (!ok) {
      if (elect_one()) tc_commit(drain_bar);
      __syncwarp();
      const unsigned long long t0 = global_ns();
      while (!mbar_try_wait(drain_bar, 0) && global_ns() - t0 < a.wait_ns) {}
    }
  } else {
    // ------------------------------------------------------------ softmax: thread r of the tile, every other tile of keys
    const int group = (warp - 2) >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t s_addr = lane_addr + group * 128u, o_addr = lane_addr + 256u + group * 128u;
    const float sc = a.scale_log2;
    const uint64_t sc2 = pack2(sc, sc);
    float top = -INFINITY, sum = 0.f;
    bool has_o = false, ok = true;
    for (int t = group; ok && t < T; t += 2) {
      ok = mbar_wait(s_full_bar(group), (uint32_t)(t >> 1) & 1u, abort_flag, a.status, a.wait_ns);
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
      }
      float p0, p1;
      unpack2(add2(add2(part[0], part[1]), add2(part[2], part[3])), p0, p1);
      sum += p0 + p1;
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(p_ready_bar(group));
      has_o = true;
    }
    // ------------------------------------------------------------ the groups' halves meet; each writes 64 channels
    xchg[group][r] = make_float2(has_o ? top : -INFINITY, has_o ? sum : 0.f);
    asm volatile("bar.sync 1, 256;" ::: "memory");         // reached by all eight warps, aborted or not
    if (ok) ok = mbar_wait(o_full_bar, 0, abort_flag, a.status, a.wait_ns);
    ok = __all_sync(0xffffffffu, ok);
    if (ok) {
      tc_fence_after();
      const float2 e0 = xchg[0][r], e1 = xchg[1][r];       // (group 0 always has a tile)
      const float m = fmaxf(e0.x, e1.x);
      const float f0 = m == -INFINITY ? 1.f : fast_exp2(e0.x - m), f1 = T > 1 ? (m == -INFINITY ? 1.f : fast_exp2(e1.x - m)) : 0.f;
      const size_t part = (((size_t)p * a.tiles + tile) * a.chunks + chunk) * kTileRows;
      const int used = a.seqs * a.tokens * a.group;
      if (group == 0 && r < used) a.part_ml[part + r] = make_float2(m, f0 * e0.y + f1 * e1.y);
      // Rows go through shared memory (all tiles of the ring are done with), so that a warp writes 128 contiguous bytes of
      // four rows at a time; a row's eight places are permuted against bank conflicts.
      unsigned char* stage = base_ptr + kPrefixSlot0 + (warp - 2) * 4096;
#pragma unroll 1
      for (int c0 = 64 * group; c0 < 64 * group + 64; c0 += 32) {
        float v[32], w[32];
        tmem_ld32(lane_addr + 256u + c0, v);
        if (T > 1) tmem_ld32(lane_addr + 384u + c0, w);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          float4 o;
          o.x = v[4 * c] * f0 + (T > 1 ? w[4 * c] * f1 : 0.f);
          o.y = v[4 * c + 1] * f0 + (T > 1 ? w[4 * c + 1] * f1 : 0.f);
          o.z = v[4 * c + 2] * f0 + (T > 1 ? w[4 * c + 2] * f1 : 0.f);
          o.w = v[4 * c + 3] * f0 + (T > 1 ? w[4 * c + 3] * f1 : 0.f);
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
