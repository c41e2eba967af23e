// New rows join a generation-phase cache and rows of least weight leave it, in place: the eviction step of a cache whose rows
// are ranked by weights that the caller keeps (curdkv_cache_push).
//
// Keys as in the selection: forced rows (sinks and the most recent, found by position) on top, then weights; of equal ones
// the row in the lower slot stays.  In steady state a step evicts as many rows as come, a handful at most, so nothing is
// sorted: one sweep over the head's weights and positions (8 bytes a row, what bounds the kernel beside its start and
// end) leaves every thread with the least key of its slots, and each eviction takes the least of all, whose owner
// then looks for its next one.  8 heads of 1703 slots 4.8 us, 1024 of 2049 11.6, 64 of 65537 20 (floor 5.1).  Slots are read
// four at a time where the capacity is a multiple of four, which a budget and the rows of one step need not be: 64 heads of
// 65540 with four rows to go 24 us, 59 with slots one at a time; 8 heads, which keep eight SMs busy, take as long (floor 0.6).
#pragma once
#include "cache.cuh"

namespace curdkv {

constexpr int kPushMost = 8;                               // rows a step may evict

struct PushArgs {
  AppendArgs append;                 // raw_new: [batch][heads][t] or nullptr (0)
  int budget, num_sink, window;
  int32_t* tickets;                  // [batch], zero on entry; nullptr: the heads of a sequence are a cluster
};

// One CTA per head; capacity at most budget + kPushMost.  With t rows of real slots 0 .. n - 1 (held rows, then new ones)
// the result is what append and in-place compression leave, and slots at or beyond the new count stay as they were.
__global__ void __launch_bounds__(1024) cache_push_kernel(const PushArgs s) {
  __shared__ unsigned long long s_least[32];
  __shared__ int s_leave[kPushMost];
  const AppendArgs& a = s.append;
  const int p = blockIdx.x, b = p / a.heads, h = p % a.heads, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");       // launched behind the kernel before it without waiting for its end
  const int cap = a.cache.capacity;
  int tb = a.t_new != nullptr ? a.t_new[b] : a.t;
  tb = tb < 0 ? 0 : (tb > a.t ? a.t : tb);
  const int was = a.cache.count[b], held = min(max(was, 0), cap), first_pos = a.cache.total[b], offered = tb;
  if (was != held && tid == 0) flag_status(a.status, CURDKV_DEV_BAD_INDEX);
  if (tb > cap - held) {
    if (tid == 0) flag_status(a.status, CURDKV_DEV_CACHE_FULL);
    tb = cap - held;
  }
  const int n = held + tb, kept = min(s.budget, n), leave = n - kept;        // leave <= capacity - budget <= kPushMost
  const int recent = first_pos + offered - s.window;
  float* raw = a.cache.raw + (size_t)p * cap;
  int32_t* pos = a.cache.pos + (size_t)p * cap;
  const float* raw_new = a.raw_new != nullptr ? a.raw_new + (size_t)p * a.t : nullptr;

  // rank of a slot: key above, then the lower slot above
  auto rank = [&](int j) {
    const int at = j < held ? pos[j] : first_pos + (j - held);
    const float w = j < held ? raw[j] : (raw_new != nullptr ? raw_new[j - held] : 0.f);
    const uint32_t key = at < s.num_sink || at >= recent ? kForcedKey : score_key(w);
    return ((unsigned long long)key << 32) | (uint32_t)~j;
  };
  constexpr unsigned long long kNone = ~0ull;
  // Held slots come four at a time where rows of weights and positions are 16-byte aligned, two such loads of each in flight.
  const bool wide = (cap & 3) == 0 && ((reinterpret_cast<uintptr_t>(a.cache.raw) | reinterpret_cast<uintptr_t>(a.cache.pos)) & 15u) == 0;
  const int quads = wide ? held >> 2 : 0;
  auto least_above = [&](unsigned long long last, bool any) {                // of this thread's slots
    unsigned long long best = kNone;
    auto take = [&](int j, int at, float w) {
      const uint32_t key = at < s.num_sink || at >= recent ? kForcedKey : score_key(w);
      const unsigned long long x = ((unsigned long long)key << 32) | (uint32_t)~j;
      if ((!any || x > last) && x < best) best = x;
    };
    for (int q = tid; q < quads; q += 2 * blockDim.x) {
      const int q1 = q + blockDim.x;
      const bool two = q1 < quads;
      const int4 p0 = reinterpret_cast<const int4*>(pos)[q], p1 = reinterpret_cast<const int4*>(pos)[two ? q1 : q];
      const float4 w0 = reinterpret_cast<const float4*>(raw)[q], w1 = reinterpret_cast<const float4*>(raw)[two ? q1 : q];
      take(4 * q, p0.x, w0.x); take(4 * q + 1, p0.y, w0.y); take(4 * q + 2, p0.z, w0.z); take(4 * q + 3, p0.w, w0.w);
      if (two) { take(4 * q1, p1.x, w1.x); take(4 * q1 + 1, p1.y, w1.y); take(4 * q1 + 2, p1.z, w1.z); take(4 * q1 + 3, p1.w, w1.w); }
    }
    for (int j = 4 * quads + tid; j < n; j += blockDim.x) {
      const unsigned long long x = rank(j);
      if ((!any || x > last) && x < best) best = x;
    }
    return best;
  };
  if (leave > 0) {
    unsigned long long mine = least_above(0ull, false);
    for (int e = 0; e < leave; ++e) {
      unsigned long long x = mine;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long y = __shfl_xor_sync(0xffffffffu, x, o);
        x = y < x ? y : x;
      }
      if (lane == 0) s_least[warp] = x;
      __syncthreads();
      unsigned long long all = lane < (int)(blockDim.x >> 5) ? s_least[lane] : kNone;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long y = __shfl_xor_sync(0xffffffffu, all, o);
        all = y < all ? y : all;
      }
      if (tid == 0) s_leave[e] = (int)~(uint32_t)all;
      __syncthreads();
      if (e + 1 < leave && mine == all) mine = least_above(all, true);
    }
  }
  // Row x of the moves: the i-th row kept at or behind `kept` goes to the i-th place given up below it, new rows with a slot
  // of their own below `kept` go there.  leave is small: every warp works the list out for itself.
  const int own0 = min(held, kept), own_rows = kept - own0;                  // new rows in slots own0 .. kept - 1
  auto left = [&](int slot) {
    bool gone = false;
    for (int e = 0; e < leave; ++e) gone = gone || s_leave[e] == slot;
    return gone;
  };
  auto hole = [&](int i) {                                 // the i-th place below `kept` that was given up, or -1
    for (int e = 0; e < leave; ++e) {
      const int x = s_leave[e];
      if (x >= kept) continue;
      int before = 0;
      for (int f = 0; f < leave; ++f) before += s_leave[f] < x;
      if (before == i) return x;
    }
    return -1;
  };
  auto mover = [&](int i) {                                // the i-th slot at or behind `kept` whose row stays
    for (int j = kept; j < n; ++j)
      if (!left(j) && i-- == 0) return j;
    return -1;
  };
  const int jobs = own_rows + leave, half = lane >> 4, l16 = lane & 15, chunks = a.d >> 3;
  const KvView& T = half ? a.V_new : a.K_new;
  const __nv_bfloat16* new_rows = T.base + b * T.stride_b + h * T.stride_h;
  __nv_bfloat16* rows = (half ? a.cache.V : a.cache.K) + (size_t)p * cap * a.d;
  for (int x = warp; x < jobs; x += blockDim.x >> 5) {
    int from, to;
    if (x < own_rows) {
      from = to = own0 + x;
      if (left(from)) continue;                            // (its place is a hole)
    } else {
      to = hole(x - own_rows);
      from = to < 0 ? -1 : mover(x - own_rows);
      if (to < 0 || from < 0) continue;
    }
    const __nv_bfloat16* src = from < held ? rows + (size_t)from * a.d : new_rows + (int64_t)(from - held) * T.stride_n;
    for (int c = l16; c < chunks; c += 16)
      reinterpret_cast<uint4*>(rows + (size_t)to * a.d)[c] = reinterpret_cast<const uint4*>(src)[c];
    if (lane == 0) {
      const float w = from < held ? raw[from] : (raw_new != nullptr ? raw_new[from - held] : 0.f);
      const int at = from < held ? pos[from] : first_pos + (from - held);
      raw[to] = w;
      pos[to] = at;
    }
  }
  // counters, when every head of the sequence has read them
  if (s.tickets == nullptr) {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (h == 0 && tid == 0) {
      a.cache.count[b] = kept;
      a.cache.total[b] = first_pos + offered;
    }
  } else {
    __threadfence();
    __syncthreads();
    if (tid == 0 && atomicAdd(s.tickets + b, 1) == a.heads - 1) {
      a.cache.count[b] = kept;
      a.cache.total[b] = first_pos + offered;
    }
  }
}

}  // namespace curdkv
