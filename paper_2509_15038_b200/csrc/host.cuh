// Host-side helpers that the serving calls share: checks of arguments and launch bookkeeping.
#pragma once
#include <atomic>
#include <cstdint>

#include "common.cuh"

namespace curdkv {
namespace host {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t x) { return (x + 255) & ~size_t(255); }

inline bool launched() {
  count_launch();
  return cudaGetLastError() == cudaSuccess;
}

// SMs of the current device (asked of the driver once per device), or a B200's where none can be asked
// (workspace sizes).
inline int sms() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) == cudaSuccess) {
    if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0) {
      if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
      return n;
    }
  }
  cudaGetLastError();
  return 148;
}

inline bool status_ok(const void* workspace) { return (reinterpret_cast<uintptr_t>(workspace) & 255u) == 0; }

// Lets `kernel` use `bytes` of shared memory on the current device; asked of the driver once per device.
template <typename Kernel>
bool allow_smem(Kernel kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  done.fetch_or(bit, std::memory_order_relaxed);
  return true;
}

// Whether a TMA map can hold these strides: positive and below 2^40 bytes (for sequences and heads: where there are
// several).
inline bool map_strides_ok(int64_t batch, int64_t heads, int64_t sb, int64_t sh, int64_t sn) {
  const int64_t most = (int64_t)1 << 38;
  return (batch <= 1 || (sb > 0 && sb < most)) && (heads <= 1 || (sh > 0 && sh < most)) && sn < most;
}

inline bool query_strides_ok(const void* x, int64_t sb, int64_t sh, int64_t sn) {
  return x != nullptr && aligned16(x) && sb >= 0 && sh >= 0 && sn >= 128 && sb % 8 == 0 && sh % 8 == 0 && sn % 8 == 0;
}

// Rows that are written may not share memory with one another: by ascending stride, each axis has to step over all
// that the ones before it reach.  (An axis of one never steps.)
inline bool rows_apart(int64_t batch, int64_t heads, int64_t rows, int64_t sb, int64_t sh, int64_t sn) {
  int64_t size[3] = {batch, heads, rows}, step[3] = {sb, sh, sn};
  __int128 reach = 128;
  for (int done = 0; done < 3; ++done) {
    int least = -1;
    for (int i = 0; i < 3; ++i)
      if (size[i] > 1 && (least < 0 || step[i] < step[least])) least = i;
    if (least < 0) break;
    if (step[least] < reach) return false;
    reach += (__int128)(size[least] - 1) * step[least];
    size[least] = 1;
  }
  return true;
}

inline bool overlap(const void* a, const void* b, __int128 bytes) {
  const __int128 x = (__int128)reinterpret_cast<uintptr_t>(a), y = (__int128)reinterpret_cast<uintptr_t>(b);
  return x < y + bytes && y < x + bytes;
}

}  // namespace host
}  // namespace curdkv
