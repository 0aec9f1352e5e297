// The paged key-value cache as the kernels see it: tables, positions of new tokens, conversions.  sm_100a only.
#pragma once

#include "device_utils.cuh"
#include "marlin_internal.cuh"

namespace marlin_b200 {

// These kernels start while the one before them in the stream still runs, and wait for its end (pdl_wait_prior_grids) before they read
// anything: what it writes, such as the output of the qkv layer, lengths or a page table, changes while they live.  A load through the
// read-only path (__ldg, ld.global.nc) is for memory that nobody writes during the whole kernel, and may be moved in front of the wait; these
// are ordinary loads, which the compiler keeps behind it, in their order, but is free to move over stores.
__device__ __forceinline__ int load(const int* p) {
  int x;
  asm volatile("ld.global.b32 %0, [%1];" : "=r"(x) : "l"(p));
  return x;
}
__device__ __forceinline__ float load(const float* p) {
  float x;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(x) : "l"(p));
  return x;
}
__device__ __forceinline__ uint4 load(const uint4* p) {
  uint4 x;
  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
  return x;
}

// A call that reaches outside of the cache says so in a word of its own: a wait that runs out, there or in a later call on the workspace,
// finds the status word free, and neither hides the other.  (Any number of threads write the same.)
__device__ __forceinline__ void report_cache(int* status) { *(volatile int*)(status + kWsCacheWord) = MARLIN_ERR_CACHE; }

constexpr int kLongest = 1 << 30;  // tokens of a sequence: positions, windows in front of them and tiles asked for ahead fit in 32 bits

// Length of sequence b.  One that its row of the table cannot hold is bad and taken as 0, so that none of its new tokens has a
// position: cut down to what the row holds, it would put them over tokens that are there already.
// (`bad` is for the caller to report, behind the loads of other sequences, which an atomic in between would hold back.)
__device__ __forceinline__ int cache_length(const KvCacheView& c, int b, bool& bad) {
  const int len = load(c.lengths + b);
  const bool fits = len >= 0 && len <= min((long long)c.max_pages << c.page_shift, (long long)kLongest);
  bad |= !fits;
  return fits ? len : 0;
}

// Offset (in elements) of the token at position pos < max_pages * page_size, head h; -1 where its page is not there.
__device__ __forceinline__ long long cache_offset(const KvCacheView& c, int page, int h, int pos, int* status) {
  if ((unsigned)page >= (unsigned)c.pages) {
    report_cache(status);
    return -1;
  }
  return page * c.s_page + h * c.s_head + (pos & ((1 << c.page_shift) - 1)) * c.s_token;
}

// two fp32 values -> two e4m3 bytes (lo in the lower one): to nearest even, saturating at 448, NaN kept
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// two e4m3 bytes (the lower 16 bits) -> two fp16 values, exact
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
  return r;
}

}  // namespace marlin_b200
