// Internal: the paged cache as kernels see it, and where a call's tokens go in it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "paged_plan.h"

namespace sirius {

// Keys [page][kv head][position][column], values [page][kv head][column][position].
struct PagedView {
  uint16_t* k_pages;
  uint16_t* v_pages;
  const int32_t* table;  // [B][max_pages]
  const int32_t* pos;    // [B]: rows in the cache before the call's tokens
  const int32_t* start;  // [B + 1]: a sequence's first token, or null: n tokens each
  int B, T, n;           // n: tokens of a sequence, at most (start set) or exactly
  int n_pages, page_size, max_pages;
  uint32_t page_magic;   // ceil(2^32 / page_size): row / page_size = row * magic >> 32
};

constexpr int kMaxPageSize = 4096;     // row * (magic * page_size - 2^32) < 2^20 * 2^12 stays below 2^32

__device__ __forceinline__ int page_of(const PagedView& c, int row) {
  return (int)__umulhi((uint32_t)row, c.page_magic);
}

// A sequence's tokens [first, first + n), inside [0, T) whatever the offsets say.
__device__ __forceinline__ int2 tokens_of(const PagedView& c, int b) {
  if (c.start == nullptr) return make_int2(b * c.n, c.n);
  const int s = min(max(c.start[b], 0), c.T), e = min(max(c.start[b + 1], s), c.T);
  return make_int2(s, e - s);
}

// Whether n tokens at rows p .. p + n - 1 lie inside the sequence's table.
__device__ __forceinline__ bool rows_fit(const PagedView& c, int p, int n) {
  return p >= 0 && (long)p + n <= (long)c.max_pages * c.page_size;
}

// The sequence that token t belongs to (the last whose first token is not behind t), -1 outside all.
// Uniform over the wave: 64 offsets are looked at together, so 65535 sequences take three loads.
__device__ __forceinline__ int sequence_of_wave(const PagedView& c, int t) {
  if (c.start == nullptr) return t / c.n;
  const int lane = threadIdx.x & (kWave - 1);
  int lo = 0, n = c.B + 1;  // the answer is the last entry <= t of [lo, lo + n)
  while (true) {
    const int step = (n + kWave - 1) / kWave;
    const int at = lane * step;
    const uint64_t le = __ballot(at < n && c.start[lo + at] <= t);
    if (le == 0) return -1;  // before the first token (only in the first turn)
    const int last = (63 - __builtin_clzll(le)) * step;
    lo += last;
    n = min(step, n - last);
    if (step == 1) break;
  }
  return lo < c.B ? lo : -1;
}

// The same by one lane alone.
__device__ __forceinline__ int sequence_of_lane(const PagedView& c, int t) {
  if (c.start == nullptr) return t / c.n;
  if (c.start[0] > t || c.start[c.B] <= t) return -1;
  int lo = 0, hi = c.B;  // start[lo] <= t < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (c.start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

}  // namespace sirius
