// Device code that the page kernels over bf16 / fp32 pools (halo_pages.hip) and
// over 4-bit ones (halo_kv4_pages.hip) share.
#pragma once

#include <hip/hip_runtime.h>

#include "halo_internal.h"

namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// V pages keep the tokens of a dim row in the slot order 0-3, 8-11, 4-7,
// 12-15 (bits 2 and 3 of the index swapped; the map is its own inverse).
__device__ __forceinline__ int v_token_at_slot(int s) { return (s & 3) | ((s & 4) << 1) | ((s & 8) >> 1); }

// The last index s < n with indptr[s] <= x, for a nondecreasing indptr with
// indptr[0] <= x (wave-uniform x): the wave compares 64 evenly spaced
// entries at once and keeps the bracket that holds the answer, so up to 4095
// entries take two rounds of loads where a binary search takes twelve.
__device__ __forceinline__ int last_at_or_below(const int32_t* indptr, int n, int64_t x, int lane) {
  int lo = 0, len = n;
  while (len > 64) {
    const int stride = (len + 63) / 64;
    const int off = lane * stride;
    const bool hit = off < len && indptr[lo + off] <= x;
    const uint64_t mask = __ballot(hit);
    const int top = 63 - __clzll(mask);          // lane 0 always hits
    lo += top * stride;
    len = min(stride, len - top * stride);
  }
  const bool hit = lane < len && indptr[lo + lane] <= x;
  const uint64_t mask = __ballot(hit);
  return lo + 63 - __clzll(mask);
}

// Pages touched by tokens start .. start + count - 1 of one sequence: a first
// and a last one that may be partial, and nfull whole pages from slot f0.
struct PageRange {
  int first, last, f0, nfull;
  bool head, tail;   // the first / last page is partly touched (last != first)
  __device__ __forceinline__ PageRange(int start, int count) {
    const int end = start + count;
    first = start / 16;
    last = (end - 1) / 16;
    head = (start & 15) != 0 || end < 16 * (first + 1);
    tail = last > first && (end & 15) != 0;
    f0 = first + (head ? 1 : 0);
    nfull = last - (tail ? 1 : 0) - f0 + 1;
  }
};

// Inclusive sum over the lanes of a wave: shifts by 1, 2, 4 and 8 inside each
// row of 16 lanes, then the last lane of a row to the next row (rows 1 and 3)
// and lane 31 to the upper half.
__device__ __forceinline__ int wave_inclusive_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return x;
}

}  // namespace
