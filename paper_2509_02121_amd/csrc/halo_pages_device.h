// Device code that the page kernels over bf16 / fp32 pools (halo_pages.hip) and
// over 4-bit ones (halo_kvq_pages.hip) share.
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

// How many lanes before this one the mask has, and `more`.
__device__ __forceinline__ int lanes_before(uint64_t mask, int more) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, more));
}

constexpr int kBins = 2048;      // 11 bits

// The largest of the kBins counts' places with `left` or more at or above it, and how
// many of `left` fall into it, by the whole workgroup.
template <int W>
__device__ __forceinline__ void find_bin(const int (&count)[kBins], int (&sums)[W], int (&found)[2], int& left, int& bin) {
  constexpr int N = kBins / (64 * W);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  int c[N], mine = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) mine += c[j] = count[kBins - 1 - (N * tid + j)];
  const int upto = wave_inclusive_sum(mine);
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int above = upto - mine;
#pragma unroll
  for (int v = 0; v < W; ++v) above += v < wave ? sums[v] : 0;
  if (above < left && above + mine >= left) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (above < left && above + c[j] >= left) {
        found[0] = kBins - 1 - (N * tid + j);
        found[1] = left - above;
        above = INT32_MAX / 2;
      } else {
        above += c[j];
      }
    }
  }
  __syncthreads();
  bin = found[0];
  left = found[1];
}

// The range of one sequence, and its whole-page tiles (none where the range
// does not fit its page list: its own workgroup flags that).
struct SeqRange {
  int start, base, tiles, f0;
  int64_t off;
  // a: the arrays of a scatter's arguments; per_page: tiles of a page
  template <typename Args>
  __device__ __forceinline__ SeqRange(const Args& a, int per_page, int seq) {
    start = a.seq_start[seq];
    const int count = a.seq_count[seq];
    base = a.seq_page_indptr[seq];
    const int next = a.seq_page_indptr[seq + 1];
    off = a.in_token_offset[seq];
    const PageRange r(start, count);
    f0 = r.f0;
    const bool fits = count > 0 && start >= 0 && (int64_t)start + count <= (int64_t)(next - base) * 16;
    tiles = fits ? r.nfull * per_page : 0;
  }
};

// Sequences whose tiles one workgroup sums.
constexpr int kTileSeqs = 4096;

// Whole pages: the tiles of up to kTileSeqs sequences, shared equally by the
// waves. Up to 64 sequences every wave sums by itself, one sequence per lane,
// and finds its tiles in the lanes' registers, without a barrier or a second
// look at the metadata (32 chunks of 512 tokens, K and V: 30.6 us; by the
// workgroup 33.5); it takes every turns-th tile, so that neighbouring waves
// move neighbouring heads of one page (32 fp32 chunks of 512 tokens after other
// work: 83 us with contiguous runs, 72 so). More are summed by the workgroup,
// thread i those of sequences i, i + 256, ..., in LDS (1024 appends: 18 us,
// against 22.7 when every wave sums all of them), and a wave takes a contiguous
// run. A sequence with fewer than 16 new tokens has no whole page: only its
// count is read.
// `tile` is called with the dense row of the sequence's token 0, its page list, a
// page's place in it and the tile's number in the page.
template <typename Args, typename Tile>
__device__ __forceinline__ void whole_tiles(const Args& a, int per_page, int s0, int n_seqs, int turn, int turns,
                                            int (&sums)[260], int wave, int lane, Tile tile) {
  const bool by_wave = n_seqs <= 64;
  int mine = 0, l_start = 0, l_base = 0, l_f0 = 0, upto, total;
  int64_t l_off = 0;
  if (by_wave) {
    if (lane < n_seqs) {
      const SeqRange r(a, per_page, s0 + lane);
      mine = r.tiles;
      l_start = r.start;
      l_base = r.base;
      l_f0 = r.f0;
      l_off = r.off;
    }
    if (!__any(mine > 0)) return;
    upto = wave_inclusive_sum(mine);
    total = __builtin_amdgcn_readlane(upto, 63);
  } else {
    constexpr int kAhead = 4;   // counts in flight per thread
    for (int i0 = threadIdx.x; i0 < n_seqs; i0 += kAhead * 256) {
      int count[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) count[u] = i0 + 256 * u < n_seqs ? a.seq_count[s0 + i0 + 256 * u] : 0;
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (count[u] >= 16) mine += SeqRange(a, per_page, s0 + i0 + 256 * u).tiles;
    }
    if (!__syncthreads_or(mine)) return;
    upto = wave_inclusive_sum(mine);
    if (lane == 63) sums[256 + wave] = upto;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      upto += w < wave ? sums[256 + w] : 0;
      total += sums[256 + w];
    }
    sums[threadIdx.x] = upto;
    __syncthreads();
  }
  const int per = (int)(((int64_t)total + turns - 1) / turns);
  int k = by_wave ? turn : (int)min((int64_t)total, (int64_t)turn * per);
  const int k_end = by_wave ? total : (int)min((int64_t)total, (int64_t)k + per);
  while (k < k_end) {
    int t, n, base, f0;
    int64_t at;   // dense row of the sequence's token 0
    if (by_wave) {
      const int lo = __popcll(__ballot(upto <= k));   // the lane whose sequence holds tile k
      t = k - (lo ? __builtin_amdgcn_readlane(upto, lo - 1) : 0);
      n = __builtin_amdgcn_readlane(mine, lo);
      base = __builtin_amdgcn_readlane(l_base, lo);
      f0 = __builtin_amdgcn_readlane(l_f0, lo);
      at = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(l_off >> 32), lo) << 32) |
                     (uint32_t)__builtin_amdgcn_readlane((int)l_off, lo)) -
           __builtin_amdgcn_readlane(l_start, lo);
    } else {
      int lo = 0;   // the thread whose sequences hold tile k
#pragma unroll
      for (int j = 0; j < 4; ++j) lo += __popcll(__ballot(sums[64 * j + lane] <= k));
      t = k - (lo ? sums[lo - 1] : 0);
      t = __builtin_amdgcn_readfirstlane(t);
      int seq = s0 + lo;
      SeqRange r(a, per_page, seq);
      while (t >= r.tiles) {
        t -= r.tiles;
        seq += 256;
        r = SeqRange(a, per_page, seq);
      }
      n = r.tiles;
      base = r.base;
      f0 = r.f0;
      at = r.off - r.start;
    }
    // tiles t .. t_end - 1 of one sequence, a page's next to each other
    const int t_end = by_wave ? t + 1 : min(n, t + (k_end - k));
    k += by_wave ? turns : t_end - t;
#pragma nounroll
    for (; t < t_end; ++t) tile(at, base, f0 + t / per_page, t % per_page);
  }
}

}  // namespace
