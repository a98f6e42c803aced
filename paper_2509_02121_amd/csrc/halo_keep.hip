// gfx950 kernels and entry points of the C ABI that shorten cached sequences:
// evict_kernel: which tokens of a sequence each head keeps, by their weights;
// keep_kernel: the kept tokens' keys and values, to the front or to other pages;
// release_kernel: the pages past a sequence's new length, back on the free list.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "halo_host.h"
#include "halo_internal.h"
#include "halo_kvq_format.h"
#include "halo_pages_device.h"

using namespace halo;

namespace {

// ---------------------------------------------------------------- which tokens stay

struct EvictArgs {
  halo_evict_sizes_t s;
  const float* weights;
  const int32_t* seq_len;
  int32_t* kept;
  float* weights_out;
  int32_t* new_len;
  int32_t* error_flag;
};

// A weight's place among all: larger weights have larger keys, NaN the lowest (0),
// and -0 that of 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  uint32_t u = __float_as_uint(w);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if (u == 0x80000000u) u = 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kListed = 4096;    // keys of one bin that are looked at in LDS

// A workgroup of W waves for each (sequence, head); wave v has tokens v * 64 R .. + 64 R - 1 of
// each chunk of 64 R W, R of them a lane, and a row of one chunk stays in its
// registers. Of the tokens between the sinks and the recent ones `left` stay. The
// left-th largest key is found from the top: the keys are counted by their first 11
// bits, and those of the bin that holds it, few as a rule, go to a list in LDS,
// which the next 11 and the last 10 bits are counted from (a bin that
// holds more is counted from the row again). Then the
// tokens are written in order: those of a larger key stay, and of those of the same
// key the first ones. A wave knows its places from what the waves before it count.
// Bound by the VALU of the CUs that have a row, of short rows by latency: 512 rows of 2048-2816 tokens 14.9 us, 32 rows of
// 40000-70000 tokens 47 (a row needs 24 instructions a token and pass, as it is passed three times).
template <int W, int R>
__global__ __launch_bounds__(64 * W) void evict_kernel(EvictArgs a) {
  constexpr int T = 64 * W, kChunk = T * R;
  __shared__ int count[kBins];
  __shared__ uint32_t list[kListed];
  __shared__ int sums[W], stay[W], same[W];
  __shared__ int found[2], listed;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, H = a.s.num_kv_heads;
  const int seq = (int)(blockIdx.x / H), h = (int)(blockIdx.x % H);
  const int len = a.seq_len[seq];
  const int64_t row = ((int64_t)seq * H + h) * a.s.width;
  const float* w = a.weights + row;
  float* out = a.weights_out + row;
  const bool bad = len < 0 || len > a.s.width;
  if (h == 0 && tid == 0) {
    a.new_len[seq] = !bad && len > a.s.trigger ? a.s.budget : len;
    if (bad && a.error_flag) a.error_flag[0] = 1;
  }
  if (bad) return;
  if (len <= a.s.trigger) {
    if (a.weights != a.weights_out)
      for (int t = tid; t < len; t += T) out[t] = w[t];
    return;
  }
  const bool one = len <= kChunk;
  const int mine = wave * 64 * R + lane;   // a lane's first token of a chunk; the others are 64 apart
  float x[R];
  // the tokens of a chunk, and those of them between the sinks and the recent ones
  int n, lo, hi;
  auto load = [&](int64_t t0) {
    const int64_t rest = len - t0;
    n = (int)min((int64_t)kChunk, rest);
    lo = (int)min(max((int64_t)a.s.sinks - t0, (int64_t)0), (int64_t)kChunk);
    hi = (int)min(max(rest - a.s.recent, (int64_t)0), (int64_t)kChunk);
    const float* at = w + t0 + mine;
    if (n == kChunk) {
#pragma unroll
      for (int i = 0; i < R; ++i) x[i] = at[64 * i];
    } else {
#pragma unroll
      for (int i = 0; i < R; ++i) x[i] = mine + 64 * i < n ? at[64 * i] : 0.f;
    }
  };
  load(0);
  int left = a.s.budget - a.s.sinks - a.s.recent;
  const bool chosen = left > 0;
  uint32_t key = 0;   // the left-th largest key
  if (chosen) {
    // counts the keys that begin with `key` above bit `top` by the bits from `shift` up to there
    auto count_row = [&](int top, int shift, int bins) {
      for (int64_t t0 = 0; t0 < len; t0 += kChunk) {
        if (!one) load(t0);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const int t = mine + 64 * i;
          const uint32_t k = weight_key(x[i]);
          if (t >= lo && t < hi && (top == 32 || (k ^ key) >> (top & 31) == 0)) atomicAdd(&count[(k >> shift) & (bins - 1)], 1);
        }
      }
    };
    int bin;
    for (int i = tid; i < kBins; i += T) count[i] = 0;
    if (tid == 0) listed = 0;
    __syncthreads();
    count_row(32, 21, kBins);
    __syncthreads();
    find_bin<W>(count, sums, found, left, bin);
    key = (uint32_t)bin << 21;
    const int in_bin = count[bin];
    const bool short_list = in_bin <= kListed;
    if (short_list) {
      for (int64_t t0 = 0; t0 < len; t0 += kChunk) {
        if (!one) load(t0);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const int t = mine + 64 * i;
          const uint32_t k = weight_key(x[i]);
          if (t >= lo && t < hi && (k ^ key) >> 21 == 0) list[atomicAdd(&listed, 1)] = k;
        }
      }
    }
#pragma unroll
    for (int step = 0; step < 2; ++step) {
      const int top = step == 0 ? 21 : 10, shift = step == 0 ? 10 : 0, bins = step == 0 ? kBins : kBins / 2;
      __syncthreads();   // (the counts have been read, the list is whole)
      for (int i = tid; i < kBins; i += T) count[i] = 0;
      __syncthreads();
      if (short_list) {
        for (int i = tid; i < in_bin; i += T) {
          const uint32_t k = list[i];
          if ((k ^ key) >> top == 0) atomicAdd(&count[(k >> shift) & (bins - 1)], 1);
        }
      } else {
        count_row(top, shift, bins);
      }
      __syncthreads();
      find_bin<W>(count, sums, found, left, bin);
      key |= (uint32_t)bin << shift;
    }
  }
  int32_t* kept = a.kept + ((int64_t)seq * H + h) * a.s.budget;
  int at = 0;   // tokens written so far; left: of the ones with the key still to take
  // Weights are ordered as floats, but for NaN: where the key is a number's, comparing with it is enough.
  const float limit = __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
  for (int64_t t0 = 0; t0 < len; t0 += kChunk) {
    if (!one) load(t0);
    // Whether all of this wave's tokens are between the sinks and the recent ones. (Rows of few chunks gain nothing
    // from a loop of its own for them: 2048 tokens 14.2 us without, 15.2 with it; 40000-70000 tokens 52.7 and 46.8.)
    const int wave_first = mine - lane;
    const bool plain = W == 16 && chosen && key != 0 && lo <= wave_first && hi >= wave_first + 64 * R;
    // what stays whatever its order, and those of the key
    int n_stay = 0, n_same = 0;
    if (plain) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        n_stay += __popcll(__ballot(x[i] > limit));
        n_same += __popcll(__ballot(x[i] == limit));
      }
    } else {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int t = mine + 64 * i;
        const uint32_t k = weight_key(x[i]);
        const bool between = t >= lo && t < hi;
        n_stay += __popcll(__ballot(t < n && (!between || (chosen && k > key))));
        n_same += __popcll(__ballot(between && chosen && k == key));
      }
    }
    if (lane == 0) {
      stay[wave] = n_stay;
      same[wave] = n_same;
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();   // (every read of this chunk has ended: in place, what is written lies before the next one)
    int to = at, rest = left;
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const int take = min(same[v], left);
      if (v < wave) {
        to += stay[v] + take;
        rest -= take;
      }
      at += stay[v] + take;
      left -= take;
    }
    auto write = [&](int i, bool keep, bool equal) {
      const uint64_t equals = __ballot(equal);
      if (equals) {
        keep |= equal && lanes_before(equals, 0) < rest;
        rest -= min((int)__popcll(equals), rest);
      }
      const uint64_t keeps = __ballot(keep);
      if (keep) {
        const int place = lanes_before(keeps, to);
        kept[place] = (int32_t)(t0 + mine + 64 * i);
        out[place] = x[i];
      }
      to += __popcll(keeps);
    };
    if (plain) {
#pragma unroll
      for (int i = 0; i < R; ++i) write(i, x[i] > limit, x[i] == limit);
    } else {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int t = mine + 64 * i;
        const uint32_t k = weight_key(x[i]);
        const bool between = t >= lo && t < hi;
        write(i, t < n && (!between || (chosen && k > key)), between && chosen && k == key);
      }
    }
    __syncthreads();   // (the counts are overwritten)
  }
}

// ---------------------------------------------------------------- moving them

struct KeepArgs {
  uint8_t* k_pool;
  uint8_t* v_pool;
  const int32_t* page_ids;
  const int32_t* seq_page_indptr;
  const int32_t* seq_len;
  const int32_t* new_len;
  const int32_t* kept;
  const int32_t* dst_page_ids;
  const int32_t* dst_page_indptr;
  int32_t* error_flag;
  int64_t num_pool_pages;
  int32_t num_seqs, num_kv_heads, kept_width;
};

// A sequence as the call gives it.
struct KeepSeq {
  int len, count, base, to;
  bool bad, whole;
  __device__ __forceinline__ KeepSeq(const KeepArgs& a, int seq) {
    len = a.seq_len[seq];
    count = a.new_len[seq];
    base = a.seq_page_indptr[seq];
    to = a.dst_page_indptr[seq];
    const int64_t have = (int64_t)(a.seq_page_indptr[seq + 1] - base) * 16;
    const int64_t room = (int64_t)(a.dst_page_indptr[seq + 1] - to) * 16;
    bad = len < 0 || count < 0 || count > len || len > have || count > room || (count < len && count > a.kept_width);
    whole = count == len;
  }
};

// One (page, head) tile of a new list, and where its 16 tokens come from: lanes 0 .. 15
// have a token each, the others repeat them. The kept indices, the source pages'
// ids and the tokens are loads that need each other, so each is a step of its own, and
// a wave takes the first ones of its next tiles before the last of this one.
struct TileSource {
  int base, len, h;
  int token;         // of the sequence; -1: none is to come here
  int page, slot;    // page -1: the place stays as it is
  int dst_page;
  bool asked;
  __device__ __forceinline__ void find_tokens(const KeepArgs& a, const KeepSeq& s, int seq, int head, int p, int lane) {
    base = s.base;
    len = s.len;
    h = head;
    dst_page = a.dst_page_ids[s.to + p];
    const int j = 16 * p + (lane & 15);
    token = j;
    if (j >= s.count) token = -1;
    else if (!s.whole) token = a.kept[((int64_t)seq * a.num_kv_heads + head) * a.kept_width + j];
    if (j < s.count && token < 0) token = -2;
  }
  __device__ __forceinline__ void find_pages(const KeepArgs& a) {
    page = -1;
    slot = token & 15;
    asked = dst_page >= 0 && dst_page < a.num_pool_pages && token >= 0 && token < len;
    if (asked) page = a.page_ids[base + token / 16];
    else if (token != -1 && a.error_flag) a.error_flag[0] = 1;
  }
  __device__ __forceinline__ void check(const KeepArgs& a) {
    if (asked && (page < 0 || page >= a.num_pool_pages)) {
      page = -1;
      if (a.error_flag) a.error_flag[0] = 1;
    }
  }
};

__device__ __forceinline__ int lane_of(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// K tiles: a token's dims lie in 16-byte units (4-bit codes: units of D / 8 bytes), a unit's 16 tokens next to
// each other. Lane (token, g) moves units g, g + 4, ... of its token.
template <typename T, bool KVQ, int D>
struct KTile {
  static constexpr int kUnit = KVQ ? D / 8 : 16;
  static constexpr int kUnits = KVQ ? 4 : D * (int)sizeof(T) / 16;
  static constexpr int kBytes = KVQ ? kvq_k_tile<D>() : 16 * D * (int)sizeof(T);
  using Unit = typename std::conditional<kUnit == 16, u32x4_t, uint64_t>::type;
  using Scale = typename std::conditional<D == 128, uint32_t, uint16_t>::type;
  Unit x[kUnits / 4];
  Scale scale;
  __device__ __forceinline__ void load(const KeepArgs& a, const TileSource& s, int lane) {
    if (s.page < 0) return;
    const uint8_t* src = a.k_pool + ((int64_t)s.page * a.num_kv_heads + s.h) * kBytes;
#pragma unroll
    for (int i = 0; i < kUnits / 4; ++i)
      x[i] = *reinterpret_cast<const Unit*>(src + (((lane >> 4) + 4 * i) * 16 + s.slot) * kUnit);
    if constexpr (KVQ) scale = reinterpret_cast<const Scale*>(src + D * 8)[s.slot];
  }
  __device__ __forceinline__ void store(const KeepArgs& a, const TileSource& s, int lane) const {
    if (s.page < 0) return;
    uint8_t* dst = a.k_pool + ((int64_t)s.dst_page * a.num_kv_heads + s.h) * kBytes;
#pragma unroll
    for (int i = 0; i < kUnits / 4; ++i)
      *reinterpret_cast<Unit*>(dst + (((lane >> 4) + 4 * i) * 16 + (lane & 15)) * kUnit) = x[i];
    if constexpr (KVQ)
      if (lane < 16) reinterpret_cast<Scale*>(dst + D * 8)[lane] = scale;
  }
};

// V tiles: a dim's 16 tokens lie next to each other, so a token is one element of
// every row, and every row of each source page is read whole. A lane has the rows of
// D / 64 dims. The tokens come from few pages, in order (a page's are next to each other): one
// after the other, the page's rows are loaded and the tokens that are in it are
// picked, the same slot in every lane, so that a row's word is chosen by a uniform index.
template <typename T, bool KVQ, int D>
struct VTile {
  static constexpr int kBytes = 16 * D * (int)sizeof(T);
  static constexpr int N = D / 64, W = 4 * (int)sizeof(T);   // rows a lane, words a row
  typedef uint32_t words_t __attribute__((ext_vector_type(W)));
  words_t x[N];
  uint64_t live;   // the tokens that come from somewhere
  // 16-byte loads and stores of a wave are contiguous. Of a bf16 tile's that gives each lane of
  // a pair a half of two rows; they swap, so that the even one has row 64 n + lane / 2 whole and
  // the odd one that row + 32.
  static __device__ __forceinline__ void swap_halves(u32x4_t& p, u32x4_t& q, bool odd) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int got = __builtin_amdgcn_update_dpp(0, (int)(odd ? p[i] : q[i]), 0xB1, 0xf, 0xf, true);   // quad_perm 1,0,3,2
      p[i] = odd ? (uint32_t)got : p[i];
      q[i] = odd ? q[i] : (uint32_t)got;
    }
  }
  static __device__ __forceinline__ void load_rows(const uint8_t* tile, int lane, words_t (&y)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if constexpr (sizeof(T) == 2) {
        u32x4_t p = reinterpret_cast<const u32x4_t*>(tile)[128 * n + lane];
        u32x4_t q = reinterpret_cast<const u32x4_t*>(tile)[128 * n + 64 + lane];
        swap_halves(p, q, lane & 1);
        y[n] = __builtin_shufflevector(p, q, 0, 1, 2, 3, 4, 5, 6, 7);
      } else {
        y[n] = reinterpret_cast<const words_t*>(tile)[64 * n + lane];
      }
    }
  }
  __device__ __forceinline__ void load(const KeepArgs& a, const TileSource& s, int lane) {
    live = __ballot(s.page >= 0) & 0xffff;
    if (!live) return;
    // (slots that get no token keep what they hold)
    if (live != 0xffff) load_rows(a.v_pool + ((int64_t)s.dst_page * a.num_kv_heads + s.h) * kBytes, lane, x);
    uint64_t rest = live;
    while (rest) {
      const int page = lane_of(s.page, __builtin_ctzll(rest));
      const uint64_t here = __ballot(s.page == page) & rest;
      rest &= ~here;
      words_t y[N];
      load_rows(a.v_pool + ((int64_t)page * a.num_kv_heads + s.h) * kBytes, lane, y);
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        if (!(here >> t & 1)) continue;
        const int from = v_token_at_slot(lane_of(s.slot, t));   // (the map is its own inverse)
        const int to = (t & 3) | ((t & 4) << 1) | ((t & 8) >> 1);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int n = 0; n < N; ++n) x[n][to] = y[n][from];
        } else {
          // half `from & 1` of a word becomes half `to & 1` of another
          const uint32_t pick = to & 1 ? (from & 1 ? 0x07060100u : 0x05040100u) : (from & 1 ? 0x03020706u : 0x03020504u);
#pragma unroll
          for (int n = 0; n < N; ++n) x[n][to / 2] = __builtin_amdgcn_perm(y[n][from / 2], x[n][to / 2], pick);
        }
      }
    }
  }
  __device__ __forceinline__ void store(const KeepArgs& a, const TileSource& s, int lane) const {
    if (!live) return;
    uint8_t* dst = a.v_pool + ((int64_t)s.dst_page * a.num_kv_heads + s.h) * kBytes;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if constexpr (sizeof(T) == 2) {
        u32x4_t p = __builtin_shufflevector(x[n], x[n], 0, 1, 2, 3), q = __builtin_shufflevector(x[n], x[n], 4, 5, 6, 7);
        swap_halves(p, q, lane & 1);
        reinterpret_cast<u32x4_t*>(dst)[128 * n + lane] = p;
        reinterpret_cast<u32x4_t*>(dst)[128 * n + 64 + lane] = q;
      } else {
        reinterpret_cast<words_t*>(dst)[64 * n + lane] = x[n];
      }
    }
  }
};

// 4-bit values: a word holds the codes of 8 slots of a dim, [D / 64][half][64 dims]. Of
// every token the words of its half are loaded, all at once, and its code put into
// place; a place that stays takes its own.
template <typename T, int D>
struct VTile<T, true, D> {
  static constexpr int kBytes = kvq_v_tile<D>();
  static constexpr int N = D / 64;
  uint32_t x[N][2];
  uint16_t scale;
  bool any;
  __device__ __forceinline__ void load(const KeepArgs& a, const TileSource& s, int lane) {
    any = __ballot(s.page >= 0) != 0;
    if (!any) return;
    const int page = s.page >= 0 ? s.page : s.dst_page, slot = s.page >= 0 ? s.slot : lane & 15;
    scale = reinterpret_cast<const uint16_t*>(a.v_pool + ((int64_t)page * a.num_kv_heads + s.h) * kBytes + D * 8)[v_token_at_slot(slot)];
    uint32_t y[16][N];
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const uint8_t* src = a.v_pool + ((int64_t)lane_of(page, t) * a.num_kv_heads + s.h) * kBytes;
      const int half = v_token_at_slot(lane_of(slot, t)) >> 3;
#pragma unroll
      for (int n = 0; n < N; ++n) y[t][n] = reinterpret_cast<const uint32_t*>(src)[(2 * n + half) * 64 + lane];
    }
#pragma unroll
    for (int n = 0; n < N; ++n) x[n][0] = x[n][1] = 0;
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      const int from = 4 * (v_token_at_slot(lane_of(slot, t)) & 7);
      const int to = (t & 3) | ((t & 4) << 1) | ((t & 8) >> 1);
#pragma unroll
      for (int n = 0; n < N; ++n) x[n][to >> 3] |= (y[t][n] >> from & 15) << (4 * (to & 7));
    }
  }
  __device__ __forceinline__ void store(const KeepArgs& a, const TileSource& s, int lane) const {
    if (!any) return;
    uint8_t* dst = a.v_pool + ((int64_t)s.dst_page * a.num_kv_heads + s.h) * kBytes;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int half = 0; half < 2; ++half) reinterpret_cast<uint32_t*>(dst)[(2 * n + half) * 64 + lane] = x[n][half];
    if (lane < 16) reinterpret_cast<uint16_t*>(dst + D * 8)[v_token_at_slot(lane)] = scale;
  }
};

// To other pages: the new lists' (slot, head) tiles are cut into equal runs, one a
// wave, as in the gather; every other wave moves K tiles, the others V tiles. The ids of the
// next two tiles are on their way while one is moved. Bound by HBM, and by what is read of the source pages for tokens
// that are not kept: 64 sequences of 2048-2816 bf16 tokens to 2048, 8 heads of d 128, 1.08 GB moved, 272 us (4.0 TB/s);
// 4 of 40000-70000 4-bit tokens to 8192, of a page's 16 about 3 kept, 51 us.
template <typename T, bool KVQ, int D>
__global__ __launch_bounds__(256) void keep_kernel(KeepArgs a) {
  const int lane = threadIdx.x & 63, H = a.num_kv_heads;
  const int first = a.dst_page_indptr[0];
  const int64_t total = ((int64_t)a.dst_page_indptr[a.num_seqs] - first) * H;
  const int64_t waves = (int64_t)gridDim.x * 2, wave = (int64_t)blockIdx.x * 2 + (threadIdx.x >> 7);
  const bool values = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 1;
  const int64_t per = (total + waves - 1) / waves;
  const int64_t begin = wave * per;
  int64_t left = min(total, begin + per) - begin;   // tiles of the run that are still to come
  if (blockIdx.x == 0 && threadIdx.x < 64) {
    // (a malformed sequence may have no new page to be found by)
    for (int i = lane; i < a.num_seqs; i += 64)
      if (KeepSeq(a, i).bad && a.error_flag) a.error_flag[0] = 1;
  }
  if (left <= 0) return;
  int slot = first + (int)(begin / H), h = (int)(begin % H) - 1;
  int seq = last_at_or_below(a.dst_page_indptr, a.num_seqs, slot, lane), next = a.dst_page_indptr[seq + 1];
  KeepSeq s(a, seq);
  // goes to the run's next tile that gets a token
  auto advance = [&] {
    while (left-- > 0) {
      if (++h == H) {
        h = 0;
        ++slot;
      }
      if (slot >= next) {
        while (slot >= next) next = a.dst_page_indptr[++seq + 1];   // (ends at num_seqs - 1)
        s = KeepSeq(a, seq);
      }
      if (!s.bad && (int64_t)(slot - s.to) * 16 < s.count) return true;
    }
    return false;
  };
  TileSource now, soon, then;
  bool has_now = false, has_soon = false, has_then = true;
  while (has_now || has_soon || has_then) {
    if (has_then) has_then = advance();
    if (has_then) then.find_tokens(a, s, seq, h, slot - s.to, lane);
    if (has_soon) soon.find_pages(a);
    if (has_now) {
      now.check(a);
      if (values) {
        VTile<T, KVQ, D> v;
        v.load(a, now, lane);
        v.store(a, now, lane);
      } else {
        KTile<T, KVQ, D> k;
        k.load(a, now, lane);
        k.store(a, now, lane);
      }
    }
    now = soon;
    soon = then;
    has_now = has_soon;
    has_soon = has_then;
  }
}

// In place: a workgroup for each (sequence, head, pool) goes through the pages in order, a
// page a wave. Kept indices are ascending, so a page reads only what lies at it or
// behind it: the pages of one round are loaded, and stored when all are; what the next
// round reads lies behind all of these. Bound by HBM where there are sequences enough (64 of 2500 bf16 tokens to
// 2048: 264 us, 4-bit 87), by the rounds' waits where there are few (4 of 65000 4-bit tokens to 8192: 107 us, bf16 413).
constexpr int kInPlaceWaves = 16;
template <typename T, bool KVQ, int D>
__global__ __launch_bounds__(64 * kInPlaceWaves) void keep_in_place_kernel(KeepArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, H = a.num_kv_heads;
  const int z = (int)(blockIdx.x % 2), h = (int)(blockIdx.x / 2 % H), seq = (int)(blockIdx.x / 2 / H);
  const KeepSeq s(a, seq);
  if (s.bad) {
    if (threadIdx.x == 0 && a.error_flag) a.error_flag[0] = 1;
    return;
  }
  if (s.whole) return;
  auto move = [&](auto tile) {
    for (int64_t p0 = 0; p0 * 16 < s.count; p0 += kInPlaceWaves) {
      const int64_t p = p0 + wave;
      const bool mine = p * 16 < s.count;
      TileSource src;
      if (mine) {
        src.find_tokens(a, s, seq, h, (int)p, lane);
        src.find_pages(a);
        src.check(a);
        tile.load(a, src, lane);
      }
      __builtin_amdgcn_s_waitcnt(0x0f70);   // every load has ended, not only begun
      __syncthreads();
      if (mine) tile.store(a, src, lane);
    }
  };
  if (z == 0) move(KTile<T, KVQ, D>{});
  else move(VTile<T, KVQ, D>{});
}

// ---------------------------------------------------------------- pages given back

struct ReleaseArgs {
  const int32_t* block_table;
  const int32_t* seq_len;
  const int32_t* new_len;
  const int32_t* free_pages;
  const int32_t* free_next;
  int32_t* free_pages_out;
  int32_t* free_next_out;
  int32_t* error_flag;
  int32_t num_seqs, table_width, num_free;
  int32_t per;      // sequences of a group
  int32_t splits;   // workgroups of a group, which share its rows
};

__device__ __forceinline__ uint32_t sum_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

// A sequence's pages that go: from `first`, `count` of them.
struct Released {
  int first, count;
  bool bad;
  __device__ __forceinline__ Released(const ReleaseArgs& a, int i) {
    const int len = a.seq_len[i], now = a.new_len[i];
    bad = now < 0 || len < now || (int64_t)len > (int64_t)a.table_width * 16;
    first = bad ? 0 : (int)(((int64_t)now + 15) >> 4);
    count = bad ? 0 : (int)(((int64_t)len + 15) >> 4) - first;
  }
};

// As the step tables: every workgroup sums over all sequences itself (8 bytes
// each), so there is one launch and no wait between workgroups. Bound by latency: 2.6 us for 4 sequences, 4.8 for 64
// that give back up to 48 pages each.
__global__ __launch_bounds__(256) void release_kernel(ReleaseArgs a) {
  __shared__ uint32_t sums[4][3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int group = (int)blockIdx.x / a.splits, split = (int)blockIdx.x % a.splits;
  const int first = (int)min((int64_t)a.num_seqs, (int64_t)group * a.per);
  const int last = (int)min((int64_t)a.num_seqs, (int64_t)first + a.per);
  uint32_t s[3] = {0, 0, 0};   // pages before the group, of all; malformed ones
  for (int64_t i = tid; i < a.num_seqs; i += 256) {
    const Released r(a, (int)i);
    s[1] = sum_sat(s[1], r.count);
    s[2] |= r.bad ? 1u : 0u;
    if (i < first) s[0] = sum_sat(s[0], r.count);
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s[k] = sum_sat(s[k], __shfl_xor(s[k], m));
    if (lane == 0) sums[wave][k] = s[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) s[k] = sum_sat(sum_sat(sums[0][k], sums[1][k]), sum_sat(sums[2][k], sums[3][k]));
  const int next = a.free_next[0];
  const bool in = next >= 0 && next <= a.num_free;
  const bool fits = in && s[1] <= (uint32_t)next;
  if (blockIdx.x == 0 && tid == 0) {
    a.free_next_out[0] = fits ? next - (int)s[1] : next;
    if ((s[2] || !fits) && a.error_flag) a.error_flag[0] = 1;
  }
  if (fits) {
    int64_t at = (int64_t)next - s[1] + s[0];
    for (int i = first; i < last; ++i) {
      const Released r(a, i);
      const int32_t* row = a.block_table + (int64_t)i * a.table_width + r.first;
      for (int j = split * 256 + tid; j < r.count; j += a.splits * 256) a.free_pages_out[at + j] = row[j];
      at += r.count;
    }
  }
  if (in && a.free_pages_out != a.free_pages)
    for (int64_t j = (int64_t)next + (int64_t)blockIdx.x * 256 + tid; j < a.num_free; j += (int64_t)gridDim.x * 256)
      a.free_pages_out[j] = a.free_pages[j];
}

// ---------------------------------------------------------------- host side

halo_status_t page_keep(bool kvq, void* k_pool, void* v_pool, const halo_attn_params_t* params, const int32_t* page_ids,
                        const int32_t* seq_page_indptr, const int32_t* seq_len, const int32_t* new_len,
                        const int32_t* kept, int32_t kept_width, const int32_t* dst_page_ids,
                        const int32_t* dst_page_indptr, int32_t num_seqs, int32_t* error_flag, void* stream) {
  clear_error();
  if (!params) return fail(HALO_ERR_INVALID_ARGUMENT, "params must not be NULL");
  if (num_seqs < 0 || kept_width < 0) return fail(HALO_ERR_INVALID_ARGUMENT, "num_seqs and kept_width must be >= 0");
  const halo_status_t st = check_cache_params(params);
  if (st != HALO_OK) return st;
  if (num_seqs == 0) return HALO_OK;
  if (!k_pool || !v_pool || !page_ids || !seq_page_indptr || !seq_len || !new_len || (!kept && kept_width > 0) ||
      !dst_page_ids || !dst_page_indptr)
    return fail(HALO_ERR_INVALID_ARGUMENT, "k_pool, v_pool, page_ids, seq_page_indptr, seq_len, new_len, kept, "
                                           "dst_page_ids, dst_page_indptr must not be NULL");
  if (!aligned16(k_pool) || !aligned16(v_pool)) return fail(HALO_ERR_INVALID_ARGUMENT, "pools must be 16-byte aligned");
  if ((dst_page_ids == page_ids) != (dst_page_indptr == seq_page_indptr))
    return fail(HALO_ERR_INVALID_ARGUMENT, "in place, both dst_page_ids and dst_page_indptr are those of the sequences");
  const int64_t blocks = (int64_t)num_seqs * params->num_kv_heads * 2;
  if (blocks > 1 << 24) return fail(HALO_ERR_UNSUPPORTED, "num_seqs * num_kv_heads must be at most 2^23");
  const bool in_place = dst_page_ids == page_ids;
  if (in_place && blocks * 64 * kInPlaceWaves > UINT32_MAX)   // (threads of a launch)
    return fail(HALO_ERR_UNSUPPORTED, "in place, num_seqs * num_kv_heads must be less than 2^21");
  KeepArgs g{static_cast<uint8_t*>(k_pool), static_cast<uint8_t*>(v_pool), page_ids, seq_page_indptr, seq_len, new_len,
             kept, dst_page_ids, dst_page_indptr, error_flag, params->num_pool_pages, num_seqs, params->num_kv_heads,
             kept_width};
  (void)hipGetLastError();
  by_type_and_dim(params, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    using W = typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type;
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto launch = [&](auto t, auto kvq) {
      using U = decltype(t);
      constexpr bool Q = decltype(kvq)::value;
      if (in_place)
        hipLaunchKernelGGL((keep_in_place_kernel<U, Q, D>), dim3((unsigned)blocks), dim3(64 * kInPlaceWaves), 0, s, g);
      else
        hipLaunchKernelGGL((keep_kernel<U, Q, D>), dim3(4096), dim3(256), 0, s, g);
    };
    if (kvq) launch(uint8_t{}, std::true_type{});
    else launch(W{}, std::false_type{});
  });
  return hip_check("keep launch");
}

}  // namespace

extern "C" halo_status_t halo_kv_evict_select(const halo_evict_sizes_t* sizes, const float* weights,
                                              const int32_t* seq_len, int32_t* kept, float* weights_out,
                                              int32_t* new_len, int32_t* error_flag, void* stream) {
  clear_error();
  if (!sizes) return fail(HALO_ERR_INVALID_ARGUMENT, "sizes must not be NULL");
  if (sizes->num_seqs < 0 || sizes->width < 0 || sizes->sinks < 0 || sizes->recent < 0)
    return fail(HALO_ERR_INVALID_ARGUMENT, "num_seqs, width, sinks and recent must be >= 0");
  if (sizes->num_kv_heads < 1 || sizes->budget < 1)
    return fail(HALO_ERR_INVALID_ARGUMENT, "num_kv_heads and budget must be >= 1");
  if ((int64_t)sizes->sinks + sizes->recent > sizes->budget || sizes->trigger < sizes->budget)
    return fail(HALO_ERR_INVALID_ARGUMENT, "sinks + recent must be <= budget, and trigger >= budget");
  const int64_t n = sizes->num_seqs, rows = n * sizes->num_kv_heads;
  const bool long_rows = sizes->width > 4096;
  if (rows * (long_rows ? 1024 : 256) > UINT32_MAX)   // (threads of a launch)
    return fail(HALO_ERR_UNSUPPORTED, "num_seqs * num_kv_heads must be less than 2^24, of rows of more than 4096 tokens 2^22");
  if (n == 0) return HALO_OK;
  if (!seq_len || !kept || !new_len || (sizes->width > 0 && (!weights || !weights_out)))
    return fail(HALO_ERR_INVALID_ARGUMENT, "weights, seq_len, kept, weights_out, new_len must not be NULL");
  const halo_status_t lap = check_overlaps(
      {{"weights", weights == weights_out ? nullptr : weights, rows * sizes->width * 4}, {"seq_len", seq_len, 4 * n}},
      {{"kept", kept, rows * sizes->budget * 4}, {"weights_out", weights_out, rows * sizes->width * 4},
       {"new_len", new_len, 4 * n}, {"error_flag", error_flag, 4}});
  if (lap != HALO_OK) return lap;
  EvictArgs g{*sizes, weights, seq_len, kept, weights_out, new_len, error_flag};
  (void)hipGetLastError();
  // as many tokens in registers as the rows may hold
  auto launch = [&](auto waves, auto per_lane) {
    constexpr int W = decltype(waves)::value, R = decltype(per_lane)::value;
    hipLaunchKernelGGL((evict_kernel<W, R>), dim3((unsigned)rows), dim3(64 * W), 0, static_cast<hipStream_t>(stream), g);
  };
  if (sizes->width <= 1024) launch(std::integral_constant<int, 4>{}, std::integral_constant<int, 4>{});
  else if (!long_rows) launch(std::integral_constant<int, 4>{}, std::integral_constant<int, 16>{});
  else launch(std::integral_constant<int, 16>{}, std::integral_constant<int, 16>{});
  return hip_check("evict launch");
}

extern "C" halo_status_t halo_kv_page_keep_kv(void* k_pool, void* v_pool, const halo_attn_params_t* params,
                                              const int32_t* page_ids, const int32_t* seq_page_indptr,
                                              const int32_t* seq_len, const int32_t* new_len, const int32_t* kept,
                                              int32_t kept_width, const int32_t* dst_page_ids,
                                              const int32_t* dst_page_indptr, int32_t num_seqs, int32_t* error_flag,
                                              void* stream) {
  return page_keep(false, k_pool, v_pool, params, page_ids, seq_page_indptr, seq_len, new_len, kept, kept_width,
                   dst_page_ids, dst_page_indptr, num_seqs, error_flag, stream);
}

extern "C" halo_status_t halo_kvq_page_keep_kv(void* k_pool, void* v_pool, const halo_attn_params_t* params,
                                               const int32_t* page_ids, const int32_t* seq_page_indptr,
                                               const int32_t* seq_len, const int32_t* new_len, const int32_t* kept,
                                               int32_t kept_width, const int32_t* dst_page_ids,
                                               const int32_t* dst_page_indptr, int32_t num_seqs, int32_t* error_flag,
                                               void* stream) {
  return page_keep(true, k_pool, v_pool, params, page_ids, seq_page_indptr, seq_len, new_len, kept, kept_width,
                   dst_page_ids, dst_page_indptr, num_seqs, error_flag, stream);
}

extern "C" halo_status_t halo_kv_release_pages(const halo_step_sizes_t* sizes, const int32_t* block_table,
                                               const int32_t* seq_len, const int32_t* new_len,
                                               const int32_t* free_pages, const int32_t* free_next,
                                               int32_t* free_pages_out, int32_t* free_next_out, int32_t* error_flag,
                                               void* stream) {
  clear_error();
  if (!sizes) return fail(HALO_ERR_INVALID_ARGUMENT, "sizes must not be NULL");
  if (sizes->num_seqs < 0 || sizes->table_width < 0 || sizes->num_free < 0)
    return fail(HALO_ERR_INVALID_ARGUMENT, "every size must be >= 0");
  if (sizes->page_size != 16) return fail(HALO_ERR_UNSUPPORTED, "page_size must be 16");
  const int64_t n = sizes->num_seqs;
  if (!free_next || !free_next_out || (n > 0 && (!seq_len || !new_len)) ||
      (n > 0 && sizes->table_width > 0 && !block_table) || (sizes->num_free > 0 && (!free_pages || !free_pages_out)))
    return fail(HALO_ERR_INVALID_ARGUMENT, "only error_flag (and arrays of no elements) may be NULL");
  const halo_status_t lap = check_overlaps(
      {{"block_table", block_table, 4 * n * sizes->table_width}, {"seq_len", seq_len, 4 * n},
       {"new_len", new_len, 4 * n}, {"free_next", free_next, 4},
       {"free_pages", free_pages == free_pages_out ? nullptr : free_pages, 4 * (int64_t)sizes->num_free}},
      {{"free_pages_out", free_pages_out, 4 * (int64_t)sizes->num_free}, {"free_next_out", free_next_out, 4},
       {"error_flag", error_flag, 4}});
  if (lap != HALO_OK) return lap;
  // up to 256 groups of sequences, and more workgroups for one where rows or the
  // list are long and sequences few
  const int groups = std::min(std::max((int)n, 1), kNumCUs);
  ReleaseArgs g{block_table, seq_len, new_len, free_pages, free_next, free_pages_out, free_next_out, error_flag,
                sizes->num_seqs, sizes->table_width, sizes->num_free, (int)((n + groups - 1) / groups), 1};
  const int64_t longest = std::max<int64_t>((sizes->table_width + 511) / 512, sizes->num_free / 512 / groups);
  g.splits = (int)std::max<int64_t>(1, std::min<int64_t>(longest, kNumCUs / groups));
  (void)hipGetLastError();
  hipLaunchKernelGGL(release_kernel, dim3(groups * g.splits), dim3(256), 0, static_cast<hipStream_t>(stream), g);
  return hip_check("release launch");
}
