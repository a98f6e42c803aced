// gfx950 kernels and entry points of the C ABI for beam search:
// beam_scan_kernel, beam_pick_kernel: the best candidates (beam, token) of each
//   request by score + logit - ln sum exp(logits);
// beam_freed_kernel, beam_rows_kernel: the beams' rows of the page table follow
//   their parents.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "halo_host.h"
#include "halo_internal.h"
#include "halo_pages_device.h"

using namespace halo;

namespace {

constexpr int kMaxBeams = 64;
constexpr int kMaxBest = 64;
constexpr int kMaxVocab = 1 << 24;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kMinusInf = -__builtin_huge_valf();

// ---------------------------------------------------------------- one pass over the logits

// What a wave found in its part of a row.
struct BeamPart {
  float top;    // the largest logit, or the lowest finite number
  double sum;   // of exp(logit - top)
};
struct Candidate {
  float value;
  int32_t token;   // -1: none
};

struct BeamArgs {
  const void* logits;
  const float* scores;
  const int32_t* ended;
  BeamPart* parts;         // [rows][parts]
  Candidate* candidates;   // [rows][parts][best]
  float* out_scores;
  int32_t* out_tokens;
  int32_t* out_parents;
  int64_t stride;
  int32_t beams, vocab, best, end_token;
  int32_t per;             // elements of a part, a multiple of 512
  int32_t num_parts;
};

__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ bool is_finite(double x) {
  return ((uint64_t)__double_as_longlong(x) & 0x7ff0000000000000ull) != 0x7ff0000000000000ull;
}
// Larger numbers have larger keys; of -0 and 0 the same.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_order_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// A number that at least n of the wave's N keys a lane are no smaller than (0 if there
// are fewer keys), and as few more as ties allow: the n-th largest key, or one between it and the
// next smaller. Bit by bit from the top, from the keys' ballots, until it is as
// good (or, of the upper bits alone, no larger than that).
template <int LOWEST_BIT = 0, int N>
__device__ __forceinline__ uint32_t wave_nth_key(const uint32_t (&key)[N], int n) {
  uint32_t t = 0;
  for (int bit = 31; bit >= LOWEST_BIT; --bit) {
    const uint32_t next = t | 1u << bit;
    int c = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) c += __popcll(__ballot(key[j] >= next));
    if (c >= n) t = next;
    if (c == n) break;
  }
  return t;
}

// LDS that a wave alone writes and reads: what was written can be read by its other lanes.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kBoundBit = 14;    // of a bound on logits the bits from here on
constexpr int kTile = 512;       // elements a wave looks at together
// Candidates a wave holds. (Of rows in any order 64 best need about 800 places until the part ends, 16 best 230: 64 of
// 16 x 16 rows of 128256 bf16 logits take 97 us with 640 places, 78 with 1024; 32 of them 44 and 50, as more registers and
// LDS leave fewer waves; 64 of 8 x 64 rows of 32000 fp32 logits, parts of 8 tiles, 37 and 47.)
constexpr int kListCap = 640, kLongListCap = 1024, kLongListFrom = 33, kLongPart = 16 * kTile;

// Keeps the `best` first of the list's n candidates (by value, then token), N a lane.
template <int N>
__device__ __forceinline__ int prune_of(float* value, int32_t* token, int n, int best, int lane) {
  uint32_t key[N], id[N];   // (larger: earlier)
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = 64 * j + lane;
    key[j] = i < n ? order_key(value[i]) : 0;
    id[j] = i < n ? ~(uint32_t)token[i] : 0;
  }
  const uint32_t least = wave_nth_key(key, best);
  int count = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) count += __popcll(__ballot(key[j] >= least));
  uint32_t last = 0;   // of the candidates at `least` those of this id and larger ones
  if (count > best) {  // (then `least` is a key, and these are ties)
    uint32_t of_ties[N];
    int above = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      above += __popcll(__ballot(key[j] > least));
      of_ties[j] = key[j] == least ? id[j] : 0;
    }
    last = wave_nth_key(of_ties, best - above);
  }
  int at = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const bool keep = key[j] > least || (key[j] == least && id[j] >= last);
    const uint64_t mask = __ballot(keep);
    if (keep) {
      const int to = lanes_before(mask, at);
      value[to] = from_order_key(key[j]);
      token[to] = (int32_t)~id[j];
    }
    at += __popcll(mask);
  }
  return at;
}
template <int CAP>
__device__ __forceinline__ int prune(float* value, int32_t* token, int n, int best, int lane) {
  wave_lds_fence();
  if (n > best) {
    if (n <= 64) n = prune_of<1>(value, token, n, best, lane);
    else if (n <= 128) n = prune_of<2>(value, token, n, best, lane);
    else n = prune_of<CAP / 64>(value, token, n, best, lane);
    wave_lds_fence();
  }
  return n;
}

// Elements x[0 .. 511] of a row, eight a lane, of which those from n on are -inf. Loads
// are of 16 bytes at any alignment of the row, so that which lane adds what goes by
// the token alone: two beams of the same logits have the same sum.
template <typename T>
struct Tile {
  static constexpr int E = 16 / (int)sizeof(T);
  T w[8];
  __device__ __forceinline__ void load(const T* x, int64_t n, int lane) {
    if (n >= kTile) {
#pragma unroll
      for (int u = 0; u < 8 / E; ++u) __builtin_memcpy(w + u * E, x + (u * 64 + lane) * E, 16);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = place(k, lane) < n ? x[place(k, lane)] : (T)kMinusInf;
    }
  }
  // place of a lane's element k in the tile
  static __device__ __forceinline__ int place(int k, int lane) { return ((k / E) * 64 + lane) * E + k % E; }
};

// A wave passes its part of a row once. A lane follows the largest of its logits and
// the sum of their exponentials (fp32; the lanes' are joined in 64 bits). Candidates go to a
// list in LDS: those at or above the best-th largest lane maximum, since as many lanes have
// seen one; it is found anew after 1, 2, 4, 8, ... tiles, so that of a part in any order about
// `best` more are listed each time the part seen doubles. A full list is cut to the
// first `best`; then only what is above the last of these counts (ties with it are later tokens).
// Bound by HBM: 1024 rows of 200019 fp32 logits, 819 MB, 16 best, 138 us (5.9 TB/s); with fewer tiles a wave by its start
// and end: 256 rows of 128256 bf16 logits, 66 MB, 8 best, 23 us.
template <typename T, int CAP>
__global__ __launch_bounds__(256) void beam_scan_kernel(BeamArgs a) {
  __shared__ float list_value[4][CAP];
  __shared__ int32_t list_token[4][CAP];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int row = (int)blockIdx.y, part = (int)blockIdx.x * 4 + wave;
  if (part >= a.num_parts) return;
  BeamPart* out = a.parts + (int64_t)row * a.num_parts + part;
  // (a beam that has ended or is dead: its logits are not looked at)
  if ((a.ended && a.ended[row]) || !is_finite(a.scores[row])) return;
  const T* x = static_cast<const T*>(a.logits) + (int64_t)row * a.stride;
  const int64_t begin = (int64_t)part * a.per, end = min(begin + a.per, (int64_t)a.vocab);
  float* value = list_value[wave];
  int32_t* token = list_token[wave];
  float top = kLowest, sum = 0.f, bound = kMinusInf;
  int n = 0, seen = 0, renew = 1;
  Tile<T> now, next, then;
  if (begin < end) now.load(x + begin, end - begin, lane);
  if (begin + kTile < end) next.load(x + begin + kTile, end - begin - kTile, lane);
  for (int64_t t = begin; t < end; t += kTile) {
    if (t + 2 * kTile < end) then.load(x + t + 2 * kTile, end - t - 2 * kTile, lane);
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)now.w[k];
    float most = v[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) most = fmaxf(most, v[k]);
    const float high = fmaxf(top, most);
    sum *= __builtin_amdgcn_exp2f((top - high) * 1.44269504088896340736f);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += __builtin_amdgcn_exp2f((v[k] - high) * 1.44269504088896340736f);
    top = high;
    if (++seen == renew) {
      renew *= 2;
      // just below the best-th largest lane maximum, as long as that is no lane without a logit
      const uint32_t key[1] = {order_key(top)};
      uint32_t k = wave_nth_key<kBoundBit>(key, a.best);
      if (k > order_key(kLowest)) {
        if (--k == order_key(0.f) - 1) --k;   // (the key of -0)
        bound = fmaxf(bound, from_order_key(k));
      }
    }
    if (__any(most > bound)) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const bool hit = v[k] > bound;
        const uint64_t mask = __ballot(hit);
        if (mask) {
          if (hit) {
            const int to = lanes_before(mask, n);
            value[to] = v[k];
            token[to] = (int32_t)t + Tile<T>::place(k, lane);
          }
          n += __popcll(mask);
        }
      }
      if (n > CAP - kTile) {
        n = prune<CAP>(value, token, n, a.best, lane);
        if (n >= a.best) {
          float least = -kMinusInf;
          for (int i = lane; i < n; i += 64) least = fminf(least, value[i]);
#pragma unroll
          for (int m = 32; m >= 1; m >>= 1) least = fminf(least, __shfl_xor(least, m));
          bound = fmaxf(bound, least);
        }
      }
    }
    now = next;
    next = then;
  }
  n = prune<CAP>(value, token, n, a.best, lane);
  Candidate* c = a.candidates + ((int64_t)row * a.num_parts + part) * a.best;
  for (int i = lane; i < a.best; i += 64) c[i] = i < n ? Candidate{value[i], token[i]} : Candidate{kMinusInf, -1};
  float most = top;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
  double s = (double)sum * exp2(((double)top - (double)most) * 1.44269504088896340736);
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
  if (lane == 0) *out = BeamPart{most, s};
}

// ---------------------------------------------------------------- the best of an item

__device__ __forceinline__ uint64_t order_key(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return u & 0x8000000000000000ull ? ~u : u | 0x8000000000000000ull;
}
__device__ __forceinline__ double from_order_key(uint64_t k) {
  return __longlong_as_double((long long)(k & 0x8000000000000000ull ? k & 0x7fffffffffffffffull : ~k));
}

constexpr int kPickCap = 512;    // candidates that are put in order together
// Candidates of an item that workgroups of 16 waves are taken from on (16 beams of 16 parts with 16 best, 4096: 24.5 us
// by 4 waves, 12 by 16).
constexpr int kManyCandidates = 2048;
constexpr uint64_t kLastId = (1ull << 38) - 1;   // ids: beam, token

struct Ranked {
  uint64_t key, id;   // larger keys first, then smaller ids
};

// A workgroup of NW waves for each item. ln sum exp of every beam comes from its parts. Of the beams'
// candidates those at or above a bound go to a list in LDS, and each one's place is how
// many of the list come before it. The bound: of each wave's lane maxima the best-th largest
// one (in the upper 32 bits), of the waves' the largest. Where the list does not hold them all, the candidates
// from the bound up are counted in 2048 equal parts of their range, then those of the part that holds the last one
// of the best, and so on, of equal keys by their ids, until what is left fits. Bound by latency: 4 beams of 16 parts with
// 8 best 6.9 us; 16 beams of 16 parts with 64 best, 16384 candidates, 54 us (a round for each of the best: 2100).
template <int NW>
__global__ __launch_bounds__(64 * NW) void beam_pick_kernel(BeamArgs a) {
  constexpr int T = 64 * NW;
  // ln sum exp of a beam's logits is top + ln_sum, not added: of logits of 1e20 the sum would be top
  __shared__ double ln_sum[kMaxBeams];
  __shared__ float top_of[kMaxBeams];
  __shared__ int32_t live[kMaxBeams];   // 0 dead, 1 live, 2 ended
  __shared__ __align__(16) Ranked list[kPickCap];
  __shared__ int count[kBins];
  __shared__ int sums[NW], found[2];
  __shared__ uint32_t bounds[NW], tops[NW];
  __shared__ int32_t listed;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int item = (int)blockIdx.x, W = a.beams, P = a.num_parts;
  if (tid == 0) listed = 0;
  for (int b = wave; b < W; b += NW) {
    const int row = item * W + b;
    const BeamPart* parts = a.parts + (int64_t)row * P;
    const bool open = is_finite(a.scores[row]);
    const bool ended = a.ended && a.ended[row];
    const bool read = open && !ended;   // (its parts are written)
    float most = kLowest;
    for (int p = lane; p < P; p += 64) most = fmaxf(most, read ? parts[p].top : kLowest);
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) most = fmaxf(most, __shfl_xor(most, m));
    double s = 0;
    for (int p = lane; p < P; p += 64)
      s += read ? parts[p].sum * exp2(((double)parts[p].top - (double)most) * 1.44269504088896340736) : 0;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if (lane == 0) {
      // (a NaN or +inf among the logits makes the sum no number)
      const bool sound = is_finite(s) && s > 0 && is_finite(most);
      top_of[b] = most;
      ln_sum[b] = sound ? log(s) : 0;
      live[b] = !open ? 0 : ended ? 2 : sound ? 1 : 0;
    }
  }
  __syncthreads();
  const int per_row = P * a.best, all = W * per_row;
  // A candidate's key (larger: better; 0: none) and, of equal keys, its order.
  auto candidate = [&](int i, uint64_t& key, uint64_t& id) {
    const bool in = i < all;
    i = in ? i : 0;
    const int b = i / per_row, j = i - b * per_row;
    const int row = item * W + b, how = live[b];
    const Candidate x = a.candidates[(int64_t)row * per_row + j];   // (of a beam that is not live: anything)
    const double score = (double)a.scores[row];
    const bool of_live = in && how == 1 && x.token >= 0, of_ended = in && how == 2 && j == 0;
    key = order_key(of_ended ? score : (((double)x.value - (double)top_of[b]) - ln_sum[b]) + score);
    if (!of_live && !of_ended) key = 0;
    id = (uint64_t)b << 32 | (uint32_t)(of_ended ? a.end_token : x.token);
  };
  // each(key, id) of this thread's candidates, R of which it keeps; more are looked up again, several at once
  constexpr int R = 4;
  uint64_t keys[R], ids[R];
#pragma unroll
  for (int j = 0; j < R; ++j) candidate(tid + T * j, keys[j], ids[j]);
  auto pass = [&](auto each) {
#pragma unroll
    for (int j = 0; j < R; ++j) each(keys[j], ids[j]);
    for (int i = tid + T * R; i < all; i += T * R) {
      uint64_t k[R], d[R];
#pragma unroll
      for (int j = 0; j < R; ++j) candidate(i + T * j, k[j], d[j]);
#pragma unroll
      for (int j = 0; j < R; ++j) each(k[j], d[j]);
    }
  };
  uint32_t most[1] = {0};
  pass([&](uint64_t key, uint64_t) { most[0] = max(most[0], (uint32_t)(key >> 32)); });
  const uint32_t mine = wave_nth_key(most, a.best);
  uint32_t top = most[0];
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  if (lane == 0) {
    bounds[wave] = mine;
    tops[wave] = top;
  }
  __syncthreads();
  uint32_t bound = 0;
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    bound = max(bound, bounds[v]);
    top = max(top, tops[v]);
  }
  auto offer = [&](uint64_t key, uint64_t id) {
    const int at = atomicAdd(&listed, 1);
    if (at < kPickCap) list[at] = Ranked{key, id};
  };
  pass([&](uint64_t key, uint64_t id) {
    if (key != 0 && (uint32_t)(key >> 32) >= bound) offer(key, id);
  });
  __syncthreads();
  int n = listed;
  if (n > kPickCap) {
    // The best are those above a range and `left` of the ones in it: first of keys, then of the ids (counted from
    // the last one) of those with one key. (There are more than a.best from the bound on.)
    uint64_t lo = bound ? (uint64_t)bound << 32 : 1, hi = (uint64_t)top << 32 | 0xffffffffu, tie = 0;
    bool of_tie = false;
    int left = a.best;
    for (int step = 0; step < 10; ++step) {   // (64 bits of a key and 38 of an id, 11 at a time)
      const int shift = max(0, 53 - (int)__clzll((hi - lo) | 1));   // (to 11 bits)
      for (int i = tid; i < kBins; i += T) count[i] = 0;
      __syncthreads();
      pass([&](uint64_t key, uint64_t id) {
        const uint64_t x = of_tie ? kLastId - id : key;
        if ((!of_tie || key == tie) && x >= lo && x <= hi) atomicAdd(&count[(x - lo) >> shift], 1);
      });
      __syncthreads();
      int bin;
      find_bin<NW>(count, sums, found, left, bin);
      const int in_bin = count[bin];
      lo += (uint64_t)bin << shift;
      hi = min(hi, lo + (((uint64_t)1 << shift) - 1));
      if (tid == 0) listed = 0;
      __syncthreads();   // (the counts have been read)
      if (a.best - left + in_bin <= kPickCap) break;
      if (lo == hi) {   // (no two candidates have one key and one id)
        tie = lo;
        of_tie = true;
        lo = 0;
        hi = kLastId;
      }
    }
    pass([&](uint64_t key, uint64_t id) {
      if (of_tie ? key > tie || (key == tie && kLastId - id >= lo) : key >= lo) offer(key, id);
    });
    __syncthreads();
    n = listed;
  }
  auto write = [&](int place, uint64_t key, uint64_t id) {
    const int64_t to = (int64_t)item * a.best + place;
    a.out_scores[to] = key ? (float)from_order_key(key) : kMinusInf;
    a.out_tokens[to] = key ? (int32_t)(uint32_t)id : -1;
    a.out_parents[to] = key ? (int32_t)(id >> 32) : -1;
  };
  for (int i = tid; i < n; i += T) {
    const Ranked me = list[i];
    int place = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
      const Ranked x = list[j];
      place += (int)(x.key > me.key) | ((int)(x.key == me.key) & (int)(x.id < me.id));
    }
    if (place < a.best) write(place, me.key, me.id);
  }
  for (int i = n + tid; i < a.best; i += T) write(i, 0, 0);
}

// ---------------------------------------------------------------- the tables

struct ItemCount {
  int32_t taken, freed, bad, pad;
};

struct BeamTableArgs {
  halo_beam_table_sizes_t s;
  halo_beam_tables_t out;
  const int32_t* parents;
  const int32_t* seq_len;
  const int32_t* block_table;
  const int32_t* free_pages;
  const int32_t* free_next;
  ItemCount* counts;   // [items]
  int32_t* freed;      // [items][beams * width]
  int32_t* error_flag;
  int32_t splits;      // workgroups of an item, which share its rows and its part of the free list
};

// An item's beams in LDS: parents, lengths, and which beam is its parent's first
// child. One that is malformed is its own parents' item, with no pages in a row whose
// length does not fit.
struct ItemBeams {
  int32_t parent[kMaxBeams], len[kMaxBeams], pages[kMaxBeams], copied[kMaxBeams];
  uint64_t mothers;   // beams with children
  int32_t bad;
  // A beam's parent and length, by the lane of the same number.
  static __device__ __forceinline__ void read(const BeamTableArgs& a, int item, int lane, int& p, int& n) {
    const int W = a.s.num_beams;
    p = lane < W ? a.parents[(int64_t)item * a.s.parents_stride + lane] : -1;
    n = lane < W ? a.seq_len[(int64_t)item * W + lane] : 0;
  }
  // Takes them, by one wave; to be read after a barrier. as_it_is: as if the item were malformed.
  __device__ __forceinline__ void take(const BeamTableArgs& a, int p, int n, bool as_it_is, int lane) {
    const int W = a.s.num_beams;
    const bool fits = n >= 0 && (int64_t)n <= (int64_t)a.s.table_width * 16;
    const bool wrong = __any(p < -1 || p >= W || !fits);
    if ((wrong || as_it_is) && lane < W) p = lane;
    uint64_t children = 0;
    bool later = false;
    for (int k = 0; k < W; ++k) {
      const int of = __builtin_amdgcn_readlane(p, k);
      if (of >= 0) children |= 1ull << of;
      later |= k < lane && of == p;
    }
    const int of_parent = __shfl(n, max(p, 0));
    if (lane < W) {
      parent[lane] = p;
      len[lane] = n;
      pages[lane] = fits ? (int)(((int64_t)n + 15) >> 4) : 0;
      copied[lane] = p >= 0 && later && (of_parent & 15) != 0;
    }
    if (lane == 0) {
      mothers = children;
      bad = wrong;
    }
  }
};

// Beams whose places in a column a thread holds at a time.
constexpr int kHeld = 8;

// A workgroup for each item: how many pages it takes, and which ones it frees. Beams
// of an item share pages only in the same place of their rows, so a page of a
// beam without children is free if no beam with children has it there, nor an
// earlier beam without: each place of the rows is looked at by itself, W x W
// comparisons, without counts of references. A thread has a place, and the pages of all
// beams there (of more than kHeld beams: of kHeld at a time, against the others). Bound by latency: 4 items of 4 beams
// 3.8 us, 256 items of 8 beams of up to 256 pages 7.4.
__global__ __launch_bounds__(256) void beam_freed_kernel(BeamTableArgs a) {
  __shared__ ItemBeams m;
  __shared__ int sums[4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, item = (int)blockIdx.x, W = a.s.num_beams;
  if (wave == 0) {
    int p, n;
    ItemBeams::read(a, item, lane, p, n);
    m.take(a, p, n, false, lane);
  }
  __syncthreads();
  const int32_t* table = a.block_table + (int64_t)item * W * a.s.table_width;
  int32_t* list = a.freed + (int64_t)item * W * a.s.table_width;
  const uint64_t mothers = m.mothers;
  int most = 0;   // places that hold a page which may be free
  for (int b = 0; b < W; ++b) most = max(most, mothers >> b & 1 ? 0 : m.pages[b]);
  int done = 0;
  for (int c0 = 0; c0 < most; c0 += 256) {
    const int c = c0 + tid;
    uint64_t gone = 0;
    int mine = 0;
    int32_t page[kHeld];
    for (int b0 = 0; b0 < W; b0 += kHeld) {
#pragma unroll
      for (int j = 0; j < kHeld; ++j)
        page[j] = b0 + j < W && c < m.pages[b0 + j] ? table[(int64_t)(b0 + j) * a.s.table_width + c] : 0;
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
        const int b = b0 + j;
        if (b >= W || (mothers >> b & 1)) continue;
        bool held = c >= m.pages[b];
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
          if (b0 + k < W && (k < j || (mothers >> (b0 + k) & 1))) held |= c < m.pages[b0 + k] && page[k] == page[j];
        if (W > kHeld && !held)
          for (int k = 0; k < W; ++k)
            if (k < b0 || (k >= b0 + kHeld && (mothers >> k & 1)))
              held |= c < m.pages[k] && table[(int64_t)k * a.s.table_width + c] == page[j];
        gone |= held ? 0ull : 1ull << b;
      }
    }
    mine = __popcll(gone);
    const int upto = wave_inclusive_sum(mine);
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int at = done + upto - mine;
    for (int w = 0; w < 4; ++w) {
      at += w < wave ? sums[w] : 0;
      done += sums[w];
    }
    if (W <= kHeld) {
#pragma unroll
      for (int j = 0; j < kHeld; ++j)
        if (gone >> j & 1) list[at++] = page[j];
    } else {
      while (gone) {
        const int b = __builtin_ctzll(gone);
        gone &= gone - 1;
        list[at++] = table[(int64_t)b * a.s.table_width + c];
      }
    }
  }
  if (tid < 64) {
    const int taken = __popcll(__ballot(tid < W && m.copied[tid]));
    if (tid == 0) a.counts[item] = ItemCount{taken, done, m.bad, 0};
  }
}

// The items' rows, copies and freed pages at their places: sums over the items before
// each one, which every workgroup makes itself (in a launch of its own, as it needs all counts). Bound by latency: 4
// items of 4 beams 5.5 us, 256 items of 8 beams of up to 256 pages 7.5.
__global__ __launch_bounds__(256) void beam_rows_kernel(BeamTableArgs a) {
  __shared__ ItemBeams m;
  __shared__ int32_t sums[4][5];   // (a table has less than 2^31 pages)
  __shared__ int32_t fresh[kMaxBeams];   // the pages that the copies take
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, W = a.s.num_beams;
  const int item = (int)(blockIdx.x / a.splits), split = (int)(blockIdx.x % a.splits);
  const bool any = item < a.s.num_items;
  const int first = a.free_next[0];
  int p = -1, n = 0;   // (loaded beside the counts)
  if (any && wave == 0) ItemBeams::read(a, item, lane, p, n);
  int32_t s[5] = {0, 0, 0, 0, 0};   // taken and freed before the item, of all; malformed items
  for (int i = tid; i < a.s.num_items; i += 256) {
    const ItemCount c = a.counts[i];
    s[2] += c.taken;
    s[3] += c.freed;
    s[4] += c.bad;
    if (i < item) {
      s[0] += c.taken;
      s[1] += c.freed;
    }
  }
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    s[k] = wave_inclusive_sum(s[k]);
    if (lane == 63) sums[wave][k] = s[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 5; ++k) s[k] = sums[0][k] + sums[1][k] + sums[2][k] + sums[3][k];
  const bool in = first >= 0 && first <= a.s.num_free;
  const bool fits = in && s[2] <= a.s.num_free - first && first + s[2] >= s[3];
  const int64_t rest = fits ? first + s[2] : first;   // from here on the free list stays
  if (any && wave == 0) {
    m.take(a, p, n, !fits, lane);
    const bool copy = lane < W && m.copied[lane];
    const uint64_t mask = __ballot(copy);
    const int before = lanes_before(mask, 0);
    if (lane < W) fresh[lane] = copy ? a.free_pages[first + s[0] + before] : -1;
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.out.free_next[0] = (int)(fits ? rest - s[3] : first);
    if ((s[4] || !fits) && a.error_flag) a.error_flag[0] = 1;
  }
  if (in)
    for (int64_t j = rest + (int64_t)blockIdx.x * 256 + tid; j < a.s.num_free; j += (int64_t)gridDim.x * 256)
      a.out.free_pages[j] = a.free_pages[j];
  if (!any) return;
  __syncthreads();
  if (fits) {
    const int32_t* list = a.freed + (int64_t)item * W * a.s.table_width;
    const int freed = a.counts[item].freed;
    for (int64_t j = (int64_t)split * 256 + tid; j < freed; j += (int64_t)a.splits * 256)
      a.out.free_pages[rest - s[3] + s[1] + j] = list[j];
  }
  const int32_t* table = a.block_table + (int64_t)item * W * a.s.table_width;
  int32_t* out = a.out.block_table + (int64_t)item * W * a.s.table_width;
  if (split == 0 && tid < W) {
    const int p = m.parent[tid];
    const int64_t row = (int64_t)item * W + tid;
    const bool copy = m.copied[tid] && m.pages[p] > 0;
    a.out.seq_len[row] = p < 0 ? 0 : m.len[p];
    a.out.copy_src[row] = copy ? table[(int64_t)p * a.s.table_width + m.pages[p] - 1] : -1;
    a.out.copy_dst[row] = fresh[tid];
  }
  int most = 0;
  for (int k = 0; k < W; ++k) most = max(most, m.parent[k] < 0 ? 0 : m.pages[m.parent[k]]);
  for (int64_t c = (int64_t)split * 256 + tid; c < most; c += (int64_t)a.splits * 256)
    for (int k0 = 0; k0 < W; k0 += kHeld) {
      int32_t page[kHeld];
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
        const int p = k0 + j < W ? m.parent[k0 + j] : -1;
        page[j] = p >= 0 && c < m.pages[p] ? table[(int64_t)p * a.s.table_width + c] : 0;
      }
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
        const int k = k0 + j, p = k < W ? m.parent[k] : -1;
        if (p >= 0 && c < m.pages[p])
          out[(int64_t)k * a.s.table_width + c] = m.copied[k] && c == m.pages[p] - 1 ? fresh[k] : page[j];
      }
    }
}

// ---------------------------------------------------------------- host side

halo_status_t check_sizes(const halo_beam_sizes_t* s) {
  if (!s) return fail(HALO_ERR_INVALID_ARGUMENT, "sizes must not be NULL");
  if (s->num_items < 0) return fail(HALO_ERR_INVALID_ARGUMENT, "num_items must be >= 0");
  if (s->num_beams < 1 || s->vocab < 1 || s->num_best < 1)
    return fail(HALO_ERR_INVALID_ARGUMENT, "num_beams, vocab and num_best must be >= 1");
  if (s->num_beams > kMaxBeams || s->num_best > kMaxBest || s->vocab > kMaxVocab)
    return fail(HALO_ERR_UNSUPPORTED, "at most 64 beams, 64 candidates and 2^24 tokens");
  if (s->logits_stride < s->vocab) return fail(HALO_ERR_INVALID_ARGUMENT, "logits_stride must be >= vocab");
  if (s->dtype != HALO_F32 && s->dtype != HALO_BF16)
    return fail(HALO_ERR_UNSUPPORTED, "dtype must be HALO_F32 or HALO_BF16");
  if ((int64_t)s->num_items * s->num_beams > 65535)
    return fail(HALO_ERR_UNSUPPORTED, "num_items * num_beams must be at most 65535");
  return HALO_OK;
}

// Elements of a wave's part of a row, and the parts of a row: about 4096 waves in
// all, of at least four tiles each.
void parts_of(const halo_beam_sizes_t* s, int32_t& per, int32_t& parts) {
  const int64_t rows = std::max<int64_t>((int64_t)s->num_items * s->num_beams, 1);
  const int64_t span = s->vocab;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(4096 / rows, (span + 2047) / 2048));
  per = (int32_t)((span + want * kTile - 1) / (want * kTile) * kTile);
  parts = (int32_t)((span + per - 1) / per);
}

int64_t parts_bytes(const halo_beam_sizes_t* s, int32_t parts) {
  return ((int64_t)s->num_items * s->num_beams * parts * (int64_t)sizeof(BeamPart) + 255) / 256 * 256;
}

halo_status_t check_sizes(const halo_beam_table_sizes_t* s) {
  if (!s) return fail(HALO_ERR_INVALID_ARGUMENT, "sizes must not be NULL");
  if (s->num_items < 0 || s->table_width < 0 || s->num_free < 0)
    return fail(HALO_ERR_INVALID_ARGUMENT, "num_items, table_width and num_free must be >= 0");
  if (s->num_beams < 1) return fail(HALO_ERR_INVALID_ARGUMENT, "num_beams must be >= 1");
  if (s->num_beams > kMaxBeams) return fail(HALO_ERR_UNSUPPORTED, "at most 64 beams");
  if (s->page_size != 16) return fail(HALO_ERR_UNSUPPORTED, "page_size must be 16");
  if (s->parents_stride < s->num_beams)
    return fail(HALO_ERR_INVALID_ARGUMENT, "parents_stride must be >= num_beams");
  if ((int64_t)s->num_items * s->num_beams * s->table_width > INT32_MAX || s->num_items > 1 << 20)
    return fail(HALO_ERR_UNSUPPORTED, "at most 2^20 items and 2^31 - 1 elements of a table");
  return HALO_OK;
}

int64_t counts_bytes(const halo_beam_table_sizes_t* s) {
  return ((int64_t)s->num_items * (int64_t)sizeof(ItemCount) + 255) / 256 * 256;
}

bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255) == 0; }

}  // namespace

extern "C" int64_t halo_beam_workspace_bytes(const halo_beam_sizes_t* sizes) {
  clear_error();
  if (check_sizes(sizes) != HALO_OK) return -1;
  int32_t per, parts;
  parts_of(sizes, per, parts);
  return parts_bytes(sizes, parts) +
         (int64_t)sizes->num_items * sizes->num_beams * parts * sizes->num_best * (int64_t)sizeof(Candidate);
}

extern "C" halo_status_t halo_beam_select(const halo_beam_sizes_t* sizes, const void* logits, const float* scores,
                                          const int32_t* ended, int32_t end_token, float* out_scores,
                                          int32_t* out_tokens, int32_t* out_parents, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  clear_error();
  const halo_status_t st = check_sizes(sizes);
  if (st != HALO_OK) return st;
  if (ended && (end_token < 0 || end_token >= sizes->vocab))
    return fail(HALO_ERR_INVALID_ARGUMENT, "end_token must be in [0, vocab)");
  if (sizes->num_items == 0) return HALO_OK;
  if (!logits || !scores || !out_scores || !out_tokens || !out_parents || !workspace)
    return fail(HALO_ERR_INVALID_ARGUMENT, "only ended may be NULL");
  const int elt = sizes->dtype == HALO_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % elt) return fail(HALO_ERR_INVALID_ARGUMENT, "logits must be aligned to their elements");
  if (!aligned256(workspace)) return fail(HALO_ERR_INVALID_ARGUMENT, "workspace must be 256-byte aligned");
  const int64_t need = halo_beam_workspace_bytes(sizes);
  if (workspace_bytes < (size_t)need)
    return fail(HALO_ERR_WORKSPACE_TOO_SMALL, "workspace has " + std::to_string(workspace_bytes) + " bytes, needs " +
                                                  std::to_string(need));
  const int64_t rows = (int64_t)sizes->num_items * sizes->num_beams, out = (int64_t)sizes->num_items * sizes->num_best * 4;
  const halo_status_t lap = check_overlaps(
      {{"logits", logits, ((rows - 1) * sizes->logits_stride + sizes->vocab) * elt}, {"scores", scores, rows * 4},
       {"ended", ended, rows * 4}},
      {{"out_scores", out_scores, out}, {"out_tokens", out_tokens, out}, {"out_parents", out_parents, out},
       {"workspace", workspace, need}});
  if (lap != HALO_OK) return lap;
  BeamArgs g{};
  g.logits = logits;
  g.scores = scores;
  g.ended = ended;
  parts_of(sizes, g.per, g.num_parts);
  g.parts = static_cast<BeamPart*>(workspace);
  g.candidates = reinterpret_cast<Candidate*>(static_cast<uint8_t*>(workspace) + parts_bytes(sizes, g.num_parts));
  g.out_scores = out_scores;
  g.out_tokens = out_tokens;
  g.out_parents = out_parents;
  g.stride = sizes->logits_stride;
  g.beams = sizes->num_beams;
  g.vocab = sizes->vocab;
  g.best = sizes->num_best;
  g.end_token = end_token;
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const dim3 grid((unsigned)((g.num_parts + 3) / 4), (unsigned)rows);
  const bool bf16 = sizes->dtype == HALO_BF16, many = sizes->num_best >= kLongListFrom && g.per >= kLongPart;
  if (bf16 && many) hipLaunchKernelGGL((beam_scan_kernel<__bf16, kLongListCap>), grid, dim3(256), 0, s, g);
  else if (bf16) hipLaunchKernelGGL((beam_scan_kernel<__bf16, kListCap>), grid, dim3(256), 0, s, g);
  else if (many) hipLaunchKernelGGL((beam_scan_kernel<float, kLongListCap>), grid, dim3(256), 0, s, g);
  else hipLaunchKernelGGL((beam_scan_kernel<float, kListCap>), grid, dim3(256), 0, s, g);
  if ((int64_t)sizes->num_beams * g.num_parts * sizes->num_best > kManyCandidates)
    hipLaunchKernelGGL(beam_pick_kernel<16>, dim3(sizes->num_items), dim3(1024), 0, s, g);
  else
    hipLaunchKernelGGL(beam_pick_kernel<4>, dim3(sizes->num_items), dim3(256), 0, s, g);
  return hip_check("beam selection launch");
}

extern "C" int64_t halo_beam_tables_workspace_bytes(const halo_beam_table_sizes_t* sizes) {
  clear_error();
  if (check_sizes(sizes) != HALO_OK) return -1;
  return counts_bytes(sizes) + (int64_t)sizes->num_items * sizes->num_beams * sizes->table_width * 4;
}

extern "C" halo_status_t halo_kv_beam_tables(const halo_beam_table_sizes_t* sizes, const int32_t* parents,
                                             const int32_t* seq_len, const int32_t* block_table,
                                             const int32_t* free_pages, const int32_t* free_next,
                                             const halo_beam_tables_t* tables, void* workspace,
                                             size_t workspace_bytes, int32_t* error_flag, void* stream) {
  clear_error();
  const halo_status_t st = check_sizes(sizes);
  if (st != HALO_OK) return st;
  if (!tables) return fail(HALO_ERR_INVALID_ARGUMENT, "tables must not be NULL");
  const int64_t items = sizes->num_items, rows = items * sizes->num_beams, cells = rows * sizes->table_width * 4;
  if (!free_next || !tables->free_next ||
      (rows > 0 && (!parents || !seq_len || !tables->seq_len || !tables->copy_src || !tables->copy_dst || !workspace)) ||
      (cells > 0 && (!block_table || !tables->block_table)) ||
      (sizes->num_free > 0 && (!free_pages || !tables->free_pages)))
    return fail(HALO_ERR_INVALID_ARGUMENT, "only error_flag (and arrays of no elements) may be NULL");
  if (!aligned256(workspace)) return fail(HALO_ERR_INVALID_ARGUMENT, "workspace must be 256-byte aligned");
  const int64_t need = halo_beam_tables_workspace_bytes(sizes);
  if (workspace_bytes < (size_t)need)
    return fail(HALO_ERR_WORKSPACE_TOO_SMALL, "workspace has " + std::to_string(workspace_bytes) + " bytes, needs " +
                                                  std::to_string(need));
  const int64_t free_bytes = 4 * (int64_t)sizes->num_free;
  const halo_status_t lap = check_overlaps(
      {{"parents", parents, items ? ((items - 1) * sizes->parents_stride + sizes->num_beams) * 4 : 0},
       {"seq_len", seq_len, 4 * rows}, {"block_table", block_table, cells}, {"free_pages", free_pages, free_bytes},
       {"free_next", free_next, 4}},
      {{"tables' block_table", tables->block_table, cells}, {"tables' seq_len", tables->seq_len, 4 * rows},
       {"tables' free_pages", tables->free_pages, free_bytes}, {"tables' free_next", tables->free_next, 4},
       {"tables' copy_src", tables->copy_src, 4 * rows}, {"tables' copy_dst", tables->copy_dst, 4 * rows},
       {"workspace", workspace, need}, {"error_flag", error_flag, 4}});
  if (lap != HALO_OK) return lap;
  BeamTableArgs g{*sizes, *tables, parents, seq_len, block_table, free_pages, free_next,
                  static_cast<ItemCount*>(workspace),
                  reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + counts_bytes(sizes)), error_flag, 1};
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  // more workgroups for an item where rows or the free list are long and items few (both launches, 1 item of 4 beams: with
  // 10^6 free pages 1021 -> 11.2 us, with rows of 40000 tokens 22.1 -> 15.3)
  const int64_t groups = std::max<int64_t>(items, 1);
  const int64_t longest = std::max<int64_t>((sizes->table_width + 511) / 512, sizes->num_free / 512 / groups);
  g.splits = (int)std::max<int64_t>(1, std::min<int64_t>(longest, kNumCUs / groups));
  if (items > 0) hipLaunchKernelGGL(beam_freed_kernel, dim3((unsigned)items), dim3(256), 0, s, g);
  hipLaunchKernelGGL(beam_rows_kernel, dim3((unsigned)(groups * g.splits)), dim3(256), 0, s, g);
  return hip_check("beam tables launch");
}
