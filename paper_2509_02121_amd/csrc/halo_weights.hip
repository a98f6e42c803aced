// gfx950 kernels and entry points of the C ABI for the attention weight that
// cached tokens get from the queries of a step:
//
//   w[i, h, t] = decay * w[i, h, t] + sum over rows r that see t, heads g of h:
//                exp(scale q[r, g] . k[t, h] - lse[r, g])
//
// lse is known (attention has run), so there is no maximum to follow and no V:
// a wave holds the keys of a few pages in registers and passes the rows by them,
// 16 or 32 at a time. A key's sum stays with its lanes, from the first row to the
// last or (weights_wide, held rows) for 256 rows at a time, each of which is added
// to weights_out by the same lanes, so it has one order and needs no atomics.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "halo_device.h"
#include "halo_host.h"
#include "halo_internal.h"
#include "halo_kvq_format.h"
#include "halo_pages_device.h"

using namespace halo;

namespace {

struct WeightArgs {
  const void* k_pool;
  const void* q;
  const float* lse;
  const float* weights;
  float* weights_out;
  const int32_t* page_ids;
  const int32_t* seq_page_indptr;
  const int32_t* seq_start;
  const int32_t* seq_end;
  const int32_t* row_indptr;
  const int32_t* rows;
  const int32_t* row_end;
  int32_t* error_flag;
  int64_t num_pool_pages;
  int32_t num_seqs, num_rows, num_entries, width;
  int32_t num_kv_heads, group;   // group: q heads of a kv head
  float scale_log2, decay;
};

// How keys lie in the pool and what they become: fragments of the products.
// bf16 queries and keys: one product of bf16 fragments. fp32 ones: fp32 products.
// 4-bit keys are exact in bf16, so fp32 queries go there in three bf16 parts.
template <typename T, bool KVQ, int D>
struct KeyFormat {
  static constexpr int kParts = KVQ && sizeof(T) == 4 ? 3 : 1;
  using F = typename std::conditional<KVQ, bf16x8_t, typename FragOf<T>::type>::type;
  static constexpr int64_t kTile = KVQ ? kvq_k_tile<D>() : 16 * D * (int)sizeof(T);

  // The fragments of the 16 keys of a tile: lane (key = lane & 15, grp) holds dims
  // 32 s + 8 grp .. + 7 of its key. NT: past the caches.
  template <bool NT = false>
  static __device__ __forceinline__ void load_keys(const uint8_t* tile, int lane, F (&k)[D / 32]) {
    const int key = lane & 15, grp = lane >> 4;
    if constexpr (KVQ) {
      uint32_t codes[D / 32], scales;
      const uint8_t* at = tile + (grp * 16 + key) * (D / 8);
      const uint8_t* sc = tile + D * 8 + key * (D / 32);
      if constexpr (D == 128) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(at);
#pragma unroll
        for (int s = 0; s < 4; ++s) codes[s] = x[s];
        scales = *reinterpret_cast<const uint32_t*>(sc);
      } else {
        const u32x2_t x = *reinterpret_cast<const u32x2_t*>(at);
        codes[0] = x[0];
        codes[1] = x[1];
        scales = *reinterpret_cast<const uint16_t*>(sc);
      }
#pragma unroll
      for (int s = 0; s < D / 32; ++s) k[s] = kvq_decode_bf16(codes[s], kvq_scale_byte(scales, s));
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
        k[s] = __builtin_bit_cast(bf16x8_t, ld16<NT>(tile + ((4 * s + grp) * 16 + key) * 16));
    } else {
#pragma unroll
      for (int s = 0; s < D / 32; ++s) k[s] = load_k8<NT>(reinterpret_cast<const float*>(tile), key, 32 * s + 8 * grp);
    }
  }

  // A row's fragments, dims 32 s + 8 grp .. + 7.
  static __device__ __forceinline__ void load_query(const T* row, int grp, F (&q)[kParts][D / 32]) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      const auto x = load8(row + 32 * s + 8 * grp);
      if constexpr (kParts == 1) {
        q[0][s] = x;
      } else {
        float v[8];
        bf16x8_t f[kParts];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[j];
        split(v, f);
#pragma unroll
        for (int n = 0; n < kParts; ++n) q[n][s] = f[n];
      }
    }
  }
};

// Keys that a wave holds at a time.
template <typename T, bool KVQ, int D>
constexpr int weight_pages() { return sizeof(T) == 4 && !KVQ && D == 128 ? 2 : 4; }

// One sequence as the call gives it.
struct WeightSeq {
  int base, next, end, start, e0, e1;
  bool bad, bad_rows;   // (entries that are no range of the list: none)
  __device__ __forceinline__ WeightSeq(const WeightArgs& a, int seq) {
    base = a.seq_page_indptr[seq];
    next = a.seq_page_indptr[seq + 1];
    end = a.seq_end[seq];
    start = a.seq_start ? a.seq_start[seq] : end;
    bad = end < 0 || end > a.width || (int64_t)(next - base) * 16 < end;
    e0 = a.row_indptr ? a.row_indptr[seq] : seq;
    e1 = a.row_indptr ? a.row_indptr[seq + 1] : seq + 1;
    bad_rows = a.row_indptr && (e0 < 0 || e1 < e0 || e1 > a.num_entries);
    if (bad_rows) e0 = e1 = 0;
  }
};

// Flags sequences without pages, which no job comes by, that are to have tokens or whose entries are no range: 64 a
// wave, from the last wave on, as small calls leave it without a job.
__device__ __forceinline__ void flag_without_pages(const WeightArgs& a) {
  if (!a.error_flag) return;
  for (uint32_t i = (gridDim.x - blockIdx.x) * 256 - 1 - threadIdx.x; i < (uint32_t)a.num_seqs; i += gridDim.x * 256) {
    if (a.seq_page_indptr[i + 1] != a.seq_page_indptr[i]) continue;
    const WeightSeq s(a, (int)i);
    if (s.end != 0 || s.bad_rows) a.error_flag[0] = 1;
  }
}

// The (page slot, head) tiles are dealt to the waves in jobs of `run` slots of one
// head, which may span sequences; of a job a wave takes up to NP pages of one
// sequence at a time, and passes all its rows by them. Rows are the A operand and keys the B
// operand of 16x16x32 MFMAs, so that a lane has four rows of one key: their
// exponentials are summed in the lane, and the four lane groups once at the end. Bound by HBM for up to 16 rows (32
// sequences of 1000-8000 bf16 keys, a row of 4 heads on each: 75 us, 4.0 TB/s). More rows come here as fp32 ones, 16 at a
// time from global memory beside fp32 products (32 rows of 4 heads: 900 us, 42 TFLOP/s), and as bf16 ones where the rows of
// weights are short (2048 sequences of 30-64 tokens, 8 rows of 4 heads: 135 us).
template <typename T, bool KVQ, int D>
__global__ __launch_bounds__(256) void weights_kernel(WeightArgs a) {
  using Fmt = KeyFormat<T, KVQ, D>;
  using F = typename Fmt::F;
  constexpr int NS = D / 32, NP = weight_pages<T, KVQ, D>(), PARTS = Fmt::kParts;
  flag_without_pages(a);
  const int lane = threadIdx.x & 63, key = lane & 15, grp = lane >> 4;
  const int H = a.num_kv_heads, G = a.group;
  const int first = a.seq_page_indptr[0];
  const int64_t slots = (int64_t)a.seq_page_indptr[a.num_seqs] - first;
  const int64_t waves = (int64_t)gridDim.x * 4, wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  // as many slots a job as keep every wave busy once, whole groups of NP pages
  const int64_t run = min((int64_t)64, max((int64_t)NP, ((slots * H + waves - 1) / waves + NP - 1) / NP * NP));
  const int64_t jobs = (slots + run - 1) / run * H;
  for (int64_t job = wave; job < jobs; job += waves) {
    const int h = (int)(job % H);
    int64_t slot = job / H * run;
    const int64_t last = min(slots, slot + run);
    int seq = last_at_or_below(a.seq_page_indptr, a.num_seqs, first + slot, lane);
    int loaded = -1;   // the sequence whose only tile of rows is in q
    F q[PARTS][NS];
    float l2[4];
    int sees[4];
    while (slot < last) {
      while (first + slot >= a.seq_page_indptr[seq + 1]) ++seq;   // (ends at num_seqs - 1: slot < slots)
      const WeightSeq s(a, seq);
      const int from = (int)(first + slot - s.base);              // the page's place in its list
      const int n = (int)min(min(last - slot, (int64_t)(s.next - s.base - from)), (int64_t)(NP - from % NP));
      slot += n;
      if ((s.bad || s.bad_rows || a.num_pool_pages == 0) && lane == 0 && a.error_flag) a.error_flag[0] = 1;
      if (s.bad || a.num_pool_pages == 0) continue;
      if ((int64_t)from * 16 >= s.end) continue;   // (a list may have more pages than 32-bit tokens)
      const int t0 = from * 16;
      F k[NP][NS];
      bool ok[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const bool asked = p < n && t0 + 16 * p < s.end;
        const int pid = asked ? a.page_ids[s.base + from + p] : -1;
        ok[p] = pid >= 0 && pid < a.num_pool_pages;
        if (asked && !ok[p] && lane == 0 && a.error_flag) a.error_flag[0] = 1;
        // (a page that is none is read as page 0 and not written)
        Fmt::load_keys(static_cast<const uint8_t*>(a.k_pool) + ((int64_t)(ok[p] ? pid : 0) * H + h) * Fmt::kTile, lane, k[p]);
      }
      float sum[NP] = {}, old[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int t = t0 + 16 * p + key;
        old[p] = a.decay != 0.f && p < n && t < s.end && t < s.start ? a.weights[((int64_t)seq * H + h) * a.width + t] : 0.f;
      }
      const int64_t rows = (int64_t)(s.e1 - s.e0) * G;
      for (int64_t r0 = 0; r0 < rows; r0 += 16) {
        if (rows > 16 || loaded != seq) {
          loaded = seq;
          // lane (row = lane & 15) brings its row's fragments; then rows 4 grp + i
          auto row_of = [&](int64_t r, int& e) {
            e = (int)(s.e0 + r / G);
            if (r >= rows) return -1;
            const int at = a.rows ? a.rows[e] : e;
            return at >= 0 && at < a.num_rows ? at : -1;
          };
          int e;
          const int64_t r = r0 + key;
          const int at = row_of(r, e);
          if (r < rows && at < 0 && a.error_flag) a.error_flag[0] = 1;
          const T* qp = static_cast<const T*>(a.q) + ((int64_t)max(at, 0) * H * G + (int64_t)h * G + r % G) * D;
          if (at >= 0) Fmt::load_query(qp, grp, q);
          else
#pragma unroll
            for (int x = 0; x < PARTS; ++x)
#pragma unroll
              for (int y = 0; y < NS; ++y) q[x][y] = zero_frag<F>();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t ri = r0 + 4 * grp + i;
            const int ai = row_of(ri, e);
            const float l = ai >= 0 ? a.lse[(int64_t)ai * H * G + (int64_t)h * G + ri % G] : kNegInf;
            sees[i] = l == kNegInf ? 0 : a.row_end ? min(a.row_end[e], s.end) : s.end;
            l2[i] = l == kNegInf ? 0.f : l * kLog2e;
          }
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          f32x4_t x = {};
#pragma unroll
          for (int m = 0; m < PARTS; ++m)
#pragma unroll
            for (int y = 0; y < NS; ++y) x = mma(q[PARTS - 1 - m][y], k[p][y], x);
          const int t = t0 + 16 * p + key;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], a.scale_log2, -l2[i]));
            sum[p] += t < sees[i] ? w : 0.f;
          }
        }
      }
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const float w = rows_sum(sum[p]);
        const int t = t0 + 16 * p + key;
        if (ok[p] && p < n && t < s.end && grp == 0) {
          a.weights_out[((int64_t)seq * H + h) * a.width + t] = __builtin_fmaf(a.decay, old[p], w);
        }
      }
    }
  }
}

// ---------------------------------------------------------------- a row for each sequence

// What a lane loads of a page's 16 keys: fragments, or the codes and scales that make them.
template <typename T, bool KVQ, int D>
struct PageKeys {
  using Fmt = KeyFormat<T, KVQ, D>;
  using F = typename Fmt::F;
  F k[D / 32];
  template <bool NT>
  __device__ __forceinline__ void load(const uint8_t* tile, int lane) { Fmt::template load_keys<NT>(tile, lane, k); }
  __device__ __forceinline__ F fragment(int s) const { return k[s]; }
};
template <typename T, int D>
struct PageKeys<T, true, D> {
  uint32_t codes[D / 32], scales;
  template <bool NT>
  __device__ __forceinline__ void load(const uint8_t* tile, int lane) {
    const uint8_t* at = tile + lane * (D / 8);
    const uint8_t* sc = tile + D * 8 + (lane & 15) * (D / 32);   // (lane 16 grp + key is unit (grp, key))
    if constexpr (D == 128) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(at);
#pragma unroll
      for (int s = 0; s < 4; ++s) codes[s] = x[s];
      scales = *reinterpret_cast<const uint32_t*>(sc);
    } else {
      const u32x2_t x = *reinterpret_cast<const u32x2_t*>(at);
      codes[0] = x[0];
      codes[1] = x[1];
      scales = *reinterpret_cast<const uint16_t*>(sc);
    }
  }
  __device__ __forceinline__ bf16x8_t fragment(int s) const { return kvq_decode_bf16(codes[s], kvq_scale_byte(scales, s)); }
};
// Pages on their way, and waves a SIMD whose registers hold as many.
template <typename T, bool KVQ, int D>
constexpr int step_ring() { return KVQ ? 6 : sizeof(T) == 4 && D == 128 ? 2 : D == 128 ? 3 : 4; }
// (fp32 rows, and their parts, take more)
template <typename T> constexpr int step_waves() { return sizeof(T) == 2 ? 4 : 2; }

// A decode step: one entry a sequence and at most 16 q heads of a kv head, so one tile of
// rows, which stays in registers while the sequence's pages pass by. A wave has one run of slots of one
// head, as long as keeps the chip full once; pages are loaded a ring ahead of their use, and a
// page's old weights are waited for when its place in the ring comes round. Bound by HBM: each
// key is read once. Keys of more than kStepCached bytes are loaded past the caches, as the gather's tiles
// are (64 sequences of 2112-2560 tokens, 300 MB: 66.6 -> 61.2 us, 5.1 TB/s).
constexpr int64_t kStepCached = (int64_t)64 << 20;
template <typename T, bool KVQ, int D, bool NT>
__device__ __forceinline__ void weights_step(const WeightArgs& a) {
  using Fmt = KeyFormat<T, KVQ, D>;
  using F = typename Fmt::F;
  constexpr int NS = D / 32, R = step_ring<T, KVQ, D>(), PARTS = Fmt::kParts;
  const int lane = threadIdx.x & 63, key = lane & 15, grp = lane >> 4;
  const int H = a.num_kv_heads, G = a.group;
  const int first = a.seq_page_indptr[0];
  const int64_t slots = (int64_t)a.seq_page_indptr[a.num_seqs] - first;
  const int64_t waves = (int64_t)gridDim.x * 4, wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int run = (int)min((int64_t)64, max((int64_t)1, (slots * H + waves - 1) / waves));
  const int64_t jobs = (slots + run - 1) / run * H;
  for (int64_t job = wave; job < jobs; job += waves) {
    const int h = (int)(job % H);
    const int64_t chunk = job / H * run;
    const int n = (int)min((int64_t)run, slots - chunk);
    const int from = first + (int)chunk;
    const int ids = a.page_ids[from + min(lane, n - 1)];
    int seq = last_at_or_below(a.seq_page_indptr, a.num_seqs, from, lane);
    const uint8_t* pool = static_cast<const uint8_t*>(a.k_pool) + h * Fmt::kTile;
    PageKeys<T, KVQ, D> keys[R];
    float w[R], old[R];
    int64_t to[R];   // of the ring's pages: where their weights go, and how many (the same in every lane)
    int count[R];
    auto load = [&](int i, int r) {   // (behind the last page: that one again)
      const int pid = __builtin_amdgcn_readlane(ids, min(i, n - 1));
      keys[r].template load<NT>(pool + (int64_t)(pid >= 0 && pid < a.num_pool_pages ? pid : 0) * H * Fmt::kTile, lane);
    };
    auto finish = [&](int r) {
      if (lane < count[r]) a.weights_out[to[r] + lane] = __builtin_fmaf(a.decay, old[r], w[r]);
    };
#pragma unroll
    for (int r = 0; r < R; ++r) {
      to[r] = count[r] = 0;
      w[r] = old[r] = 0.f;
      load(r, r);
    }
    int next = from;   // the first slot of another sequence than the one in q
    int base = 0, end = 0, start = 0, sees = 0;
    bool bad = false;
    F q[PARTS][NS];
    float l2[4];
    for (int i0 = 0; i0 < n; i0 += R) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int i = i0 + r, slot = from + min(i, n - 1);
        finish(r);
        count[r] = 0;
        if (i < n) {
          if (slot >= next) {   // another sequence: its row
            while (slot >= a.seq_page_indptr[seq + 1]) ++seq;   // (ends at num_seqs - 1)
            const WeightSeq s(a, seq);
            next = s.next;
            base = s.base;
            end = s.end;
            start = a.decay != 0.f ? s.start : 0;
            bad = s.bad;
            const int at = a.rows ? a.rows[seq] : seq;
            const bool fine = at >= 0 && at < a.num_rows;
            sees = fine ? a.row_end ? min(a.row_end[seq], end) : end : 0;
            if ((bad || !fine) && lane == 0 && a.error_flag) a.error_flag[0] = 1;
            const int64_t row = (int64_t)(fine ? at : 0) * H * G + (int64_t)h * G;
            if (fine && key < G) Fmt::load_query(static_cast<const T*>(a.q) + (row + key) * D, grp, q);
            else
#pragma unroll
              for (int x = 0; x < PARTS; ++x)
#pragma unroll
                for (int y = 0; y < NS; ++y) q[x][y] = zero_frag<F>();
#pragma unroll
            for (int j = 0; j < 4; ++j) l2[j] = fine && 4 * grp + j < G ? a.lse[row + 4 * grp + j] * kLog2e : kNegInf;
          }
          const int64_t token = (int64_t)(slot - base) * 16;   // (a list may have more pages than 32-bit tokens)
          const int t0 = (int)token, pid = __builtin_amdgcn_readlane(ids, i);
          const bool ok = pid >= 0 && pid < a.num_pool_pages, here = !bad && token < end;
          if (here && !ok && lane == 0 && a.error_flag) a.error_flag[0] = 1;
          if (here && ok) {
            f32x4_t x = {};
#pragma unroll
            for (int y = 0; y < NS; ++y) {
              const F k = keys[r].fragment(y);
#pragma unroll
              for (int m = 0; m < PARTS; ++m) x = mma(q[PARTS - 1 - m][y], k, x);
            }
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], a.scale_log2, -l2[j]));
              sum += l2[j] == kNegInf ? 0.f : p;   // (no such row, or it saw no key)
            }
            sum = rows_sum(sum);
            w[r] = t0 + key < sees ? sum : 0.f;
            to[r] = ((int64_t)seq * H + h) * a.width + t0;
            count[r] = min(16, end - t0);
            old[r] = lane < min(min(start, end) - t0, 16) ? a.weights[to[r] + lane] : 0.f;
          }
        }
        load(i + R, r);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) finish(r);
  }
}
template <typename T, bool KVQ, int D>
__global__ __launch_bounds__(256, step_waves<T>()) void weights_step_kernel(WeightArgs a) {
  flag_without_pages(a);
  const int64_t slots = (int64_t)a.seq_page_indptr[a.num_seqs] - a.seq_page_indptr[0];
  if (!KVQ && slots * a.num_kv_heads * KeyFormat<T, KVQ, D>::kTile > kStepCached) weights_step<T, KVQ, D, !KVQ>(a);
  else weights_step<T, KVQ, D, false>(a);
}

// ---------------------------------------------------------------- many rows

// Fragments of 32 keys for 32x32x16 products: lane (c, hh) holds dims 16 s + 8 hh .. + 7 of
// key c % 16 of page c / 16 (`tile`: that page's).
template <bool KVQ, int D>
struct Keys32 {
  u32x4_t x[D / 16];
  __device__ __forceinline__ void load(const uint8_t* tile, int key, int hh) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) x[s] = *reinterpret_cast<const u32x4_t*>(tile + ((2 * s + hh) * 16 + key) * 16);
  }
  __device__ __forceinline__ void fragments(bf16x8_t (&k)[D / 16]) const {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) k[s] = __builtin_bit_cast(bf16x8_t, x[s]);
  }
};
template <int D>
struct Keys32<true, D> {
  // dims 16 s + 8 hh are in group 2 (s & 1) + hh
  using Codes = typename std::conditional<D == 128, u32x4_t, u32x2_t>::type;
  using Scales = typename std::conditional<D == 128, uint32_t, uint16_t>::type;
  Codes codes[2];
  Scales scales;
  __device__ __forceinline__ void load(const uint8_t* tile, int key, int hh) {
#pragma unroll
    for (int z = 0; z < 2; ++z) codes[z] = *reinterpret_cast<const Codes*>(tile + ((2 * z + hh) * 16 + key) * (D / 8));
    scales = *reinterpret_cast<const Scales*>(tile + D * 8 + key * (D / 32));
  }
  __device__ __forceinline__ void fragments(bf16x8_t (&k)[D / 16]) const {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) k[s] = kvq_decode_bf16(codes[s & 1][s >> 1], kvq_scale_byte(scales, s >> 1));
  }
};

// A workgroup takes jobs of one head, groups of 16 slots (which may span sequences), a wave four of a group's pages, 64
// keys, as fragments in registers. Rows are the A operand of 32x32x16 MFMAs, 32 of them a tile, so a lane
// has 16 rows of a key. Bound by the VALU: a product's 64 results take a multiply-add, an
// exponential (four times as long) and an addition.
// Rows go to LDS by direct loads, in batches of four tiles, with their lse and limits. What a batch's loads need
// to know are two lists, one of which is read from the other.
// HELD: a sequence's rows are passed by its pages 256 at a time, and stay where they are for all of a job's
// groups, so the waves work without a barrier; the next group's keys are on their way while the last
// tile's exponentials are taken. A job is as long as fills the chip once: 32 sequences of 1000-8000 tokens with
// 32 tokens' queries (32 + 8 heads), 4 bits, 95.5 -> 61 us; that is 4500 groups of 4 tiles a wave, whose lists and rows
// had taken twice as long to arrive as the products take.
// Otherwise, for more rows, a job is one group, and a batch is loaded while the one before is worked on: its lists are loaded
// three batches ahead, and what they point to one batch later (8 sequences of 4608 tokens, 512 tokens each:
// 183 us, 0.8 PFLOP/s).
// 16-byte unit u of row r of a tile lies at place u ^ r (mod the units of a row; at d 64 r / 2), so that
// the 32 rows' units of one fragment are in different banks.
constexpr int kHeldRows = 256;
template <bool KVQ, int D, bool HELD>
__device__ __forceinline__ void weights_wide(const WeightArgs& a) {
  constexpr int NS = D / 16, U = D / 8, RB = 2 * D, kSlots = 16, NI = D / 64, kRowsPer = 64 / U;
  constexpr int64_t kTile = KVQ ? kvq_k_tile<D>() : 32 * D;
  // (two arrays, and nothing on its way where the loop begins: the compiler then knows that reads of one do not
  // wait for loads to the other)
  __shared__ __align__(1024) uint8_t q0[128 * RB], q1[128 * RB];
  __shared__ int64_t row_lds[4][128];   // where the rows begin
  __shared__ int sees_lds[4][128];
  __shared__ __align__(16) float l_lds[4][128];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 31, hh = lane >> 5;
  const int H = a.num_kv_heads, G = a.group;
  const int first = a.seq_page_indptr[0];
  const int64_t slots = (int64_t)a.seq_page_indptr[a.num_seqs] - first;
  int64_t run = kSlots;
  if constexpr (HELD) run *= max((int64_t)1, ((slots + kSlots - 1) / kSlots * H + gridDim.x - 1) / gridDim.x);
  const int64_t jobs = (slots + run - 1) / run * H;
  const int64_t row_bytes = (int64_t)H * G * RB;
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int h = (int)(job % H);
    const int64_t chunk = job / H * run, chunk_end = min(slots, chunk + run);
    int64_t mine = chunk + 4 * wave;   // the wave's first slot
    Keys32<KVQ, D> keys[2];
    int pid[2];   // this lane's pages
    bool ok[2];
    auto load_ids = [&](int64_t from) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int64_t at = from + 2 * b + (c >> 4);
        pid[b] = at < chunk_end ? a.page_ids[first + at] : -1;
      }
    };
    auto in_pool = [&](int id) { return id >= 0 && id < a.num_pool_pages; };
    auto load_page = [&](int b) {   // (a page that is none is read as page 0 and not written)
      keys[b].load(static_cast<const uint8_t*>(a.k_pool) + ((int64_t)(in_pool(pid[b]) ? pid[b] : 0) * H + h) * kTile, c & 15, hh);
    };
    auto load_keys = [&] {
      load_page(0);
      load_page(1);
    };
    bf16x8_t k[2][NS];
    auto take_keys = [&] {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        ok[b] = in_pool(pid[b]);
        keys[b].fragments(k[b]);
      }
    };
    if constexpr (!HELD) {
      load_ids(mine);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        ok[b] = in_pool(pid[b]);
        if (a.num_pool_pages == 0) continue;
        load_page(b);
        keys[b].fragments(k[b]);
      }
    }
    int seq = last_at_or_below(a.seq_page_indptr, a.num_seqs, first + chunk, lane);
    int64_t slot = chunk;
    while (slot < chunk_end) {
      while (first + slot >= a.seq_page_indptr[seq + 1]) ++seq;   // (ends at num_seqs - 1: slot < slots)
      const WeightSeq s(a, seq);
      const int64_t from = slot, upto = min(chunk_end, (int64_t)s.next - first);
      slot = upto;
      if ((s.bad || s.bad_rows || a.num_pool_pages == 0) && tid == 0 && a.error_flag) a.error_flag[0] = 1;
      const int64_t place = first - (int64_t)s.base;   // of slot 0 in the sequence's list
      if (s.bad || a.num_pool_pages == 0 || (place + from) * 16 >= s.end) continue;
      const int64_t rows = (int64_t)(s.e1 - s.e0) * G;   // (below INT32_MAX - 1024)
      const int64_t keys_end = min(upto, ((int64_t)s.end + 15) / 16 - place);
      int64_t row0 = 0, group = from;
      if constexpr (HELD) {
        load_ids(from + 4 * wave);
        load_keys();
      }
      do {
        if constexpr (HELD) {
          take_keys();
          mine = group + 4 * wave;
          load_ids((group + kSlots < keys_end ? group + kSlots : from) + 4 * wave);   // (behind the last one: the next rows')
        }
        // this wave's keys in the sequence
        const int64_t k0 = max(from, mine), k1 = min(upto, mine + 4);
        const int key_lo = k0 < k1 ? (int)min((place + k0) * 16, (int64_t)s.end) : s.end;
        const int key_hi = k0 < k1 ? (int)min((place + k1) * 16, (int64_t)s.end) : s.end;
        const bool whole = k1 - k0 == 4;
        int t[2];   // this lane's tokens; past every row's end: none
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int64_t at = mine + 2 * b + (c >> 4);
          const bool in = at >= k0 && at < k1;
          t[b] = in ? (int)min((place + at) * 16 + (c & 15), (int64_t)INT32_MAX) : INT32_MAX;
          if (in && !ok[b] && (place + at) * 16 < s.end && a.error_flag) a.error_flag[0] = 1;
        }
        float sum[2] = {0.f, 0.f}, old[2] = {0.f, 0.f};
        const int64_t to = ((int64_t)seq * H + h) * a.width;
#pragma unroll
        for (int z = 0; z < 2; ++z)
          if (HELD && hh == 0 && ok[z] && t[z] < min(s.start, s.end) && a.decay != 0.f && row0 == 0) old[z] = a.weights[to + t[z]];
        if (rows > 0) {
          // A batch's rows, one to each of 128 threads (the other half does the same, and at the start the second
          // batch): the entry, then its row of q, then that row's lse and limit. Rows behind the last one see nothing.
          int e = 0, g = 0, row = 0, sees = 0;
          bool fine = false;
          float l = 0.f;
          auto find = [&](int64_t first_row) {
            const int r = (int)min(first_row, rows);
            e = (int)((uint32_t)r / (uint32_t)G);
            g = r - e * G;
            e += s.e0;
            const int in = min(e, s.e1 - 1);   // (there is one)
            row = a.rows ? a.rows[in] : in;
            if (r >= rows) e = -1;
          };
          auto place_row = [&](int at, int r) {
            fine = row >= 0 && row < a.num_rows;
            if (!fine && e >= 0 && a.error_flag) a.error_flag[0] = 1;
            if (!fine) row = 0;
            row_lds[at][r] = row * row_bytes + (int64_t)(h * G + g) * RB;
          };
          auto look = [&] {
            l = a.num_rows > 0 ? a.lse[(int64_t)row * H * G + (int64_t)h * G + g] : kNegInf;
            sees = a.row_end ? a.row_end[max(e, s.e0)] : s.end;
            if (!fine || e < 0) sees = 0;
          };
          auto keep = [&](int at, int r) {
            const bool none = l == kNegInf;   // (it saw no key)
            l_lds[at][r] = none ? 0.f : -l * kLog2e;
            sees_lds[at][r] = none ? 0 : min(sees, s.end);
          };
          const int64_t tiles = ((HELD ? min(rows - row0, (int64_t)kHeldRows) : rows) + 31) / 32;
          auto issue = [&](int64_t batch, uint8_t* q) {
            if (a.num_rows == 0) return;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (batch * 4 + i >= tiles) break;
#pragma unroll
              for (int j = 0; j < NI; ++j) {
                const int r = wave * 8 + j * kRowsPer + lane / U;
                const int unit = (lane % U) ^ (D == 128 ? r & 15 : (r >> 1) & 7);
                __builtin_amdgcn_global_load_lds(static_cast<const uint8_t*>(a.q) + row_lds[batch & 3][32 * i + r] + unit * 16,
                                                 q + (32 * i + wave * 8 + j * kRowsPer) * RB, 16, 0, 0);
              }
            }
          };
          // A tile's scores go to x while the exponentials of the one before are taken from y: the matrix
          // products of one wave run beside its own VALU instructions. A tile that no key of the wave is
          // seen by is left out; one whose rows see all of them needs no limits.
          uint64_t sees_any[2], sees_part[2];   // of a batch's rows: those that see a key of the wave, and not all of them
          auto look_at = [&](int64_t batch) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int limit = sees_lds[batch & 3][64 * j + lane];
              sees_any[j] = __ballot(limit > key_lo);
              sees_part[j] = __ballot(limit < key_hi);
            }
          };
          auto read_q = [&](const uint8_t* q_lds, bf16x8_t (&q)[NS]) {
#pragma unroll
            for (int x = 0; x < NS; ++x)
              q[x] = *reinterpret_cast<const bf16x8_t*>(q_lds + c * RB + ((2 * x + hh) ^ (D == 128 ? c & 15 : (c >> 1) & 7)) * 16);
          };
          auto read_l = [&](int64_t tile, float (&nl)[16]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const f32x4_t l = *reinterpret_cast<const f32x4_t*>(&l_lds[(tile >> 2) & 3][(tile & 3) * 32 + 8 * j + 4 * hh]);
#pragma unroll
              for (int i = 0; i < 4; ++i) nl[4 * j + i] = l[i];
            }
          };
          auto product = [&](int y, const bf16x8_t (&q)[NS], f32x16_t (&x)[2]) {
#pragma unroll
            for (int z = 0; z < 2; ++z) x[z] = mma32(q[y], k[z][y], y == 0 ? f32x16_t{} : x[z]);
          };
          auto exponentials = [&](int i, const f32x16_t (&y)[2], const float (&nl)[16]) {
#pragma unroll
            for (int z = 0; z < 2; ++z) sum[z] += __builtin_amdgcn_exp2f(__builtin_fmaf(y[z][i], a.scale_log2, nl[i]));
          };
          auto masked = [&](int64_t tile, const f32x16_t (&y)[2]) {
            float nl[16];
            read_l(tile, nl);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int end = sees_lds[(tile >> 2) & 3][(tile & 3) * 32 + 8 * (i >> 2) + 4 * hh + (i & 3)];
#pragma unroll
              for (int z = 0; z < 2; ++z) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(y[z][i], a.scale_log2, nl[i]));
                sum[z] += t[z] < end ? w : 0.f;
              }
            }
          };
          bool held_any = false, held_full = false;   // of the tile whose scores are held
          // tile 4 batch + i's scores to x, the exponentials of the one before, whose scores are in y
          auto step = [&](int64_t batch, int i, const uint8_t* q_lds, f32x16_t (&x)[2], const f32x16_t (&y)[2]) {
            const bool more = i < 4;
            const bool any = more && (uint32_t)(sees_any[(i & 2) / 2] >> (32 * (i & 1))) != 0;
            const bool full = any && whole && (uint32_t)(sees_part[(i & 2) / 2] >> (32 * (i & 1))) == 0;
            const int64_t tile = batch * 4 + i;
            if (any && held_full) {
              bf16x8_t q[NS];
              float nl[16];
              read_l(tile - 1, nl);
              read_q(q_lds, q);
              // (in this order: the two chains of products in turn, each with its share of the rest)
#pragma unroll
              for (int s = 0; s < NS; ++s) {
                product(s, q, x);
#pragma unroll
                for (int j = 0; j < 16 / NS; ++j) exponentials(16 / NS * s + j, y, nl);
                __builtin_amdgcn_sched_barrier(0);
              }
            } else {
              if (any) {
                bf16x8_t q[NS];
                read_q(q_lds, q);
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                  product(s, q, x);
                  __builtin_amdgcn_sched_barrier(0);
                }
              }
              if (held_full) {
                float nl[16];
                read_l(tile - 1, nl);
#pragma unroll
                for (int j = 0; j < 16; ++j) exponentials(j, y, nl);
              } else if (held_any) {
                masked(tile - 1, y);
              }
            }
            held_any = any;
            held_full = full;
          };
          f32x16_t x[2], y[2];
          // one batch: the next one's loads begin, and those of what the ones behind it need
          auto work = [&](int64_t batch, const uint8_t* q, uint8_t* next) {
            look_at(batch);
            const bool behind = (batch + 2) * 4 < tiles;
            if (behind) {
              place_row((int)(batch + 2) & 3, tid & 127);
              look();
            }
            issue(batch + 1, next);
            step(batch, 0, q, x, y);
            step(batch, 1, q + 32 * RB, y, x);
            if (behind) {
              keep((int)(batch + 2) & 3, tid & 127);
              find((batch + 3) * 128 + (tid & 127));
            }
            step(batch, 2, q + 64 * RB, x, y);
            step(batch, 3, q + 96 * RB, y, x);
            wait_vmcnt<0>();
            __syncthreads();
          };
          if (!HELD || group == from) {
            find(row0 + tid);
            place_row(tid >> 7, tid & 127);
            __syncthreads();
            issue(0, q0);
            if constexpr (HELD) issue(1, q1);
            look();
            keep(tid >> 7, tid & 127);
            if (!HELD && tiles > 8) find(256 + (tid & 127));
            wait_vmcnt<0>();
            __syncthreads();
          }
          if constexpr (HELD) {
            for (int64_t batch = 0; batch * 4 < tiles; ++batch) {
              const uint8_t* q = batch ? q1 : q0;
              look_at(batch);
              step(batch, 0, q, x, y);
              step(batch, 1, q + 32 * RB, y, x);
              step(batch, 2, q + 64 * RB, x, y);
              step(batch, 3, q + 96 * RB, y, x);
            }
          } else {
            for (int64_t batch = 0; batch * 4 < tiles; batch += 2) {
              work(batch, q0, q1);
              if ((batch + 1) * 4 < tiles) work(batch + 1, q1, q0);
            }
          }
          if constexpr (HELD) load_keys();   // (the next group's: nothing needs this one's any more)
          step((tiles - 1) / 4, 4, q0, x, y);   // (whole batches, so that the last scores are in y)
          // (the next first batches go where the last rows and limits may still be read)
          if (!HELD || group + kSlots >= keys_end) __syncthreads();
        }
        if constexpr (!HELD) {
#pragma unroll
          for (int z = 0; z < 2; ++z)
            if (hh == 0 && ok[z] && t[z] < min(s.start, s.end) && a.decay != 0.f) old[z] = a.weights[to + t[z]];
        }
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const float w = halves_sum(sum[z]);
          if (hh == 0 && ok[z] && t[z] < s.end) {
            if (row0 > 0) a.weights_out[to + t[z]] += w;
            else a.weights_out[to + t[z]] = __builtin_fmaf(a.decay, old[z], w);   // (without an old weight: decay * 0)
          }
        }
        group += kSlots;
        if (HELD && group >= keys_end) {
          group = from;
          row0 += kHeldRows;
        }
      } while (HELD && (group > from || row0 < rows));
    }
  }
}

// (the body in a function of its own: the host's pass does not know the direct loads)
template <bool KVQ, int D, bool HELD>
__global__ __launch_bounds__(256, 2) void weights_wide_kernel(WeightArgs a) {
  flag_without_pages(a);
  weights_wide<KVQ, D, HELD>(a);
}

// Whether a sequence has `rows` rows or more on average. The wide kernel takes bf16 queries from 17 on, where
// the general one passes a second tile (window of 8 tokens, G 4, sequences of 1000-8000 tokens: 113 us general, 73 wide;
// of 4 tokens: 93 and 83; 512 sequences of 50-200 tokens: 85 and 81, of 4 tokens 55 and 89). It holds them up to 512: 128
// tokens, 224 us a batch at a time, 205 held; 256 tokens, 397 and 427. Short sequences do not pay for what a
// workgroup waits for at their beginning: 2048 of 30-64 tokens with windows of 8, 16 and 32 take 135, 201 and 351 us by
// the general kernel, 179, 217 and 293 a batch at a time, 249, 281 and 336 held; 512 of 200-300 tokens 130, 193 and 324,
// 106, 121 and 152, 106, 115 and 134. What is known here are averages and capacities: how many tokens there are by the
// weights' width alone, so that short sequences in wide rows of weights take the held kernel's times, and rows by all
// entries, so that one prefix with the rows of a thousand requests and their private lists in one call take the general
// kernel's; such calls are better made apart.
constexpr int kShortWidth = 80, kHeldWidth = 129;   // five pages; more than eight
bool many_rows(const halo_weight_sizes_t& s, bool lists, int group, int rows) {
  return (int64_t)(lists ? s.num_entries : s.num_seqs) * group >= rows * (int64_t)s.num_seqs;
}

halo_status_t page_weights(bool kvq, const void* k_pool, const halo_attn_params_t* params,
                           const halo_weight_sizes_t* sizes, const int32_t* page_ids, const int32_t* seq_page_indptr,
                           const int32_t* seq_start, const int32_t* seq_end, const int32_t* row_indptr,
                           const int32_t* rows, const int32_t* row_end, const void* q, const float* lse, float decay,
                           const float* weights, float* weights_out, int32_t* error_flag, void* stream) {
  clear_error();
  if (!params || !sizes) return fail(HALO_ERR_INVALID_ARGUMENT, "params and sizes must not be NULL");
  if (sizes->num_seqs < 0 || sizes->num_rows < 0 || sizes->num_entries < 0 || sizes->width < 0)
    return fail(HALO_ERR_INVALID_ARGUMENT, "every size must be >= 0");
  const halo_status_t st = check_cache_params(params);
  if (st != HALO_OK) return st;
  const int H = params->num_kv_heads;
  if (params->num_q_heads < H || params->num_q_heads % H != 0)
    return fail(HALO_ERR_INVALID_ARGUMENT, "num_q_heads must be a multiple of num_kv_heads");
  if (!finite(params->sm_scale) || params->sm_scale <= 0.f)
    return fail(HALO_ERR_INVALID_ARGUMENT, "sm_scale must be positive and finite");
  if (!finite(decay) || decay < 0.f) return fail(HALO_ERR_INVALID_ARGUMENT, "decay must be finite and >= 0");
  if (sizes->num_seqs == 0 || sizes->width == 0) return HALO_OK;
  if (!k_pool || !page_ids || !seq_page_indptr || !seq_end || !weights_out || (sizes->num_rows > 0 && (!q || !lse)))
    return fail(HALO_ERR_INVALID_ARGUMENT,
                "k_pool, page_ids, seq_page_indptr, seq_end, q, lse, weights_out must not be NULL");
  if (!weights && decay != 0.f) return fail(HALO_ERR_INVALID_ARGUMENT, "weights must not be NULL unless decay is 0");
  if (!row_indptr && (rows || row_end) && sizes->num_entries < sizes->num_seqs)
    return fail(HALO_ERR_INVALID_ARGUMENT, "without row_indptr, rows and row_end have an element for each sequence");
  if (!aligned16(k_pool) || !aligned16(q)) return fail(HALO_ERR_INVALID_ARGUMENT, "k_pool and q must be 16-byte aligned");
  if ((int64_t)sizes->num_entries * (params->num_q_heads / H) >= INT32_MAX - 1023)
    return fail(HALO_ERR_UNSUPPORTED, "num_entries * num_q_heads / num_kv_heads must be less than 2^31 - 1024");
  const int64_t n = sizes->num_seqs, cells = n * H * sizes->width * 4, elt = params->kv_dtype == HALO_BF16 ? 2 : 4;
  const int64_t rows_h = (int64_t)sizes->num_rows * params->num_q_heads, entries = 4 * (int64_t)sizes->num_entries;
  const int64_t tile = kvq ? params->head_dim * 8 + params->head_dim / 2 : 16 * params->head_dim * elt;
  const halo_status_t lap = check_overlaps(
      {{"k_pool", k_pool, params->num_pool_pages * H * tile}, {"q", q, rows_h * params->head_dim * elt},
       {"lse", lse, rows_h * 4}, {"weights", weights == weights_out ? nullptr : weights, cells},
       {"seq_page_indptr", seq_page_indptr, 4 * (n + 1)}, {"seq_start", seq_start, 4 * n}, {"seq_end", seq_end, 4 * n},
       {"row_indptr", row_indptr, 4 * (n + 1)}, {"rows", rows, entries}, {"row_end", row_end, entries}},
      {{"weights_out", weights_out, cells}, {"error_flag", error_flag, 4}});
  if (lap != HALO_OK) return lap;
  WeightArgs g{k_pool, q, lse, weights, weights_out, page_ids, seq_page_indptr, seq_start, seq_end, row_indptr, rows,
               row_end, error_flag, params->num_pool_pages, sizes->num_seqs, sizes->num_rows, sizes->num_entries,
               sizes->width, H, params->num_q_heads / H, params->sm_scale * kLog2e, decay};
  (void)hipGetLastError();
  const bool step = !row_indptr && g.group <= 16 && params->num_pool_pages > 0;
  const bool wide = params->kv_dtype == HALO_BF16 && many_rows(*sizes, row_indptr != nullptr, g.group, sizes->width <= kShortWidth ? 65 : 17);
  const bool held = sizes->width >= kHeldWidth && !many_rows(*sizes, row_indptr != nullptr, g.group, 2 * kHeldRows + 1);
  by_type_and_dim(params, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    const dim3 grid(2048), block(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (step && kvq) hipLaunchKernelGGL((weights_step_kernel<T, true, D>), dim3(kNumCUs * step_waves<T>()), block, 0, s, g);
    else if (step) hipLaunchKernelGGL((weights_step_kernel<T, false, D>), dim3(kNumCUs * step_waves<T>()), block, 0, s, g);
    else if (wide && held && kvq) hipLaunchKernelGGL((weights_wide_kernel<true, D, true>), dim3(2 * kNumCUs), block, 0, s, g);
    else if (wide && held) hipLaunchKernelGGL((weights_wide_kernel<false, D, true>), dim3(2 * kNumCUs), block, 0, s, g);
    else if (wide && kvq) hipLaunchKernelGGL((weights_wide_kernel<true, D, false>), grid, block, 0, s, g);
    else if (wide) hipLaunchKernelGGL((weights_wide_kernel<false, D, false>), grid, block, 0, s, g);
    else if (kvq) hipLaunchKernelGGL((weights_kernel<T, true, D>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((weights_kernel<T, false, D>), grid, block, 0, s, g);
  });
  return hip_check("attention weights launch");
}

}  // namespace

extern "C" halo_status_t halo_kv_page_weights(const void* k_pool, const halo_attn_params_t* params,
                                              const halo_weight_sizes_t* sizes, const int32_t* page_ids,
                                              const int32_t* seq_page_indptr, const int32_t* seq_start,
                                              const int32_t* seq_end, const int32_t* row_indptr, const int32_t* rows,
                                              const int32_t* row_end, const void* q, const float* lse, float decay,
                                              const float* weights, float* weights_out, int32_t* error_flag,
                                              void* stream) {
  return page_weights(false, k_pool, params, sizes, page_ids, seq_page_indptr, seq_start, seq_end, row_indptr, rows,
                      row_end, q, lse, decay, weights, weights_out, error_flag, stream);
}

extern "C" halo_status_t halo_kvq_page_weights(const void* k_pool, const halo_attn_params_t* params,
                                               const halo_weight_sizes_t* sizes, const int32_t* page_ids,
                                               const int32_t* seq_page_indptr, const int32_t* seq_start,
                                               const int32_t* seq_end, const int32_t* row_indptr, const int32_t* rows,
                                               const int32_t* row_end, const void* q, const float* lse, float decay,
                                               const float* weights, float* weights_out, int32_t* error_flag,
                                               void* stream) {
  return page_weights(true, k_pool, params, sizes, page_ids, seq_page_indptr, seq_start, seq_end, row_indptr, rows,
                      row_end, q, lse, decay, weights, weights_out, error_flag, stream);
}
