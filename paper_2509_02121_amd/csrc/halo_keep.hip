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

constexpr int kEvictThreads = 1024;

// The sum of x over the workgroup, and of the threads before this one.
__device__ __forceinline__ int block_exclusive_sum(int x, int& total, int (&sums)[kEvictThreads / 64]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int upto = wave_inclusive_sum(x);
  __syncthreads();
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kEvictThreads / 64; ++w) {
    before += w < wave ? sums[w] : 0;
    total += sums[w];
  }
  return before + upto - x;
}

// A workgroup for each (sequence, head). Of the tokens between the sinks and the recent
// ones m stay: the m-th largest key is found byte by byte from the top, by
// counting how many keys with the bytes found so far have each next one. Then the
// tokens are passed in order: those of a larger key stay, and of those of the same
// key the first ones.
__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictArgs a) {
  __shared__ int count[256];
  __shared__ int sums[kEvictThreads / 64];
  __shared__ int found[2];
  const int tid = threadIdx.x, H = a.s.num_kv_heads;
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
      for (int t = tid; t < len; t += kEvictThreads) out[t] = w[t];
    return;
  }
  const int lo = a.s.sinks, hi = len - a.s.recent;
  int left = a.s.budget - a.s.sinks - a.s.recent;   // of the tokens lo .. hi - 1
  uint32_t key = 0;   // the left-th largest key's bytes found so far
  const bool chosen = left > 0;
  if (chosen) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) count[tid] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += kEvictThreads) {
        const uint32_t k = weight_key(w[t]);
        if (shift == 24 || (k ^ key) >> (shift + 8) == 0) atomicAdd(&count[(k >> shift) & 255], 1);
      }
      __syncthreads();
      // the largest byte with `left` or more keys at or above it
      if (tid < 64) {
        int c[4], mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) mine += c[j] = count[255 - (4 * tid + j)];
        const int upto = wave_inclusive_sum(mine);
        int above = upto - mine;
        if (above < left && upto >= left) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (above < left && above + c[j] >= left) {
              found[0] = 255 - (4 * tid + j);
              found[1] = left - above;
              above = INT32_MAX / 2;
            } else {
              above += c[j];
            }
          }
        }
      }
      __syncthreads();
      key |= (uint32_t)found[0] << shift;
      left = found[1];
    }
  }
  // in order: of the tokens with this key the first `left`
  int32_t* kept = a.kept + ((int64_t)seq * H + h) * a.s.budget;
  int done = 0, equal_done = 0;
  for (int t0 = 0; t0 < len; t0 += kEvictThreads) {
    const int t = t0 + tid;
    const bool in = t < len, between = t >= lo && t < hi;
    const float x = in ? w[t] : 0.f;
    const uint32_t k = weight_key(x);
    const bool equal = chosen && in && between && k == key;
    int equals, total;
    const int rank = block_exclusive_sum(equal, equals, sums);
    const bool keep = in && (!between || (chosen && (k > key || (equal && equal_done + rank < left))));
    const int at = done + block_exclusive_sum(keep, total, sums);
    // (every read of this round is done: the places written are behind them)
    if (keep && at < a.s.budget) {
      kept[at] = t;
      out[at] = x;
    }
    done += total;
    equal_done += equals;
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
  int32_t num_kv_heads, kept_width;
  bool in_place;
};

// Where one token of a sequence comes from.
struct Source {
  int64_t page;   // -1: nowhere
  int slot;       // its place in the page
};

template <typename T, bool KVQ, int D>
struct KeepFormat {
  static constexpr int kK = KVQ ? kvq_k_tile<D>() : 16 * D * (int)sizeof(T);
  static constexpr int kV = KVQ ? kvq_v_tile<D>() : 16 * D * (int)sizeof(T);
};

__device__ __forceinline__ int v_slot_of_token(int t) { return v_token_at_slot(t); }   // (its own inverse)

// A workgroup for each (sequence, head, pool), which goes through the new pages in
// order. Kept indices are ascending, so what is written to a page has already been
// read for every page before it, and the pages behind it read only what lies
// further back: between the loads of a page and its stores there is one barrier,
// and no other workgroup touches these tiles, so that it works in place.
template <typename T, bool KVQ, int D>
__global__ __launch_bounds__(256) void keep_kernel(KeepArgs a) {
  using Fmt = KeepFormat<T, KVQ, D>;
  __shared__ int64_t from[16];   // byte offset of the source tile
  __shared__ int at[16];         // place in it; -1: none
  const int tid = threadIdx.x, H = a.num_kv_heads;
  const int z = (int)(blockIdx.x % 2), h = (int)(blockIdx.x / 2 % H), seq = (int)(blockIdx.x / 2 / H);
  const int len = a.seq_len[seq], count = a.new_len[seq];
  const int base = a.seq_page_indptr[seq], to = a.dst_page_indptr[seq];
  const int64_t have = (int64_t)(a.seq_page_indptr[seq + 1] - base) * 16;
  const int64_t room = (int64_t)(a.dst_page_indptr[seq + 1] - to) * 16;
  if (len < 0 || count < 0 || count > len || len > have || count > room || (count < len && count > a.kept_width)) {
    if (z == 0 && h == 0 && tid == 0 && a.error_flag) a.error_flag[0] = 1;
    return;
  }
  const bool whole = count == len;
  if (whole && a.in_place) return;
  const int32_t* kept = a.kept + ((int64_t)seq * H + h) * a.kept_width;
  uint8_t* pool = z ? a.v_pool : a.k_pool;
  const int tile = z ? Fmt::kV : Fmt::kK;
  for (int p = 0; p * 16 < count; ++p) {
    const int page = a.dst_page_ids[to + p];
    const bool there = page >= 0 && page < a.num_pool_pages;
    if (tid < 16) {
      const int j = 16 * p + tid;
      int src = -1;
      bool bad = !there;
      if (j < count) {
        const int t = whole ? j : kept[j];
        bad |= t < 0 || t >= len;
        if (t >= 0 && t < len) {
          const int id = a.page_ids[base + t / 16];
          if (id >= 0 && id < a.num_pool_pages) {
            src = t & 15;
            from[tid] = ((int64_t)id * H + h) * tile;
          } else {
            bad = true;
          }
        }
        if (bad && a.error_flag) a.error_flag[0] = 1;
      }
      at[tid] = src;
    }
    __syncthreads();
    if (!there) continue;
    uint8_t* dst = pool + ((int64_t)page * H + h) * tile;
    if constexpr (!KVQ) {
      constexpr int E = 16 / (int)sizeof(T), U = D / E, N = 16 * U / 256;   // 16-byte units a thread moves
      constexpr int M = N > 0 ? N : 1;
      u32x4_t x[M];
      bool live[M];
#pragma unroll
      for (int i = 0; i < M; ++i) {
        const int u = tid + 256 * i;
        live[i] = false;
        if (u >= 16 * U) continue;
        if (z == 0) {   // unit u / 16 of token u % 16
          const int s = at[u & 15];
          live[i] = s >= 0;
          if (live[i]) x[i] = *reinterpret_cast<const u32x4_t*>(pool + from[u & 15] + ((u >> 4) * 16 + s) * 16);
        } else {        // E slots of a dim
          const int dim = u / (16 / E), part = u % (16 / E);
          // (slots that get no token keep what they hold)
          x[i] = *reinterpret_cast<const u32x4_t*>(dst + u * 16);
          T* e = reinterpret_cast<T*>(&x[i]);
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const int tok = v_token_at_slot(part * E + j), s = at[tok];
            if (s >= 0) e[j] = reinterpret_cast<const T*>(pool + from[tok])[dim * 16 + v_slot_of_token(s)];
            live[i] |= s >= 0;
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < M; ++i) {
        const int u = tid + 256 * i;
        if (live[i]) *reinterpret_cast<u32x4_t*>(dst + u * 16) = x[i];
      }
    } else if (z == 0) {
      // codes: 4 groups of D / 8 bytes a token; scales: D / 32 bytes a token
      constexpr int W = D / 32;   // dwords of a token's codes in a group
      uint32_t c[W] = {};
      uint32_t sc = 0;
      const int tok = tid & 15, g = tid >> 4;   // (64 threads)
      const int s = tid < 64 ? at[tok] : -1;
      if (s >= 0) {
        const uint8_t* src = pool + from[tok];
#pragma unroll
        for (int i = 0; i < W; ++i) c[i] = reinterpret_cast<const uint32_t*>(src + (g * 16 + s) * (D / 8))[i];
        if (g == 0) {
          if constexpr (D == 128) sc = *reinterpret_cast<const uint32_t*>(src + D * 8 + s * 4);
          else sc = *reinterpret_cast<const uint16_t*>(src + D * 8 + s * 2);
        }
      }
      __syncthreads();
      if (s >= 0) {
#pragma unroll
        for (int i = 0; i < W; ++i) reinterpret_cast<uint32_t*>(dst + (g * 16 + tok) * (D / 8))[i] = c[i];
        if (g == 0) {
          if constexpr (D == 128) *reinterpret_cast<uint32_t*>(dst + D * 8 + tok * 4) = sc;
          else *reinterpret_cast<uint16_t*>(dst + D * 8 + tok * 2) = (uint16_t)sc;
        }
      }
    } else {
      // a dword: the codes of 8 slots of a dim; [D / 64][half][16][4] of them
      uint32_t x = 0;
      uint16_t sc = 0;
      bool live = false;
      if (tid < D * 2) {
        const int half = (tid >> 6) & 1, in_half = (tid >> 7) * 128 + (tid & 63);
        x = reinterpret_cast<const uint32_t*>(dst)[tid];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int tok = v_token_at_slot(8 * half + j), s = at[tok];
          if (s < 0) continue;
          const int slot = v_slot_of_token(s);
          const uint32_t w = (pool + from[tok])[(in_half + 64 * (slot >> 3)) * 4 + ((slot & 7) >> 1)];
          const uint32_t code = slot & 1 ? w >> 4 : w & 15;
          x = (x & ~(15u << (4 * j))) | code << (4 * j);
          live = true;
        }
      }
      const int s = tid < 16 ? at[v_token_at_slot(tid)] : -1;
      if (s >= 0) sc = reinterpret_cast<const uint16_t*>(pool + from[v_token_at_slot(tid)] + D * 8)[v_slot_of_token(s)];
      __syncthreads();
      if (live) reinterpret_cast<uint32_t*>(dst)[tid] = x;
      if (s >= 0) reinterpret_cast<uint16_t*>(dst + D * 8)[tid] = sc;
    }
    __syncthreads();
  }
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
  int32_t per;   // sequences of a workgroup
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
// each), so there is one launch and no wait between workgroups.
__global__ __launch_bounds__(256) void release_kernel(ReleaseArgs a) {
  __shared__ uint32_t sums[4][3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int first = (int)min((int64_t)a.num_seqs, (int64_t)blockIdx.x * a.per);
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
      for (int j = tid; j < r.count; j += 256) a.free_pages_out[at + j] = row[j];
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
  KeepArgs g{static_cast<uint8_t*>(k_pool), static_cast<uint8_t*>(v_pool), page_ids, seq_page_indptr, seq_len, new_len,
             kept, dst_page_ids, dst_page_indptr, error_flag, params->num_pool_pages, params->num_kv_heads, kept_width,
             dst_page_ids == page_ids};
  (void)hipGetLastError();
  by_type_and_dim(params, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    using W = typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type;
    const dim3 grid((unsigned)blocks), block(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!kvq) hipLaunchKernelGGL((keep_kernel<W, false, D>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((keep_kernel<uint8_t, true, D>), grid, block, 0, s, g);
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
  if (rows > 1 << 24) return fail(HALO_ERR_UNSUPPORTED, "num_seqs * num_kv_heads must be at most 2^24");
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
  hipLaunchKernelGGL(evict_kernel, dim3((unsigned)rows), dim3(kEvictThreads), 0, static_cast<hipStream_t>(stream), g);
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
  // up to 256 workgroups, a group of sequences each; without sequences one copies the list
  const int want = std::max((int)n, (int)std::min<int64_t>(64, (sizes->num_free + 2047) / 2048));
  const int blocks = std::min(std::max(want, 1), kNumCUs);
  ReleaseArgs g{block_table, seq_len, new_len, free_pages, free_next, free_pages_out, free_next_out, error_flag,
                sizes->num_seqs, sizes->table_width, sizes->num_free, (int)((n + blocks - 1) / blocks)};
  (void)hipGetLastError();
  hipLaunchKernelGGL(release_kernel, dim3(blocks), dim3(256), 0, static_cast<hipStream_t>(stream), g);
  return hip_check("release launch");
}
