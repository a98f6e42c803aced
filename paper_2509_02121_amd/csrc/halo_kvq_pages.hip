// gfx950 kernels and entry points of the C ABI that write tokens into 4-bit
// pages and read them back:
// kvq_scatter_kernel: new tokens quantised into their pages, K and V;
// kvq_gather_kernel: paged tokens out into dense buffers, K and V.
//
// A wave takes one (page, head) tile of 16 tokens at a time, lane 4 sl + g
// holding dims 32 s + 8 g .. + 7 (s < D / 32) of the token in slot sl. A K scale
// block of 32 dims is then the four lanes of a slot, and a V one (the whole head)
// their D / 32 vectors. 8 dims are one dword of K codes as they are; V codes have
// the 8 tokens of a half (slots 8 h .. + 7) of one dim in a dword, which is a
// transposition of 8 x 8 codes between the 8 lanes of a half and the 8 codes of a
// lane: three rounds of lane exchanges, no LDS (CodeTransposer).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "halo_internal.h"
#include "halo_kvq_format.h"
#include "halo_pages_device.h"

using namespace halo;

namespace {

typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// 8 consecutive elements of a dense row as floats, and back.
__device__ __forceinline__ void load8(const __bf16* p, float (&v)[8]) {
  const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(x[j] << 16);
    v[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4_t x = *reinterpret_cast<const f32x4_t*>(p), y = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = x[j];
    v[4 + j] = y[j];
  }
}
__device__ __forceinline__ void store_decoded(__bf16* p, uint32_t w, float scale) {
  *reinterpret_cast<u32x4_t*>(p) = __builtin_bit_cast(u32x4_t, kvq_decode_bf16(w, scale));
}
__device__ __forceinline__ void store_decoded(float* p, uint32_t w, float scale) {
  float v[8];
  kvq_decode_f32(w, scale, v);
  *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
}

// Codes i of the lanes 4 (8 h + j) + g become codes j of the lanes
// 4 (8 h + i) + g (its own inverse): bit b of i and of j are swapped by an
// exchange with the lane 4 << b away, on the VALU and without branches (with
// __shfl_xor and a choice between two results, 12 branches and LDS waits a tile: 64
// appends 4.65 -> 4.36 us, 60 with 4 chunks 7.2 -> 6.8).
struct CodeTransposer {
  uint32_t rot, keep, bytes, halves;
  __device__ __forceinline__ explicit CodeTransposer(int lane) {
    rot = lane & 4 ? 4 : 28;
    keep = lane & 4 ? 0xf0f0f0f0u : 0x0f0f0f0fu;
    bytes = lane & 8 ? 0x03070105u : 0x06020400u;
    halves = lane & 16 ? 0x07060302u : 0x05040100u;
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t x) const {
    // 4 lanes away: reversed in 8 lanes, then in 4
    const int half = __builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true);        // row_half_mirror
    uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, half, 0x1B, 0xf, 0xf, true);   // quad_perm 3,2,1,0
    x = (x & keep) | (__builtin_amdgcn_alignbit(y, y, rot) & ~keep);
    y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true);           // row_ror:8
    x = __builtin_amdgcn_perm(y, x, bytes);
    // the even and the odd row's
    const auto rows = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return __builtin_amdgcn_perm(rows[1], rows[0], halves);
  }
};

// The dword of a V tile that holds dim 32 s + 8 g + i for half h.
__device__ __forceinline__ int v_dword(int s, int g, int i, int h) {
  const int b = 2 * s + (g >> 1), c = 8 * (g & 1) + i;
  return (((b >> 2) * 2 + h) * 16 + c) * 4 + (b & 3);
}

// The maximum of x over the four lanes of a slot.
__device__ __forceinline__ uint32_t slot_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));   // quad_perm 1,0,3,2
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));   // quad_perm 2,3,0,1
}

// ---------------------------------------------------------------- write path

struct KvqScatterArgs {
  uint8_t* pool[2];
  const void* in[2];
  const int32_t* page_ids;
  const int32_t* seq_page_indptr;
  const int32_t* seq_start;
  const int32_t* seq_count;
  const int64_t* in_token_offset;
  int32_t* error_flag;
  int64_t num_pool_pages;
  int32_t num_seqs;
  int32_t num_kv_heads;
  int32_t seq_blocks;    // workgroups by sequence (partly touched pages)
  int32_t splits;        // of them per sequence
  int32_t tile_blocks;   // workgroups for the whole pages' tiles
};

// Tokens lo .. hi - 1 (of 0 .. 15) of one tile; src: the dense row of token 0 of
// the page (only those of the tokens are read), `row` elements per token.
template <typename T, int D, bool V>
__device__ __forceinline__ void write_tile(const T* src, int64_t row, uint8_t* tile, int lo, int hi, int lane) {
  constexpr int S = D / 32;
  const int sl = lane >> 2, g = lane & 3;
  const int t = v_token_at_slot(sl);
  const bool live = t >= lo && t < hi;
  float v[S][8];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    if (live) {
      load8(src + t * row + 32 * s + 8 * g, v[s]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[s][j] = 0.f;
    }
  }
  uint32_t top[S];   // (bits: a NaN's are the largest)
#pragma unroll
  for (int s = 0; s < S; ++s) {
    top[s] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top[s] = max(top[s], __float_as_uint(v[s][j]) & 0x7fffffffu);
  }
  if constexpr (!V) {
    uint32_t w[S], scales = 0;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int e = kvq_exponent(slot_max(top[s]));
      w[s] = kvq_encode(v[s], kvq_scale(e)) & (e == 255 ? 0u : 0xffffffffu);
      scales |= (uint32_t)e << (8 * s);
    }
    if (!live) return;
    uint32_t* at = reinterpret_cast<uint32_t*>(tile) + (g * 16 + t) * S;
    if constexpr (S == 4) *reinterpret_cast<u32x4_t*>(at) = u32x4_t{w[0], w[1], w[2], w[3]};
    else *reinterpret_cast<u32x2_t*>(at) = u32x2_t{w[0], w[1]};
    if (g == 0) {
      if constexpr (S == 4) *reinterpret_cast<uint32_t*>(tile + D * 8 + t * 4) = scales;
      else *reinterpret_cast<uint16_t*>(tile + D * 8 + t * 2) = (uint16_t)scales;
    }
  } else {
    uint32_t m = top[0];
#pragma unroll
    for (int s = 1; s < S; ++s) m = max(m, top[s]);
    const int e = kvq_exponent(slot_max(m));
    // the codes of this lane's half that are written
    const int h = sl >> 3, i = sl & 7;
    uint32_t mask = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int tok = v_token_at_slot(8 * h + j);
      mask |= tok >= lo && tok < hi ? 0xfu << (4 * j) : 0u;
    }
    uint32_t* codes = reinterpret_cast<uint32_t*>(tile);
    const CodeTransposer transpose(lane);
    const uint32_t real = e == 255 ? 0u : 0xffffffffu;
    uint32_t w[S];
#pragma unroll
    for (int s = 0; s < S; ++s) w[s] = transpose(kvq_encode(v[s], kvq_scale(e)) & real);
    if (lo != 0 || hi != 16) {
#pragma unroll
      for (int s = 0; s < S; ++s) w[s] = (w[s] & mask) | (mask != 0xffffffffu ? codes[v_dword(s, g, i, h)] & ~mask : 0u);
    }
    if (mask) {
#pragma unroll
      for (int s = 0; s < S; ++s) codes[v_dword(s, g, i, h)] = w[s];
    }
    if (live && g == 0)
      *reinterpret_cast<uint16_t*>(tile + D * 8 + 2 * sl) = (uint16_t)(e == 255 ? 0x7fc0 : e << 7);
  }
}

// A tile of page `pslot` of a page list: K and V of the heads in turn.
template <typename T, int D>
__device__ __forceinline__ void scatter_tile(const KvqScatterArgs& a, int64_t at, int base, int pslot, int hv, int lo,
                                             int hi, int lane) {
  const int H = a.num_kv_heads, h = hv >> 1;
  const int64_t row = (int64_t)H * D;
  const int pid = a.page_ids[base + pslot];
  if (pid < 0 || pid >= a.num_pool_pages) {
    if (lane == 0 && a.error_flag) a.error_flag[0] = 1;
    return;
  }
  const int64_t from = (at + (int64_t)pslot * 16) * row + (int64_t)h * D;   // token 0 of the page
  const int64_t tile = (int64_t)pid * H + h;
  if (hv & 1)
    write_tile<T, D, true>(static_cast<const T*>(a.in[1]) + from, row, a.pool[1] + tile * kvq_v_tile<D>(), lo, hi, lane);
  else
    write_tile<T, D, false>(static_cast<const T*>(a.in[0]) + from, row, a.pool[0] + tile * kvq_k_tile<D>(), lo, hi, lane);
}

// Two kinds of workgroups, as in scatter_kernel: `splits` for each sequence take the
// tiles of its partly touched first and last pages (an append: one page, a wave for
// each of its tiles), and tile_blocks share the whole pages of all sequences
// equally. Against splits of every sequence's tiles, whole pages or not: 64
// appends 8.7 -> 4.6 us, 496 appends and 16 chunks 87 -> 18 us (8 heads, d 128).
// 32 chunks of 512-1024 tokens (137 MB) 23.4 us, 5.9 TB/s out of the caches.
// Five waves per SIMD: with the four that its registers would ask for 32 chunks of
// 512-1024 tokens (after other work) take 36.2 us, so 30.7, 1024 appends 19.0 and 17.8;
// six spill (64 appends 4.34 us, so 4.10).
template <typename T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(5))) void kvq_scatter_kernel(KvqScatterArgs a) {
  __shared__ int sums[260];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int H = a.num_kv_heads;
  if ((int)blockIdx.x < a.seq_blocks) {
    const int first_tile = (int)blockIdx.x % a.splits * 4 + wave;
    for (int seq = (int)blockIdx.x / a.splits; seq < a.num_seqs; seq += a.seq_blocks / a.splits) {
      const int start = a.seq_start[seq], count = a.seq_count[seq];
      const int base = a.seq_page_indptr[seq], next = a.seq_page_indptr[seq + 1];
      const int64_t off = a.in_token_offset[seq];
      if (count <= 0) continue;
      if (start < 0 || (int64_t)start + count > (int64_t)(next - base) * 16) {
        if (first_tile == 0 && lane == 0 && a.error_flag) a.error_flag[0] = 1;
        continue;
      }
      const PageRange r(start, count);
      const int pages = (r.head ? 1 : 0) + (r.tail ? 1 : 0);
      for (int k = first_tile; k < pages * 2 * H; k += 4 * a.splits) {
        const bool second = k >= 2 * H;   // the last page, after the first
        const int p = r.head && !second ? r.first : r.last;
        scatter_tile<T, D>(a, off - start, base, p, second ? k - 2 * H : k, max(start - p * 16, 0),
                           min(start + count - p * 16, 16), lane);
      }
    }
    return;
  }
  const int tb = (int)blockIdx.x - a.seq_blocks;
  const int groups = (a.num_seqs + kTileSeqs - 1) / kTileSeqs;
  for (int g = tb % groups; g < groups; g += a.tile_blocks) {
    // the workgroups of this group, and this one's turn among them
    const int of = a.tile_blocks >= groups ? (a.tile_blocks - g + groups - 1) / groups : 1;
    const int s0 = g * kTileSeqs, n = min(a.num_seqs - s0, kTileSeqs);
    whole_tiles(a, 2 * H, s0, n, tb / groups * 4 + wave, of * 4, sums, wave, lane,
                [&](int64_t at, int base, int pslot, int hv) { scatter_tile<T, D>(a, at, base, pslot, hv, 0, 16, lane); });
    __syncthreads();   // the sums are overwritten for the next group
  }
}

// ---------------------------------------------------------------- gather

struct KvqGatherArgs {
  const uint8_t* pool[2];
  void* out[2];
  const int32_t* page_ids;
  const int32_t* seq_page_indptr;
  const int32_t* seq_len;
  const int64_t* out_token_offset;
  int32_t* error_flag;
  int64_t num_pool_pages;
  int32_t num_seqs;
  int32_t num_kv_heads;
};

// Tokens 0 .. n - 1 of one tile; dst: the dense row of token 0.
template <typename T, int D, bool V>
__device__ __forceinline__ void read_tile(const uint8_t* tile, T* dst, int64_t row, int n, int lane) {
  constexpr int S = D / 32;
  const int sl = lane >> 2, g = lane & 3;
  const int t = v_token_at_slot(sl);
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(tile);
  uint32_t w[S];
  float scale[S];
  if constexpr (!V) {
    const uint32_t* at = codes + (g * 16 + t) * S;
    uint32_t scales;
    if constexpr (S == 4) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(at);
      scales = *reinterpret_cast<const uint32_t*>(tile + D * 8 + t * 4);
#pragma unroll
      for (int s = 0; s < S; ++s) w[s] = x[s];
    } else {
      const u32x2_t x = *reinterpret_cast<const u32x2_t*>(at);
      scales = *reinterpret_cast<const uint16_t*>(tile + D * 8 + t * 2);
#pragma unroll
      for (int s = 0; s < S; ++s) w[s] = x[s];
    }
#pragma unroll
    for (int s = 0; s < S; ++s) scale[s] = kvq_scale((scales >> (8 * s)) & 0xff);
  } else {
    const CodeTransposer transpose(lane);
    const uint32_t e = *reinterpret_cast<const uint16_t*>(tile + D * 8 + 2 * sl);
#pragma unroll
    for (int s = 0; s < S; ++s) w[s] = codes[v_dword(s, g, sl & 7, sl >> 3)];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      w[s] = transpose(w[s]);
      scale[s] = __uint_as_float(e << 16);
    }
  }
  if (t >= n) return;
#pragma unroll
  for (int s = 0; s < S; ++s) store_decoded(dst + t * row + 32 * s + 8 * g, w[s], scale[s]);
}

// The tiles of all sequences (pages, then heads, K before V) are cut into equal
// contiguous runs, one per wave, so that a few long sequences among many short
// ones spread over the chip. 8192 workgroups: 256 sequences of 100-500 tokens after
// other work (400 MB) 115 us, with 2048 127; 25000 tokens 39 and 43; 16384 cost
// small calls more than they bring large ones.
template <typename T, int D>
__global__ __launch_bounds__(256) void kvq_gather_kernel(KvqGatherArgs a) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int H = a.num_kv_heads;
  const int64_t row = (int64_t)H * D;
  // page-list slots first .. last-1 are read; first need not be 0
  const int first = a.seq_page_indptr[0];
  const int64_t total = ((int64_t)a.seq_page_indptr[a.num_seqs] - first) * 2 * H;
  const int64_t waves = (int64_t)gridDim.x * 4;
  const int64_t per = (total + waves - 1) / waves;
  const int64_t begin = ((int64_t)blockIdx.x * 4 + wave) * per, end = min(total, begin + per);
  if (begin >= end) return;
  // indptr[0] <= first + begin / 2H < indptr[num_seqs]: a sequence in [0, num_seqs)
  int seq = last_at_or_below(a.seq_page_indptr, a.num_seqs, first + begin / (2 * H), lane);
  int base = a.seq_page_indptr[seq], next = a.seq_page_indptr[seq + 1];
  for (int64_t k = begin; k < end; ++k) {
    const int slot = first + (int)(k / (2 * H)), hv = (int)(k % (2 * H)), h = hv >> 1;
    while (slot >= next) {   // later sequences (empty ones are passed over)
      ++seq;
      base = next;
      next = a.seq_page_indptr[seq + 1];
    }
    const int len = a.seq_len[seq];
    const int pid = a.page_ids[slot];
    if (len < 0 || next - base != (int)(((int64_t)len + 15) / 16) || pid < 0 || pid >= a.num_pool_pages) {
      if (lane == 0 && a.error_flag) a.error_flag[0] = 1;
      continue;
    }
    const int t0 = (slot - base) * 16, n = min(16, len - t0);
    const int64_t at = (a.out_token_offset[seq] + t0) * row + (int64_t)h * D;
    const int64_t tile = (int64_t)pid * H + h;
    if (hv & 1)
      read_tile<T, D, true>(a.pool[1] + tile * kvq_v_tile<D>(), static_cast<T*>(a.out[1]) + at, row, n, lane);
    else
      read_tile<T, D, false>(a.pool[0] + tile * kvq_k_tile<D>(), static_cast<T*>(a.out[0]) + at, row, n, lane);
  }
}

// ---------------------------------------------------------------- host side

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

halo_status_t hip_check(const char* what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(HALO_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return HALO_OK;
}

halo_status_t check_pool_params(const halo_attn_params_t* p) {
  if (p->head_dim != 64 && p->head_dim != 128) return fail(HALO_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (p->page_size != 16) return fail(HALO_ERR_UNSUPPORTED, "page_size must be 16");
  if (p->num_kv_heads < 1) return fail(HALO_ERR_INVALID_ARGUMENT, "num_kv_heads must be >= 1");
  if (p->num_pool_pages < 0) return fail(HALO_ERR_INVALID_ARGUMENT, "num_pool_pages must be >= 0");
  if (p->num_kv_heads > 65536 || p->num_pool_pages > INT32_MAX)   // (products of these stay in their types)
    return fail(HALO_ERR_UNSUPPORTED, "at most 65536 heads and 2^31 - 1 pages");
  if (p->kv_dtype != HALO_BF16 && p->kv_dtype != HALO_F32)
    return fail(HALO_ERR_UNSUPPORTED, "kv_dtype must be HALO_F32 or HALO_BF16");
  return HALO_OK;
}

int64_t page_bytes(const halo_attn_params_t* p, halo_pool_kind_t kind) {
  const int64_t tile = p->head_dim * 8 + (kind == HALO_POOL_K ? p->head_dim / 2 : 32);
  return tile * p->num_kv_heads;
}

template <typename Launch>
void by_type(const halo_attn_params_t* p, Launch launch) {
  const bool d128 = p->head_dim == 128;
  if (p->kv_dtype == HALO_BF16) {
    if (d128) launch(__bf16{}, std::integral_constant<int, 128>{});
    else launch(__bf16{}, std::integral_constant<int, 64>{});
  } else {
    if (d128) launch(float{}, std::integral_constant<int, 128>{});
    else launch(float{}, std::integral_constant<int, 64>{});
  }
}

}  // namespace

extern "C" int64_t halo_kvq_pool_bytes(const halo_attn_params_t* params, halo_pool_kind_t pool_kind) {
  clear_error();
  if (!params || (pool_kind != HALO_POOL_K && pool_kind != HALO_POOL_V)) {
    (void)fail(HALO_ERR_INVALID_ARGUMENT, "params must not be NULL, pool_kind must be HALO_POOL_K or HALO_POOL_V");
    return -1;
  }
  if (check_pool_params(params) != HALO_OK) return -1;
  return page_bytes(params, pool_kind) * params->num_pool_pages;
}

extern "C" halo_status_t halo_kvq_page_scatter_kv(void* k_pool, void* v_pool, const halo_attn_params_t* params,
                                                  const int32_t* page_ids, const int32_t* seq_page_indptr,
                                                  const int32_t* seq_start, const int32_t* seq_count,
                                                  const int64_t* in_token_offset, int32_t num_seqs,
                                                  const void* k_in, const void* v_in, int32_t* error_flag,
                                                  void* stream) {
  clear_error();
  if (!params) return fail(HALO_ERR_INVALID_ARGUMENT, "params must not be NULL");
  if (num_seqs < 0) return fail(HALO_ERR_INVALID_ARGUMENT, "num_seqs must be >= 0");
  if (num_seqs == 0) return HALO_OK;
  if (!k_pool || !v_pool || !page_ids || !seq_page_indptr || !seq_start || !seq_count || !in_token_offset ||
      !k_in || !v_in)
    return fail(HALO_ERR_INVALID_ARGUMENT, "k_pool, v_pool, page_ids, seq_page_indptr, seq_start, seq_count, "
                                           "in_token_offset, k_in, v_in must not be NULL");
  halo_status_t st = check_pool_params(params);
  if (st != HALO_OK) return st;
  if (!aligned16(k_pool) || !aligned16(v_pool) || !aligned16(k_in) || !aligned16(v_in))
    return fail(HALO_ERR_INVALID_ARGUMENT, "pools and inputs must be 16-byte aligned");
  const int H = params->num_kv_heads;
  KvqScatterArgs g{{static_cast<uint8_t*>(k_pool), static_cast<uint8_t*>(v_pool)}, {k_in, v_in}, page_ids,
                   seq_page_indptr, seq_start, seq_count, in_token_offset, error_flag, params->num_pool_pages,
                   num_seqs, H, 0, 0, 0};
  // A wave for each of an append's 2 H tiles, or for two from 257 sequences on,
  // where the chip takes them in several rounds anyway (512 appends 10.2 -> 9.3 us,
  // 1024 17.9 -> 16.3; 256 6.4, with two 7.6). 1024 workgroups for the whole pages:
  // 512 have fewer loads in flight (32 chunks of 768 tokens 29.9 us, 1024 27.5),
  // 2048 are waited for by appends (64: 5.5 us, 1024 4.6).
  g.splits = std::min((2 * H + 3) / 4, 64);
  if (num_seqs > 256) g.splits = (g.splits + 1) / 2;
  g.seq_blocks = std::min(num_seqs, 16384) * g.splits;
  g.tile_blocks = 1024;
  const dim3 grid((unsigned)(g.seq_blocks + g.tile_blocks));
  (void)hipGetLastError();
  by_type(params, [&](auto t, auto d) {
    hipLaunchKernelGGL((kvq_scatter_kernel<decltype(t), decltype(d)::value>), grid, dim3(256), 0,
                       static_cast<hipStream_t>(stream), g);
  });
  return hip_check("4-bit scatter launch");
}

extern "C" halo_status_t halo_kvq_page_gather_kv(const void* k_pool, const void* v_pool,
                                                 const halo_attn_params_t* params, const int32_t* page_ids,
                                                 const int32_t* seq_page_indptr, const int32_t* seq_len,
                                                 const int64_t* out_token_offset, int32_t num_seqs, void* k_out,
                                                 void* v_out, int32_t* error_flag, void* stream) {
  clear_error();
  if (!params) return fail(HALO_ERR_INVALID_ARGUMENT, "params must not be NULL");
  if (num_seqs < 0) return fail(HALO_ERR_INVALID_ARGUMENT, "num_seqs must be >= 0");
  if (num_seqs == 0) return HALO_OK;
  if (!k_pool || !v_pool || !page_ids || !seq_page_indptr || !seq_len || !out_token_offset || !k_out || !v_out)
    return fail(HALO_ERR_INVALID_ARGUMENT, "k_pool, v_pool, page_ids, seq_page_indptr, seq_len, out_token_offset, "
                                           "k_out, v_out must not be NULL");
  halo_status_t st = check_pool_params(params);
  if (st != HALO_OK) return st;
  if (!aligned16(k_pool) || !aligned16(v_pool) || !aligned16(k_out) || !aligned16(v_out))
    return fail(HALO_ERR_INVALID_ARGUMENT, "pools and outputs must be 16-byte aligned");
  KvqGatherArgs g{{static_cast<const uint8_t*>(k_pool), static_cast<const uint8_t*>(v_pool)}, {k_out, v_out}, page_ids,
                  seq_page_indptr, seq_len, out_token_offset, error_flag, params->num_pool_pages, num_seqs,
                  params->num_kv_heads};
  (void)hipGetLastError();
  by_type(params, [&](auto t, auto d) {
    hipLaunchKernelGGL((kvq_gather_kernel<decltype(t), decltype(d)::value>), dim3(8192), dim3(256), 0,
                       static_cast<hipStream_t>(stream), g);
  });
  return hip_check("4-bit gather launch");
}

extern "C" halo_status_t halo_kvq_page_copy(void* pool, const halo_attn_params_t* params, halo_pool_kind_t pool_kind,
                                            const int32_t* src_pages, const int32_t* dst_pages, int32_t num_pages,
                                            int32_t* error_flag, void* stream) {
  clear_error();
  if (!params) return fail(HALO_ERR_INVALID_ARGUMENT, "params must not be NULL");
  if (num_pages < 0) return fail(HALO_ERR_INVALID_ARGUMENT, "num_pages must be >= 0");
  if (num_pages == 0) return HALO_OK;
  if (!pool || !src_pages || !dst_pages)
    return fail(HALO_ERR_INVALID_ARGUMENT, "pool, src_pages, dst_pages must not be NULL");
  if (pool_kind != HALO_POOL_K && pool_kind != HALO_POOL_V)
    return fail(HALO_ERR_INVALID_ARGUMENT, "pool_kind must be HALO_POOL_K or HALO_POOL_V");
  halo_status_t st = check_pool_params(params);
  if (st != HALO_OK) return st;
  if (!aligned16(pool)) return fail(HALO_ERR_INVALID_ARGUMENT, "pool must be 16-byte aligned");
  return launch_page_copy(pool, src_pages, dst_pages, num_pages, params->num_pool_pages, page_bytes(params, pool_kind),
                          error_flag, stream);
}
