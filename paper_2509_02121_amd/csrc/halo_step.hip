// gfx950 kernels and entry points of the C ABI for what a step needs around
// its cache writes and its attention:
// step_tables_kernel: page lists, slots and positions of a step's tokens from
//   the lengths of its sequences, with new pages out of a free list;
// rope_kernel: queries and keys turned by their positions.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <string>
#include <type_traits>

#include "halo_internal.h"

using namespace halo;

namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- step tables

struct StepArgs {
  halo_step_tables_t out;
  const int32_t* seq_len;
  const int32_t* seq_new;
  int32_t* block_table;
  const int32_t* free_pages;
  const int32_t* free_next;
  int32_t* error_flag;
  int32_t num_seqs, table_width, num_free, max_tokens, max_pages;
  int32_t per;      // sequences of a group
  int32_t splits;   // workgroups of a group, which share its rows
  int32_t team;     // threads that take a sequence together: 64 or 256
};

// One sequence's cached and new tokens, and its pages. A sequence whose lengths
// are negative, or whose tokens do not fit its row of the table, takes part as
// an empty one.
struct StepSeq {
  int32_t len, count, have, need;
  bool bad;
  __device__ __forceinline__ StepSeq(const StepArgs& a, int i) {
    len = a.seq_len[i];
    count = a.seq_new[i];
    const int64_t room = min((int64_t)a.table_width * 16, (int64_t)INT32_MAX - 15);
    bad = len < 0 || count < 0 || (int64_t)len + count > room;
    if (bad) len = count = 0;
    have = (int)(((int64_t)len + 15) >> 4);
    need = (int)(((int64_t)len + count + 15) >> 4);
  }
};

// Sums that stay at 2^32 - 1 once they pass it: what does not fit an int32
// never seems to.
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }

__device__ __forceinline__ uint32_t wave_sum_sat(uint32_t x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x = add_sat(x, __shfl_xor(x, m));
  return x;
}

// The step's arrays are sums over the sequences before each one. Every
// workgroup sums the lengths of all sequences itself (8 bytes each, from the
// caches), those before its own group apart from the rest, and then writes its
// group's rows: one launch, without a second one or a wait between workgroups.
// The rows of a group are shared by `splits` workgroups. Bound by the launch
// (3.3 us for one sequence, 3.7 for 64) until the page lists are megabytes (1024
// sequences of 256-10240 tokens, 2.8 MB: 6.5 us).
__global__ __launch_bounds__(256) void step_tables_kernel(StepArgs a) {
  __shared__ uint32_t sums[4][7];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.num_seqs;
  const int group = (int)blockIdx.x / a.splits, split = (int)blockIdx.x % a.splits;
  const int first = (int)min((int64_t)n, (int64_t)group * a.per), last = (int)min((int64_t)n, (int64_t)first + a.per);
  // before the group: pages, new pages, tokens; of all: the same; malformed ones
  uint32_t s[7] = {0, 0, 0, 0, 0, 0, 0};
  for (int64_t i = tid; i < n; i += 256) {
    const StepSeq q(a, (int)i);
    s[3] = add_sat(s[3], q.need);
    s[4] = add_sat(s[4], q.need - q.have);
    s[5] = add_sat(s[5], q.count);
    s[6] |= q.bad ? 1u : 0u;
    if (i < first) {
      s[0] = add_sat(s[0], q.need);
      s[1] = add_sat(s[1], q.need - q.have);
      s[2] = add_sat(s[2], q.count);
    }
  }
#pragma unroll
  for (int k = 0; k < 7; ++k) s[k] = wave_sum_sat(s[k]);
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < 7; ++k) sums[wave][k] = s[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 7; ++k) s[k] = add_sat(add_sat(sums[0][k], sums[1][k]), add_sat(sums[2][k], sums[3][k]));
  const int free0 = a.free_next[0];
  const bool fits = free0 >= 0 && free0 <= a.num_free && s[4] <= (uint32_t)(a.num_free - free0) &&
                    s[3] <= (uint32_t)a.max_pages && s[5] <= (uint32_t)a.max_tokens;
  const bool lead = blockIdx.x == 0 && tid == 0;
  if (lead) {
    a.out.seq_page_indptr[n] = fits ? (int32_t)s[3] : 0;
    a.out.free_next[0] = fits ? free0 + (int32_t)s[4] : free0;
    if ((s[6] || !fits) && a.error_flag) a.error_flag[0] = 1;
  }
  // the group's sequences, a team of threads each
  const int teams = 256 / a.team, team = tid / a.team, member = tid % a.team;
  const int64_t at = (int64_t)split * a.team + member, stride = (int64_t)a.splits * a.team;
  uint32_t pages = s[0], taken = s[1], tokens = s[2];
  for (int i = first; i < last; ++i) {
    const StepSeq q(a, i);
    if ((i - first) % teams == team) {
      if (split == 0 && member == 0) {
        a.out.seq_page_indptr[i] = fits ? (int32_t)pages : 0;
        a.out.seq_start[i] = fits ? q.len : 0;
        a.out.seq_count[i] = fits ? q.count : 0;
        a.out.seq_end[i] = a.seq_len[i] + (fits ? q.count : 0);
        a.out.in_token_offset[i] = fits ? (int64_t)tokens : 0;
      }
      if (fits) {
        int32_t* row = a.block_table + (int64_t)i * a.table_width;
        const int32_t* fresh = a.free_pages + free0 + taken;   // page `have` on
        for (int64_t j = at; j < q.need; j += stride) {
          int32_t page;
          if (j < q.have) {
            page = row[j];
          } else {
            page = fresh[j - q.have];
            row[j] = page;
          }
          a.out.page_ids[pages + j] = page;
        }
        for (int64_t t = at; t < q.count; t += stride) {
          const int pos = q.len + (int)t, j = pos >> 4;
          const int32_t page = j < q.have ? row[j] : fresh[j - q.have];
          if (a.out.positions) a.out.positions[tokens + t] = pos;
          if (a.out.slots) a.out.slots[tokens + t] = page < 0 ? -1 : (int64_t)page * 16 + (pos & 15);
        }
      }
    }
    pages += q.need;
    taken += q.need - q.have;
    tokens += q.count;
  }
  // tokens behind the last
  for (int64_t t = (fits ? (int64_t)s[5] : 0) + (int64_t)blockIdx.x * 256 + tid; t < a.max_tokens;
       t += (int64_t)gridDim.x * 256) {
    if (a.out.positions) a.out.positions[t] = 0;
    if (a.out.slots) a.out.slots[t] = -1;
  }
}

// ---------------------------------------------------------------- rotary positions

struct RopeArgs {
  const void* in[2];   // q and k: [tokens][heads][D], tokens in_stride elements apart
  void* out[2];
  int64_t in_stride[2], out_stride[2];
  const int32_t* positions;
  const uint64_t* turns;
  float amplitude;
  int32_t tokens, heads0, heads;   // heads0 of q, heads of both
  int32_t rotary;
  int32_t slots;                   // threads of a token that share a unit, each with every slots-th head
};

// sin and cos of 2 pi x / 2^32. The top two bits of x + 2^29 are the quadrant;
// what is left is an angle within pi / 4, where the Taylor series to x^9 and
// x^10 end below 2^-28.
__device__ __forceinline__ void sincos_turn(uint32_t x, float& sn, float& cs) {
  const uint32_t quad = (x + 0x20000000u) >> 30;
  const float r = (float)(int32_t)(x - (quad << 30)) * 1.46291807926716e-9f;   // 2 pi / 2^32
  const float z = r * r;
  float s = 1.f / 362880.f, c = -1.f / 3628800.f;
  s = __builtin_fmaf(s, z, -1.f / 5040.f);
  s = __builtin_fmaf(s, z, 1.f / 120.f);
  s = __builtin_fmaf(s, z, -1.f / 6.f);
  s = __builtin_fmaf(s * z, r, r);
  c = __builtin_fmaf(c, z, 1.f / 40320.f);
  c = __builtin_fmaf(c, z, -1.f / 720.f);
  c = __builtin_fmaf(c, z, 1.f / 24.f);
  c = __builtin_fmaf(c, z, -0.5f);
  c = __builtin_fmaf(c, z, 1.f);
  const float a = quad & 1 ? c : s, b = quad & 1 ? s : c;
  sn = quad & 2 ? -a : a;
  cs = (quad + 1) & 2 ? -b : b;
}

// 16 bytes as floats, and back.
__device__ __forceinline__ void unpack(u32x4_t x, float (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(x[j]);
}
__device__ __forceinline__ void unpack(u32x4_t x, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(x[j] << 16);
    v[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u);
  }
}
__device__ __forceinline__ u32x4_t pack(const float (&v)[4]) {
  return __builtin_bit_cast(u32x4_t, f32x4_t{v[0], v[1], v[2], v[3]});
}
__device__ __forceinline__ u32x4_t pack(const float (&v)[8]) {
  bf16x8_t r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = (__bf16)v[j];
  return __builtin_bit_cast(u32x4_t, r);
}

// A thread holds one unit of a token: two 16-byte vectors of a head, E pairs of
// the rotary part (its neighbours, or the vectors R / 2 apart), or of the part
// that stays as it is. It works out the E angles once and turns the unit in
// every slots-th head.
//
// The angle in turns, position * f mod 1, is a product of integers: f is held
// as 64 bits after the point, and the product is cut to 32, so that it is less than
// 2^-32 of a turn (1.5e-9 rad) short, and off by f's rounding (up to 2^-34 at
// position 2^31), where a product in fp32 is off by whole radians at 10^6.
// Products and sums in fp32, rounded once to the output's type. Bound by HBM:
// q and k read and written once (16384 tokens of 32 + 8 heads, d 128, bf16: 336 MB
// in 67.7 us, 4.96 TB/s, where a device copy reaches 5.17).
template <typename T, int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int E = 16 / (int)sizeof(T);
  constexpr int U = D / (2 * E);   // units of a head
  const int unit = threadIdx.x % U;
  const int slot = (int)threadIdx.x / U % a.slots;
  const int64_t token = (int64_t)blockIdx.x * (256 / U / a.slots) + (int)threadIdx.x / U / a.slots;
  if (token >= a.tokens) return;
  const int turned = a.rotary / (2 * E);   // units of the rotary part
  const bool turn = unit < turned;
  int lo, hi;   // elements of the unit's vectors
  if (INTERLEAVED || !turn) {
    lo = 2 * E * unit;
    hi = lo + E;
  } else {
    lo = E * unit;
    hi = lo + a.rotary / 2;
  }
  float sn[E], cs[E];
  if (turn) {
    const uint32_t pos = (uint32_t)max(a.positions[token], 0);
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const uint64_t f = a.turns[E * unit + j];
      sincos_turn((uint32_t)(pos * f >> 32), sn[j], cs[j]);
      sn[j] *= a.amplitude;
      cs[j] *= a.amplitude;
    }
  }
#pragma unroll 4
  for (int h = slot; h < a.heads; h += a.slots) {
    const int z = h >= a.heads0 ? 1 : 0;
    const int64_t head = (int64_t)(h - (z ? a.heads0 : 0)) * D;
    const T* src = static_cast<const T*>(a.in[z]) + token * a.in_stride[z] + head;
    T* dst = static_cast<T*>(a.out[z]) + token * a.out_stride[z] + head;
    if (!turn && src == dst) continue;
    u32x4_t x = *reinterpret_cast<const u32x4_t*>(src + lo);
    u32x4_t y = *reinterpret_cast<const u32x4_t*>(src + hi);
    if (turn) {
      float v[E], w[E], p[E], q[E];
      unpack(x, v);
      unpack(y, w);
      if constexpr (INTERLEAVED) {
#pragma unroll
        for (int j = 0; j < E / 2; ++j) {
          p[2 * j] = v[2 * j] * cs[j] - v[2 * j + 1] * sn[j];
          p[2 * j + 1] = v[2 * j] * sn[j] + v[2 * j + 1] * cs[j];
          q[2 * j] = w[2 * j] * cs[E / 2 + j] - w[2 * j + 1] * sn[E / 2 + j];
          q[2 * j + 1] = w[2 * j] * sn[E / 2 + j] + w[2 * j + 1] * cs[E / 2 + j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) {
          p[j] = v[j] * cs[j] - w[j] * sn[j];
          q[j] = v[j] * sn[j] + w[j] * cs[j];
        }
      }
      x = pack(p);
      y = pack(q);
    }
    *reinterpret_cast<u32x4_t*>(dst + lo) = x;
    *reinterpret_cast<u32x4_t*>(dst + hi) = y;
  }
}

// ---------------------------------------------------------------- host side

// Memory that a call reads or writes.
struct Range {
  const char* name;
  const void* p;
  int64_t bytes;
};
bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + b.bytes && y < x + a.bytes;
}

// Whether two operands of `tokens` rows share memory. Rows the same stride apart may
// lie between each other (q and k in the rows of one projection).
struct Rows {
  const void* p;
  int64_t stride, width;   // bytes
};
bool rows_overlap(const Rows& a, const Rows& b, int64_t tokens) {
  const Range x{"", a.p, (tokens - 1) * a.stride + a.width}, y{"", b.p, (tokens - 1) * b.stride + b.width};
  if (!overlap(x, y)) return false;
  if (a.stride != b.stride) return true;
  const int64_t s = a.stride, d = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
  const int64_t ahead = ((d % s) + s) % s;   // from a row of a to the next one of b
  return ahead < a.width || s - ahead < b.width;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

halo_status_t hip_check(const char* what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(HALO_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return HALO_OK;
}

}  // namespace

extern "C" halo_status_t halo_kv_step_tables(const halo_step_sizes_t* sizes, const int32_t* seq_len,
                                             const int32_t* seq_new, int32_t* block_table,
                                             const int32_t* free_pages, const int32_t* free_next,
                                             const halo_step_tables_t* tables, int32_t* error_flag, void* stream) {
  clear_error();
  if (!sizes || !tables) return fail(HALO_ERR_INVALID_ARGUMENT, "sizes and tables must not be NULL");
  if (sizes->num_seqs < 0 || sizes->table_width < 0 || sizes->num_free < 0 || sizes->max_tokens < 0 ||
      sizes->max_pages < 0)
    return fail(HALO_ERR_INVALID_ARGUMENT, "every size must be >= 0");
  if (sizes->page_size != 16) return fail(HALO_ERR_UNSUPPORTED, "page_size must be 16");
  const bool seqs = sizes->num_seqs > 0;
  if (!free_next || !tables->free_next || !tables->seq_page_indptr ||
      (seqs && (!seq_len || !seq_new || !tables->seq_start || !tables->seq_count || !tables->seq_end ||
                !tables->in_token_offset)) ||
      (seqs && sizes->table_width > 0 && !block_table) || (sizes->num_free > 0 && !free_pages) ||
      (sizes->max_pages > 0 && !tables->page_ids))
    return fail(HALO_ERR_INVALID_ARGUMENT, "only positions, slots and error_flag (and arrays of no elements) may be NULL");
  // every workgroup reads the lengths and the free list while others write their
  // outputs
  const int64_t n = sizes->num_seqs;
  const Range reads[] = {{"seq_len", seq_len, 4 * n}, {"seq_new", seq_new, 4 * n},
                         {"free_pages", free_pages, 4 * (int64_t)sizes->num_free}, {"free_next", free_next, 4}};
  const Range writes[] = {{"block_table", block_table, 4 * n * sizes->table_width},
                          {"tables' seq_page_indptr", tables->seq_page_indptr, 4 * (n + 1)},
                          {"tables' page_ids", tables->page_ids, 4 * (int64_t)sizes->max_pages},
                          {"tables' seq_start", tables->seq_start, 4 * n},
                          {"tables' seq_count", tables->seq_count, 4 * n},
                          {"tables' seq_end", tables->seq_end, 4 * n},
                          {"tables' in_token_offset", tables->in_token_offset, 8 * n},
                          {"tables' positions", tables->positions, 4 * (int64_t)sizes->max_tokens},
                          {"tables' slots", tables->slots, 8 * (int64_t)sizes->max_tokens},
                          {"tables' free_next", tables->free_next, 4},
                          {"error_flag", error_flag, 4}};
  for (const Range& w : writes) {
    for (const Range& r : reads)
      if (overlap(w, r)) return fail(HALO_ERR_INVALID_ARGUMENT, std::string(r.name) + " must not overlap " + w.name);
    for (const Range* v = writes; v != &w; ++v)
      if (overlap(w, *v)) return fail(HALO_ERR_INVALID_ARGUMENT, std::string(v->name) + " must not overlap " + w.name);
  }
  StepArgs g{*tables, seq_len, seq_new, block_table, free_pages, free_next, error_flag,
             sizes->num_seqs, sizes->table_width, sizes->num_free, sizes->max_tokens, sizes->max_pages, 0, 0, 0};
  // A group of sequences for each of up to 512 workgroups (2000 sequences 6.6 us,
  // with 256 8.0), and more workgroups for a group where rows or tokens are long
  // and sequences few.
  const int groups = std::min(std::max(sizes->num_seqs, 1), 2 * kNumCUs);
  g.per = (std::max(sizes->num_seqs, 1) + groups - 1) / groups;
  g.team = g.per >= 4 ? 64 : 256;
  const int64_t longest = std::max<int64_t>((sizes->table_width + 511) / 512, (sizes->max_tokens + 1023) / 1024);
  g.splits = (int)std::max<int64_t>(1, std::min<int64_t>(longest, 2 * kNumCUs / groups));
  (void)hipGetLastError();
  hipLaunchKernelGGL(step_tables_kernel, dim3(groups * g.splits), dim3(256), 0, static_cast<hipStream_t>(stream), g);
  return hip_check("step tables launch");
}

extern "C" halo_status_t halo_rope_qk(const halo_rope_params_t* rope, float amplitude, const uint64_t* turns,
                                      const int32_t* positions, int32_t num_tokens, int32_t num_q_heads,
                                      int32_t num_kv_heads, halo_dtype_t dtype, const void* q, int64_t q_stride,
                                      const void* k, int64_t k_stride, void* q_out, int64_t q_out_stride,
                                      void* k_out, int64_t k_out_stride, void* stream) {
  clear_error();
  if (!rope) return fail(HALO_ERR_INVALID_ARGUMENT, "rope must not be NULL");
  if (rope->head_dim != 64 && rope->head_dim != 128)
    return fail(HALO_ERR_UNSUPPORTED, "head_dim must be 64 or 128, got " + std::to_string(rope->head_dim));
  if (rope->rotary_dim < 16 || rope->rotary_dim > rope->head_dim || rope->rotary_dim % 16 != 0)
    return fail(HALO_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 in [16, head_dim], got " +
                                          std::to_string(rope->rotary_dim));
  if (dtype != HALO_F32 && dtype != HALO_BF16) return fail(HALO_ERR_UNSUPPORTED, "dtype must be HALO_F32 or HALO_BF16");
  if (num_tokens < 0 || num_q_heads < 0 || num_kv_heads < 0)
    return fail(HALO_ERR_INVALID_ARGUMENT, "num_tokens, num_q_heads and num_kv_heads must be >= 0");
  uint32_t bits;
  memcpy(&bits, &amplitude, 4);   // (NaN is told by its bits, since the build drops float tests for it)
  if ((bits & 0x7f800000u) == 0x7f800000u) return fail(HALO_ERR_INVALID_ARGUMENT, "amplitude must be finite");
  if ((int64_t)num_q_heads + num_kv_heads > 65536)
    return fail(HALO_ERR_UNSUPPORTED, "at most 65536 heads");
  if (num_tokens == 0 || num_q_heads + num_kv_heads == 0) return HALO_OK;
  if (!turns || !positions) return fail(HALO_ERR_INVALID_ARGUMENT, "turns and positions must not be NULL");
  if ((reinterpret_cast<uintptr_t>(turns) & 7) != 0)
    return fail(HALO_ERR_INVALID_ARGUMENT, "turns must be 8-byte aligned");
  const int elt = dtype == HALO_BF16 ? 2 : 4, D = rope->head_dim;
  RopeArgs g{};
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const int64_t in_stride[2] = {q_stride, k_stride}, out_stride[2] = {q_out_stride, k_out_stride};
  const int heads[2] = {num_q_heads, num_kv_heads};
  for (int z = 0; z < 2; ++z) {
    if (heads[z] == 0) continue;
    if (!in[z] || !out[z]) return fail(HALO_ERR_INVALID_ARGUMENT, "q, k and their outputs must not be NULL");
    if (in_stride[z] < (int64_t)heads[z] * D || out_stride[z] < (int64_t)heads[z] * D)
      return fail(HALO_ERR_INVALID_ARGUMENT, "a token's stride must be >= its heads * head_dim elements");
    if (!aligned16(in[z]) || !aligned16(out[z]) || in_stride[z] * elt % 16 != 0 || out_stride[z] * elt % 16 != 0)
      return fail(HALO_ERR_INVALID_ARGUMENT, "q, k, their outputs and their tokens must be 16-byte aligned");
    if (in[z] == out[z] && in_stride[z] != out_stride[z])
      return fail(HALO_ERR_INVALID_ARGUMENT, "in place, the strides must be equal");
    g.in[z] = in[z];
    g.out[z] = out[z];
    g.in_stride[z] = in_stride[z];
    g.out_stride[z] = out_stride[z];
  }
  for (int z = 0; z < 2; ++z) {
    if (heads[z] == 0) continue;
    const int64_t width = (int64_t)heads[z] * D * elt;
    const Rows to{out[z], out_stride[z] * elt, width};
    for (int y = 0; y < 2; ++y) {
      if (heads[y] == 0) continue;
      const int64_t w = (int64_t)heads[y] * D * elt;
      if ((y != z || in[y] != out[z]) && rows_overlap(to, Rows{in[y], in_stride[y] * elt, w}, num_tokens))
        return fail(HALO_ERR_INVALID_ARGUMENT, "an output must be its operand, or overlap none");
      if (y < z && rows_overlap(to, Rows{out[y], out_stride[y] * elt, w}, num_tokens))
        return fail(HALO_ERR_INVALID_ARGUMENT, "q_out and k_out must not overlap");
    }
  }
  g.positions = positions;
  g.turns = turns;
  g.amplitude = amplitude;
  g.tokens = num_tokens;
  g.heads0 = num_q_heads;
  g.heads = num_q_heads + num_kv_heads;
  g.rotary = rope->rotary_dim;
  // Of a workgroup's 256 threads `slots` share each unit of a token: one for
  // every head, as far as they go. Fewer work out the angles less often, but have
  // fewer loads in flight: 16384 tokens of 32 + 8 heads (d 128) take 67.7 us with
  // 32, 70.9 with 8, 76.0 with 4; 64 tokens 3.7, 4.8 and 7.1.
  const int units = D * elt / 32, most = 256 / units;
  int slots = 1;
  while (slots < most && slots < g.heads) slots *= 2;
  g.slots = slots;
  const int per_block = most / slots;
  const int64_t blocks = ((int64_t)num_tokens + per_block - 1) / per_block;
  if (blocks >= 1 << 24) return fail(HALO_ERR_UNSUPPORTED, "too many tokens for one call (2^32 threads)");
  const dim3 grid((unsigned)blocks);
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  auto launch = [&](auto t, auto d, auto i) {
    hipLaunchKernelGGL((rope_kernel<decltype(t), decltype(d)::value, decltype(i)::value>), grid, dim3(256), 0, st, g);
  };
  auto by_layout = [&](auto t, auto d) {
    if (rope->interleaved) launch(t, d, std::true_type{});
    else launch(t, d, std::false_type{});
  };
  auto by_dim = [&](auto t) {
    if (D == 128) by_layout(t, std::integral_constant<int, 128>{});
    else by_layout(t, std::integral_constant<int, 64>{});
  };
  if (dtype == HALO_BF16) by_dim(__bf16{});
  else by_dim(float{});
  return hip_check("rope launch");
}
