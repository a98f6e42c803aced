// Device code that the attention kernels over bf16 / fp32 pools
// (halo_kernels.hip) and over 4-bit ones (halo_kvq_attn.hip) share: fragments
// and MFMA wrappers, reductions inside a wave, spans and steps, and the wide
// items.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "halo_internal.h"
#include "halo_kvq_format.h"

namespace halo {

struct AttnArgs {
  const void* q;
  const void* k_pool;
  const void* v_pool;
  void* o;
  float* lse;
  void* part_o;      // partial O rows, in the output element type
  float* part_lse;   // (4-bit pools, bf16 output: pairs with a scale, see store_half)
  const int32_t* seg_page_off;
  const int32_t* seg_len;
  const int32_t* page_ids;
  const Item* items;        // narrow item slots: slot k of narrow workgroup b is item b * narrow_slots + k
  const ItemRec* item_recs; // their lane records
  const Item* wide_items;   // wide items (one workgroup each)
  const Span* spans;
  const Row* rows;
  int32_t n_items;
  int32_t n_wide;
  int32_t wide_blocks;     // grid blocks of the wide role (n_wide padded, see xcd_remap)
  int32_t narrow_blocks;   // grid blocks of the narrow role (a multiple of 8)
  int32_t narrow_slots;    // item slots per narrow workgroup (one per wave)
  int32_t wide_group;      // consecutive wide items kept on one XCD
  int32_t wide_span;       // launch rounds (of 8 blocks) the wide rounds are spread over
  int32_t num_kv_heads;
  float scale_log2;   // sm_scale * log2(e)
};

// The items of a plan over 4-bit pools (halo_kvq_attn.hip).
void launch_attention_kvq(AttnArgs args, const halo_plan& plan, hipStream_t stream);

}  // namespace halo

using namespace halo;

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLog2e = 1.44269504088896340736f;

// ---------------------------------------------------------------- fragments
// A fragment is the 8 K-slot values one lane feeds to a 16x16x32 MFMA.

template <typename T> struct FragOf;
template <> struct FragOf<__bf16> { using type = bf16x8_t; };
template <> struct FragOf<float> { using type = f32x8_t; };

__device__ __forceinline__ bf16x8_t load8(const __bf16* p) {
  return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p));
}
__device__ __forceinline__ f32x8_t load8(const float* p) {
  return *reinterpret_cast<const f32x8_t*>(p);
}

template <typename F> __device__ __forceinline__ F zero_frag() { return F{}; }

// 16-byte global load; NT marks data read once (non-temporal: streamed past
// the caches, measured 7.2 TB/s vs 5.8 TB/s for plain loads on a read stream).
template <bool NT>
__device__ __forceinline__ u32x4_t ld16(const void* p) {
  if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  else return *reinterpret_cast<const u32x4_t*>(p);
}
// A load from an address told to be global. From an integer the compiler makes
// flat loads, which count as LDS accesses too and which it can only wait for all
// together.
template <typename V, bool NT = false>
__device__ __forceinline__ V load_global(int64_t at) {
  typedef const V __attribute__((address_space(1))) * global_t;
  if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<global_t>(at));
  else return *reinterpret_cast<global_t>(at);
}
// K fragment: dims d0..d0+7 of key t in a K tile stored as [D/E][16][E]
// (E elements per 16-byte unit).
template <bool NT>
__device__ __forceinline__ f32x8_t load_k8(const float* tile, int t, int d0) {
  const u32x4_t lo = ld16<NT>(tile + ((d0 >> 2) * 16 + t) * 4);
  const u32x4_t hi = ld16<NT>(tile + (((d0 >> 2) + 1) * 16 + t) * 4);
  return __builtin_bit_cast(f32x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// V fragment: the 8 slot-ordered keys at element offset off of a V tile
// stored dim-major as [D][16] (one dim row holds tokens 0-3, 8-11, 4-7,
// 12-15, so slots 8h..8h+7 are the keys one lane multiplies).
template <bool NT>
__device__ __forceinline__ f32x8_t load_v8(const float* page, int off) {
  const u32x4_t lo = ld16<NT>(page + off);
  const u32x4_t hi = ld16<NT>(page + off + 4);
  return __builtin_bit_cast(f32x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Key (relative to the first key of a 32-key step) behind slot j of a lane
// in lane group grp. QK tile X (X = j / 4) takes its 16 A rows as keys
// 8X..8X+7 of page 0 (rows 0-7) and of page 1 (rows 8-15); MFMA output
// register i of lane group grp is tile row 4 grp + i, i.e. page grp / 2,
// key 8X + 4 (grp % 2) + i.
__device__ __forceinline__ int slot_key(int grp, int j) {
  return 16 * (grp >> 1) + 8 * (j >> 2) + 4 * (grp & 1) + (j & 3);
}

// D(16x16) += A(16x32) B(32x16). bf16: one MFMA. fp32: the same 32-deep
// contraction as eight 16x16x4 MFMAs, slot j of every lane in the j-th one,
// so both element types share one register layout.
__device__ __forceinline__ f32x4_t mma(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mma(f32x8_t a, f32x8_t b, f32x4_t c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// D(32x32) += A(32x16) B(16x32), bf16 operands, fp32 accumulate. Lane
// (c = lane % 32, h = lane / 32): A row c and B column c, k = 8h..8h+7;
// result register i holds row 8 (i / 4) + 4h + i % 4, column c.
__device__ __forceinline__ f32x16_t mma32(bf16x8_t a, bf16x8_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bf16x8_t to_frag(const float (&p)[8], bf16x8_t*) {
  bf16x8_t r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = (__bf16)p[j];
  return r;
}
__device__ __forceinline__ f32x8_t to_frag(const float (&p)[8], f32x8_t*) {
  f32x8_t r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = p[j];
  return r;
}

// x as a sum of N bf16 fragments, the largest first.
template <int N>
__device__ __forceinline__ void split(const float (&x)[8], bf16x8_t (&f)[N]) {
  float r[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = x[j];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      f[n][j] = (__bf16)r[j];
      if (n + 1 < N) r[j] -= (float)f[n][j];
    }
}

__device__ __forceinline__ void store4(float* dst, f32x4_t v) {
  *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
}
// Partial results (read once, by the merge launch): four elements of a row
// per lane, so a row's line is written in 16-byte (fp32) or 8-byte (bf16)
// pieces by several instructions. fp32 pieces go past the caches; bf16
// pieces are half as large, and written past the caches they cost more than
// they save (measured on the 70B-shaped decode: 966 against 934 us of
// attention for fp32 partials), so they go through L2, which assembles the
// lines before they reach HBM.
__device__ __forceinline__ void store4_part(float* dst, f32x4_t v) {
  __builtin_nontemporal_store(v, reinterpret_cast<f32x4_t*>(dst));
}
__device__ __forceinline__ void store4(__bf16* dst, f32x4_t v) {
  typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
  bf16x4_t r;
  r[0] = (__bf16)v[0];
  r[1] = (__bf16)v[1];
  r[2] = (__bf16)v[2];
  r[3] = (__bf16)v[3];
  *reinterpret_cast<uint2*>(dst) = __builtin_bit_cast(uint2, r);
}
__device__ __forceinline__ void store4_part(__bf16* dst, f32x4_t v) { store4(dst, v); }

// Partial results over 4-bit pools with a bf16 output: as long as bf16 ones, but in
// fp16 with a power of two for each row, the largest finite element's (an infinity
// stays one in fp16, and leaves the row's other dims as they are), so that each is off
// by at most 2^-11 of itself (or 2^-25 of the row's largest) where bf16 is by 2^-8:
// rows of three or more partials were otherwise further off than the output's
// rounding (70B-shaped decode: 0.0027 of the row, 0.0022 so; 64 requests on 2048 keys
// 0.0024 and 0.0018). The scale stands beside the row's LSE, one load for both.
template <typename V, int N>
__device__ __forceinline__ float largest_finite(const V (&acc)[N]) {
  constexpr int kPer = sizeof(V) / 4;
  const float inf = -kNegInf;
  float top = 0.f;
#pragma unroll
  for (int b = 0; b < N; ++b)
#pragma unroll
    for (int j = 0; j < kPer; ++j) top = fmaxf(top, fabsf(acc[b][j]));
  if (__any(top == inf)) {
    top = 0.f;
#pragma unroll
    for (int b = 0; b < N; ++b)
#pragma unroll
      for (int j = 0; j < kPer; ++j) top = fmaxf(top, fabsf(acc[b][j]) == inf ? 0.f : fabsf(acc[b][j]));
  }
  return top;
}
__device__ __forceinline__ float row_scale(float top) {
  const uint32_t e = min(__float_as_uint(top) & 0x7f800000u, 0x7e800000u);
  return __uint_as_float(e ? e : 0x3f800000u);
}
__device__ __forceinline__ float reciprocal_of_scale(float scale) {   // of a power of two in [2^-126, 2^126]
  return __uint_as_float(0x7f000000u - __float_as_uint(scale));
}
__device__ __forceinline__ void store_half(void* dst, f32x4_t v) {
  typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
  f16x4_t r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = (_Float16)v[j];
  *reinterpret_cast<uint2*>(dst) = __builtin_bit_cast(uint2, r);
}

// Reductions over the four 16-lane rows of a wave (lanes l, l^16, l^32,
// l^48) with the gfx950 row-swap instructions, which stay on the VALU
// instead of going through the LDS crossbar like a generic shuffle. Each
// swap leaves, in every lane, the pair {own value, value of lane l^16} (or
// l^32), in some order; max and sum are symmetric in the pair.
__device__ __forceinline__ float rows_max(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Reductions over the two 32-lane halves of a wave (lanes l and l^32).
__device__ __forceinline__ float halves_max(float x) {
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// ---------------------------------------------------------------- attention

// Workgroups are dealt to the 8 XCDs round-robin by block index, and each
// XCD has its own L2. Blocks that read the same pages (the row groups of one
// shared chunk) are made consecutive on one XCD: physical block p of a
// segment (p % 8 = XCD, p / 8 = its turn there) runs logical block
//   ((p / 8) / S * 8 + p % 8) * S + (p / 8) % S,
// i.e. groups of S logical blocks go round-robin to XCDs, in order. The
// segment length is a multiple of 8 S, so this is a permutation.
// Within an XCD, workgroups are dispatched in order and in turn to its 4
// shader engines (the XCD's j-th workgroup goes to engine j % 4, in a fixed
// order): a workgroup waits for its engine even when another engine has a
// free CU. The launch therefore mixes wide and narrow workgroups in whole
// cycles of kSeCycle rounds, so every engine gets the same kinds at the same
// time.
constexpr int kSeCycle = 4;

__device__ __forceinline__ int xcd_remap(int p, int S) {
  const int x = p & 7, j = p >> 3;
  return ((j / S) * 8 + x) * S + j % S;
}

// s_waitcnt with only the vector-memory counter limited (gfx9 encoding:
// vmcnt low bits [3:0] and high bits [15:14]; expcnt and lgkmcnt at their
// "no wait" maxima).
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x70 | 0xF00);
}
__device__ __forceinline__ void wait_lgkmcnt0() { __builtin_amdgcn_s_waitcnt(0xC07F); }

// A span's keys and its page ids, one page per lane (a span has at most 64
// pages), so a step finds its page ids with two lane reads instead of
// dependent memory loads.
struct SpanState {
  int kb, ke, causal;
  int vpid;      // lane l: page id of the span's l-th page
  bool valid;
};

// Position of one 32-key step.
struct StepPos {
  int t0;          // first key of the step (segment-local, multiple of 32)
  int key_end;     // end of its span
  int causal;
  int pid0, pid1;  // page ids of the step's two pages (pid1 == pid0 if absent)
  bool has1;
  bool valid;
  bool full;       // all 32 keys visible to every row: inside the span, no causal mask
};

// Field-wise choice between two step positions (a conditional on the
// structs themselves would select their addresses and keep them in memory).
__device__ __forceinline__ StepPos pick(bool c, const StepPos& x, const StepPos& y) {
  StepPos r;
  r.t0 = c ? x.t0 : y.t0;
  r.key_end = c ? x.key_end : y.key_end;
  r.causal = c ? x.causal : y.causal;
  r.pid0 = c ? x.pid0 : y.pid0;
  r.pid1 = c ? x.pid1 : y.pid1;
  r.has1 = c ? x.has1 : y.has1;
  r.valid = c ? x.valid : y.valid;
  r.full = c ? x.full : y.full;
  return r;
}

// Operand registers of one step: K for the two 16-key QK tiles, V^T for
// the NB output blocks.
template <typename F, int NS, int NB>
struct StepRegs {
  F k[2][NS];
  F v[NB];
};

// The LSE bits of a partial result. A NaN sum (NaN or +inf scores) gives +inf,
// which makes the row's weights NaN in the merge: O = NaN and LSE = -inf, as
// when one item holds the row. (With -inf, as where the row has no key, a merge
// would skip the partial. NaN is told by its bits, since the build drops float
// tests for it. The merges stay as they are: a case of its own there costs a
// decode of 64 requests on 2048 keys 0.25 us of 21.)
__device__ __forceinline__ int part_lse_bits(float lse2, float sum) {
  const bool nan = (__float_as_int(sum) & 0x7fffffff) > 0x7f800000;
  return nan ? 0x7f800000 : __float_as_int(lse2);
}

// This lane's words of a narrow item's record: its row's q_row and second
// word (lane % 16), and page lane % 32 of the first span.
struct RecLane {
  int32_t q_row, aux, page;
};

// The end of a narrow item: lane (col, grp) holds dims 16b + 4grp .. + 3 of row
// col in acc[b], and its share of the row's sum.
// HALF: partial results by store_half.
template <typename T, int D, typename TO, bool HALF = false>
__device__ __forceinline__ void finish_item(const AttnArgs& a, const Item& it, const Row& row, int col, int grp,
                                            f32x4_t (&acc)[D / 16], float m, float lsum) {
  constexpr int NB = D / 16;
  lsum = rows_sum(lsum);
  const bool has_row = col < it.n_rows;
  const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
  const float lse2 = lsum > 0.f ? m + __log2f(lsum) : kNegInf;
  if (it.part_base >= 0) {
    if (sizeof(T) == 4 && has_row && (it.flags & kItemPiece)) {   // (bf16 pieces are wide items)
      const int64_t prow = (int64_t)it.part_base + col;
      float* dst = static_cast<float*>(a.part_o) + prow * D + 4 * grp;
#pragma unroll
      for (int b = 0; b < NB; ++b) store4(dst + 16 * b, acc[b] * inv);
      if (grp == 0) reinterpret_cast<int*>(a.part_lse)[prow] = part_lse_bits(lse2, lsum);
    } else if constexpr (HALF) {
      const float scale = row_scale(rows_max(largest_finite(acc)) * inv), x = inv * reciprocal_of_scale(scale);
      if (has_row) {
        const int64_t prow = row.slot;
        uint16_t* dst = static_cast<uint16_t*>(a.part_o) + prow * D + 4 * grp;
#pragma unroll
        for (int b = 0; b < NB; ++b) store_half(dst + 16 * b, acc[b] * x);
        if (grp == 0)
          reinterpret_cast<int2*>(a.part_lse)[prow] = make_int2(part_lse_bits(lse2, lsum), __float_as_int(scale));
      }
    } else if (has_row) {
      const int64_t prow = row.slot;
      TO* dst = static_cast<TO*>(a.part_o) + prow * D + 4 * grp;
#pragma unroll
      for (int b = 0; b < NB; ++b) store4_part(dst + 16 * b, acc[b] * inv);
      if (grp == 0) reinterpret_cast<int*>(a.part_lse)[prow] = part_lse_bits(lse2, lsum);
    }
  } else if (has_row) {
    TO* dst = static_cast<TO*>(a.o) + (int64_t)row.q_row * D + 4 * grp;
#pragma unroll
    for (int b = 0; b < NB; ++b) store4(dst + 16 * b, acc[b] * inv);
    if (grp == 0 && a.lse) a.lse[row.q_row] = lse2 == kNegInf ? kNegInf : lse2 * kLn2;
  }
}

// Waves per workgroup: 8 for bf16 (two per SIMD, so one wave's softmax
// overlaps another's MFMAs), 4 for fp32, whose operand registers allow only
// one wave per SIMD.
template <typename T> constexpr int block_waves() { return sizeof(T) == 2 ? 8 : 4; }

// ---------------------------------------------------------------- wide items
// A wide item holds up to W * 32 query rows of one kv head against a span
// list: a workgroup of W waves (kWideWaves, or kSmallWideWaves in
// wide_kernel), 32 rows per wave, all rows sharing the key stream. Used for
// the grouped prefix pass (many rows share one segment, §2 intra-batch prefix
// sharing) and for chunked prefill (§4.1).
//
// Loads. Each 32-key step's K and V (two pages) are read once per workgroup,
// by direct global-to-LDS loads into a ring of S step images, so no registers
// hold data in transit. A step image is 2 * D/32 + D/16 blocks of 1 KB (16 KB
// at d = 128), each from one page. With c = L % 32, h = L / 32 of lane L:
//   K block (page g, units 4j..4j+3): as stored; lane L fetches key L % 16 of
//     unit 4j + L / 16. The fragment of dims 16s..16s+15 is then, per lane,
//     page c / 16, key c % 16, unit 2s + h: four runs of 256 bytes;
//   V block (page g, dims 32b..+31): lane L fetches dim 32b + c, slots
//     8h..8h+7, and every lane reads its own 16 bytes back.
// Both reads are free of bank conflicts.
//
// Products use v_mfma_f32_32x32x16_bf16, the shape that reaches the bf16
// peak on gfx950 (measured 2.48 PFLOP/s, against 1.39 for 16x16x32):
//   S^T (32 keys x 32 rows) = K Q^T, 8 products over d = 128; lane (c, h)
//     holds row c, keys 8 (i / 4) + 4 h + i % 4 in register i;
//   O^T (32 dims x 32 rows) += V^T P^T per page of the step: the B operand of
//     page g is registers 8g..8g+7 of that lane, i.e. keys 8j/4 + 4h + j%4 of
//     page g, which the V slot order keeps in 16 contiguous bytes.
//
// Compute. Iteration t issues the MFMAs of P V for step t-1 and of Q K^T for
// step t+1, and meanwhile runs the softmax of step t on the VALU: the three
// are independent, so the matrix cores and the VALU overlap inside each
// wave (and the two waves of a SIMD fill each other's stalls).
//
// Softmax rescaling is lazy: a row's reference maximum only moves when a
// step's maximum exceeds it by more than kRescaleLog2 (so weights stay below
// 2^kRescaleLog2); the result is the same softmax, and the accumulator
// rescale runs only on the rare steps where some row moves.
constexpr float kRescaleLog2 = 8.f;

// Bytes of the wide items' LDS ring: S step images of 2 * D/32 + D/16 blocks
// of 1 KB.
template <int D, int S> constexpr int wide_ring_bytes() { return S * (D / 16 + 2 * (D / 32)) * 1024; }

// 4-bit pools (KVQ, workgroups of four waves). The loads go to registers instead: a
// wave has half of one page's K tile and half of its V tile. An iteration later it
// converts them to bf16, scales included, and writes them into the step image in
// the form above, which from there on is read as any other; every value is
// converted once for the workgroup's rows. K is one conversion per two values. V
// scales run along the keys of a dim: see kvq_decode_keys. (On the softmax's weights
// instead, 16 products and 4 LDS reads a step for every wave, they took registers
// that had to be spilled inside the loop: chunked prefill 1765 us, at the conversion 1290.) Only in a
// step with masked keys, whose scales may be NaN, are they put on the weights, with
// the masked ones at 0. The conversion has no branch and runs between the MFMAs of
// the step before: with a K or a V tile to a wave, ahead of them, it cost 280 of
// 1219 us.
constexpr int kKvqStages = 4;
template <int D> constexpr int kvq_image_bytes() { return (D / 16 + 2 * (D / 32)) * 1024 + 128; }

// What a lane holds of a step: ND dwords of K codes and their scale bytes, ND of V
// codes and the scales of their 8 keys in bf16.
template <int ND> struct KvqRegs {
  uint32_t k[ND], v[ND];
  uint32_t k_scale;
  u32x4_t v_scale;
};

// A step's softmax weights between their softmax and their product with V: the
// bf16 operands, one per page. Or, where the output is fp32 and every other
// operand of P V exact in bf16 (4-bit V), the weights in fp32, which are split into
// three bf16 parts at the product: the output then has fp32's accuracy, not that of
// bf16 weights (2^-9 each).
template <bool EXACT> struct Weights {
  bf16x8_t f[2];
};
template <> struct Weights<true> {
  float p[16];
};

// A workgroup of W waves and an S-stage ring, for the item's rows from row0 on.
template <int D, typename TO, int W, int S, bool KVQ = false>
__device__ __forceinline__ void wide_item(const AttnArgs& a, int item_id, uint8_t* smem, int row0 = 0) {
  using T = __bf16;
  using F = bf16x8_t;
  constexpr int NK = D / 16;                      // 16-dim slices of Q K^T
  constexpr int NO = D / 32;                      // 32-dim output blocks
  constexpr int kBlocks = NK + 2 * NO;            // 1 KB blocks per step image
  constexpr int kStepBytes = kBlocks * 1024;
  static_assert(kBlocks % W == 0, "step blocks must split evenly over the waves");
  constexpr int kLoadsPerWave = kBlocks / W;
  static_assert(S >= 4 && S % 2 == 0, "the ring needs >= 4 stages, an even count keeps tile parity static");
  constexpr int64_t kTile = 16 * D;
  static_assert(S * kStepBytes == (wide_ring_bytes<D, S>()), "ring size");
  constexpr int kImageBytes = KVQ ? kvq_image_bytes<D>() : kStepBytes;
  constexpr int kImages = KVQ ? kKvqStages : S;
  static_assert(!KVQ || S == kKvqStages, "an image for each stage of the step ring");
  uint8_t (*lds)[kImageBytes] = reinterpret_cast<uint8_t (*)[kImageBytes]>(smem);

  const int wave = threadIdx.x >> 6;
  const int uwave = __builtin_amdgcn_readfirstlane(wave);   // on the scalar unit, for addresses
  const int lane = threadIdx.x & 63;
  const int c = lane & 31;
  const int h = lane >> 5;
  const Item it = a.wide_items[item_id];
  if (KVQ && row0 >= it.n_rows) return;   // (a run past the rows of a shorter item)
  // waves without rows still load their share of every step image
  const bool computes = row0 + wave * 32 < it.n_rows;

  // This lane's row: row c of this wave's block.
  const int r = row0 + wave * 32 + c;
  const Row row = r < it.n_rows ? a.rows[it.row_begin + r] : Row{-1, 0, -1, -1};
  F qf[NK];
  {
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(row.q_row < 0 ? 0 : row.q_row) * D + 8 * h;
#pragma unroll
    for (int s = 0; s < NK; ++s) qf[s] = row.q_row >= 0 ? load8(qp + 16 * s) : zero_frag<F>();
  }

  const int64_t page_stride = (int64_t)a.num_kv_heads * kTile;
  const T* kbase = static_cast<const T*>(a.k_pool) + (int64_t)it.kv_head * kTile;
  const T* vbase = static_cast<const T*>(a.v_pool) + (int64_t)it.kv_head * kTile;

  // ---- span cursor (identical, wave-uniform, in every wave)
  auto load_span = [&](int si) {
    SpanState st;
    st.valid = si < it.n_spans;
    st.kb = st.ke = st.causal = 0;
    st.vpid = 0;
    if (st.valid) {
      const Span sp = a.spans[it.span_begin + si];
      st.kb = sp.key_begin;
      st.ke = sp.key_end;
      st.causal = sp.causal;
      const int np = (sp.key_end - sp.key_begin + 15) >> 4;
      st.vpid = lane < np ? a.page_ids[sp.page_off + lane] : 0;
    }
    return st;
  };
  int si = 0;
  SpanState cur = load_span(0);
  SpanState nxt = load_span(1);
  int t_next = cur.kb;
  auto advance = [&]() {
    if (t_next >= cur.ke) {
      cur = nxt;
      ++si;
      nxt = load_span(si + 1);
      t_next = cur.kb;
    }
    StepPos p;
    p.valid = cur.valid;
    p.t0 = t_next;
    p.key_end = cur.ke;
    p.causal = cur.causal;
    const int j = (t_next - cur.kb) >> 4;
    p.has1 = t_next + 16 < cur.ke;
    p.full = t_next + kKeysPerStep <= cur.ke && !cur.causal;
    p.pid0 = __builtin_amdgcn_readlane(cur.vpid, j);
    p.pid1 = __builtin_amdgcn_readlane(cur.vpid, j + (p.has1 ? 1 : 0));
    t_next += kKeysPerStep;
    return p;
  };

  // ---- loads: this wave writes blocks wave + W * k of a step image. A block
  // lies in one page, so its address is a wave-uniform base and a lane offset
  // that never changes: the addresses cost no vector instructions (with lanes
  // of one block in both pages, ~20 a step and wave beside ~100 of softmax:
  // chunked prefill 1200 -> 1163 us, short chunks 88 -> 79 us).
  const uint32_t k_off = lane * 16, v_off = c * 32 + h * 16;
  // (readfirstlane keeps a base whole: the compiler would otherwise add the
  // lane offset to the pool's address first and the page's to that, per lane)
  auto uniform64 = [](int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
  };
  auto issue = [&](const StepPos& p, uint8_t* img) {
    const int64_t o0 = uniform64((int64_t)(uint32_t)p.pid0 * page_stride * (int64_t)sizeof(T));
    const int64_t o1 = uniform64((int64_t)(uint32_t)p.pid1 * page_stride * (int64_t)sizeof(T));
#pragma unroll
    for (int k = 0; k < kLoadsPerWave; ++k) {
      // kind and page of block uwave + W * k: known here when W divides the
      // blocks of a page
      constexpr bool kStatic = (NK / 2) % W == 0;
      const int blk = (kStatic ? 0 : uwave) + W * k;
      const bool is_k = blk < NK;
      const int of_kind = is_k ? blk : blk - NK;
      const bool p1 = of_kind >= NK / 2;
      const int in_page = of_kind % (NK / 2) + (kStatic ? uwave : 0);
      uint32_t off = is_k ? k_off : v_off;
      asm volatile("" : "+v"(off));   // (not widened outside the loop: the load adds it itself)
      const uint8_t* base = reinterpret_cast<const uint8_t*>(is_k ? kbase : vbase) + in_page * 1024;
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const uint8_t*>(uniform64(reinterpret_cast<int64_t>(base) + (p1 ? o1 : o0))) + off,
          img + (uwave + W * k) * 1024, 16, 0, 0);
    }
  };
  // ---- 4-bit loads: half q_half of page q_page's tiles
  static_assert(!KVQ || W == 4, "a wave for each half of a page's tiles");
  constexpr int ND = NO / 2;   // dwords of codes per lane, of K and of V
  using Regs = KvqRegs<ND>;
  const int q_page = uwave & 1, q_half = uwave >> 1;
  // K: dwords ND half .. of unit (g, token) = lane. V: unit (bq, h, c) = lane
  // modulo their number, dwords ND sub .. of its four
  constexpr int kUnits = D / 2;
  const int q_unit = lane % kUnits, q_sub = lane / kUnits + 64 / kUnits * q_half;
  const uint32_t q_k_off = lane * (D / 8) + q_half * ND * 4, q_ks_off = D * 8 + (lane & 15) * NO + q_half * ND;
  const uint32_t q_v_off = q_unit * 16 + q_sub * ND * 4, q_vs_off = D * 8 + 16 * ((q_unit >> 4) & 1);
  const int64_t q_k_base = reinterpret_cast<int64_t>(a.k_pool) + (int64_t)it.kv_head * kvq_k_tile<D>();
  const int64_t q_v_base = reinterpret_cast<int64_t>(a.v_pool) + (int64_t)it.kv_head * kvq_v_tile<D>();
  // The registers are loaded again right after their conversion, half a step
  // earlier than at the step's end, where the step is short (d 64: 32 chunks of 512
  // tokens on 4096 888 -> 859 us; d 128: 1209 -> 1215, 16 chunks of 16-128 on 2048
  // 90.8 -> 92.1).
  constexpr bool kFetchEarly = KVQ && D == 64;
  // where the first dword's 8 values go in an image
  const int q_v_blk = 4 * (q_unit / 32) + q_sub * ND;   // its 16-dim block
  const uint32_t q_k_to = (q_page * (NK / 2) + q_half * ND) * 1024 + lane * 16;
  const uint32_t q_v_to = (NK + q_page * NO + (q_v_blk >> 1)) * 1024 + ((q_unit >> 4) & 1) * 512 + (q_v_blk & 1) * 256 +
                          (q_unit & 15) * 16;
  auto q_fetch = [&](const StepPos& p, Regs& r) {
    const int64_t page = (int64_t)(uint32_t)(q_page ? p.pid1 : p.pid0) * a.num_kv_heads;
    const int64_t kb = uniform64(q_k_base + page * kvq_k_tile<D>()), vb = uniform64(q_v_base + page * kvq_v_tile<D>());
    if constexpr (ND == 2) {
      const u32x2_t x = load_global<u32x2_t>(kb + q_k_off), y = load_global<u32x2_t>(vb + q_v_off);
      r.k[0] = x[0];
      r.k[1] = x[1];
      r.v[0] = y[0];
      r.v[1] = y[1];
      r.k_scale = load_global<uint16_t>(kb + q_ks_off);
    } else {
      r.k[0] = load_global<uint32_t>(kb + q_k_off);
      r.v[0] = load_global<uint32_t>(vb + q_v_off);
      r.k_scale = load_global<uint8_t>(kb + q_ks_off);
    }
    r.v_scale = load_global<u32x4_t>(vb + q_vs_off);
  };
  // (full: of the step the registers hold)
  auto q_convert = [&](bool full, const Regs& r, uint8_t* img) {
#pragma unroll
    for (int k = 0; k < ND; ++k)
      *reinterpret_cast<bf16x8_t*>(img + q_k_to + k * 1024) = kvq_decode_bf16(r.k[k], kvq_scale_byte(r.k_scale, k));
    float scale[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = full ? r.v_scale[i] : 0x3f803f80u;
      scale[2 * i] = __uint_as_float(x << 16);
      scale[2 * i + 1] = __uint_as_float(x);   // (of a scale only the exponent counts)
    }
    F f[2];
    kvq_decode_keys(r.v[0], ND == 2 ? r.v[ND - 1] : 0u, scale, f[0], f[1]);
    *reinterpret_cast<F*>(img + q_v_to) = f[0];
    if constexpr (ND == 2) *reinterpret_cast<F*>(img + q_v_to + 256) = f[1];
  };
  // The V scales of a step with masked keys, in token order.
  auto q_scales = [&](const Regs& r, uint8_t* img) {
    if (q_sub == 0 && (q_unit & ~16) == 0) {
      // slots 8 hh + j are keys 8 (j / 4) + 4 hh + j % 4 of the page
      const int hh = q_unit >> 4;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        reinterpret_cast<uint32_t*>(img + kStepBytes)[16 * q_page + 8 * (j >> 2) + 4 * hh + (j & 3)] =
            j & 1 ? r.v_scale[j >> 1] & 0xffff0000u : r.v_scale[j >> 1] << 16;
    }
  };
  // The V scales of this lane's 16 keys of a step that has masked ones.
  auto read_scales = [&](const uint8_t* img, float (&sc)[16]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(img + kStepBytes + (8 * q + 4 * h) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[4 * q + i] = x[i];
    }
  };

  // K fragment s of a step image: this lane's key and units 2s + h.
  const int k_rd = (c >> 4) * (NK / 2) * 1024 + h * 256 + (c & 15) * 16;
  auto k_at = [&](const uint8_t* img, int s) { return img + k_rd + s / 2 * 1024 + s % 2 * 512; };

  float m = kNegInf, lsum = 0.f;
  f32x16_t acc[NO];
#pragma unroll
  for (int b = 0; b < NO; ++b) acc[b] = f32x16_t{};

  // Key (within the step) of score register i of this lane.
  auto skey = [&](int i) { return 8 * (i >> 2) + 4 * h + (i & 3); };

  // Q K^T of one step (one accumulation chain over the 16-dim slices).
  auto qk = [&](const uint8_t* img, f32x16_t& sacc) {
    F kf[NK];
#pragma unroll
    for (int s = 0; s < NK; ++s) kf[s] = __builtin_bit_cast(F, *reinterpret_cast<const u32x4_t*>(k_at(img, s)));
    f32x16_t sn = f32x16_t{};
#pragma unroll
    for (int s = 0; s < NK; ++s) sn = mma32(kf[s], qf[s], sn);
    sacc = sn;
  };

  // P V of one step. Keys past the span end may be NaN page tails: their V
  // slots are zeroed (P = 0 times NaN would still poison the sum).
  auto read_v = [&](const uint8_t* img, F (&vf)[2][NO]) {
    const uint8_t* rd = img + lane * 16;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int b = 0; b < NO; ++b)
        vf[g][b] = __builtin_bit_cast(F, *reinterpret_cast<const u32x4_t*>(rd + (NK + g * NO + b) * 1024));
  };
  auto mask_v = [&](const StepPos& p, F (&vf)[2][NO]) {
    if (p.t0 + kKeysPerStep > p.key_end) {
      const int lim = p.key_end - p.t0;
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int b = 0; b < NO; ++b) {
          u32x4_t w = __builtin_bit_cast(u32x4_t, vf[g][b]);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            // 32-bit word q holds slots 2q, 2q+1 = registers 8g + 2q, 8g + 2q + 1
            const unsigned keep_lo = skey(8 * g + 2 * q) < lim ? 0xFFFFu : 0u;
            const unsigned keep_hi = skey(8 * g + 2 * q + 1) < lim ? 0xFFFF0000u : 0u;
            w[q] &= keep_lo | keep_hi;
          }
          vf[g][b] = __builtin_bit_cast(F, w);
        }
    }
  };
  constexpr bool kExact = KVQ && sizeof(TO) == 4;
  using P = Weights<kExact>;
  auto pv = [&](const F (&vf)[2][NO], const P& w) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      if constexpr (kExact) {
        float half[8];
        F part[3];
#pragma unroll
        for (int j = 0; j < 8; ++j) half[j] = w.p[8 * g + j];
        split(half, part);
#pragma unroll
        for (int n = 2; n >= 0; --n)
#pragma unroll
          for (int b = 0; b < NO; ++b) acc[b] = mma32(vf[g][b], part[n], acc[b]);
      } else {
#pragma unroll
        for (int b = 0; b < NO; ++b) acc[b] = mma32(vf[g][b], w.f[g], acc[b]);
      }
    }
  };
  auto put_weights = [&](const float (&pr)[16], P& w) {
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      if constexpr (kExact) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w.p[8 * g + j] = pr[8 * g + j];
      } else {
        float half[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) half[j] = pr[8 * g + j];
        w.f[g] = to_frag(half, (F*)nullptr);
      }
    }
  };

  // Online softmax of one step's scores into P (bf16, RNE), one operand per
  // page of the step (registers 0-7: page 0, 8-15: page 1).
  auto softmax = [&](const StepPos& p, const f32x16_t& sacc, const uint8_t* img, P& pf) {
    // raw scores (masked ones -inf); the scale is applied inside the exponent
    // with one FMA (scale > 0, so it commutes with the max)
    float sv[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sv[i] = sacc[i];
    if (p.t0 + kKeysPerStep > p.key_end || p.causal) {
      const int lim = (p.causal ? min(p.key_end, row.qpos + 1) : p.key_end) - p.t0;
#pragma unroll
      for (int i = 0; i < 16; ++i) sv[i] = skey(i) < lim ? sv[i] : kNegInf;
    }
    float mt = sv[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mt = fmaxf(mt, sv[i]);
    mt = halves_max(mt) * a.scale_log2;
    const bool move = mt > m + kRescaleLog2;
    if (__any(move)) {
      const float m_new = move ? mt : m;
      const float alpha = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
      lsum *= alpha;
#pragma unroll
      for (int b = 0; b < NO; ++b) acc[b] *= alpha;
      m = m_new;
    }
    const float m_use = m == kNegInf ? 0.f : m;
    float pr[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[i], a.scale_log2, -m_use));
    float ps = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 4) ps += (pr[i] + pr[i + 1]) + (pr[i + 2] + pr[i + 3]);
    lsum += ps;
    if (KVQ && !p.full) {
      float sc[16];
      read_scales(img, sc);
      const int lim = (p.causal ? min(p.key_end, row.qpos + 1) : p.key_end) - p.t0;
#pragma unroll
      for (int i = 0; i < 16; ++i) pr[i] = skey(i) < lim ? pr[i] * sc[i] : 0.f;
    }
    put_weights(pr, pf);
  };

  // One iteration on full, unmasked steps as a single basic block: the 16
  // MFMAs (P V of step t-1, Q K^T of step t+1) are interleaved with the
  // softmax VALU work of step t, so a wave keeps issuing independent VALU
  // instructions while each MFMA runs. V of step t-1 arrives in registers
  // (read during the previous iteration); the K reads of step t+1 go out
  // first and arrive behind the P V products, and the V reads of step t,
  // for the next iteration, go out behind the Q K^T products. The
  // accumulator rescale, which must wait for the P V products, is returned
  // (alpha) and applied afterwards.
  // KVQ: `convert` turns the registers' step into its image.
  auto fast_iter = [&](F (&vf)[2][NO], const uint8_t* img_qk, const uint8_t* img_v, const P& pf_prev,
                       const f32x16_t& sacc_cur, f32x16_t& sacc_nxt, P& pf_cur, float& alpha, auto convert) {
    F kf[NK];
#pragma unroll
    for (int s = 0; s < NK; ++s) kf[s] = __builtin_bit_cast(F, *reinterpret_cast<const u32x4_t*>(k_at(img_qk, s)));
    pv(vf, pf_prev);
    f32x16_t sn = f32x16_t{};
#pragma unroll
    for (int s = 0; s < NK; ++s) sn = mma32(kf[s], qf[s], sn);
    read_v(img_v, vf);
    // softmax of step t (no masks: full step); the max as a tree of
    // three-input maxima (v_max3_f32, 8 instructions for 16 scores)
    auto max3 = [](float x, float y, float z) { return fmaxf(fmaxf(x, y), z); };
    const float m0 = max3(sacc_cur[0], sacc_cur[1], sacc_cur[2]);
    const float m1 = max3(sacc_cur[3], sacc_cur[4], sacc_cur[5]);
    const float m2 = max3(sacc_cur[6], sacc_cur[7], sacc_cur[8]);
    const float m3 = max3(sacc_cur[9], sacc_cur[10], sacc_cur[11]);
    const float m4 = max3(sacc_cur[12], sacc_cur[13], sacc_cur[14]);
    float mt = fmaxf(max3(m0, m1, m2), max3(m3, m4, sacc_cur[15]));
    mt = halves_max(mt) * a.scale_log2;
    const bool move = mt > m + kRescaleLog2;
    const float m_new = move ? mt : m;
    alpha = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    const float m_use = m == kNegInf ? 0.f : m;
    float pr[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) pr[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc_cur[i], a.scale_log2, -m_use));
    put_weights(pr, pf_cur);
    float ps = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 4) ps += (pr[i] + pr[i + 1]) + (pr[i + 2] + pr[i + 3]);
    lsum = __builtin_fmaf(lsum, alpha, ps);
    sacc_nxt = sn;
    convert();
    // keep the softmax results in this block (they are consumed only after
    // the next barrier, and would otherwise sink below the rescale branch)
    if constexpr (kExact) {
#pragma unroll
      for (int i = 0; i < 16; ++i) asm volatile("" ::"v"(pf_cur.p[i]));
    } else {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const u32x4_t w = __builtin_bit_cast(u32x4_t, pf_cur.f[g]);
        asm volatile("" ::"v"(w[0]), "v"(w[1]), "v"(w[2]), "v"(w[3]));
      }
    }
    asm volatile("" ::"v"(lsum));
    // schedule: the K reads, the P V MFMAs, then the Q K^T MFMAs with the V
    // reads of step t after the first of them; each MFMA followed by VALU
    // work
    // (KVQ: half of the K reads after three of the P V products, which leaves
    // registers for the conversion, and more VALU work to the Q K^T products: 4 and 6
    // instructions, chunked prefill 1184 us, 4 and 4 1191, 5 and 6 1191, 6 and 6 1228;
    // d 64: 3 and 6 843, 4 and 4 850)
    constexpr int kBetween = KVQ ? (D == 128 ? 4 : 3) : 5, kBehind = KVQ ? 6 : 5, kAhead = KVQ ? NK / 2 : NK;
    __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
    for (int k = 0; k < 2 * NO + 1; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, kBetween, 0);
      if (KVQ && k >= 3 && k - 3 < (NK - kAhead) / 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * NO, 0);
#pragma unroll
    for (int k = 0; k < NK - 1; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, kBehind, 0);
    }
  };

  // ---- pipeline. Step t lives in stage t % S. Iteration t:
  //   wait for this wave's loads of step t+1 (steps t+2..t+S-2 may still be
  //   in flight) and retire its LDS reads (lgkmcnt 0); barrier: step t+1 is
  //   visible to every wave, and step t-1's stage is free (its K was read in
  //   iteration t-2, its V in iteration t-1); issue step t+S-1 into it;
  //   MFMA: P V of step t-1 (V already in registers), Q K^T of step t+1;
  //   VALU: softmax of step t; LDS: K of step t+1, V of step t.
  // Score and probability tiles alternate by step parity (S is even, so the
  // parity of each unrolled position is fixed). Positions past the end
  // re-load the current step's pages (in bounds, never read) so the count of
  // loads in flight stays fixed.
  StepPos ps[S];
  ps[0] = advance();
  if (ps[0].valid) {
    Regs qr;
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
      if (i > 0) ps[i] = advance();
      if constexpr (KVQ) {
        q_fetch(pick(ps[i].valid, ps[i], ps[0]), qr);
        if (i < 2) {
          q_convert(ps[i].full, qr, lds[i]);
          if (!ps[i].full) q_scales(qr, lds[i]);
        }
      } else {
        issue(pick(ps[i].valid, ps[i], ps[0]), lds[i]);
      }
    }
    f32x16_t sacc[2];
    P pf[2];
    F vf[2][NO];
    if constexpr (KVQ) {
      asm volatile("" ::: "memory");
      wait_lgkmcnt0();
    } else {
      wait_vmcnt<(S - 3) * kLoadsPerWave>();
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (computes) qk(lds[0], sacc[0]);
    bool first = true, done = false;
    while (!done) {
#pragma unroll
      for (int st = 0; st < S; ++st) {
        const int cur_p = st & 1, nxt_p = cur_p ^ 1;
        const int nx = (st + 1) % S, pv_st = (st + S - 1) % S;
        if constexpr (KVQ) asm volatile("" ::: "memory");
        else wait_vmcnt<(S - 3) * kLoadsPerWave>();
        wait_lgkmcnt0();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const StepPos prev = ps[pv_st];   // step t-1, whose V is in vf
        ps[pv_st] = advance();
        if constexpr (!KVQ) issue(pick(ps[pv_st].valid, ps[pv_st], ps[st]), lds[pv_st]);
        const bool more = ps[nx].valid;
        // KVQ: step t+2 into its image (that of step t-2), then step t+S-1 into
        // the registers. (A fast step is one in which that step is full too, so that
        // its conversion chooses no scales: with the scales' mantissas left as they
        // are, 8 instructions fewer, chunked prefill 1207 -> 1193 us.)
        const bool full2 = ps[(st + 2) % S].full;
        const bool fast = !first && more && ps[st].full && prev.full && (!KVQ || full2);
        auto fetch = [&]() { q_fetch(pick(ps[pv_st].valid, ps[pv_st], ps[st]), qr); };
        auto convert = [&]() {
          if constexpr (KVQ) q_convert(full2, qr, lds[(st + 2) % kImages]);
        };
        auto convert_fast = [&]() {
          if constexpr (KVQ) {
            if constexpr (!kFetchEarly) {
              // (of its own: what it shares with the one below would be computed
              // before the branch, and the loads waited for there; 70B-shaped decode
              // 501 -> 494 us)
#pragma unroll
              for (int k = 0; k < ND; ++k) asm volatile("" : "+v"(qr.k[k]), "+v"(qr.v[k]));
              asm volatile("" : "+v"(qr.k_scale), "+v"(qr.v_scale));
            }
            q_convert(true, qr, lds[(st + 2) % kImages]);
          }
          if constexpr (kFetchEarly) fetch();
        };
        if (computes && fast) {
          float alpha;
          fast_iter(vf, lds[nx % kImages], lds[st % kImages], pf[nxt_p], sacc[cur_p], sacc[nxt_p], pf[cur_p], alpha,
                    convert_fast);
          if (__any(alpha != 1.f)) {
#pragma unroll
            for (int b = 0; b < NO; ++b) acc[b] *= alpha;
          }
        } else {
          convert();
          if (computes) {
            if (!first) {
              if constexpr (!KVQ) mask_v(prev, vf);   // (4-bit codes are finite, and the weights 0)
              pv(vf, pf[nxt_p]);
            }
            if (more) qk(lds[nx % kImages], sacc[nxt_p]);
            softmax(ps[st], sacc[cur_p], lds[st % kImages], pf[cur_p]);
            read_v(lds[st % kImages], vf);
            if (!more) {
              if constexpr (!KVQ) mask_v(ps[st], vf);
              pv(vf, pf[cur_p]);
            }
          }
        }
        if constexpr (KVQ) {
          if (!full2) q_scales(qr, lds[(st + 2) % kImages]);
          if (!(kFetchEarly && computes && fast)) fetch();
        }
        first = false;
        if (!more) {
          done = true;
          break;
        }
      }
    }
  }
  // drain the loads still in flight before the workgroup's LDS is released
  wait_vmcnt<0>();

  // ---- epilogue: lane (c, h) holds dims 32b + 8(i/4) + 4h + i%4 of row c
  const float l = halves_sum(lsum);
  constexpr bool kHalf = KVQ && sizeof(TO) == 2;   // partial results by store_half
  float top = 0.f;
  if constexpr (kHalf) top = halves_max(largest_finite(acc));
  if (computes && r < it.n_rows) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const float lse2 = l > 0.f ? m + __log2f(l) : kNegInf;
    if (W == kSmallWideWaves && (it.flags & kItemPiece)) {
      const int64_t prow = (int64_t)it.part_base + r;
      float* dst = static_cast<float*>(a.part_o) + prow * D + 4 * h;
#pragma unroll
      for (int b = 0; b < NO; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          store4(dst + 32 * b + 8 * q, f32x4_t{acc[b][4 * q], acc[b][4 * q + 1], acc[b][4 * q + 2], acc[b][4 * q + 3]} * inv);
      if (h == 0) reinterpret_cast<int*>(a.part_lse)[prow] = part_lse_bits(lse2, l);
    } else if (kHalf && it.part_base >= 0) {
      const int64_t prow = row.slot;
      const float scale = row_scale(top * inv), x = inv * reciprocal_of_scale(scale);
      uint16_t* dst = static_cast<uint16_t*>(a.part_o) + prow * D + 4 * h;
#pragma unroll
      for (int b = 0; b < NO; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          store_half(dst + 32 * b + 8 * q, f32x4_t{acc[b][4 * q], acc[b][4 * q + 1], acc[b][4 * q + 2], acc[b][4 * q + 3]} * x);
      if (h == 0)
        reinterpret_cast<int2*>(a.part_lse)[prow] = make_int2(part_lse_bits(lse2, l), __float_as_int(scale));
    } else if (it.part_base >= 0) {
      const int64_t prow = row.slot;
      TO* dst = static_cast<TO*>(a.part_o) + prow * D + 4 * h;
#pragma unroll
      for (int b = 0; b < NO; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          store4_part(dst + 32 * b + 8 * q, f32x4_t{acc[b][4 * q], acc[b][4 * q + 1], acc[b][4 * q + 2], acc[b][4 * q + 3]} * inv);
      if (h == 0) reinterpret_cast<int*>(a.part_lse)[prow] = part_lse_bits(lse2, l);
    } else {
      TO* dst = static_cast<TO*>(a.o) + (int64_t)row.q_row * D + 4 * h;
#pragma unroll
      for (int b = 0; b < NO; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          store4(dst + 32 * b + 8 * q, f32x4_t{acc[b][4 * q], acc[b][4 * q + 1], acc[b][4 * q + 2], acc[b][4 * q + 3]} * inv);
      if (h == 0 && a.lse) a.lse[row.q_row] = lse2 == kNegInf ? kNegInf : lse2 * kLn2;
    }
  }
}

// ---------------------------------------------------------------- host side

int pad_to(int n, int m) { return (n + m - 1) / m * m; }

// Share (percent) of the narrow rounds interleaved with the wide ones; the
// rest run after the last wide round.
constexpr int kWideSpanNarrowPct = 80;

int lcm_int(int a, int b) {
  int x = a, y = b;
  while (y) {
    const int t = x % y;
    x = y;
    y = t;
  }
  return a / x * b;
}

// The wide role's blocks: whole dispatch cycles of wide rounds, each a multiple
// of wide_group rounds.
void lay_out_rounds(AttnArgs& args, bool wide, int narrow_pct = kWideSpanNarrowPct) {
  args.wide_blocks =
      (wide && args.n_wide > 0) ? pad_to(args.n_wide, 8 * lcm_int(args.wide_group, kSeCycle)) : 0;
  {
    const int ws = args.wide_blocks / (8 * kSeCycle), ns = args.narrow_blocks / (8 * kSeCycle);
    args.wide_span = ws + (int)((int64_t)ns * narrow_pct / 100);
  }
}

}  // namespace
