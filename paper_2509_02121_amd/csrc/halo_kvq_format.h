// The 4-bit page format in device code: E2M1 codes to and from floats, and the
// scales.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace halo {

// Bytes of a (page, head) tile: 16 * D codes, then a scale byte for each 32 dims
// of a token (K) or a bf16 scale for each token (V).
template <int D> constexpr int kvq_k_tile() { return D * 8 + D / 2; }
template <int D> constexpr int kvq_v_tile() { return D * 8 + 32; }

}  // namespace halo

namespace {

typedef __bf16 kvq_bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 kvq_bf16x2_t __attribute__((ext_vector_type(2)));
typedef float kvq_f32x2_t __attribute__((ext_vector_type(2)));

// 8 codes (the lowest four bits first) times a power of two (of which the
// conversion uses the exponent; 255 there gives NaN). Exact: an E2M1 value has
// two significant bits.
__device__ __forceinline__ kvq_bf16x8_t kvq_decode_bf16(uint32_t w, float scale) {
  const kvq_bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const kvq_bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const kvq_bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const kvq_bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return kvq_bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void kvq_decode_f32(uint32_t w, float scale, float (&v)[8]) {
  const kvq_f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
  const kvq_f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const kvq_f32x2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
  const kvq_f32x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
  v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
}
// 8 codes each of two dims of the same 8 keys, times the keys' scales: a byte of
// two codes of one key is put together first, so that one conversion does both
// dims with the key's scale.
__device__ __forceinline__ void kvq_decode_keys(uint32_t w0, uint32_t w1, const float (&scale)[8], kvq_bf16x8_t& f0,
                                                kvq_bf16x8_t& f1) {
  constexpr uint32_t kLow = 0x0f0f0f0fu;
  const uint32_t a = (w0 & kLow) | ((w1 << 4) & ~kLow);   // keys 0, 2, 4, 6
  const uint32_t b = ((w0 >> 4) & kLow) | (w1 & ~kLow);   // keys 1, 3, 5, 7
  const uint32_t c[8] = {
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale[0], 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b, scale[1], 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale[2], 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b, scale[3], 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale[4], 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b, scale[5], 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(a, scale[6], 3)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b, scale[7], 3))};
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  u32x4 lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
    hi[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
  }
  f0 = __builtin_bit_cast(kvq_bf16x8_t, lo);
  f1 = __builtin_bit_cast(kvq_bf16x8_t, hi);
}
// The nearest codes of 8 values over a power of two, ties to the even code,
// magnitudes past 6 to 6.
__device__ __forceinline__ uint32_t kvq_encode(const float (&v)[8], float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
  return w;
}
// The biased exponent of a block's scale from the bits of its largest magnitude:
// that of the magnitude rounded to two significant bits, less two, so that it
// becomes 3.5 to 7 and the largest code (6) is at most one unit off; 255 for a
// block that holds an infinity or a NaN (whose bits are the largest).
__device__ __forceinline__ int kvq_exponent(uint32_t bits) {
  const int e = (int)((bits + 0x200000u) >> 23) - 2;
  return bits >= 0x7f800000u ? 255 : min(max(e, 1), 254);
}
__device__ __forceinline__ float kvq_scale(int e) { return __uint_as_float((uint32_t)e << 23); }

// The scale of byte i of four, in one instruction (a shift and a mask otherwise).
__device__ __forceinline__ float kvq_scale_byte(uint32_t bytes, int i) {
  uint32_t r;
  const uint32_t n = 23;
  if (i == 0) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(n), "v"(bytes));
  else if (i == 1) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(n), "v"(bytes));
  else if (i == 2) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(n), "v"(bytes));
  else r = (bytes >> 24) << 23;
  return __uint_as_float(r);
}

}  // namespace
