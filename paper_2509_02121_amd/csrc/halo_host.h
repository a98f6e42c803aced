// Checks that the entry points of the operators between two steps share (host
// code of the .hip files).
#pragma once

#include <hip/hip_runtime.h>

#include <cstring>
#include <initializer_list>
#include <string>

#include "halo_internal.h"

namespace {

// Memory that a call reads or writes.
struct Range {
  const char* name;
  const void* p;
  int64_t bytes;
};
inline bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + b.bytes && y < x + a.bytes;
}
// No array that is written may overlap another one.
inline halo_status_t check_overlaps(std::initializer_list<Range> reads, std::initializer_list<Range> writes) {
  for (const Range& w : writes) {
    for (const Range& r : reads)
      if (overlap(w, r))
        return halo::fail(HALO_ERR_INVALID_ARGUMENT, std::string(r.name) + " must not overlap " + w.name);
    for (const Range& v : writes)
      if (&v < &w && overlap(w, v))
        return halo::fail(HALO_ERR_INVALID_ARGUMENT, std::string(v.name) + " must not overlap " + w.name);
  }
  return HALO_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool finite(float x) {   // (by its bits: the build drops float tests for NaN)
  uint32_t bits;
  memcpy(&bits, &x, 4);
  return (bits & 0x7f800000u) != 0x7f800000u;
}

inline halo_status_t hip_check(const char* what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return halo::fail(HALO_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return HALO_OK;
}

// What a call over pools needs of its params, whatever their format.
inline halo_status_t check_cache_params(const halo_attn_params_t* p) {
  if (p->head_dim != 64 && p->head_dim != 128)
    return halo::fail(HALO_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (p->page_size != 16) return halo::fail(HALO_ERR_UNSUPPORTED, "page_size must be 16");
  if (p->num_kv_heads < 1) return halo::fail(HALO_ERR_INVALID_ARGUMENT, "num_kv_heads must be >= 1");
  if (p->num_pool_pages < 0) return halo::fail(HALO_ERR_INVALID_ARGUMENT, "num_pool_pages must be >= 0");
  if (p->num_kv_heads > 65536 || p->num_pool_pages > INT32_MAX)
    return halo::fail(HALO_ERR_UNSUPPORTED, "at most 65536 heads and 2^31 - 1 pages");
  if (p->kv_dtype != HALO_BF16 && p->kv_dtype != HALO_F32)
    return halo::fail(HALO_ERR_UNSUPPORTED, "kv_dtype must be HALO_F32 or HALO_BF16");
  return HALO_OK;
}

// Calls launch(type, head_dim) for params' kv_dtype and head_dim.
template <typename Launch>
void by_type_and_dim(const halo_attn_params_t* p, Launch launch) {
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
