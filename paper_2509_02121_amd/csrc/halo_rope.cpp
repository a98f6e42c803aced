// Rotary frequencies (host): the angle of each pair per position, for the plain
// rotation and for its extensions to positions beyond the trained ones.

#include <algorithm>
#include <cmath>
#include <string>

#include "halo_internal.h"

using namespace halo;

namespace {

halo_status_t check_rope(const halo_rope_params_t* p) {
  if (!p) return fail(HALO_ERR_INVALID_ARGUMENT, "rope must not be NULL");
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(HALO_ERR_UNSUPPORTED, "head_dim must be 64 or 128, got " + std::to_string(p->head_dim));
  if (p->rotary_dim < 16 || p->rotary_dim > p->head_dim || p->rotary_dim % 16 != 0)
    return fail(HALO_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 16 in [16, head_dim], got " +
                                          std::to_string(p->rotary_dim));
  if (!std::isfinite(p->base) || !(p->base > 1.0))
    return fail(HALO_ERR_INVALID_ARGUMENT, "base must be finite and > 1");
  if (p->scaling < HALO_ROPE_NONE || p->scaling > HALO_ROPE_BANDS)
    return fail(HALO_ERR_UNSUPPORTED, "unknown rope scaling");
  if (p->scaling != HALO_ROPE_NONE && (!std::isfinite(p->factor) || !(p->factor >= 1.0)))
    return fail(HALO_ERR_INVALID_ARGUMENT, "factor must be finite and >= 1");
  if (p->scaling == HALO_ROPE_YARN || p->scaling == HALO_ROPE_BANDS) {
    if (p->original_positions < 1) return fail(HALO_ERR_INVALID_ARGUMENT, "original_positions must be >= 1");
    if (!std::isfinite(p->fast_turns) || !std::isfinite(p->slow_turns) || !(p->slow_turns > 0) ||
        !(p->fast_turns > p->slow_turns))
      return fail(HALO_ERR_INVALID_ARGUMENT, "fast_turns must be finite and > slow_turns > 0");
  }
  return HALO_OK;
}

}  // namespace

extern "C" void halo_rope_params_default(halo_rope_params_t* rope, int32_t head_dim) {
  if (!rope) return;
  *rope = halo_rope_params_t{head_dim, head_dim, 0, HALO_ROPE_NONE, 10000.0, 1.0, 8192, 0.0, 0.0};
}

extern "C" halo_status_t halo_rope_turns(const halo_rope_params_t* rope, uint64_t* turns, float* amplitude) {
  clear_error();
  if (rope && (rope->fast_turns == 0 && rope->slow_turns == 0)) {
    // the defaults of the scaling
    halo_rope_params_t p = *rope;
    p.fast_turns = p.scaling == HALO_ROPE_BANDS ? 4.0 : 32.0;
    p.slow_turns = 1.0;
    return halo_rope_turns(&p, turns, amplitude);
  }
  halo_status_t st = check_rope(rope);
  if (st != HALO_OK) return st;
  if (!turns || !amplitude) return fail(HALO_ERR_INVALID_ARGUMENT, "turns and amplitude must not be NULL");
  const int R = rope->rotary_dim;
  const double f = rope->factor, two_pi = 6.283185307179586476925;
  long double base = rope->base;
  if (rope->scaling == HALO_ROPE_NTK) base *= powl(f, (long double)R / (R - 2));
  *amplitude = 1.f;
  double lo = 0, span = 1;
  if (rope->scaling == HALO_ROPE_YARN) {
    auto index = [&](double n) {   // of the pair that makes n turns over the original positions
      return R * std::log(rope->original_positions / (n * two_pi)) / (2 * std::log(rope->base));
    };
    lo = std::max(std::floor(index(rope->fast_turns)), 0.0);
    const double hi = std::min(std::ceil(index(rope->slow_turns)), R - 1.0);
    span = hi > lo ? hi - lo : 0.001;
    if (f > 1) *amplitude = (float)(0.1 * std::log(f) + 1.0);
  }
  const long double two64 = 18446744073709551616.0L, pi2 = 6.283185307179586476925286766559L;
  for (int i = 0; i < R / 2; ++i) {
    long double w = powl(base, -2.0L * i / R);
    if (rope->scaling == HALO_ROPE_LINEAR) w /= f;
    if (rope->scaling == HALO_ROPE_YARN) {
      const double slowed = std::min(1.0, std::max(0.0, (i - lo) / span));
      w = w * (1 - slowed) + w / f * slowed;
    }
    if (rope->scaling == HALO_ROPE_BANDS) {
      const long double n = rope->original_positions * w / pi2;   // turns over the original positions
      const long double kept =
          std::min(1.0L, std::max(0.0L, (n - rope->slow_turns) / (rope->fast_turns - rope->slow_turns)));
      w = w * kept + w / f * (1 - kept);
    }
    turns[i] = (uint64_t)(w / pi2 * two64 + 0.5L);   // w <= 1: less than 2^62
  }
  return HALO_OK;
}
