// gfx950 kernels for attention over 4-bit pools: the items of the same plans as
// over bf16 and fp32 pools (see halo_kernels.hip for the work decomposition, the
// layouts of the products and the merge, which are shared).
//
//   S = scale q K^T, P = softmax(S), O = P V with K = k_scale * k_code,
//   V = v_scale * v_code, codes E2M1 and scales powers of two.
//
// A K code times its scale is exact in bf16 and takes one conversion per two
// values. A V scale belongs to a key, i.e. runs along the contraction of P V, so
// it is multiplied onto P (exactly) after the sum of P is taken, and V codes are
// converted with scale 1.
//
// Narrow items convert in registers, between the loads and the MFMAs; wide items
// once per workgroup, on the way into LDS (wide_item). Per step of 32 keys and
// wave a narrow item reads 4.3 KB at d = 128 where bf16 pages take 16 KB, and adds
// 64 conversions (about 5 cycles each, measured) and 40 instructions for the scales
// to the softmax and the 16 MFMAs.
//
// fp32 queries: K and V are exact in bf16, so a product with fp32 accuracy needs
// only q and P split into three bf16 parts each (8 + 8 + 8 bits): three MFMAs of
// 16x16x32 in place of eight 16x16x4 fp32 ones.

#include <hip/hip_runtime.h>

#include <algorithm>

#include "halo_device.h"
#include "halo_internal.h"
#include "halo_kvq_format.h"

using namespace halo;

namespace {

// bf16 parts of an operand: 1 for bf16 (rounded, as over bf16 pools), 3 for fp32.
template <typename T> constexpr int parts() { return sizeof(T) == 2 ? 1 : 3; }

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

// Loads marked non-temporal for keys that one item reads only (see ld16).
template <bool NT, typename V>
__device__ __forceinline__ V ld(const void* p) {
  if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}

// One step's codes and scales of a lane: K dwords of 8 dims for the two 16-key
// tiles, their scale bytes, V dwords of 8 keys, and those keys' scales in bf16.
template <int D>
struct KvqStep {
  uint32_t k[2][D / 32];
  uint32_t ks[2];
  uint32_t v[D / 16];
  u32x4_t vs;
};

// One work item on one wavefront: run_item over 4-bit pages. Lane (col, grp) has
// the same keys and dims there and here: for tile X its K row is key 8X + col % 8
// of page col / 8, of which it holds unit (grp, key), dims 32 s + 8 grp .. + 7 for
// every s, in one load; for P V dims 16 b + col of the keys in half grp % 2 of
// page grp / 2, one dword for each b.
template <typename T, int D, typename TO, bool NT, int P>
__device__ __forceinline__ void run_item_kvq(const AttnArgs& a, const Item& it, const RecLane& rl, int lane) {
  using F = bf16x8_t;
  constexpr int NS = D / 32, NB = D / 16, NP = parts<T>();
  constexpr int kTile = kvq_k_tile<D>(), vTile = kvq_v_tile<D>();
  using Regs = KvqStep<D>;
  const int col = lane & 15;
  const int grp = lane >> 4;
  const Row row{rl.q_row, rl.aux, -1, rl.aux};

  F qf[NP][NS];
  {
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(row.q_row < 0 ? 0 : row.q_row) * D + 8 * grp;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      if constexpr (sizeof(T) == 2) {
        qf[0][s] = row.q_row >= 0 ? load8(qp + 32 * s) : zero_frag<F>();
      } else {
        const f32x8_t x = row.q_row >= 0 ? load8(qp + 32 * s) : f32x8_t{};
        float v[8];
        F f[NP];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[j];
        split(v, f);
#pragma unroll
        for (int n = 0; n < NP; ++n) qf[n][s] = f[n];
      }
    }
  }

  const uint8_t* kbase = static_cast<const uint8_t*>(a.k_pool) + (int64_t)it.kv_head * kTile;
  const uint8_t* vbase = static_cast<const uint8_t*>(a.v_pool) + (int64_t)it.kv_head * vTile;
  const int64_t k_stride = (int64_t)a.num_kv_heads * kTile, v_stride = (int64_t)a.num_kv_heads * vTile;

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
  auto step_at = [&](const SpanState& st, int t0) {
    StepPos p;
    p.valid = st.valid;
    p.t0 = t0;
    p.key_end = st.ke;
    p.causal = st.causal;
    const int j = (t0 - st.kb) >> 4;
    p.has1 = t0 + 16 < st.ke;
    p.full = t0 + kKeysPerStep <= st.ke && !st.causal;
    p.pid0 = __builtin_amdgcn_readlane(st.vpid, j);
    p.pid1 = p.has1 ? __builtin_amdgcn_readlane(st.vpid, j + 1) : p.pid0;
    return p;
  };
  // A step's addresses are, per lane, a scalar base chosen by page and an offset
  // that never changes. A position past the item's end loads, in every lane, words
  // at the start of the item table instead (all within its first 2 KB; a table has
  // at least 8 workgroups of 4 items), so that the count of loads in flight stays
  // fixed without reading pages again.
  auto uniform64 = [](int64_t x) {   // on the scalar unit
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
  };
  const uint32_t k_lane = (grp * 16 + (col & 7)) * (D / 8);
  const uint32_t ks_lane = D * 8 + (col & 7) * NS;
  const uint32_t v_lane = ((grp & 1) * 16 + col) * 16;
  const uint32_t vs_lane = D * 8 + (grp & 1) * 16;
  auto fetch = [&](const StepPos& p, Regs& r) {
    const bool live = p.valid;
    const int64_t idle = reinterpret_cast<int64_t>(a.items);
    const int64_t k0 = uniform64(live ? reinterpret_cast<int64_t>(kbase) + (int64_t)(uint32_t)p.pid0 * k_stride : idle);
    const int64_t k1 = uniform64(live ? reinterpret_cast<int64_t>(kbase) + (int64_t)(uint32_t)p.pid1 * k_stride : idle);
    const int64_t v0 = uniform64(live ? reinterpret_cast<int64_t>(vbase) + (int64_t)(uint32_t)p.pid0 * v_stride : idle);
    const int64_t v1 = uniform64(live ? reinterpret_cast<int64_t>(vbase) + (int64_t)(uint32_t)p.pid1 * v_stride : idle);
    const uint8_t* kq = reinterpret_cast<const uint8_t*>((col < 8 ? k0 : k1) + (live ? k_lane : 0u));
    const uint8_t* kz = reinterpret_cast<const uint8_t*>((col < 8 ? k0 : k1) + (live ? ks_lane : 0u));
    const uint8_t* vq = reinterpret_cast<const uint8_t*>((grp < 2 ? v0 : v1) + (live ? v_lane : 0u));
    const uint8_t* vz = reinterpret_cast<const uint8_t*>((grp < 2 ? v0 : v1) + (live ? vs_lane : 0u));
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if constexpr (D == 128) {
        const u32x4_t w = ld<NT, u32x4_t>(kq + x * D);
#pragma unroll
        for (int s = 0; s < NS; ++s) r.k[x][s] = w[s];
        r.ks[x] = ld<NT, uint32_t>(kz + x * 8 * NS);
      } else {
        const u32x2_t w = ld<NT, u32x2_t>(kq + x * D);
#pragma unroll
        for (int s = 0; s < NS; ++s) r.k[x][s] = w[s];
        r.ks[x] = ld<NT, uint16_t>(kz + x * 8 * NS);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; b += 4) {
      const u32x4_t w = ld<NT, u32x4_t>(vq + b * 128);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[b + i] = w[i];
    }
    r.vs = ld<NT, u32x4_t>(vz);
  };

  // The span cursor of run_item: a later span's page ids are loaded, and waited
  // for, when the walk reaches it.
  int si = 0;
  SpanState cur;
  cur.valid = it.n_spans > 0;
  cur.kb = it.s0_key_begin;
  cur.ke = it.s0_key_end;
  cur.causal = it.s0_causal;
  cur.vpid = rl.page;
  int gs = 0, sb = 0;
  auto advance = [&]() {
    while (cur.valid && gs >= sb + ((cur.ke - cur.kb + kKeysPerStep - 1) >> 5)) {
      sb += (cur.ke - cur.kb + kKeysPerStep - 1) >> 5;
      ++si;
      cur = load_span(si);
      wait_vmcnt<0>();
    }
    StepPos p = step_at(cur, cur.kb + (gs - sb) * kKeysPerStep);
    ++gs;
    return p;
  };

  float m = kNegInf;
  float lsum = 0.f;
  f32x4_t acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto compute = [&](const StepPos& p, Regs& r) {
    f32x4_t sacc[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      sacc[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const F kf = kvq_decode_bf16(r.k[x][s], kvq_scale((r.ks[x] >> (8 * s)) & 0xff));
#pragma unroll
        for (int n = NP - 1; n >= 0; --n) sacc[x] = mma(kf, qf[n][s], sacc[x]);
      }
    }
    // slot j = 4X + i holds key t0 + slot_key(grp, j)
    const bool full = p.t0 + kKeysPerStep <= p.key_end && !p.causal;
    float sv[8], vs[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sv[j] = sacc[j >> 2][j & 3] * a.scale_log2;
      vs[j] = __uint_as_float(j & 1 ? r.vs[j >> 1] & 0xffff0000u : r.vs[j >> 1] << 16);
    }
    if (!full) {
      // (a key that is not seen may have any scales: NaN scores, and a weight of
      // 0 times a NaN)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = p.t0 + slot_key(grp, j);
        const bool vis = key < p.key_end && (!p.causal || key <= row.qpos);
        sv[j] = vis ? sv[j] : kNegInf;
        vs[j] = vis ? vs[j] : 0.f;
      }
    }
    float mt = sv[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) mt = fmaxf(mt, sv[j]);
    mt = rows_max(mt);
    // the sums are rescaled only when some row's maximum moves
    if (__any(mt > m)) {
      const float m_new = fmaxf(m, mt);
      const float x = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
      lsum *= x;
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b] *= x;
      m = m_new;
    }
    const float m_use = m == kNegInf ? 0.f : m;
    float pr[8];
    float psum = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      pr[j] = __builtin_amdgcn_exp2f(sv[j] - m_use);
      psum += pr[j];
      pr[j] *= vs[j];
    }
    lsum += psum;
    F pf[NP];
    split(pr, pf);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const F vf = kvq_decode_bf16(r.v[b], 1.f);
#pragma unroll
      for (int n = NP - 1; n >= 0; --n) acc[b] = mma(vf, pf[n], acc[b]);
    }
  };

  // P register stages rotate: while step s is computed, the next P - 1 steps are
  // in flight.
  Regs r[P];
  StepPos ps[P];
  ps[0] = advance();
  if (ps[0].valid) {
    fetch(ps[0], r[0]);
#pragma unroll
    for (int i = 1; i < P - 1; ++i) {
      ps[i] = advance();
      fetch(ps[i], r[i]);
    }
    bool done = false;
    while (!done) {
#pragma unroll
      for (int s = 0; s < P; ++s) {
        const int w = (s + P - 1) % P;
        ps[w] = advance();
        fetch(ps[w], r[w]);
        compute(ps[s], r[s]);
        if (!ps[(s + 1) % P].valid) {
          done = true;
          break;
        }
      }
    }
  }
  finish_item<T, D, TO>(a, it, row, col, grp, acc, m, lsum);
}

constexpr int kKvqNarrowStages = 3;

template <typename T, int D, typename TO>
__device__ __forceinline__ void narrow_block_kvq(const AttnArgs& a, int block) {
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int lane = threadIdx.x & 63;
  const int64_t item_id = (int64_t)block * block_waves<T>() + wave;
  const Item it = a.items[item_id];
  const ItemRec* rec = a.item_recs + item_id;
  const int col = lane & 15;
  const RecLane rl{rec->q_row[col], rec->aux[col], rec->page[lane & 31]};
  if (it.flags & kItemStream) run_item_kvq<T, D, TO, true, kKvqNarrowStages>(a, it, rl, lane);
  else run_item_kvq<T, D, TO, false, kKvqNarrowStages>(a, it, rl, lane);
}

// Both roles in one launch, dealt as in attn_kernel.
constexpr int kKvqStepStages = kKvqStages;

template <typename T, int D, typename TO, int RB>
__global__ __launch_bounds__(64 * block_waves<T>())
__attribute__((amdgpu_waves_per_eu(block_waves<T>() / 4)))
void attn_kvq_kernel(AttnArgs a) {
  static_assert(RB == 0 || block_waves<T>() == kWideWaves, "wide items need kWideWaves-wave blocks");
  constexpr int kSmem = RB > 0 ? kKvqStages * kvq_image_bytes<D>() : 16;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kSmem];
  const int b = blockIdx.x;
  const int x = b & 7, r = b >> 3;
  if constexpr (RB > 0) {
    const int ws = a.wide_blocks / (8 * kSeCycle);
    const int sp = a.wide_span;
    const int cyc = r / kSeCycle, q = r % kSeCycle;
    const int w_before = cyc < sp ? (int)((int64_t)cyc * ws / sp) : ws;
    const int w_upto = cyc < sp ? (int)((int64_t)(cyc + 1) * ws / sp) : ws;
    if (w_upto > w_before) {
      const int item = xcd_remap((w_before * kSeCycle + q) * 8 + x, a.wide_group);
      if (item < a.n_wide) wide_item<D, TO, kWideWaves, kKvqStepStages, true>(a, item, smem);
      return;
    }
    narrow_block_kvq<T, D, TO>(a, ((cyc - w_upto) * kSeCycle + q) * 8 + x);
  } else {
    (void)smem;
    narrow_block_kvq<T, D, TO>(a, b);
  }
}

// Wide items of at most kSmallWideRows rows and nothing else (prefill).
template <int D, typename TO>
__global__ __launch_bounds__(64 * kSmallWideWaves) __attribute__((amdgpu_waves_per_eu(2)))
void wide_kvq_kernel(AttnArgs a) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kKvqStages * kvq_image_bytes<D>()];
  const int item = xcd_remap(blockIdx.x, a.wide_group);
  if (item < a.n_wide) wide_item<D, TO, kSmallWideWaves, kKvqStepStages, true>(a, item, smem);
}

template <typename T, int D, typename TO>
void launch_items(AttnArgs args, const halo_plan& plan, hipStream_t stream) {
  const int rb = sizeof(T) == 2 ? plan.wide_rb : 0;
  lay_out_rounds(args, rb > 0);
  const int grid = args.wide_blocks + args.narrow_blocks;
  if (grid == 0) return;
  constexpr int W = block_waves<T>();
  if constexpr (sizeof(T) == 2) {
    if (rb > 0 && plan.small_wide) {
      hipLaunchKernelGGL((wide_kvq_kernel<D, TO>), dim3(pad_to(args.n_wide, 8 * args.wide_group)),
                         dim3(64 * kSmallWideWaves), 0, stream, args);
      return;
    }
    if (rb > 0) {
      hipLaunchKernelGGL((attn_kvq_kernel<T, D, TO, 1>), dim3(grid), dim3(64 * W), 0, stream, args);
      return;
    }
  }
  hipLaunchKernelGGL((attn_kvq_kernel<T, D, TO, 0>), dim3(grid), dim3(64 * W), 0, stream, args);
}

}  // namespace

void halo::launch_attention_kvq(AttnArgs args, const halo_plan& plan, hipStream_t stream) {
  const halo_attn_params_t& p = plan.params;
  const bool d128 = p.head_dim == 128, f32 = p.out_dtype == HALO_F32;
  if (p.kv_dtype == HALO_BF16) {
    if (d128) {
      if (f32) launch_items<__bf16, 128, float>(args, plan, stream);
      else launch_items<__bf16, 128, __bf16>(args, plan, stream);
    } else {
      if (f32) launch_items<__bf16, 64, float>(args, plan, stream);
      else launch_items<__bf16, 64, __bf16>(args, plan, stream);
    }
  } else {
    if (d128) launch_items<float, 128, float>(args, plan, stream);
    else launch_items<float, 64, float>(args, plan, stream);
  }
}
