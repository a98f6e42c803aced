// gfx950 kernels for attention over 4-bit pools: the items of the same plans as
// over bf16 and fp32 pools (see halo_kernels.hip for the work decomposition, the
// layouts of the products and the merge, which are shared).
//
//   S = scale q K^T, P = softmax(S), O = P V with K = k_scale * k_code,
//   V = v_scale * v_code, codes E2M1 and scales powers of two.
//
// A K code times its scale is exact in bf16 and takes one conversion per two
// values. A V scale belongs to a key, i.e. runs along the contraction of P V.
// Narrow items multiply it onto P (exactly) after the sum of P is taken, and
// convert V codes with scale 1; wide items put it into V at the conversion, but in
// steps with masked keys onto P too.
//
// Narrow items convert in registers, between the loads and the MFMAs; wide items
// once per workgroup, on the way into LDS (wide_item). Per step of 32 keys and
// wave a narrow item reads 4.3 KB at d = 128 where bf16 pages take 16 KB, and adds
// 64 conversions (about 5 cycles each, measured) and 40 instructions for the scales
// to the softmax and the 16 MFMAs.
//
// What bounds them (d 128, bf16): narrow items over private keys read at the rate of
// the memory (1024 requests of 256-2048 keys, 1.24 GB: 252 us, 4.9 TB/s), those over
// shared keys wait for their instructions (VALU 926 cycles a step and SIMD); wide
// items for products (busy 42% of the cycles) and VALU instructions (54%), which
// overlap little (32 chunks of 512 tokens on 4096 keys 1175-1257 us by the card, 0.93
// to 0.99 PFLOP/s, 8 prefixes of 8192 under 1024 requests 300 us). A launch of both
// kinds takes nearly the sum of the two (70B-shaped decode 492-518 us); small calls
// are chains of dependent loads in two launches (8 requests of 300 keys 6.8-7.6 us).
//
// fp32 queries and outputs: K and V are exact in bf16, so products with fp32
// accuracy need only q (fp32 queries) and P (fp32 outputs) split into three bf16
// parts each (8 + 8 + 8 bits): three MFMAs of 16x16x32 in place of eight 16x16x4
// fp32 ones (4 requests of 12000-24000 keys 32 us: 16 steps in a chain, of 0.9 us
// alone on a SIMD and 1.4 where two share it). With bf16 queries and fp32 outputs P V
// is three products for one: 32 chunks of 512 tokens on 4096 keys 2061-2080
// us, 70B-shaped decode 740-753.
//
// Registers: at d 128 the wide kernels use all 256. With bf16 outputs 7 (8 in a launch
// of both kinds) are stored to scratch before the loop and loaded after it, none
// inside; with fp32 outputs 14 (9), of which 4 (1) are loaded again in each step.

#include <hip/hip_runtime.h>

#include <algorithm>

#include "halo_device.h"
#include "halo_internal.h"
#include "halo_kvq_format.h"

using namespace halo;

namespace {

// bf16 parts of an operand whose products go to type T: 1 for bf16 (rounded, as
// over bf16 pools), 3 for fp32.
template <typename T> constexpr int parts() { return sizeof(T) == 2 ? 1 : 3; }

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
  constexpr int NW = parts<TO>();   // of the softmax's weights
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
  // A lane's addresses of a step are page id * page bytes + an address that never
  // changes, one instruction each for codes and scales of K and V. A position past
  // the item's end loads from page 0 (of every wave the same few lines), so that
  // the count of loads in flight stays fixed without reading pages again.
  const uint32_t k_stride = a.num_kv_heads * kTile, v_stride = a.num_kv_heads * vTile;
  const uint64_t k_at = reinterpret_cast<uint64_t>(a.k_pool) + (uint64_t)it.kv_head * kTile + (grp * 16 + (col & 7)) * (D / 8);
  const uint64_t ks_at = reinterpret_cast<uint64_t>(a.k_pool) + (uint64_t)it.kv_head * kTile + D * 8 + (col & 7) * NS;
  const uint64_t v_at = reinterpret_cast<uint64_t>(a.v_pool) + (uint64_t)it.kv_head * vTile + ((grp & 1) * 16 + col) * 16;
  const uint64_t vs_at = reinterpret_cast<uint64_t>(a.v_pool) + (uint64_t)it.kv_head * vTile + D * 8 + (grp & 1) * 16;
  auto fetch = [&](const StepPos& p, Regs& r) {
    const uint32_t k_page = col < 8 ? p.pid0 : p.pid1, v_page = grp < 2 ? p.pid0 : p.pid1;
    const int64_t kq = k_at + (uint64_t)k_page * k_stride, kz = ks_at + (uint64_t)k_page * k_stride;
    const int64_t vq = v_at + (uint64_t)v_page * v_stride, vz = vs_at + (uint64_t)v_page * v_stride;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if constexpr (D == 128) {
        const u32x4_t w = load_global<u32x4_t, NT>(kq + x * D);
#pragma unroll
        for (int s = 0; s < NS; ++s) r.k[x][s] = w[s];
        r.ks[x] = load_global<uint32_t, NT>(kz + x * 8 * NS);
      } else {
        const u32x2_t w = load_global<u32x2_t, NT>(kq + x * D);
#pragma unroll
        for (int s = 0; s < NS; ++s) r.k[x][s] = w[s];
        r.ks[x] = load_global<uint16_t, NT>(kz + x * 8 * NS);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; b += 4) {
      const u32x4_t w = load_global<u32x4_t, NT>(vq + b * 128);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[b + i] = w[i];
    }
    r.vs = load_global<u32x4_t, NT>(vz);
  };

  // The span cursor: a later span's page ids are loaded, and waited for, when the
  // walk reaches it (see run_item).
  int si = 0;
  SpanState cur;
  cur.valid = it.n_spans > 0;
  cur.kb = it.s0_key_begin;
  cur.ke = it.s0_key_end;
  cur.causal = it.s0_causal;
  cur.vpid = rl.page;
  int t_next = cur.kb;
  auto advance = [&]() {
    while (cur.valid && t_next >= cur.ke) {
      cur = load_span(++si);
      wait_vmcnt<0>();
      t_next = cur.kb;
    }
    StepPos p;
    p.valid = cur.valid;
    p.t0 = t_next;
    p.key_end = cur.ke;
    p.causal = cur.causal;
    p.has1 = t_next + 16 < cur.ke;
    p.full = t_next + kKeysPerStep <= cur.ke && !cur.causal;
    const int j = (t_next - cur.kb) >> 4;
    p.pid0 = cur.valid ? __builtin_amdgcn_readlane(cur.vpid, j) : 0;
    p.pid1 = p.has1 ? __builtin_amdgcn_readlane(cur.vpid, j + 1) : p.pid0;
    t_next += kKeysPerStep;
    return p;
  };

  float m = kNegInf;
  float lsum = 0.f;
  f32x4_t acc[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto compute = [&](const StepPos& p, Regs& r) {
    f32x4_t sacc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const F kf = kvq_decode_bf16(r.k[x][s], kvq_scale_byte(r.ks[x], s));
#pragma unroll
        for (int n = NP - 1; n >= 0; --n) sacc[x] = mma(kf, qf[n][s], sacc[x]);
      }
    // slot j = 4X + i holds key t0 + slot_key(grp, j); raw scores, the scale is
    // applied with the maximum's subtraction (scale > 0)
    float sv[8], vs[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sv[j] = sacc[j >> 2][j & 3];
      vs[j] = __uint_as_float(j & 1 ? r.vs[j >> 1] & 0xffff0000u : r.vs[j >> 1] << 16);
    }
    if (!p.full) {
      // (a key that is not seen may have any scales: NaN scores, and a weight of
      // 0 times a NaN)
      asm volatile("");   // (a branch, not selects in every step)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = p.t0 + slot_key(grp, j);
        const bool vis = key < p.key_end && (!p.causal || key <= row.qpos);
        sv[j] = vis ? sv[j] : kNegInf;
        vs[j] = vis ? vs[j] : 0.f;
      }
    }
    const float m4[2] = {fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7]))};
    const float mt = rows_max(fmaxf(m4[0], m4[1])) * a.scale_log2;
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
#pragma unroll
    for (int j = 0; j < 8; ++j) pr[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(sv[j], a.scale_log2, -m_use));
    const float psum = ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
#pragma unroll
    for (int j = 0; j < 8; ++j) pr[j] *= vs[j];
    lsum += psum;
    F pf[NW];
    split(pr, pf);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const F vf = kvq_decode_bf16(r.v[b], 1.f);
#pragma unroll
      for (int n = NW - 1; n >= 0; --n) acc[b] = mma(vf, pf[n], acc[b]);
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
  finish_item<T, D, TO, sizeof(TO) == 2>(a, it, row, col, grp, acc, m, lsum);
}

// (3 and 4 stages: 64 requests on 2048 keys 16.4 and 16.6 us, 2: 16.1; loads are
// not what a step waits for)
constexpr int kKvqNarrowStages = 2;

// Launches with wide items have workgroups of four waves for either role, of which
// a CU holds two: narrow slots are taken in runs of four (two for a plan's bf16
// workgroup of eight), wide items in runs of 128 rows. Next to each other on a CU, a
// wide workgroup's products and a narrow one's loads and conversions overlap
// (70B-shaped decode 492 us; when it took 526, workgroups of eight took 545).
// Launches of narrow items alone keep the plan's workgroups, one to a CU: with two
// half as large the dispatcher fills some CUs twice and leaves others empty (64
// requests on 2048 shared keys 16.4 us, with eight 12.8).
constexpr int kKvqWaves = 4;
constexpr int kKvqRows = kKvqWaves * 32;

// Share (percent) of the narrow rounds dealt among the wide ones (see
// kWideSpanNarrowPct), by the number of wide workgroups. Up to one for each CU start
// first, all at once, and the narrow ones run beside and behind them: those that start
// later would end the launch. More are spread out, so that the two kinds share CUs.
// (us, with 0, 20 and 40) 256 workgroups: 128 requests of 64 query heads in 4 groups
// of 8192 shared and 128-512 own keys 71, 82, 83; 600 of 32 in 8 of 4096 151, 153,
// 177; 384: 300 of 64 in 6 of 4096 99, 98, 113, 700 in 8 of 2048 with up to 2048 own
// 255, 253, 246; 512: 512 in 4 of 8192 with up to 4096 own 442, 408, 394; 1024: the
// 70B-shaped decode 554, 521, 508 (with 60 517; 492 since).
int kvq_narrow_pct(int wide_units) { return wide_units <= kNumCUs ? 0 : wide_units < 2 * kNumCUs ? 20 : 40; }

template <typename T, int RB> constexpr int kvq_waves() { return RB > 0 ? kKvqWaves : block_waves<T>(); }

template <typename T, int D, typename TO, int W>
__device__ __forceinline__ void narrow_block_kvq(const AttnArgs& a, int block) {
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int lane = threadIdx.x & 63;
  // A plan's workgroup stays on its XCD (its index modulo 8), and its runs come
  // one dispatch cycle after the other.
  constexpr int kRuns = block_waves<T>() / W;
  const int round = block >> 3, rounds = a.narrow_blocks / (8 * kRuns);
  const int cycle = round / (kRuns * kSeCycle), width = min(kSeCycle, rounds - cycle * kSeCycle);
  const int at = round - cycle * kRuns * kSeCycle;
  const int of = kRuns == 1 ? block : (cycle * kSeCycle + at % width) * 8 + (block & 7);
  const int64_t item_id = (int64_t)of * block_waves<T>() + (kRuns == 1 ? 0 : at / width * W) + wave;
  const Item it = a.items[item_id];
  const ItemRec* rec = a.item_recs + item_id;
  const int col = lane & 15;
  const RecLane rl{rec->q_row[col], rec->aux[col], rec->page[lane & 31]};
  if (it.flags & kItemStream) run_item_kvq<T, D, TO, true, kKvqNarrowStages>(a, it, rl, lane);
  else run_item_kvq<T, D, TO, false, kKvqNarrowStages>(a, it, rl, lane);
}

// Both roles in one launch, dealt as in attn_kernel; wide unit u is run
// u % runs of 128 rows of item u / runs.
template <typename T, int D, typename TO, int RB>
__global__ __launch_bounds__((64 * kvq_waves<T, RB>())) __attribute__((amdgpu_waves_per_eu(2)))
void attn_kvq_kernel(AttnArgs a, int runs) {
  constexpr int W = kvq_waves<T, RB>();
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
      const int unit = xcd_remap((w_before * kSeCycle + q) * 8 + x, a.wide_group);
      if (unit < a.n_wide) wide_item<D, TO, W, kKvqStages, true>(a, unit / runs, smem, unit % runs * kKvqRows);
      return;
    }
    narrow_block_kvq<T, D, TO, W>(a, ((cyc - w_upto) * kSeCycle + q) * 8 + x);
  } else {
    (void)smem;
    narrow_block_kvq<T, D, TO, W>(a, b);
  }
}

// Wide items and nothing else (prefill).
template <int D, typename TO>
__global__ __launch_bounds__(64 * kKvqWaves) __attribute__((amdgpu_waves_per_eu(2)))
void wide_kvq_kernel(AttnArgs a, int runs) {
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kKvqStages * kvq_image_bytes<D>()];
  const int unit = xcd_remap(blockIdx.x, a.wide_group);
  if (unit < a.n_wide)
    wide_item<D, TO, kKvqWaves, kKvqStages, true>(a, unit / runs, smem, unit % runs * kKvqRows);
}

template <typename T, int D, typename TO>
void launch_items(AttnArgs args, const halo_plan& plan, hipStream_t stream) {
  const bool wide = sizeof(T) == 2 && plan.wide_rb > 0;
  const int runs = (plan.max_wide_rows + kKvqRows - 1) / kKvqRows;
  if (wide) {
    args.n_wide *= runs;
    args.wide_group *= runs;
  }
  args.narrow_blocks *= block_waves<T>() / (wide ? kKvqWaves : block_waves<T>());
  lay_out_rounds(args, wide, kvq_narrow_pct(args.n_wide));
  const int grid = args.wide_blocks + args.narrow_blocks;
  if (grid == 0) return;
  if constexpr (sizeof(T) == 2) {
    if (wide && args.narrow_blocks == 0) {
      hipLaunchKernelGGL((wide_kvq_kernel<D, TO>), dim3(pad_to(args.n_wide, 8 * args.wide_group)),
                         dim3(64 * kKvqWaves), 0, stream, args, runs);
      return;
    }
    if (wide) {
      hipLaunchKernelGGL((attn_kvq_kernel<T, D, TO, 1>), dim3(grid), dim3(64 * kKvqWaves), 0, stream, args, runs);
      return;
    }
  }
  hipLaunchKernelGGL((attn_kvq_kernel<T, D, TO, 0>), dim3(grid), dim3(64 * block_waves<T>()), 0, stream, args, runs);
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
