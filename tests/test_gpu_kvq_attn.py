"""GPU parity of attention over 4-bit pools with 64 bits over the values that
they stand for, with a derived bound for every output; and a serving step
made of the step operators together."""

import numpy as np
import pytest
import torch

import oracle
from kvq_helpers import assert_close, check, expected, fill_pools, run, values
from paper_2509_02121_amd import halo
from test_step import rope_frequencies
from workloads import build_workload, make_config, random_forest

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
TYPES = [(BF16, BF16), (BF16, FP32), (FP32, FP32)]


def _w(seg_len, paths, q_len=None, heads=(4, 2), D=128, dtype=BF16, seed=5):
    return build_workload("kvq", seed, *heads, D, dtype, seg_len, paths, q_len, poison=False, extra_pages=3)


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 511, 512, 513, 1025])
def test_decode_one_request(gpu_lib, n, D, dtype, out):
    """Lengths around a page, a step, a span."""
    check(_w([n], [[0]], D=D, dtype=dtype), out, label=f"one of {n}")


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("heads,D", [((1, 1), 64), ((16, 1), 128), ((6, 3), 128), ((32, 8), 64), ((20, 1), 128)])
def test_decode_heads(gpu_lib, heads, D, dtype, out):
    check(_w([100, 40, 0, 77], [[0, 1], [0, 2], [0, 3]], heads=heads, D=D, dtype=dtype), out, label=f"heads {heads}")


@pytest.mark.parametrize("dtype,out", TYPES)
def test_decode_without_keys(gpu_lib, dtype, out):
    """Rows that see nothing beside rows that do."""
    check(_w([0, 40, 0], [[0], [1, 2], [], [0, 2]], dtype=dtype), out, label="no keys")
    check(_w([0], [[0]], dtype=dtype), out, label="no keys at all")


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("dtype,out", TYPES)
def test_decode_random_forests(gpu_lib, seed, dtype, out):
    rng = np.random.default_rng(seed)
    seg_len, paths, _ = random_forest(rng, int(rng.integers(1, 24)), max_len=int(rng.choice([40, 300, 1500])))
    check(_w(seg_len, paths, heads=(8, 2), D=int(rng.choice([64, 128])), dtype=dtype, seed=seed), out, label=f"forest {seed}")


@pytest.mark.parametrize("out", [BF16, FP32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [0, 32, 96, 256])
def test_decode_wide(gpu_lib, rows, D, out):
    """Shared prefixes whose rows run as wide items, over prefixes that end
    inside a page, a step and a span, beside private keys."""
    seg_len = [777, 40, 1025, 3] + [int(x) for x in np.random.default_rng(1).integers(0, 90, 40)]
    paths = [[0, 2, 4 + r] if r % 2 else [1, 3, 4 + r] for r in range(40)]
    att, _ = check(_w(seg_len, paths, heads=(16, 2), D=D), out, {"wide": 1, "wide_rows": rows}, f"wide {rows}")
    assert att.plan.stats()["num_wide_items"] > 0


@pytest.mark.parametrize("n", [1, 5, 16, 17, 32, 33, 64, 95, 96, 97, 128, 129, 160, 192, 224, 4100])
def test_wide_lengths(gpu_lib, n):
    """Few steps: fewer than the pipeline holds, and around its length."""
    check(_w([n, 1], [[0], [0, 1]] * 8, heads=(8, 1), seed=n), FP32, {"wide": 1}, f"wide length {n}")


@pytest.mark.parametrize("options", [{"kc_shared": 64, "kc_private": 32}, {"kc_private": 64, "wide": 0},
                                     {"kc_wide": 96, "wide": 1, "wide_rows": 64}, {"items_per_block": 1},
                                     {"shared_unit": 1, "wide": 0}])
@pytest.mark.parametrize("dtype,out", TYPES)
def test_decode_split_keys(gpu_lib, options, dtype, out):
    """Keys cut into many pieces, merged."""
    if dtype == FP32:
        options = {k: v for k, v in options.items() if "wide" not in k}
    seg_len, paths = [600, 257, 900, 31, 1400], [[0, 1], [0, 2], [0, 3], [4]]
    check(_w(seg_len, paths, heads=(8, 2), dtype=dtype), out, options, f"split {options}")


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_prefill(gpu_lib, D, dtype, out):
    """Chunks around a wave's and a workgroup's rows over cached segments that
    end inside a page, a step and a span; among them none."""
    q_len = [1, 31, 32, 33, 127, 129, 200]
    seg_len = [0, 5, 48, 1023, 1025] + q_len
    paths = [[i % 5, 5 + i] if i else [5] for i in range(len(q_len))]
    check(_w(seg_len, paths, q_len, heads=(3, 3), D=D, dtype=dtype), out, label=f"prefill d{D}")


@pytest.mark.parametrize("options", [{"wide_rows": 32}, {"wide_rows": 256}])
@pytest.mark.parametrize("D", [64, 128])
def test_prefill_workgroups(gpu_lib, D, options):
    q_len = [257, 40, 100]
    check(_w([300, 70] + q_len, [[0, 2], [1, 3], [4]], q_len, heads=(4, 1), D=D), BF16, options, f"prefill {options}")


@pytest.mark.parametrize("dtype,out", TYPES)
@pytest.mark.parametrize("prefix,q_len", [(3001, [70]), (1500, [1, 200, 33]), (0, [900]), (7000, [1])])
def test_prefill_pieces(gpu_lib, prefix, q_len, dtype, out):
    """Few items whose keys are cut, and the same without the workspace."""
    seg_len = [prefix // 3, prefix - prefix // 3] + q_len
    w = _w(seg_len, [[0, 1, 2 + i] for i in range(len(q_len))], q_len, heads=(6, 2), dtype=dtype)
    att, pools = check(w, out, label=f"pieces {prefix}")
    assert att.plan.workspace_bytes > 0
    o, lse = att.alloc_outputs(w.q)
    halo.prefix_attn_prefill_kvq(att.plan, att.meta, w.q, *pools, o, lse, None)
    torch.cuda.synchronize()
    assert_close(w, out, o.double().cpu().numpy(), lse.double().cpu().numpy(), expected(w, pools), False, "uncut")


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("dtype,out", TYPES)
def test_prefill_random_forests(gpu_lib, seed, dtype, out):
    rng = np.random.default_rng(100 + seed)
    seg_len, paths, q_len = random_forest(rng, int(rng.integers(1, 12)), max_len=200, prefill=True, max_q=150)
    check(_w(seg_len, paths, q_len, heads=(8, 4), D=int(rng.choice([64, 128])), dtype=dtype, seed=seed), out,
          label=f"prefill forest {seed}")


@pytest.mark.parametrize("dtype,out", TYPES)
def test_strong_channels(gpu_lib, dtype, out):
    """A few key dims 30 times the others: scores of hundreds, one key with
    all the weight."""
    strong = torch.ones(128)
    strong[::29] = 30.0
    check(_w([900, 33, 20], [[0, 1], [0, 2]], dtype=dtype), out, label="strong", strong=strong)


@pytest.mark.parametrize("prefill", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_fp32_keeps_every_bit(gpu_lib, D, prefill):
    """fp32 queries of one dim, so that a score is one product: q in two bf16
    parts instead of three would be off by 2^-17 of it, and so would weights.
    Here a score has at most 8 roundings (three parts' sums, the scale, the
    maximum, exp2 and its argument), of scores up to B, and an output 24 more."""
    w = _w([3, 2], [[0, 1]], [2] if prefill else None, heads=(4, 4), D=D, dtype=FP32)
    w.q[:, :, 1:] = 0.0
    w.q[:, :, 0] = torch.tensor([3.1415927, -2.7182817, 17.123457, 0.57721567]) * D ** 0.5
    pools = fill_pools(w)
    o, lse, _ = run(w, pools, FP32)
    ro, rl, A, B, _ = expected(w, pools)
    sums = 2.0 ** -24 * 8 * (B + 1)
    assert (np.abs(lse - rl) <= 2 * sums + 2.0 ** -22 * np.abs(rl)).all()
    assert (np.abs(o - ro) <= A * (4 * sums[..., None] + 24 * 2.0 ** -24)).all()


@pytest.mark.parametrize("prefill", [False, True])
def test_nan_tokens_stay_in_their_rows(gpu_lib, prefill):
    """A cached NaN token makes NaN of the rows that see it and of no other:
    another request's, an earlier chunk row's."""
    if prefill:
        w = _w([40, 50, 50], [[0, 1], [0, 2]], [50, 50], heads=(2, 1))
    else:
        w = _w([40, 50, 50], [[0, 1], [0, 2]], heads=(2, 1))
    pools = fill_pools(w)
    clean, _, _ = run(w, pools, FP32)
    page, D = int(w.seg_pages[1][1]), 128   # tokens 16 .. 31 of segment 1
    pools[0][page, 0, D * 8 + 3 * 4 + 2] = 255                     # K of token 3: position 19
    o, lse, _ = run(w, pools, FP32)
    first = 19 if prefill else 0
    rows = 50 if prefill else 1
    assert np.isnan(o[first:rows]).all() and not np.isnan(o[:first]).any() and not np.isnan(o[rows:]).any()
    if prefill:
        assert np.array_equal(o[:16], clean[:16])
    pools[0][page, 0, D * 8 + 3 * 4 + 2] = 127
    slot = oracle.paged_kv.v_slot(3)
    pools[1][page, 0, D * 8 + 2 * slot:D * 8 + 2 * slot + 2] = torch.tensor([0xc0, 0x7f], dtype=torch.uint8)
    o, lse, _ = run(w, pools, FP32)
    assert np.isnan(o[first:rows]).all() and not np.isnan(o[:first]).any() and not np.isnan(o[rows:]).any()
    assert np.isfinite(lse).all()


@pytest.mark.parametrize("wide", [0, 1])
def test_wide_and_narrow_nan_tail(gpu_lib, wide):
    """Random bytes behind the last token of every segment (NaN scales among
    them) never show: two fillings of the rest give the same bits."""
    w = _w([37, 1, 70, 16], [[0, 1], [0, 2], [0, 3]] * 6, heads=(8, 2))
    a, la, _ = run(w, fill_pools(w, 1), BF16, {"wide": wide})
    b, lb, _ = run(w, fill_pools(w, 2), BF16, {"wide": wide})
    assert np.array_equal(a, b) and np.array_equal(la, lb) and np.isfinite(a).all()


def test_same_as_dequantised_pools(gpu_lib):
    """Over bf16 pools of the same values the result is the same to the
    rounding of either."""
    w = _w([500, 33, 70, 800], [[0, 1], [0, 2], [0, 3]], heads=(8, 2))
    pools = fill_pools(w)
    o, lse, _ = run(w, pools, FP32)
    k, v = (torch.from_numpy(values(p.cpu().numpy(), z, 128)).cuda() for z, p in enumerate(pools))
    dense_k = k.permute(0, 2, 1, 3).reshape(-1, 2, 16, 16, 8).permute(0, 1, 3, 2, 4).to(BF16).contiguous()
    slots = torch.tensor([oracle.paged_kv.v_slot(t) for t in range(16)], device="cuda")
    dense_v = v[:, slots].permute(0, 2, 3, 1).to(BF16).contiguous()
    o2, lse2, _ = run(w, (dense_k, dense_v), FP32)
    want = expected(w, pools)
    assert_close(w, FP32, o, lse, want, True, "4-bit pools")
    # (over bf16 pools the weights are rounded to bf16 for an fp32 output too)
    assert_close(w, BF16, o2, lse2, want, True, "bf16 pools")


def test_configured_workloads(gpu_lib):
    """The 8B-shaped decode, the tree and a chunked prefill at their sizes
    (fewer requests), through the planner's own choices."""
    for name, out in (("llama8b_decode", BF16), ("two_level_tree_decode", FP32)):
        w = make_config(name, poison=False)
        w.req_paths = w.req_paths[:24]
        w.q = w.q[:24]
        check(w, out, label=name)
    rng = np.random.default_rng(4)
    w = _w([2048] + list(rng.integers(256, 600, 64)), [[0, 1 + r] for r in range(64)], heads=(64, 8))
    check(w, BF16, label="70B-shaped group")


def test_long_offsets(gpu_lib):
    """Pages past 4 GiB of a pool."""
    w = _w([100, 20], [[0, 1]], heads=(8, 8))
    small = fill_pools(w)
    n_pool = (5 << 30) // (8 * 1056)
    move = np.random.default_rng(0).permutation(np.arange(n_pool - 1000, n_pool))[:w.num_pool_pages]
    big = []
    for p in small:
        t = torch.empty((n_pool, *p.shape[1:]), dtype=torch.uint8, device="cuda")
        t[torch.from_numpy(move).cuda()] = p
        big.append(t)
    want, lse, _ = run(w, small, FP32)
    w.seg_pages = [move[p] for p in w.seg_pages]
    w.num_pool_pages = n_pool
    o, lse2, _ = run(w, big, FP32)
    assert np.array_equal(o, want) and np.array_equal(lse, lse2)


def test_bound_captured_and_on_streams(gpu_lib):
    """A bound call, two graphs of one plan replayed at once on two streams,
    and eager calls between them."""
    w = _w([2000, 300, 900, 40], [[0, 1], [0, 2], [0, 3]], heads=(8, 2))
    pools = fill_pools(w)
    _, _, att = run(w, pools, BF16)
    assert att.plan.workspace_bytes > 0
    qs = [w.q, -w.q]
    want = [att.run(q, *pools) for q in qs]
    bound = [att.alloc_outputs(w.q) for _ in qs]
    for q, out in zip(qs, bound):
        att.bind(q, *pools, *out)()
    graphs, outs = [], []
    for q in qs:
        out, g = att.alloc_outputs(w.q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            att.run(q, *pools, *out)
        graphs.append(g)
        outs.append(out)
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for i in range(5):
        for out in outs:
            out[0].zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        again = att.run(qs[i % 2], *pools)
        torch.cuda.synchronize()
        for got in (outs, bound):
            for (o, lse), (eo, el) in zip(got, want):
                assert torch.equal(o, eo) and torch.equal(lse, el)
        assert torch.equal(again[0], want[i % 2][0])


def test_mixed_pools_are_refused(gpu_lib):
    w = _w([20], [[0]])
    pools = fill_pools(w)
    _, _, att = run(w, pools, BF16)
    with pytest.raises(ValueError):
        att.run(w.q, pools[0], w.v_pool.cuda())
    with pytest.raises(ValueError):
        att.run(w.q, w.k_pool.cuda(), pools[1])
    with pytest.raises(ValueError):
        att.run(w.q, pools[0][:-1], pools[1])


# ------------------------------------------------------------------- a serving loop

@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_serving_loop(gpu_lib, dtype):
    """Decode steps as a serving loop makes them: the step's tables from the
    lengths on the GPU, queries and keys turned by their positions, the new
    tokens quantised into their pages, the plan brought up to date on the
    host (which knows which page went where), attention. Checked at every
    step against 64 bits over what was written."""
    n, steps, H, Hq, D = 6, 20, 2, 8, 64
    rng = np.random.default_rng(8)
    prefix, own = 50, rng.integers(1, 40, n)
    used = -(-prefix // 16)
    p = halo.make_params(Hq, H, D, dtype, 80, D ** -0.5)
    pools = halo.alloc_kvq_pools(p)
    order = rng.permutation(80).astype(np.int32)
    free, nxt = order[used:], 0
    width = 8
    table = np.zeros((n, width), np.int32)
    rope = halo.Rope(D, base=10000.0)
    freq = np.array(rope_frequencies(D, 10000.0, "none", 1.0, 8192, 32, 1)[0])
    gen = torch.Generator().manual_seed(3)

    def cuda(x, dt=torch.int32):
        return torch.tensor(np.asarray(x), dtype=dt, device="cuda")

    def step(lens, new, first_pos):
        """One step's writes; returns what was turned and written."""
        T = int(sum(new))
        rows = torch.randn((T, (Hq + 2 * H) * D), generator=gen).to(dtype).cuda()
        q, k, v = (x.view(T, -1, D) for x in rows.split([Hq * D, H * D, H * D], 1))
        tabs = halo.StepTables(n, T, n * width)
        flag = cuda([0])
        halo.kv_step_tables(tabs, cuda(lens), cuda(new), d_table, d_free, d_next, flag)
        pos = tabs.positions + first_pos   # the private tokens follow the prefix
        plain = [t.double().cpu().numpy() for t in (q, k)]
        halo.rope_qk(q, k, pos, rope)
        halo.kvq_page_scatter_kv(*pools, p, tabs.page_ids, tabs.seq_page_indptr, tabs.seq_start, tabs.seq_count,
                                 tabs.in_token_offset, k.contiguous(), v.contiguous(), flag)
        d_next.copy_(tabs.free_next)
        angle = pos.cpu().numpy()[:, None, None] * freq
        for x, got in zip(plain, (q, k)):
            a, b = x[..., :D // 2], x[..., D // 2:]
            turned = np.concatenate([a * np.cos(angle) - b * np.sin(angle), a * np.sin(angle) + b * np.cos(angle)], -1)
            assert np.abs(got.double().cpu().numpy() - turned).max() <= np.abs(x).max() * 2 * (
                2.0 ** -8 if dtype == BF16 else 2.0 ** -20)
        assert flag.item() == 0
        return q, tabs

    # the prefix and the private prompts
    d_table, d_free, d_next = cuda(table), cuda(free), cuda([0])
    kv = [torch.randn((prefix, H, D), generator=gen).to(dtype).cuda() for _ in range(2)]
    halo.kvq_page_scatter_kv(*pools, p, cuda(order[:used]), cuda([0, used]), cuda([0]), cuda([prefix]),
                             cuda([0], torch.int64), *kv)
    lens = np.zeros(n, np.int64)
    new, att = own, None
    for i in range(steps):
        q, tabs = step(lens, new, prefix)
        # the host's own account of the pages
        for r in range(n):
            for j in range(-(-lens[r] // 16), -(-(lens[r] + new[r]) // 16)):
                table[r, j] = free[nxt]
                nxt += 1
        lens = lens + new
        assert np.array_equal(d_table.cpu().numpy(), table)
        pages = [order[:used]] + [table[r, :-(-lens[r] // 16)] for r in range(n)]
        csr = {"seg_len": np.array([prefix, *lens], np.int32),
               "seg_page_indptr": np.cumsum([0] + [len(x) for x in pages]).astype(np.int32),
               "seg_page_ids": np.concatenate(pages), "req_seg_indptr": np.arange(0, 2 * n + 1, 2, dtype=np.int32),
               "req_seg_ids": np.array([[0, 1 + r] for r in range(n)], np.int32).ravel(), "q_len": None}
        last = (np.cumsum(new) - 1).tolist()
        q = q[last].contiguous()
        if att is None:
            att = halo.PrefixAttention(p, csr)
        else:
            att.update(csr)
        o, lse = att.run(q, *pools)
        w = build_workload("loop", 0, Hq, H, D, dtype, csr["seg_len"], [[0, 1 + r] for r in range(n)], poison=False)
        w.seg_pages, w.num_pool_pages, w.scale = pages, 80, float(np.float32(D ** -0.5))
        assert_close(w, dtype, o.double().cpu().numpy(), lse.double().cpu().numpy(), expected(w, pools, q), True, f"step {i}")
        new = np.ones(n, np.int64)
