"""GPU checks of calls over 4-bit pools that stand beside each other: the
workspace, values at the ends of the range, cuts that must not show."""

import gc
import weakref

import numpy as np
import pytest
import torch

import oracle
from kvq_helpers import assert_close, check, expected, fill_pools, run, values
from paper_2509_02121_amd import halo
from workloads import build_workload

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def _w(seg_len, paths, q_len=None, heads=(4, 2), D=128, dtype=BF16, seed=5):
    return build_workload("kvq", seed, *heads, D, dtype, seg_len, paths, q_len, poison=False, extra_pages=3)


@pytest.mark.parametrize("out", [BF16, FP32])
def test_workspace_of_a_fresh_object(gpu_lib, out):
    """PrefixAttention.workspace is enough for a call over 4-bit pools, also
    before the first one, which then makes no other."""
    w = _w([600, 33, 257], [[0, 1], [0, 2]])
    pools = fill_pools(w)
    params = halo.make_params(4, 2, 128, BF16, w.num_pool_pages, w.scale, out)
    att = halo.PrefixAttention(params, w.forest_csr())
    assert att.plan.stats()["num_merge_rows"] > 0
    q, ws = w.q.cuda(), att.workspace
    o, lse = att.alloc_outputs(q)
    halo.prefix_attn_decode_kvq(att.plan, att.meta, q, *pools, o, lse, ws)
    o2, lse2 = att.run(q, *pools)
    torch.cuda.synchronize()
    assert att.workspace is ws
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def _token(w, seg, t):
    """(page, place in it) of token t of a segment."""
    return int(w.seg_pages[seg][t // 16]), t % 16


def _set_scale(pools, kind, D, page, head, t, scale, codes=None):
    """The scale of one token (K: of its first 32 dims), and for V its codes,
    as {dim: code}, the others 0."""
    tile = pools[kind][page, head].cpu().numpy()
    if kind == halo.HALO_POOL_K:
        tile[D * 8 + t * (D // 32)] = scale
    else:
        at = D * 8 + 2 * oracle.paged_kv.v_slot(t)
        tile[at], tile[at + 1] = scale & 0xff, scale >> 8
    for c in range(D) if codes is not None else ():
        n = oracle.paged_kvq.code_number(kind, D, t, c)
        byte, code = int(tile[n // 2]), codes.get(c, 0)
        tile[n // 2] = (byte & 0x0f) | code << 4 if n % 2 else (byte & 0xf0) | code
    pools[kind][page, head] = torch.from_numpy(tile).cuda()


# keys cut into few and into many pieces, by narrow and by wide items; merged by
# either kernel (rows of few partials, few rows of many)
CUTS = {"few": ({"wide": 0, "kc_shared": 512}, 3),
        "many": ({"wide": 0, "kc_shared": 32, "kc_private": 32}, 2), "wide": ({"wide": 1, "kc_wide": 512}, 12),
        "wide many": ({"wide": 1, "kc_wide": 64, "kc_private": 32}, 12)}


def _cut(name, D):
    """Groups of requests on segments 0 and 1, which are not multiples of a
    step, with a few keys of their own; one query for all, so that one key of
    segment 0 is the first of every row that sees it."""
    options, n = CUTS[name]
    w = _w([1000, 700] + [5 + 7 * r for r in range(2 * n)], [[r % 2, 2 + r] for r in range(2 * n)], heads=(8, 1), D=D)
    w.q[:] = w.q[:1, :1].clone()
    pools = fill_pools(w)
    k = values(pools[0].cpu().numpy()[np.asarray(w.seg_pages[0])], 0, D).reshape(-1, D)[:1000]
    return w, pools, options, int(np.argmax(k @ w.q[0, 0].double().numpy()))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cut", CUTS)
def test_infinite_value_leaves_other_dims(gpu_lib, cut, D):
    """A cached value whose dim 5 is an infinity (code 6 at the scale 2^126),
    with the largest weight: dim 5 of the rows that see it is infinite, and
    every other dim what it would be if that one were 0, however keys are cut."""
    w, pools, options, key = _cut(cut, D)
    page, t = _token(w, 0, key)
    _set_scale(pools, 1, D, page, 0, t, 0x7e80, {})
    clean, lse0, att = run(w, pools, BF16, options)
    stats = att.plan.stats()
    split = stats["num_merge_rows"] > 0
    assert split and (stats["num_wide_items"] > 0) == ("wide" in cut)
    assert (stats["num_partial_rows"] > 8 * stats["num_merge_rows"]) == ("many" in cut)   # (which merge runs)
    want = expected(w, pools)
    assert_close(w, BF16, clean, lse0, want, split, f"{cut}: clean")
    _set_scale(pools, 1, D, page, 0, t, 0x7e80, {5: 7})
    o, lse, _ = run(w, pools, BF16, options)
    sees = np.arange(len(w.req_paths)) % 2 == 0
    assert np.isposinf(o[sees, :, 5]).all() and np.array_equal(o[~sees], clean[~sees])
    o[sees, :, 5] = want[0][sees, :, 5]
    assert_close(w, BF16, o, lse, want, split, f"{cut}: with an infinity")
    assert np.array_equal(lse, lse0)


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cut", CUTS)
def test_nan_in_cut_keys(gpu_lib, cut, D, kind):
    """A NaN key or value makes NaN of the bf16 rows that see it and leaves
    the others' bits, however keys are cut; a NaN score has the LSE -inf, a
    NaN value leaves it."""
    w, pools, options, key = _cut(cut, D)
    clean, lse0, _ = run(w, pools, BF16, options)
    page, t = _token(w, 0, key)
    _set_scale(pools, kind, D, page, 0, t, 0x7fc0 if kind else 255)
    o, lse, _ = run(w, pools, BF16, options)
    sees = np.arange(len(w.req_paths)) % 2 == 0
    assert np.isnan(o[sees]).all()
    assert np.array_equal(o[~sees], clean[~sees]) and np.array_equal(lse[~sees], lse0[~sees])
    assert np.array_equal(lse[sees], lse0[sees]) if kind else np.isneginf(lse[sees]).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("D", [64, 128])
def test_gather_at_the_ends_of_the_range(gpu_lib, D, dtype):
    """All codes at the smallest and largest scales read back exactly:
    subnormals (2^-127 is one in either type) stay, 2^128 and more are
    infinities."""
    exps = [1, 2, 253, 254]
    rng = np.random.default_rng(D)
    pools, want = [], []
    for kind in (0, 1):
        tile = rng.integers(0, 256, (1, 1, oracle.paged_kvq.tile_bytes(kind, D)), dtype=np.uint8)
        if kind == halo.HALO_POOL_K:
            tile[0, 0, D * 8:] = np.resize(exps, D // 2)
        else:
            tile[0, 0, D * 8:] = (np.resize(exps, 16).astype(np.uint16) << 7).view(np.uint8)
        pools.append(torch.from_numpy(tile).cuda())
        x = np.stack([oracle.paged_kvq.read_token(tile[0, 0], kind, D, t) for t in range(16)])
        want.append(np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x))
        assert np.isinf(want[-1]).any() and (np.abs(want[-1]) == 2.0 ** -127).any()
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    outs = [torch.full((16, 1, D), 3.0, dtype=dtype, device="cuda") for _ in range(2)]
    params = halo.make_params(1, 1, D, dtype, 1, 0.125)
    halo.kvq_page_gather_kv(*pools, params, one, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), one + 16,
                            one.long(), *outs)
    for got, x in zip(outs, want):
        assert np.array_equal(got.double().cpu().numpy()[:, 0], x)


@pytest.mark.parametrize("out", [BF16, FP32])
@pytest.mark.parametrize("D", [64, 128])
def test_prefill_narrow(gpu_lib, D, out):
    """bf16 chunks as narrow items."""
    q_len = [257, 40, 100, 1]
    w = _w([300, 70] + q_len, [[0, 2], [1, 3], [4], [0, 5]], q_len, heads=(4, 1), D=D)
    att, _ = check(w, out, {"wide": 0}, f"narrow prefill d{D}")
    assert att.plan.stats()["num_wide_items"] == 0


@pytest.mark.parametrize("prefill", [False, True])
def test_calls_repeat_themselves(gpu_lib, prefill):
    """Two calls give the same bits (no result depends on an order of
    workgroups), with other work between them."""
    q_len = [200, 33] if prefill else None
    w = _w([1500, 300, 900] + (q_len or []), [[0, 1, 3], [0, 2, 4]] if prefill else [[0, 1], [0, 2]] * 20, q_len,
           heads=(16, 2))
    pools = fill_pools(w)
    o, lse, att = run(w, pools, BF16)
    for _ in range(5):
        torch.randn(1 << 22, device="cuda").sum()
        o2, lse2 = att.run(w.q, *pools)
        assert np.array_equal(o2.double().cpu().numpy(), o) and np.array_equal(lse2.double().cpu().numpy(), lse)


@pytest.mark.parametrize("seg_len", [[20], [600, 33]])
def test_bound_call_holds_its_plan(gpu_lib, seg_len):
    """bind() of an object that is dropped: the plan and its metadata live as
    long as the callable, with a workspace and without one."""
    w = _w(seg_len, [[*range(len(seg_len))]])
    pools = fill_pools(w)
    o, lse, att = run(w, pools, FP32)
    assert bool(att.plan.workspace_bytes) == (len(seg_len) > 1)
    out = att.alloc_outputs(w.q)
    call = att.bind(w.q, *pools, *out)
    held = [weakref.ref(att.plan), weakref.ref(att.meta)]
    del att
    gc.collect()
    assert all(x() is not None for x in held)
    call()
    torch.cuda.synchronize()
    assert np.array_equal(out[0].double().cpu().numpy(), o) and np.array_equal(out[1].double().cpu().numpy(), lse)
    del call
    gc.collect()
    assert all(x() is None for x in held)
