"""GPU checks of calls over 4-bit pools that stand beside each other: the
workspace, values at the ends of the range, cuts that must not show."""

import numpy as np
import pytest
import torch

import oracle
from kvq_helpers import assert_close, expected, fill_pools, run, values
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
