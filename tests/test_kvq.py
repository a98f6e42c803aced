"""The 4-bit cache on the CPU: the oracle's format pinned by worked examples
and invariants, and what the entry points refuse."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged_kvq
from paper_2509_02121_amd import halo


@pytest.fixture(scope="module")
def lib():
    return halo.load_library()


@pytest.mark.parametrize("y,code", [(0, 0), (0.25, 0), (0.26, 1), (0.5, 1), (0.75, 2), (1.25, 2), (1.3, 3), (1.75, 4),
                                    (2.5, 4), (2.51, 5), (3.5, 6), (5, 6), (5.01, 7), (6, 7), (6.99, 7), (-0.0, 8),
                                    (-0.75, 10), (-6.5, 15)])
def test_nearest_code(y, code):
    assert paged_kvq.nearest_code(y) == code


@pytest.mark.parametrize("top,e", [(1.0, -2), (1.74, -2), (1.75, -1), (1.99, -1), (2.0, -1), (6.0, 0), (7.0, 1),
                                   (0.0, -126), (1e-45, -126), (2.0 ** -124, -126), (2.0 ** -123, -125),
                                   (3.4e38, 126), (math.inf, None), (math.nan, None)])
def test_scale_exponent(top, e):
    assert paged_kvq.scale_exponent([0.1 * top if math.isfinite(top) else 0.5, -top]) == e


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("D", [64, 128])
def test_tile_layout(kind, D):
    """Every code has a place of its own, and a written token reads back as
    its nearest values with the others left alone."""
    numbers = {paged_kvq.code_number(kind, D, t, c) for t in range(16) for c in range(D)}
    assert numbers == set(range(16 * D))
    rng = np.random.default_rng(D + kind)
    tile = rng.integers(0, 255, paged_kvq.tile_bytes(kind, D)).astype(np.uint8)
    if kind:   # (a random bf16 may be an infinity, times 0)
        tile[D * 8:] = np.tile(np.array([0x80, 0x3f], np.uint8), 16)
    before = [paged_kvq.read_token(tile, kind, D, t) for t in range(16)]
    x = rng.standard_normal(D)
    paged_kvq.write_token(tile, kind, D, 5, x)
    for t in range(16):
        if t != 5:
            assert np.array_equal(paged_kvq.read_token(tile, kind, D, t), before[t], equal_nan=True)
    got = paged_kvq.read_token(tile, kind, D, 5)
    block = 32 if kind == 0 else D
    for s in range(0, D, block):
        unit = 2.0 ** paged_kvq.scale_exponent(x[s:s + block])
        # half of the widest step, or what lies between 6 and the largest 7
        assert np.abs(got[s:s + block] - x[s:s + block]).max() <= unit


def test_hand_worked_block():
    """Largest magnitude 6: the unit is 1, and these are the values."""
    x = np.zeros(64)
    x[:8] = [6, -5, 3.4, 2.5, 1.75, 0.75, 0.25, -0.3]
    tile = np.zeros(paged_kvq.tile_bytes(0, 64), np.uint8)
    paged_kvq.write_token(tile, 0, 64, 0, x)
    # token 0, g = 0, s = 0: the first four bytes
    assert tile[:4].tolist() == [0x7 | 0xe << 4, 0x5 | 0x4 << 4, 0x4 | 0x2 << 4, 0x0 | 0x9 << 4]
    assert tile[512] == 127 and tile[513] == 1
    assert paged_kvq.read_token(tile, 0, 64, 0)[:8].tolist() == [6, -4, 3, 2, 2, 1, 0, -0.5]


def _params(**given):
    p = halo.make_params(8, 2, 64, torch.bfloat16, 10, 0.125)
    for k, v in given.items():
        setattr(p, k, v)
    return p


def test_pool_bytes(lib):
    assert halo.kvq_pool_bytes(_params(), halo.HALO_POOL_K) == 10 * 2 * (512 + 32)
    assert halo.kvq_pool_bytes(_params(), halo.HALO_POOL_V) == 10 * 2 * (512 + 32)
    assert halo.kvq_pool_bytes(_params(head_dim=128), halo.HALO_POOL_K) == 10 * 2 * 1088
    assert halo.kvq_pool_bytes(_params(head_dim=128), halo.HALO_POOL_V) == 10 * 2 * 1056
    k, v = halo.alloc_kvq_pools(_params(head_dim=128), "cpu")
    assert k.shape == (10, 2, 1088) and v.shape == (10, 2, 1056)
    for bad in ({"head_dim": 96}, {"page_size": 32}, {"num_kv_heads": 0}, {"kv_dtype": 7}, {"num_pool_pages": -1},
                {"num_kv_heads": 1 << 30}, {"num_pool_pages": 1 << 60}):
        with pytest.raises(halo.HaloError):
            halo.kvq_pool_bytes(_params(**bad), halo.HALO_POOL_K)
    with pytest.raises(halo.HaloError):
        halo.kvq_pool_bytes(_params(), 2)


def _address():
    buf = np.zeros(64, np.int64)
    return buf, (buf.ctypes.data + 15) // 16 * 16


@pytest.mark.parametrize("call", ["scatter", "gather", "copy"])
def test_refusals(lib, call):
    """Calls with host addresses: each is refused before any launch."""
    keep, at = _address()
    fn, n_ptr = {"scatter": (lib.halo_kvq_page_scatter_kv, 9), "gather": (lib.halo_kvq_page_gather_kv, 8),
                 "copy": (lib.halo_kvq_page_copy, 3)}[call]

    def run(params=None, null=None, n=2, off=None, kind=0):
        p = _params() if params is None else params
        ptrs = [at] * n_ptr
        if null is not None:
            ptrs[null] = None
        if off is not None:
            ptrs[off] = at + 4
        ref = ctypes.byref(p) if p != 0 else None
        if call == "copy":
            return fn(ptrs[0], ref, kind, ptrs[1], ptrs[2], n, None, None)
        k, v, lists, data = ptrs[0], ptrs[1], ptrs[2:-2], ptrs[-2:]
        return fn(k, v, ref, *lists, n, *data, None, None)

    assert run(n=0) == halo.HALO_OK
    assert run(n=-1) == halo.HALO_ERR_INVALID_ARGUMENT
    assert run(params=0) == halo.HALO_ERR_INVALID_ARGUMENT
    for i in range(n_ptr):
        assert run(null=i) == halo.HALO_ERR_INVALID_ARGUMENT, i
    for i in (0, 1, n_ptr - 2, n_ptr - 1) if call != "copy" else (0,):
        assert run(off=i) == halo.HALO_ERR_INVALID_ARGUMENT, i
    assert run(params=_params(head_dim=80)) == halo.HALO_ERR_UNSUPPORTED
    assert run(params=_params(page_size=8)) == halo.HALO_ERR_UNSUPPORTED
    assert run(params=_params(kv_dtype=3)) == halo.HALO_ERR_UNSUPPORTED
    assert run(params=_params(num_kv_heads=0)) == halo.HALO_ERR_INVALID_ARGUMENT
    assert run(params=_params(num_pool_pages=-1)) == halo.HALO_ERR_INVALID_ARGUMENT
    assert run(params=_params(num_kv_heads=1 << 30)) == halo.HALO_ERR_UNSUPPORTED
    assert run(params=_params(num_pool_pages=1 << 40)) == halo.HALO_ERR_UNSUPPORTED
    if call == "copy":
        assert run(kind=2) == halo.HALO_ERR_INVALID_ARGUMENT


def test_arguments(lib):
    p = _params()
    k, v = halo.alloc_kvq_pools(p, "cpu")
    i32, i64 = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int64)
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    one = i32[:1]
    good = [k, v, p, i32, i32, one, one, i64, x, x]
    for at, bad in ((0, k[:9]), (1, v.view(torch.int8)), (4, i32.long()), (5, one.long()), (6, torch.zeros(0, dtype=torch.int32)),
                    (7, one), (8, x.float()), (9, x.transpose(1, 2)), (None, None)):   # the last: not on a GPU
        args = list(good)
        if at is not None:
            args[at] = bad
        with pytest.raises(ValueError):
            halo.kvq_page_scatter_kv(*args)
    for at, bad in ((0, k[:9]), (5, i64), (6, one), (7, x.float()), (None, None)):
        args = [k, v, p, i32, i32, one, i64, x, x]
        if at is not None:
            args[at] = bad
        with pytest.raises(ValueError):
            halo.kvq_page_gather_kv(*args)
    with pytest.raises(ValueError):
        halo.kvq_page_copy(k, p, halo.HALO_POOL_K, i32, one)


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("D", [64, 128])
def test_vectorised_reading(kind, D):
    """The helper that the GPU tests read whole pools with."""
    from kvq_helpers import values
    rng = np.random.default_rng(kind + D)
    tiles = rng.integers(0, 256, (3, 2, paged_kvq.tile_bytes(kind, D)), dtype=np.uint8)
    got = values(tiles, kind, D)
    for n in range(3):
        for h in range(2):
            for t in range(16):
                with np.errstate(all="ignore"):
                    assert np.array_equal(got[n, t, h], paged_kvq.read_token(tiles[n, h], kind, D, t), equal_nan=True)


def test_attention_arguments(lib):
    """Pools too small, of another type than the other one, or on the host."""
    from workloads import build_workload
    w = build_workload("args", 1, 4, 2, 64, torch.bfloat16, [20, 5], [[0, 1]])
    p = halo.make_params(4, 2, 64, torch.bfloat16, w.num_pool_pages, w.scale)
    plan = halo.Plan.from_csr(p, w.forest_csr())
    k, v = halo.alloc_kvq_pools(p, "cpu")
    meta = torch.zeros(plan.device_meta_bytes, dtype=torch.uint8)
    o, lse = torch.zeros_like(w.q), torch.zeros(w.q.shape[:2])
    ws = torch.zeros(max(plan.workspace_bytes, 1), dtype=torch.uint8)
    for bad in ((k[:-1], v), (k, v[:, :, :-1]), (k, v.view(torch.int8)), (w.k_pool, v), (k, v)):
        with pytest.raises(ValueError):
            halo.prefix_attn_decode_kvq(plan, meta, w.q, *bad, o, lse, ws)


@pytest.mark.parametrize("name,prefill", [("halo_prefix_attn_decode_kvq", False), ("halo_prefix_attn_prefill_kvq", True)])
def test_attention_refusals(lib, name, prefill):
    from workloads import build_workload
    w = build_workload("args", 1, 4, 2, 64, torch.bfloat16, [300, 5], [[0, 1]], [5] if prefill else None)
    p = halo.make_params(4, 2, 64, torch.bfloat16, w.num_pool_pages, w.scale)
    csr = w.forest_csr()
    plan = halo.Plan.from_csr(p, csr)
    other = halo.Plan.from_csr(p, {**csr, "q_len": None if prefill else np.array([5], np.int32)})
    keep, at = _address()
    at = (at + 255) // 256 * 256
    fn = getattr(lib, name)
    good = [plan._handle, at, at, at, at, at, at, at, 1 << 40, None]
    for i, bad in ((0, None), (0, other._handle), (1, None), (2, None), (3, None), (4, None), (5, None), (1, at + 16),
                   (2, at + 4), (3, at + 8), (4, at + 2), (5, at + 1)):
        args = list(good)
        args[i] = bad
        assert fn(*args) == halo.HALO_ERR_INVALID_ARGUMENT, i
    if not prefill:
        assert plan.kvq_workspace_bytes > plan.workspace_bytes > 0   # (bf16 output: a scale for each partial)
        for n in (0, plan.workspace_bytes, plan.kvq_workspace_bytes - 1):
            assert fn(*good[:8], n, None) == halo.HALO_ERR_WORKSPACE_TOO_SMALL


def test_workspace_bytes(lib):
    from workloads import build_workload
    w = build_workload("ws", 1, 4, 2, 64, torch.bfloat16, [300, 5, 7], [[0, 1], [0, 2]])
    for out, scales in ((torch.bfloat16, True), (torch.float32, False)):
        plan = halo.Plan.from_csr(halo.make_params(4, 2, 64, torch.bfloat16, w.num_pool_pages, w.scale, out), w.forest_csr())
        slots = len(plan.inspect()["merge_parts"])
        assert plan.stats()["num_merge_rows"] > 0
        more = plan.kvq_workspace_bytes - plan.workspace_bytes
        assert more >= 4 * slots and more % 256 == 0 if scales else more == 0
    assert lib.halo_plan_kvq_workspace_bytes(None) == 0
