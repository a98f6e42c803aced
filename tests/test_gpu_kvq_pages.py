"""GPU checks of the 4-bit pages, bit for bit against the oracle: tokens
quantised into pages (appends, chunks, ragged ones), read back, and pages
copied."""

import math

import numpy as np
import pytest
import torch

from oracle import paged_kv, paged_kvq
from paper_2509_02121_amd import halo

pytestmark = pytest.mark.gpu

K, V = halo.HALO_POOL_K, halo.HALO_POOL_V


def _cuda(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def _lists(seqs):
    indptr = np.cumsum([0] + [len(p) for p, *_ in seqs])
    ids = np.concatenate([np.asarray(p, np.int64) for p, *_ in seqs] + [np.zeros(1, np.int64)])
    return _cuda(ids), _cuda(indptr)


def _params(D, H, n_pool, dtype):
    return halo.make_params(H, H, D, dtype, n_pool, 0.125, dtype)


def _random_pools(D, H, n_pool, rng):
    """Pools of random bytes with finite scales."""
    k = rng.integers(0, 256, (n_pool, H, paged_kvq.tile_bytes(K, D)), dtype=np.uint8)
    v = rng.integers(0, 256, (n_pool, H, paged_kvq.tile_bytes(V, D)), dtype=np.uint8)
    k[:, :, D * 8:] = rng.integers(100, 150, k[:, :, D * 8:].shape)
    v[:, :, D * 8:] = (rng.integers(100, 150, (n_pool, H, 16)) << 7).astype(np.uint16).view(np.uint8)
    return k, v


def _write(D, H, n_pool, seqs, dtype, values, rng, flag=False):
    """Scatter and compare every byte of both pools with the oracle's.
    seqs: (page ids, start, count); values: [tokens, H, D] for K and V."""
    pools = _random_pools(D, H, n_pool, rng)
    offs = np.cumsum([0] + [max(c, 0) for _, _, c in seqs])[:-1]
    dev = [torch.from_numpy(p).cuda() for p in pools]
    src = [torch.tensor(x, dtype=torch.float32).to(dtype) for x in values]
    exp, flags = zip(*(paged_kvq.scatter(pools[z], z, D, [p for p, _, _ in seqs], [s for _, s, _ in seqs],
                                         [c for _, _, c in seqs], offs, src[z].double().numpy()) for z in (K, V)))
    ids, indptr = _lists(seqs)
    err = _cuda([0])
    args = (*dev, _params(D, H, n_pool, dtype), ids, indptr, _cuda([s for _, s, _ in seqs]),
            _cuda([c for _, _, c in seqs]), _cuda(offs, torch.int64), src[0].cuda(), src[1].cuda(), err)
    halo.kvq_page_scatter_kv(*args)
    for z in (K, V):
        assert np.array_equal(dev[z].cpu().numpy(), exp[z]), "KV"[z]
    assert bool(err.item()) == any(flags) == flag
    return dev


def _normal(rng, seqs, H, D):
    n = sum(max(c, 0) for _, _, c in seqs)
    return [rng.standard_normal((max(n, 1), H, D)) * np.exp(rng.uniform(-9, 9, (max(n, 1), 1, 1))) for _ in range(2)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,H", [(64, 1), (64, 3), (128, 1), (128, 2)])
def test_appends(gpu_lib, D, H, dtype):
    """One token at each place of a page."""
    rng = np.random.default_rng(D + H)
    seqs = [([2 * i, 2 * i + 1], start, 1) for i, start in enumerate(list(range(18)) + [31])]
    _write(D, H, 2 * len(seqs), seqs, dtype, _normal(rng, seqs, H, D), rng)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,H", [(64, 2), (128, 1)])
def test_chunks(gpu_lib, D, H, dtype):
    """Chunks that begin and end inside a page, and whole pages."""
    rng = np.random.default_rng(D + 1)
    spans = [(0, 16), (0, 33), (5, 4), (3, 13), (15, 2), (7, 41), (16, 16), (30, 20), (1, 1), (0, 7), (9, 0), (4, 9)]
    pages = rng.permutation(60)
    seqs, at = [], 0
    for start, count in spans:
        need = max(1, -(-(start + count) // 16))
        seqs.append((pages[at:at + need], start, count))
        at += need
    _write(D, H, 64, seqs, dtype, _normal(rng, seqs, H, D), rng)


@pytest.mark.parametrize("n", [70, 257, 530])
def test_many_sequences(gpu_lib, n):
    rng = np.random.default_rng(n)
    seqs = [([i], int(rng.integers(0, 15)), 1) for i in range(n)]
    _write(64, 1, n, seqs, torch.bfloat16, _normal(rng, seqs, 1, 64), rng)


@pytest.mark.parametrize("H", [8, 40, 130])
def test_many_heads(gpu_lib, H):
    rng = np.random.default_rng(H)
    seqs = [([0], 14, 2), ([1], 0, 1)]
    _write(64, H, 2, seqs, torch.bfloat16, _normal(rng, seqs, H, 64), rng)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_special_values(gpu_lib, dtype):
    """Zeros of both signs, ties, the bound between two scales, the smallest
    and largest numbers, infinities and NaN: in one block, the others stay."""
    rng = np.random.default_rng(0)
    D, n = 128, 24
    x = rng.standard_normal((n, 1, D))
    x[0] = 0.0
    x[1, 0, ::2] = -0.0
    x[1, 0, 1::2] = 0.0
    x[2, 0] = np.resize([0.25, -0.75, 1.25, -1.75, 2.5, -3.5, 5.0, 6.0], D)
    for i, top in enumerate([7.0, 6.96875, 3.5, 3.484375, 1.75, 1e-40, 2.0 ** -126, 3e38, 2.0 ** 127]):
        x[3 + i, 0, :] *= 0.1 * min(top, 1e37)
        x[3 + i, 0, 77] = top
    x[12, 0, 40] = np.inf
    x[13, 0, 40] = -np.inf
    x[14, 0, 3] = np.nan
    x[15, 0, 100:] = np.nan
    x[16] = 1e-45
    x[17] *= 1e-38
    seqs = [([0, 1], 2, n)]
    _write(D, 1, 2, seqs, dtype, [x, x[::-1].copy()], rng)


def test_bad_ranges_and_pages(gpu_lib):
    """Sequences whose range does not fit are left out whole, pages out of
    range are passed over, and the flag says so."""
    rng = np.random.default_rng(3)
    good = ([4], 3, 2)
    for bad in (([0], -1, 2), ([0], 15, 2), ([0, -1], 10, 10), ([0, 9, 1], 0, 48), ([2 ** 31 - 1], 0, 1),
                ([0], 2 ** 31 - 1, 1)):
        seqs = [bad, good] if bad[1] < 100 else [good, bad]
        _write(64, 2, 9, seqs, torch.bfloat16, _normal(rng, seqs, 2, 64), rng, flag=True)


# ------------------------------------------------------------------- read back

def _gather(D, H, pools, seqs, dtype, first=0):
    """Tokens of seqs (page ids, length) in dense buffers, against the
    oracle's values; other rows keep their bits."""
    total = sum(n for _, n in seqs)
    offs = np.cumsum([2] + [n for _, n in seqs])[:-1]
    ids, indptr = _lists([([7] * first, 0)] + seqs) if first else _lists(seqs)
    if first:
        indptr = indptr[1:].contiguous()
    outs = [torch.full((total + 5, H, D), 77.0, dtype=dtype, device="cuda") for _ in range(2)]
    err = _cuda([0])
    p = _params(D, H, len(pools[0]), dtype)
    halo.kvq_page_gather_kv(*[torch.from_numpy(x).cuda() for x in pools], p, ids, indptr, _cuda([n for _, n in seqs]),
                            _cuda(offs, torch.int64), *outs, err)
    for z in (K, V):
        exp = np.full((total + 5, H, D), 77.0)
        for (pages, n), off in zip(seqs, offs):
            if len(pages) != -(-n // 16):
                continue
            for t in range(n):
                if 0 <= pages[t // 16] < len(pools[0]):
                    for h in range(H):
                        exp[off + t, h] = paged_kvq.read_token(pools[z][pages[t // 16], h], z, D, t % 16)
        assert np.array_equal(outs[z].double().cpu().numpy(), exp, equal_nan=True), "KV"[z]
    return err.item()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,H", [(64, 3), (128, 2)])
@pytest.mark.parametrize("first", [0, 3])
def test_gather(gpu_lib, D, H, dtype, first):
    rng = np.random.default_rng(D)
    pools = _random_pools(D, H, 40, rng)
    pages = rng.permutation(40)
    seqs, at = [], 0
    for n in (1, 0, 16, 17, 40, 0, 95, 31):
        need = -(-n // 16)
        seqs.append((pages[at:at + need].tolist(), n))
        at += need
    assert _gather(D, H, pools, seqs, dtype, first) == 0


def test_gather_nan_scales_and_bad_lists(gpu_lib):
    rng = np.random.default_rng(9)
    D, pools = 128, _random_pools(128, 1, 6, np.random.default_rng(9))
    pools[0][2, 0, D * 8 + 5] = 255
    pools[1][2, 0, D * 8 + 6:D * 8 + 8] = [0xc0, 0x7f]
    assert _gather(D, 1, pools, [([2, 3], 20)], torch.bfloat16) == 0
    assert _gather(D, 1, pools, [([0], 17), ([1], 3)], torch.bfloat16) == 1
    assert _gather(D, 1, pools, [([0, 6], 17), ([1, -1, 2], 48)], torch.float32) == 1
    del rng


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_written_again_the_same(gpu_lib, D, dtype):
    """What a cache stands for is quantised to itself: written, read and
    written again, every byte of the written tokens is the same (and an
    append writes the bits that a chunk does)."""
    gen = torch.Generator(device="cuda").manual_seed(D)
    H, n = 4, 1000
    p = _params(D, H, 64, dtype)
    x = [torch.randn((n, H, D), generator=gen, device="cuda").to(dtype) for _ in range(2)]
    ids, indptr = _cuda(torch.randperm(64).numpy()), _cuda([0, 63])
    zero64 = _cuda([0], torch.int64)
    pools = halo.alloc_kvq_pools(p)
    halo.kvq_page_scatter_kv(*pools, p, ids, indptr, _cuda([0]), _cuda([n]), zero64, *x)
    out = [torch.empty_like(t) for t in x]
    halo.kvq_page_gather_kv(*pools, p, ids, _cuda([0, 63]), _cuda([n]), zero64, *out)
    again = halo.alloc_kvq_pools(p)
    halo.kvq_page_scatter_kv(*again, p, ids, indptr, _cuda([0]), _cuda([n]), zero64, *out)
    single = halo.alloc_kvq_pools(p)
    for t in range(0, 40):
        halo.kvq_page_scatter_kv(*single, p, ids, indptr, _cuda([t]), _cuda([1]), _cuda([t], torch.int64), *x)
    for a, b, c in zip(pools, again, single):
        assert torch.equal(a, b)
        assert torch.equal(a[ids[:2].long()], c[ids[:2].long()])


def test_page_copy(gpu_lib):
    rng = np.random.default_rng(1)
    for D in (64, 128):
        pools = _random_pools(D, 3, 12, rng)
        p = _params(D, 3, 12, torch.bfloat16)
        src, dst = [1, 1, 5, -1, 7], [2, 3, 11, 4, 12]
        for z in (K, V):
            dev, err = torch.from_numpy(pools[z]).cuda(), _cuda([0])
            halo.kvq_page_copy(dev, p, z, _cuda(src), _cuda(dst), err)
            want, flagged = paged_kv.page_copy(pools[z].reshape(-1), 3 * pools[z].shape[2], 12, src, dst)
            assert np.array_equal(dev.cpu().numpy().reshape(-1), want) and flagged and err.item() == 1
            again, lists = torch.from_numpy(pools[z]).cuda(), (_cuda(src), _cuda(dst))
            call = halo.bind_kvq_page_copy(again, p, z, *lists)
            call()
            assert torch.equal(again, dev)


def test_long_offsets(gpu_lib):
    """Pages past 4 GiB of a pool."""
    D, H = 128, 8
    n_pool = (5 << 30) // (H * 1056)
    p = _params(D, H, n_pool, torch.bfloat16)
    k, v = (torch.empty((n_pool, H, b), dtype=torch.uint8, device="cuda") for b in (1088, 1056))
    ids = _cuda([n_pool - 1, 3])
    x = [torch.randn((20, H, D), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    for t in (k, v):
        t[3].zero_(), t[n_pool - 1].zero_()
    args = (_cuda([0, 2]), _cuda([0]), _cuda([20]), _cuda([0], torch.int64))
    halo.kvq_page_scatter_kv(k, v, p, ids, *args, *x)
    out = [torch.empty_like(t) for t in x]
    halo.kvq_page_gather_kv(k, v, p, ids, args[0], _cuda([20]), args[3], *out)
    for z, pool in enumerate((k, v)):
        tiles = [pool[i].cpu().numpy() for i in (n_pool - 1, 3)]
        for t in (0, 15, 16, 19):
            for h in (0, 7):
                assert np.array_equal(out[z][t, h].double().cpu().numpy(),
                                      paged_kvq.read_token(tiles[t // 16][h], z, D, t % 16))
        # half a unit of the widest step and what the largest code cuts off
        top = x[z].float().abs().amax(-1, keepdim=True)
        assert ((out[z].float() - x[z].float()).abs() <= 2.0 / 7.0 * top).all()


def test_in_a_graph_and_on_a_stream(gpu_lib):
    """A captured write and read, replayed with new tokens."""
    D, H = 64, 2
    p = _params(D, H, 8, torch.bfloat16)
    pools, ref = halo.alloc_kvq_pools(p), halo.alloc_kvq_pools(p)
    ids, indptr, start, count = _cuda([5, 2, 0]), _cuda([0, 2, 3]), _cuda([14, 3]), _cuda([4, 1])
    off, total, out_off = _cuda([0, 4], torch.int64), _cuda([18, 4]), _cuda([0, 18], torch.int64)
    x = [torch.zeros((5, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out = [torch.zeros((22, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    want = [torch.zeros_like(t) for t in out]
    write = halo.bind_kvq_page_scatter_kv(*ref, p, ids, indptr, start, count, off, *x)
    read = halo.bind_kvq_page_gather_kv(*ref, p, ids, indptr, total, out_off, *want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        halo.kvq_page_scatter_kv(*pools, p, ids, indptr, start, count, off, *x)
        halo.kvq_page_gather_kv(*pools, p, ids, indptr, total, out_off, *out)
    for i in range(4):
        for t in x:
            t.copy_(torch.randn(t.shape, device="cuda"))
        graph.replay()
        write(), read()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*out, *pools), (*want, *ref)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    halo.kvq_page_gather_kv(*ref, p, ids, indptr, total, out_off, *out, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_largest_magnitudes(gpu_lib, dtype):
    """From 3.5 * 2^126 on a value is stored as 2^128: an infinity, where one below
    it is finite, and so are its neighbours."""
    p = _params(64, 1, 2, dtype)
    k, v = halo.alloc_kvq_pools(p)
    x = torch.zeros(2, 1, 64, dtype=dtype, device="cuda")
    x[0, 0, 5], x[0, 0, 6] = 2.0 ** 126 * 3.5, -2.0 ** 126
    x[1, 0, 5], x[1, 0, 6] = 2.0 ** 126 * 3.375, -2.0 ** 126
    lists = (_cuda([0]), _cuda([0, 1]))
    halo.kvq_page_scatter_kv(k, v, p, *lists, _cuda([0]), _cuda([2]), _cuda([0], torch.int64), x, x)
    out = [torch.empty_like(x) for _ in range(2)]
    halo.kvq_page_gather_kv(k, v, p, *lists, _cuda([2]), _cuda([0], torch.int64), *out)
    for o in out:
        assert o[0, 0, 5] == math.inf and o[1, 0, 5] == 2.0 ** 126 * 3 and (o[:, 0, 6] == -2.0 ** 126).all()
        assert (o[:, 0, 7:] == 0).all()
