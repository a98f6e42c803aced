"""Shared helpers of the tests of attention over 4-bit pools: a workload's
keys and values written into 4-bit pools, read back by the format's
definition, and a bound on the kernels' rounding for each output."""

import functools

import numpy as np
import torch

import oracle
from oracle import paged_kvq
from paper_2509_02121_amd import halo

U32 = 2.0 ** -24


@functools.cache
def _places(kind, D):
    """Code number of (token, dim), and the index of its scale."""
    n = np.array([[paged_kvq.code_number(kind, D, t, c) for c in range(D)] for t in range(16)])
    if kind == paged_kvq.POOL_K:
        s = np.array([[t * (D // 32) + c // 32 for c in range(D)] for t in range(16)])
    else:
        s = np.array([[oracle.paged_kv.v_slot(t)] * D for t in range(16)])
    return n, s


def values(tiles, kind, D):
    """[n, 16, H, D] float64 of tiles [n, H, bytes] (numpy)."""
    number, scale = _places(kind, D)
    code = (tiles[:, :, (number // 2).ravel()].reshape(*tiles.shape[:2], 16, D) >> (4 * (number % 2)).astype(np.uint8)) & 15
    mag = np.array(paged_kvq.MAGNITUDES)[code & 7] * np.where(code & 8, -1.0, 1.0)
    if kind == paged_kvq.POOL_K:
        e = tiles[:, :, D * 8:].astype(np.float64)
        with np.errstate(over="ignore"):
            unit = np.where(e == 255, np.nan, 2.0 ** (e - 127))
    else:
        unit = np.ascontiguousarray(tiles[:, :, D * 8:]).view(np.uint16).astype(np.uint32)
        with np.errstate(invalid="ignore"):
            unit = (unit << 16).view(np.float32).astype(np.float64)
    with np.errstate(invalid="ignore"):
        return (mag * unit[:, :, scale]).transpose(0, 2, 1, 3)


def fill_pools(w, seed=0, strong=None):
    """4-bit pools on the GPU that hold w's segments, every other byte random
    (scales of NaN and of any size among them)."""
    D, H, n = w.head_dim, w.num_kv_heads, w.num_pool_pages
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pools = [torch.randint(0, 256, (n, H, paged_kvq.tile_bytes(kind, D)), generator=gen, device="cuda", dtype=torch.uint8)
             for kind in (0, 1)]
    pools[0][:, :, D * 8:] |= (torch.rand(pools[0][:, :, D * 8:].shape, generator=gen, device="cuda") < 0.5) * 255
    src, lists, lens = [[], []], [], []
    for s in range(len(w.seg_len)):
        if w.seg_len[s]:
            for z, x in enumerate(w.segment_kv(s)):
                src[z].append(x.cuda())
            lists.append(np.asarray(w.seg_pages[s]))
            lens.append(int(w.seg_len[s]))
    if lists:
        def cuda(x, dtype=torch.int32):
            return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")
        src = [torch.cat(x) for x in src]
        if strong is not None:
            src[0] = (src[0].float() * strong.cuda()).to(src[0].dtype)
        params = halo.make_params(w.num_q_heads, H, D, w.dtype, n, w.scale, w.dtype)
        halo.kvq_page_scatter_kv(*pools, params, cuda(np.concatenate(lists)), cuda(np.cumsum([0] + [len(x) for x in lists])),
                                 cuda([0] * len(lens)), cuda(lens), cuda(np.cumsum([0] + lens[:-1]), torch.int64), *src)
    return pools


def expected(w, pools, q=None):
    """(o, lse, o bound per weight rounding, score bound) in 64 bits: for each
    output the average A of |v| under the row's weights, and for each row
    scale * sum |q| max |k|, which bounds every sum of products behind a score."""
    D = w.head_dim
    seg_k, seg_v, top = {}, {}, {}
    host = [p.cpu().numpy() for p in pools]
    for s in range(len(w.seg_len)):
        pages, n = np.asarray(w.seg_pages[s], np.int64), int(w.seg_len[s])
        seg_k[s], seg_v[s] = (values(host[z][pages], z, D).reshape(-1, w.num_kv_heads, D)[:n] for z in (0, 1))
        top[s] = np.abs(seg_k[s]).max(0) if n else np.zeros((w.num_kv_heads, D))
    qq = (w.q if q is None else q).double().cpu().numpy()
    ab = {s: np.abs(x) for s, x in seg_v.items()}
    if w.is_prefill:
        o, lse = oracle.prefill(qq, w.q_len, seg_k, seg_v, w.req_paths, w.scale)
        A, _ = oracle.prefill(qq, w.q_len, seg_k, ab, w.req_paths, w.scale)
        owner = np.repeat(np.arange(w.num_requests), w.q_len)
    else:
        o, lse = oracle.decode(qq, seg_k, seg_v, w.req_paths, w.scale)
        A, _ = oracle.decode(qq, seg_k, ab, w.req_paths, w.scale)
        owner = np.arange(w.num_requests)
    G = w.num_q_heads // w.num_kv_heads
    B = np.zeros(lse.shape)
    keys = np.zeros(len(owner))
    for r, path in enumerate(w.req_paths):
        at = owner == r
        if path:
            most = np.max([top[s] for s in path], 0).repeat(G, 0)
            B[at] = w.scale * (np.abs(qq[at]) * most).sum(-1)
        keys[at] = sum(int(w.seg_len[s]) for s in path)
    return o, lse, A, B, keys


def assert_close(w, out_dtype, o, lse, want, split, label=""):
    """Rounding of the kernels, worst case.

    Every term relative to A (weights are positive, so sums of weights times
    |v| bound sums of products): a weight is 2^x of an x off by the score's
    error, which is at most (D + 16) roundings of sums bounded by B (products,
    three parts for fp32, the scale, the maximum); exp2 and its argument 4 more;
    n roundings in a sum of n keys, in the numerator and in the denominator, 16
    for rescaling and merging. bf16 outputs: a weight is rounded to bf16 for P V
    (half a step, 2^-8), a partial result to fp16 (2^-11, or 2^-25 of the row's
    largest element, which is at most the largest A), and the output itself."""
    ro, rl, A, B, keys = want
    D = w.head_dim
    sums = U32 * ((D + 16) * B + 4 * (1 + B) + keys[:, None] + 16)
    coarse, floor = 0.0, 1e-30
    if out_dtype == torch.bfloat16:
        coarse = 2 * 2.0 ** -8 + (2.0 ** -11 if split else 0.0)
        floor += 2.0 ** -25 * A.max(-1, keepdims=True) if split else 0.0
    seen = np.isfinite(rl)
    assert np.isneginf(lse[~seen]).all() and (o[~seen] == 0).all(), f"{label}: rows without keys"
    tol = A * (coarse + 2 * 2 * sums[..., None]) + floor
    err = np.abs(o - ro)
    assert (err[seen] <= tol[seen]).all(), f"{label}: {np.nanmax(err[seen] / tol[seen]):.3f} of the bound, " \
                                           f"finite {np.isfinite(o).all()}"
    ltol = 2 * sums + 4 * U32 * np.where(seen, np.abs(rl), 0)
    lerr = np.abs(np.where(seen, lse - np.where(seen, rl, 0), 0))
    assert (lerr <= ltol + 1e-30).all(), f"{label}: lse {np.nanmax(lerr / (ltol + 1e-30)):.3f} of the bound"
    return float(np.nanmax(err[seen] / tol[seen])) if seen.any() else 0.0


def run(w, pools, out_dtype, options=None):
    """(o, lse) of PrefixAttention over the pools as float64 arrays, and it."""
    params = halo.make_params(w.num_q_heads, w.num_kv_heads, w.head_dim, w.dtype, w.num_pool_pages, w.scale, out_dtype)
    att = halo.PrefixAttention(params, w.forest_csr(), "cuda", options)
    w.q = w.q.cuda()
    o, lse = att.run(w.q, *pools)
    torch.cuda.synchronize()
    return o.double().cpu().numpy(), lse.double().cpu().numpy(), att


def check(w, out_dtype, options=None, label="", seed=0, strong=None):
    """The whole path against the oracle; returns the PrefixAttention."""
    pools = fill_pools(w, seed, strong)
    o, lse, att = run(w, pools, out_dtype, options)
    split = att.plan.stats()["num_merge_rows"] > 0
    share = assert_close(w, out_dtype, o, lse, expected(w, pools), split, label)
    print(f"{label}: {share:.3f} of the bound", flush=True)
    return att, pools
