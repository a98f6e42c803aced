"""Shared helpers of the tests of the operators between two steps: pools of
random bits and where tokens lie in them, read and written by the formats'
definitions."""

import functools

import numpy as np
import torch

import kvq_helpers
from oracle import paged_kv, paged_kvq
from paper_2509_02121_amd import halo

BF16, F32 = torch.bfloat16, torch.float32
PAGE = 16


def cuda(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x)).to(dtype).cuda()


def csr(lists):
    """(indptr, flat) of page lists, on the GPU."""
    indptr = np.cumsum([0] + [len(x) for x in lists])
    flat = np.concatenate([np.asarray(x, np.int32) for x in lists]) if lists else np.zeros(0, np.int32)
    return cuda(indptr), cuda(flat)


def params(hq, hkv, dim, dtype, pages, scale=None):
    return halo.make_params(hq, hkv, dim, dtype, pages, dim ** -0.5 if scale is None else scale)


@functools.cache
def _places(kind, D, elems):
    """Flat place of (token, dim) in a tile of a bf16 or fp32 pool."""
    return np.array([[paged_kv.elem_offset(kind, 1, D, elems, 0, 0, t, c) for c in range(D)] for t in range(PAGE)])


def tile_bytes(kind, D, dtype, kvq):
    return paged_kvq.tile_bytes(kind, D) if kvq else PAGE * D * dtype.itemsize


def random_pool(kind, pages, H, D, dtype, kvq, gen, scale=1.0):
    """A pool whose bytes read as finite numbers of about `scale`."""
    if not kvq:
        x = torch.randn((pages, H, PAGE * D), generator=gen, device="cuda") * scale
        return x.to(dtype)
    pool = torch.randint(0, 256, (pages, H, tile_bytes(kind, D, dtype, True)), generator=gen, device="cuda",
                         dtype=torch.uint8)
    if kind == paged_kv.POOL_K:
        e = torch.randint(123, 127, pool[:, :, D * 8:].shape, generator=gen, device="cuda")
        pool[:, :, D * 8:] = e.to(torch.uint8)
    else:
        e = torch.randint(123, 127, (pages, H, PAGE), generator=gen, device="cuda") << 7
        pool[:, :, D * 8:] = e.to(torch.int16).view(torch.uint8).view(pages, H, 2 * PAGE)
    return pool


def values(pool, kind, D, kvq):
    """[pages, 16, H, D] float64 of a pool (a numpy array: bf16 as float32)."""
    if kvq:
        return kvq_helpers.values(pool, kind, D)
    elems = 8 if pool.dtype == np.uint16 else 4
    x = pool[:, :, _places(kind, D, elems)]
    if x.dtype == np.uint16:
        x = (x.astype(np.uint32) << 16).view(np.float32)
    return x.astype(np.float64).transpose(0, 2, 1, 3)


def to_numpy(pool):
    """The pool's bits: uint16 (bf16), float32 or uint8."""
    x = pool.detach()
    return x.view(torch.int16).cpu().numpy().view(np.uint16) if x.dtype == BF16 else x.cpu().numpy()


@functools.cache
def _token_bits(kind, D, kvq, elems):
    """For each token of a tile, the indices of its pieces: (bytes or elements, their halves: -1 whole, 0 low, 1
    high) in one fixed order."""
    if not kvq:
        return [(p, np.full(D, -1)) for p in _places(kind, D, elems)]
    out = []
    for t in range(PAGE):
        n = np.array([paged_kvq.code_number(kind, D, t, c) for c in range(D)])
        if kind == paged_kv.POOL_K:
            s = D * 8 + t * (D // 32) + np.arange(D // 32)
        else:
            s = D * 8 + 2 * paged_kv.v_slot(t) + np.arange(2)
        out.append((np.concatenate([n // 2, s]), np.concatenate([n % 2, np.full(len(s), -1)])))
    return out


def read_bits(tile, t, kind, D, kvq):
    """Token t of a (page, head) tile as its pieces."""
    at, half = _token_bits(kind, D, kvq, 8 if tile.dtype == np.uint16 else 4)[t]
    x = tile[at]
    return np.where(half < 0, x, (x >> (4 * np.maximum(half, 0))) & 15).astype(x.dtype) if kvq else x.copy()


def write_bits(tile, t, bits, kind, D, kvq):
    at, half = _token_bits(kind, D, kvq, 8 if tile.dtype == np.uint16 else 4)[t]
    if not kvq:
        tile[at] = bits
        return
    for a, h, b in zip(at, half, bits):
        b = int(b)
        if h >= 0:
            b = (int(tile[a]) & 0x0f) | b << 4 if h else (int(tile[a]) & 0xf0) | b
        tile[a] = b
