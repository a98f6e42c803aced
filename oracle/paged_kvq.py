"""4-bit paged KV cache reference (TEST INFRASTRUCTURE ONLY).

The format in plain numpy, in 64 bits, one block and one code at a time:
E2M1 codes, a power of two as scale for each 32 dims of a token's K and for
each token's V of a head, and where a code lies in a tile of 16 tokens:
  * K: code (token t, dim c) is number
    ``((c % 32 // 8 * 16 + t) * (D // 32) + c // 32) * 8 + c % 8`` of the tile,
    the scale of dims ``32 s ..`` byte ``8 D + t * (D // 32) + s``;
  * V: number ``((((c // 64) * 2 + u // 8) * 16 + c % 16) * 4 + c // 16 % 4) * 8
    + u % 8`` with ``u`` the slot of token t (``paged_kv.v_slot``), the scale
    the bf16 at byte ``8 D + 2 u``;
code number n is the low (n even) or high half of byte ``n // 2``.
"""

import math

import numpy as np

from .paged_kv import PAGE, POOL_K, v_slot

MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def tile_bytes(kind, head_dim):
    return head_dim * 8 + (head_dim // 2 if kind == POOL_K else 32)


def scale_exponent(block):
    """The exponent of a block's scale (None: NaN)."""
    top = max(abs(float(x)) for x in block)
    if any(not math.isfinite(float(x)) for x in block):
        return None
    if top == 0:
        return -126
    m, e = math.frexp(top)          # top = m 2^e, m in [0.5, 1)
    if m >= 0.875:                  # two significant bits: to the next power of two
        e += 1
    return max(e - 3, -126)


def nearest_code(y):
    """The code of the nearest magnitude to y, ties to the even code."""
    sign = 8 if math.copysign(1.0, y) < 0 else 0
    best = min(range(8), key=lambda c: (abs(MAGNITUDES[c] - min(abs(y), 6.0)), c % 2))
    return sign + best


def code_number(kind, head_dim, t, c):
    if kind == POOL_K:
        return ((c % 32 // 8 * 16 + t) * (head_dim // 32) + c // 32) * 8 + c % 8
    u = v_slot(t)
    return ((((c // 64) * 2 + u // 8) * 16 + c % 16) * 4 + c // 16 % 4) * 8 + u % 8


def write_token(tile, kind, head_dim, t, values):
    """Quantise one token (head_dim values) into slot t of a tile (bytes)."""
    block = 32 if kind == POOL_K else head_dim
    for s in range(head_dim // block):
        part = values[s * block:(s + 1) * block]
        e = scale_exponent(part)
        if kind == POOL_K:
            tile[head_dim * 8 + t * (head_dim // 32) + s] = 255 if e is None else e + 127
        else:
            bits = 0x7fc0 if e is None else (e + 127) << 7
            at = head_dim * 8 + 2 * v_slot(t)
            tile[at], tile[at + 1] = bits & 0xff, bits >> 8
        for i, x in enumerate(part):
            code = 0 if e is None else nearest_code(float(x) * 2.0 ** -e)
            n = code_number(kind, head_dim, t, s * block + i)
            byte = int(tile[n // 2])
            tile[n // 2] = (byte & 0x0f) | (code << 4) if n % 2 else (byte & 0xf0) | code


def read_token(tile, kind, head_dim, t):
    """The values (float64) of slot t of a tile."""
    out = np.empty(head_dim)
    for c in range(head_dim):
        n = code_number(kind, head_dim, t, c)
        code = (int(tile[n // 2]) >> (4 * (n % 2))) & 15
        value = MAGNITUDES[code & 7] * (-1 if code & 8 else 1)
        if kind == POOL_K:
            e = int(tile[head_dim * 8 + t * (head_dim // 32) + c // 32])
            out[c] = math.nan if e == 255 else value * 2.0 ** (e - 127)
        else:
            at = head_dim * 8 + 2 * v_slot(t)
            bits = np.uint32(int(tile[at]) | int(tile[at + 1]) << 8) << np.uint32(16)
            out[c] = value * float(np.uint32(bits).view(np.float32))
    return out


def scatter(pool, kind, head_dim, page_lists, starts, counts, in_offsets, src):
    """The pool ([pages, H, tile bytes] uint8) after writing tokens start ..
    start + count - 1 of each sequence from rows in_offsets[i] .. of src
    [T, H, D]; sequences and pages that do not fit are skipped. Returns
    (pool, flagged)."""
    out = pool.copy()
    flagged = False
    for pages, start, count, off in zip(page_lists, starts, counts, in_offsets):
        if count <= 0:
            continue
        if start < 0 or start + count > PAGE * len(pages):
            flagged = True
            continue
        for i in range(count):
            page = int(pages[(start + i) // PAGE])
            if not 0 <= page < len(pool):
                flagged = True
                continue
            for h in range(pool.shape[1]):
                write_token(out[page, h], kind, head_dim, (start + i) % PAGE, src[off + i, h])
    return out, flagged
