"""The operators around a 4-bit KV cache, as a serving step calls them.

A case is a dict of plain values. ``listed()`` holds the named ones, ``draw(rng)`` makes another one of the same
ranges, and for a case

  prepare(case, seed)  what a program holds before the call: inputs, pools, page lists, the plan (from the seed);
  run(state)           one pass: with ``own`` the framework's operators, without it elementary torch operations;
  work(case)           the bytes and flops that one pass cannot do without;
  exact(case, seed)    the outputs from the definition, in 64 bits.

Kinds: "tables" (page lists, slots and positions of a step from lengths on the GPU), "rope" (queries and keys turned
by their positions), "write" (new tokens into the 4-bit pages, then the sequences' tokens read back), "decode" and
"prefill" (attention over the 4-bit cache of a prefix forest).

The 4-bit cache. Codes are E2M1 (sign, and a magnitude of 0, 0.5, 1, 1.5, 2, 3, 4 or 6). A token's key has a power of
two as scale for each 32 dims of a head, held as its biased exponent in a byte (255: NaN); a token's value has one for
the head, held in bf16. The scale's exponent is that of the largest magnitude, rounded to two significant bits, less
two. Pages of 16 tokens are [head][tile]; a tile is D * 8 bytes of codes, then the scales of its 16 tokens:
  K codes  [g: 4][token: 16][s: D/32][i: 8]           dim 32 s + 8 g + i
  K scales [token: 16][s: D/32]
  V codes  [bq: D/64][h: 2][c: 16][b: 4][j: 8]        dim 16 (4 bq + b) + c, token slot 8 h + j
  V scales [slot: 16]
with the slots of a V tile in the token order 0-3, 8-11, 4-7, 12-15 and two codes to a byte, the first one low.
"""

import functools
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
# token in slot s of a V tile (and slot of token s: the map is its own inverse)
SLOTS = [0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15]
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
ROPE_BASE = 500000.0
ORIGINAL_POSITIONS = 8192


# ------------------------------------------------------------------- cases

def _tables(name=None, *, sequences, length, new=(1, 1), chunks=0, chunk=(1, 1), spare=0):
    """`chunks` of the sequences take a prompt chunk, the others a few tokens;
    `spare`: padding tokens behind the step's last (a captured step's)."""
    case = {"kind": "tables", "sequences": sequences, "length_lo": length[0], "length_hi": length[1],
            "new_lo": new[0], "new_hi": new[1], "chunks": chunks, "chunk_lo": chunk[0], "chunk_hi": chunk[1],
            "spare": spare}
    return {**case, "name": name} if name else case


def _rope(name=None, *, tokens, heads=(32, 8), dim=128, rotary=128, interleaved=False, dtype="bf16", scaling="none",
          factor=1.0, span=4096, fused=True):
    """`tokens` tokens at positions below `span`; fused: q and k are parts of
    one projection's rows."""
    case = {"kind": "rope", "tokens": tokens, "q_heads": heads[0], "kv_heads": heads[1], "head_dim": dim,
            "rotary": rotary, "interleaved": interleaved, "dtype": dtype, "scaling": scaling, "factor": factor,
            "span": span, "fused": fused}
    return {**case, "name": name} if name else case


def _write(name=None, *, sequences, length, chunks=0, chunk=(1, 1), heads=8, dim=128, dtype="bf16"):
    """Sequences with cached tokens: `chunks` of them write a chunk, the
    others one token; then all are read back."""
    case = {"kind": "write", "sequences": sequences, "length_lo": length[0], "length_hi": length[1],
            "chunks": chunks, "chunk_lo": chunk[0], "chunk_hi": chunk[1], "kv_heads": heads, "head_dim": dim,
            "dtype": dtype}
    return {**case, "name": name} if name else case


def _attention(kind, name=None, *, requests, groups=1, root=0, prefix=0, private=(0, 0), chunk=(0, 0), heads=(32, 8),
               dim=128, dtype="bf16", out=None):
    """A forest: an optional root shared by all, `groups` prefixes shared by
    runs of requests, a private segment each and, for a prefill, a chunk."""
    case = {"kind": kind, "requests": requests, "groups": groups, "root": root, "prefix": prefix,
            "private_lo": private[0], "private_hi": private[1], "chunk_lo": chunk[0], "chunk_hi": chunk[1],
            "q_heads": heads[0], "kv_heads": heads[1], "head_dim": dim, "dtype": dtype, "out": out or dtype}
    return {**case, "name": name} if name else case


def listed():
    return [
        # One decode step of 64 workflows: a token each, latency only.
        _tables("tables_step", sequences=64, length=(64, 2560)),
        # A full batch: most sequences append, 32 bring a chunk, with the
        # padding of a captured step. Page lists of long histories.
        _tables("tables_mixed", sequences=1024, length=(256, 10240), new=(0, 2), chunks=32, chunk=(64, 512), spare=1000),
        # Queries and keys of one decode step, out of a fused projection.
        _rope("rope_step", tokens=64, scaling="bands", factor=8.0, span=131072),
        # A prompt batch: 16384 tokens, neighbouring pairs, half of each head.
        _rope("rope_prompt", tokens=16384, rotary=64, interleaved=True, scaling="yarn", factor=4.0, span=16384),
        # A mixed step's cache writes into 4 bits, read back by a consumer of
        # dense tokens (ragged, small).
        _write("kv4_write_mixed", sequences=64, length=(16, 256), chunks=4, chunk=(64, 512)),
        # 32 prompt chunks written and read back: the copy-bound end.
        _write("kv4_write_prompt", sequences=32, length=(1, 100), chunks=32, chunk=(512, 1024)),
        # A handful of agents on a short prompt: launches and latency.
        _attention("decode", "decode_tiny", requests=8, prefix=256, private=(16, 64), heads=(4, 4), dim=64, out="fp32"),
        # One layer of an 8B-shaped model: 64 workflows on a 2048-token prompt.
        _attention("decode", "decode_8b", requests=64, prefix=2048, private=(64, 512)),
        # A 70B-shaped layer at full batch, the largest call.
        _attention("decode", "decode_70b", requests=1024, groups=8, prefix=8192, private=(256, 2048), heads=(64, 8)),
        # A few long conversations in fp32: keys split over the whole chip.
        _attention("decode", "decode_long_fp32", requests=4, private=(12000, 24000), dtype="fp32"),
        # Chunked prefill at full batch over a cached prompt.
        _attention("prefill", "prefill_chunked", requests=32, prefix=4096, chunk=(512, 512)),
        # Short ragged continuations over a shared prompt and a history.
        _attention("prefill", "prefill_short", requests=16, prefix=2048, private=(100, 1000), chunk=(16, 128)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _range(rng, lo, hi):
    a, b = sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))
    return a, b


def _draw_once(rng):
    kind = rng.choice(["tables", "rope", "write", "decode", "decode", "decode", "prefill", "prefill"])
    dim = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    heads = rng.choice([(4, 4), (16, 16), (32, 8), (32, 8), (64, 8), (16, 1)])
    if kind == "tables":
        n = _log_int(rng, 1, 2048)
        return _tables(sequences=n, length=_range(rng, 1, 12000), new=(rng.randint(0, 1), rng.randint(1, 3)),
                       chunks=min(n, rng.choice([0, rng.randint(0, 32)])), chunk=_range(rng, 2, 1024),
                       spare=rng.choice([0, rng.randint(1, 1000)]))
    if kind == "rope":
        scaling = rng.choice(["none", "linear", "ntk", "yarn", "bands"])
        return _rope(tokens=_log_int(rng, 1, 16384), heads=heads, dim=dim, rotary=rng.choice([dim, dim, dim // 2, 16]),
                     interleaved=rng.random() < 0.5, dtype=dtype, scaling=scaling,
                     factor=1.0 if scaling == "none" else float(rng.choice([2, 4, 8, 40])),
                     span=_log_int(rng, 100, 1000000), fused=rng.random() < 0.7)
    if kind == "write":
        n = _log_int(rng, 1, 512)
        return _write(sequences=n, length=_range(rng, 1, 500), chunks=min(n, rng.choice([0, rng.randint(0, 32)])),
                      chunk=_range(rng, 2, 1024), heads=rng.choice([1, 4, 8]), dim=dim, dtype=dtype)
    out = "fp32" if dtype == "fp32" or rng.random() < 0.25 else dtype
    requests = _log_int(rng, 1, {"decode": 1024, "prefill": 32}[kind])
    prefix = rng.choice([0, _log_int(rng, 16, 8192)])
    root = rng.choice([0, 0, _log_int(rng, 16, 2048)])
    rest = {"requests": requests, "groups": _log_int(rng, 1, max(1, requests // 2)), "root": root, "prefix": prefix,
            "heads": heads, "dim": dim, "dtype": dtype, "out": out}
    if kind == "prefill":
        return _attention(kind, private=rng.choice([(0, 0), _range(rng, 1, 5000)]), chunk=_range(rng, 1, 1024), **rest)
    return _attention(kind, private=_range(rng, 1, 24000), **rest)


def draw(rng):
    """One more case of these ranges, no more costly than the largest listed ones."""
    top = {c["name"]: work(c) for c in listed()}
    while True:
        case = _draw_once(rng)
        w = work(case)
        if case["kind"] in ("decode", "prefill"):
            # (fp32: three products for one)
            share = 4 if case["dtype"] == "fp32" else 1
            if w["bytes"] <= top["decode_70b"]["bytes"] and w["flops"] * share <= top["prefill_chunked"]["flops"]:
                return case
        else:
            largest = {"tables": "tables_mixed", "rope": "rope_prompt", "write": "kv4_write_prompt"}[case["kind"]]
            if w["bytes"] <= top[largest]["bytes"]:
                return case


# ------------------------------------------------------------------- sizes

def _lengths(case, lo, hi, n, what):
    """n lengths in [lo, hi], the same for every seed of one case."""
    rng = random.Random(what + repr(sorted((k, v) for k, v in case.items() if k != "name")))
    return [rng.randint(lo, hi) for _ in range(n)]


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _sequences(case):
    """(cached tokens, new tokens) of each sequence of a table or write case."""
    n = case["sequences"]
    length = _lengths(case, case["length_lo"], case["length_hi"], n, "length")
    new = _lengths(case, case.get("new_lo", 1), case.get("new_hi", 1), n, "new")
    for i, c in enumerate(_lengths(case, case["chunk_lo"], case["chunk_hi"], case["chunks"], "chunk")):
        new[i * n // case["chunks"]] = c
    return length, new


def _forest(case):
    """(segment lengths, paths, chunk lengths or None)."""
    R = case["requests"]
    seg, paths = [], [[] for _ in range(R)]
    if case["root"]:
        seg.append(case["root"])
        for p in paths:
            p.append(0)
    if case["prefix"]:
        first = len(seg)
        seg += [case["prefix"]] * case["groups"]
        for r, p in enumerate(paths):
            p.append(first + r * case["groups"] // R)
    own_len, chunk = None, None
    if case["private_hi"]:
        own_len = _lengths(case, case["private_lo"], case["private_hi"], R, "private")
    if case["kind"] == "prefill":
        chunk = _lengths(case, case["chunk_lo"], case["chunk_hi"], R, "chunk")
    for lens in (own_len, chunk):
        for p, n in zip(paths, lens or []):
            p.append(len(seg))
            seg.append(n)
    return seg, paths, chunk


def _csr(lists):
    indptr = np.zeros(len(lists) + 1, dtype=np.int32)
    indptr[1:] = np.cumsum([len(x) for x in lists])
    flat = np.concatenate([np.asarray(x, dtype=np.int32) for x in lists]) if lists else np.zeros(0, np.int32)
    return indptr, flat.astype(np.int32)


def _place(page_counts, seed, spare=1.25):
    """Page ids of each list, at random in a pool a quarter larger."""
    need = sum(page_counts)
    size = max(1, math.ceil(need * spare))
    ids = np.random.default_rng(seed).permutation(size)[:need].astype(np.int32)
    cuts = np.cumsum([0] + list(page_counts))
    return [ids[a:b] for a, b in zip(cuts[:-1], cuts[1:])], size


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _cuda(values, dtype=torch.int32):
    return torch.tensor(np.asarray(values), dtype=dtype, device="cuda")


def _tile_bytes(dim):
    """Bytes of a (page, head) tile: (K, V)."""
    return dim * 8 + dim // 2, dim * 8 + 32


# ------------------------------------------------------------------- the 4-bit format in torch

def _exponent(amax):
    """Biased exponent of the scale: that of amax rounded to two significant bits, less two."""
    e = ((amax.view(torch.int32) + 0x200000) >> 23) - 2
    return torch.where(torch.isfinite(amax), e.clamp(1, 254), torch.full_like(e, 255))


def _code(y):
    """E2M1 code of y, ties to the even code, up to 6."""
    a = y.abs()
    c = (a > 0.25).to(torch.uint8)
    for bound, at in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        c += (a >= bound) if at else (a > bound)
    return c | (torch.signbit(y).to(torch.uint8) << 3)


def _quantise(x, block):
    """(codes uint8 of x's shape, biased exponents [..., D / block]) of [..., D]."""
    x = x.float()
    b = x.view(*x.shape[:-1], x.shape[-1] // block, block)
    e = _exponent(b.abs().amax(-1))
    inverse = ((254 - e) << 23).view(torch.float32)   # 2 ** (127 - e)
    y = b * inverse[..., None]
    c = torch.where(e[..., None] == 255, 0, _code(y))
    return c.view(x.shape), e


def _pack(codes):
    """Two codes to a byte along the last axis, the first one low."""
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _k_tiles(codes, e):
    """K tiles [n, H, bytes] of codes [n, 16, H, D], exponents [n, 16, H, D/32]."""
    n, _, h, d = codes.shape
    c = codes.view(n, 16, h, d // 32, 4, 8).permute(0, 2, 4, 1, 3, 5).reshape(n, h, d * 16)
    return torch.cat([_pack(c), e.permute(0, 2, 1, 3).reshape(n, h, d // 2).to(torch.uint8)], -1)


def _v_bits(e):
    """The V scales' bf16 bits of biased exponents (255: NaN)."""
    return torch.where(e == 255, 0x7fc0, e << 7).to(torch.int16)


def _v_tiles(codes, e):
    """V tiles of codes [n, 16, H, D] and exponents [n, 16, H]."""
    n, _, h, d = codes.shape
    c = codes[:, _slots()].view(n, 2, 8, h, d // 64, 4, 16).permute(0, 3, 4, 1, 6, 5, 2).reshape(n, h, d * 16)
    s = _v_bits(e[:, _slots()]).permute(0, 2, 1).contiguous().view(torch.uint8)
    return torch.cat([_pack(c), s], -1)


def _v_codes(tiles, d):
    """Codes [n, 16 slots, H, D] of V tiles [n, H, bytes]."""
    n, h = tiles.shape[:2]
    c = _unpack(tiles[:, :, :d * 8]).view(n, h, d // 64, 2, 16, 4, 8)
    return c.permute(0, 3, 6, 1, 2, 5, 4).reshape(n, 16, h, d)


@functools.cache
def _slots():
    return torch.tensor(SLOTS, device="cuda")


@functools.cache
def _lut(dtype=torch.float32):
    return torch.tensor(E2M1 + [-x for x in E2M1], dtype=dtype, device="cuda")


@functools.cache
def _scale_lut(dtype=torch.float32):
    return torch.tensor([2.0 ** (e - 127) for e in range(255)] + [math.nan], dtype=dtype, device="cuda")


def _k_values(tiles, d):
    """Values [n, 16, H, D] of K tiles [n, H, bytes], in 32 bits."""
    n, h = tiles.shape[:2]
    c = _unpack(tiles[:, :, :d * 8]).view(n, h, 4, 16, d // 32, 8)
    x = _lut()[c.int()] * _scale_lut()[tiles[:, :, d * 8:].int()].view(n, h, 1, 16, d // 32, 1)
    return x.permute(0, 3, 1, 4, 2, 5).reshape(n, 16, h, d)


def _v_values(tiles, d):
    """Values [n, 16, H, D] of V tiles, in 32 bits."""
    s = tiles[:, :, d * 8:].contiguous().view(torch.bfloat16).float()   # [n, H, slots]
    return (_lut()[_v_codes(tiles, d).int()] * s.permute(0, 2, 1)[..., None])[:, _slots()]


def _pools(case, size, gen):
    """4-bit pools of normal keys and values; the keys have a few strong dims,
    as trained models' keys have."""
    h, d = case["kv_heads"], case["head_dim"]
    kb, vb = _tile_bytes(d)
    k = torch.empty((size, h, kb), dtype=torch.uint8, device="cuda")
    v = torch.empty((size, h, vb), dtype=torch.uint8, device="cuda")
    strong = torch.ones(d, device="cuda")
    strong[::29] = 4.0
    step = max(1, (1 << 25) // (16 * h * d))
    for a in range(0, size, step):
        n = min(step, size - a)
        x = torch.randn((n, 16, h, d), generator=gen, device="cuda")
        c, e = _quantise(x * strong, 32)
        k[a:a + n] = _k_tiles(c, e)
        c, e = _quantise(torch.randn((n, 16, h, d), generator=gen, device="cuda"), d)
        v[a:a + n] = _v_tiles(c, e[..., 0])
    return k, v


# ------------------------------------------------------------------- prepare

def _inputs(case, seed):
    """Everything but the framework's own objects."""
    gen = _generator(seed)
    if case["kind"] == "tables":
        length, new = _sequences(case)
        have = [_pages(a) for a in length]
        need = [_pages(a + b) for a, b in zip(length, new)]
        used = sum(n - h for n, h in zip(need, have))
        first, spare = seed % 7, 5 + seed % 11   # entries used up before, and left after the step
        pages, _ = _place(have + [first + used + spare], seed)
        width = max(need) + 3
        table = np.full((len(have), width), -1, np.int32)
        for row, p in zip(table, pages):
            row[:len(p)] = p
        return {"seq_len": _cuda(length), "seq_new": _cuda(new), "block_table": _cuda(table),
                "free_pages": _cuda(pages[-1]), "free_next": _cuda([first]),
                "max_tokens": sum(new) + case["spare"], "max_pages": sum(need) + 17}
    if case["kind"] == "rope":
        T, hq, hk, d = case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
        dt = DTYPES[case["dtype"]]
        if case["fused"]:
            rows = torch.randn((T, (hq + 2 * hk) * d), generator=gen, device="cuda").to(dt)
            q, k = rows[:, :hq * d].view(T, hq, d), rows[:, hq * d:(hq + hk) * d].view(T, hk, d)
        else:
            q = torch.randn((T, hq, d), generator=gen, device="cuda").to(dt)
            k = torch.randn((T, hk, d), generator=gen, device="cuda").to(dt)
        pos = torch.randint(0, case["span"], (T,), generator=gen, device="cuda", dtype=torch.int32)
        return {"q": q, "k": k, "pos": pos}
    if case["kind"] == "write":
        length, new = _sequences(case)
        pages, size = _place([_pages(a + b) for a, b in zip(length, new)], seed)
        k, v = _pools(case, size, gen)
        shape = (sum(new), case["kv_heads"], case["head_dim"])
        kn, vn = (torch.randn(shape, generator=gen, device="cuda").to(DTYPES[case["dtype"]]) for _ in range(2))
        indptr, ids = _csr(pages)
        return {"length": length, "new": new, "pages": pages, "size": size, "k": k, "v": v, "k_new": kn, "v_new": vn,
                "indptr": _cuda(indptr), "ids": _cuda(ids), "start": _cuda(length), "count": _cuda(new),
                "in_offset": _cuda(np.cumsum([0] + new[:-1]), torch.int64),
                "total": _cuda([a + b for a, b in zip(length, new)]),
                "out_offset": _cuda(np.cumsum([0] + [a + b for a, b in zip(length, new)][:-1]), torch.int64)}
    seg, paths, chunk = _forest(case)
    pages, size = _place([_pages(n) for n in seg], seed)
    k, v = _pools(case, size, gen)
    rows = sum(chunk) if chunk else case["requests"]
    # scores of standard deviation about 2: a few keys carry most of a row
    q = torch.randn((rows, case["q_heads"], case["head_dim"]), generator=gen, device="cuda") * 1.5
    return {"seg": seg, "paths": paths, "chunk": chunk, "pages": pages, "size": size, "k": k, "v": v,
            "q": q.to(DTYPES[case["dtype"]])}


def _params(case, size):
    from paper_2509_02121_amd import halo
    return halo.make_params(case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["head_dim"],
                            DTYPES[case["dtype"]], size, case["head_dim"] ** -0.5, DTYPES[case.get("out", case["dtype"])])


def prepare(case, seed):
    x = _inputs(case, seed)
    return _prepare_own(case, x) if own else _prepare_plain(case, x)


def _prepare_own(case, x):
    """A step's calls are bound once to their buffers and made every step."""
    from paper_2509_02121_amd import halo
    halo.load_library(require_gpu=True)
    state = {"x": x}
    if case["kind"] == "tables":
        t = state["tables"] = halo.StepTables(case["sequences"], x["max_tokens"], x["max_pages"])
        t.page_ids.fill_(-1)
        state["calls"] = [halo.bind_kv_step_tables(t, x["seq_len"], x["seq_new"], x["block_table"], x["free_pages"],
                                                   x["free_next"])]
        state["out"] = (x["block_table"], t.seq_page_indptr, t.page_ids, t.seq_start, t.seq_count, t.seq_end,
                        t.in_token_offset, t.positions, t.slots, t.free_next)
    elif case["kind"] == "rope":
        rope = state["rope"] = halo.Rope(case["head_dim"], case["rotary"], base=ROPE_BASE,
                                         interleaved=case["interleaved"], scaling=case["scaling"],
                                         factor=case["factor"], original_positions=ORIGINAL_POSITIONS)
        state["out"] = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in (x["q"], x["k"])]
        state["calls"] = [halo.bind_rope_qk(x["q"], x["k"], x["pos"], rope, *state["out"])]
    elif case["kind"] == "write":
        p = state["params"] = _params(case, x["size"])
        shape = (sum(x["length"]) + sum(x["new"]), case["kv_heads"], case["head_dim"])
        state["out"] = [torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda") for _ in range(2)]
        state["calls"] = [halo.bind_kv4_page_scatter_kv(x["k"], x["v"], p, x["ids"], x["indptr"], x["start"],
                                                        x["count"], x["in_offset"], x["k_new"], x["v_new"]),
                          halo.bind_kv4_page_gather_kv(x["k"], x["v"], p, x["ids"], x["indptr"], x["total"],
                                                       x["out_offset"], *state["out"])]
    else:
        page_indptr, page_ids = _csr(x["pages"])
        req_indptr, req_ids = _csr(x["paths"])
        csr = {"seg_len": np.asarray(x["seg"], np.int32), "seg_page_indptr": page_indptr, "seg_page_ids": page_ids,
               "req_seg_indptr": req_indptr, "req_seg_ids": req_ids,
               "q_len": None if x["chunk"] is None else np.asarray(x["chunk"], np.int32)}
        att = state["att"] = halo.PrefixAttention(_params(case, x["size"]), csr, "cuda")
        state["out"] = att.alloc_outputs(x["q"])
        state["calls"] = [att.bind(x["q"], x["k"], x["v"], *state["out"])]
    return state


def _prepare_plain(case, x):
    state = {"case": case, "x": x}
    if case["kind"] == "rope":
        freq, state["amplitude"] = _rope_frequencies(case)
        state["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
    elif case["kind"] == "write":
        # where each new token goes and each token lies
        page, slot, touched, index = [], [], {}, []
        for p, a, n in zip(x["pages"], x["length"], x["new"]):
            for t in range(a, a + n):
                page.append(int(p[t // PAGE]))
                slot.append(t % PAGE)
                index.append(touched.setdefault(page[-1], len(touched)))
        state["page"], state["slot"] = _cuda(page, torch.int64), _cuda(slot, torch.int64)
        state["touched"], state["index"] = _cuda(list(touched), torch.int64), _cuda(index, torch.int64)
        ends = [a + n for a, n in zip(x["length"], x["new"])]
        pages, at = np.unique(np.concatenate([np.repeat(p, PAGE)[:n] for p, n in zip(x["pages"], ends)]),
                              return_inverse=True)
        state["all"], state["all_at"] = _cuda(pages, torch.int64), _cuda(at.reshape(-1), torch.int64)
        state["all_slot"] = _cuda(np.concatenate([np.arange(n) % PAGE for n in ends]), torch.int64)
    elif case["kind"] != "tables":
        state["ids"] = [_cuda(p, torch.int64) for p in x["pages"]]
        state["groups"] = _groups(x)
    return state


def _groups(x):
    """For each segment the requests whose paths hold it and their query rows."""
    chunk = x["chunk"] or [1] * len(x["paths"])
    first = np.cumsum([0] + chunk)
    users = [[] for _ in x["seg"]]
    for r, p in enumerate(x["paths"]):
        for s in p:
            users[s].append(r)
    rows = [_cuda(np.concatenate([np.arange(first[r], first[r + 1]) for r in u]) if u else [], torch.int64) for u in users]
    causal = [bool(x["chunk"]) and bool(u) and s == x["paths"][u[0]][-1] for s, u in enumerate(users)]
    return rows, causal


# ------------------------------------------------------------------- run

def run(state):
    if own:
        for call in state["calls"]:
            call()
        return state["out"]
    plain = {"tables": _plain_tables, "rope": _plain_rope, "write": _plain_write, "decode": _plain_attention,
             "prefill": _plain_attention}
    return plain[state["case"]["kind"]](state)


def _plain_tables(state):
    x = state["x"]
    start, new = x["seq_len"], x["seq_new"]
    end = start + new
    have, need = (start + 15) // 16, (end + 15) // 16
    indptr = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), need.cumsum(0, dtype=torch.int32)])
    taken = (need - have).cumsum(0)
    first = x["free_next"].long() + taken - (need - have)   # of each sequence's new pages in the free list
    col = torch.arange(x["block_table"].shape[1], device="cuda")
    fresh = (col >= have[:, None]) & (col < need[:, None])
    source = (first[:, None] + col - have[:, None]).clamp(0, x["free_pages"].numel() - 1)
    table = torch.where(fresh, x["free_pages"][source], x["block_table"])
    # one place behind the end takes what is not listed
    pages = torch.full((x["max_pages"] + 1,), -1, dtype=torch.int32, device="cuda")
    at = torch.where(col < need[:, None], indptr[:-1, None] + col, x["max_pages"])
    pages[at.long()] = torch.where(col < need[:, None], table, -1)
    offset = new.cumsum(0, dtype=torch.int64) - new
    token = torch.arange(x["max_tokens"], device="cuda")
    seq = torch.searchsorted(offset + new, token, right=True)
    inside = seq < start.numel()
    seq = seq.clamp(max=start.numel() - 1)
    pos = torch.where(inside, start[seq] + token - offset[seq], 0)
    slot = torch.where(inside, table[seq, pos // 16].long() * 16 + pos % 16, -1)
    free = x["free_next"] + taken[-1:].to(torch.int32)
    return (table, indptr, pages[:-1], start.clone(), new.clone(), end, offset, pos.to(torch.int32), slot, free)


def _rope_frequencies(case):
    """Angle of each pair per position, and the factor on the rotated values
    (in 64 bits; once per model)."""
    R, f, orig = case["rotary"], case["factor"], ORIGINAL_POSITIONS
    base = ROPE_BASE
    if case["scaling"] == "ntk":
        base *= f ** (R / (R - 2))
    freq = [base ** (-2.0 * i / R) for i in range(R // 2)]
    if case["scaling"] == "linear":
        freq = [w / f for w in freq]
    if case["scaling"] == "yarn":
        # pairs of more than 32 turns over the original positions stay, those
        # of fewer than one are slowed, between them a ramp over the index
        def index(turns):
            return R * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(index(32.0)), 0), min(math.ceil(index(1.0)), R - 1)
        span = hi - lo if hi > lo else 0.001
        ramp = [min(1.0, max(0.0, (i - lo) / span)) for i in range(R // 2)]
        freq = [w * (1 - r) + w / f * r for w, r in zip(freq, ramp)]
        return freq, 0.1 * math.log(f) + 1.0 if f > 1 else 1.0
    if case["scaling"] == "bands":
        # by turns over the original positions: more than 4 stay, fewer than 1
        # are slowed, between them a ramp over the turns
        def band(w):
            keep = min(1.0, max(0.0, (orig * w / (2 * math.pi) - 1.0) / 3.0))
            return w * keep + w / f * (1 - keep)
        freq = [band(w) for w in freq]
    return freq, 1.0


def _plain_rope(state):
    x, case = state["x"], state["case"]
    angle = x["pos"].double()[:, None] * state["freq"]
    cos, sin = ((t * state["amplitude"]).float()[:, None] for t in (angle.cos(), angle.sin()))
    R, out = case["rotary"], []
    for t in (x["q"], x["k"]):
        v = t.float()
        if case["interleaved"]:
            a, b = v[..., 0:R:2], v[..., 1:R:2]
        else:
            a, b = v[..., :R // 2], v[..., R // 2:R]
        y = [a * cos - b * sin, a * sin + b * cos]
        y = torch.stack(y, -1).flatten(-2) if case["interleaved"] else torch.cat(y, -1)
        out.append(torch.cat([y, v[..., R:]], -1).to(t.dtype))
    return out


def _plain_write(state):
    x, d = state["x"], state["case"]["head_dim"]
    T, h = x["k_new"].shape[:2]
    c, e = _quantise(x["k_new"], 32)
    codes = x["k"][:, :, :d * 8].view(-1, h, 4, 16, d // 32, 4)
    packed = _pack(c.view(T, h, d // 32, 4, 8).permute(0, 1, 3, 2, 4))
    codes[state["page"], :, :, state["slot"]] = packed
    scales = x["k"][:, :, d * 8:].view(-1, h, 16, d // 32)
    scales[state["page"], :, state["slot"]] = e.to(torch.uint8)
    c, e = _quantise(x["v_new"], d)
    old = x["v"][state["touched"]]
    at = _slots()[state["slot"]]
    all_codes = _v_codes(old, d)
    all_codes[state["index"], at] = c
    bits = old[:, :, d * 8:].contiguous().view(torch.int16)
    bits[state["index"], :, at] = _v_bits(e[..., 0])
    n = all_codes.shape[0]
    packed = _pack(all_codes.view(n, 2, 8, h, d // 64, 4, 16).permute(0, 3, 4, 1, 6, 5, 2).reshape(n, h, d * 16))
    x["v"][state["touched"]] = torch.cat([packed, bits.view(torch.uint8)], -1)
    out = []
    for pool, values in ((x["k"], _k_values), (x["v"], _v_values)):
        out.append(values(pool[state["all"]], d)[state["all_at"], state["all_slot"]].to(x["k_new"].dtype))
    return out


def _plain_attention(state):
    """Segment by segment with a running maximum and sum for each query row."""
    x, case = state["x"], state["case"]
    h, d, hq = case["kv_heads"], case["head_dim"], case["q_heads"]
    g = hq // h
    q = x["q"].float().view(-1, h, g, d)
    rows = q.shape[0]
    m = torch.full((rows, h, g), -math.inf, device="cuda")
    l = torch.zeros((rows, h, g), device="cuda")
    o = torch.zeros((rows, h, g, d), device="cuda")
    for s, (at, causal) in enumerate(zip(*state["groups"])):
        n = x["seg"][s]
        if not n or not at.numel():
            continue
        k = _k_values(x["k"][state["ids"][s]], d).view(-1, h, d)[:n].permute(1, 2, 0).contiguous()
        v = _v_values(x["v"][state["ids"][s]], d).reshape(-1, h, d)[:n].permute(1, 0, 2).contiguous()
        qs = q[at].permute(1, 0, 2, 3).reshape(h, -1, d)
        score = torch.matmul(qs, k).view(h, -1, g, n) * d ** -0.5
        if causal:
            t = torch.arange(n, device="cuda")
            score = score.masked_fill((t[None, :] > t[:, None])[:, None, :], -math.inf)
        top = torch.maximum(m[at].permute(1, 0, 2), score.amax(-1))
        p = torch.exp(score - top[..., None])
        down = torch.exp(m[at].permute(1, 0, 2) - top)
        l[at] = (l[at].permute(1, 0, 2) * down + p.sum(-1)).permute(1, 0, 2)
        pv = torch.matmul(p.view(h, -1, n), v).view(h, -1, g, d)
        o[at] = (o[at].permute(1, 0, 2, 3) * down[..., None] + pv).permute(1, 0, 2, 3)
        m[at] = top.permute(1, 0, 2)
    o = (o / l[..., None]).view(rows, hq, d).to(DTYPES[case["out"]])
    return o, (m + torch.log(l)).view(rows, hq)


# ------------------------------------------------------------------- work

def work(case):
    if case["kind"] == "tables":
        length, new = _sequences(case)
        have = sum(_pages(a) for a in length)
        need = sum(_pages(a + b) for a, b in zip(length, new))
        n, tokens = case["sequences"], sum(new) + case["spare"]
        # lengths, old and new pages read; page lists, table entries, arrays of sequences and of tokens written
        return {"bytes": 8 * n + 4 * need + 4 * need + 4 * (need - have) + 24 * n + 12 * tokens, "flops": 0}
    if case["kind"] == "rope":
        elt = 2 if case["dtype"] == "bf16" else 4
        heads = case["tokens"] * (case["q_heads"] + case["kv_heads"])
        return {"bytes": 2 * heads * case["head_dim"] * elt + 4 * case["tokens"], "flops": 3 * heads * case["rotary"]}
    if case["kind"] == "write":
        length, new = _sequences(case)
        elt = 2 if case["dtype"] == "bf16" else 4
        h, d = case["kv_heads"], case["head_dim"]
        packed = h * (d + d // 32 + 2)   # a token's K and V
        total = sum(length) + sum(new)
        return {"bytes": sum(new) * (2 * h * d * elt + packed) + total * (packed + 2 * h * d * elt), "flops": 0}
    seg, paths, chunk = _forest(case)
    h, d, hq = case["kv_heads"], case["head_dim"], case["q_heads"]
    pairs = 0
    for r, p in enumerate(paths):
        n = sum(seg[s] for s in p)
        pairs += chunk[r] * (n - chunk[r]) + chunk[r] * (chunk[r] + 1) // 2 if chunk else n
    rows = sum(chunk) if chunk else case["requests"]
    sizes = {"bf16": 2, "fp32": 4}
    io = rows * hq * (d * (sizes[case["dtype"]] + sizes[case["out"]]) + 4)
    return {"bytes": sum(seg) * h * (d + d // 32 + 2) + io, "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    if case["kind"] == "tables":
        return None   # whole numbers: the plain form is the definition
    x = _inputs(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(case, x)
    if case["kind"] == "write":
        return _exact_write(case, x)
    return _exact_attention(case, x)


def _exact_rope(case, x):
    freq, amplitude = _rope_frequencies(case)
    turn = torch.polar(torch.full((case["tokens"], len(freq)), amplitude, dtype=torch.float64, device="cuda"),
                       torch.outer(x["pos"].double(), torch.tensor(freq, dtype=torch.float64, device="cuda")))
    R = case["rotary"]
    out = []
    for t in (x["q"], x["k"]):
        y = t.double().clone()
        first = slice(0, R, 2) if case["interleaved"] else slice(0, R // 2)
        second = slice(1, R, 2) if case["interleaved"] else slice(R // 2, R)
        z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return out


def _nearest(x, block):
    """The values that x's 4-bit form stands for."""
    b = x.double().view(*x.shape[:-1], -1, block)
    top = b.abs().amax(-1, keepdim=True)
    mant, ex = torch.frexp(top)                               # top = mant 2^ex, mant in [0.5, 1)
    ex = torch.where(mant >= 0.875, ex + 1, ex)               # two significant bits: 0.875 goes to 1
    unit = torch.exp2((ex - 3).clamp(min=-126).double())      # 2 ** (exponent - 2)
    y = (b / unit).clamp(-6.0, 6.0)
    # steps of 0.5 below 2, of 1 below 4, of 2 above; a tie goes to an even multiple of the step
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    return (torch.round(y / step) * step * unit).view(x.shape)


def _tile_index(d):
    """For K and V, where code (token, dim) of a tile lies, in codes."""
    t, c = np.meshgrid(np.arange(16), np.arange(d), indexing="ij")
    k = ((c % 32 // 8 * 16 + t) * (d // 32) + c // 32) * 8 + c % 8
    slot = np.asarray(SLOTS)[t]
    v = ((((c // 64) * 2 + slot // 8) * 16 + c % 16) * 4 + c // 16 % 4) * 8 + slot % 8
    return _cuda(k, torch.int64), _cuda(v, torch.int64)


def _read_tokens(pool, ids, n, d, which):
    """[n, H, D] float64 of the first n tokens of pages ids, code by code."""
    tiles = pool[torch.as_tensor(np.asarray(ids, np.int64), device="cuda")]
    at = _tile_index(d)[which]
    byte = tiles[:, :, (at // 2).flatten()].view(*tiles.shape[:2], 16, d).int()
    code = torch.where((at % 2).bool(), byte >> 4, byte & 15)
    value = _lut(torch.float64)[code]
    if which == 0:
        e = tiles[:, :, d * 8:].view(*tiles.shape[:2], 16, d // 32).int()
        value = value * _scale_lut(torch.float64)[e].repeat_interleave(32, -1)
    else:
        s = tiles[:, :, d * 8:].contiguous().view(torch.bfloat16).double()[:, :, _slots()]
        value = value * s[..., None]
    return value.permute(0, 2, 1, 3).reshape(-1, tiles.shape[1], d)[:n]


def _exact_write(case, x):
    d = case["head_dim"]
    out = []
    for which, (pool, new, block) in enumerate(((x["k"], x["k_new"], 32), (x["v"], x["v_new"], d))):
        fresh = _nearest(new, block)
        parts, at = [], 0
        for p, a, n in zip(x["pages"], x["length"], x["new"]):
            parts += [_read_tokens(pool, p[:_pages(a)], a, d, which), fresh[at:at + n]]
            at += n
        out.append(torch.cat(parts))
    return out


def _exact_attention(case, x):
    """Softmax attention of every request over its path's keys."""
    h, d, hq = case["kv_heads"], case["head_dim"], case["q_heads"]
    uses = [0] * len(x["seg"])
    for p in x["paths"]:
        for s in p:
            uses[s] += 1
    kept = {}

    def keys_of(s):
        if s not in kept:
            k, v = (_read_tokens(x[n], x["pages"][s], x["seg"][s], d, i).permute(1, 0, 2) for i, n in enumerate("kv"))
            kv = k.transpose(1, 2).contiguous(), v.contiguous()
            if uses[s] == 1:
                return kv
            kept[s] = kv
        return kept[s]

    o = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(x["q"].shape[:2], dtype=torch.float64, device="cuda")
    row = 0
    for r, p in enumerate(x["paths"]):
        n = x["chunk"][r] if x["chunk"] else 1
        q = x["q"][row:row + n].double().view(n, h, hq // h, d).permute(1, 0, 2, 3).reshape(h, -1, d)
        kv = [keys_of(s) for s in p]
        score = torch.cat([torch.matmul(q, k) for k, _ in kv], dim=2) / math.sqrt(d)
        if x["chunk"]:
            pos = torch.arange(n, device="cuda").repeat_interleave(hq // h)
            score[:, :, -n:].masked_fill_(torch.arange(n, device="cuda")[None, :] > pos[:, None], -math.inf)
        z = torch.logsumexp(score, dim=2)
        weight = torch.exp(score - z[..., None])
        out, at = 0, 0
        for _, v in kv:
            out = out + torch.matmul(weight[:, :, at:at + v.shape[1]].contiguous(), v)
            at += v.shape[1]
        o[row:row + n] = out.view(h, n, hq // h, d).permute(1, 0, 2, 3).reshape(n, hq, d)
        lse[row:row + n] = z.view(h, n, hq // h).permute(1, 0, 2).reshape(n, hq)
        row += n
    return o, lse
