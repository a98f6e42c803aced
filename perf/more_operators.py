"""The operators that decide between two steps what stays in the cache, as a serving loop calls them.

A case is a dict of plain values. ``listed()`` holds the named ones, ``draw(rng)`` makes another one of the same
ranges, and for a case

  prepare(case, seed)  what a program holds before the call: pools, tables, lists, bound calls (from the seed);
  run(state)           one pass: with ``own`` the framework's operators, without it elementary torch operations;
  work(case)           the bytes and flops that one pass cannot do without;
  exact(case, seed)    the computed outputs from the definition, in 64 bits.

Kinds:
  "weights"  of every cached token the attention weight that a step's queries gave it, added to what it had:
               w[i, h, t] = decay * w[i, h, t] + sum over rows r that see t, heads g of h: exp(scale q[r, g] . k[t, h] - lse[r, g])
             (no decayed part for tokens that are new in the step);
  "evict"    of sequences longer than `trigger` each head keeps `budget` tokens: the first `sinks`, the last `recent`
             and the heaviest of the others (ties: the earlier token); the tokens move to other pages, in order, and
             the old pages go back to the free list;
  "select"   beam search: of the candidates (beam, token) of a request with score + logit - logsumexp(logits) the
             best K, in order (ties: the lower beam, then the lower token); a beam that has ended offers its end
             token alone, at its own score; a dead beam (score -inf) offers nothing;
  "reorder"  the beams' rows of the page table follow their parents: whole pages are shared, a page that is partly
             filled is copied for every child but the first, pages that no beam holds any more are freed.

Pools have pages of 16 tokens, [page][head][tile]. E = 16 / sizeof(element):
  K [D/E][token: 16][E];  V [D][slot: 16], slots in the token order 0-3, 8-11, 4-7, 12-15;
and in the 4-bit cache (E2M1 codes, two to a byte, the first one low)
  K codes  [g: 4][token: 16][s: D/32][i: 8]           dim 32 s + 8 g + i
  K scales [token: 16][s: D/32]                       biased exponents of powers of two
  V codes  [bq: D/64][h: 2][c: 16][b: 4][j: 8]        dim 16 (4 bq + b) + c, slot 8 h + j
  V scales [slot: 16] bf16
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
DECAY = 0.9375


# ------------------------------------------------------------------- cases

def _weights(name=None, *, mode, sequences, length, rows=(1, 1), heads=(32, 8), dim=128, dtype="bf16", cache="same"):
    """mode "step": a query for each sequence, its last token's. "chunk": `rows` queries, the last tokens', causal.
    "window": the same, and the weights start anew. "shared": a prefix and the queries of `rows` requests on it."""
    case = {"kind": "weights", "mode": mode, "sequences": sequences, "length_lo": length[0], "length_hi": length[1],
            "rows_lo": rows[0], "rows_hi": rows[1], "q_heads": heads[0], "kv_heads": heads[1], "head_dim": dim,
            "dtype": dtype, "cache": cache}
    return {**case, "name": name} if name else case


def _evict(name=None, *, sequences, length, budget, trigger, sinks, recent, heads=8, dim=128, dtype="bf16",
           cache="same"):
    case = {"kind": "evict", "sequences": sequences, "length_lo": length[0], "length_hi": length[1], "budget": budget,
            "trigger": trigger, "sinks": sinks, "recent": recent, "kv_heads": heads, "head_dim": dim, "dtype": dtype,
            "cache": cache}
    return {**case, "name": name} if name else case


def _select(name=None, *, items, beams, vocab, best, dtype, ended=0.0, first=0.0):
    """`ended`: share of beams that have ended; `first`: share of requests at their first step (one live beam)."""
    case = {"kind": "select", "items": items, "beams": beams, "vocab": vocab, "best": best, "dtype": dtype,
            "ended": ended, "first": first}
    return {**case, "name": name} if name else case


def _reorder(name=None, *, items, beams, length, done=0.0, heads=1, dim=128, dtype="bf16"):
    """`done`: share of requests whose beams are all given up."""
    case = {"kind": "reorder", "items": items, "beams": beams, "length_lo": length[0], "length_hi": length[1],
            "done": done, "kv_heads": heads, "head_dim": dim, "dtype": dtype}
    return {**case, "name": name} if name else case


def listed():
    return [
        # A handful of agents on short prompts, one decode step: launches and latency.
        _weights("weights_tiny", mode="step", sequences=8, length=(272, 320), heads=(4, 4), dim=64, dtype="fp32"),
        # One layer of an 8B-shaped model, a decode step of 64 workflows on prompts of about 2300 tokens.
        _weights("weights_step", mode="step", sequences=64, length=(2112, 2560)),
        # A prompt's last queries say what of a 4-bit cache is worth keeping (ragged lengths).
        _weights("weights_window_kv4", mode="window", sequences=32, length=(1000, 8000), rows=(32, 32), cache="kv4"),
        # Chunked prefill over cached prompts: every query of the chunk counts, the largest call.
        _weights("weights_chunk", mode="chunk", sequences=8, length=(4608, 4608), rows=(512, 512)),
        # Four short fp32 sequences, just past their budget.
        _evict("evict_tiny", sequences=4, length=(272, 320), budget=256, trigger=256, sinks=4, recent=32, heads=4,
               dim=64, dtype="fp32"),
        # A full batch that is cut back to 2048 tokens, some sequences not yet.
        _evict("evict_batch", sequences=64, length=(2048, 2816), budget=2048, trigger=2112, sinks=4, recent=256),
        # A few long conversations in 4 bits, to a fraction.
        _evict("evict_long_kv4", sequences=4, length=(40000, 70000), budget=8192, trigger=8192, sinks=16, recent=1024,
               cache="kv4"),
        # One request's four beams over a small vocabulary.
        _select("select_step", items=1, beams=4, vocab=32000, best=4, dtype="fp32"),
        # A batch of requests, twice as many candidates as beams, some beams ended, some requests at their first step.
        _select("select_batch", items=64, beams=4, vocab=128256, best=8, dtype="bf16", ended=0.1, first=0.1),
        # The widest call: 1024 rows of an odd vocabulary in fp32.
        _select("select_large", items=128, beams=8, vocab=200019, best=16, dtype="fp32", ended=0.05),
        # Four requests of a few pages.
        _reorder("reorder_step", items=4, beams=4, length=(64, 400), heads=8),
        # A full batch of long histories.
        _reorder("reorder_batch", items=256, beams=8, length=(512, 4096), done=0.03),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _range(rng, lo, hi):
    a, b = sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))
    return a, b


def _draw_once(rng):
    kind = rng.choice(["weights", "weights", "weights", "evict", "evict", "select", "select", "reorder"])
    dim = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    cache = rng.choice(["same", "same", "kv4"])
    if kind == "weights":
        mode = rng.choice(["step", "step", "chunk", "window", "shared"])
        rows = {"step": (1, 1), "chunk": _range(rng, 1, 512), "window": (rng.randint(1, 64),) * 2,
                "shared": _range(rng, 1, 256)}[mode]
        return _weights(mode=mode, sequences=_log_int(rng, 1, 256), length=_range(rng, 1, 40000), rows=rows,
                        heads=rng.choice([(4, 4), (16, 16), (32, 8), (32, 8), (64, 8), (16, 1)]), dim=dim, dtype=dtype,
                        cache=cache)
    if kind == "evict":
        budget = _log_int(rng, 16, 8192)
        sinks, recent = rng.randint(0, budget // 8), rng.randint(0, budget // 2)
        return _evict(sequences=_log_int(rng, 1, 128), length=_range(rng, 1, 70000), budget=budget,
                      trigger=budget + rng.choice([0, rng.randint(0, 256)]), sinks=sinks, recent=recent,
                      heads=rng.choice([1, 4, 8]), dim=dim, dtype=dtype, cache=cache)
    if kind == "select":
        beams = _log_int(rng, 1, 16)
        return _select(items=_log_int(rng, 1, 256), beams=beams, vocab=_log_int(rng, 1000, 260000),
                       best=rng.choice([beams, 2 * beams]), dtype=dtype, ended=rng.choice([0.0, 0.1, 0.3]),
                       first=rng.choice([0.0, 0.2, 1.0]))
    return _reorder(items=_log_int(rng, 1, 512), beams=_log_int(rng, 1, 16), length=_range(rng, 1, 6000),
                    done=rng.choice([0.0, 0.1]), heads=rng.choice([1, 4, 8]), dim=dim, dtype=dtype)


def draw(rng):
    """One more case of these ranges, no more costly than the largest listed ones."""
    top = {c["name"]: work(c) for c in listed()}
    while True:
        case = _draw_once(rng)
        w = work(case)
        if case["kind"] == "weights":
            # (in fp32 a product is several)
            share = 16 if case["dtype"] == "fp32" and case["mode"] != "step" else 1
            length, rows = _sequences(case)
            widest = max(length) * max(rows) * case["q_heads"] * case["sequences"]
            if (w["bytes"] <= top["weights_step"]["bytes"] and w["flops"] * share <= top["weights_chunk"]["flops"] and
                    widest <= 1 << 30):
                return case
        elif case["kind"] == "evict":
            if w["bytes"] <= top["evict_batch"]["bytes"]:
                return case
        elif case["kind"] == "select":
            if w["bytes"] <= top["select_large"]["bytes"]:
                return case
        elif w["bytes"] <= top["reorder_batch"]["bytes"] and case["items"] * case["beams"] <= 4096:
            return case


# ------------------------------------------------------------------- sizes

def _lengths(case, lo, hi, n, what):
    """n lengths in [lo, hi], the same for every seed of one case."""
    rng = random.Random(what + repr(sorted((k, v) for k, v in case.items() if k != "name")))
    return [rng.randint(lo, hi) for _ in range(n)]


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _sequences(case):
    """(tokens, queries) of each sequence of a weights case."""
    n = case["sequences"]
    length = _lengths(case, case["length_lo"], case["length_hi"], n, "length")
    rows = _lengths(case, case["rows_lo"], case["rows_hi"], n, "rows")
    return length, rows if case["mode"] == "shared" else [min(a, b) for a, b in zip(length, rows)]


def _kept(case):
    """(tokens before, tokens after) of each sequence of an evict case."""
    length = _lengths(case, case["length_lo"], case["length_hi"], case["sequences"], "length")
    return length, [case["budget"] if n > case["trigger"] else n for n in length]


def _histories(case):
    """Of each request of a reorder case: tokens, and the pages up to which its beams share in eights, in pairs."""
    length = _lengths(case, case["length_lo"], case["length_hi"], case["items"], "length")
    return length, [(n // PAGE * 3 // 4, n // PAGE * 7 // 8) for n in length]


def _tile_bytes(case):
    """Bytes of a (page, head) tile: (K, V)."""
    d = case["head_dim"]
    if case.get("cache") == "kv4":
        return d * 8 + d // 2, d * 8 + 32
    return (16 * d * DTYPES[case["dtype"]].itemsize,) * 2


def work(case):
    """Each input read once, each output written once."""
    if case["kind"] == "weights":
        length, rows = _sequences(case)
        elt = DTYPES[case["dtype"]].itemsize
        h, d = case["kv_heads"], case["head_dim"]
        pairs = 0
        for n, r in zip(length, rows):
            pairs += n * r - (r * (r - 1) // 2 if case["mode"] in ("chunk", "window") else 0)
        old = 4 if case["mode"] != "window" else 0
        total = sum(length) * h * (_tile_bytes(case)[0] / 16 + 4 + old) + sum(rows) * case["q_heads"] * (d * elt + 4)
        return {"bytes": total + sum(_pages(n) for n in length) * 4, "flops": 2.0 * pairs * case["q_heads"] * d}
    if case["kind"] == "evict":
        before, after = _kept(case)
        h = case["kv_heads"]
        moved = sum(after) * h * (sum(_tile_bytes(case)) / 8 + 4)            # K and V read and written, weights
        return {"bytes": moved + sum(before) * h * 4 + sum(_pages(n) for n in before) * 8, "flops": 0}
    if case["kind"] == "select":
        rows = case["items"] * case["beams"]
        elt = DTYPES[case["dtype"]].itemsize
        # an exponential and a sum, and a comparison, for each logit
        return {"bytes": rows * (case["vocab"] * elt + 8) + case["items"] * case["best"] * 12,
                "flops": 3.0 * rows * case["vocab"]}
    length, _ = _histories(case)
    pages = sum(_pages(n) for n in length) * case["beams"]
    # rows read and written; about half of the beams are not their parent's first child, and copy a page
    copies = sum(n % PAGE != 0 for n in length) * case["beams"] * 0.5
    return {"bytes": pages * 8 + copies * case["kv_heads"] * sum(_tile_bytes(case)) * 2, "flops": 0}


# ------------------------------------------------------------------- inputs

def _place(page_counts, seed, spare=1.25):
    """Page ids of each list, at random in a pool a quarter larger."""
    need = int(sum(page_counts))
    size = max(1, math.ceil(need * spare))
    ids = np.random.default_rng(seed).permutation(size)[:need].astype(np.int32)
    cuts = np.cumsum([0] + list(page_counts))
    return [ids[a:b] for a, b in zip(cuts[:-1], cuts[1:])], size


def _csr(lists):
    indptr = np.zeros(len(lists) + 1, dtype=np.int32)
    indptr[1:] = np.cumsum([len(x) for x in lists])
    return _cuda(indptr), _cuda(np.concatenate(lists).astype(np.int32))


def _table(lists, width):
    """Rows of page ids, -1 behind a row's pages."""
    table = np.full((len(lists), width), -1, np.int32)
    for row, p in zip(table, lists):
        row[:len(p)] = p
    return _cuda(table)


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _cuda(values, dtype=torch.int32):
    return torch.tensor(np.asarray(values), dtype=dtype, device="cuda")


@functools.cache
def _slots():
    return torch.tensor(SLOTS, device="cuda")


@functools.cache
def _values_of_codes(dtype=torch.float32):
    return torch.tensor(E2M1 + [-x for x in E2M1], dtype=dtype, device="cuda")


def _codes(gen, shape):
    """Bytes of two E2M1 codes each, of normal values."""
    x = torch.randn((*shape, 2), generator=gen, device="cuda", dtype=torch.bfloat16)
    c = torch.zeros(x.shape, dtype=torch.uint8, device="cuda")
    for bound in (0.125, 0.375, 0.625, 0.875, 1.25, 1.75, 2.5):
        c += x.abs() > bound
    c |= torch.signbit(x).to(torch.uint8) << 3
    return c[..., 0] | (c[..., 1] << 4)


def _pools(case, size, gen):
    """A K and a V pool of normal values; some heads' keys are stronger in a few dims, as trained models' are."""
    h, d = case["kv_heads"], case["head_dim"]
    if case.get("cache") == "kv4":
        k = torch.empty((size, h, d * 8 + d // 2), dtype=torch.uint8, device="cuda")
        v = torch.empty((size, h, d * 8 + 32), dtype=torch.uint8, device="cuda")
        for a in range(0, size, 4096):
            n = min(4096, size - a)
            k[a:a + n, :, :d * 8] = _codes(gen, (n, h, d * 8))
            v[a:a + n, :, :d * 8] = _codes(gen, (n, h, d * 8))
        k[:, :, d * 8:] = 126 + torch.randint(0, 8, (size, h, d // 2), generator=gen, device="cuda").eq(0).to(torch.uint8)
        s = torch.exp2(torch.randint(-2, 1, (size, h, 16), generator=gen, device="cuda").float()).to(torch.bfloat16)
        v[:, :, d * 8:] = s.view(torch.uint8)
        return k, v
    dt, e = DTYPES[case["dtype"]], 16 // DTYPES[case["dtype"]].itemsize
    k = torch.randn((size, h, d // e, 16, e), generator=gen, device="cuda", dtype=dt)
    k[:, ::2, ::8] *= 2
    return k, torch.randn((size, h, d, 16), generator=gen, device="cuda", dtype=dt)


def _k_values(case, pool, pages, dtype=torch.float32):
    """Keys [..., 16, H, D] of the pages `pages`."""
    h, d = case["kv_heads"], case["head_dim"]
    x = pool[pages]
    lead = x.shape[:-2] if case["cache"] == "kv4" else x.shape[:-4]
    n = math.prod(lead)
    if case["cache"] == "kv4":
        x = x.view(n, h, -1)
        c = torch.stack([x[:, :, :d * 8] & 15, x[:, :, :d * 8] >> 4], -1).view(n, h, 4, 16, d // 32, 8)
        scale = torch.exp2(x[:, :, d * 8:].to(dtype) - 127).view(n, h, 1, 16, d // 32, 1)
        x = (_values_of_codes(dtype)[c.int()] * scale).permute(0, 3, 1, 4, 2, 5)
    else:
        x = x.view(n, h, d // pool.shape[4], 16, pool.shape[4]).to(dtype).permute(0, 3, 1, 2, 4)
    return x.reshape(*lead, 16, h, d)


def _scores(x, case, dtype=torch.float32):
    """Scores [n, H, rows * G, L] of every sequence's padded rows and tokens, and where they count [n, rows, L]."""
    n, r = x["q_at"].shape
    h, hq, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    k = _k_values(case, x["k"], x["table"].clamp(min=0).long(), dtype)      # [n, pages, 16, H, D]
    k = k.view(n, -1, h, d)
    L = k.shape[1]
    q = x["q"][x["q_at"].long()].to(dtype).view(n, r, h, hq // h, d).permute(0, 2, 1, 3, 4).reshape(n, h, -1, d)
    s = torch.matmul(q * d ** -0.5, k.permute(0, 2, 3, 1).contiguous())
    return s, torch.arange(L, device="cuda") < x["sees"][..., None]


def _weights_inputs(case, seed):
    gen = _generator(seed)
    length, rows = _sequences(case)
    hq, h, d, n = case["q_heads"], case["kv_heads"], case["head_dim"], case["sequences"]
    lists, size = _place([_pages(a) for a in length], seed)
    k, _ = _pools(case, size, gen)
    total = sum(rows)
    q = (torch.randn((total, hq, d), generator=gen, device="cuda") * 1.5).to(DTYPES[case["dtype"]])
    first = np.cumsum([0] + rows)
    at = np.zeros((n, max(rows)), np.int32)
    sees = np.zeros((n, max(rows)), np.int32)    # 0: no such row
    # the requests on a shared prefix are rows of q in any order
    order = np.random.default_rng(seed + 1).permutation(total) if case["mode"] == "shared" else np.arange(total)
    for i, r in enumerate(rows):
        at[i, :r] = order[first[i]:first[i + 1]]
        sees[i, :r] = length[i] if case["mode"] == "shared" else length[i] - r + 1 + np.arange(r)
    start = {"step": [a - 1 for a in length], "chunk": [a - b for a, b in zip(length, rows)],
             "window": [0] * n, "shared": length}[case["mode"]]
    width = max(length) + 5
    indptr, ids = _csr(lists)
    x = {"k": k, "q": q, "table": _table(lists, max(map(len, lists))), "ids": ids, "indptr": indptr, "size": size,
         "start": _cuda(start), "end": _cuda(length), "q_at": _cuda(at), "sees": _cuda(sees),
         "row_indptr": _cuda(first), "rows": _cuda(order),
         "row_end": _cuda(np.concatenate([s[:r] for s, r in zip(sees, rows)])),
         # what earlier steps gave: most tokens little
         "old": torch.exp(2 * torch.randn((n, h, width), generator=gen, device="cuda")),
         "out": torch.zeros((n, h, width), device="cuda")}
    s, seen = _scores(x, case)
    s = s.view(n, h, at.shape[1], hq // h, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
    z = torch.logsumexp(s, -1).permute(0, 2, 1, 3).reshape(n, -1, hq)      # [n, rows, Hq]
    x["lse"] = torch.zeros((total, hq), device="cuda")
    live = x["sees"] > 0
    x["lse"][x["q_at"][live].long()] = z[live]
    return x


def _evict_inputs(case, seed):
    gen = _generator(seed)
    before, after = _kept(case)
    n, h = case["sequences"], case["kv_heads"]
    lists, size = _place([_pages(a) for a in before] + [_pages(a) for a in after] + [19], seed, 1.05)
    k, v = _pools(case, size, gen)
    width = max(before) + 3
    w = torch.exp(2 * torch.randn((n, h, width), generator=gen, device="cuda"))
    w[torch.rand((n, h, width), generator=gen, device="cuda") < 0.02] = 0      # never looked at
    old, new = lists[:n], lists[n:2 * n]
    indptr, ids = _csr(old)
    new_indptr, new_ids = _csr(new)
    used = sum(map(len, old))
    free = np.concatenate([np.full(used + 2, -1, np.int32), lists[-1]])       # as many entries are taken already
    return {"k": k, "v": v, "size": size, "w": w, "len": _cuda(before), "table": _table(old, max(map(len, old))),
            "ids": ids, "indptr": indptr, "new_ids": new_ids, "new_indptr": new_indptr,
            "new_table": _table(new, max(map(len, new))), "none": torch.zeros(n, dtype=torch.int32, device="cuda"),
            "kept": torch.full((n, h, case["budget"]), -1, dtype=torch.int32, device="cuda"),
            "new_len": torch.zeros(n, dtype=torch.int32, device="cuda"), "w_out": torch.zeros_like(w),
            "free": _cuda(free), "free_next": _cuda([used + 2]), "free_out": torch.full_like(_cuda(free), -1),
            "free_next_out": _cuda([0])}


def _select_inputs(case, seed):
    gen = _generator(seed)
    n, w = case["items"], case["beams"]
    logits = torch.randn((n * w, case["vocab"]), generator=gen, device="cuda", dtype=DTYPES[case["dtype"]])
    logits *= 3
    # tokens that the request may not use
    banned = torch.randint(0, case["vocab"], (max(1, case["vocab"] // 500),), generator=gen, device="cuda")
    logits[:, banned] = -math.inf
    scores = -torch.rand((n, w), generator=gen, device="cuda").mul_(0.7 * w + 0.5).sort(-1).values - 12
    first = torch.rand(n, generator=gen, device="cuda") < case["first"]
    scores[first, 1:] = -math.inf
    scores[first, 0] = 0
    ended = torch.rand((n, w), generator=gen, device="cuda") < case["ended"]
    ended &= ~first[:, None]
    return {"logits": logits, "scores": scores, "ended": ended.int().contiguous(), "end": seed % case["vocab"]}


def _reorder_inputs(case, seed):
    gen = _generator(seed)
    rng = np.random.default_rng(seed)
    length, shared = _histories(case)
    n, w = case["items"], case["beams"]
    width = max(map(_pages, length)) + 4
    column = np.arange(width)[None, None, :]
    have = np.asarray([_pages(a) for a in length])[:, None, None]
    all_, pairs = (np.asarray([s[j] for s in shared])[:, None, None] for j in range(2))
    beam = np.arange(w)[None, :, None]
    # the first beam that holds the same page in the same column
    holder = np.where(column < all_, 0, np.where(column < pairs, beam // 2 * 2, beam))
    mine = (column < have) & (holder == beam)
    count = int(mine.sum())
    spare = n * w + 37
    size = count + spare
    ids = rng.permutation(size).astype(np.int32)
    table = np.full((n, w, width), -1, np.int32)
    table[mine] = ids[:count]
    table = np.where(column < have, np.take_along_axis(table, np.broadcast_to(holder, table.shape), 1), -1)
    # the best few beams carry most of the next ones
    parents = np.minimum(rng.geometric(min(0.9, 1.5 / w), (n, w)) - 1, w - 1)
    parents[rng.random(n) < case["done"]] = -1
    free = np.concatenate([np.full(count, -1, np.int32), ids[count:]])
    k, v = _pools(case, size, gen)
    rows = n * w
    return {"parents": _cuda(parents), "len": _cuda(np.repeat(length, w)), "table": _cuda(table).view(rows, width),
            "free": _cuda(free), "free_next": _cuda([count]), "k": k, "v": v, "size": size}


INPUTS = {"weights": _weights_inputs, "evict": _evict_inputs, "select": _select_inputs, "reorder": _reorder_inputs}


# ------------------------------------------------------------------- prepare and run

def _params(case, size):
    from paper_2509_02121_amd import halo
    return halo.make_params(case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["head_dim"],
                            DTYPES[case["dtype"]], size, case["head_dim"] ** -0.5)


def prepare(case, seed):
    state = {"case": case, "x": INPUTS[case["kind"]](case, seed)}
    if own:
        _bind(state)
    return state


def _bind(state):
    """The framework's calls, bound once to the loop's buffers, and what they write."""
    from paper_2509_02121_amd import halo
    halo.load_library(require_gpu=True)
    case, x = state["case"], state["x"]
    kv4 = case.get("cache") == "kv4"
    if case["kind"] == "weights":
        rows = {"step": {}, "chunk": {"row_indptr": x["row_indptr"], "row_end": x["row_end"]},
                "window": {"row_indptr": x["row_indptr"], "row_end": x["row_end"]},
                "shared": {"row_indptr": x["row_indptr"], "rows": x["rows"]}}[case["mode"]]
        bind = halo.bind_kvq_page_weights if kv4 else halo.bind_kv_page_weights
        state["calls"] = [bind(x["old"], x["k"], _params(case, x["size"]), x["ids"], x["indptr"], x["start"], x["end"],
                               x["q"], x["lse"], decay=DECAY, weights_out=x["out"], **rows)]
        state["out"] = x["out"]
    elif case["kind"] == "evict":
        keep = halo.bind_kvq_page_keep_kv if kv4 else halo.bind_kv_page_keep_kv
        state["calls"] = [
            halo.bind_kv_evict_select(x["w"], x["len"], x["kept"], x["new_len"], trigger=case["trigger"],
                                      sinks=case["sinks"], recent=case["recent"], weights_out=x["w_out"]),
            keep(x["k"], x["v"], _params(case, x["size"]), x["ids"], x["indptr"], x["len"], x["new_len"], x["kept"],
                 x["new_ids"], x["new_indptr"]),
            halo.bind_kv_release_pages(x["table"], x["len"], x["none"], x["free"], x["free_next"], x["free_out"],
                                       x["free_next_out"])]
        state["out"] = [x[name] for name in ("kept", "new_len", "w_out", "k", "v", "free_out", "free_next_out")]
    elif case["kind"] == "select":
        out = halo.BeamSelect(case["items"], case["beams"], case["vocab"], case["best"])
        state["calls"] = [halo.bind_beam_select(out, x["logits"], x["scores"], x["ended"], x["end"])]
        state["out"] = [out.scores, out.tokens, out.parents]
    else:
        out = halo.BeamTables(case["items"], case["beams"], x["table"].shape[1], x["free"].numel())
        p = _params(case, x["size"])
        state["calls"] = [
            halo.bind_kv_beam_tables(out, x["parents"], x["len"], x["table"], x["free"], x["free_next"]),
            halo.bind_kv_page_copy(x["k"], p, out.copy_src, out.copy_dst),
            halo.bind_kv_page_copy(x["v"], p, out.copy_src, out.copy_dst)]
        state["out"] = [out.block_table, out.seq_len, out.free_pages, out.free_next, out.copy_src, out.copy_dst, x["k"],
                        x["v"]]


def run(state):
    if own:
        for call in state["calls"]:
            call()
        return state["out"]
    return PLAIN[state["case"]["kind"]](state["case"], state["x"])


# ------------------------------------------------------------------- plain forms

def _plain_weights(case, x):
    n, h = x["old"].shape[:2]
    s, seen = _scores(x, case)
    r = x["q_at"].shape[1]
    s = s.view(n, h, r, -1, s.shape[-1])
    lse = x["lse"][x["q_at"].long()].view(n, r, h, -1).permute(0, 2, 1, 3)[..., None]
    p = torch.exp(s.sub_(lse).masked_fill_(~seen[:, None, :, None], -math.inf))
    w = p.sum((2, 3))                                                     # [n, H, L]
    width = x["old"].shape[2]
    w = torch.nn.functional.pad(w, (0, max(0, width - w.shape[2])))[..., :width]
    t = torch.arange(width, device="cuda")
    w += torch.where((t < x["start"][:, None])[:, None], x["old"] * DECAY, 0)
    x["out"].copy_(torch.where((t < x["end"][:, None])[:, None], w, x["out"]))
    return x["out"]


def _moved_tokens(case, x, kept_rows, new_len):
    """Of every token after the move: (old page, old place, new page, new place), pages and places of new ones [T] and
    of old ones [T, H]."""
    n = x["len"].shape[0]
    j = torch.arange(x["new_table"].shape[1] * PAGE, device="cuda")
    live = j < new_len[:, None]
    i, j = live.nonzero(as_tuple=True)
    whole = (new_len == x["len"])[i]
    old = torch.where(whole[:, None], j[:, None], kept_rows[i, :, j.clamp(max=case["budget"] - 1)]).long()   # [T, H]
    old_page = x["table"].reshape(-1)[i[:, None] * x["table"].shape[1] + old // PAGE].long()
    return old_page, old % PAGE, x["new_table"][i, j // PAGE].long(), j % PAGE


def _plain_evict(case, x):
    w, n_tokens = x["w"], x["len"][:, None, None]
    n, h, width = w.shape
    budget, sinks, recent = case["budget"], case["sinks"], case["recent"]
    t = torch.arange(width, device="cuda")
    evicted = x["len"] > case["trigger"]
    new_len = torch.where(evicted, budget, x["len"]).int()
    middle = (t >= sinks) & (t < n_tokens - recent)
    order = torch.where(middle, w, -1.0).sort(dim=-1, descending=True, stable=True).indices
    keep = torch.zeros(w.shape, dtype=torch.bool, device="cuda")
    keep.scatter_(2, order[..., :budget - sinks - recent], True)
    keep = torch.where(evicted[:, None, None], (keep | ~middle) & (t < n_tokens), False)
    x["kept"][evicted] = keep[evicted].nonzero()[:, 2].view(-1, h, budget).int()
    x["new_len"].copy_(new_len)
    # the kept weights, in order
    at = torch.arange(budget, device="cuda").expand(n, h, budget)
    index = torch.where(evicted[:, None, None], x["kept"], at).long().clamp(max=width - 1)
    kept_w = torch.nn.functional.pad(w.gather(2, index), (0, max(0, width - budget)))[..., :width]
    moved = torch.where(evicted[:, None, None], kept_w, w)
    x["w_out"].copy_(torch.where(t < new_len[:, None, None], moved, x["w_out"]))
    # keys and values
    old_page, old_at, page, place = _moved_tokens(case, x, x["kept"], new_len)
    head = torch.arange(h, device="cuda")
    slots = _slots()
    d = case["head_dim"]
    if case["cache"] == "kv4":
        k, v = x["k"], x["v"]
        codes = k[:, :, :d * 8].view(-1, h, 4, 16, d // 8)       # (views: the tiles' bytes lie as they are)
        scales = k[:, :, d * 8:].view(-1, h, 16, d // 32)
        codes[page[:, None], head, :, place[:, None]] = codes[old_page, head, :, old_at]
        scales[page[:, None], head, place[:, None]] = scales[old_page, head, old_at]
        codes = v[:, :, :d * 8].view(-1, h, d // 64, 2, 64, 4)   # [bq][half][c, b][pair of slots]
        a, b = slots[old_at], slots[place][:, None]
        moved = codes[old_page, head, :, a // 8, :, a % 8 // 2]
        moved = torch.where((a % 2 == 1)[..., None, None], moved >> 4, moved & 15)      # [T, H, bq, 64]
        for odd in (0, 1):   # a byte holds two tokens: the low codes, then the high ones
            some = place % 2 == odd                                                       # (a slot is odd as its token is)
            at_ = (page[some, None], head, slice(None), b[some] // 8, slice(None), b[some] % 8 // 2)
            codes[at_] = (codes[at_] & (0x0f if odd else 0xf0)) | (moved[some] << (4 * odd))
        scales = v[:, :, d * 8:].view(torch.int16)
        scales[page[:, None], head, b] = scales[old_page, head, a]
    else:
        x["k"][page[:, None], head, :, place[:, None]] = x["k"][old_page, head, :, old_at]
        x["v"][page[:, None], head, :, slots[place][:, None]] = x["v"][old_page, head, :, slots[old_at]]
    # the old pages, in order, before what is still free
    pages = x["table"][torch.arange(x["table"].shape[1], device="cuda") < ((x["len"] + 15) // PAGE)[:, None]]
    first = x["free_next"].long()
    begin = first - pages.numel()
    at = torch.arange(x["free"].numel(), device="cuda")
    x["free_out"].copy_(torch.where(at >= first, x["free"], x["free_out"]))
    x["free_out"][begin + torch.arange(pages.numel(), device="cuda")] = pages
    x["free_next_out"].copy_(begin)
    return [x[name] for name in ("kept", "new_len", "w_out", "k", "v", "free_out", "free_next_out")]


def _plain_select(case, x):
    n, w, vocab, best = case["items"], case["beams"], case["vocab"], case["best"]
    y = x["logits"].double()      # scores of different beams lie close together
    top = y.amax(1, keepdim=True)
    z = top + torch.exp(y - top).sum(1, keepdim=True).log()
    y = y.sub_(z).add_(x["scores"].double().view(-1, 1)).nan_to_num_(-math.inf, math.inf, -math.inf)
    ended = x["ended"].view(-1) != 0
    y.masked_fill_(ended[:, None], -math.inf)
    y[:, x["end"]] = torch.where(ended, x["scores"].double().view(-1), y[:, x["end"]])
    y = y.view(n, w * vocab)
    least = y.topk(best, 1).values[:, -1:]
    i, c = ((y >= least) & (y > -math.inf)).nonzero(as_tuple=True)          # a request's candidates, in order
    value = y[i, c]
    order = value.sort(descending=True, stable=True).indices
    order = order[i[order].sort(stable=True).indices]                       # by request, value, place
    i, c, value = i[order], c[order], value[order]
    rank = torch.arange(i.numel(), device="cuda") - torch.searchsorted(i, i)
    i, c, value, rank = (v[rank < best] for v in (i, c, value, rank))
    scores = torch.full((n, best), -math.inf, device="cuda")
    tokens, parents = (torch.full((n, best), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    scores[i, rank] = value.float()
    tokens[i, rank] = (c % vocab).int()
    parents[i, rank] = (c // vocab).int()
    return [scores, tokens, parents]


def _plain_reorder(case, x):
    n, w = case["items"], case["beams"]
    width = x["table"].shape[1]
    table, length = x["table"].view(n, w, width), x["len"].view(n, w)
    p = x["parents"].long()
    live = p >= 0
    at = p.clamp(min=0)
    column = torch.arange(width, device="cuda")
    new_len = torch.where(live, length.gather(1, at), 0)
    have = (new_len + 15) // PAGE
    new = torch.where(column < have[..., None], table.gather(1, at[..., None].expand(-1, -1, width)), -1)
    # a partly filled page stays with its holder's first child
    later = torch.tril((p[:, :, None] == p[:, None, :]), -1).any(2)
    copied = live & later & (new_len % PAGE != 0)
    number = copied.view(-1).cumsum(0).view(n, w)
    taken = number[-1, -1]
    first = x["free_next"].long()
    fresh = x["free"][(first + number - 1).clamp(0, x["free"].numel() - 1)]
    last = (have - 1).clamp(min=0)[..., None].long()
    source = new.gather(2, last)[..., 0]
    new = torch.where(copied[..., None] & (column == last), fresh[..., None], new)
    copy_src, copy_dst = (torch.where(copied, v, -1).int().view(-1) for v in (source, fresh))
    # pages of the old rows that no new row holds, once each
    valid = column < ((length + 15) // PAGE)[..., None]
    gone = valid.clone()
    first_holder = torch.ones_like(valid)
    for j in range(w):
        held = (new[:, j:j + 1] == table) & (new[:, j:j + 1] >= 0)
        gone &= ~held
        first_holder[:, j + 1:] &= ~((table[:, j:j + 1] == table[:, j + 1:]) & valid[:, j:j + 1])
    gone &= first_holder
    pages = table.transpose(1, 2)[gone.transpose(1, 2)]                     # by request, column, beam
    begin = first + taken - pages.numel()
    place = torch.arange(x["free"].numel(), device="cuda")
    free = torch.where(place >= first + taken, x["free"], -1)
    free[begin + torch.arange(pages.numel(), device="cuda")] = pages
    source, fresh = copy_src[copied.view(-1)].long(), copy_dst[copied.view(-1)].long()
    for pool in (x["k"], x["v"]):
        pool[fresh] = pool[source]
    return [new.view(n * w, width), new_len.int().view(-1), free, begin.int(), copy_src, copy_dst, x["k"], x["v"]]


PLAIN = {"weights": _plain_weights, "evict": _plain_evict, "select": _plain_select, "reorder": _plain_reorder}


# ------------------------------------------------------------------- in 64 bits

def _tokens_of(case, pool, ids, n):
    """The first n keys of a page list [n, H, D], element by element, in 64 bits."""
    d = case["head_dim"]
    token, dim = np.meshgrid(np.arange(16), np.arange(d), indexing="ij")
    tiles = pool[torch.as_tensor(np.asarray(ids, np.int64), device="cuda")].flatten(2)
    if case["cache"] == "kv4":
        at = _cuda(((dim % 32 // 8 * 16 + token) * (d // 32) + dim // 32) * 8 + dim % 8, torch.int64)
        byte = tiles[:, :, (at // 2).flatten()].view(*tiles.shape[:2], 16, d).int()
        value = _values_of_codes(torch.float64)[torch.where((at % 2).bool(), byte >> 4, byte & 15)]
        e = tiles[:, :, _cuda(d * 8 + token * (d // 32) + dim // 32, torch.int64).flatten()]
        value = torch.ldexp(value, e.view(value.shape).int() - 127)
    else:
        e = 16 // DTYPES[case["dtype"]].itemsize
        at = _cuda((dim // e * 16 + token) * e + dim % e, torch.int64)
        value = tiles[:, :, at.flatten()].view(*tiles.shape[:2], 16, d).double()
    return value.permute(0, 2, 1, 3).reshape(-1, tiles.shape[1], d)[:n]


def _exact_weights(case, x):
    length, rows = _sequences(case)
    h, hq, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    out = x["out"].double()
    indptr, ids, start = (x[k].cpu().numpy() for k in ("indptr", "ids", "start"))
    for i, (n, r) in enumerate(zip(length, rows)):
        k = _tokens_of(case, x["k"], ids[indptr[i]:indptr[i + 1]], n)
        at, sees = x["q_at"][i, :r].long(), x["sees"][i, :r]
        for head in range(h):
            group = slice(head * (hq // h), (head + 1) * (hq // h))
            s = x["q"][at, group].double().flatten(0, 1) @ k[:, head].T.contiguous() / math.sqrt(d)
            p = torch.exp(s - x["lse"][at, group].double().flatten()[:, None]).view(r, -1, n)
            total = p.masked_fill_(torch.arange(n, device="cuda") >= sees[:, None, None], 0).sum((0, 1))
            total[:start[i]] += DECAY * x["old"][i, head, :start[i]].double()
            out[i, head, :n] = total
    return out


def _exact_select(case, x):
    scores = torch.full((case["items"], case["best"]), -math.inf, dtype=torch.float64, device="cuda")
    ended, given = x["ended"].cpu(), x["scores"].cpu()
    for i in range(case["items"]):
        values = []
        for b in range(case["beams"]):
            if given[i, b] == -math.inf:
                continue
            if ended[i, b]:
                values.append(given[i, b:b + 1].double().cuda())
            else:
                y = x["logits"][i * case["beams"] + b].double()
                values.append(float(given[i, b]) + y - torch.logsumexp(y, 0))
        every = torch.cat(values) if values else torch.zeros(0, dtype=torch.float64, device="cuda")
        best = every.sort(descending=True).values[:case["best"]]
        scores[i, :best.numel()] = best
    return [scores, None, None]


def exact(case, seed):
    """None where a pass computes no numbers: tokens and pages move bit for bit."""
    if case["kind"] == "weights" and case["sequences"] * case["kv_heads"] <= 4096:
        return _exact_weights(case, INPUTS["weights"](case, seed))
    if case["kind"] == "select":
        return _exact_select(case, _select_inputs(case, seed))
    return None
