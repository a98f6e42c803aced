"""GPU checks of the step operators: page lists, positions and slots against
a sequential statement of them, and the rotation against 64 bits."""

import math

import numpy as np
import pytest
import torch

from paper_2509_02121_amd import halo
from test_step import rope_frequencies

pytestmark = pytest.mark.gpu

I32 = torch.int32


def _cuda(x, dtype=I32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


# ------------------------------------------------------------------- tables

def expected_tables(seq_len, seq_new, table, free, start, max_tokens, max_pages, page_ids):
    """The step's arrays, sequence by sequence, token by token."""
    table, page_ids = table.copy(), page_ids.copy()
    n, width = len(seq_len), table.shape[1]
    bad = [a < 0 or b < 0 or a + b > min(16 * width, 2 ** 31 - 16) for a, b in zip(seq_len, seq_new)]
    lens = [(0, 0) if x else (int(a), int(b)) for a, b, x in zip(seq_len, seq_new, bad)]
    pages = [(-(-a // 16), -(-(a + b) // 16)) for a, b in lens]
    taken = sum(q - p for p, q in pages)
    fits = (0 <= start <= len(free) and start + taken <= len(free) and sum(q for _, q in pages) <= max_pages and
            sum(b for _, b in lens) <= max_tokens)
    indptr, ids, first, count, offset, pos, slot = [0], [], [], [], [], [], []
    nxt = start
    for i in range(n):
        (a, b), (p, q) = (lens[i], pages[i]) if fits else ((0, 0), (0, 0))
        for j in range(p, q):
            table[i, j] = free[nxt]
            nxt += 1
        offset.append(len(pos) if fits else 0)
        first.append(a)
        count.append(b)
        ids += list(table[i, :q])
        indptr.append(len(ids))
        for t in range(a, a + b):
            page = int(table[i, t // 16])
            pos.append(t)
            slot.append(-1 if page < 0 else page * 16 + t % 16)
    page_ids[:len(ids)] = ids
    pad = max_tokens - len(pos)
    return dict(block_table=table, seq_page_indptr=indptr, page_ids=page_ids, seq_start=first, seq_count=count,
                seq_end=[int(a) + c for a, c in zip(seq_len, count)], in_token_offset=offset,
                positions=pos + [0] * pad, slots=slot + [-1] * pad, free_next=[nxt], flag=int(not fits or any(bad)))


def check_tables(seq_len, seq_new, width=None, num_free=None, start=0, spare_tokens=0, spare_pages=0, max_tokens=None,
                 seed=0, repeat=2):
    rng = np.random.default_rng(seed)
    n = len(seq_len)
    need = [-(-max(int(a) + int(b), 0) // 16) for a, b in zip(seq_len, seq_new)]
    width = max(need + [1]) if width is None else width
    table = rng.integers(0, 1 << 30, (n, width)).astype(np.int32)
    taken = sum(q + max(int(a), 0) // -16 for q, a in zip(need, seq_len))
    free = rng.integers(0, 1 << 30, max(start + taken, 0) if num_free is None else num_free).astype(np.int32)
    max_tokens = sum(max(int(b), 0) for b in seq_new) + spare_tokens if max_tokens is None else max_tokens
    tabs = halo.StepTables(n, max_tokens, sum(need) + spare_pages)
    tabs.page_ids.fill_(-7)
    old_ids = tabs.page_ids.cpu().numpy()
    exp = expected_tables(seq_len, seq_new, table, free, start, max_tokens, tabs.max_pages, old_ids)
    flag = _cuda([0])
    d_table = _cuda(table)
    args = (tabs, _cuda(seq_len), _cuda(seq_new), d_table, _cuda(free), _cuda([start]), flag)
    for _ in range(repeat):
        halo.kv_step_tables(*args)
    got = {"block_table": d_table, "flag": flag, **{k: getattr(tabs, k) for k in exp if hasattr(tabs, k)}}
    for k, want in exp.items():
        assert np.array_equal(got[k].cpu().numpy().ravel(), np.asarray(want).ravel()), k
    return got


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 256, 257, 1000, 1024, 1025, 3000])
@pytest.mark.parametrize("kind", ["append", "mixed", "chunks"])
def test_tables(gpu_lib, n, kind):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 700, n)
    lens[rng.random(n) < 0.2] = rng.choice([0, 1, 15, 16, 17, 31, 32])
    new = {"append": np.ones(n, int), "mixed": rng.integers(0, 3, n), "chunks": rng.integers(0, 90, n)}[kind]
    check_tables(lens, new, spare_tokens=int(rng.integers(0, 50)), spare_pages=int(rng.integers(0, 9)), start=3, seed=n)


@pytest.mark.parametrize("n", [0, 1, 5])
def test_tables_empty(gpu_lib, n):
    check_tables([0] * n, [0] * n, spare_tokens=5)
    check_tables([0] * n, [0] * n)
    check_tables([40] * n, [0] * n, spare_tokens=300)


def test_tables_long_rows(gpu_lib):
    check_tables([1000003], [1], width=70000)
    check_tables([0, 16, 5], [20000, 0, 33000], width=4000, spare_tokens=100)
    check_tables([131072] * 3, [1, 2, 3], seed=4)


@pytest.mark.parametrize("n", [3, 300, 2000])
def test_tables_malformed_sequences(gpu_lib, n):
    """Negative lengths, lengths past the row and past int32: those sequences
    are left out, the others are served."""
    rng = np.random.default_rng(n)
    lens, new = rng.integers(0, 64, n), rng.integers(0, 30, n)
    for bad in ((-1, 3), (5, -1), (2 ** 31 - 1, 2 ** 31 - 1), (60, 100), (-2 ** 31, 1)):
        at = rng.integers(0, n)
        lens[at], new[at] = bad
    check_tables(lens, new, width=6, num_free=4 * n, max_tokens=30 * n)


@pytest.mark.parametrize("n", [1, 40, 1500])
def test_tables_refused_whole(gpu_lib, n):
    """A step that lacks a free page, a token's or a page's place takes
    nothing; with exactly enough it does."""
    lens, new = np.full(n, 15), np.full(n, 2)
    check_tables(lens, new, num_free=n)
    assert check_tables(lens, new, num_free=n - 1)["flag"].item() == 1
    assert check_tables(lens, new, num_free=n + 2, start=3)["free_next"].item() == 3
    check_tables(lens, new, num_free=n + 3, start=3)
    check_tables(lens, new, num_free=n, max_tokens=2 * n - 1)
    check_tables(lens, new, num_free=n, spare_pages=-1)
    check_tables(lens, new, num_free=n, start=-1)
    check_tables(lens, new, num_free=2, start=3)


def test_tables_negative_page_ids(gpu_lib):
    tabs = halo.StepTables(1, 4, 2)
    table, free = _cuda([[-5, 0]]), _cuda([9])
    halo.kv_step_tables(tabs, _cuda([14]), _cuda([4]), table, free, _cuda([0]))
    assert tabs.slots.tolist() == [-1, -1, 144, 145] and tabs.page_ids.tolist() == [-5, 9]


def test_tables_without_positions_and_slots(gpu_lib):
    tabs = halo.StepTables(2, 8, 4)
    tabs.positions = tabs.slots = None
    halo.kv_step_tables(tabs, _cuda([3, 16]), _cuda([4, 4]), _cuda([[1, 0], [2, 0]]), _cuda([7]), _cuda([0]))
    assert tabs.page_ids.tolist() == [1, 2, 7, 0] and tabs.seq_end.tolist() == [7, 20]


def test_tables_loop_in_a_graph(gpu_lib):
    """A captured step whose outputs are fed back advances by its new tokens at
    every replay, as the sequential statement does."""
    n, steps = 37, 40
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 60, n)
    new = np.ones(n, int)
    table = np.zeros((n, 8), np.int32)
    table[:, :4] = rng.integers(0, 1000, (n, 4))
    free = np.arange(2000, 2000 + 4 * n).astype(np.int32)
    tabs = halo.StepTables(n, n, 8 * n)
    d = [_cuda(lens), _cuda(new), _cuda(table), _cuda(free), _cuda([0])]
    call = halo.bind_kv_step_tables(tabs, *d)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        halo.kv_step_tables(tabs, *d)
        d[0].copy_(tabs.seq_end)
        d[4].copy_(tabs.free_next)
    start = 0
    for step in range(steps):
        exp = expected_tables(lens, new, table, free, start, n, 8 * n, tabs.page_ids.cpu().numpy())
        if step % 3 == 2:   # an eager step between the replays
            call()
            d[0].copy_(tabs.seq_end)
            d[4].copy_(tabs.free_next)
        else:
            graph.replay()
        for k in ("seq_page_indptr", "page_ids", "slots", "positions", "seq_end", "free_next"):
            assert np.array_equal(getattr(tabs, k).cpu().numpy(), np.asarray(exp[k])), (step, k)
        table, lens, start = exp["block_table"], np.array(exp["seq_end"]), exp["free_next"][0]
        assert np.array_equal(d[2].cpu().numpy(), table)


# ------------------------------------------------------------------- rope

# What the kernel adds up for y = x cos - y sin in fp32, relative to |x| + |y|:
# the angle's rounding to fp32 (pi/4 * 2^-24 on sin and cos) and one rounding of
# the quadrant's factor, the two series (each about 3 roundings at values up to
# 1), the amplitude (1), two products and a sum (2): under 8 * 2^-24. Then the
# rounding to the output's type, at most half its step.
def _rope_tolerance(x, y, dtype, amplitude):
    t = 8 * 2.0 ** -24 * amplitude * (x.abs() + y.abs())
    if dtype == torch.bfloat16:
        t = t + (amplitude * (x.abs() + y.abs())) * (torch.finfo(dtype).eps / 2)
    return t + 1e-38


def _rope_reference(t, pos, w, amplitude, interleaved):
    """(expected, tolerance) in 64 bits."""
    v = t.double().cpu()
    R = 2 * len(w)
    angle = pos.cpu().clamp(min=0).double()[:, None, None] * torch.tensor(w, dtype=torch.float64)
    c, s = amplitude * angle.cos(), amplitude * angle.sin()
    a, b = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    out, tol = v.clone(), torch.zeros_like(v)
    out[..., a], out[..., b] = v[..., a] * c - v[..., b] * s, v[..., a] * s + v[..., b] * c
    tol[..., a] = tol[..., b] = _rope_tolerance(v[..., a], v[..., b], t.dtype, amplitude)
    return out, tol


def _check_rope(q, k, pos, rope, w, amplitude, q_out=None, k_out=None):
    refs = [_rope_reference(t, pos, w, amplitude, bool(rope.params.interleaved)) for t in (q, k)]
    halo.rope_qk(q, k, pos, rope, q_out, k_out)
    for name, t, (want, tol) in zip("qk", (q if q_out is None else q_out, k if k_out is None else k_out), refs):
        err = (t.double().cpu() - want).abs()
        assert (err <= tol).all(), f"{name}: {(err / tol.clamp(min=1e-300)).max():.2f} of the tolerance"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rotary", [(128, 128), (128, 64), (128, 16), (64, 64), (64, 48), (64, 16)])
@pytest.mark.parametrize("tokens,heads", [(1, (1, 1)), (3, (32, 8)), (65, (4, 4)), (700, (16, 2)), (2500, (7, 1))])
def test_rope(gpu_lib, tokens, heads, dim, rotary, interleaved, dtype):
    gen = torch.Generator().manual_seed(tokens + dim + rotary)
    q, k = (torch.randn((tokens, h, dim), generator=gen).to(dtype).cuda() for h in heads)
    pos = torch.randint(0, 1 << 20, (tokens,), generator=gen, dtype=I32).cuda()
    rope = halo.Rope(dim, rotary, base=500000.0, interleaved=interleaved, scaling="yarn", factor=8.0)
    w, amplitude = rope_frequencies(rotary, 500000.0, "yarn", 8.0, 8192, 32, 1)
    _check_rope(q, k, pos, rope, w, amplitude, torch.full_like(q, math.nan), torch.full_like(k, math.nan))
    _check_rope(q, k, pos, rope, w, amplitude)   # in place


def test_rope_far_positions(gpu_lib):
    """Positions up to the largest int32, and negative ones (taken as 0)."""
    pos = _cuda([2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30, 10 ** 7, 1, 0, -1, -2 ** 31])
    q, k = torch.randn((8, 2, 128), device="cuda"), torch.randn((8, 1, 128), device="cuda")
    rope = halo.Rope(128)
    w, _ = rope_frequencies(128, 10000.0, "none", 1.0, 8192, 32, 1)
    # (the reference's product of 2^31 and a frequency is itself off by 2^-22)
    halo.rope_qk(q, k, pos, rope, qo := torch.empty_like(q), ko := torch.empty_like(k))
    for t, o in ((q, qo), (k, ko)):
        want, tol = _rope_reference(t, pos, w, 1.0, False)
        assert ((o.double().cpu() - want).abs() <= tol + 2.0 ** -20 * t.abs().max().item()).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope_fused_projection(gpu_lib, dtype):
    """q and k as parts of the rows of one projection, in place: the values
    and what lies between are left alone."""
    T, hq, hk, d = 77, 8, 2, 128
    rows = torch.randn((T, (hq + 2 * hk) * d + 64), device="cuda").to(dtype)
    q, k = rows[:, :hq * d].view(T, hq, d), rows[:, hq * d:(hq + hk) * d].view(T, hk, d)
    rest = rows[:, (hq + hk) * d:].clone()
    pos = torch.arange(T, dtype=I32, device="cuda")
    w, _ = rope_frequencies(d, 10000.0, "none", 1.0, 8192, 32, 1)
    _check_rope(q, k, pos, halo.Rope(d), w, 1.0)
    assert torch.equal(rows[:, (hq + hk) * d:], rest)


def test_rope_one_operand_and_none(gpu_lib):
    d = 64
    w, _ = rope_frequencies(d, 10000.0, "none", 1.0, 8192, 32, 1)
    q, none = torch.randn((5, 3, d), device="cuda"), torch.empty((5, 0, d), device="cuda")
    pos = torch.arange(5, dtype=I32, device="cuda") * 1000
    _check_rope(q, none, pos, halo.Rope(d), w, 1.0)
    _check_rope(none, q, pos, halo.Rope(d), w, 1.0)
    halo.rope_qk(q[:0], q[:0], pos[:0], halo.Rope(d))


def test_rope_special_values(gpu_lib):
    """A NaN or infinity stays in its own pair."""
    q = torch.zeros((2, 1, 64), device="cuda")
    q[0, 0, 3], q[1, 0, 40] = math.nan, math.inf
    k = torch.ones((2, 1, 64), device="cuda")
    halo.rope_qk(q, k, _cuda([5, 9]), halo.Rope(64))
    bad = ~torch.isfinite(q)
    assert bad[0, 0].nonzero().flatten().tolist() == [3, 35] and bad[1, 0].nonzero().flatten().tolist() == [8, 40]
    assert torch.isfinite(k).all()


def test_rope_in_a_graph_and_on_streams(gpu_lib):
    q, k = torch.randn((9, 4, 128), device="cuda"), torch.randn((9, 1, 128), device="cuda")
    pos, rope = torch.arange(9, dtype=I32, device="cuda"), halo.Rope(128)
    want = [t.clone() for t in (q, k)]
    halo.rope_qk(*want, pos, rope)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        halo.rope_qk(q, k, pos, rope, qo, ko)
    for _ in range(3):
        qo.zero_(), ko.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        qo.zero_(), ko.zero_()
        halo.rope_qk(q, k, pos, rope, qo, ko)
    other.synchronize()
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
