"""beam_select and kv_beam_tables on the GPU: candidates, rows, copies and the
free list equal to the oracle's.

Scores: fp32 roundings of 64-bit sums, whose ln sum exp comes from fp32
exponentials of d = logit - largest (each off by 2^-21 and, by the rounding of d and of
log2(e), 3 |d| 2^-24, with a weight of e^d: |d| e^d <= 0.37), added in fp32 in
runs of at most 512 / 64 * the tiles of a part."""

import numpy as np
import pytest
import torch

from oracle import upkeep
from paper_2509_02121_amd import halo
from upkeep_helpers import BF16, F32, cuda, random_pool

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def check_select(logits, scores, best, ended=None, end_token=0):
    """logits [items, beams, vocab] (a GPU tensor, any strides of rows)."""
    n, w, vocab = logits.shape
    out = halo.BeamSelect(n, w, vocab, best)
    for t in (out.scores, out.tokens, out.parents):
        t.fill_(77)
    out.workspace.fill_(255)
    # (a view: rows any stride apart)
    rows = logits.as_strided((n * w, vocab), (logits.stride(1), 1)) if n * w else logits.reshape(0, vocab)
    halo.beam_select(out, rows, cuda(scores, F32), None if ended is None else cuda(ended), end_token)
    torch.cuda.synchronize()
    x = logits.double().cpu().numpy()
    got_s, got_t, got_p = (t.cpu().numpy() for t in (out.scores, out.tokens, out.parents))
    scores = np.asarray(scores, np.float32).reshape(n, w)
    for i in range(n):
        s, t, p = upkeep.select(x[i], scores[i], None if ended is None else np.asarray(ended).reshape(n, w)[i], end_token,
                                best)
        s = np.array(s)
        assert got_t[i].tolist() == t and got_p[i].tolist() == p, (i, got_t[i], t, got_p[i], p, got_s[i], s)
        live = np.isfinite(s)
        assert (got_s[i][~live] == -np.inf).all()
        bound = U * np.abs(s[live]) + (vocab / 64 + 40) * U
        assert (np.abs(got_s[i][live] - s[live]) <= bound).all(), (i, got_s[i], s)
    return out


def _random(n, w, vocab, dtype, seed, scale=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    logits = (torch.randn((n, w, vocab), generator=gen, device="cuda") * scale).to(dtype)
    scores = -np.random.default_rng(seed).random((n, w)) * w - 5
    return logits, scores


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 65, 511, 512, 513, 2047, 2049, 5000, 32003])
def test_select(gpu_lib, vocab, dtype):
    for n, w, best in ((1, 1, 1), (3, 4, 4), (2, 5, 10), (2, 2, 64)):
        logits, scores = _random(n, w, vocab, dtype, vocab + best)
        check_select(logits, scores, best)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,w,best", [(1, 64, 64), (70, 3, 6), (300, 1, 2), (5, 16, 32)])
def test_select_shapes(gpu_lib, n, w, best, dtype):
    logits, scores = _random(n, w, 1501, dtype, w)
    check_select(logits, scores, best)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_large(gpu_lib, dtype):
    logits, scores = _random(2, 4, 262147, dtype, 5)
    check_select(logits, scores, 8)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two", "steps", "zeros"])
def test_select_ties_and_orders(gpu_lib, kind, dtype):
    """Ties go to the lower beam, then the lower token; rising logits renew every
    list in every tile."""
    vocab = 9001
    t = torch.arange(vocab, device="cuda")
    row = {"equal": t * 0 - 3.0, "rising": t / 500, "falling": -t / 500, "two": (t % 2) * 1.0, "steps": t // 1500 * 0.5,
           "zeros": torch.where(t % 3 == 0, -0.0, 0.0)}[kind]
    logits = row.to(dtype).expand(2, 3, vocab).contiguous()
    for best in (1, 3, 16, 64):
        check_select(logits, [[-1.0, -1.0, -2.0], [-1.0, -np.inf, -1.0]], best)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["random", "equal", "few", "close"])
@pytest.mark.parametrize("n,w,vocab,best", [(1, 16, 20011, 64), (2, 64, 3001, 64), (2, 3, 40009, 33), (1, 1, 70001, 64)])
def test_select_many_candidates(gpu_lib, n, w, vocab, best, kind, dtype):
    """More candidates than are put in order together: all apart, all the same, of few values, and of nearly one."""
    logits, scores = _random(n, w, vocab, dtype, 31)
    if kind == "equal":
        logits.fill_(0.5)
    elif kind == "few":
        logits = logits.round().clamp(-1, 2)
    elif kind == "close":
        logits = (4 + torch.arange(w, device="cuda")[None, :, None] * 2.0 ** -6 + 0 * logits.float()).to(dtype)
        logits[:, :, ::7] += 2.0 ** -5
    if kind != "random":
        scores[:] = -6.25
    check_select(logits, scores, best)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_masked_logits(gpu_lib, dtype):
    logits, scores = _random(4, 3, 3001, dtype, 7)
    low = torch.finfo(dtype).min
    logits[0, :, ::2] = -float("inf")
    logits[0, 1] = -float("inf")             # nothing left
    logits[1, :, 5:] = -float("inf")         # fewer than `best` in all
    logits[2, :, 1:] = low                   # masked by the lowest number: candidates still
    logits[2, 1] = low
    logits[3, 0, 2000:] = -float("inf")
    logits[3, 1, :2999] = -float("inf")
    for best in (3, 20, 64):
        check_select(logits, scores, best)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_no_numbers(gpu_lib, dtype):
    """A beam with a NaN or +inf among its logits, or with a score that is none, offers nothing."""
    logits, scores = _random(5, 3, 1500, dtype, 8)
    logits[0, 1, 700] = float("nan")
    logits[1, 0, 3] = float("inf")
    logits[2, :, 1499] = -float("nan")
    logits[3, 2] = float("inf")
    scores[4] = [np.nan, np.inf, -np.inf]
    logits[4, 1, 4] = float("nan")
    check_select(logits, scores, 6)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_ended_and_dead(gpu_lib, dtype):
    logits, scores = _random(6, 4, 2000, dtype, 9)
    ended = np.random.default_rng(9).integers(0, 2, (6, 4))
    ended[0], ended[1] = 1, 0
    logits[0] = float("nan")                 # not looked at
    logits[2, :, 1999] = -float("inf")
    scores[3, 1:] = -np.inf
    scores[4] = -np.inf
    ended[5] = [5, 0, -1, 0]                 # any value but 0
    scores[5, 0] = 0.0
    check_select(logits, scores, 8, ended, 1999)
    check_select(logits, scores, 4, ended, 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset", range(1, 8))
def test_select_strided_rows_at_any_alignment(gpu_lib, offset, dtype):
    """Rows inside wider ones: what lies beside them is NaN."""
    n, w, vocab = 2, 3, 1030
    base = torch.full((n * w, vocab + 13), float("nan"), dtype=dtype, device="cuda")
    logits, scores = _random(n, w, vocab, dtype, offset)
    view = base[:, offset:offset + vocab]
    view.copy_(logits.view(n * w, vocab))
    check_select(view.as_strided((n, w, vocab), (w * view.stride(0), view.stride(0), 1)), scores, 7)


def test_select_rows_past_32_bits(gpu_lib):
    """Rows that begin past 2^32 bytes."""
    stride, vocab = (1 << 30) + 3, 3000
    base = torch.empty(2 * stride + vocab, device="cuda")
    logits, scores = _random(1, 3, vocab, F32, 4)
    view = base.as_strided((1, 3, vocab), (3 * stride, stride, 1))
    view.copy_(logits)
    check_select(view, scores, 5)


def test_select_of_the_largest_sizes(gpu_lib):
    """2^24 tokens, and 65535 beams."""
    logits, scores = _random(1, 2, 2 ** 24, F32, 17)
    check_select(logits, scores, 8)
    logits, scores = _random(13107, 5, 9, BF16, 18)
    check_select(logits, scores, 3)


def test_select_of_no_items(gpu_lib):
    check_select(torch.zeros((0, 3, 10), device="cuda"), np.zeros((0, 3)), 2)


def test_select_extreme_logits(gpu_lib):
    logits, scores = _random(3, 2, 700, F32, 3)
    logits[0, 0, 9] = 3e38
    logits[0, 1] = -3e38
    logits[1] *= 1e30
    logits[2] *= 1e-30
    # a difference of 1e-30 is none beside the score: only what is certain is compared
    logits[2, :, 10:20] = torch.arange(10, device="cuda") + 1.0
    check_select(logits, scores, 2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [2, 700, 5000])
@pytest.mark.parametrize("high", [False, True])
def test_select_a_beam_whose_tokens_are_all_masked_alike(gpu_lib, high, vocab, dtype):
    """Every logit the type's lowest (or largest) number: ln sum exp is that number in 64 bits too, and each token has
    1 / vocab of the beam."""
    logits, _ = _random(1, 2, vocab, dtype, vocab)
    logits[0, 0] = torch.finfo(dtype).max if high else torch.finfo(dtype).min
    logits[0, 1] = 0.0
    logits[0, 1, 1] = 1.0                      # (the largest of the other beam, and better than any of the masked one)
    out = check_select(logits, [[-1.0, -1.0]], 2 * vocab if vocab == 2 else 3)
    own = 1.0 - np.log(vocab - 1 + np.e)
    want = sorted([(-1 + own, 1, 1)] + [(-1 - np.log(vocab), 0, t) for t in range(2)] +
                  [(-1 - np.log(vocab - 1 + np.e), 1, 0)], key=lambda x: (-x[0], x[1], x[2]))[:out.num_best]
    assert out.parents[0].tolist() == [x[1] for x in want] and out.tokens[0].tolist() == [x[2] for x in want]
    # (a fp32 rounding of a number below 16, an exponential and a sum)
    assert np.allclose(out.scores[0].double().cpu().numpy(), [x[0] for x in want], rtol=0, atol=(16 + vocab / 64 + 40) * U)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_sums_are_joined_in_64_bits(gpu_lib, dtype):
    """Two beams whose sums of exponentials, 504 and 8 times e^-20 or e^-21, are one number in 32 bits: the candidates
    of the one with the smaller sum come first. (The 8 tokens of small logits are one lane's: in its fp32 sum they
    have nothing larger beside them.)"""
    logits = torch.zeros((1, 2, 512), dtype=dtype, device="cuda")
    per = 16 // dtype.itemsize
    tokens = [(u * 64 + 5) * per + i for u in range(8 // per) for i in range(per)]
    assert np.float32(504 + 8 * np.exp(-20.0)) == np.float32(504 + 8 * np.exp(-21.0))
    for small in ((-20.0, -21.0), (-21.0, -20.0)):
        for b in range(2):
            logits[0, b, tokens] = small[b]
        out = check_select(logits, [[-1.0, -1.0]], 4)
        assert out.parents[0].tolist() == [int(small[1] < small[0])] * 4 and out.tokens[0].tolist() == [0, 1, 2, 3]


# ------------------------------------------------------------------ the tables

class Beams:
    """Items whose beams share pages as beams do, a free list and parents."""

    def __init__(self, items, beams, longest, seed=0, width=None, gone=0.1, spare=None, before=None):
        rng = np.random.default_rng(seed)
        self.items, self.beams = items, beams
        rows = items * beams
        self.len = np.zeros(rows, np.int64)
        per = upkeep.pages_of(longest)
        width = per + 2 if width is None else width
        table = rng.integers(-9, 10 ** 7, (rows, width)).astype(np.int32)    # (what lies past a row's pages is anything)
        ids = iter(rng.permutation(rows * width + rows + 50).tolist())
        for i in range(items):
            n = int(rng.integers(0, longest + 1))
            for b in range(beams):
                r = i * beams + b
                # most beams as long as their siblings, some shorter
                self.len[r] = n if rng.random() < 0.8 else rng.integers(0, n + 1)
                common = 0
                if b and rng.random() < 0.9:
                    o = i * beams + int(rng.integers(0, b))
                    whole = min(self.len[o] // 16, self.len[r] // 16)
                    common = int(rng.integers(0, whole + 1))
                    table[r, :common] = table[o, :common]
                for c in range(common, upkeep.pages_of(self.len[r])):
                    table[r, c] = next(ids)
        self.table = table
        self.parents = np.minimum(rng.geometric(0.4, (items, beams)) - 1, beams - 1)
        self.parents[rng.random((items, beams)) < gone / 2] = -1
        self.parents[rng.random(items) < gone] = -1
        most = int(sum(upkeep.pages_of(x) for x in self.len))
        rest = list(ids)[:rows + 20 if spare is None else spare]
        self.next = most if before is None else before
        self.free = np.array([-3] * self.next + rest, np.int64)

    def call(self, out=None, parents=None, **given):
        rows, width = self.table.shape
        out = halo.BeamTables(self.items, self.beams, width, len(self.free)) if out is None else out
        out.workspace.fill_(255)
        flag = cuda([0])
        a = dict(parents=cuda(self.parents if parents is None else parents), seq_len=cuda(self.len),
                 block_table=cuda(self.table), free_pages=cuda(self.free), free_next=cuda([self.next]), error_flag=flag)
        a.update(given)
        halo.kv_beam_tables(out, **a)
        torch.cuda.synchronize()
        return out, int(flag)

    def check(self, out, flag, flagged=False):
        new, lengths, free, nxt, src, dst, want_flag = upkeep.beam_tables(self.items, self.beams, self.parents, self.len,
                                                                          self.table, self.free.tolist(), self.next)
        assert want_flag == flagged and flag == int(flagged)
        assert out.seq_len.tolist() == lengths
        assert out.copy_src.tolist() == src and out.copy_dst.tolist() == dst
        got = out.block_table.cpu().numpy()
        for row, pages in zip(got, new):
            assert row[:len(pages)].tolist() == pages and (row[len(pages):] == -1).all()
        assert int(out.free_next) == nxt
        if 0 <= self.next <= len(self.free):
            assert out.free_pages[nxt:].tolist() == free[nxt:] and (out.free_pages[:nxt] == -1).all()
        else:
            assert (out.free_pages == -1).all()


@pytest.mark.parametrize("items", [1, 2, 7, 300])
@pytest.mark.parametrize("beams", [1, 2, 5, 16])
def test_tables(gpu_lib, items, beams):
    for longest in (5, 16, 200, 1000):
        case = Beams(items, beams, longest if items < 300 else longest // 4, seed=items + beams + longest)
        case.check(*case.call())


def test_tables_of_many_beams_and_long_rows(gpu_lib):
    case = Beams(3, 64, 900, seed=1)
    case.check(*case.call())
    case = Beams(2, 4, 40000, seed=2)
    case.check(*case.call())
    case = Beams(1500, 2, 60, seed=3)
    case.check(*case.call())


@pytest.mark.parametrize("items", [0, 1, 2, 40, 257])
def test_tables_with_long_free_lists_and_rows(gpu_lib, items):
    """More of the free list, and of a row, than an item's workgroup passes at once, in calls that fit and that do not."""
    case = Beams(items, 3, 300 if items else 0, seed=15 + items, spare=150001)
    case.check(*case.call())
    if items:
        case.next = 3
        case.parents[:] = -1
        case.check(*case.call(), flagged=True)
    if 0 < items <= 2:
        case = Beams(items, 5, 30000, seed=16, width=3000, spare=70000, gone=0.0)
        case.check(*case.call())


def test_tables_more_parents_than_beams(gpu_lib):
    """The first of an item's candidates, as a selection of twice as many gives them."""
    case = Beams(6, 4, 300, seed=4)
    wide = np.concatenate([case.parents, np.full((6, 5), 99)], 1)
    out, flag = case.call(parents=wide)
    case.check(out, flag)


@pytest.mark.parametrize("kind", ["same", "first", "all gone", "one gone", "swap"])
def test_tables_parents(gpu_lib, kind):
    case = Beams(5, 4, 500, seed=5)
    case.parents = np.array({"same": [0, 1, 2, 3], "first": [0, 0, 0, 0], "all gone": [-1] * 4, "one gone": [0, 0, -1, 2],
                             "swap": [3, 2, 1, 0]}[kind] * 5).reshape(5, 4)
    case.check(*case.call())


def test_tables_no_items_or_width(gpu_lib):
    case = Beams(0, 3, 0, seed=6)
    case.free, case.next = np.arange(9), 4
    case.check(*case.call())
    case = Beams(3, 2, 0, seed=6, width=0)
    case.check(*case.call())


def test_tables_malformed_items_stay(gpu_lib):
    case = Beams(6, 3, 200, seed=7, gone=0.0)
    case.parents[1, 2] = 3
    case.parents[3, 0] = -2
    case.len[4 * 3 + 1] = -1
    case.len[5 * 3] = 16 * case.table.shape[1] + 1
    case.check(*case.call(), flagged=True)
    case.parents[0, 1] = 2 ** 31 - 1
    case.len[2 * 3] = 2 ** 31 - 1
    case.check(*case.call(), flagged=True)


def test_tables_refused_whole(gpu_lib):
    # too few pages for the copies
    case = Beams(4, 4, 300, seed=8, spare=0, gone=0.0)
    case.parents[:] = 0
    case.len[:] = np.maximum(case.len // 16 * 16 - 3, 5)
    case.check(*case.call(), flagged=True)
    # more freed than came from the list
    case = Beams(4, 4, 300, seed=9, before=2)
    case.parents[:] = -1
    case.check(*case.call(), flagged=True)
    for bad in (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31):
        case = Beams(4, 4, 300, seed=10)
        case.next = bad
        case.check(*case.call(), flagged=True)


def test_tables_with_just_enough_pages(gpu_lib):
    case = Beams(4, 4, 300, seed=11, gone=0.0)
    taken = sum(d >= 0 for d in upkeep.beam_tables(4, 4, case.parents, case.len, case.table, case.free.tolist(),
                                                   case.next)[5])
    assert taken > 0
    case.free = case.free[:case.next + taken]
    case.check(*case.call())


def test_tables_in_a_graph_and_on_a_stream(gpu_lib):
    case = Beams(9, 4, 300, seed=12)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, flag = case.call(stream=side)
    case.check(out, flag)
    a = dict(parents=cuda(case.parents), seq_len=cuda(case.len), block_table=cuda(case.table),
             free_pages=cuda(case.free), free_next=cuda([case.next]))
    out = halo.BeamTables(9, 4, case.table.shape[1], len(case.free))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        halo.kv_beam_tables(out, **a)
    for _ in range(3):
        for t in (out.block_table, out.seq_len, out.free_pages, out.free_next, out.copy_src, out.copy_dst):
            t.fill_(-1)
        out.workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        case.check(out, 0)
        case.check(*case.call())


def test_select_in_a_graph_and_on_a_stream(gpu_lib):
    logits, scores = _random(6, 4, 5000, BF16, 13)
    rows, s = logits.view(24, 5000), cuda(scores, F32)
    want = check_select(logits, scores, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = halo.BeamSelect(6, 4, 5000, 8)
    torch.cuda.synchronize()
    halo.bind_beam_select(out, rows, s, stream=side)()
    side.synchronize()
    assert all(torch.equal(getattr(out, x), getattr(want, x)) for x in ("scores", "tokens", "parents"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        halo.beam_select(out, rows, s)
    for _ in range(3):
        out.tokens.fill_(-9)
        out.workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(out, x), getattr(want, x)) for x in ("scores", "tokens", "parents"))
        check_select(logits, scores, 8)


def test_two_selections_at_once(gpu_lib):
    """An object each on two streams."""
    data = [_random(4, 4, 20000, F32, 20 + i) for i in range(2)]
    outs = [halo.BeamSelect(4, 4, 20000, 8) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    s = [cuda(x[1], F32) for x in data]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            halo.beam_select(outs[i], data[i][0].view(16, 20000), s[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        want = check_select(*data[i], 8)
        assert all(torch.equal(getattr(outs[i], x), getattr(want, x)) for x in ("scores", "tokens", "parents"))


def test_copies_of_pages(gpu_lib):
    """The copies that the tables ask for, in both pools."""
    case = Beams(8, 4, 200, seed=14)
    size = int(max(case.table.max(), case.free.max())) + 1
    case.table %= size
    gen = torch.Generator(device="cuda").manual_seed(1)
    pool = random_pool(0, 2000, 2, 64, BF16, False, gen)
    out, _ = case.call()
    p = halo.make_params(2, 2, 64, BF16, 2000, 0.125)
    before = pool.clone()
    halo.kv_page_copy(pool, p, out.copy_src, out.copy_dst)
    for a, b in zip(out.copy_src.tolist(), out.copy_dst.tolist()):
        if 0 <= a < 2000 and 0 <= b < 2000:
            assert torch.equal(pool[b], before[a])
            before[b] = before[a]
    assert torch.equal(pool, before)
