"""kv_page_weights and kvq_page_weights on the GPU against the formula in 64
bits, element by element.

The bound on an element sums, over the rows that count, p times what p may be off
by: the score's products and sums (D + 2 roundings of 2^-24 of the products'
magnitudes each, twice that for what an MFMA may cut), the roundings of scale and of
log2(e) times score and lse (four of 2^-24), the exponential (2^-21) and the sum
(a rounding a term)."""

import numpy as np
import pytest
import torch

import oracle
from oracle import upkeep
from paper_2509_02121_amd import halo
from upkeep_helpers import BF16, F32, cuda, csr, params, random_pool, to_numpy, values

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


class Case:
    """Sequences of `lengths` tokens with `rows` query rows each (any number), in a pool with NaN wherever no token
    is; every input random."""

    def __init__(self, lengths, rows, heads=(4, 2), dim=128, dtype=BF16, kvq=False, seed=0, width=None, causal=True,
                 strong=1.0, extra_pages=3):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        hq, h = heads
        self.h, self.hq, self.dim, self.kvq, self.dtype = h, hq, dim, kvq, dtype
        self.lengths, self.rows = list(lengths), list(rows)
        n, need = len(lengths), [upkeep.pages_of(a) for a in lengths]
        size = sum(need) + extra_pages
        ids = rng.permutation(size)
        cuts = np.cumsum([0] + need)
        self.lists = [ids[a:b] for a, b in zip(cuts, cuts[1:])]
        self.pool = random_pool(0, size, h, dim, dtype, kvq, gen, 0.7)
        keys = values(to_numpy(self.pool), 0, dim, kvq)
        self.keys = [keys[p].reshape(-1, h, dim)[:a] for p, a in zip(self.lists, lengths)]
        self._poison()
        self.params = params(hq, h, dim, dtype, size)
        total = sum(rows)
        self.q = (torch.randn((total + 2, hq, dim), generator=gen, device="cuda") * strong).to(dtype)
        self.order = rng.permutation(total + 2)[:total]       # rows of q in any order
        self.row_indptr = np.cumsum([0] + list(rows))
        self.row_end = np.concatenate([np.zeros(0, int)] + [rng.integers(0, a + 3, r) if causal else np.full(r, a)
                                                             for a, r in zip(lengths, rows)]).astype(int)
        self.start = np.array([rng.integers(-1, a + 2) for a in lengths])
        # what attention gives: every row over the tokens it sees
        q64 = self.q.double().cpu().numpy()
        lse = np.full((total + 2, hq), np.nan)
        for i, k in enumerate(self.keys):
            for e in range(self.row_indptr[i], self.row_indptr[i + 1]):
                r, m = self.order[e], min(self.row_end[e], len(k))
                for g in range(hq):
                    s = dim ** -0.5 * (k[:m, g // (hq // h)] @ q64[r, g])
                    lse[r, g] = upkeep.log_sum_exp(s) if m else -np.inf
        self.lse = cuda(lse, F32)
        self.q64, self.lse64 = q64, self.lse.double().cpu().numpy()
        self.width = (max(lengths, default=0) + 5) if width is None else width
        self.old = torch.exp(2 * torch.randn((n, h, self.width), generator=gen, device="cuda"))
        self.indptr, self.ids = csr(self.lists)

    def _poison(self):
        """NaN in the slots behind each sequence's tokens and in pages of none."""
        used = {int(p) for x in self.lists for p in x}
        spare = [p for p in range(len(self.pool)) if p not in used]
        if self.kvq:
            self.pool[spare, :, self.dim * 8:] = 255
            scales = self.pool[:, :, self.dim * 8:].view(len(self.pool), self.h, 16, -1)
            for x, a in zip(self.lists, self.lengths):
                if a % 16:
                    scales[int(x[-1]), :, a % 16:] = 255
            return
        self.pool[spare] = float("nan")
        e = 16 // self.dtype.itemsize
        units = self.pool.view(len(self.pool), self.h, self.dim // e, 16, e)
        for x, a in zip(self.lists, self.lengths):
            if a % 16:
                units[int(x[-1]), :, :, a % 16:] = float("nan")

    def arguments(self, **given):
        a = dict(weights=self.old, k_pool=self.pool, params=self.params, page_ids=self.ids, seq_page_indptr=self.indptr,
                 seq_start=cuda(self.start), seq_end=cuda(self.lengths), q=self.q, lse=self.lse,
                 row_indptr=cuda(self.row_indptr), rows=cuda(self.order), row_end=cuda(self.row_end), decay=0.75,
                 weights_out=torch.full_like(self.old, -7.0))
        a.update(given)
        return a

    def expected(self, i, decay=0.75, start=None, entries=None, order=None, row_end=None):
        """(weights, bound on the error) of sequence i, [H, tokens] each."""
        order = self.order if order is None else order
        entries = range(self.row_indptr[i], self.row_indptr[i + 1]) if entries is None else entries
        r = [order[e] for e in entries]
        ends = [(self.row_end if row_end is None else row_end)[e] for e in entries]
        scale = float(np.float32(self.dim ** -0.5))
        old = self.old[i].double().cpu().numpy()
        w, products, sizes = upkeep.weights(self.keys[i], self.q64[r], self.lse64[r], ends, scale, old,
                                            self.start[i] if start is None else start, decay)
        terms = len(r) * (self.hq // self.h)
        return w, 2 * (self.dim + 2) * U * products + 4 * U * sizes + (2.0 ** -21 + (terms + 4) * U) * w

    def check(self, out, which=None, **given):
        got = out.double().cpu().numpy()
        for i, a in enumerate(self.lengths) if which is None else which:
            w, bound = self.expected(i, **given)
            off = np.abs(got[i, :, :a] - w) - bound
            assert (off <= 0).all(), f"sequence {i}: {off.max():.3g} past the bound at {np.unravel_index(off.argmax(), off.shape)}"
            assert (got[i, :, a:] == -7.0).all(), f"sequence {i}: written past its end"


def _call(case, **given):
    a = case.arguments(**given)
    (halo.kvq_page_weights if case.kvq else halo.kv_page_weights)(**a)
    torch.cuda.synchronize()
    return a["weights_out"]


LENGTHS = [0, 1, 15, 16, 17, 100, 333, 64]
ROWS = [2, 1, 0, 17, 5, 40, 3, 1]
FORMATS = [(BF16, False), (F32, False), (BF16, True), (F32, True)]


@pytest.mark.parametrize("dtype,kvq", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (4, 2), (32, 8), (16, 1), (10, 2), (40, 2)])
def test_weights(gpu_lib, heads, dim, dtype, kvq):
    case = Case(LENGTHS, ROWS, heads, dim, dtype, kvq, seed=sum(heads))
    case.check(_call(case))


@pytest.mark.parametrize("dtype,kvq", FORMATS)
def test_many_rows(gpu_lib, dtype, kvq):
    case = Case([700, 33, 1], [150, 300, 64], (8, 2), 64, dtype, kvq, seed=3)
    case.check(_call(case))
    case = Case([130, 257], [513, 77], (4, 1), 128, dtype, kvq, seed=4, causal=False)
    case.check(_call(case))


@pytest.mark.parametrize("dtype,kvq", FORMATS)
def test_decode_step(gpu_lib, dtype, kvq):
    """A row for each sequence, no lists."""
    n = 70
    rng = np.random.default_rng(5)
    lengths = rng.integers(1, 400, n)
    case = Case(lengths, [1] * n, (8, 4), 128, dtype, kvq, seed=5, causal=False)
    case.order, case.start = np.arange(n), lengths - 1
    q64 = case.q64
    lse = np.array([[upkeep.log_sum_exp(case.dim ** -0.5 * (case.keys[i][:, g // 2] @ q64[i, g])) for g in range(8)]
                    for i in range(n)] + [[0.0] * 8] * 2)
    case.lse = cuda(lse, F32)
    case.lse64 = case.lse.double().cpu().numpy()
    out = _call(case, row_indptr=None, rows=None, row_end=None, seq_start=cuda(case.start))
    case.check(out)
    # nothing is new: the old weight counts everywhere
    case.check(_call(case, row_indptr=None, rows=None, row_end=None, seq_start=None), start=10 ** 6)


@pytest.mark.parametrize("dtype,kvq", FORMATS)
@pytest.mark.parametrize("heads", [(1, 1), (32, 2), (34, 2), (64, 1)])
def test_decode_step_with_rows_and_ends(gpu_lib, heads, dtype, kvq):
    """An entry for each sequence, with its row and end from lists; q heads of a kv head that fill a tile, and more."""
    rng = np.random.default_rng(23)
    lengths = [0, 1, 16, *rng.integers(0, 200, 20), 1000]
    case = Case(lengths, [1] * len(lengths), heads, 64, dtype, kvq, seed=23)
    case.check(_call(case, row_indptr=None))
    ends = np.array([len(k) for k in case.keys])
    case.check(_call(case, row_indptr=None, row_end=None), row_end=ends)


@pytest.mark.parametrize("dtype,kvq,dim", [(BF16, False, 128), (F32, False, 64), (F32, False, 128), (BF16, True, 128)])
def test_decode_step_of_many_pages(gpu_lib, dtype, kvq, dim):
    """More pages than waves, several sequences to a run of them; keys of more than 64 MiB (those of 2 bytes and 4)."""
    rng = np.random.default_rng(24)
    lengths = [*rng.integers(1, 40, 60), *rng.integers(500, 1500, 34)]
    rng.shuffle(lengths)
    case = Case(lengths, [1] * len(lengths), (8, 8), dim, dtype, kvq, seed=24)
    assert sum(len(x) for x in case.lists) * 8 > 4 * 4096
    case.check(_call(case, row_indptr=None))


@pytest.mark.parametrize("kvq", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_more_rows_than_are_held(gpu_lib, dim, kvq):
    """Rows in many batches, some of them one row longer; rows that see none, some or all of the keys in turn."""
    case = Case([300, 40, 700], [1100, 129, 343], (3, 1), dim, BF16, kvq, seed=25)
    case.check(_call(case))
    case = Case([513, 64], [1025, 128], (2, 2), dim, BF16, kvq, seed=26, causal=False)
    case.row_end[::3] = 0
    case.row_end[200:500] = 100
    # (lse over all of the keys: a row that sees fewer of them has smaller weights)
    case.check(_call(case))


@pytest.mark.parametrize("kvq", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_window_of_rows(gpu_lib, dim, kvq):
    """Some rows for many pages: several groups of pages with the same rows, sequences that begin and end inside of
    them, and one with more rows than are held at once."""
    rng = np.random.default_rng(27)
    lengths = [*rng.integers(0, 3000, 12), 17000, 1, 256, 4096]
    rows = [*rng.integers(0, 60, 12), 64, 3, 300, 128]
    case = Case(lengths, rows, (4, 2), dim, BF16, kvq, seed=27)
    case.check(_call(case))
    once = case.old.clone()
    _call(case, weights=once, weights_out=once)
    case.check(torch.where(torch.arange(case.width, device="cuda") < cuda(lengths)[:, None, None], once, -7.0))


@pytest.mark.parametrize("kvq", [False, True])
@pytest.mark.parametrize("longest", [50, 100, 200])
@pytest.mark.parametrize("rows", [10, 30, 90])
def test_short_sequences(gpu_lib, rows, longest, kvq):
    """Many sequences to a job, some empty, with rows for each of the kernels that weights of this width may go to."""
    rng = np.random.default_rng(32)
    lengths = [*rng.integers(0, longest, 60), longest]
    case = Case(lengths, rng.integers(rows // 2, rows, 61), (4, 2), 64, BF16, kvq, seed=32)
    case.check(_call(case))


@pytest.mark.parametrize("dtype,rows", [(F32, 3), (BF16, 1), (BF16, 3), (BF16, 40), (BF16, 700)])
def test_slices_of_longer_lists(gpu_lib, rows, dtype):
    """Page lists and entries that begin inside of their arrays."""
    case = Case([130, 0, 40, 257], [rows] * 4, (2, 1), 64, dtype, seed=36)
    ids = torch.cat([torch.full((13,), -9, dtype=torch.int32, device="cuda"), case.ids])
    given = dict(page_ids=ids, seq_page_indptr=case.indptr + 13)
    if rows == 1:
        given["row_indptr"] = None
    else:
        pad = np.full(7, 2 ** 30)
        given.update(rows=cuda(np.concatenate([pad, case.order])), row_end=cuda(np.concatenate([pad, case.row_end])),
                     row_indptr=cuda(case.row_indptr + 7))
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    case.check(_call(case, error_flag=flag, **given))
    assert int(flag) == 0


def test_lists_of_no_pages_are_refused(gpu_lib):
    """An array of no elements has no address; one of any element is taken."""
    case = Case([0, 0], [1, 1], (2, 1), 64, BF16, seed=37, width=5)
    with pytest.raises(halo.HaloError, match="page_ids"):
        _call(case, page_ids=cuda([]))
    case.check(_call(case, page_ids=cuda([0])))


def test_lists_that_are_left_out(gpu_lib):
    case = Case([50, 20, 90], [3, 0, 20], seed=6, causal=False)
    case.check(_call(case, row_end=None))
    # rows NULL: entry e is token e
    plain = Case([50, 20, 90], [3, 0, 20], seed=6)
    plain.order = np.arange(23)
    lse = plain.lse64.copy()
    lse[:23] = 3.0
    plain.lse, plain.lse64 = cuda(lse, F32), lse
    plain.check(_call(plain, rows=None))


@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
def test_decay_and_in_place(gpu_lib, decay):
    case = Case([77, 200], [4, 30], seed=7)
    old = case.old.clone()
    if decay == 0.0:
        old.fill_(float("nan"))       # not read
    old[0, :, 77:] = old[1, :, 200:] = -7.0
    for i in range(2):
        old[i, :, max(case.start[i], 0):case.lengths[i]] = float("nan")   # a new token's old weight is not read
    out = old.clone()
    _call(case, weights=out, weights_out=None, decay=decay)
    case.check(out, decay=decay)
    if decay == 0.0:
        out = torch.full_like(case.old, -7.0)
        _call(case, weights=None, weights_out=out, decay=0.0)
        case.check(out, decay=decay)


def test_accumulates_over_steps(gpu_lib):
    """Three calls in a row with decay 1 add up."""
    case = Case([60, 35], [5, 2], seed=8)
    case.start = np.array([60, 35])
    out = case.old.clone()
    for _ in range(3):
        _call(case, weights=out, weights_out=None, decay=1.0, seq_start=None)
    for i, a in enumerate(case.lengths):
        w, bound = case.expected(i, decay=0.0)
        old = case.old[i, :, :a].double().cpu().numpy()
        off = np.abs(out[i, :, :a].double().cpu().numpy() - (old + 3 * w)) - 3 * (bound + U * (old + 3 * w))
        assert (off <= 0).all()


def test_rows_that_see_nothing(gpu_lib):
    case = Case([40, 40], [3, 20], seed=9)
    case.row_end[:] = 0
    case.row_end[5] = -4
    out = _call(case, row_end=cuda(case.row_end))
    case.check(out, which=[(0, 40), (1, 40)], row_end=np.zeros(23, int))
    # lse = -inf adds nothing, whatever the row would see
    case.lse.fill_(-float("inf"))
    case.check(_call(case, row_end=None), row_end=np.zeros(23, int))


def test_no_sequences_and_no_rows(gpu_lib):
    empty = Case([], [], seed=1, width=4)
    _call(empty)
    none = Case([20, 0], [0, 0], seed=1)
    none.check(_call(none))


def test_special_values(gpu_lib):
    """A NaN or infinite key spoils its own token, a NaN row the tokens it sees."""
    case = Case([48, 48], [2, 2], (2, 1), 64, BF16, seed=11, causal=False)
    units = case.pool.view(len(case.pool), 1, 8, 16, 8)
    page = int(case.lists[0][1])
    units[page, 0, 3, 5, 2] = float("nan")
    out = _call(case).cpu().numpy()
    assert np.isnan(out[0, 0, 21])
    w, bound = case.expected(0)
    keep = np.arange(48) != 21
    assert (np.abs(out[0, 0, :48] - w[0])[keep] <= bound[0][keep]).all()
    q = case.q.clone()
    q[case.order[2], 0, 7] = float("nan")
    ends = case.row_end.copy()
    ends[2] = 30
    out = _call(case, q=q, row_end=cuda(ends)).cpu().numpy()
    assert np.isnan(out[1, 0, :30]).all() and np.isfinite(out[1, 0, 30:48]).all()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,kvq,rows,width", [(BF16, False, 1, 210), (BF16, True, 1, 210), (F32, False, 1, 210),
                                                  (BF16, False, 40, 210), (BF16, True, 40, 210), (BF16, False, 300, 210),
                                                  (BF16, True, 300, 210), (BF16, False, 700, 210), (BF16, True, 700, 210),
                                                  (F32, False, 40, 210), (F32, True, 40, 210)])
def test_special_values_stay_where_they_are(gpu_lib, rows, width, causal, dtype, kvq):
    """In each of the kernels a key that is no number spoils its own token and a row that is none the tokens that it
    sees, whether rows see all keys of a wave or not; a row with lse -inf adds nothing."""
    case = Case([200, 130, 70], [rows] * 3, (2, 1), 64, dtype, kvq, seed=35, width=width, causal=causal)
    lists = dict(row_indptr=None) if rows == 1 else {}
    keys = case.pool.clone()
    page = int(case.lists[0][4])                       # token 70
    if kvq:
        keys[page, :, 64 * 8:].view(1, 16, 2)[:, 6] = 255
    else:
        e = 16 // dtype.itemsize
        keys.view(len(keys), 1, 64 // e, 16, e)[page, 0, 1, 6, 2] = float("nan")
    others = np.arange(200) != 70
    case.row_end[0] = 200                              # (a row sees that token)
    out = _call(case, k_pool=keys, row_end=cuda(case.row_end), **lists).double().cpu().numpy()
    want, bound = case.expected(0)
    assert np.isnan(out[0, 0, 70]) and (np.abs(out[0, :, :200] - want)[:, others] <= bound[:, others]).all()
    for i, n in ((1, 130), (2, 70)):
        want, bound = case.expected(i)
        assert (np.abs(out[i, :, :n] - want) <= bound).all()
    # the middle row of sequence 1: no number, then without a key that it saw
    e = rows + rows // 2
    q, lse = case.q.clone(), case.lse.clone()
    q[case.order[e], 1, 9] = float("nan")
    for end in (130, 50):
        ends = case.row_end.copy()
        ends[e] = end
        out = _call(case, q=q, row_end=cuda(ends), **lists).double().cpu().numpy()
        entries = [x for x in range(rows, 2 * rows) if x != e]
        want, bound = case.expected(1, entries=entries, row_end=ends)
        assert np.isnan(out[1, 0, :end]).all() and (np.abs(out[1, :, end:130] - want[:, end:]) <= bound[:, end:]).all()
        for i, n in ((0, 200), (2, 70)):
            want, bound = case.expected(i)
            assert (np.abs(out[i, :, :n] - want) <= bound).all()
    lse[case.order[e]] = -float("inf")
    case.check(_call(case, q=q, lse=lse, **lists), which=[(1, 130)], entries=entries)


def test_large_scores(gpu_lib):
    """Scores of hundreds: few tokens hold all of a row's weight."""
    case = Case([100, 300], [10, 20], (4, 2), 128, BF16, seed=12, strong=60.0)
    case.check(_call(case))
    case = Case([100, 300], [10, 20], (4, 2), 64, F32, seed=12, strong=60.0)
    case.check(_call(case))


@pytest.mark.parametrize("kvq", [False, True])
def test_what_does_not_fit_is_flagged(gpu_lib, kvq):
    """Malformed sequences, pages, entries: left out, flagged, and nothing else is touched."""
    case = Case([40, 50, 60, 70, 80], [3, 2, 4, 3, 2], kvq=kvq, seed=13)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(expect_flag=1, **given):
        flag.zero_()
        out = _call(case, error_flag=flag, **given)
        assert int(flag) == expect_flag
        return out

    case.check(run(0))
    ends = np.array(case.lengths)
    for bad in (-1, case.width + 1, 49 + 16):       # negative, past the rows, past the pages
        e = ends.copy()
        e[1] = bad
        out = run(seq_end=cuda(e))
        case.check(out, which=[(0, 40), (2, 60), (3, 70), (4, 80)])
        assert (out[1] == -7.0).all()
    ids = case.ids.clone()
    for bad in (-1, len(case.pool), 2 ** 31 - 1):
        ids[4] = bad                                  # the second page of sequence 1
        out = run(page_ids=ids)
        case.check(out, which=[(0, 40), (2, 60), (3, 70), (4, 80)])
        got = out[1].double().cpu().numpy()
        w, bound = case.expected(1)
        seen = np.r_[0:16, 32:50]
        assert (np.abs(got[:, seen] - w[:, seen]) <= bound[:, seen]).all() and (got[:, 16:32] == -7.0).all()
    order = case.order.copy()
    for bad in (-1, len(case.q), 2 ** 31 - 1, -2 ** 31):
        order[4] = bad                                # the second row of sequence 1
        out = run(rows=cuda(order))
        case.check(out, which=[(0, 40), (2, 60), (3, 70), (4, 80)])
        case.check(out, which=[(1, 50)], entries=[3])
    for bad in (-3, 15, 2 ** 31 - 1):                 # (sequences 1 and 2 have no rows then, one way or the other)
        indptr = case.row_indptr.copy()
        indptr[2] = bad
        out = run(row_indptr=cuda(indptr))
        case.check(out, which=[(0, 40), (3, 70), (4, 80)])
        case.check(out, which=[(1, 50), (2, 60)], entries=[])
    out = run(params=params(4, 2, 128, BF16, 0))      # a pool of no pages
    assert (out == -7.0).all()


@pytest.mark.parametrize("rows", [1, 3, 40, 700])
def test_tokens_without_pages_are_flagged(gpu_lib, rows):
    """A sequence of no pages at all whose end says that it has tokens: skipped and flagged; without any it is not."""
    for at in (0, 1, 2):
        lengths = [30, 20]
        lengths.insert(at, 0)
        case = Case(lengths, [rows] * 3, (2, 1), 64, BF16, seed=28)
        ends = list(lengths)
        for end, want in ((0, 0), (5, 1), (-1, 1)):
            ends[at] = end
            flag = torch.zeros(1, dtype=torch.int32, device="cuda")
            lists = dict(row_indptr=None) if rows == 1 else {}
            case.check(_call(case, seq_end=cuda(ends), error_flag=flag, **lists))
            assert int(flag) == want, (at, end)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    none = Case([0, 0], [rows] * 2, (2, 1), 64, BF16, seed=29)
    none.check(_call(none, page_ids=cuda([0]), seq_end=cuda([0, 3]), error_flag=flag))
    assert int(flag) == 1


@pytest.mark.parametrize("dtype,rows", [(F32, 3), (BF16, 3), (BF16, 40), (BF16, 700)])
def test_entries_of_a_sequence_without_tokens_are_checked(gpu_lib, rows, dtype):
    """The last sequence has no pages, no tokens and entries that are no range of the list."""
    case = Case([30, 20, 0], [rows] * 3, (2, 1), 64, dtype, seed=34)
    for end, want in ((3 * rows, 0), (2 * rows, 0), (2 * rows - 1, 1), (3 * rows + 1, 1), (-3, 1), (2 ** 31 - 1, 1)):
        indptr = case.row_indptr.copy()
        indptr[3] = end
        flag = torch.zeros(1, dtype=torch.int32, device="cuda")
        case.check(_call(case, row_indptr=cuda(indptr), error_flag=flag))
        assert int(flag) == want, end


@pytest.mark.parametrize("dtype,rows", [(F32, 1), (F32, 3), (BF16, 1), (BF16, 3), (BF16, 40), (BF16, 700)])
@pytest.mark.parametrize("bad", [-1, -2, -2 ** 31, 5, 2 ** 31 - 1])
def test_any_bad_page_is_flagged(gpu_lib, bad, dtype, rows):
    case = Case([30, 20], [rows] * 2, (2, 1), 64, dtype, seed=30, extra_pages=1)
    assert len(case.pool) == 5
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    ids = case.ids.clone()
    ids[3] = bad                                          # the second page of the second sequence
    out = _call(case, page_ids=ids, error_flag=flag, **(dict(row_indptr=None) if rows == 1 else {}))
    assert int(flag) == 1 and (out[1, :, 16:] == -7.0).all()
    want, bound = case.expected(1)
    assert (np.abs(out[1, :, :16].double().cpu().numpy() - want[:, :16]) <= bound[:, :16]).all()
    case.check(out, which=[(0, 30)])


def test_no_lists_and_too_few_rows(gpu_lib):
    case = Case([40, 50], [1, 1], seed=14)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = _call(case, row_indptr=None, rows=None, row_end=None, q=case.q[:1].contiguous(), error_flag=flag)
    assert int(flag) == 1
    old = case.old[1, :, :50].cpu() * 0.75
    old[:, max(case.start[1], 0):] = 0
    assert torch.equal(out[1, :, :50].cpu(), old)


def test_rows_of_weights_past_32_bits(gpu_lib):
    """The second sequence's weights begin past 2^32 bytes."""
    width = (1 << 29) + 100
    case = Case([300, 300], [2, 2], (2, 2), 64, BF16, seed=15, width=320)
    out = torch.empty((2, 2, width), device="cuda")
    out[:, :, :340] = -7.0
    _call(case, weights=None, weights_out=out, decay=0.0)
    case.check(out[:, :, :340], decay=0.0)


@pytest.mark.parametrize("rows,lists,kvq", [(1, False, True), (2, True, False), (40, True, True), (700, True, False)])
def test_page_lists_past_32_bits(gpu_lib, rows, lists, kvq):
    """A list of more pages than a sequence has, whose last ones would begin past token 2^31: they are not looked at."""
    case = Case([100, 40], [rows] * 2, (2, 1), 64, BF16, kvq, seed=33, width=200)
    much = (1 << 27) + 50
    ids = torch.full((much + 3,), -1, dtype=torch.int32, device="cuda")
    ids[:7], ids[much:] = cuda(case.lists[0]), cuda(case.lists[1])
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = _call(case, page_ids=ids, seq_page_indptr=cuda([0, much, much + 3]), error_flag=flag,
                **({} if lists else dict(row_indptr=None)))
    assert int(flag) == 0
    case.check(out)


def test_pools_past_32_bits(gpu_lib):
    """Pages behind 2^32 bytes of a pool."""
    case = Case([300, 64], [4, 2], (8, 8), 128, BF16, seed=16)
    pages = (1 << 32) // (8 * 16 * 128 * 2) + 40
    pool = torch.empty((pages, 8, 16 * 128), dtype=BF16, device="cuda")
    shift = pages - len(case.pool)
    pool[shift:] = case.pool
    pool[:len(case.pool)] = float("nan")
    out = _call(case, k_pool=pool, page_ids=case.ids + shift, params=params(8, 8, 128, BF16, pages))
    case.check(out)


def test_long_sequence(gpu_lib):
    case = Case([20000, 5], [2, 1], (4, 1), 64, BF16, seed=17)
    case.check(_call(case))


@pytest.mark.parametrize("rows", [[1] * 6, [40, 0, 3, 100, 1, 17]])
def test_repeats_are_bitwise_equal_on_any_stream_and_in_graphs(gpu_lib, rows):
    case = Case([100, 1, 33, 260, 16, 70], rows, (8, 2), 128, BF16, seed=18)
    want = _call(case)
    side = torch.cuda.Stream()
    a = case.arguments()
    side.wait_stream(torch.cuda.current_stream())
    halo.kv_page_weights(**a, stream=side)
    side.synchronize()
    assert torch.equal(a["weights_out"], want)
    graph = torch.cuda.CUDAGraph()
    b = case.arguments()
    call = None
    with torch.cuda.graph(graph):
        call = halo.bind_kv_page_weights(**b)
        call()
    for _ in range(3):
        b["weights_out"].fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b["weights_out"], want)
        assert torch.equal(_call(case), want)


def test_weights_of_attention(gpu_lib):
    """The lse that decode attention gives: the weights of a decode step sum to the
    number of q heads of a kv head."""
    rng = np.random.default_rng(19)
    lengths = rng.integers(20, 300, 9)
    case = Case(lengths, [1] * 9, (8, 2), 128, BF16, seed=19, causal=False)
    case.pool.nan_to_num_()
    pages = [len(x) for x in case.lists]
    forest = dict(seg_len=lengths, seg_page_indptr=np.cumsum([0] + pages), seg_page_ids=np.concatenate(case.lists),
                  req_seg_indptr=np.arange(10), req_seg_ids=np.arange(9))
    att = halo.PrefixAttention(case.params, forest)
    q = case.q[:9].contiguous()
    _, lse = att.run(q, case.pool, torch.zeros_like(case.pool))
    out = torch.zeros_like(case.old)
    halo.kv_page_weights(out, case.pool, case.params, case.ids, case.indptr, None, cuda(lengths), q, lse)
    assert torch.allclose(out.double().sum(2), torch.full((9, 2), 4.0, dtype=torch.float64, device="cuda"), rtol=1e-5)
