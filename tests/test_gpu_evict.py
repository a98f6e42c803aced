"""kv_evict_select, kv_page_keep_kv, kvq_page_keep_kv and kv_release_pages on
the GPU: which tokens stay, where their bits go and which pages come back, equal
to the oracle's, with everything else left as it was."""

import numpy as np
import pytest
import torch

from oracle import upkeep
from paper_2509_02121_amd import halo
from upkeep_helpers import BF16, F32, cuda, csr, params, random_pool, read_bits, to_numpy, write_bits

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ which tokens stay

def _weights(rng, n, h, width, kind):
    w = np.exp(2 * rng.normal(size=(n, h, width))).astype(np.float32)
    if kind == "ties":
        w = np.round(w)
    elif kind == "equal":
        w[:] = 0.25
    elif kind == "special":
        pick = rng.integers(0, 9, w.shape)
        for i, x in enumerate((np.nan, np.inf, -np.inf, -0.0, 0.0, 1e-42, -3.0)):
            w[pick == i] = x
        w[0, 0, ::7] = -np.float32("nan")
    elif kind == "rising":
        w = np.broadcast_to(np.arange(width, dtype=np.float32), w.shape).copy()
    return w


def check_evict(n, h, lengths, budget, trigger=None, sinks=0, recent=0, kind="random", seed=0, width=None, in_place=False,
                flagged=False):
    rng = np.random.default_rng(seed)
    width = max(max(lengths, default=0), 0) + 3 if width is None else width
    w = _weights(rng, n, h, width, kind)
    wt = torch.from_numpy(w).cuda()
    kept = torch.full((n, h, budget), -5, dtype=torch.int32, device="cuda")
    new_len = torch.full((n,), -5, dtype=torch.int32, device="cuda")
    out = None if in_place else torch.full_like(wt, -7.0)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    halo.kv_evict_select(wt, cuda(lengths), kept, new_len, trigger=trigger, sinks=sinks, recent=recent, weights_out=out,
                         error_flag=flag)
    torch.cuda.synchronize()
    assert int(flag) == int(flagged)
    kept, new_len = kept.cpu().numpy(), new_len.cpu().numpy()
    got = (wt if in_place else out).cpu().numpy()
    for i, a in enumerate(lengths):
        for j in range(h):
            bad = a < 0 or a > width
            want = None if bad else upkeep.evict(w[i, j], a, budget, budget if trigger is None else trigger, sinks, recent)
            if want is None:
                assert new_len[i] == a and (kept[i, j] == -5).all()
                assert np.array_equal(got[i, j, :0 if bad else a].view(np.uint32), w[i, j, :0 if bad else a].view(np.uint32))
                m = 0 if bad else a
            else:
                assert new_len[i] == budget and kept[i, j].tolist() == want
                assert np.array_equal(got[i, j, :budget].view(np.uint32), w[i, j, want].view(np.uint32))
                m = budget
            if not in_place:
                assert (got[i, j, m:] == -7.0).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "special", "rising"])
def test_evict(gpu_lib, kind, in_place):
    lengths = [0, 1, 7, 8, 9, 15, 16, 17, 63, 64, 65, 100, 255, 256, 257, 1023, 1024, 1025, 3000]
    check_evict(len(lengths), 3, lengths, 8, sinks=1, recent=2, kind=kind, in_place=in_place)
    check_evict(len(lengths), 1, lengths, 64, trigger=100, sinks=4, recent=32, kind=kind, in_place=in_place, seed=1)
    check_evict(len(lengths), 2, lengths, 1000, trigger=1024, sinks=0, recent=0, kind=kind, in_place=in_place, seed=2)


@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (2, 1, 1), (40, 20, 20), (40, 40, 0),
                                                 (40, 0, 40), (40, 0, 0), (41, 20, 20)])
def test_evict_edges(gpu_lib, budget, sinks, recent):
    check_evict(6, 2, [1, 2, budget, budget + 1, 500, 2100], budget, sinks=sinks, recent=recent, kind="ties", seed=budget)


@pytest.mark.parametrize("kind", ["random", "equal", "ties", "special"])
def test_evict_long(gpu_lib, kind):
    check_evict(2, 2, [150001, 70000], 8192, sinks=16, recent=1024, kind=kind, seed=3)
    check_evict(1, 1, [200000], 100001, trigger=150000, kind=kind, seed=4, in_place=True)


def test_evict_malformed_and_empty(gpu_lib):
    check_evict(4, 2, [30, -1, 34, 20], 8, width=33, flagged=True)
    check_evict(3, 2, [-2 ** 31, 2 ** 31 - 1, 25], 8, width=33, flagged=True)
    check_evict(0, 2, [], 8, width=33)
    check_evict(2, 2, [0, 0], 8, width=0)


def test_evict_repeats_in_a_graph(gpu_lib):
    w = torch.rand((5, 4, 700), device="cuda").round(decimals=2)
    n = cuda([700, 90, 128, 129, 333])

    def buffers():
        return (torch.full((5, 4, 128), -1, dtype=torch.int32, device="cuda"),
                torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros_like(w))

    def call(b):
        halo.kv_evict_select(w, n, b[0], b[1], sinks=2, recent=9, weights_out=b[2])

    want, got = buffers(), buffers()
    call(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(got)
    for _ in range(3):
        for t in got:
            t.fill_(-1 if t.dtype == torch.int32 else 0)
        graph.replay()
        torch.cuda.synchronize()
        again = buffers()
        call(again)
        for a, b, c in zip(want, got, again):
            assert torch.equal(a, b) and torch.equal(a, c)


def test_evict_as_many_rows_as_a_launch_holds(gpu_lib):
    n, h = 2 ** 16 - 1, 2 ** 8
    w = torch.rand((n, h, 2), device="cuda").round(decimals=1)
    kept = torch.full((n, h, 1), -1, dtype=torch.int32, device="cuda")
    new_len, out = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros_like(w)
    halo.kv_evict_select(w, torch.full_like(new_len, 2), kept, new_len, weights_out=out)
    assert torch.equal(kept[..., 0], (w[..., 1] > w[..., 0]).int()) and bool((new_len == 1).all())
    assert torch.equal(out[..., 0], w.amax(2)) and not bool(out[..., 1].any())


# ------------------------------------------------------------------ moving them

class Keep:
    """Sequences in pools of random bits, and kept tokens at random."""

    def __init__(self, lengths, new_lens, h=2, dim=128, dtype=BF16, kvq=False, seed=0, in_place=False, spare=2):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.h, self.dim, self.dtype, self.kvq, self.in_place = h, dim, dtype, kvq, in_place
        self.lengths, self.new_lens = list(lengths), list(new_lens)
        n = len(lengths)
        need = [upkeep.pages_of(a) + int(rng.integers(0, 2)) for a in lengths]
        dst = [upkeep.pages_of(b) + int(rng.integers(0, 2)) for b in new_lens]
        size = sum(need) + sum(dst) + spare
        ids = rng.permutation(size)
        cuts = np.cumsum([0] + need + dst)
        lists = [ids[a:b] for a, b in zip(cuts, cuts[1:])]
        self.src = lists[:n]
        self.dst = self.src if in_place else lists[n:]
        self.pools = []
        for kind in (0, 1):   # any bits: NaN payloads among them
            if kvq:
                x = torch.randint(0, 256, random_pool(kind, 1, h, dim, dtype, True, gen).shape[1:], generator=gen,
                                  device="cuda", dtype=torch.uint8)
                x = torch.randint(0, 256, (size, *x.shape), generator=gen, device="cuda", dtype=torch.uint8)
            else:
                x = torch.randint(-2 ** 31, 2 ** 31 - 1, (size, h, 16 * dim * dtype.itemsize // 4), generator=gen,
                                  device="cuda", dtype=torch.int64).to(torch.int32).view(dtype)
            self.pools.append(x)
        width = max([b for a, b in zip(lengths, new_lens) if b < a], default=1) + 2
        self.kept = np.full((n, h, width), -1, np.int32)
        for i, (a, b) in enumerate(zip(lengths, new_lens)):
            for j in range(h):
                if b < a:
                    self.kept[i, j, :b] = np.sort(rng.permutation(a)[:b])
        self.params = params(h, h, dim, dtype, size)

    def bits(self, kind):
        x = to_numpy(self.pools[kind])
        return x.view(np.uint32) if x.dtype == np.float32 else x

    def expected(self, skip_sequences=(), skip_tokens=()):
        out = []
        for kind in (0, 1):
            x = self.bits(kind)
            y = x.copy()
            for i, (a, b) in enumerate(zip(self.lengths, self.new_lens)):
                if i in skip_sequences or (a == b and self.in_place):
                    continue
                for j in range(self.h):
                    for t in range(b):
                        s = int(self.kept[i, j, t]) if b < a else t
                        if (i, j, t) in skip_tokens:
                            continue
                        bits = read_bits(x[self.src[i][s // 16], j], s % 16, kind, self.dim, self.kvq)
                        write_bits(y[self.dst[i][t // 16], j], t % 16, bits, kind, self.dim, self.kvq)
            out.append(y)
        return out

    def call(self, **given):
        indptr, ids = csr(self.src)
        a = dict(k_pool=self.pools[0], v_pool=self.pools[1], params=self.params, page_ids=ids, seq_page_indptr=indptr,
                 seq_len=cuda(self.lengths), new_len=cuda(self.new_lens), kept=cuda(self.kept))
        if not self.in_place:
            a["dst_page_indptr"], a["dst_page_ids"] = csr(self.dst)
        a.update(given)
        (halo.kvq_page_keep_kv if self.kvq else halo.kv_page_keep_kv)(**a)
        torch.cuda.synchronize()

    def check(self, want):
        for kind, y in enumerate(want):
            got = self.bits(kind)
            assert np.array_equal(got, y), f"pool {kind}: {np.argwhere(got != y)[:5]} of {got.shape}"


LENGTHS = [0, 1, 5, 16, 17, 40, 64, 100, 33, 129]
NEW = [0, 1, 3, 16, 16, 17, 20, 99, 1, 31]
FORMATS = [(BF16, False), (F32, False), (BF16, True), (F32, True)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,kvq", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("h", [1, 3])
def test_keep(gpu_lib, h, dim, dtype, kvq, in_place):
    case = Keep(LENGTHS, NEW, h, dim, dtype, kvq, seed=h + dim, in_place=in_place)
    want = case.expected()
    case.call()
    case.check(want)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kvq", [False, True])
def test_keep_many_pages(gpu_lib, kvq, in_place):
    """Kept tokens from the whole of a long sequence, and nearly all of one."""
    case = Keep([1500, 1200, 700], [600, 1190, 699], 2, 64, BF16, kvq, seed=5, in_place=in_place)
    want = case.expected()
    case.call()
    case.check(want)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kvq", [False, True])
def test_keep_slices_of_longer_lists(gpu_lib, kvq, in_place):
    """Old and new lists that begin inside of their arrays."""
    case = Keep([100, 0, 33, 64], [40, 0, 33, 20], 2, 64, BF16, kvq, seed=10, in_place=in_place)
    want = case.expected()
    pad = torch.full((5,), -9, dtype=torch.int32, device="cuda")
    given = {}
    for names, lists in ((("seq_page_indptr", "page_ids"), case.src), (("dst_page_indptr", "dst_page_ids"), case.dst)):
        indptr, ids = csr(lists)
        given[names[0]], given[names[1]] = indptr + 5, torch.cat([pad, ids])
    if in_place:
        given["dst_page_indptr"], given["dst_page_ids"] = given["seq_page_indptr"], given["page_ids"]
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    case.call(error_flag=flag, **given)
    case.check(want)
    assert int(flag) == 0


def test_keep_lists_that_are_refused(gpu_lib):
    """A list of no elements, which has no address; one array for both lists with two indptr, or the other way round."""
    case = Keep([20, 33], [0, 0], seed=11)
    want = [case.bits(0), case.bits(1)]
    (indptr, ids), (dst_indptr, dst_ids) = csr(case.src), csr(case.dst)
    for given, match in ((dict(dst_page_ids=cuda([])), "dst_page_ids"), (dict(page_ids=cuda([])), "page_ids"),
                         (dict(page_ids=ids, dst_page_ids=ids), "in place"),
                         (dict(seq_page_indptr=indptr, dst_page_indptr=indptr), "in place")):
        with pytest.raises(halo.HaloError, match=match):
            case.call(**given)
    case.check(want)


@pytest.mark.parametrize("kvq", [False, True])
def test_keep_nothing(gpu_lib, kvq):
    """A sequence that keeps no token, none at all, and rows of no width."""
    case = Keep([20, 33], [0, 0], kvq=kvq, seed=6)
    want = [case.bits(0), case.bits(1)]
    case.call()
    case.check(want)
    case.call(seq_len=cuda([0, 0]), kept=torch.zeros((2, 2, 0), dtype=torch.int32, device="cuda"))
    case.check(want)


@pytest.mark.parametrize("kvq", [False, True])
def test_keep_what_does_not_fit_is_flagged(gpu_lib, kvq):
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")

    def fresh():
        flag.zero_()
        return Keep([40, 50, 70], [18, 35, 70], kvq=kvq, seed=7)

    case = fresh()
    want = case.expected()
    case.call(error_flag=flag)
    case.check(want)
    assert int(flag) == 0
    for name, bad in (("seq_len", [40, -1, 70]), ("seq_len", [40, 34, 70]), ("seq_len", [40, 16 * 5 + 1, 70]),
                      ("new_len", [18, -1, 70]), ("new_len", [18, 49, 70]), ("new_len", [18, 2 ** 31 - 1, 70])):
        case = fresh()
        want = case.expected(skip_sequences=[1])
        case.call(error_flag=flag, **{name: cuda(bad)})
        case.check(want)
        assert int(flag) == 1
    for bad in (-1, 50, 2 ** 31 - 1, -2 ** 31):
        case = fresh()
        case.kept[1, 0, 20] = bad
        want = case.expected(skip_tokens=[(1, 0, 20)])
        case.call(error_flag=flag)
        case.check(want)
        assert int(flag) == 1
    for bad in (-1, len(case.pools[0]), 2 ** 31 - 1):
        case = fresh()
        gone = [(1, j, t) for j in range(2) for t in range(35) if case.kept[1, j, t] // 16 == 1]
        want = case.expected(skip_tokens=gone)
        lists = [x.copy() for x in case.src]
        lists[1][1] = bad
        case.call(error_flag=flag, page_ids=csr(lists)[1])
        case.check(want)
        assert int(flag) == 1
        case = fresh()
        want = case.expected(skip_tokens=[(1, j, t) for j in range(2) for t in range(16, 32)])
        lists = [x.copy() for x in case.dst]
        lists[1][1] = bad
        case.call(error_flag=flag, dst_page_ids=csr(lists)[1])
        case.check(want)
        assert int(flag) == 1
    case = fresh()
    want = [case.bits(0), case.bits(1)]
    case.call(error_flag=flag, params=params(2, 2, 128, BF16, 0))
    case.check(want)
    assert int(flag) == 1


def test_keep_in_place_of_as_many_rows_as_a_launch_holds(gpu_lib):
    """2^21 - 256 (sequence, head) pairs, of which the last sequence's keep their second token."""
    n, h = 2 ** 13 - 1, 2 ** 8
    pool = torch.randn((1, h, 16 * 64), device="cuda").to(BF16)
    want = pool.clone()
    k = want.view(h, 8, 16, 8)
    k[:, :, 0] = k[:, :, 1]
    got = pool.clone()
    v = torch.zeros_like(pool)
    lengths, new = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    lengths[-1], new[-1] = 2, 1
    indptr = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    indptr[-1] = 1
    kept = torch.ones((n, h, 1), dtype=torch.int32, device="cuda")
    halo.kv_page_keep_kv(got, v, params(h, h, 64, BF16, 1), cuda([0]), indptr, lengths, new, kept)
    assert torch.equal(got, want)


def test_keep_pools_past_32_bits(gpu_lib):
    pages = (1 << 32) // (8 * 16 * 128 * 2) + 200
    case = Keep([500, 90], [200, 64], 8, 128, BF16, seed=8)
    want = case.expected()
    shift = pages - len(case.pools[0])
    big = [torch.empty((pages, 8, 16 * 128), dtype=BF16, device="cuda") for _ in range(2)]
    for x, y in zip(big, case.pools):
        x[shift:] = y
    case.src, case.dst = [x + shift for x in case.src], [x + shift for x in case.dst]
    small, case.pools = case.pools, big
    case.params = params(8, 8, 128, BF16, pages)
    case.call()
    case.pools = [x[shift:] for x in big]
    case.check(want)
    assert len(small) == 2


@pytest.mark.parametrize("in_place", [False, True])
def test_keep_in_a_graph_and_on_a_stream(gpu_lib, in_place):
    case = Keep([100, 300], [50, 200], seed=9, in_place=in_place)
    want = case.expected()
    start = [x.clone() for x in case.pools]
    indptr, ids = csr(case.src)
    more = {} if in_place else dict(zip(("dst_page_indptr", "dst_page_ids"), csr(case.dst)))
    a = dict(k_pool=case.pools[0], v_pool=case.pools[1], params=case.params, page_ids=ids, seq_page_indptr=indptr,
             seq_len=cuda(case.lengths), new_len=cuda(case.new_lens), kept=cuda(case.kept), **more)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    halo.kv_page_keep_kv(**a, stream=side)
    side.synchronize()
    case.check(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        halo.kv_page_keep_kv(**a)
    for _ in range(3):
        for x, y in zip(case.pools, start):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        case.check(want)


# ------------------------------------------------------------------ pages given back

def check_release(lengths, new, free_next, num_free, in_place, width=None, seed=0, flagged=False):
    rng = np.random.default_rng(seed)
    n = len(lengths)
    width = max([upkeep.pages_of(max(a, 0)) for a in lengths] + [1]) if width is None else width
    table = rng.integers(0, 10 ** 6, (n, width)).astype(np.int32)
    free = rng.integers(0, 10 ** 6, num_free).astype(np.int32)
    want, want_next, want_flag = upkeep.release(table, lengths, new, free.tolist(), free_next)
    assert want_flag == flagged
    free_t = cuda(free)
    out = free_t if in_place else torch.full_like(free_t, -9)
    next_out, flag = cuda([-9]), cuda([0])
    table_t = cuda(table)
    halo.kv_release_pages(table_t, cuda(lengths), cuda(new), free_t, cuda([free_next]), out, next_out, error_flag=flag)
    torch.cuda.synchronize()
    assert int(next_out) == want_next and int(flag) == int(flagged) and torch.equal(table_t, cuda(table))
    got = out.cpu().numpy()
    if in_place:
        assert got.tolist() == want
    elif 0 <= free_next <= num_free:
        assert got[want_next:].tolist() == want[want_next:] and (got[:want_next] == -9).all()
    else:
        assert (got == -9).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n", [1, 3, 255, 256, 257, 1000, 5000])
def test_release(gpu_lib, n, in_place):
    rng = np.random.default_rng(n)
    lengths = rng.integers(0, 400, n)
    new = (lengths * rng.choice([0.0, 0.5, 0.9, 1.0], n)).astype(int)
    total = sum(upkeep.pages_of(a) - upkeep.pages_of(b) for a, b in zip(lengths, new))
    check_release(lengths, new, total, total + 5, in_place)
    check_release(lengths, new, total + 3, total + 3, in_place, seed=1)
    check_release(lengths, new, total - 1, total + 9, in_place, flagged=True) if total else None


@pytest.mark.parametrize("in_place", [False, True])
def test_release_edges(gpu_lib, in_place):
    check_release([], [], 3, 5, in_place)
    check_release([], [], 0, 0, in_place)
    check_release([160, 16, 17], [0, 16, 16], 100, 30000, in_place)     # a long list is passed on
    check_release([50, -1, 60, 30, 97], [20, -1, 70, 20, 3], 9, 9, in_place, width=6, flagged=True)
    check_release([50, 2 ** 31 - 1], [20, 0], 9, 9, in_place, width=6, flagged=True)
    for bad in (-1, 10, -2 ** 31, 2 ** 31 - 1):
        check_release([50], [20], bad, 9, in_place, flagged=True)
    check_release([0, 0], [0, 0], 2, 4, in_place, width=0)


def test_release_is_the_inverse_of_the_step_tables(gpu_lib):
    """Pages that a step takes and a release gives back are the list's next ones again."""
    n = 40
    rng = np.random.default_rng(2)
    lengths = rng.integers(1, 100, n)
    new = rng.integers(0, 60, n)
    table = cuda(np.arange(n * 12).reshape(n, 12))
    free, first = cuda(rng.permutation(400) + 1000), cuda([7])
    t = halo.StepTables(n, 3000, 1000)
    halo.kv_step_tables(t, cuda(lengths), cuda(new), table, free, first)
    out, back = torch.full_like(free, -1), cuda([0])
    halo.kv_release_pages(table, t.seq_end, cuda(lengths), free, t.free_next, out, back)
    assert int(back) == 7 and torch.equal(out[7:], free[7:])
