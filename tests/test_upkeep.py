"""CPU tests of the operators between two steps: the oracle's pins, and the
library's and the binding's refusals (no GPU is touched)."""

import ctypes
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import upkeep
from paper_2509_02121_amd import halo

BAD, UNSUPPORTED, SMALL = (halo.HALO_ERR_INVALID_ARGUMENT, halo.HALO_ERR_UNSUPPORTED,
                           halo.HALO_ERR_WORKSPACE_TOO_SMALL)


@pytest.fixture(scope="module")
def lib():
    return halo.load_library()


# ------------------------------------------------------------------ the oracle

def test_weights_by_hand():
    # two keys, one head of one dim: scores ln 1 and ln 3, lse ln 4
    keys = np.array([[[0.0]], [[math.log(3.0)]]])
    w, _, _ = upkeep.weights(keys, np.array([[[1.0]]]), np.array([[math.log(4.0)]]), [2], 1.0, np.array([[8.0, 8.0]]), 1, 0.5)
    assert np.allclose(w, [[0.25 + 4.0, 0.75]], rtol=1e-15)


def test_weights_of_a_row_sum_to_one():
    rng = np.random.default_rng(0)
    k, q = rng.normal(size=(40, 2, 8)), rng.normal(size=(5, 6, 8))
    _, lse = oracle.decode(q, {0: k}, {0: k}, [[0]] * 5, 0.3)
    w, _, _ = upkeep.weights(k, q, lse, [40] * 5, 0.3, np.zeros((2, 40)), 0, 0.0)
    assert np.allclose(w.sum(1), 15.0)
    probs = sum(oracle.attention_probs(q[r, g][None], k[:, 0], 0.3)[0] for r in range(5) for g in range(3))
    assert np.allclose(w[0], probs)


def test_weights_of_rows_that_see_nothing():
    k = np.ones((3, 1, 2))
    q, lse = np.ones((2, 1, 2)), np.array([[-np.inf], [0.0]])
    w, _, _ = upkeep.weights(k, q, lse, [3, 0], 1.0, np.full((1, 3), 2.0), 3, 1.0)
    assert (w == 2.0).all()


def test_evict_by_hand():
    w = [9.0, 1.0, 5.0, 5.0, float("nan"), 2.0, 0.0]
    assert upkeep.evict(w, 7, 4, 4, 1, 1) == [0, 2, 3, 6]
    assert upkeep.evict(w, 7, 3, 3, 1, 1) == [0, 2, 6]        # equal weights: the earlier token
    assert upkeep.evict(w, 7, 6, 6, 0, 0) == [0, 1, 2, 3, 5, 6]
    assert upkeep.evict(w, 7, 4, 7, 1, 1) is None
    assert upkeep.evict(w, 7, 2, 3, 1, 1) == [0, 6]


def test_release_by_hand():
    table = [[4, 5, 6, -1], [7, 8, -1, -1]]
    assert upkeep.release(table, [33, 20], [16, 20], [9, 9, 9, 1], 3) == ([9, 5, 6, 1], 1, False)
    assert upkeep.release(table, [33, 20], [0, 0], [9, 9, 9, 1], 3) == ([9, 9, 9, 1], 3, True)
    assert upkeep.release(table, [65, 20], [0, 0], [9, 9, 9, 1], 3) == ([9, 7, 8, 1], 1, True)


def test_select_by_hand():
    ln = math.log
    logits = [[ln(1), ln(3), -np.inf], [ln(2), ln(2), ln(4)], [0, 0, 0]]
    s, t, p = upkeep.select(logits, [0.0, ln(0.4), -np.inf], None, 0, 4)
    assert t == [1, 0, 2, 0] and p == [0, 0, 1, 1]     # (the last: ties, the lower token)
    assert np.allclose(np.exp(s), [0.75, 0.25, 0.2, 0.1])
    s, t, p = upkeep.select([logits[1]] * 2, [-1.0, -1.0], None, 0, 3)
    assert t == [2, 2, 0] and p == [0, 1, 0]           # (ties: the lower beam)
    s, t, p = upkeep.select(logits, [ln(0.3), ln(0.5), -1.0], [1, 0, 1], 2, 3)
    assert t == [2, 2, 2] and p == [2, 0, 1]
    assert upkeep.select(logits, [-np.inf] * 3, None, 0, 2) == ([-np.inf] * 2, [-1, -1], [-1, -1])


def test_select_of_logits_that_are_all_the_lowest_number():
    """Each of n tokens has 1 / n of the beam, also where ln n is nothing beside the logits."""
    low = float(np.finfo(np.float32).min)
    s, t, p = upkeep.select([[low] * 4, [0.0] * 3 + [-np.inf]], [-1.0, -1.0], None, 0, 4)
    assert t == [0, 1, 2, 0] and p == [1, 1, 1, 0]
    assert np.allclose(s, [-1 - math.log(3)] * 3 + [-1 - math.log(4)], rtol=1e-15)


def test_beam_tables_by_hand():
    # beams 0 and 1 share page 3; both go on from beam 1, whose page 5 is partly filled
    new = upkeep.beam_tables(1, 2, [[1, 1]], [20, 20], [[3, 4, -1], [3, 5, -1]], [8, 6, 7], 1)
    assert new == ([[3, 5], [3, 6]], [20, 20], [8, 4, 7], 1, [-1, 5], [-1, 6], False)
    new = upkeep.beam_tables(1, 2, [[1, -1]], [32, 32], [[3, 4, -1], [3, 5, -1]], [8, 6, 7], 1)
    assert new == ([[3, 5], []], [32, 0], [4, 6, 7], 0, [-1, -1], [-1, -1], False)
    # no room for a copy: as it was
    new = upkeep.beam_tables(1, 2, [[1, 1]], [20, 20], [[3, 4, -1], [3, 5, -1]], [8], 1)
    assert new == ([[3, 4], [3, 5]], [20, 20], [8], 1, [-1, -1], [-1, -1], True)


# ------------------------------------------------------------------ refusals of the C ABI

def _params(**given):
    p = dict(num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, num_pool_pages=3, kv_dtype=halo.HALO_BF16,
             out_dtype=halo.HALO_BF16, sm_scale=0.125)
    p.update(given)
    return halo.AttnParams(**p)


class Buffers:
    """Host memory in the place of device arrays: what is refused is not read."""

    def __init__(self, *names):
        self.room = {n: np.zeros(1 << 16, np.uint8) for n in names}
        self.at = {n: (b.ctypes.data + 255) // 256 * 256 for n, b in self.room.items()}

    def take(self, none=(), same=None, **offset):
        at = {n: None if n in none else a for n, a in self.at.items()}
        for n, other in (same or {}).items():
            at[n] = at[other]
        for n, by in offset.items():
            at[n] += by
        return at


WEIGHTS = ("k_pool", "page_ids", "indptr", "start", "end", "row_indptr", "rows", "row_end", "q", "lse", "weights",
           "out", "flag")


def _weights_call(lib, params=None, sizes=(2, 3, 4, 40), decay=1.0, kvq=False, none=(), same=None, **offset):
    bufs = Buffers(*WEIGHTS)
    a = bufs.take(none, same, **offset)
    p, s = _params(**(params or {})), halo.WeightSizes(*sizes)
    fn = lib.halo_kvq_page_weights if kvq else lib.halo_kv_page_weights
    return fn(a["k_pool"], ctypes.byref(p), ctypes.byref(s), a["page_ids"], a["indptr"], a["start"], a["end"],
              a["row_indptr"], a["rows"], a["row_end"], a["q"], a["lse"], decay, a["weights"], a["out"], a["flag"], None)


@pytest.mark.parametrize("kvq", [False, True])
def test_weights_refusals(lib, kvq):
    def call(*a, **k):
        return _weights_call(lib, *a, kvq=kvq, **k)

    for name in ("k_pool", "page_ids", "indptr", "end", "q", "lse", "out", "weights"):
        assert call(none=(name,)) == BAD, name
    for params, want in (({"head_dim": 96}, UNSUPPORTED), ({"page_size": 32}, UNSUPPORTED), ({"kv_dtype": 7}, UNSUPPORTED),
                         ({"num_kv_heads": 0}, BAD), ({"num_q_heads": 3}, BAD), ({"num_q_heads": 1}, BAD),
                         ({"num_kv_heads": 65537, "num_q_heads": 65537}, UNSUPPORTED), ({"num_pool_pages": -1}, BAD),
                         ({"num_pool_pages": 2 ** 31}, UNSUPPORTED), ({"sm_scale": 0.0}, BAD),
                         ({"sm_scale": math.nan}, BAD), ({"sm_scale": math.inf}, BAD)):
        assert call(params) == want, params
    for sizes in ((-1, 3, 4, 40), (2, -1, 4, 40), (2, 3, -1, 40), (2, 3, 4, -1)):
        assert call(sizes=sizes) == BAD
    for decay in (-0.5, math.nan, math.inf):
        assert call(decay=decay) == BAD
    assert call(sizes=(2, 3, (2 ** 31 - 1024) // 2, 40)) == UNSUPPORTED  # (entries times q heads of a kv head)
    assert call(sizes=(2, 3, 1, 40), none=("row_indptr",)) == BAD        # an entry for each sequence
    assert call(k_pool=8) == BAD and call(q=2) == BAD
    for written in ("out", "flag"):
        for other in ("k_pool", "q", "lse", "indptr", "start", "end", "row_indptr", "rows", "row_end"):
            assert call(same={written: other}) == BAD, (written, other)
            assert b"overlap" in lib.halo_last_error_message()
    assert call(same={"weights": "out"}, out=4) == BAD                   # neither the same nor apart
    assert call(same={"flag": "out"}) == BAD
    fn = lib.halo_kvq_page_weights if kvq else lib.halo_kv_page_weights
    assert fn(*[None] * 12, 1.0, *[None] * 4) == BAD
    assert call(sizes=(0, 0, 0, 40)) == halo.HALO_OK and call(sizes=(2, 3, 4, 0)) == halo.HALO_OK


def _evict_call(lib, sizes=(2, 2, 40, 8, 8, 1, 2), none=(), same=None, **offset):
    a = Buffers("weights", "len", "kept", "out", "new_len", "flag").take(none, same, **offset)
    s = halo.EvictSizes(*sizes)
    return lib.halo_kv_evict_select(ctypes.byref(s), a["weights"], a["len"], a["kept"], a["out"], a["new_len"],
                                    a["flag"], None)


def test_evict_refusals(lib):
    for name in ("weights", "len", "kept", "out", "new_len"):
        assert _evict_call(lib, none=(name,)) == BAD
    for i, bad in enumerate((-1, 0, -1, 0, 7, -1, -1)):
        sizes = [2, 2, 40, 8, 8, 1, 2]
        sizes[i] = bad
        assert _evict_call(lib, tuple(sizes)) == BAD, sizes
    assert _evict_call(lib, (2, 2, 40, 8, 8, 5, 4)) == BAD
    assert _evict_call(lib, (2, 2, 40, 8, 8, 2 ** 31 - 1, 2 ** 31 - 1)) == BAD
    assert _evict_call(lib, (2 ** 20, 2 ** 8, 0, 8, 8, 1, 2)) == UNSUPPORTED
    for written, other in (("kept", "weights"), ("out", "len"), ("new_len", "len"), ("new_len", "weights"),
                           ("kept", "out"), ("flag", "kept"), ("flag", "new_len"), ("kept", "len")):
        assert _evict_call(lib, same={written: other}) == BAD
        assert b"overlap" in lib.halo_last_error_message()
    assert _evict_call(lib, same={"weights": "out"}, out=4) == BAD
    assert _evict_call(lib, (0, 2, 40, 8, 8, 1, 2)) == halo.HALO_OK
    assert lib.halo_kv_evict_select(*[None] * 8) == BAD


def test_evict_refuses_more_rows_than_a_launch_holds(lib):
    """A launch has less than 2^32 threads: 256 a row, 1024 where rows have more than 4096 tokens."""
    for sizes in ((2 ** 14, 2 ** 8, 4097, 8, 8, 1, 2), (2 ** 16, 2 ** 8, 4096, 8, 8, 1, 2), (2 ** 16, 2 ** 8, 0, 8, 8, 1, 2)):
        assert _evict_call(lib, sizes) == UNSUPPORTED, sizes
        assert b"num_seqs * num_kv_heads" in lib.halo_last_error_message()
    assert _evict_call(lib, (2 ** 14, 2 ** 8, 4096, 8, 8, 1, 2)) == BAD     # (looked at further: arrays that overlap)


def _keep_call(lib, params=None, width=8, seqs=2, kvq=False, none=(), same=None, **offset):
    a = Buffers("k", "v", "ids", "indptr", "len", "new_len", "kept", "dst_ids", "dst_indptr", "flag").take(none, same,
                                                                                                          **offset)
    p = _params(**(params or {}))
    fn = lib.halo_kvq_page_keep_kv if kvq else lib.halo_kv_page_keep_kv
    return fn(a["k"], a["v"], ctypes.byref(p), a["ids"], a["indptr"], a["len"], a["new_len"], a["kept"], width,
              a["dst_ids"], a["dst_indptr"], seqs, a["flag"], None)


@pytest.mark.parametrize("kvq", [False, True])
def test_keep_refusals(lib, kvq):
    def call(*a, **k):
        return _keep_call(lib, *a, kvq=kvq, **k)

    for name in ("k", "v", "ids", "indptr", "len", "new_len", "kept", "dst_ids", "dst_indptr"):
        assert call(none=(name,)) == BAD, name
    for params, want in (({"head_dim": 96}, UNSUPPORTED), ({"page_size": 32}, UNSUPPORTED), ({"kv_dtype": 7}, UNSUPPORTED),
                         ({"num_kv_heads": 0}, BAD), ({"num_pool_pages": -1}, BAD)):
        assert call(params) == want, params
    assert call(width=-1) == BAD and call(seqs=-1) == BAD
    assert call(seqs=2 ** 22, params={"num_kv_heads": 4}) == UNSUPPORTED
    assert call(k=4) == BAD and call(v=8) == BAD
    assert call(same={"dst_ids": "ids"}) == BAD and call(same={"dst_indptr": "indptr"}) == BAD
    assert call(seqs=0) == halo.HALO_OK
    fn = lib.halo_kvq_page_keep_kv if kvq else lib.halo_kv_page_keep_kv
    assert fn(*[None] * 8, 0, None, None, 1, None, None) == BAD


@pytest.mark.parametrize("kvq", [False, True])
def test_keep_in_place_refuses_more_rows_than_a_launch_holds(lib, kvq):
    """Two workgroups of 1024 threads a (sequence, head), and a launch has less than 2^32."""
    same = {"dst_ids": "ids", "dst_indptr": "indptr"}
    assert _keep_call(lib, {"num_kv_heads": 4}, seqs=2 ** 19, kvq=kvq, same=same) == UNSUPPORTED
    assert b"in place" in lib.halo_last_error_message()


def _release_call(lib, sizes=(2, 16, 4, 8, 0, 0), none=(), same=None, **offset):
    a = Buffers("table", "len", "new_len", "free", "next", "out", "next_out", "flag").take(none, same, **offset)
    s = halo.StepSizes(*sizes)
    return lib.halo_kv_release_pages(ctypes.byref(s), a["table"], a["len"], a["new_len"], a["free"], a["next"], a["out"],
                                     a["next_out"], a["flag"], None)


def test_release_refusals(lib):
    for name in ("table", "len", "new_len", "free", "next", "out", "next_out"):
        assert _release_call(lib, none=(name,)) == BAD
    for sizes in ((-1, 16, 4, 8, 0, 0), (2, 16, -1, 8, 0, 0), (2, 16, 4, -1, 0, 0)):
        assert _release_call(lib, sizes) == BAD
    assert _release_call(lib, (2, 32, 4, 8, 0, 0)) == UNSUPPORTED
    for written, other in (("out", "table"), ("next_out", "next"), ("out", "len"), ("next_out", "new_len"),
                           ("flag", "out"), ("next_out", "free"), ("flag", "next")):
        assert _release_call(lib, same={written: other}) == BAD
        assert b"overlap" in lib.halo_last_error_message()
    assert _release_call(lib, same={"out": "free"}, free=4) == BAD
    assert lib.halo_kv_release_pages(*[None] * 10) == BAD


def _select_call(lib, sizes=(2, 3, 100, 4, 100, halo.HALO_F32), end=5, bytes_=None, none=(), same=None, **offset):
    a = Buffers("logits", "scores", "ended", "out_scores", "tokens", "parents", "workspace").take(none, same, **offset)
    s = halo.BeamSizes(*sizes)
    need = lib.halo_beam_workspace_bytes(ctypes.byref(s))
    return lib.halo_beam_select(ctypes.byref(s), a["logits"], a["scores"], a["ended"], end, a["out_scores"], a["tokens"],
                                a["parents"], a["workspace"], max(need, 0) if bytes_ is None else bytes_, None)


def test_select_refusals(lib):
    for name in ("logits", "scores", "out_scores", "tokens", "parents", "workspace"):
        assert _select_call(lib, none=(name,)) == BAD
    for sizes, want in (((-1, 3, 100, 4, 100, 0), BAD), ((2, 0, 100, 4, 100, 0), BAD), ((2, 3, 0, 4, 100, 0), BAD),
                        ((2, 3, 100, 0, 100, 0), BAD), ((2, 65, 100, 4, 100, 0), UNSUPPORTED),
                        ((2, 3, 100, 65, 100, 0), UNSUPPORTED), ((2, 3, 2 ** 24 + 1, 4, 2 ** 24 + 1, 0), UNSUPPORTED),
                        ((2, 3, 100, 4, 99, 0), BAD), ((2, 3, 100, 4, 100, 9), UNSUPPORTED),
                        ((22000, 3, 100, 4, 100, 0), UNSUPPORTED)):
        assert _select_call(lib, sizes) == want, sizes
        assert lib.halo_beam_workspace_bytes(ctypes.byref(halo.BeamSizes(*sizes))) == -1
    assert lib.halo_beam_workspace_bytes(None) == -1
    assert _select_call(lib, end=-1) == BAD and _select_call(lib, end=100) == BAD
    assert _select_call(lib, bytes_=10) == SMALL
    assert _select_call(lib, workspace=16) == BAD and _select_call(lib, logits=2) == BAD
    for written, other in (("out_scores", "scores"), ("tokens", "logits"), ("parents", "ended"), ("workspace", "logits"),
                           ("tokens", "parents"), ("workspace", "out_scores")):
        assert _select_call(lib, same={written: other}) == BAD
        assert b"overlap" in lib.halo_last_error_message()
    assert _select_call(lib, (0, 3, 100, 4, 100, 0)) == halo.HALO_OK
    assert lib.halo_beam_select(None, None, None, None, 0, None, None, None, None, 0, None) == BAD


TABLES = ("block_table", "seq_len", "free_pages", "free_next", "copy_src", "copy_dst")


def _tables_call(lib, sizes=(2, 3, 16, 4, 8, 3), bytes_=None, none=(), same=None, **offset):
    a = Buffers("parents", "len", "table", "free", "next", "workspace", "flag", *TABLES).take(none, same, **offset)
    s = halo.BeamTableSizes(*sizes)
    need = lib.halo_beam_tables_workspace_bytes(ctypes.byref(s))
    out = halo._BeamTables(**{n: a[n] for n in TABLES})
    return lib.halo_kv_beam_tables(ctypes.byref(s), a["parents"], a["len"], a["table"], a["free"], a["next"],
                                   ctypes.byref(out), a["workspace"], max(need, 0) if bytes_ is None else bytes_,
                                   a["flag"], None)


def test_tables_refusals(lib):
    for name in ("parents", "len", "table", "free", "next", "workspace", *TABLES):
        assert _tables_call(lib, none=(name,)) == BAD, name
    for sizes, want in (((-1, 3, 16, 4, 8, 3), BAD), ((2, 0, 16, 4, 8, 3), BAD), ((2, 65, 16, 4, 8, 65), UNSUPPORTED),
                        ((2, 3, 32, 4, 8, 3), UNSUPPORTED), ((2, 3, 16, -1, 8, 3), BAD), ((2, 3, 16, 4, -1, 3), BAD),
                        ((2, 3, 16, 4, 8, 2), BAD), ((2 ** 20 + 1, 1, 16, 1, 8, 1), UNSUPPORTED),
                        ((2 ** 20, 64, 16, 64, 8, 64), UNSUPPORTED)):
        assert _tables_call(lib, sizes) == want, sizes
        assert lib.halo_beam_tables_workspace_bytes(ctypes.byref(halo.BeamTableSizes(*sizes))) == -1
    assert _tables_call(lib, bytes_=10) == SMALL
    assert _tables_call(lib, workspace=16) == BAD
    for written, other in (("block_table", "table"), ("seq_len", "len"), ("free_pages", "free"), ("free_next", "next"),
                           ("copy_src", "parents"), ("copy_dst", "copy_src"), ("workspace", "table"),
                           ("flag", "free_next"), ("block_table", "free")):
        assert _tables_call(lib, same={written: other}) == BAD
        assert b"overlap" in lib.halo_last_error_message()
    assert lib.halo_kv_beam_tables(*[None] * 8, 0, None, None) == BAD


# ------------------------------------------------------------------ refusals of the binding

def _bad(fn, good, **wrong):
    """fn refuses `good` with each of `wrong`'s values, and `good` itself for not being on a GPU."""
    for name, values in wrong.items():
        for value in values:
            with pytest.raises((ValueError, TypeError, halo.HaloError)):
                fn(**{**good, name: value})
    with pytest.raises(ValueError, match="GPU"):
        fn(**good)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("fn,kvq", [(halo.kv_page_weights, False), (halo.bind_kvq_page_weights, True)])
def test_weights_arguments(lib, fn, kvq):
    p = _params()
    pool = torch.zeros(3 * 2 * 16 * 64, dtype=torch.bfloat16)
    if kvq:
        pool = torch.zeros(3 * 2 * (64 * 8 + 32), dtype=torch.uint8)
    good = dict(weights=torch.zeros(2, 2, 40), k_pool=pool, params=p, page_ids=_i32(3), seq_page_indptr=_i32(3),
                seq_start=_i32(2), seq_end=_i32(2), q=torch.zeros(3, 4, 64, dtype=torch.bfloat16), lse=torch.zeros(3, 4),
                row_indptr=_i32(3), rows=_i32(3), row_end=_i32(3))
    _bad(fn, good, weights=[None, torch.zeros(2, 40), torch.zeros(1, 2, 40), torch.zeros(2, 2, 40).double(),
                            torch.zeros(2, 40, 2).transpose(1, 2)],
         weights_out=[torch.zeros(2, 2, 39), torch.zeros(2, 3, 40)], k_pool=[pool[:-1], pool.float()],
         page_ids=[_i32(3).long()], seq_page_indptr=[_i32(0)], seq_start=[_i32(1)], seq_end=[_i32(1), None],
         q=[torch.zeros(3, 4, 64), torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(12, 64, dtype=torch.bfloat16)],
         lse=[torch.zeros(2, 4), torch.zeros(3, 4, dtype=torch.bfloat16)], row_indptr=[_i32(2)], rows=[_i32(3).long()],
         row_end=[torch.zeros(3)])


def test_evict_arguments(lib):
    good = dict(weights=torch.zeros(2, 2, 40), seq_len=_i32(2), kept=_i32(2, 2, 8), new_len=_i32(2))
    _bad(halo.kv_evict_select, good, weights=[torch.zeros(2, 40), torch.zeros(2, 2, 40).double()],
         weights_out=[torch.zeros(2, 2, 39)], seq_len=[_i32(1)], kept=[_i32(2, 8), _i32(2, 3, 8), _i32(2, 2, 8).long()],
         new_len=[_i32(1), _i32(2).long()])
    _bad(halo.bind_kv_evict_select, good)


@pytest.mark.parametrize("fn,kvq", [(halo.bind_kv_page_keep_kv, False), (halo.kvq_page_keep_kv, True)])
def test_keep_arguments(lib, fn, kvq):
    k = v = torch.zeros(3 * 2 * 16 * 64, dtype=torch.bfloat16)
    if kvq:
        k, v = (torch.zeros(3 * 2 * (64 * 8 + 32), dtype=torch.uint8) for _ in range(2))
    good = dict(k_pool=k, v_pool=v, params=_params(), page_ids=_i32(3), seq_page_indptr=_i32(3), seq_len=_i32(2),
                new_len=_i32(2), kept=_i32(2, 2, 8))
    _bad(fn, good, k_pool=[k[:-1]], v_pool=[v.float()], page_ids=[_i32(3).long()], seq_len=[_i32(1)], new_len=[_i32(1)],
         kept=[_i32(2, 8), _i32(1, 2, 8), _i32(2, 3, 8)], dst_page_ids=[_i32(3)], dst_page_indptr=[_i32(3)])


def test_release_arguments(lib):
    good = dict(block_table=_i32(2, 4), seq_len=_i32(2), new_len=_i32(2), free_pages=_i32(8), free_next=_i32(1),
                free_pages_out=_i32(8), free_next_out=_i32(1))
    _bad(halo.kv_release_pages, good, block_table=[_i32(8), _i32(4, 2).t()], seq_len=[_i32(1)], new_len=[_i32(1)],
         free_pages_out=[_i32(7)], free_next=[_i32(1).long()], free_next_out=[_i32(0)])
    _bad(halo.bind_kv_release_pages, good)


def test_beam_arguments(lib):
    out = halo.BeamSelect(2, 3, 100, 4, device="cpu")
    good = dict(out=out, logits=torch.zeros(6, 100), scores=torch.zeros(2, 3), ended=_i32(2, 3), end_token=5)
    _bad(halo.beam_select, good, logits=[torch.zeros(6, 99), torch.zeros(5, 100), torch.zeros(100, 6).t(), torch.zeros(600),
                                         torch.zeros(6, 100, dtype=torch.float16), torch.zeros(100).expand(6, 100), None],
         scores=[torch.zeros(5), torch.zeros(6).double()], ended=[_i32(5), torch.zeros(6, dtype=torch.bool)])
    _bad(halo.bind_beam_select, good)
    for bad in ((2, 65, 100, 4), (2, 3, 100, 65), (2, 0, 100, 4), (-1, 3, 100, 4)):
        with pytest.raises(halo.HaloError):
            halo.BeamSelect(*bad, device="cpu")
    tables = halo.BeamTables(2, 3, 4, 8, device="cpu")
    good = dict(out=tables, parents=_i32(2, 3), seq_len=_i32(6), block_table=_i32(6, 4), free_pages=_i32(8),
                free_next=_i32(1))
    _bad(halo.kv_beam_tables, good, parents=[_i32(6), _i32(2, 2), _i32(3, 3), _i32(2, 3).long()], seq_len=[_i32(5)],
         block_table=[_i32(6, 5), _i32(24)], free_pages=[_i32(7), _i32(9)], free_next=[_i32(0)])
    _bad(halo.bind_kv_beam_tables, good)
    with pytest.raises(halo.HaloError):
        halo.BeamTables(2, 65, 4, 8, device="cpu")
