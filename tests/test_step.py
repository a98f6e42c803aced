"""Host checks of the step operators: rotary angles against the formulas, and
what halo_rope_turns, halo_rope_qk and halo_kv_step_tables refuse."""

import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2509_02121_amd import halo


@pytest.fixture(scope="module")
def lib():
    return halo.load_library()


def rope_frequencies(R, base, scaling, factor, original, fast, slow):
    """The angle of each pair per position, and the amplitude, in 64 bits."""
    if scaling == "ntk":
        base *= factor ** (R / (R - 2))
    w = [base ** (-2 * i / R) for i in range(R // 2)]
    if scaling == "linear":
        w = [x / factor for x in w]
    if scaling == "yarn":
        lo, hi = (R * math.log(original / (n * 2 * math.pi)) / (2 * math.log(base)) for n in (fast, slow))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), R - 1)
        ramp = [min(1.0, max(0.0, (i - lo) / (hi - lo if hi > lo else 0.001))) for i in range(R // 2)]
        return [x * (1 - r) + x / factor * r for x, r in zip(w, ramp)], 0.1 * math.log(factor) + 1
    if scaling == "bands":
        keep = [min(1.0, max(0.0, (original * x / (2 * math.pi) - slow) / (fast - slow))) for x in w]
        w = [x * k + x / factor * (1 - k) for x, k in zip(w, keep)]
    return w, 1.0


@pytest.mark.parametrize("scaling,fast,slow", [("none", 32, 1), ("linear", 32, 1), ("ntk", 32, 1), ("yarn", 32, 1),
                                               ("yarn", 16, 2), ("bands", 4, 1), ("bands", 8, 0.5)])
@pytest.mark.parametrize("R,base", [(16, 10000.0), (64, 500000.0), (128, 1000000.0)])
def test_turns(lib, R, base, scaling, fast, slow):
    defaults = {"yarn": (32, 1), "bands": (4, 1)}.get(scaling) == (fast, slow)
    given = {} if defaults else {"fast_turns": fast, "slow_turns": slow}
    rope = halo.Rope(128, R, base=base, scaling=scaling, factor=4.0, original_positions=8192, device="cpu", **given)
    w, amplitude = rope_frequencies(R, base, scaling, 4.0, 8192, fast, slow)
    got = rope.host_turns.astype(np.float64) * 2.0 ** -64 * 2 * math.pi
    # a pow, a division and a few products in 64 bits on the reference's side;
    # the angle's 64 bits after the point are off by half of the last one at most
    # (2 pi * 2^-65 = 1.7e-19, where the smallest angles are below 1e-6)
    bound = 16 * np.finfo(np.float64).eps * math.log(base) * np.array(w) + 2 * math.pi * 2.0 ** -65
    assert (np.abs(got - np.array(w)) <= bound).all()
    assert abs(rope.amplitude - amplitude) <= 2.0 ** -24 * amplitude


@pytest.mark.parametrize("given", [
    {"head_dim": 96}, {"rotary_dim": 0}, {"rotary_dim": 24}, {"rotary_dim": 144}, {"base": 1.0}, {"base": math.nan},
    {"base": math.inf}, {"scaling": "linear", "factor": 0.5}, {"scaling": "ntk", "factor": math.nan},
    {"scaling": "yarn", "original_positions": 0}, {"scaling": "bands", "fast_turns": 1.0, "slow_turns": 4.0},
    {"scaling": "yarn", "fast_turns": math.nan, "slow_turns": 1.0}])
def test_turns_refusals(lib, given):
    args = {"head_dim": 128, "rotary_dim": 64, "factor": 2.0, **given}
    with pytest.raises(halo.HaloError):
        halo.Rope(device="cpu", **args)


def test_rope_arguments(lib):
    with pytest.raises(ValueError):
        halo.Rope(128, scaling="longer", device="cpu")
    with pytest.raises(ValueError):
        halo.Rope(128, fast_turns=3.0, device="cpu")
    with pytest.raises(halo.HaloError):
        halo._check(lib.halo_rope_turns(None, None, None))
    rope = halo.Rope(128, device="cpu")
    q, k, pos = torch.zeros(3, 4, 128), torch.zeros(3, 2, 128), torch.zeros(3, dtype=torch.int32)
    for bad in ((q[:2], k, pos), (q, k[:, :, :64], pos), (q, k.bfloat16(), pos), (q.double(), k, pos),
                (q.transpose(0, 1), k, pos), (q, k, pos)):   # the last: not on a GPU
        with pytest.raises(ValueError):
            halo.rope_qk(*bad, rope)


def _rope_call(lib, **given):
    """halo_rope_qk with host addresses (a call that is refused reads none)."""
    buf = np.zeros(4096, np.float32)
    at = (buf.ctypes.data + 15) // 16 * 16
    p = halo.RopeParams()
    lib.halo_rope_params_default(ctypes.byref(p), 128)
    for n in ("rotary_dim", "head_dim"):
        setattr(p, n, given.pop(n, getattr(p, n)))
    a = dict(rope=ctypes.byref(p), amplitude=1.0, turns=at, positions=at, tokens=2, hq=2, hk=1, dtype=0, q=at, qs=256,
             k=at, ks=128, qo=at, qos=256, ko=at, kos=128, stream=None)
    a.update(given)
    return lib.halo_rope_qk(*a.values())


@pytest.mark.parametrize("given", [
    {"rope": None}, {"rotary_dim": 8}, {"head_dim": 80}, {"dtype": 2}, {"tokens": -1}, {"hq": -1}, {"hk": -2},
    {"amplitude": math.nan}, {"amplitude": math.inf}, {"turns": None}, {"positions": None}, {"q": None}, {"ko": None},
    {"qs": 255}, {"qs": 258}, {"kos": 64}, {"qos": 512}, {"hq": 70000}])
def test_rope_qk_refusals(lib, given):
    assert _rope_call(lib, **given) in (halo.HALO_ERR_INVALID_ARGUMENT, halo.HALO_ERR_UNSUPPORTED)
    assert lib.halo_last_error_message()


def test_rope_qk_unaligned(lib):
    buf = np.zeros(64, np.float32)
    at = (buf.ctypes.data + 15) // 16 * 16
    assert _rope_call(lib, q=at + 4) == halo.HALO_ERR_INVALID_ARGUMENT
    assert _rope_call(lib, turns=at + 4) == halo.HALO_ERR_INVALID_ARGUMENT


def test_rope_qk_overlaps(lib):
    """Two tokens of two query heads (256 elements) and one key head (128), rows of
    384 elements at byte 0 of the buffer, or of 256 and 128."""
    buf = np.zeros(4096, np.float32)
    at = (buf.ctypes.data + 15) // 16 * 16
    far = {"q": at, "k": at + 4 * 1024, "qo": at + 4 * 2048, "ko": at + 4 * 3000}
    bad = [{"qo": at + 16}, {"qo": at + 4 * 512 - 16}, {"qo": far["k"]}, {"ko": at}, {"ko": at + 4 * 255 + 4},
           {"ko": far["k"] + 32}, {"ko": far["qo"] + 4 * 256}, {"qo": far["k"] - 4 * 256},
           {"qs": 384, "qos": 384, "qo": at + 4 * 128},   # a row apart by less than its width
           {"qs": 384, "qo": at, "ks": 384, "kos": 384, "qos": 384, "ko": at + 4 * 240},
           {"qs": 384, "kos": 512, "ko": at + 4 * 256}]   # strides that differ
    for given in bad:
        assert _rope_call(lib, **{**far, **given}) == halo.HALO_ERR_INVALID_ARGUMENT, given
        assert b"overlap" in lib.halo_last_error_message(), given


def test_rope_qk_too_many_tokens(lib):
    """A workgroup takes the 40 heads of one token: 2^24 of them are 2^32 threads."""
    a = 1 << 20   # (addresses far enough apart, read by nobody)
    far = {"q": a, "k": a + (1 << 50), "qo": a, "ko": a + (1 << 51)}
    assert _rope_call(lib, **far, tokens=1 << 24, hq=32, hk=8, qs=4096, qos=4096, ks=1024,
                      kos=1024) == halo.HALO_ERR_UNSUPPORTED


def test_rope_qk_nothing_to_do(lib):
    assert _rope_call(lib, tokens=0) == halo.HALO_OK
    assert _rope_call(lib, hq=0, hk=0) == halo.HALO_OK


def _tables_call(lib, sizes=None, none=(), **given):
    bufs = {n: np.zeros(64, np.int64) for n in
            ("seq_len", "seq_new", "block_table", "free_pages", "in_next", "error", "seq_page_indptr", "page_ids",
             "seq_start", "seq_count", "seq_end", "in_token_offset", "positions", "slots", "free_next")}
    at = {n: None if n in none else b.ctypes.data for n, b in bufs.items()}
    for n, other in given.items():
        at[n] = at[other]
    s = dict(num_seqs=2, page_size=16, table_width=4, num_free=3, max_tokens=8, max_pages=8)
    s.update(sizes or {})
    st = halo.StepSizes(*s.values())
    out = halo._StepTables(**{n: at[n] for n, _ in halo._StepTables._fields_})
    return lib.halo_kv_step_tables(ctypes.byref(st), at["seq_len"], at["seq_new"], at["block_table"], at["free_pages"],
                                   at["in_next"], ctypes.byref(out), at["error"], None)


def test_step_tables_refusals(lib):
    for name in ("num_seqs", "table_width", "num_free", "max_tokens", "max_pages"):
        assert _tables_call(lib, {name: -1}) == halo.HALO_ERR_INVALID_ARGUMENT
    assert _tables_call(lib, {"page_size": 32}) == halo.HALO_ERR_UNSUPPORTED
    for name in ("seq_len", "seq_new", "block_table", "free_pages", "in_next", "seq_page_indptr", "page_ids",
                 "seq_start", "seq_count", "seq_end", "in_token_offset", "free_next"):
        assert _tables_call(lib, none=(name,)) == halo.HALO_ERR_INVALID_ARGUMENT
    assert _tables_call(lib, seq_end="seq_len") == halo.HALO_ERR_INVALID_ARGUMENT
    assert _tables_call(lib, seq_count="seq_new") == halo.HALO_ERR_INVALID_ARGUMENT
    assert _tables_call(lib, free_next="in_next") == halo.HALO_ERR_INVALID_ARGUMENT
    for written, other in (("page_ids", "free_pages"), ("slots", "block_table"), ("error", "free_next"),
                           ("positions", "slots"), ("seq_start", "seq_new"), ("block_table", "free_pages")):
        assert _tables_call(lib, **{written: other}) == halo.HALO_ERR_INVALID_ARGUMENT
        assert b"overlap" in lib.halo_last_error_message()
    assert lib.halo_kv_step_tables(None, *[None] * 8) == halo.HALO_ERR_INVALID_ARGUMENT


def test_step_tables_arguments(lib):
    t = halo.StepTables(2, 8, 8, device="cpu")
    one, two = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    table, free = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad in ((one, two, table, free, one), (two, two.long(), table, free, one), (two, two, table[:1], free, one),
                (two, two, table.flatten(), free, one), (two, two, table.t(), free, one),
                (two, two, table, free, one)):   # the last: not on a GPU
        with pytest.raises(ValueError):
            halo.kv_step_tables(t, *bad)
