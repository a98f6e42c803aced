"""Host checks of how the step operators and the 4-bit calls are reached: the
names that programs use, the status of a refusal."""

import ast
import gc
import os
import weakref

import numpy as np
import pytest
import torch

from paper_2509_02121_amd import halo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("call", ["page_scatter_kv", "page_gather_kv", "page_copy"])
def test_both_names_of_the_page_calls(call):
    for prefix in ("", "bind_"):
        assert getattr(halo, f"{prefix}kv4_{call}") is getattr(halo, f"{prefix}kvq_{call}")


def test_operator_cases_call_what_there_is():
    """Every name that the cases of perf/operators.py take from the package."""
    with open(os.path.join(ROOT, "perf", "operators.py")) as f:
        tree = ast.parse(f.read())
    names = {n.attr for n in ast.walk(tree)
             if isinstance(n, ast.Attribute) and isinstance(n.value, ast.Name) and n.value.id == "halo"}
    assert len(names) > 5
    assert sorted(n for n in names if not hasattr(halo, n)) == []


@pytest.fixture
def on_host(monkeypatch):
    """The bound calls' arguments are taken from host tensors (nothing is
    called)."""
    halo.load_library()
    monkeypatch.setattr(halo, "_gpu", lambda t, *a: t)
    monkeypatch.setattr(halo, "_one_gpu", lambda *a: None)
    monkeypatch.setattr(halo, "_rope_operand", lambda t, *a: (t.shape[1], t.stride(0)))
    monkeypatch.setattr(halo, "_stream_handle", lambda s: None)


def test_bound_rope_holds_its_angles(on_host):
    """A Rope made in the call's expression lives as long as the callable."""
    q, k, pos = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32)
    ropes = [halo.Rope(64, device="cpu")]
    turns = weakref.ref(ropes[0].turns)
    call = halo.bind_rope_qk(q, k, pos, ropes.pop())
    gc.collect()
    assert turns() is not None
    del call
    gc.collect()
    assert turns() is None


def test_bound_step_tables_hold_their_arrays(on_host):
    """So do the arrays of a StepTables of which the caller keeps only some:
    the calls write all of them."""
    def ints(*shape):
        return torch.zeros(shape, dtype=torch.int32)
    tabs = halo.StepTables(2, 4, 8, device="cpu")
    arrays = [weakref.ref(t) for t in vars(tabs).values() if isinstance(t, torch.Tensor)]
    assert len(arrays) == 9
    call = halo.bind_kv_step_tables(tabs, ints(2), ints(2), ints(2, 4), ints(8), ints(1))
    del tabs
    gc.collect()
    assert all(t() is not None for t in arrays)
    del call
    gc.collect()
    assert all(t() is None for t in arrays)


@pytest.mark.parametrize("bad,status", [({"head_dim": 96}, halo.HALO_ERR_UNSUPPORTED), ({"page_size": 32}, halo.HALO_ERR_UNSUPPORTED),
                                        ({"kv_dtype": 7}, halo.HALO_ERR_UNSUPPORTED),
                                        ({"num_kv_heads": 1 << 30}, halo.HALO_ERR_UNSUPPORTED),
                                        ({"num_pool_pages": 1 << 60}, halo.HALO_ERR_UNSUPPORTED),
                                        ({"num_kv_heads": 0}, halo.HALO_ERR_INVALID_ARGUMENT),
                                        ({"num_pool_pages": -1}, halo.HALO_ERR_INVALID_ARGUMENT)])
def test_pool_bytes_status(bad, status):
    """A size that is refused has the status that the page calls give."""
    lib = halo.load_library()
    p = halo.make_params(8, 2, 64, torch.bfloat16, 10, 0.125)
    for k, v in bad.items():
        setattr(p, k, v)
    for call in (lambda: halo.kvq_pool_bytes(p, halo.HALO_POOL_K), lambda: halo.alloc_kvq_pools(p, "cpu")):
        with pytest.raises(halo.HaloError) as e:
            call()
        assert e.value.status == status
    assert lib.halo_last_error_status() == status
    assert halo.kvq_pool_bytes(halo.make_params(8, 2, 64, torch.bfloat16, 10, 0.125), halo.HALO_POOL_V) > 0
    assert lib.halo_last_error_status() == halo.HALO_OK


@pytest.mark.parametrize("prefill", [False, True])
def test_attention_over_pools_that_are_not_built(prefill):
    """A plan of more heads than a 4-bit pool has: the kernels' page offsets
    would pass 32 bits for some of them, so the call refuses it, like
    halo_kvq_pool_bytes."""
    lib = halo.load_library()
    n = 65537
    csr = {"seg_len": np.array([1], np.int32), "seg_page_indptr": np.array([0, 1], np.int32),
           "seg_page_ids": np.array([0], np.int32), "req_seg_indptr": np.array([0, 1], np.int32),
           "req_seg_ids": np.array([0], np.int32), "q_len": np.array([1], np.int32) if prefill else None}
    plan = halo.Plan.from_csr(halo.make_params(n, n, 64, torch.bfloat16, 1, 0.125), csr)
    assert plan.is_prefill == prefill
    fn = lib.halo_prefix_attn_prefill_kvq if prefill else lib.halo_prefix_attn_decode_kvq
    keep = np.zeros(128, np.int64)
    at = (keep.ctypes.data + 255) // 256 * 256
    assert fn(plan._handle, at, at, at, at, at, at, at, 1 << 40, None) == halo.HALO_ERR_UNSUPPORTED
    assert b"65536" in lib.halo_last_error_message()
