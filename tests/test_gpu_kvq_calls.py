"""GPU checks of calls over 4-bit pools that stand beside each other: the
workspace, values at the ends of the range, cuts that must not show."""

import numpy as np
import pytest
import torch

from kvq_helpers import fill_pools
from paper_2509_02121_amd import halo
from workloads import build_workload

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def _w(seg_len, paths, q_len=None, heads=(4, 2), D=128, dtype=BF16, seed=5):
    return build_workload("kvq", seed, *heads, D, dtype, seg_len, paths, q_len, poison=False, extra_pages=3)


@pytest.mark.parametrize("out", [BF16, FP32])
def test_workspace_of_a_fresh_object(gpu_lib, out):
    """PrefixAttention.workspace is enough for a call over 4-bit pools, also
    before the first one, which then makes no other."""
    w = _w([600, 33, 257], [[0, 1], [0, 2]])
    pools = fill_pools(w)
    params = halo.make_params(4, 2, 128, BF16, w.num_pool_pages, w.scale, out)
    att = halo.PrefixAttention(params, w.forest_csr())
    assert att.plan.stats()["num_merge_rows"] > 0
    q, ws = w.q.cuda(), att.workspace
    o, lse = att.alloc_outputs(q)
    halo.prefix_attn_decode_kvq(att.plan, att.meta, q, *pools, o, lse, ws)
    o2, lse2 = att.run(q, *pools)
    torch.cuda.synchronize()
    assert att.workspace is ws
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
