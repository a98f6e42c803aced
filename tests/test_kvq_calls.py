"""Host checks of how the step operators and the 4-bit calls are reached: the
names that programs use, the status of a refusal."""

import ast
import os

import pytest

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
