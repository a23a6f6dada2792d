"""Which kernel a call of paged_attn is planned to (host code)."""
import pytest

import paper_2505_15781_amd as P
from paged_shapes import CALLS, plan_of


@pytest.mark.parametrize("cache_dtype", [P.BF16, P.E4M3])
@pytest.mark.parametrize("name", CALLS)
def test_the_calls_of_the_gpu_tests_take_the_kernels_they_are_there_for(name, cache_dtype):
    """A threshold that moves must not take a kernel out of the tests: then these shapes move with it."""
    assert plan_of(name, cache_dtype).kernel == CALLS[name][6]


def test_the_calls_take_every_kernel():
    assert {c[6] for c in CALLS.values()} == {"split", "split+", "wide1", "wide1+", "wide2", "wide2+"}
    assert {(c[6], c[5]) for c in CALLS.values() if c[6].startswith("wide")} == {
        ("wide1", 64), ("wide1", 128), ("wide2", 64), ("wide2", 128), ("wide1+", 64), ("wide2+", 128)}       # what make_plan hands out


@pytest.mark.parametrize("name", CALLS)
def test_fp32_rows_have_one_kernel(name):
    assert plan_of(name, P.FP32, P.FP32).kernel in ("split", "split+")
