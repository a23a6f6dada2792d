"""Which kernel a call of paged_attn is planned to (host code)."""
import ctypes as C

import pytest

import paper_2505_15781_amd as P
from paged_shapes import CALLS, plan_of
from paper_2505_15781_amd import binding as B
from plans import paged_plan


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


def need(plan, batch, heads, dh):
    """Bytes of a plan's records: (first slice, slices) of each sequence, then max, sum and output of each slice, K/V head and query row."""
    return -(-batch * 8 // 16) * 16 + plan.cap * heads * plan.q_groups * plan.q_tiles * 16 * (dh + 4) * 4 if plan.split else 0


@pytest.mark.parametrize("group,heads,dh,batch,keys,dtype,cache_dtype", [
    (7, 4, 128, 8, 4096, P.BF16, P.BF16), (7, 4, 128, 1, 32768, P.BF16, P.E4M3), (1, 32, 128, 4, 2100, P.BF16, P.E4M3), (16, 1, 64, 6, 9000, P.BF16, P.BF16),
    (4, 8, 64, 2, 100000, P.BF16, P.E4M3), (3, 8, 32, 3, 5000, P.BF16, P.BF16), (4, 2, 128, 5, 1000, P.FP32, P.FP32), (8, 24, 128, 2, 700, P.BF16, P.BF16),
    (2, 8, 64, 30, 3000, P.BF16, P.E4M3), (1, 1, 128, 100, 2000, P.BF16, P.E4M3)])
def test_a_workspace_for_many_rows_is_enough_for_fewer(group, heads, dh, batch, keys, dtype, cache_dtype):
    """An active set that shrinks keeps its workspace: the bytes of a call cover every call of fewer rows and of a smaller bound on the same cache."""
    sizes = dict(batch=batch, max_pages=-(-keys // 16), page_size=16, n_kv_heads=heads, head_dim=dh, cache_dtype=cache_dtype)
    d = B.PagedCacheDesc(16, 16, 16, 16, 16, 16, batch, batch * sizes["max_pages"], sizes["max_pages"], 16, heads, dh, cache_dtype)
    most = (1, 2, 3, 5, 8, 12, 16, 20, 33, 40, 64, 80, 96, 128, 130, 200, 300, 513, 1000)
    largest = 0
    for m in most:
        for rows in sorted({m, m + 1, batch * m // 3, batch * m * 3 // 4, batch * m - 1, batch * m}):
            if not 1 <= rows <= batch * m:
                continue
            largest = max(largest, need(paged_plan(group * heads, rows, m, dtype, **sizes), batch, heads, dh))
        assert B.lib.dkv_paged_attn_workspace_bytes(C.byref(d), group * heads, batch * m, m, dtype) >= largest, m
        assert B.lib.dkv_paged_attn_workspace_bytes(C.byref(d), group * heads, batch * 1000, 1000, dtype) < 32 << 20
    assert largest > 0


@pytest.mark.parametrize("batch,cut", [(13, True), (14, True), (15, True), (16, False), (19, False)])
def test_long_sequences_of_a_ragged_batch_are_cut_where_it_gains(batch, cut):
    """28/4 heads, up to 40 rows and 3000 keys: 20 slices run at once, and cutting gains down to four for three sequences."""
    rows = sum(-(-40 * (batch - b) // batch) for b in range(batch))
    p = paged_plan(28, rows, 40, P.BF16, batch, 48, 64, 4, 128, P.E4M3)
    assert p.kernel == ("wide2+" if cut else "wide2" if p.wide == 2 else "wide1")
