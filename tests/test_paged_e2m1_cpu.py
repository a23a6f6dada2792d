"""Paged K/V cache in 4 bits without a GPU: the oracle's quantiser, the plans, and what the calls refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import paged as O
from paged_shapes import CALLS, E2M1_CALLS, plan_of
from paper_2505_15781_amd import binding as B
from plans import paged_plan
from test_paged_cpu import ALL, CACHE_FAULTS, attn, calls, desc, load, store
from test_paged_plan_cpu import need


def test_codes_and_rounding_of_the_oracle():
    v = O.e2m1_values()
    for c in range(16):                                    # from the fields: sign, exponent, mantissa
        s, e, m = c >> 3, c >> 1 & 3, c & 1
        assert v[c] == (-1.0) ** s * (m * 0.5 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1))
    # every border: half way goes to the even code, a little less down, a little more up
    for c in range(7):
        half = (v[c] + v[c + 1]) / 2
        assert O.round_e2m1(np.array([half]))[0] == v[c + c % 2]
        assert O.round_e2m1(np.array([half - 1e-9]))[0] == v[c] and O.round_e2m1(np.array([half + 1e-9]))[0] == v[c + 1]
        assert O.round_e2m1(np.array([-half]))[0] == -v[c + c % 2]
    assert (O.round_e2m1(v) == v).all()


@pytest.mark.parametrize("top,e", [(6.0, 0), (6.01, 1), (3.0, -1), (3.01, 0), (1.0, -2), (1.5, -2), (1.5000001, -1), (0.0, -110), (1e-38, -110),
                                   (6 * 2.0 ** -110, -110), (6.1 * 2.0 ** -110, -109), (3.3895e38, 126), (np.inf, 128), (np.nan, 128)])
def test_scale_of_the_oracle(top, e):
    x = np.concatenate([[np.float32(top)], -0.3 * np.ones(31) * (top if np.isfinite(top) else 1.0), np.ones(32)])
    held, got = O.quantise_e2m1(x)
    assert got.tolist() == [e, -2] and (held[32:] == 1.0).all()
    if e == 128:
        assert np.isnan(held[:32]).all()
        return
    assert np.isfinite(held.astype(np.float32)).all()
    if e < 126:
        assert (np.abs(held - x) <= np.maximum(2.0 ** -2 * np.abs(x), 2.0 ** (e - 2)))[:32].all()


def test_held_values_are_the_nearest_of_their_block():
    """Against a search over all 16 codes, for blocks of many sizes and distributions."""
    g = np.random.default_rng(2)
    x = (g.standard_normal((300, 32)) * 2.0 ** g.integers(-60, 60, (300, 1)) * 2.0 ** g.integers(-3, 4, (300, 32))).astype(np.float32).astype(np.float64)
    held, e = O.quantise_e2m1(x)
    assert (np.abs(x).max(-1) <= 6 * 2.0 ** e[:, 0]).all() and (np.abs(x).max(-1) > 3 * 2.0 ** e[:, 0]).all()
    grid = O.e2m1_values() * (2.0 ** e)[..., None]
    assert np.array_equal(np.abs(held - x), np.abs(grid - x[..., None]).min(-1))


FOUR = dict(cache_dtype=B.E2M1)


@pytest.mark.parametrize("fault,code", [f for f in CACHE_FAULTS if "cache_dtype" not in f[0]])
def test_every_call_refuses_a_bad_cache(fault, code):
    for call in (store, load, attn):
        assert call(**FOUR, **fault) == code and B.last_error()
    assert B.lib.dkv_paged_attn_workspace_bytes(C.byref(desc(**FOUR, **fault)), 4, 3, 2, 0) == 0


def test_what_is_refused_and_what_is_not():
    for call in (store, load):
        assert call(**FOUR, k=None) == call(**FOUR, rows=-1) == call(**FOUR, dtype=B.E2M1) == -1
        assert call(**FOUR, rows=0, k=None, v=None, pos=None) == 0
        assert call(**FOUR, rows=1 << 24) == -3
    assert attn(**FOUR, rows=0, q=None, out=None, ws=None, nbytes=0) == 0 == attn(**FOUR, dtype=B.FP32, rows=0)
    assert attn(**FOUR, dtype=B.E2M1) == attn(**FOUR, seq_len=None) == attn(**FOUR, stride=255) == -1
    assert store(cache_dtype=5) == -1 and "dtype" in B.last_error()


@pytest.mark.parametrize("name", E2M1_CALLS)
def test_the_calls_of_the_gpu_tests_take_the_kernels_they_are_there_for(name):
    """A threshold that moves must not take a kernel out of the tests: then these shapes move with it."""
    assert plan_of(name, P.E2M1, calls=E2M1_CALLS).kernel == E2M1_CALLS[name][6]
    assert plan_of(name, P.E2M1, P.FP32, E2M1_CALLS).kernel in ("split", "split+")


def test_the_calls_take_every_kernel():
    kinds = lambda calls: {(c[6], c[5] if c[6].startswith("wide") else 0) for c in calls.values()}
    assert kinds(E2M1_CALLS) == kinds(CALLS)


@pytest.mark.parametrize("group,heads,dh,batch,keys,dtype", [
    (7, 4, 128, 8, 4096, P.BF16), (7, 4, 128, 1, 32768, P.BF16), (1, 32, 128, 4, 2100, P.BF16), (16, 1, 64, 6, 9000, P.BF16), (4, 8, 64, 2, 100000, P.BF16),
    (3, 8, 32, 3, 5000, P.BF16), (4, 2, 128, 5, 1000, P.FP32), (8, 24, 128, 2, 700, P.BF16), (1, 1, 128, 100, 2000, P.BF16), (16, 1, 128, 2, 50000, P.BF16),
    (1, 32, 128, 8, 9000, P.BF16), (7, 4, 128, 64, 8192, P.BF16)])
def test_a_workspace_for_many_rows_is_enough_for_fewer(group, heads, dh, batch, keys, dtype):
    sizes = dict(batch=batch, max_pages=-(-keys // 16), page_size=16, n_kv_heads=heads, head_dim=dh, cache_dtype=P.E2M1)
    d = B.PagedCacheDesc(16, 16, 16, 16, 16, 16, batch, batch * sizes["max_pages"], sizes["max_pages"], 16, heads, dh, P.E2M1)
    largest = 0
    for m in (1, 2, 3, 5, 8, 12, 16, 20, 33, 40, 64, 80, 96, 128, 130, 200, 300, 513, 1000):
        for rows in sorted({m, m + 1, batch * m // 3, batch * m * 3 // 4, batch * m - 1, batch * m}):
            if 1 <= rows <= batch * m:
                largest = max(largest, need(paged_plan(group * heads, rows, m, dtype, **sizes), batch, heads, dh))
        assert B.lib.dkv_paged_attn_workspace_bytes(C.byref(d), group * heads, batch * m, m, dtype) >= largest, m
    assert largest > 0


@pytest.mark.parametrize("heads,rows,keys,kernel", [
    (32, 64, 1000, "wide2"), (31, 64, 1000, "split"),      # up to two rounds of 256 groups of 32 query rows: 8 sequences of 64 (31 heads: 496)
    (4, 1024, 12320, "wide2+"), (4, 1024, 12256, "split+")])
def test_where_blocks_of_128_rows_begin(heads, rows, keys, kernel):
    """128 dims: from 513 groups on, or from 6144 keys a slice of 256 on (4 heads, 128 groups: 12288 keys)."""
    batch = 8 if rows == 64 else 1
    extra = 1 if rows == 64 and kernel == "wide2" else 0
    p = paged_plan(heads, batch * rows + extra * batch, rows + extra, P.BF16, batch, -(-keys // 32), 32, heads, 128, P.E2M1)
    assert p.kernel == kernel


@pytest.mark.parametrize("batch,keys,rows,dh,dtype,kernel", [
    (32, 8192, 1, 128, P.BF16, "split+"), (32, 8160, 1, 128, P.BF16, "split"), (33, 8192, 1, 128, P.BF16, "split"), (32, 8192, 17, 128, P.BF16, "split"),
    (32, 8192, 1, 64, P.BF16, "split+"), (32, 8192, 1, 128, P.FP32, "split"), (31, 8160, 1, 128, P.BF16, "split+")])
def test_where_a_compute_unit_has_two_slices(batch, keys, rows, dh, dtype, kernel):
    """8 K/V heads: 32 slices of each with one workgroup a unit, 64 with two, which serve up to 32 sequences of at least 8192 positions."""
    p = paged_plan(8, batch * rows, rows, dtype, batch, keys // 32, 32, 8, dh, P.E2M1)
    assert p.kernel == kernel and (not p.split or p.want == (64 if batch == 32 else 32))


@pytest.mark.parametrize("batch,heads,group,rows,keys,tiles,groups", [
    (3, 32, 1, 90, 300, 1, 6),                             # 288 groups of 32, 576 of 16: two rounds against one and a bit
    (19, 8, 4, 10, 700, 1, 3), (12, 8, 4, 17, 1500, 1, 5), (64, 4, 7, 5, 1000, 1, 3),
    (4, 4, 7, 64, 1024, 2, 14), (8, 32, 1, 64, 1024, 2, 2), (20, 32, 1, 17, 2000, 2, 1),
    (16, 4, 7, 40, 2000, 8, 3)])                           # blocks of 128
def test_where_groups_of_16_query_rows_are_taken(batch, heads, group, rows, keys, tiles, groups):
    p = paged_plan(heads * group, batch * rows, rows, P.BF16, batch, -(-keys // 16), 16, heads, 128, P.E2M1)
    assert p.kernel == ("split" if tiles < 8 else "wide2") and (p.q_tiles, p.q_groups) == (tiles, groups)


def tensors():
    pages = torch.zeros((5, 2, 16, 32), dtype=torch.uint8).view(torch.float4_e2m1fn_x2)
    scale = torch.zeros((5, 2, 16, 2), dtype=torch.uint8).view(torch.float8_e8m0fnu)
    return P.PagedCache(pages, pages.clone(), torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32), scale, scale.clone())


def refused(which, cache, text, **kw):
    for name, call in calls(cache, **kw).items():
        if name in which:
            with pytest.raises(ValueError, match=text):
                call()


def test_the_binding_refuses_tensors_that_are_not_what_a_call_reads():
    c = tensors()
    refused(ALL, c, "not on a GPU")                        # everything else is as it should be
    refused(ALL, c._replace(k_scale=None), "need k_scale")
    refused(ALL, c._replace(v_scale=c.v_scale.view(torch.uint8)), "v_scale")
    refused(ALL, c._replace(k_scale=c.k_scale[..., 0].contiguous()), "k_scale")
    refused(ALL, c._replace(k_scale=c.k_scale[..., :1].contiguous()), "k_scale")
    refused(ALL, c._replace(v_scale=c.v_scale[:4]), "v_scale")
    refused(ALL, c._replace(v_pages=c.v_pages.view(torch.uint8)), "v_pages")
    refused(ALL, c._replace(k_pages=c.k_pages.view(torch.uint8), v_pages=c.v_pages.view(torch.uint8)), "not supported")
    refused(("store", "load"), c, "k_", k=torch.zeros((6, 2, 32), dtype=torch.bfloat16))      # rows of the packed length
    refused(("attn",), c, "q", q=torch.zeros((6, 4, 32), dtype=torch.bfloat16))
    huge = torch.empty((1, 1, 1, 2 ** 31 - 1), dtype=torch.uint8, device="meta").view(torch.float4_e2m1fn_x2)
    refused(ALL, c._replace(k_pages=huge, v_pages=huge), "32 bits")


@pytest.mark.parametrize("heads,group,dh,batch,keys", [(8, 4, 128, 4, 9000), (32, 1, 64, 8, 16384), (4, 7, 32, 2, 100000), (1, 16, 128, 100, 2000)])
def test_fp32_rows_need_no_more_workspace_than_over_e4m3(heads, group, dh, batch, keys):
    """Their slices are those of one workgroup to a compute unit, whatever the cache; and enough for every call of fewer rows."""
    pages = -(-keys // 16)

    def bytes_for(dtype, m):
        d = B.PagedCacheDesc(16, 16, 16, 16, 16, 16, batch, batch * pages, pages, 16, heads, dh, dtype)
        return B.lib.dkv_paged_attn_workspace_bytes(C.byref(d), group * heads, batch * m, m, P.FP32)

    for m in (1, 2, 7, 33, 150):
        have = bytes_for(P.E2M1, m)
        assert have == bytes_for(P.E4M3, m) > 0
        for fewer in {1, m // 2, m} - {0}:
            plan = paged_plan(group * heads, batch * fewer, fewer, P.FP32, batch, pages, 16, heads, dh, P.E2M1)
            assert need(plan, batch, heads, dh) <= have


def test_sequences_are_ordered_by_their_lengths_where_that_gains():
    """Whole sequences in two to four rounds of workgroups over tables of 1024 positions and more: up to 64 of them, which are in order as a whole."""
    def ordered(batch, heads, max_pages=32, cache_dtype=P.E2M1, dtype=P.BF16, group=1, page=64, dh=128):
        p = paged_plan(heads * group, batch, 1, dtype, batch, max_pages, page, heads, dh, cache_dtype)
        assert p.kernel == "split"
        return p.longest_first

    assert ordered(32, 32) and ordered(64, 8) and ordered(64, 16, max_pages=16) and ordered(12, 32) and ordered(32, 32, dtype=P.FP32)
    assert not ordered(33, 32) and not ordered(8, 32, max_pages=8) and not ordered(64, 8, max_pages=15)
    assert not ordered(65, 8) and not ordered(100, 4, group=7) and not ordered(1000, 1, group=16) and not ordered(128, 8, group=4)
    assert not ordered(32, 32, cache_dtype=P.E4M3) and not ordered(32, 32, cache_dtype=P.BF16)
