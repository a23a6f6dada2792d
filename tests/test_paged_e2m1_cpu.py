"""Paged K/V cache in 4 bits without a GPU: the oracle's quantiser, the plans, and what the calls refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import paged as O
from paged_shapes import CALLS, plan_of
from paper_2505_15781_amd import binding as B
from test_paged_cpu import ALL, CACHE_FAULTS, attn, calls, desc, load, store


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


@pytest.mark.parametrize("dtype", [P.BF16, P.FP32])
@pytest.mark.parametrize("name", CALLS)
def test_plans_are_those_of_the_other_caches(name, dtype):
    """A cache of any type takes the kernel that the calls of the GPU tests are there for."""
    a, b = plan_of(name, P.E2M1, dtype), plan_of(name, P.E4M3, dtype)
    assert [getattr(a, f) for f, _ in a._fields_] == [getattr(b, f) for f, _ in b._fields_]


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
