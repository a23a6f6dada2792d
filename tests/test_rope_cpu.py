"""Rotary positions without a GPU: frequencies and refusals."""
import copy
import ctypes as C
import math
import pickle

import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import rotary as O
from paper_2505_15781_amd import binding as B
from plans import rope_lane_heads


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("base", 8.0), ("parts", 16.0), ("parts", 0.5)])
@pytest.mark.parametrize("head_dim,rot_dim,theta", [(128, 128, 1e4), (64, 32, 5e5), (32, 10, 1e4), (128, 126, 10.0)])
def test_frequencies(scaling, factor, head_dim, rot_dim, theta):
    r = P.Rope(head_dim, rot_dim, theta, False, scaling, factor, 2048, 1.5, 30.0)
    freq, scale = O.frequencies(rot_dim, theta, scaling, factor, 2048, 1.5, 30.0)
    assert np.allclose(r.freq, freq, rtol=1e-13, atol=0) and abs(r.scale - scale) <= 2.0 ** -24 * abs(scale)
    assert r.freq[0] == pytest.approx(1.0 / factor if scaling == "linear" else 1.0) or scaling == "parts"
    if scaling == "base":                                  # the last pair is stretched by the factor
        assert r.freq[-1] == pytest.approx(theta ** -((rot_dim - 2) / rot_dim) / factor)


def test_parts_leave_fast_pairs_and_stretch_slow_ones():
    plain, r = P.Rope(128), P.Rope(128, scaling="parts", factor=8.0)
    turns = [4096 * f / (2 * math.pi) for f in plain.freq]
    for f, g, t in zip(plain.freq, r.freq, turns):
        assert g == f if t >= 32 else g == f / 8 if t <= 1 else f / 8 < g < f
    assert r.scale == pytest.approx(0.1 * math.log(8) + 1)


def test_frequencies_and_scale_can_be_set():
    r = P.Rope(64, 8)
    r.freq = [1.0, 0.5, 0.25, 0.0]
    r.scale = 2.0
    assert r.freq == [1.0, 0.5, 0.25, 0.0] and r.scale == 2.0 and r.desc.freq[0] == 1.0
    with pytest.raises(ValueError):
        r.freq = [1.0]


def init(desc=None, head_dim=128, rot=128, pairs=0, theta=1e4, scaling=0, factor=1.0, original=4096.0, slow=1.0, fast=32.0):
    return B.lib.dkv_rope_init(C.byref(desc or B.RopeDesc()), head_dim, rot, pairs, theta, scaling, factor, original, slow, fast)


def test_what_the_frequencies_refuse():
    assert init() == 0 and B.lib.dkv_rope_init(None, 128, 128, 0, 1e4, 0, 1.0, 0.0, 0.0, 0.0) == -1
    for head_dim, rot in ((48, 48), (256, 64), (128, 130), (128, 3), (128, 0), (64, -2), (32, 64)):
        assert init(head_dim=head_dim, rot=rot) == -3 and B.last_error()
    for bad in (0.0, -1.0, math.nan, math.inf):
        assert init(theta=bad) == -1
        assert init(scaling=1, factor=bad) == -1 == init(scaling=3, factor=bad)
        assert init(scaling=0, factor=bad) == 0            # not read
    assert init(scaling=4) == init(scaling=-1) == -1
    assert init(scaling=2, factor=2.0, rot=2) == -1
    assert init(scaling=3, original=0.0) == init(scaling=3, slow=32.0) == init(scaling=3, slow=-1.0) == init(scaling=3, fast=math.nan) == -1
    d = B.RopeDesc()
    d.head_dim = 7
    assert init(d, rot=3) == -3 and d.head_dim == 7        # nothing is written
    with pytest.raises(ValueError):
        P.Rope(64, scaling="cubic")
    with pytest.raises(P.DkvError):
        P.Rope(48)


def test_a_copy_has_frequencies_of_its_own():
    r = P.Rope(64, 32, interleaved=True)
    for other in (copy.copy(r), copy.deepcopy(r), pickle.loads(pickle.dumps(r))):
        assert other.address == C.addressof(other.desc) and other.freq == r.freq and other.scale == r.scale
    other.freq = [0.5] * 16
    assert r.freq[0] == 1.0 and other.freq[0] == B.RopeDesc.from_address(other.address).freq[0] == 0.5


def call(rope=None, q=16, qs=512, qo=16, qos=512, nq=4, k=16, ks=256, ko=16, kos=256, nk=2, pos=16, off=16, batch=3, rows=5, dtype=0, inverse=0):
    return B.lib.dkv_rope(C.byref(rope or P.Rope(128).desc), q, qs, qo, qos, nq, k, ks, ko, kos, nk, pos, off, batch, rows, dtype, inverse, None)


def test_refused_arguments():
    assert call(q=None) == call(qo=None) == call(k=None) == call(ko=None) == call(pos=None) == -1
    assert call(qs=511) == call(qos=511) == call(ks=255) == call(kos=255) == -1
    assert call(qos=513) == call(kos=257) == -1            # in place, with another stride
    assert call(rows=-1) == call(nq=-1) == call(nk=-1) == call(batch=0) == call(dtype=2) == call(dtype=4) == -1
    assert call(rows=0, q=None, qo=None, k=None, ko=None, pos=None) == 0
    assert call(nq=0, nk=0, q=None, qo=None, k=None, ko=None) == 0
    assert call(rows=1 << 24) == -3 == call(nq=1 << 24, qs=1 << 31, qos=1 << 31)
    assert call(rows=(1 << 24) - 1, nq=512, qs=1 << 16, qos=1 << 16) == -3
    assert B.lib.dkv_rope(None, *[16, 512, 16, 512, 4, 16, 256, 16, 256, 2], 16, 16, 3, 5, 0, 0, None) == -1
    bad = B.RopeDesc()
    assert call(rope=bad) == -3
    bad.head_dim, bad.rot_dim = 128, 5
    assert call(rope=bad) == -3


def test_the_binding_refuses_tensors_that_are_not_what_a_call_reads():
    r = P.Rope(64)
    q, k, pos = torch.zeros((6, 8, 64), dtype=torch.bfloat16), torch.zeros((6, 2, 64), dtype=torch.bfloat16), torch.zeros(6, dtype=torch.int32)

    def refused(text, q=q, k=k, pos=pos, **kw):
        with pytest.raises(ValueError, match=text):
            P.rope(r, q, k, pos, **kw)

    refused("not on a GPU")
    refused("not on a GPU", k=None)
    refused("not on a GPU", q=None, row_off=torch.zeros(2, dtype=torch.int32))
    refused("not on a GPU", q=None, k=None)
    qkv = torch.zeros((6, 12, 64))
    refused("not on a GPU", q=qkv[:, :8], k=qkv[:, 8:10], q_out=torch.zeros((6, 8, 64)))
    refused("positions", pos=pos.long())
    refused("positions", pos=pos[:5])
    refused("positions", pos=pos[::2])
    refused("positions", pos=pos[:, None])
    refused("q", q=q[..., :32])
    refused("q", q=q.half())
    refused("q", q=q[0])
    refused("q", q=q.transpose(1, 2).contiguous().transpose(1, 2))
    refused("k", k=k.float())
    refused("one for each row", k=k[:5])
    refused("q_out", q_out=q.float())
    refused("q_out", q_out=q[:, :4])
    refused("k_out", k_out=k[:5])
    refused("k_out", k=None, k_out=k)
    refused("q_out", q=None, q_out=q)
    refused("row_off", row_off=pos.long())
    refused("row_off", row_off=pos[:1])
    with pytest.raises(TypeError):
        P.rope(r, q, k, pos, inverse="yes")


def test_the_oracle_turns_pairs_by_their_angles():
    """Pairs as complex numbers, and that the inverse undoes (and is the transpose)."""
    g = np.random.default_rng(0)
    x, y = g.standard_normal((2, 5, 3, 64))
    pos = g.integers(0, 10 ** 6, 5)
    freq, _ = O.frequencies(48, 1e4)
    for pairs in (False, True):
        z, _ = O.rotate(x, pos, freq, 1.5, pairs)
        a, b = (slice(0, 48, 2), slice(1, 48, 2)) if pairs else (slice(0, 24), slice(24, 48))
        want = (x[..., a] + 1j * x[..., b]) * 1.5 * np.exp(1j * pos[:, None, None] * np.array(freq))
        assert np.allclose(z[..., a], want.real, atol=1e-12) and np.allclose(z[..., b], want.imag, atol=1e-12)
        assert np.array_equal(z[..., 48:], x[..., 48:])
        back, _ = O.rotate(y, pos, freq, 1.5, pairs, inverse=True)
        assert np.sum(z[..., :48] * y[..., :48]) == pytest.approx(np.sum(x[..., :48] * back[..., :48]))


def test_heads_of_a_lane():
    """Four where that gains; calls of the most workgroups, also of those that would be too many with one."""
    assert [rope_lane_heads(P.BF16, 8, 128, 64, n) for n in (1, 511, 512, 6144)] == [1, 1, 4, 4]
    assert [rope_lane_heads(P.BF16, 4, 128, 13, n) for n in (1023, 1024)] == [1, 4]
    assert [rope_lane_heads(t, 1, 64, 5, n) for t in (P.BF16, P.FP32) for n in (2047, 2048)] == [1, 4, 1, 4]
    assert {rope_lane_heads(P.FP32, 4, 128, 64, n) for n in (1, 512, 6144, 100000)} == {1}
    assert rope_lane_heads(P.BF16, 8, 64, 10, 6144) == rope_lane_heads(P.FP32, 1, 32, 4, 6144) == 1      # all heads in one wavefront
    # 64 heads of 128 in fp32, 16 wavefronts a row or 4: up to 2^25 of them
    assert [rope_lane_heads(P.FP32, 4, 128, 64, n) for n in ((1 << 21) - 1, 1 << 21, (1 << 23) - 1, 1 << 23)] == [1, 4, 4, 0]
    assert [rope_lane_heads(P.BF16, 8, 128, 64, n) for n in ((1 << 24) - 3, 1 << 24)] == [4, 0]
