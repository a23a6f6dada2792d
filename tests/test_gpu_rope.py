"""Rotary positions on the GPU against the oracle.

Bar of an element: the cosine and the sine are off by at most 2^-23 (their angle, within half a quarter turn, is rounded to fp32 once, 2^-25
at most, their series' terms and sums stay below 2^-24), times the scale once rounded (2^-24), and two products and a sum of 2^-24 each: 6 * 2^-24 of
scale (|a| + |b|) with room for the second order; the result's rounding to bf16 adds 2^-8 of it. Angles: position times quarter turns is off by
2^-52 of itself, 2^31 * 2^-52 * pi / 2 = 2^-20 radians at the farthest position and a frequency of one, which is counted with its position."""
import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import rotary as O
from test_gpu_paged import dev, rows

pytestmark = pytest.mark.gpu


def check(got, x, positions, r, interleaved, inverse=False):
    want, size = O.rotate(x.double().cpu().numpy(), positions, r.freq, r.scale, interleaved, inverse)
    got, n = got.double().cpu().numpy(), 2 * len(r.freq)
    far = np.abs(np.asarray(positions, dtype=np.float64))[:, None, None] * max(map(abs, r.freq)) * 2.0 ** -51
    bar = (6 * 2.0 ** -24 + far) * size + (2.0 ** -8 * np.abs(want) if x.dtype == torch.bfloat16 else 0.0) + 1e-37
    assert np.array_equal(got[..., n:], want[..., n:])
    err = np.abs(got - want)
    assert (err <= bar).all(), float((err / bar).max())


SHAPES = [  # rows, q heads, k heads, head_dim, rot_dim
    (1, 1, 1, 32, 32), (1, 32, 32, 128, 128), (7, 28, 4, 128, 64), (64, 32, 32, 128, 128), (33, 5, 3, 64, 64), (9, 16, 1, 64, 48), (5, 3, 2, 32, 24),
    (3, 2, 1, 128, 2), (3, 1, 2, 32, 10), (130, 24, 8, 128, 120), (1025, 33, 7, 128, 128), (2049, 8, 2, 64, 32), (4100, 3, 1, 32, 30), (777, 40, 0, 128, 96),
    (600, 0, 13, 64, 64)]


@pytest.mark.parametrize("act", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(s) for s in SHAPES])
def test_rows_are_rotated(act, interleaved, shape):
    """Out of place from parts of longer rows, back in place, and as the gradient."""
    n, hq, hk, dh, rot = shape
    g = np.random.default_rng(n)
    wide = rows(g, (n, hq + hk + 3, dh), act, 2.0)
    q, k = wide[:, 1:1 + hq] if hq else None, wide[:, 1 + hq:1 + hq + hk] if hk else None
    pos = g.integers(0, 1 << 20, n)
    pos[0], pos[-1] = 0, (1 << 30) - 1
    before = wide.clone()
    for scaling, inverse in (("none", False), ("parts", True)):
        r = P.Rope(dh, rot, 5e5, interleaved, scaling, 8.0)
        big = torch.full((n, hq + 2, dh), 7.0, dtype=wide.dtype, device="cuda")
        q_out, k_out = big[:, 1:1 + hq] if hq else None, torch.full((n, hk, dh), 7.0, dtype=wide.dtype, device="cuda") if hk else None
        P.rope(r, q, k, dev(pos), q_out=q_out, k_out=k_out, inverse=inverse)
        assert torch.equal(wide, before) and (big[:, 0] == 7.0).all() and (big[:, 1 + hq:] == 7.0).all()
        for x, y in ((q, q_out), (k, k_out)):
            if x is not None:
                check(y, x, pos, r, interleaved, inverse)
    P.rope(r, q, k, dev(pos))                              # in place
    for x, at in ((q, slice(1, 1 + hq)), (k, slice(1 + hq, 1 + hq + hk))):
        if x is not None:
            check(x, before[:, at], pos, r, interleaved)
    assert torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, 1 + hq + hk:], before[:, 1 + hq + hk:])


@pytest.mark.parametrize("act", ["bf16", "fp32"])
def test_rows_behind_the_last_sequence_and_odd_addresses(act):
    for n, rot, pairs in ((3, 128, False), (40, 64, True), (3000, 128, False), (3000, 126, True)):
        g = np.random.default_rng(n)
        room = rows(g, (n * 6 * 128 + 8,), act)
        x = room[3:3 + n * 6 * 128].view(n, 6, 128)
        before, pos, off = room.clone(), g.integers(-50, 5000, n), np.array([0, 1, n - 2])
        r = P.Rope(128, rot, interleaved=pairs)
        P.rope(r, x[:, :4], x[:, 4:], dev(pos), row_off=dev(off))
        was = before[3:3 + n * 6 * 128].view(n, 6, 128)
        check(x[:n - 2], was[:n - 2], pos[:n - 2], r, pairs)
        assert torch.equal(x[n - 2:], was[n - 2:]) and torch.equal(room[:3], before[:3]) and torch.equal(room[3 + x.numel():], before[3 + x.numel():])


@pytest.mark.parametrize("n,rot", [(3, 128), (520, 96)])
def test_rows_that_are_far_apart(n, rot):
    """Rows behind the first four gigabytes, in place and into others."""
    g = np.random.default_rng(5)
    step = (5 << 30) // (2 * (n - 1)) // 128 * 128
    x = rows(g, (n, 12, 128), "bf16")
    room = torch.empty((n - 1) * step + 12 * 128, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(room, (n, 12, 128), (step, 128, 1))
    far.copy_(x)
    pos, r = g.integers(0, 1 << 17, n), P.Rope(128, rot)
    out = torch.empty_like(x)
    P.rope(r, far[:, :9], far[:, 9:], dev(pos), q_out=out[:, :9], k_out=out[:, 9:])
    check(out, x, pos, r, False)
    P.rope(r, far[:, :9], far[:, 9:], dev(pos))
    assert torch.equal(far, out)
    far.fill_(0.0)
    P.rope(r, x[:, :9], x[:, 9:], dev(pos), q_out=far[:, :9], k_out=far[:, 9:])
    assert torch.equal(far, out)


def test_every_angle_of_a_wide_range_of_positions():
    """Positions of all magnitudes up to the largest, both signs, frequencies from radians to almost none: the pair (1, 0) becomes (cos, sin)."""
    pos = np.unique(np.concatenate([np.arange(-300, 300), (2.0 ** np.linspace(0, 31, 3000)).astype(np.int64) - 1, -(2.0 ** np.linspace(0, 31, 500)).astype(np.int64)]))
    pos = pos[(pos >= -2 ** 31) & (pos < 2 ** 31)]
    r = P.Rope(128, 128, 1e6)
    x = torch.zeros((len(pos), 1, 128), device="cuda")
    x[..., :64] = 1.0
    was = x.clone()
    P.rope(r, x, None, dev(pos))
    check(x, was, pos, r, False)


def test_own_frequencies_infinities_and_nan():
    r = P.Rope(64, 8, interleaved=True)
    r.freq, r.scale = [np.pi / 2, 0.0, -1.5, 100.25], 0.75
    x = rows(np.random.default_rng(1), (9, 2, 64), "fp32")
    was = x.clone()
    P.rope(r, x, None, dev(np.arange(9)))
    check(x, was, np.arange(9), r, True)
    x = was.clone()
    x[3, 0, 2], x[4, 1, 60], x[5, 0, 0] = float("nan"), float("inf"), float("inf")
    bad = x.clone()
    P.rope(r, x, None, dev(np.arange(9)))
    assert torch.isnan(x[3, 0, 2:4]).all() and not torch.isnan(x[3, 0, 4:]).any() and not torch.isnan(x[3, 1]).any()
    assert torch.equal(x[4, 1, 8:], bad[4, 1, 8:]) and not torch.isfinite(x[5, 0, :2]).any() and torch.isfinite(x[5, 0, 2:]).all()
    fine = [r0 for r0 in range(9) if r0 not in (3, 4, 5)]
    check(x[fine], was[fine], np.array(fine), r, True)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_by_differences(interleaved):
    """The loss w . rope(x), in fp32: its gradient by x is rope of w, inverse; differences of the loss along random directions, which is linear in x: the
    difference quotient is exact but for rounding, (head_dim + 8) * 2^-24 of the sum of magnitudes twice."""
    g = np.random.default_rng(2)
    r = P.Rope(64, 48, 1e4, interleaved, "parts", 4.0)
    x, w, d = (rows(g, (20, 5, 64), "fp32") for _ in range(3))
    pos = dev(g.integers(0, 1 << 17, 20))
    grad = torch.empty_like(w)
    P.rope(r, w, None, pos, q_out=grad, inverse=True)
    up, down = torch.empty_like(x), torch.empty_like(x)
    P.rope(r, x + d, None, pos, q_out=up)
    P.rope(r, x - d, None, pos, q_out=down)
    by_difference = ((up.double() - down.double()) * w.double()).sum() / 2
    along = (grad.double() * d.double()).sum()
    bar = 2 * 72 * 2.0 ** -24 * float(((x.abs() + d.abs()).double() * 2 * w.abs().double()).sum() + (grad.abs() * d.abs()).double().sum())
    assert abs(float(by_difference - along)) <= bar


def test_two_streams_and_a_captured_call():
    g = np.random.default_rng(3)
    r = P.Rope(128)
    xs, pos = [rows(g, (500, 40, 128), "bf16") for _ in range(2)], dev(g.integers(0, 1 << 17, 500))
    want = [torch.empty_like(x) for x in xs]
    for x, y in zip(xs, want):
        P.rope(r, x, None, pos, q_out=y)
    torch.cuda.synchronize()
    got, streams = [torch.empty_like(x) for x in xs], [torch.cuda.Stream() for _ in xs]
    for _ in range(10):
        for x, y, s in zip(xs, got, streams):
            with torch.cuda.stream(s):
                P.rope(r, x, None, pos, q_out=y)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.rope(r, xs[0], None, pos, q_out=got[0])
    r.freq = [0.0] * 64                                    # a captured call keeps the frequencies that it was given
    for t in range(3):
        pos.copy_(dev(g.integers(0, 1 << 17, 500)))
        xs[0].copy_(rows(g, (500, 40, 128), "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        P.rope(P.Rope(128), xs[0], None, pos, q_out=want[0])
        assert torch.equal(want[0], got[0])


@pytest.mark.parametrize("act", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", [(1100, 9, 4, 128, 120), (1100, 9, 4, 128, 124), (2100, 3, 2, 64, 30), (2048, 1, 4, 64, 62), (2047, 1, 4, 64, 62),
                                   (1024, 5, 4, 128, 128), (1023, 5, 4, 128, 64), (1030, 5, 3, 128, 128)], ids=str)
def test_heads_of_a_lane_one_or_four(act, interleaved, shape):
    """Both sides of where a lane works on four heads at once, in pieces of 8 and 4 elements and of one."""
    test_rows_are_rotated(act, interleaved, shape)
