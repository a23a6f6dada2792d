"""Attention over the paged cache on every kernel (the calls of paged_shapes.py, each checked to be planned to its own), with data that
unit normal values do not bring: scores that keep growing, large ones, infinities and NaN, odd addresses. Bars as in test_gpu_paged.py."""
import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import paged as O
from paged_shapes import BLOCKS, CALLS, plan_of
from test_gpu_paged import Cache, bars, check_attn, dev, rows, workspace

pytestmark = pytest.mark.gpu

EVERY = [(name, types) for name in CALLS for types in (("bf16 bf16", "bf16 e4m3") if name in BLOCKS else ("bf16 bf16", "bf16 e4m3", "fp32 fp32", "fp32 e4m3"))]
every_call = pytest.mark.parametrize("name,types", EVERY, ids=[n + "-" + t.replace(" ", "-") for n, t in EVERY])


def make(name, types, seed, size=1.0):
    """(cache with all positions stored, q with two rows behind the last sequence where the call takes them, rows of each sequence)"""
    act, dtype = types.split()
    lens, counts, page, heads, group, dh, kernel = CALLS[name]
    if act == "bf16":
        assert plan_of(name, {"bf16": P.BF16, "e4m3": P.E4M3}[dtype]).kernel == kernel
    c = Cache(lens, page, heads, dh, dtype, seed=seed).fill(act, size=size)
    extra = min(2, len(counts) * max(counts) - sum(counts))
    return c, rows(np.random.default_rng(seed), (sum(counts) + extra, heads * group, dh), act), counts


def store(c, b, positions, k, v):
    """Rows of sequence b on both sides."""
    n = c.o["table"].shape[0]
    off = np.concatenate([np.zeros(b + 1, int), np.full(n - b, len(positions))])
    P.paged_store(c.t, k, v, dev(positions), dev(off))
    with np.errstate(over="ignore"):
        O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), np.asarray(positions), off, c.dtype)


@every_call
def test_scores_of_hundreds(name, types):
    c, q, counts = make(name, types, 31, size=20.0)
    check_attn(c, q, counts)


@every_call
def test_scores_that_grow_and_fall_along_a_sequence(name, types):
    """Queries whose scores grow by some 60 (a factor of 2^86) from a sequence's first key to its last, others whose scores fall, and others that
    hardly move: the reference of the exponentials follows, a little at nearly every tile, and what was summed before is brought along."""
    c, q, counts = make(name, types, 32)
    heads, dh = c.heads, c.dh
    for b, n in enumerate(c.o["lengths"]):
        k, v = (rows(np.random.default_rng(b + i), (n, heads, dh), types.split()[0]) for i in (40, 50))
        k[:, :, 0] = (torch.arange(n, device="cuda")[:, None] * (8.0 / n)).to(k.dtype)
        store(c, b, np.arange(n), k, v)
    q[:, :, 0] = torch.tensor([7.5, -7.5, 0.5, 2.0], device="cuda").repeat(len(q) // 4 + 1)[:len(q), None].to(q.dtype) * dh ** 0.5
    check_attn(c, q, counts)


@every_call
def test_infinities_and_nan_act_where_they_are_seen(name, types):
    """Keys of -infinity, infinite and NaN values in the longest sequence and the last one, some in its first tile and some in its last."""
    act, dtype = types.split()
    c, q, counts = make(name, types, 33, size=0.5)            # no probability vanishes
    heads, dh = c.heads, c.dh
    for b in {int(np.argmax(c.o["lengths"])), len(counts) - 1}:
        n = int(c.o["lengths"][b])
        at = np.unique([3, n // 3, n // 2, n - 2])
        k = torch.full((len(at), heads, dh), 0.25, dtype=q.dtype, device="cuda")
        v = torch.ones_like(k)
        k[0] = k[-1] = float("-inf")
        v[0] = 1.0
        v[1, 0, 5], v[2, heads - 1, dh - 1] = float("inf"), float("nan")
        store(c, b, at, k, v)
    with np.errstate(invalid="ignore"):
        check_attn(c, q.abs(), counts)


@every_call
def test_addresses_of_any_element(name, types):
    c, q, counts = make(name, types, 34)
    room = torch.zeros(q.numel() + 8, dtype=q.dtype, device="cuda")
    inside = room[5:5 + q.numel()].view(q.shape).copy_(q)
    out = torch.full((q.numel() + 8,), 7.0, dtype=q.dtype, device="cuda")
    check_attn(c, inside, counts, out=out[3:3 + q.numel()].view(q.shape))
    assert (out[:3] == 7.0).all() and (out[3 + q.numel():] == 7.0).all()


@every_call
def test_pages_that_are_missing(name, types):
    """A table with a quarter of its pages gone, the first and the last of the longest sequence among them."""
    act, dtype = types.split()
    lens, counts, page, heads, group, dh, _ = CALLS[name]
    c = Cache(lens, page, heads, dh, dtype, seed=35, holes=0.25)
    b = int(np.argmax(lens))
    c.o["table"][b, [0, -(-lens[b] // page) - 1]] = -1
    c.t.page_table.copy_(dev(c.o["table"]))
    c.fill(act)
    check_attn(c, rows(np.random.default_rng(35), (sum(counts), heads * group, dh), act), counts)


@every_call
def test_scores_of_minus_infinity_only_give_zeros_whatever_the_values(name, types):
    """A query with -infinity where all keys are 1: its scores are -infinity, the sum of its exponentials is zero, and so is the result, also where
    the values that it sees are infinite or NaN. The other queries see those values."""
    act, dtype = types.split()
    c, q, counts = make(name, types, 36, size=0.5)
    for b, n in enumerate(c.o["lengths"]):
        k, v = (rows(np.random.default_rng(b + i), (n, c.heads, c.dh), act) for i in (60, 70))
        k[:, :, 1] = 1.0
        v[0, :, 0], v[n // 2, :, 2], v[n - 1, :, 3] = float("inf"), float("nan"), float("-inf")
        store(c, b, np.arange(n), 0.5 * k, v)
    most = float(q.double().norm(dim=-1).max() * torch.from_numpy(c.o["k"][np.isfinite(c.o["k"])]).abs().max()) * 1.01     # at least |q| |k| / sqrt(dh)
    q[::3, :, 1] = float("-inf")
    none = np.arange(len(q)) % 3 == 0
    offsets = np.concatenate([[0], np.cumsum(counts)])
    out = torch.full_like(q, 7.0)
    P.paged_attn(c.t, q, dev(offsets), out, max(counts), workspace(c, q, max(counts)))
    with np.errstate(invalid="ignore"):
        ref, spread, _ = O.attn(c.o, q.double().cpu().numpy(), offsets)
    mine = np.arange(len(q)) < offsets[-1]
    got, ref, spread = out.double().cpu().numpy()[mine], ref[mine], spread[mine]
    assert (got[none[mine]] == 0).all() and (ref[none[mine]] == 0).all()
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    fine = np.isfinite(ref)
    assert (np.abs(got[fine] - ref[fine]) <= bars(q, c, ref, spread, most)[fine]).all()


@every_call
def test_the_probabilities_that_weigh_the_values_sum_to_one(name, types):
    """All values of a sequence and head are one row: whatever the scores, and however the probabilities are rounded, that row is the result. To
    the bit in bf16: fp32 sums are off by far less than half a step of the result if the sum adds up the rounded probabilities; with the unrounded ones it is
    off by up to 2^-8, and half a step of values that end in ones is 2^-9. Two keys share the weight, 1 : 2^1 to 1 : 2^8."""
    act, dtype = types.split()
    c, q, counts = make(name, types, 37)
    heads, dh = c.heads, c.dh
    offsets = np.concatenate([[0], np.cumsum(counts)])
    want = torch.zeros((offsets[-1],) + q.shape[1:], dtype=torch.float64, device="cuda")
    for b, n in enumerate(c.o["lengths"]):
        g = np.random.default_rng(80 + b)
        k, v = torch.zeros((n, heads, dh), dtype=q.dtype, device="cuda"), torch.zeros((1, heads, dh), dtype=q.dtype, device="cuda")
        v[:] = torch.from_numpy(g.choice([-1.0, 1.0], v.shape) * (1.875 if dtype == "e4m3" else 255 / 128) * 2.0 ** g.integers(-3, 3, (1, heads, 1)))
        k[:, :, 1] = -4096.0
        k[[n // 8, n * 2 // 3]] = 0.0
        k[n * 2 // 3, :, 0] = 1.0
        store(c, b, np.arange(n), k, v.expand(n, -1, -1).contiguous())
        page, slot = O.place(c.o, b, 0)
        want[offsets[b]:offsets[b + 1]] = torch.from_numpy(c.o["v"][page, :, slot]).cuda().repeat_interleave(q.shape[1] // heads, dim=0)
    q[:] = 0.0
    q[:, :, 1] = 1.0
    q[:, :, 0] = (torch.rand(q.shape[:2], generator=torch.Generator().manual_seed(3)).cuda() * 7.0 + 1.0).to(q.dtype) * np.log(2) * dh ** 0.5
    out = torch.zeros_like(q)
    P.paged_attn(c.t, q, dev(offsets), out, max(counts), workspace(c, q, max(counts)))
    got = out[:offsets[-1]].double()
    if act == "bf16":
        assert torch.equal(got, want), int((got != want).sum())
    else:
        assert ((got - want).abs() <= (int(c.o["lengths"].max()) + 64) * 2.0 ** -23 * want.abs()).all()


def in_parts(x, n):
    """x as the sum of a[i] * 8^-i, each a[i] of 4 significant bits."""
    a = []
    for i in range(n):
        step = 2.0 ** (np.floor(np.log2(x)) - 3)
        a.append(float(np.floor(x / step) * step))
        x = 8 * (x - a[-1])
        if x < 2.0 ** -6:
            break
    return a + [0.0] * (n - len(a))


@every_call
def test_the_largest_probability_is_exactly_one(name, types):
    """Two keys with probabilities of 1 : 9 / 64 and values of 9 / 64 and -1, all others with a probability of zero: the result is zero, for
    1 and 9 / 64 are bf16 numbers. What is left are the errors of fp32 scores: sums of 9 products of at most 32, 9 * 2^-24 of the exponent 2.8, the
    same again for its scale, reference and exponential, of 9 / 73: below 1e-6. With the smaller one for reference the larger would be 64 / 9, which bf16 holds as
    228 / 32, and the result 2.4e-4; blocks of 128 rows over an e4m3 cache do that, and are off by half a step of the larger at most, 2^-8 (64 / 73) (9 / 64). The
    larger score comes last in even heads, first in odd ones."""
    act, dtype = types.split()
    c, q, counts = make(name, types, 38)
    heads, dh = c.heads, c.dh
    q[:] = 0.0
    q[:, :, :8] = 8.0 ** -torch.arange(8.0, device="cuda").to(q.dtype)
    q[:, :, 8] = 1.0
    larger = torch.tensor(in_parts(np.log(64 / 9) * dh ** 0.5, 8), device="cuda").to(q.dtype)
    for b, n in enumerate(c.o["lengths"]):
        k, v = torch.zeros((n, heads, dh), dtype=q.dtype, device="cuda"), rows(np.random.default_rng(90 + b), (n, heads, dh), act)
        k[:, :, 8] = -4096.0
        for h in range(heads):
            first, last = (n // 4, 3 * n // 4) if h % 2 == 0 else (3 * n // 4, n // 4)
            k[first, h], k[last, h] = 0.0, 0.0
            k[last, h, :8] = larger
            v[first, h], v[last, h] = -1.0, 9 / 64
        store(c, b, np.arange(n), k, v)
    out = torch.full_like(q, 7.0)
    n = sum(counts)
    P.paged_attn(c.t, q, dev(np.concatenate([[0], np.cumsum(counts)])), out, max(counts), workspace(c, q, max(counts)))
    half_a_step = 2.0 ** -8 * 9 / 73 if name in BLOCKS and dtype == "e4m3" else 0.0
    assert float(out[:n].abs().max()) <= 1e-6 + half_a_step


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_an_active_set_that_shrinks_keeps_its_workspace(dtype):
    """One workspace, asked for once for the most rows, whose plan has no slices; calls of fewer rows are cut into some."""
    lens = [4200, 300, 2100]
    c = Cache(lens, 32, 4, 128, dtype, seed=39).fill()
    q = rows(np.random.default_rng(39), (3 * 400, 16, 128), "bf16")
    ws = workspace(c, q, 400)
    for counts in ([400, 400, 400], [200, 200, 200], [130, 7, 200], [64, 64, 64], [33, 1, 20], [8, 8, 8], [1, 0, 1], [0, 0, 1]):
        n, most = sum(counts), max(counts)
        out = torch.full((n, 16, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        offsets = np.concatenate([[0], np.cumsum(counts)])
        P.paged_attn(c.t, q[:n], dev(offsets), out, most, ws)
        ref, spread, size = O.attn(c.o, q[:n].double().cpu().numpy(), offsets)
        assert (np.abs(out.double().cpu().numpy() - ref) <= bars(q, c, ref, spread, size)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_of_any_bits_are_held_and_read_back(dtype):
    """Random bit patterns, denormal numbers, infinities and NaN among them, in caches that are not quantised: the nearest value of the type."""
    g = np.random.default_rng(40)
    x = torch.from_numpy(g.integers(0, 2 ** 32, (2, 200, 64), dtype=np.uint64).astype(np.uint32).view(np.float32)).cuda()
    tiny = torch.from_numpy((g.integers(0, 2 ** 23, (2, 200, 32)) | g.integers(0, 2, (2, 200, 32)) << 31).astype(np.uint32).view(np.float32)).cuda()
    x[:, :, 32:] = tiny
    c = Cache([2], 16, 200, 64, dtype)
    P.paged_store(c.t, x, x, dev([0, 1]), dev([0, 2]))
    y = x.double().cpu().numpy()
    O.store(c.o, y, y, np.array([0, 1]), np.array([0, 2]), dtype)
    assert c.same()
    for out in ("bf16", "fp32"):
        k, v = (torch.zeros(x.shape, dtype={"bf16": torch.bfloat16, "fp32": torch.float32}[out], device="cuda") for _ in "kv")
        P.paged_load(c.t, k, v, dev([1, 0]), dev([0, 2]))
        page = int(c.o["table"][0, 0])
        want = c.o["k"][page, :, :2].transpose(1, 0, 2)[::-1]
        want = O.round_bf16(want) if out == "bf16" else want
        assert np.array_equal(k.double().cpu().numpy(), want, equal_nan=True) and np.array_equal(v.double().cpu().numpy(), want, equal_nan=True)


@every_call
def test_a_table_that_is_much_wider_than_its_sequences(name, types):
    """16384 positions, as a table for sequences that grow in a captured loop would have: the plan goes by them, the results by the lengths."""
    act, dtype = types.split()
    lens, counts, page, heads, group, dh, _ = CALLS[name]
    c = Cache(lens, page, heads, dh, dtype, seed=41, wider=16384 // page - max(-(-n // page) for n in lens)).fill(act)
    assert c.t.page_table.shape[1] == 16384 // page
    check_attn(c, rows(np.random.default_rng(41), (sum(counts), heads * group, dh), act), counts)
