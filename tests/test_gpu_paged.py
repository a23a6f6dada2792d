"""Paged K/V cache on the GPU: rows written, read back and attended to, against the oracle.

Bars of the attention, per element: bf16 results are rounded once (2^-8 of the value), the probabilities once before the product
with V while their sum adds up the rounded ones (2^-8 of sum p |v - o| / sum p, which is at most sum p |v| / sum p + |o|);
scores are fp32 sums of head_dim products (at most (head_dim + 4) 2^-24 of sum |q| |k| / sqrt(head_dim), which is also the relative error of
a probability, twice in a quotient), and the sums over the keys fp32 too ((keys + 64) 2^-23, for the order in which parts are joined as well)."""
import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import paged as O

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}


class Cache:
    """A cache on the GPU, and the oracle's of the same values. Everything that is not stored is NaN on both sides."""

    def __init__(self, lens, page, heads, dh, dtype, seed=0, holes=0.0, wider=1, lengths=None):
        g = np.random.default_rng(seed)
        self.dtype, self.heads, self.dh, self.g = dtype, heads, dh, g
        need = [-(-n // page) for n in lens]
        width = max(1, max(need)) + wider
        n_pages = sum(need) + 3
        ids = g.permutation(n_pages)
        table = np.full((len(lens), width), -1)
        for b, n in enumerate(need):
            table[b, :n] = ids[sum(need[:b]):sum(need[:b]) + n]
        bad = g.random(table.shape) < holes
        table[bad] = g.choice([-1, -7, n_pages, n_pages + 5, 2 ** 31 - 1, -2 ** 31], size=int(bad.sum()))
        nan = np.full((n_pages, heads, page, dh), np.nan)
        self.o = {"k": nan, "v": nan.copy(), "table": table, "lengths": np.array(lens if lengths is None else lengths)}
        raw = torch.full((n_pages, heads, page, dh * {"bf16": 2, "fp32": 4, "e4m3": 1}[dtype]), 0xFF, dtype=torch.uint8, device="cuda")
        scales = [None, None]
        if dtype == "e4m3":
            scales = [torch.full((n_pages, heads, page), 0xFF, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in "kv"]
        self.t = P.PagedCache(raw.view(TORCH[dtype]), raw.clone().view(TORCH[dtype]), torch.from_numpy(table.astype(np.int32)).cuda(),
                              torch.from_numpy(self.o["lengths"].astype(np.int32)).cuda(), *scales)

    def values(self, which):
        pages, scale = (self.t.k_pages, self.t.k_scale) if which == "k" else (self.t.v_pages, self.t.v_scale)
        x = pages.double()
        if scale is not None:
            x = x * torch.exp2(scale.view(torch.uint8).double() - 127.0)[..., None]
        return x.cpu().numpy()

    def same(self):
        return all(np.array_equal(self.values(w), self.o[w], equal_nan=True) for w in "kv")

    def fill(self, act="bf16", size=1.0):
        """Stores all positions of all sequences, on both sides."""
        lens = self.o["lengths"]
        off = np.concatenate([[0], np.cumsum(lens)])
        pos = np.concatenate([np.arange(n) for n in lens] + [np.zeros(0, int)])
        k, v = (rows(self.g, (len(pos), self.heads, self.dh), act, s) for s in (size, 1.0))
        O.store(self.o, k.double().cpu().numpy(), v.double().cpu().numpy(), pos, off, self.dtype)
        if len(pos):
            P.paged_store(self.t, k, v, dev(pos), dev(off))
        return self


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def rows(g, shape, act, size=1.0):
    return torch.from_numpy((size * g.standard_normal(shape)).astype(np.float32)).cuda().to(TORCH[act])


def workspace(cache, q, most):
    dt = P.BF16 if q.dtype == torch.bfloat16 else P.FP32
    n = P.paged_attn_workspace_bytes(cache.t, q.shape[1], q.shape[0], most, dt)
    assert n > 0
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")


def bars(q, cache, ref, spread, most):
    keys = int(cache.o["lengths"].max())
    rel = 2 * (cache.dh + 4) * 2.0 ** -24 * most + (keys + 64) * 2.0 ** -23
    bf = 2.0 ** -8 if q.dtype == torch.bfloat16 else 0.0
    return (bf + 2.0 ** -23) * np.abs(ref) + (bf + rel) * (1 + 2.0 ** -7) * (spread + np.abs(ref)) + 1e-37


def check_attn(cache, q, counts, most=None, off="given", out=None):
    counts = np.array(counts)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    most = int(counts.max()) if most is None else most
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda") if out is None else out
    P.paged_attn(cache.t, q, dev(offsets) if off == "given" else None, out, most, workspace(cache, q, most))
    got = out.double().cpu().numpy()
    ref, spread, size = O.attn(cache.o, q.double().cpu().numpy(), offsets)
    mine = np.arange(len(ref)) < offsets[-1]
    assert (got[~mine] == 7.0).all()                       # rows behind the last sequence
    ref, spread, got = ref[mine], spread[mine], got[mine]
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
    err, bar = np.abs(got[fine] - ref[fine]), bars(q, cache, ref, spread, size)[fine]
    assert (err <= bar).all(), (float((err / bar).max()), float(err.max()))
    return out


@pytest.mark.parametrize("act", ["bf16", "fp32"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("dh,heads,page", [(128, 4, 16), (64, 1, 32), (32, 3, 256), (128, 33, 64)])
def test_rows_are_held_to_the_bit_and_read_back(act, dtype, dh, heads, page):
    c = Cache([5, 0, 70, 1, page], page, heads, dh, dtype, seed=dh + page, holes=0.2).fill(act)
    assert c.same()
    counts = [4, 0, 33, 0, 3]
    off = np.concatenate([[0], np.cumsum(counts)])
    g = np.random.default_rng(3)
    top = c.o["table"].shape[1] * page
    pos = np.concatenate([g.permutation(np.arange(-2, top + 2))[:n] for n in counts] + [[0, 1]])     # two rows behind the last sequence
    pos[1] = -2 ** 31
    wide = rows(g, (len(pos), 3 * heads, dh), act, 3.0)
    k, v = wide[:, heads:2 * heads], wide[:, 2 * heads:]
    P.paged_store(c.t, k, v, dev(pos), dev(off))
    O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), pos, off, dtype)
    assert c.same()
    for out in ("bf16", "fp32"):
        ko, vo = (torch.full((len(pos), heads, dh), 7.0, dtype=TORCH[out], device="cuda") for _ in "kv")
        P.paged_load(c.t, ko, vo, dev(pos), dev(off))
        wk, wv = (np.full((len(pos), heads, dh), 7.0) for _ in "kv")
        O.load(c.o, pos, off, wk, wv)
        if out == "bf16" and dtype == "fp32":
            wk, wv = O.round_bf16(wk), O.round_bf16(wv)
        assert np.array_equal(ko.double().cpu().numpy(), wk, equal_nan=True) and np.array_equal(vo.double().cpu().numpy(), wv, equal_nan=True)


@pytest.mark.parametrize("out,heads,dh", [("bf16", 33, 128), ("fp32", 20, 64), ("bf16", 65, 32)])
def test_many_rows_are_read_back(out, heads, dh):
    """Calls large enough that a lane reads several pieces, the last ones of a row not all there; rows without a page, rows of no sequence."""
    c = Cache([700, 0, 850], 32, heads, dh, "e4m3", seed=heads, holes=0.1).fill()
    off = np.array([0, 700, 700, 1550])
    pos = np.concatenate([np.random.default_rng(1).permutation(700), np.random.default_rng(2).permutation(850), [3, 4, 5]])
    ko, vo = (torch.full((1553, heads, dh), 7.0, dtype=TORCH[out], device="cuda") for _ in "kv")
    P.paged_load(c.t, ko, vo, dev(pos), dev(off))
    wk, wv = (np.full((1553, heads, dh), 7.0) for _ in "kv")
    O.load(c.o, pos, off, wk, wv)
    assert np.array_equal(ko.double().cpu().numpy(), wk) and np.array_equal(vo.double().cpu().numpy(), wv)


def test_every_bf16_value_is_quantised_as_the_oracle_does():
    """All 65536 bit patterns, 32 to a row: rows of one magnitude (all exponents, zeros, infinities, NaN) and shuffled ones."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    mixed = bits[torch.randperm(65536, generator=torch.Generator().manual_seed(1))]
    x = torch.cat([bits, mixed]).view(1, -1, 32).cuda().expand(2, -1, -1).contiguous()
    c = Cache([2], 16, x.shape[1], 32, "e4m3")
    P.paged_store(c.t, x, x, dev([0, 1]), dev([0, 2]))
    O.store(c.o, x.double().cpu().numpy(), x.double().cpu().numpy(), np.array([0, 1]), np.array([0, 2]), "e4m3")
    assert c.same()
    ko, vo = (torch.zeros_like(x) for _ in "kv")
    P.paged_load(c.t, ko, vo, dev([1, 0]), dev([0, 2]))
    want = c.o["k"][int(c.o["table"][0, 0]), :, :2].transpose(1, 0, 2)[::-1]
    assert np.array_equal(ko.double().cpu().numpy(), want, equal_nan=True) and torch.equal(ko.view(torch.int16), vo.view(torch.int16))


def test_one_row_per_sequence_of_a_batch_beyond_a_wavefront():
    """Without row offsets, and with them, for 131 sequences: stored, read back, attended to."""
    lens = [int(x) for x in np.random.default_rng(5).integers(0, 50, 131)]
    c = Cache(lens, 16, 2, 64, "e4m3", seed=5).fill()
    g = np.random.default_rng(6)
    pos = np.maximum(np.array(lens) - 1, 0)
    k, v = (rows(g, (131, 2, 64), "bf16") for _ in "kv")
    P.paged_store(c.t, k, v, dev(pos))
    O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), pos, None, "e4m3")
    assert c.same()
    ko, vo = (torch.zeros((131, 2, 64), dtype=torch.float32, device="cuda") for _ in "kv")
    P.paged_load(c.t, ko, vo, dev(pos))
    wk, wv = np.zeros((131, 2, 64)), np.zeros((131, 2, 64))
    O.load(c.o, pos, None, wk, wv)
    assert np.array_equal(ko.double().cpu().numpy(), wk) and np.array_equal(vo.double().cpu().numpy(), wv)
    q = rows(g, (131, 6, 64), "bf16")
    a, b = check_attn(c, q, [1] * 131, off=None), check_attn(c, q, [1] * 131)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


ATTN = [  # lens, rows, page, kv heads, group, dh
    ([1], [1], 16, 1, 1, 128), ([0], [1], 16, 2, 2, 64), ([512], [1], 16, 4, 1, 128), ([31, 32, 33, 0, 1], [1, 2, 1, 3, 1], 16, 2, 4, 128),
    ([63, 64, 65, 127, 129], [3, 0, 17, 1, 16], 32, 2, 1, 64), ([1300, 7], [1, 5], 64, 2, 7, 128), ([5000], [2], 128, 1, 7, 128),
    ([333, 1000, 16], [40, 70, 16], 16, 3, 1, 128), ([769, 100, 257], [65, 129, 33], 32, 2, 7, 128), ([300, 513], [130, 257], 256, 2, 1, 64),
    ([200, 40], [17, 23], 16, 4, 1, 32), ([2100], [1], 16, 1, 16, 32), ([640, 448], [300, 64], 64, 8, 4, 128), ([1, 2, 3], [130, 1, 140], 16, 26, 1, 128),
    ([1333, 64, 333, 0], [200, 100, 400, 70], 16, 8, 4, 128), ([63, 129, 1024], [300, 5, 900], 128, 32, 1, 128),
    ([300, 1050, 40], [130, 257, 1], 256, 16, 2, 64), ([100, 190, 80, 70], [300, 300, 200, 100], 16, 32, 1, 64),
    ([4500, 40, 2100], [100, 70, 129], 32, 2, 4, 128), ([9000, 0, 2081], [50, 257, 130], 64, 1, 4, 64), ([5000, 2081], [150, 257], 64, 8, 4, 64),
    ([1006, 900], [65, 64], 16, 1, 16, 128), ([4500, 3000], [32, 30], 16, 1, 12, 128), ([8230], [96], 16, 1, 16, 128),
    ([700, 90, 130, 64, 33, 600, 5], [40, 64, 33, 35, 1, 7, 62], 16, 24, 1, 128), ([800, 100, 500], [300, 17, 140], 32, 1, 16, 64),
    ([6500, 40, 2100], [100, 70, 129], 32, 2, 4, 128), ([5000, 0, 4100], [257, 80, 300], 16, 4, 4, 64),
    ([4200, 1, 1500, 64, 700, 0, 33], [75, 3, 40, 9, 20, 2, 1], 16, 8, 4, 128)]


@pytest.mark.parametrize("types", ["bf16 bf16", "bf16 e4m3", "fp32 fp32", "fp32 e4m3"])
@pytest.mark.parametrize("case", range(len(ATTN)))
@pytest.mark.parametrize("holes", [0.0, 0.25])
def test_attention(types, case, holes):
    act, dtype = types.split()
    lens, counts, page, heads, group, dh = ATTN[case]
    c = Cache(lens, page, heads, dh, dtype, seed=case, holes=holes, wider=2).fill(act)
    g = np.random.default_rng(case)
    R = sum(counts)
    q = rows(g, (R + 2, heads * (group + 1), dh), act)[:, heads:]          # rows that are parts of longer ones, two behind the last sequence
    if R + 2 > len(counts) * max(counts):
        q = q[:R]
    check_attn(c, q, counts, most=max(counts) if case % 2 else max(counts) + 3)


@pytest.mark.parametrize("types", ["bf16 bf16", "bf16 e4m3", "fp32 fp32", "fp32 e4m3"])
@pytest.mark.parametrize("n,most", [(3, 3), (150, 150)])
def test_attention_to_large_scores_infinities_and_nan(types, n, most):
    """Scores of hundreds (one key takes it all), keys of -infinity, infinite and NaN values: where they are seen they act, and only
    on their own head; a sequence whose scores are all -infinity gives zeros. (e4m3 holds NaN for the infinities.)"""
    act, dtype = types.split()
    c = Cache([200, 90, 40], 16, 2, 128, dtype, seed=9).fill(act, size=20.0)
    q = rows(np.random.default_rng(9), (n + 2, 4, 128), act)
    check_attn(c, q, [n, 1, 1])
    c = Cache([200, 90, 40], 16, 2, 128, dtype, seed=10).fill(act, size=0.5)     # no probability vanishes
    special = torch.ones((3, 2, 128), dtype=TORCH[act], device="cuda")
    special[0, 0], special[1, 0] = float("-inf"), 1.0
    values = torch.ones((3, 2, 128), dtype=TORCH[act], device="cuda")
    values[1, 1, 5], values[2, 0, 100] = float("inf"), float("nan")
    pos, off = np.array([77, 80, 13]), np.array([0, 2, 3, 3])
    P.paged_store(c.t, special, values, dev(pos), dev(off))
    O.store(c.o, special.double().cpu().numpy(), values.double().cpu().numpy(), pos, off, dtype)
    q = q.abs()                                            # so that -infinity times a query is -infinity
    with np.errstate(invalid="ignore"):
        check_attn(c, q, [n, 1, 1])
    if dtype == "e4m3":
        return
    low = torch.full((40, 2, 128), float("-inf"), dtype=TORCH[act], device="cuda")
    one = torch.ones_like(low)
    P.paged_store(c.t, low, one, dev(np.arange(40)), dev([0, 0, 0, 40]))
    O.store(c.o, low.double().cpu().numpy(), one.double().cpu().numpy(), np.arange(40), np.array([0, 0, 0, 40]), dtype)
    out = check_attn(c, q, [n, 1, 1])
    assert (out[n + 1] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,group,dh,most,longest", [(1, 2, 64, 1, 1500), (1, 4, 128, 3, 2100), (4, 4, 128, 40, 300), (2, 2, 64, 40, 700), (2, 2, 128, 45, 900), (1, 4, 128, 30, 4200)])
def test_attention_of_more_sequences_than_a_wavefront_has_lanes(heads, group, dh, most, longest, dtype):
    """70 sequences, some without keys and some without rows, whose keys are cut into slices, or whose rows make blocks of 128."""
    g = np.random.default_rng(heads * dh + most)
    lens = (longest ** g.random(70)).astype(int) - 1
    lens[5], lens[69] = longest, longest - 1
    counts = g.integers(0, most + 1, 70)
    counts[5] = counts[68] = most
    c = Cache([int(n) for n in lens], 32, heads, dh, dtype, seed=most, holes=0.05).fill()
    check_attn(c, rows(g, (int(counts.sum()) + 1, heads * group, dh), "bf16"), counts, most=most + 1)


@pytest.mark.parametrize("act", ["bf16", "fp32"])
@pytest.mark.parametrize("dh,n", [(32, 1), (64, 1), (128, 1), (64, 300), (128, 300)])
def test_every_code_and_scale_comes_out_of_the_attention_as_it_is_held(act, dh, n):
    """One key in each sequence, whose probability is 1: the result is its V row, bit for bit. All 256 codes with the scales of -110
    to 120, with one row a sequence and (bf16, 64 and 128 dims) with enough for the kernel of 128-row blocks."""
    if act == "fp32" and n > 1:
        pytest.skip("one kernel")
    heads, lens = 256 // dh, [1] * (231 if n == 1 else 6)
    c = Cache(lens, 16, heads, dh, "e4m3", wider=0)
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(heads, dh)
    first = torch.from_numpy(c.o["table"][:, 0]).cuda()
    scale = (torch.arange(len(lens), device="cuda") * (230 // (len(lens) - 1)) + 17).to(torch.uint8)
    c.t.v_pages.view(torch.uint8)[first, :, 0] = codes
    c.t.v_scale.view(torch.uint8)[first, :, 0] = scale[:, None].expand(-1, heads)
    c.t.k_pages.view(torch.uint8)[first, :, 0] = 0
    c.t.k_scale.view(torch.uint8)[first, :, 0] = 127
    q = rows(np.random.default_rng(1), (n * len(lens), 8 * heads if n > 1 else heads, dh), act)
    out = torch.zeros_like(q)
    P.paged_attn(c.t, q, dev(np.arange(len(lens) + 1) * n), out, n, workspace(c, q, n))
    held = O.e4m3_values().reshape(1, heads, 1, dh) * 2.0 ** (scale.double().cpu().numpy() - 127.0)[:, None, None, None]
    want = np.broadcast_to(np.repeat(held, n, axis=0), (len(q), heads, q.shape[1] // heads, dh)).reshape(q.shape)
    got = out.double().cpu().numpy()
    finite = np.abs(want) <= 3.4e38                       # 256 * 2^120 and more is not held by a store
    assert np.array_equal(got[finite | np.isnan(want)], want[finite | np.isnan(want)], equal_nan=True)


def test_fp32_rows_of_all_magnitudes_are_quantised_as_the_oracle_does():
    """Random bit patterns: denormals, infinities, NaN among them; rows of one exponent, where ties and the border between two scales lie."""
    g = np.random.default_rng(12)
    bits = g.integers(0, 2 ** 32, (200, 64), dtype=np.uint64).astype(np.uint32)
    near = ((g.integers(1, 255, (200, 1)).astype(np.uint32) << 23) | (g.integers(0, 16, (200, 64)).astype(np.uint32) << 19)) + g.integers(0, 2, (200, 64)).astype(np.uint32)
    x = torch.from_numpy(np.concatenate([bits, near]).view(np.float32)).cuda().view(2, 200, 64)
    c = Cache([2], 16, 200, 64, "e4m3")
    P.paged_store(c.t, x, x, dev([0, 1]), dev([0, 2]))
    y = x.double().cpu().numpy()
    O.store(c.o, y, y, np.array([0, 1]), np.array([0, 2]), "e4m3")
    assert c.same()


@pytest.mark.parametrize("act", ["bf16", "fp32"])
def test_rows_that_start_at_any_element(act):
    """Rows and results in the middle of other tensors, at odd elements: every call, few rows and many."""
    for n, dh in ((2, 32), (3, 128), (300, 128)):
        c = Cache([n + 40, 30], 16, 2, dh, "e4m3", seed=n).fill(act)
        g = np.random.default_rng(n)
        inside = lambda *shape: rows(g, (int(np.prod(shape)) + 8,), act)[3:3 + int(np.prod(shape))].view(shape)
        k, v, q, out = inside(n, 2, dh), inside(n, 2, dh), inside(n + 1, 16, dh), inside(n + 1, 16, dh).fill_(7.0)
        P.paged_store(c.t, k, v, dev(np.arange(n)), dev([0, n, n]))
        O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), np.arange(n), np.array([0, n, n]), "e4m3")
        assert c.same()
        ko, vo = inside(n, 2, dh), inside(n, 2, dh)
        P.paged_load(c.t, ko, vo, dev(np.arange(n)), dev([0, n, n]))
        wk, wv = np.zeros(k.shape), np.zeros(k.shape)
        O.load(c.o, np.arange(n), np.array([0, n, n]), wk, wv)
        assert np.array_equal(ko.double().cpu().numpy(), wk) and np.array_equal(vo.double().cpu().numpy(), wv)
        check_attn(c, q, [n, 1], out=out)


def test_two_calls_at_once_on_two_streams():
    """Long enough to overlap, each with a workspace of its own: the same bits as one after the other."""
    c = Cache([9000, 7000], 64, 4, 128, "bf16", seed=21).fill()
    qs = [rows(np.random.default_rng(i), (2, 28, 128), "bf16") for i in range(2)]
    ws, want, got = [], [], []
    for q in qs:
        ws.append(workspace(c, q, 1))
        want.append(torch.zeros_like(q))
        got.append(torch.zeros_like(q))
        P.paged_attn(c.t, q, None, want[-1], 1, ws[-1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                P.paged_attn(c.t, qs[i], None, got[i], 1, ws[i])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_lengths_out_of_range_are_those_of_the_table():
    c = Cache([100, 64], 16, 2, 128, "bf16", seed=4, wider=0, lengths=[100, 64]).fill()
    q = rows(np.random.default_rng(4), (3, 2, 128), "bf16")
    top = c.o["table"].shape[1] * 16
    k, v = (rows(c.g, (top - 100, 2, 128), "bf16") for _ in "kv")
    P.paged_store(c.t, k, v, dev(np.arange(100, top)), dev([0, top - 100, top - 100]))
    O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), np.arange(100, top), np.array([0, top - 100, top - 100]), "bf16")
    c.t.seq_len.copy_(dev([2 ** 31 - 1, -5]))
    c.o["lengths"] = np.array([top, 0])
    check_attn(c, q, [2, 1])


def test_a_generation_in_a_captured_graph():
    """Project, store, attend, as a decode loop does: captured once, replayed while positions, lengths and tables move on, with eager
    work in between; each replay against the oracle's cache and attention. Another graph shares the workspace."""
    heads, dh, page = 2, 128, 16
    c = Cache([60, 33, 5], page, heads, dh, "e4m3", seed=8, wider=2).fill()
    free = iter(sorted(set(range(c.t.k_pages.shape[0])) - set(c.o["table"][c.o["table"] >= 0].tolist())))
    g = np.random.default_rng(8)
    w = (rows(g, (4 * heads * dh, 256), "bf16") * 0.1).contiguous()
    x, pos = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    qkv = torch.zeros((3, 4 * heads, dh), device="cuda")
    q, out, other = (torch.zeros((3, 2 * heads, dh), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    ws = workspace(c, q, 1)

    def step():
        qkv.copy_(P.gemm(x, w, P.BF16).view(3, 4 * heads, dh))
        P.paged_store(c.t, qkv[:, 2 * heads:3 * heads], qkv[:, 3 * heads:], pos)
        q.copy_(qkv[:, :2 * heads])
        P.paged_attn(c.t, q, None, out, 1, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                             # warm-up; its positions are written again below
    torch.cuda.current_stream().wait_stream(side)
    O.store(c.o, np.zeros((3, heads, dh)), np.zeros((3, heads, dh)), np.zeros(3, int), None, "e4m3")
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    with torch.cuda.graph(second):
        P.paged_attn(c.t, q, None, other, 1, ws)
    lens = c.o["lengths"].copy()
    for t in range(6):
        for b in range(3):
            if c.o["table"][b, lens[b] // page] < 0:       # a new page for a sequence that has filled its last one
                c.o["table"][b, lens[b] // page] = next(free)
        lens += 1
        c.o["lengths"] = lens
        c.t.page_table.copy_(dev(c.o["table"]))
        c.t.seq_len.copy_(dev(lens))
        pos.copy_(dev(lens - 1))
        x.copy_(rows(g, (3, 256), "bf16"))
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        new = qkv.double().cpu().numpy()
        O.store(c.o, new[:, 2 * heads:3 * heads], new[:, 3 * heads:], lens - 1, None, "e4m3")
        assert c.same()
        ref, spread, size = O.attn(c.o, q.double().cpu().numpy(), None)
        assert (np.abs(out.double().cpu().numpy() - ref) <= bars(q, c, ref, spread, size)).all()
        assert torch.equal(out.view(torch.int16), other.view(torch.int16))
        eager = torch.zeros_like(out)
        P.paged_attn(c.t, q, None, eager, 1, ws)
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16))


def test_calls_on_a_stream_of_their_own():
    c = Cache([300, 20], 16, 4, 128, "bf16", seed=2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.fill()
        check_attn(c, rows(np.random.default_rng(2), (9, 8, 128), "bf16"), [5, 4])
    side.synchronize()
    assert c.same()


def test_rows_beyond_the_bound_of_a_sequence_are_left_out():
    """The host's bound is too small for the first sequence: its rows beyond it stay as they are, all others are right."""
    c = Cache([50, 60], 16, 2, 128, "bf16", seed=3).fill()
    q = rows(np.random.default_rng(3), (10, 2, 128), "bf16")
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    P.paged_attn(c.t, q, dev([0, 8, 10]), out, 5, workspace(c, q, 5))
    assert (out[5:8] == 7.0).all()
    ref, spread, size = O.attn(c.o, q.double().cpu().numpy(), [0, 8, 10])
    ok = np.r_[0:5, 8:10]
    assert (np.abs(out.double().cpu().numpy() - ref) <= bars(q, c, ref, spread, size))[ok].all()


@pytest.mark.parametrize("group,n", [(4, 300), (2, 3)])
def test_offsets_that_go_on_behind_the_rows_of_a_call(group, n):
    """Sequences whose rows lie behind those of the call, with more keys than the one that has them: what is there is complete."""
    c = Cache([200, 700, 600, 650], 16, 8, 128, "bf16", seed=2).fill()
    q = rows(np.random.default_rng(2), (n, 8 * group, 128), "bf16")
    out = torch.full_like(q, 7.0)
    P.paged_attn(c.t, q, dev([0, n, 2 * n, 3 * n, 4 * n]), out, n, workspace(c, q, n))
    ref, spread, size = O.attn(c.o, q.double().cpu().numpy(), np.array([0, n, n, n, n]))
    fits = np.abs(out.double().cpu().numpy() - ref) <= bars(q, c, ref, spread, size)
    assert fits.all()


def test_positions_behind_four_gigabytes():
    """Pages whose offsets pass 32 bits: 2^18 slots of 4 heads of 128 dims behind the first ones, in bf16 2.1 GB a million rows."""
    page, heads, dh, n_pages = 4096, 4, 128, 1100
    k = torch.zeros((n_pages, heads, page, dh), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() * 2 > 1 << 32
    table = dev([[n_pages - 1, 3]])
    cache = P.PagedCache(k, v, table, dev([5000]))
    g = np.random.default_rng(7)
    kn, vn = (rows(g, (3, heads, dh), "bf16") for _ in "kv")
    pos = dev([4095, 17, 4999])
    P.paged_store(cache, kn, vn, pos, dev([0, 3]))
    assert torch.equal(k[n_pages - 1, :, 4095], kn[0]) and torch.equal(v[n_pages - 1, :, 17], vn[1]) and torch.equal(k[3, :, 903], kn[2])
    ko, vo = torch.zeros_like(kn), torch.zeros_like(vn)
    P.paged_load(cache, ko, vo, pos, dev([0, 3]))
    assert torch.equal(ko, kn) and torch.equal(vo, vn)
    q = rows(g, (1, heads, dh), "bf16")
    out = torch.zeros_like(q)
    ws = torch.empty(P.paged_attn_workspace_bytes(cache, heads, 1, 1), dtype=torch.uint8, device="cuda")
    P.paged_attn(cache, q, None, out, 1, ws)
    s = (kn.double() * q.double()).sum(-1) / dh ** 0.5                                 # scores of the three rows; 4997 of zero
    w = torch.exp(s)
    ref = (w[..., None] * vn.double()).sum(0) / (w.sum(0) + 4997.0)[:, None]
    assert ((out.double()[0] - ref).abs() <= 2.0 ** -7 * ref.abs() + 2.0 ** -7 * (w[..., None] * vn.double().abs()).sum(0) / 4997).all()
