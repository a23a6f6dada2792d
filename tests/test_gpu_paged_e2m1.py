"""Paged K/V cache in 4 bits on the GPU: rows written, read back and attended to, against the oracle. Caches, checks and bars are those of
test_gpu_paged.py (an element is exact in bf16 and fp32, so that nothing but the values that are held differs from the other caches), and
an absolute one: many held values are exactly zero, so that a result can come from keys of vanishing probability alone. Exponentials and their
factors below 2^-126 become zero. They are taken against a reference that is at most 2^8 behind the largest score (blocks of 128 rows; the
others have the largest itself), and the sum of all is at least 1 in units of the largest: what is lost is below 2^(8 - 126) of |v| for
each key."""
import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
import test_gpu_paged as paged
import test_gpu_paged_calls as calls
from oracle import paged as O
from paged_shapes import BLOCKS, E2M1_CALLS, plan_of
from plans import paged_plan
from test_gpu_paged import ATTN, TORCH, Cache, check_attn, dev, rows, workspace

pytestmark = pytest.mark.gpu


class FourBits(Cache):
    """A cache of this type; everything that is not stored is NaN on both sides."""

    def __init__(self, lens, page, heads, dh, dtype="e2m1", **kw):
        super().__init__(lens, page, heads, dh, "e4m3", **kw)
        assert dtype == "e2m1"
        self.dtype = dtype
        n_pages = self.t.k_pages.shape[0]
        pages = [torch.full((n_pages, heads, page, dh // 2), 0xFF, dtype=torch.uint8, device="cuda").view(torch.float4_e2m1fn_x2) for _ in "kv"]
        scales = [torch.full((n_pages, heads, page, dh // 32), 0xFF, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in "kv"]
        self.t = P.PagedCache(*pages, self.t.page_table, self.t.seq_len, *scales)

    def values(self, which):
        pages, scale = (self.t.k_pages, self.t.k_scale) if which == "k" else (self.t.v_pages, self.t.v_scale)
        codes, e = pages.view(torch.uint8).cpu().numpy(), scale.view(torch.uint8).cpu().numpy().astype(int)
        x = O.e2m1_values()[np.stack([codes & 15, codes >> 4], -1)].reshape(codes.shape[:-1] + (-1, 32))
        return (x * np.where(e == 255, np.nan, 2.0 ** (e - 127.0))[..., None]).reshape(codes.shape[:-1] + (-1,))


@pytest.fixture(autouse=True)
def bars_with_what_vanishes(monkeypatch):
    plain = paged.bars

    def bars(q, cache, ref, spread, most):
        v = cache.o["v"][np.isfinite(cache.o["v"])]
        return plain(q, cache, ref, spread, most) + 2.0 ** -118 * int(cache.o["lengths"].max()) * np.abs(v).max(initial=0.0)

    monkeypatch.setattr(paged, "bars", bars)
    monkeypatch.setattr(calls, "bars", bars)


def exponents(cache, which, n):
    """Exponents of the scales of the first n positions of sequence 0, [n, heads, dh / 32]."""
    scale = cache.t.k_scale if which == "k" else cache.t.v_scale
    at = [O.place(cache.o, 0, p) for p in range(n)]
    return scale.view(torch.uint8).cpu().numpy().astype(int)[[a[0] for a in at], :, [a[1] for a in at]] - 127


@pytest.mark.parametrize("act", ["bf16", "fp32"])
@pytest.mark.parametrize("dh,heads,page", [(128, 4, 16), (64, 1, 32), (32, 3, 256), (128, 33, 64), (32, 1, 16)])
def test_rows_are_held_to_the_bit_and_read_back(act, dh, heads, page):
    c = FourBits([5, 0, 70, 1, page], page, heads, dh, seed=dh + page, holes=0.2).fill(act)
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
    O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), pos, off, "e2m1")
    assert c.same()
    for out in ("bf16", "fp32"):
        ko, vo = (torch.full((len(pos), heads, dh), 7.0, dtype=TORCH[out], device="cuda") for _ in "kv")
        P.paged_load(c.t, ko, vo, dev(pos), dev(off))
        wk, wv = (np.full((len(pos), heads, dh), 7.0) for _ in "kv")
        O.load(c.o, pos, off, wk, wv)
        assert np.array_equal(ko.double().cpu().numpy(), wk, equal_nan=True) and np.array_equal(vo.double().cpu().numpy(), wv, equal_nan=True)


@pytest.mark.parametrize("out,heads,dh", [("bf16", 33, 128), ("fp32", 20, 64), ("bf16", 65, 32)])
def test_many_rows_are_read_back(out, heads, dh):
    """Calls large enough that a lane reads several pieces, the last ones of a row not all there; rows without a page, rows of no sequence."""
    c = FourBits([700, 0, 850], 32, heads, dh, seed=heads, holes=0.1).fill()
    off = np.array([0, 700, 700, 1550])
    pos = np.concatenate([np.random.default_rng(1).permutation(700), np.random.default_rng(2).permutation(850), [3, 4, 5]])
    ko, vo = (torch.full((1553, heads, dh), 7.0, dtype=TORCH[out], device="cuda") for _ in "kv")
    P.paged_load(c.t, ko, vo, dev(pos), dev(off))
    wk, wv = (np.full((1553, heads, dh), 7.0) for _ in "kv")
    O.load(c.o, pos, off, wk, wv)
    assert np.array_equal(ko.double().cpu().numpy(), wk) and np.array_equal(vo.double().cpu().numpy(), wv)


@pytest.mark.parametrize("act,heads,dh", [("bf16", 33, 128), ("fp32", 33, 128), ("fp32", 45, 64), ("bf16", 45, 64), ("bf16", 97, 32), ("fp32", 97, 32)])
def test_many_rows_are_stored(act, heads, dh):
    """Calls large enough that a wavefront has several heads, the last ones not all there: more sequences than it has lanes, some without rows, positions in any
    order, some without a page; rows of no sequence, which are parts of longer ones."""
    g = np.random.default_rng(dh)
    lens = g.integers(0, 45, 71)
    c = FourBits([int(n) for n in lens], 16, heads, dh, seed=heads, holes=0.1)
    counts = np.where(g.random(71) < 0.2, 0, lens)
    counts[70] = 0
    off = np.concatenate([[0], np.cumsum(counts)])
    n = int(off[-1]) + 3
    assert -(-n // (4096 // dh)) * 2 * heads >= 2048
    pos = np.concatenate([g.permutation(int(lens[b]))[:counts[b]] for b in range(71)] + [[0, 1, 2]]).astype(int)
    wide = rows(g, (n, 2 * heads + 1, dh), act)
    k, v = wide[:, :heads], wide[:, heads + 1:]
    P.paged_store(c.t, k, v, dev(pos), dev(off))
    O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), pos, off, "e2m1")
    assert c.same()


def test_every_bf16_value_is_quantised_as_the_oracle_does():
    """All 65536 bit patterns, 32 to a block: blocks of one magnitude (all exponents, zeros, infinities, NaN) and shuffled ones."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    mixed = bits[torch.randperm(65536, generator=torch.Generator().manual_seed(1))]
    x = torch.cat([bits, mixed]).view(1, -1, 32).cuda().expand(2, -1, -1).contiguous()
    c = FourBits([2], 16, x.shape[1], 32)
    P.paged_store(c.t, x, x, dev([0, 1]), dev([0, 2]))
    y = x.double().cpu().numpy()
    O.store(c.o, y, y, np.array([0, 1]), np.array([0, 2]), "e2m1")
    assert c.same()
    assert np.array_equal(exponents(c, "k", 2), O.quantise_e2m1(y)[1])
    ko, vo = (torch.zeros_like(x) for _ in "kv")
    P.paged_load(c.t, ko, vo, dev([1, 0]), dev([0, 2]))
    want = c.o["k"][int(c.o["table"][0, 0]), :, :2].transpose(1, 0, 2)[::-1]
    assert np.array_equal(ko.double().cpu().numpy(), want, equal_nan=True) and torch.equal(ko.view(torch.int16), vo.view(torch.int16))


@pytest.mark.parametrize("dh", [64, 128])
def test_fp32_rows_of_all_magnitudes_are_quantised_as_the_oracle_does(dh):
    """Random bit patterns: denormals, infinities, NaN among them; blocks of one exponent, where ties and the border between two scales lie."""
    g = np.random.default_rng(12)
    bits = g.integers(0, 2 ** 32, (200, dh), dtype=np.uint64).astype(np.uint32)
    near = ((g.integers(1, 255, (200, 1)).astype(np.uint32) << 23) | (g.integers(0, 8, (200, dh)).astype(np.uint32) << 20)) + g.integers(0, 2, (200, dh)).astype(np.uint32)
    x = torch.from_numpy(np.concatenate([bits, near]).view(np.float32)).cuda().view(2, 200, dh)
    c = FourBits([2], 16, 200, dh)
    P.paged_store(c.t, x, x, dev([0, 1]), dev([0, 2]))
    y = x.double().cpu().numpy()
    O.store(c.o, y, y, np.array([0, 1]), np.array([0, 2]), "e2m1")
    assert c.same() and np.array_equal(exponents(c, "v", 2), O.quantise_e2m1(y)[1])


def test_one_row_per_sequence_of_a_batch_beyond_a_wavefront():
    """Without row offsets, and with them, for 131 sequences: stored, read back, attended to."""
    lens = [int(x) for x in np.random.default_rng(5).integers(0, 50, 131)]
    c = FourBits(lens, 16, 2, 64, seed=5).fill()
    g = np.random.default_rng(6)
    pos = np.maximum(np.array(lens) - 1, 0)
    k, v = (rows(g, (131, 2, 64), "bf16") for _ in "kv")
    P.paged_store(c.t, k, v, dev(pos))
    O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), pos, None, "e2m1")
    assert c.same()
    ko, vo = (torch.zeros((131, 2, 64), dtype=torch.float32, device="cuda") for _ in "kv")
    P.paged_load(c.t, ko, vo, dev(pos))
    wk, wv = np.zeros((131, 2, 64)), np.zeros((131, 2, 64))
    O.load(c.o, pos, None, wk, wv)
    assert np.array_equal(ko.double().cpu().numpy(), wk) and np.array_equal(vo.double().cpu().numpy(), wv)
    q = rows(g, (131, 6, 64), "bf16")
    a, b = check_attn(c, q, [1] * 131, off=None), check_attn(c, q, [1] * 131)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("act", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(ATTN)))
@pytest.mark.parametrize("holes", [0.0, 0.25])
def test_attention(act, case, holes):
    lens, counts, page, heads, group, dh = ATTN[case]
    c = FourBits(lens, page, heads, dh, seed=case, holes=holes, wider=2).fill(act)
    g = np.random.default_rng(case)
    R = sum(counts)
    q = rows(g, (R + 2, heads * (group + 1), dh), act)[:, heads:]          # rows that are parts of longer ones, two behind the last sequence
    if R + 2 > len(counts) * max(counts):
        q = q[:R]
    check_attn(c, q, counts, most=max(counts) if case % 2 else max(counts) + 3)


@pytest.mark.parametrize("act", ["bf16", "fp32"])
@pytest.mark.parametrize("batch,heads,group,dh,longest,most", [(70, 4, 2, 32, 1100, 1), (20, 16, 1, 128, 1060, 3), (300, 1, 4, 64, 1500, 2), (65, 4, 1, 128, 1024, 20)])
def test_whole_sequences_in_the_order_of_their_lengths(act, batch, heads, group, dh, longest, most):
    """Several rounds of workgroups over a table of 1024 positions and more: lengths that are equal, zero, and as wide as the table; sequences without rows."""
    g = np.random.default_rng(batch)
    lens = (longest * g.random(batch) ** 6).astype(int)
    lens[g.integers(0, batch, batch // 4)] = 0
    lens[batch // 2], lens[batch - 1] = longest, longest
    counts = g.integers(0, most + 1, batch) if most > 1 else np.ones(batch, int)
    counts[[0, batch // 2, batch - 1]] = most
    p = paged_plan(heads * group, int(counts.sum()), most, {"bf16": P.BF16, "fp32": P.FP32}[act], batch, -(-longest // 16), 16, heads, dh, P.E2M1)
    assert p.kernel == "split" and 256 < p.cap * heads * p.q_groups <= 1024
    c = FourBits(lens.tolist(), 16, heads, dh, seed=batch, holes=0.1).fill(act)
    q = rows(g, (int(counts.sum()), heads * group, dh), act)
    check_attn(c, q, counts.tolist(), most=most)


@pytest.mark.parametrize("group,most,dh", [(1, 1, 128), (7, 2, 128), (7, 2, 64), (1, 3, 32)])
def test_slices_for_two_workgroups_of_a_compute_unit(group, most, dh):
    lens = [8200, 0, 200, 1] + [int(x) for x in np.random.default_rng(8).integers(0, 180, 27)] + [2500]
    counts = [most] * 16 + [1] * 16
    p = paged_plan(8 * group, sum(counts), most, P.BF16, 32, 129, 64, 8, dh, P.E2M1)
    assert p.kernel == "split+" and p.want == 64
    c = FourBits(lens, 64, 8, dh, seed=9, holes=0.05).fill("bf16")
    q = rows(np.random.default_rng(10), (sum(counts), 8 * group, dh), "bf16")
    a, b = check_attn(c, q, counts, most=most), check_attn(c, q, counts, most=most)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("dh", [64, 32])
def test_slices_of_small_heads(dh):
    lens, counts = [5000, 0, 1300], [1, 1, 2]
    p = paged_plan(4 * 7, 4, 2, P.BF16, 3, 157, 32, 4, dh, P.E2M1)
    assert p.kernel == "split+" and p.want == 128
    c = FourBits(lens, 32, 4, dh, seed=11, holes=0.1).fill("bf16")
    check_attn(c, rows(np.random.default_rng(12), (4, 28, dh), "bf16"), counts, most=2)


def make(name, types, seed, size=1.0):
    lens, counts, page, heads, group, dh, kernel = E2M1_CALLS[name]
    act, dtype = types.split()
    if act == "bf16":
        assert plan_of(name, P.E2M1, calls=E2M1_CALLS).kernel == kernel
    c = FourBits(lens, page, heads, dh, seed=seed).fill(act, size=size)
    extra = min(2, len(counts) * max(counts) - sum(counts))
    return c, rows(np.random.default_rng(seed), (sum(counts) + extra, heads * group, dh), act), counts


EVERY = [(name, act + " e2m1") for name in E2M1_CALLS for act in (("bf16",) if name in BLOCKS else ("bf16", "fp32"))]


@pytest.mark.parametrize("name,types", EVERY, ids=[n + "-" + t.replace(" ", "-") for n, t in EVERY])
@pytest.mark.parametrize("check", ["scores_of_hundreds", "scores_that_grow_and_fall_along_a_sequence", "infinities_and_nan_act_where_they_are_seen",
                                   "addresses_of_any_element", "pages_that_are_missing",
                                   "scores_of_minus_infinity_only_give_zeros_whatever_the_values",
                                   "the_probabilities_that_weigh_the_values_sum_to_one", "a_table_that_is_much_wider_than_its_sequences"])
def test_every_kernel(name, types, check, monkeypatch):
    """What test_gpu_paged_calls.py asks of the other caches (an infinity or a NaN is one of 32 dims here)."""
    monkeypatch.setattr(calls, "Cache", FourBits)
    monkeypatch.setattr(calls, "make", make)
    monkeypatch.setattr(calls, "CALLS", E2M1_CALLS)
    getattr(calls, "test_" + check)(name, types)


def test_an_active_set_that_shrinks_keeps_its_workspace(monkeypatch):
    monkeypatch.setattr(calls, "Cache", FourBits)
    calls.test_an_active_set_that_shrinks_keeps_its_workspace("e2m1")


@pytest.mark.parametrize("name,types", EVERY, ids=[n + "-" + t.replace(" ", "-") for n, t in EVERY])
def test_a_block_of_nan_is_seen_by_its_dims_only(name, types):
    """V rows with one block of NaN: its 32 dims are NaN for all that see the row, all others are as they would be."""
    act = types.split()[0]
    c, q, counts = make(name, types, 43)
    b = int(np.argmax(c.o["lengths"]))
    n, block = int(c.o["lengths"][b]), c.dh // 32 - 1
    k, v = (rows(np.random.default_rng(i), (1, c.heads, c.dh), act) for i in (44, 45))
    v[0, 0, 32 * block + 7] = float("nan")
    calls.store(c, b, [n // 2], k, v)
    out = check_attn(c, q, counts)
    r0 = sum(counts[:b])
    group = q.shape[1] // c.heads
    bad = torch.isnan(out[r0:r0 + counts[b]])
    assert bad[:, :group, 32 * block:].all() and not bad[:, :group, :32 * block].any() and not bad[:, group:].any()


@pytest.mark.parametrize("act,dh,n", [(act, dh, 1) for act in ("bf16", "fp32") for dh in (32, 64, 128)] + [("bf16", 64, 300), ("bf16", 128, 300)])
def test_every_code_and_scale_comes_out_of_the_attention_as_it_is_held(act, dh, n):
    """One key in each sequence, whose probability is 1: the result is its V row, bit for bit. All pairs of codes with the scales of -110
    to 125, and of 126 where they are held, a different one for each block of a row."""
    heads, lens = 512 // dh, [1] * (237 if n == 1 else 8)
    c = FourBits(lens, 16, heads, dh, wider=0)
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(heads, dh // 2)
    first = torch.from_numpy(c.o["table"][:, 0]).cuda()
    step = 1 if n == 1 else 29
    e = 17 + (torch.arange(len(lens), device="cuda")[:, None] * step + torch.arange(16, device="cuda")[None, :] * 7) % 237
    c.t.v_pages.view(torch.uint8)[first, :, 0] = codes
    c.t.v_scale.view(torch.uint8)[first, :, 0] = e.view(len(lens), heads, dh // 32).to(torch.uint8)
    c.t.k_pages.view(torch.uint8)[first, :, 0] = 0
    c.t.k_scale.view(torch.uint8)[first, :, 0] = 127
    q = rows(np.random.default_rng(1), (n * len(lens), 8 * heads if n > 1 else heads, dh), act)
    out = torch.zeros_like(q)
    P.paged_attn(c.t, q, dev(np.arange(len(lens) + 1) * n), out, n, workspace(c, q, n))
    pair = np.arange(256)
    held = (O.e2m1_values()[np.stack([pair & 15, pair >> 4], -1)].reshape(16, 32) * 2.0 ** (e.double().cpu().numpy() - 127.0)[..., None])
    held = held.reshape(len(lens), heads, 1, dh)
    want = np.broadcast_to(np.repeat(held, n, axis=0), (len(q), heads, q.shape[1] // heads, dh)).reshape(q.shape)
    got = out.double().cpu().numpy()
    finite = np.abs(want) <= 3.4e38                       # 4 * 2^126 is not held by a store
    assert finite.mean() > 0.9 and np.array_equal(got[finite], want[finite])


@pytest.mark.parametrize("act", ["bf16", "fp32"])
def test_rows_that_start_at_any_element(act):
    """Rows and results in the middle of other tensors, at odd elements: every call, few rows and many."""
    for n, dh in ((2, 32), (3, 128), (300, 128)):
        c = FourBits([n + 40, 30], 16, 2, dh, seed=n).fill(act)
        g = np.random.default_rng(n)
        inside = lambda *shape: rows(g, (int(np.prod(shape)) + 8,), act)[3:3 + int(np.prod(shape))].view(shape)
        k, v, q, out = inside(n, 2, dh), inside(n, 2, dh), inside(n + 1, 16, dh), inside(n + 1, 16, dh).fill_(7.0)
        P.paged_store(c.t, k, v, dev(np.arange(n)), dev([0, n, n]))
        O.store(c.o, k.double().cpu().numpy(), v.double().cpu().numpy(), np.arange(n), np.array([0, n, n]), "e2m1")
        assert c.same()
        ko, vo = inside(n, 2, dh), inside(n, 2, dh)
        P.paged_load(c.t, ko, vo, dev(np.arange(n)), dev([0, n, n]))
        wk, wv = np.zeros(k.shape), np.zeros(k.shape)
        O.load(c.o, np.arange(n), np.array([0, n, n]), wk, wv)
        assert np.array_equal(ko.double().cpu().numpy(), wk) and np.array_equal(vo.double().cpu().numpy(), wv)
        check_attn(c, q, [n, 1], out=out)


def test_positions_behind_four_gigabytes():
    """Pages whose offsets pass 32 bits, those of the scales too: 2^30 / 16 rows of 128 dims in 4 bits are 4.3 GB, their scales 268 MB; the
    last page of 1100 of 65536 slots of one head lies behind 4.6 GB."""
    page, heads, dh, n_pages = 65536, 1, 128, 1100
    k, v = (torch.zeros((n_pages, heads, page, dh // 2), dtype=torch.uint8, device="cuda") for _ in "kv")
    ks, vs = (torch.full((n_pages, heads, page, dh // 32), 127, dtype=torch.uint8, device="cuda") for _ in "kv")
    assert k.numel() > 1 << 32
    four, eight = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
    cache = P.PagedCache(k.view(four), v.view(four), dev([[n_pages - 1, 3]]), dev([65536 + 5000]), ks.view(eight), vs.view(eight))
    g = np.random.default_rng(7)
    kn, vn = (rows(g, (3, heads, dh), "bf16") for _ in "kv")
    pos = dev([65535, 17, 65536 + 4999])
    P.paged_store(cache, kn, vn, pos, dev([0, 3]))
    assert ks[n_pages - 1, :, 65535].ne(127).any() and int(ks.ne(127).any(-1).sum()) <= 3
    ko, vo = torch.zeros_like(kn), torch.zeros_like(vn)
    P.paged_load(cache, ko, vo, pos, dev([0, 3]))
    hk, hv = (O.quantise_e2m1(x.double().cpu().numpy())[0] for x in (kn, vn))
    assert np.array_equal(ko.double().cpu().numpy(), hk) and np.array_equal(vo.double().cpu().numpy(), hv)
    q = rows(g, (1, heads, dh), "bf16")
    out = torch.zeros_like(q)
    ws = torch.empty(P.paged_attn_workspace_bytes(cache, heads, 1, 1), dtype=torch.uint8, device="cuda")
    P.paged_attn(cache, q, None, out, 1, ws)
    w = np.exp((hk * q.double().cpu().numpy()).sum(-1) / dh ** 0.5)                    # of the three rows; all others have scores of zero
    total = w.sum(0) + 65536 + 5000 - 3
    ref = (w[..., None] * hv).sum(0) / total[:, None]
    bar = 2.0 ** -7 * np.abs(ref) + 2.0 ** -7 * (w[..., None] * np.abs(hv)).sum(0) / total[:, None]
    assert (np.abs(out.double().cpu().numpy()[0] - ref) <= bar).all()


@pytest.mark.parametrize("act", ["bf16", "fp32"])
@pytest.mark.parametrize("batch,heads,group,dh,longest,most", [(64, 8, 2, 64, 1100, 2), (64, 16, 1, 32, 1024, 1), (64, 5, 1, 128, 1700, 3), (2, 140, 1, 32, 1100, 1)])
def test_a_wavefront_of_sequences_in_the_order_of_their_lengths(act, batch, heads, group, dh, longest, most):
    """Up to 64 sequences, all in order; lengths that are equal, zero, and as wide as the table."""
    g = np.random.default_rng(batch + heads)
    lens = (longest * g.random(batch) ** 4).astype(int)
    lens[g.integers(0, batch, batch // 4)] = 0
    lens[batch - 1], lens[0] = longest, lens[batch // 2]
    counts = g.integers(0, most + 1, batch) if most > 1 else np.ones(batch, int)
    counts[[0, batch - 1]] = most
    p = paged_plan(heads * group, int(counts.sum()), most, {"bf16": P.BF16, "fp32": P.FP32}[act], batch, -(-longest // 16), 16, heads, dh, P.E2M1)
    assert p.kernel == "split" and p.longest_first
    c = FourBits(lens.tolist(), 16, heads, dh, seed=batch, holes=0.1, wider=0).fill(act)
    q = rows(g, (int(counts.sum()), heads * group, dh), act)
    check_attn(c, q, counts.tolist(), most=most)
