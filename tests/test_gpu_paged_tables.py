"""Page tables that follow the lengths on the GPU, against the oracle: whole numbers, all equal."""
import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import tables as O
from plans import resize_launches
from test_gpu_paged import dev

pytestmark = pytest.mark.gpu


class Both:
    """The same tables on the GPU and for the oracle."""

    def __init__(self, batch, width, n_pages, page, seed=0, first=0):
        self.g, self.page, self.n, self.batch, self.width = np.random.default_rng(seed), page, n_pages, batch, width
        self.table, self.len, self.ring, self.at = [[-1] * width for _ in range(batch)], [0] * batch, self.g.permutation(n_pages).tolist(), [first, n_pages]
        self.t = P.PagedTables(dev(self.table), dev(self.len), dev(self.ring), dev(self.at), page)
        self.ws = torch.full((P.paged_resize_workspace_bytes(batch),), 0xFF, dtype=torch.uint8, device="cuda")

    def holes(self, share):
        """Takes pages out of the tables, as somebody who gives them back early does."""
        for row in self.table:
            for j in range(self.width):
                if self.g.random() < share:
                    row[j] = int(self.g.choice([-1, -5, self.n, 2 ** 31 - 1]))
        self.t.page_table.copy_(dev(self.table))

    def resize(self, want, room=8, lists="both", short=0):
        was = list(self.len)
        n = sum(max(0, min(w, self.width * self.page) - x) for w, x in zip(want, was)) + room - short
        rows = max(1, n)
        off = torch.full((self.batch + 1,), -3, dtype=torch.int32, device="cuda")
        pos, slots = torch.full((rows,), -3, dtype=torch.int32, device="cuda"), torch.full((rows,), -3, dtype=torch.int64, device="cuda")
        self.run(want, off, pos, slots, lists)
        want_off, want_pos, want_slots = O.resize(self.table, self.len, self.ring, self.at, self.page, [int(x) for x in want], rows if lists != "none" else None)
        self.same()
        if lists == "none":
            return
        m = want_off[-1]
        assert off.tolist() == want_off
        for name, got, ref in (("positions", pos, want_pos), ("slots", slots, want_slots)):
            if lists in ("both", name):
                assert np.array_equal(got[:m].cpu().numpy(), np.array(ref, dtype=np.int64)) and (got[m:] == -3).all()
            else:
                assert (got == -3).all()

    def run(self, want, off, pos, slots, lists="both"):
        P.paged_resize(self.t, dev(want), self.ws, None if lists == "none" else off, pos if lists in ("both", "positions") else None,
                       slots if lists in ("both", "slots") else None)

    def same(self):
        assert self.t.seq_len.tolist() == self.len
        assert self.t.free_at.tolist() == self.at
        assert np.array_equal(self.t.page_table.cpu().numpy(), np.array(self.table))
        assert np.array_equal(self.t.free_pages.cpu().numpy(), np.array(self.ring))


# batch, pages of a table, pages, page size: one launch, and (many sequences, or rows) three
SIZES = [(1, 1, 1, 16), (1, 700, 600, 16), (3, 9, 20, 16), (64, 40, 1500, 32), (65, 7, 200, 256), (1000, 3, 2000, 16), (1024, 5, 3000, 64), (1025, 4, 3000, 16),
         (2500, 6, 9000, 16), (130, 300, 30000, 16)]


@pytest.mark.parametrize("size", SIZES, ids=[str(s) for s in SIZES])
@pytest.mark.parametrize("holes", [0.0, 0.3])
def test_lengths_come_and_go(size, holes):
    """Sequences that grow, shrink, leave, stay; lengths below zero and beyond the table; too few pages; too few rows; a ring that goes round."""
    batch, width, n, page = size
    b = Both(batch, width, n, page, seed=batch, first=n // 2)
    top = width * page
    b.resize(b.g.integers(0, top // 2 + 1, batch))
    for i in range(6):
        if holes and i % 2:
            b.holes(holes)
        mixed = np.where(b.g.random(batch) < 0.5, np.array(b.len) + b.g.integers(0, page + 3, batch), b.g.integers(-5, top + 7, batch))
        b.resize(np.where(b.g.random(batch) < 0.2, 0, mixed), lists=["both", "positions", "slots", "none", "both", "both"][i], short=[0, 0, 40, 0, 100, 0][i])
    b.resize(np.full(batch, top))
    b.resize(np.zeros(batch, int))
    b.resize(np.full(batch, 1))
    b.resize(np.array(b.len))                              # nothing changes


def test_the_first_that_does_not_fit_stops_those_behind_it():
    b = Both(5, 10, 12, 16)
    b.resize([40, 0, 20, 0, 0])                            # 3 + 2 pages, 7 are left
    b.resize([48, 100, 52, 10, 16])                        # 0 + 7 pages, then 2 too many, and nothing for the last two
    assert b.len == [48, 100, 20, 0, 0] and b.at[1] == 0
    b.resize([0, 100, 32, 10, 16])                         # what is given back is there for the next call
    assert b.len == [0, 100, 32, 0, 0]
    b.resize([0, 100, 32, 10, 16])
    assert b.len == [0, 100, 32, 10, 16]


def test_lengths_that_are_out_of_range_at_the_start():
    """seq_len beyond the table or below zero, a place in the ring beyond it, more free pages than there are: as the documentation takes them."""
    b = Both(3, 4, 30, 16)
    b.table = [[1, 2, 3, 4], [-1] * 4, [5, 6, -1, 40]]
    b.len, b.ring, b.at = [2 ** 31 - 1, -7, 64], list(range(30)), [7 + 60, 5]
    for x, y in ((b.t.page_table, b.table), (b.t.seq_len, b.len), (b.t.free_pages, b.ring), (b.t.free_at, b.at)):
        x.copy_(dev(y))
    b.resize([10, 20, 0])
    b.at = [3, 2 ** 31 - 1]                                # full: what is given back has no room
    b.t.free_at.copy_(dev(b.at))
    b.resize([0, 50, 30])
    b.at = [3, -9]
    b.t.free_at.copy_(dev(b.at))
    b.resize([64, 0, 0])


def test_sums_beyond_32_bits_do_not_fit():
    """1000 sequences that each want 2^30 positions (sums of 2^40 rows, and of 2^36 pages): the first two get their pages where no rows are listed (the
    ring has 2^15), none where they are."""
    batch, page, n = 1000, 65536, 1 << 15
    width = 1 << 14
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    t = P.PagedTables(table, dev(np.zeros(batch)), dev(np.arange(n)), dev([0, n]), page)
    ws = torch.empty(P.paged_resize_workspace_bytes(batch), dtype=torch.uint8, device="cuda")
    want = dev(np.full(batch, 1 << 30))
    off, pos = dev(np.zeros(batch + 1)), dev(np.full(5, -3))
    P.paged_resize(t, want, ws, off, pos)
    assert int(off.abs().max()) == 0 and int(t.seq_len.max()) == 0 and (pos == -3).all() and t.free_at.tolist() == [0, n]
    P.paged_resize(t, want, ws)
    assert t.seq_len.tolist() == [1 << 30] * 2 + [0] * (batch - 2) and t.free_at.tolist() == [0, 0]
    assert torch.equal(table[:2].flatten(), torch.arange(n, dtype=torch.int32, device="cuda")) and (table[2:] == -1).all()


@pytest.mark.parametrize("batch,rows", [(20, 700), (20, 9000), (1030, 40000)])
def test_captured_calls_follow_the_lengths(batch, rows):
    """Two graphs that share tables and workspace, replayed in turn, with eager calls between them."""
    b = Both(batch, 30, 20 * batch, 16, seed=4)
    grow, leave = dev(np.zeros(batch)), dev(np.zeros(batch))
    off, pos, slots = dev(np.zeros(batch + 1)), dev(np.full(rows, -3)), torch.full((rows,), -3, dtype=torch.int64, device="cuda")
    b.resize(np.full(batch, 7))
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        P.paged_resize(b.t, grow, b.ws, off, pos, slots)
    with torch.cuda.graph(second):
        P.paged_resize(b.t, leave, b.ws)
    for i in range(5):
        want = np.array(b.len) + b.g.integers(0, 33, batch)
        grow.copy_(dev(want))
        first.replay()
        o, p, s = O.resize(b.table, b.len, b.ring, b.at, 16, want.tolist(), rows)
        b.same()
        assert off.tolist() == o and pos[:o[-1]].tolist() == p and slots[:o[-1]].tolist() == s
        want = np.where(b.g.random(batch) < 0.3, b.g.integers(0, 5, batch), -1)
        leave.copy_(dev(want))
        second.replay()
        O.resize(b.table, b.len, b.ring, b.at, 16, want.tolist())
        b.same()
        b.resize(np.array(b.len) + 1)


@pytest.mark.parametrize("batch", [300, 1300])
def test_two_tables_on_two_streams(batch):
    both = [Both(batch, 40, 30 * batch, 16, seed=i) for i in range(2)]
    wants = [[b.g.integers(0, 640, batch) for _ in range(8)] for b in both]
    streams = [torch.cuda.Stream() for _ in both]
    dev_wants = [[dev(w) for w in ws] for ws in wants]
    torch.cuda.synchronize()
    for i in range(8):
        for b, s, w in zip(both, streams, dev_wants):
            with torch.cuda.stream(s):
                P.paged_resize(b.t, w[i], b.ws)
    torch.cuda.synchronize()
    for b, ws in zip(both, wants):
        for w in ws:
            O.resize(b.table, b.len, b.ring, b.at, 16, [int(x) for x in w])
        b.same()


# batch, pages of a table, holes: on both sides of the border between one launch and three, for calls without lists and for those with a short one
MOVES = [(1, 1500, 0.0), (7, 900, 0.2), (40, 180, 0.2), (40, 181, 0.2), (512, 13, 0.0), (1024, 7, 0.3), (75, 940, 0.1), (75, 960, 0.1), (1024, 65, 0.0)]


@pytest.mark.parametrize("case", MOVES, ids=[str(m) for m in MOVES])
def test_many_pages_move_for_few_rows_or_none(case):
    """All pages taken without lists, given back with a list of a few rows, taken and given back without, and in parts."""
    batch, width, holes = case
    b = Both(batch, width, batch * width, 16, seed=width, first=3)
    full, none = np.full(batch, 16 * width), np.zeros(batch, int)
    b.resize(full, lists="none")
    if holes:
        b.holes(holes)
    b.resize(none)                                         # with a list of 8 rows
    b.resize(b.g.integers(0, 16 * width + 1, batch), lists="none")
    b.resize(np.where(np.arange(batch) % 3 == 0, np.array(b.len) + 1, 0), room=0)
    b.resize(full, lists="none")
    b.resize(none, lists="none")


def test_the_moves_lie_on_both_sides_of_the_borders():
    forms = {(rows, resize_launches(batch, width, batch * width, rows)) for batch, width, _ in MOVES for rows in (None, 8)}
    assert forms == {(None, 1), (None, 3), (8, 1), (8, 3)}
    assert [resize_launches(40, w, 40 * w) for w in (180, 181)] == [1, 3]


@pytest.mark.parametrize("batch,width", [(60, 40), (1000, 5)])
def test_two_small_tables_on_two_streams(batch, width):
    """One launch each."""
    both = [Both(batch, width, batch * width - 7, 16, seed=i) for i in range(2)]
    assert resize_launches(batch, width, batch * width - 7) == 1
    wants = [[b.g.integers(0, 16 * width + 1, batch) for _ in range(8)] for b in both]
    streams = [torch.cuda.Stream() for _ in both]
    dev_wants = [[dev(w) for w in ws] for ws in wants]
    torch.cuda.synchronize()
    for i in range(8):
        for b, s, w in zip(both, streams, dev_wants):
            with torch.cuda.stream(s):
                P.paged_resize(b.t, w[i], b.ws)
    torch.cuda.synchronize()
    for b, ws in zip(both, wants):
        for w in ws:
            O.resize(b.table, b.len, b.ring, b.at, 16, [int(x) for x in w])
        b.same()


@pytest.mark.parametrize("batch,rows", [(500, 300), (900, 9)])
def test_captured_calls_that_move_many_pages(batch, rows):
    """A captured call with a short list over tables that take three launches for it, and one without lists, replayed in turn."""
    width = 160
    b = Both(batch, width, width * batch, 16, seed=4)
    assert resize_launches(batch, width, width * batch, rows) == resize_launches(batch, width, width * batch) == 3
    want, bulk = dev(np.zeros(batch)), dev(np.zeros(batch))
    off, pos, slots = dev(np.zeros(batch + 1)), dev(np.full(rows, -3)), torch.full((rows,), -3, dtype=torch.int64, device="cuda")
    b.resize(np.full(batch, 7), lists="none")
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        P.paged_resize(b.t, want, b.ws, off, pos, slots)
    with torch.cuda.graph(second):
        P.paged_resize(b.t, bulk, b.ws)
    for i in range(4):
        lengths = b.g.integers(0, 16 * width + 1, batch)
        bulk.copy_(dev(lengths))
        second.replay()
        O.resize(b.table, b.len, b.ring, b.at, 16, lengths.tolist())
        b.same()
        lengths = np.where(b.g.random(batch) < 0.7, 0, np.array(b.len) + b.g.integers(0, 3, batch))
        want.copy_(dev(lengths))
        first.replay()
        o, p, s = O.resize(b.table, b.len, b.ring, b.at, 16, lengths.tolist(), rows)
        b.same()
        assert off.tolist() == o and pos[:o[-1]].tolist() == p and slots[:o[-1]].tolist() == s


def test_sums_beyond_32_bits_of_many_sequences():
    """2100 sequences, three groups of 1024 in the sums, that want 2^30 positions each: sums that end at their largest number go on from group to group,
    and so does the place where the first sequence did not fit, which is in the first group or in a later one."""
    batch, page, width = 2100, 65536, 1 << 14
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    ws = torch.empty(P.paged_resize_workspace_bytes(batch), dtype=torch.uint8, device="cuda")

    def call(want, n, rows):
        t = P.PagedTables(table.fill_(-1), dev(np.zeros(batch)), torch.arange(n, dtype=torch.int32, device="cuda"), dev([0, n]), page)
        lists = () if rows is None else (dev(np.full(batch + 1, -3)), dev(np.full(rows, -3)), torch.full((rows,), -3, dtype=torch.int64, device="cuda"))
        P.paged_resize(t, dev(want), ws, *lists)
        return t, lists

    # more pages than are asked for, ten rows: the first sequence stops all, those of the third group that want a single row among them
    want = np.full(batch, 1 << 30)
    want[2048:] = 1
    t, (off, pos, slots) = call(want, 1 << 26, 10)
    assert int(off.abs().max()) == 0 and int(t.seq_len.abs().max()) == 0 and (pos == -3).all() and (slots == -3).all()
    assert t.free_at.tolist() == [0, 1 << 26] and int(table.max()) == -1
    # 1500 single rows fit, the next sequence stops the rest
    want[:1500] = 1
    t, (off, pos, slots) = call(want, 1 << 26, 2000)
    assert off.tolist() == list(range(1501)) + [1500] * 600 and t.seq_len.tolist() == [1] * 1500 + [0] * 600 and t.free_at.tolist() == [1500, (1 << 26) - 1500]
    assert (pos[:1500] == 0).all() and slots[:1500].tolist() == [page * b for b in range(1500)] and (pos[1500:] == -3).all() and (slots[1500:] == -3).all()
    assert table[:1500, 0].tolist() == list(range(1500)) and int(table[:1500, 1:].max()) == int(table[1500:].max()) == -1
    # too few pages, without lists: 1500 of one page, one of 2^14, and no further one
    t, _ = call(want, 1 << 15, None)
    assert t.seq_len.tolist() == [1] * 1500 + [1 << 30] + [0] * 599 and t.free_at.tolist() == [1500 + width, (1 << 15) - 1500 - width]
    assert torch.equal(table[1500], torch.arange(1500, 1500 + width, dtype=torch.int32, device="cuda")) and int(table[1501:].max()) == -1
    # the first two of the first group
    t, _ = call(np.full(batch, 1 << 30), 1 << 15, None)
    assert t.seq_len.tolist() == [1 << 30] * 2 + [0] * (batch - 2) and t.free_at.tolist() == [0, 0]
