"""Page tables that follow the lengths, without a GPU: the oracle, and what the calls refuse."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import tables as O
from paper_2505_15781_amd import binding as B
from plans import resize_launches


def test_the_oracle_keeps_every_page_in_one_place():
    """Random lengths, many calls: a page is in the ring or in one table, lengths are what was asked for or what was there, and new positions follow
    on the old ones."""
    g = np.random.default_rng(0)
    n, width, S = 40, 9, 16
    table, lengths, ring, at = [[-1] * width for _ in range(6)], [0] * 6, list(g.permutation(n)), [0, n]
    for _ in range(300):
        was, want = list(lengths), [int(x) for x in g.integers(-30, width * S + 10, 6)]
        rows = [None, 100][int(g.integers(2))]
        off, pos, slots = O.resize(table, lengths, ring, at, S, want, rows)
        held = [x for b in range(6) for x in table[b] if x >= 0]
        free = [ring[(at[0] + i) % n] for i in range(at[1])]
        assert sorted(held + free) == list(range(n))
        assert [sum(x >= 0 for x in t) for t in table] == [-(-x // S) for x in lengths]
        assert all(x == w or x == y for x, w, y in zip(lengths, want, was)) and len(pos) == off[-1] <= (rows or 10 ** 9)
        for b in range(6):
            assert pos[off[b]:off[b + 1]] == list(range(was[b], lengths[b]))
            assert slots[off[b]:off[b + 1]] == [table[b][p // S] * S + p % S for p in range(was[b], lengths[b])]
        refused = [b for b in range(6) if was[b] < want[b] <= width * S and lengths[b] == was[b]]
        assert not refused or not any(lengths[b] > was[b] for b in range(refused[0], 6))       # none behind the first that does not fit


def desc(**changes):
    d = B.PagedTablesDesc(16, 16, 16, 16, 3, 20, 5, 16)
    for k, v in changes.items():
        setattr(d, k, v)
    return d


def resize(lengths=16, off=16, pos=16, slots=16, rows=9, ws=16, nbytes=1 << 20, **changes):
    return B.lib.dkv_paged_resize(C.byref(desc(**changes)), lengths, off, pos, slots, rows, ws, nbytes, None)


def test_refused_arguments():
    for name in ("page_table", "seq_len", "free_pages", "free_at"):
        assert resize(**{name: None}) == -1 and B.last_error()
    assert resize(lengths=None) == resize(off=None) == resize(off=None, pos=None) == resize(rows=-1) == -1
    for name in ("batch", "n_pages", "max_pages"):
        assert resize(**{name: 0}) == -1 == resize(**{name: -4})
    for size in (8, 0, 48, 131072, -16):
        assert resize(page_size=size) == -3
    assert resize(max_pages=(1 << 26) + 1) == -3 == resize(n_pages=(1 << 30) + 1) == resize(batch=(1 << 20) + 1) == resize(rows=(1 << 30) + 1)
    assert resize(batch=32, max_pages=1 << 26) == -3 and "2^31" in B.last_error()
    assert resize(ws=None) == -4 == resize(nbytes=16) == resize(nbytes=P.paged_resize_workspace_bytes(3) - 1)
    assert resize(ws=24) == -1
    assert B.lib.dkv_paged_resize(None, 16, 16, 16, 16, 9, 16, 1 << 20, None) == -1
    assert P.paged_resize_workspace_bytes(0) == P.paged_resize_workspace_bytes((1 << 20) + 1) == 0 < P.paged_resize_workspace_bytes(1)
    assert P.paged_resize_workspace_bytes(1 << 20) >= 20 << 20


def tables():
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    return P.PagedTables(i(3, 5), i(3), i(20), i(2), 16)


def test_the_binding_refuses_tensors_that_are_not_what_a_call_reads():
    t, i = tables(), lambda *shape: torch.zeros(shape, dtype=torch.int32)
    ws = torch.zeros(4096, dtype=torch.uint8)

    def refused(text, t=t, lengths=i(3), ws=ws, off=i(4), pos=i(9), slots=torch.zeros(9, dtype=torch.int64)):
        with pytest.raises(ValueError, match=text):
            P.paged_resize(t, lengths, ws, off, pos, slots)

    refused("not on a GPU")
    refused("not on a GPU", slots=None)
    refused("not on a GPU", pos=None)
    refused("not on a GPU", off=None, pos=None, slots=None)
    refused("page_table", t._replace(page_table=i(3, 10)[:, ::2]))
    refused("page_table", t._replace(page_table=i(15)))
    refused("page_table", t._replace(page_table=i(3, 5).long()))
    refused("seq_len", t._replace(seq_len=i(4)))
    refused("free_pages", t._replace(free_pages=i(20).long()))
    refused("free_pages", t._replace(free_pages=i(4, 5)))
    refused("free_at", t._replace(free_at=i(3)))
    refused("lengths", lengths=i(2))
    refused("lengths", lengths=i(3).long())
    refused("row_off", off=i(3))
    refused("row_off", pos=None, slots=None)
    refused("positions", pos=i(9).long())
    refused("slots", slots=i(9))
    refused("slots", slots=torch.zeros(8, dtype=torch.int64))
    refused("workspace", ws=torch.zeros(8192, dtype=torch.uint8)[::2])
    with pytest.raises(TypeError):
        P.paged_resize(tuple(t)[:4], i(3), ws)
    with pytest.raises(TypeError):
        P.paged_resize(t._replace(page_size=None), i(3), ws)


def test_the_launches_go_by_the_pages_that_can_move_too():
    """One workgroup moves 4096 entries at a time: tables and pools of which many entries can move are not left to it."""
    for rows in (0, 8, 8192):                              # a server's step over ordinary tables
        assert resize_launches(64, 257, 8500, rows) == resize_launches(64, 1024, 65536, rows) == resize_launches(1024, 64, 65536, rows) == 1
        assert resize_launches(512, 256, 512 * 256, rows) == resize_launches(1024, 2048, 1 << 21, rows) == resize_launches(64, 4096, 64 * 4096, rows) == 3
    assert resize_launches(64, 100, 6400) == resize_launches(512, 8, 4096) == resize_launches(1, 256, 256) == 1
    assert resize_launches(64, 256, 64 * 256) == resize_launches(512, 256, 512 * 256) == resize_launches(1024, 2048, 1 << 21) == 3
    # wide tables over a small pool, and few sequences whatever they hold
    assert resize_launches(1000, 1 << 14, 1 << 15) == resize_launches(1000, 1 << 14, 1 << 15, 5) == 1
    assert resize_launches(1, 1 << 16, 1 << 16) == resize_launches(6, 1 << 16, 6 << 16) == 1
    # rows of the lists and sequences as before
    assert resize_launches(20, 30, 600, 8193) == resize_launches(1025, 4, 3000, 9) == resize_launches(1025, 4, 3000) == 3


@pytest.mark.parametrize("rows,most", [(None, 6144), (9, 65536)])
def test_the_border_between_the_forms(rows, most):
    for batch in (7, 40, 300, 1024):
        width = most // (batch - 6)
        assert resize_launches(batch, width, batch * width, rows) == 1 and resize_launches(batch, width + 1, batch * (width + 1), rows) == 3
        assert resize_launches(batch, width + 1, most + 6 * (width + 1), rows) == 1       # a smaller pool
