"""A server's step over a paged cache in 4 bits, as its operators are used together: tables follow the lengths, new rows are projected, rotated,
stored and attended to, in two layers whose caches share the tables. Captured once and replayed while sequences grow by different numbers of rows, leave and
come back; every replay is checked against the oracle and against the same calls made eagerly."""
import numpy as np
import pytest
import torch

import paper_2505_15781_amd as P
from oracle import paged as O
from oracle import rotary, tables
from test_gpu_paged import bars, dev, rows
from test_gpu_paged_e2m1 import FourBits

pytestmark = pytest.mark.gpu

BATCH, HEADS, GROUP, DH, PAGE, WIDTH, PAGES, ROWS = 4, 2, 3, 64, 16, 12, 30, 24


class Layer:
    def __init__(self, seed, table, lengths):
        self.c = FourBits([0] * BATCH, PAGE, HEADS, DH, seed=seed)
        new = lambda n: torch.full((PAGES, HEADS, PAGE, n), 0xFF, dtype=torch.uint8, device="cuda")
        self.c.t = P.PagedCache(new(DH // 2).view(torch.float4_e2m1fn_x2), new(DH // 2).view(torch.float4_e2m1fn_x2), table, lengths,
                                new(DH // 32).view(torch.float8_e8m0fnu), new(DH // 32).view(torch.float8_e8m0fnu))
        self.c.o = {"k": np.full((PAGES, HEADS, PAGE, DH), np.nan), "v": np.full((PAGES, HEADS, PAGE, DH), np.nan)}
        g = np.random.default_rng(seed)
        self.w = (rows(g, ((GROUP + 2) * HEADS * DH, 128), "bf16") * 0.1).contiguous()
        self.qkv = torch.zeros((ROWS, (GROUP + 2) * HEADS, DH), dtype=torch.bfloat16, device="cuda")
        self.out = torch.full((ROWS, GROUP * HEADS, DH), 7.0, dtype=torch.bfloat16, device="cuda")


@pytest.mark.parametrize("interleaved,rot_dim", [(False, 64), (True, 32)])
def test_a_server_step(interleaved, rot_dim):
    g = np.random.default_rng(11)
    table, lens, ring, at = [[-1] * WIDTH for _ in range(BATCH)], [0] * BATCH, g.permutation(PAGES).tolist(), [5, PAGES]
    t = P.PagedTables(dev(table), dev(lens), dev(ring), dev(at), PAGE)
    layers = [Layer(s, t.page_table, t.seq_len) for s in (1, 2)]
    rope = P.Rope(DH, rot_dim, 1e4, interleaved, "parts", 4.0, 64)
    off, pos, want = dev(np.zeros(BATCH + 1)), dev(np.zeros(ROWS)), dev(np.zeros(BATCH))
    x = torch.zeros((ROWS, 128), dtype=torch.bfloat16, device="cuda")
    tables_ws = torch.empty(P.paged_resize_workspace_bytes(BATCH), dtype=torch.uint8, device="cuda")
    nq = GROUP * HEADS
    bytes_ = P.paged_attn_workspace_bytes(layers[0].c.t, nq, ROWS, ROWS)
    ws = torch.full((bytes_,), 0xFF, dtype=torch.uint8, device="cuda")

    def step():
        P.paged_resize(t, want, tables_ws, off, pos)
        for l in layers:
            l.qkv.copy_(P.gemm(x, l.w, P.BF16).view(l.qkv.shape))
            q, k, v = l.qkv[:, :nq], l.qkv[:, nq:nq + HEADS], l.qkv[:, nq + HEADS:]
            P.rope(rope, q, k, pos, off)
            P.paged_store(l.c.t, k, v, pos, off)
            P.paged_attn(l.c.t, q, off, l.out, ROWS, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                             # warm-up: nothing grows, no row belongs to a sequence
    torch.cuda.current_stream().wait_stream(side)
    assert all((l.out == 7.0).all() for l in layers) and t.seq_len.tolist() == lens
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    plans = [[5, 9, 1, 3], [17, 9, 4, 3], [0, 12, 20, 5], [6, 12, 21, 17], [-1, 30, 33, 0], [9, 31, 33, 8], [40, 0, 50, 8]]
    for i, lengths in enumerate(plans):
        want.copy_(dev(lengths))
        x.copy_(rows(g, (ROWS, 128), "bf16"))
        for l in layers:
            l.out.fill_(7.0)
        if i % 3 == 2:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        offsets, positions, _ = tables.resize(table, lens, ring, at, PAGE, lengths, ROWS)
        n = offsets[-1]
        assert off.tolist() == offsets and pos[:n].tolist() == positions and t.seq_len.tolist() == lens
        assert t.page_table.tolist() == table and t.free_at.tolist() == at
        for l in layers:
            o = l.c.o
            o["table"], o["lengths"] = np.array(table), np.array(lens)
            before = P.gemm(x, l.w, P.BF16).view(l.qkv.shape).to(torch.bfloat16).double().cpu().numpy()
            got = l.qkv.double().cpu().numpy()
            turned, size = rotary.rotate(before[:n, :nq + HEADS], positions, rope.freq, rope.scale, interleaved)
            assert (np.abs(got[:n, :nq + HEADS] - turned) <= 2.0 ** -8 * np.abs(turned) + 7 * 2.0 ** -24 * size + 1e-37).all()
            assert np.array_equal(got[n:], before[n:]) and np.array_equal(got[:, nq + HEADS:], before[:, nq + HEADS:])
            O.store(o, got[:, nq:nq + HEADS], got[:, nq + HEADS:], np.array(positions + [0] * (ROWS - n)), offsets, "e2m1")
            assert l.c.same()
            ref, spread, most = O.attn(o, got[:, :nq], offsets)
            out = l.out.double().cpu().numpy()
            assert (out[n:] == 7.0).all()
            assert (np.abs(out[:n] - ref[:n]) <= bars(l.qkv, l.c, ref, spread, most)[:n]).all()
            again = torch.full_like(l.out, 7.0)
            P.paged_attn(l.c.t, l.qkv[:, :nq], off, again, ROWS, ws)
            assert torch.equal(again.view(torch.int16), l.out.view(torch.int16))
