"""Calls of the paged 8-bit KV cache at the edges of what its documentation allows."""
import math

import pytest
import torch

import paper_2504_19874_b200 as tq
from tests import kv8_reference as ref
from tests.test_gpu_kv8 import DEV, E4M3, I8, Batch, check_append, check_attend, run_attend, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("most", [1, 20])                               # either kernel
def test_rows_that_see_nothing_are_zeros_whatever_the_query(most, x):
    bt = Batch([3, 40, 64], d=64, page=16, seed=41).cuda()
    bt.t[2] = -1                                                        # tokens on no page
    starts = torch.tensor([0, 20, 40, 60], dtype=torch.int32)
    Q = bt.randn(60, 4, x)
    Q[0], Q[5, 1, 3], Q[16, 2, 63], Q[45], Q[59, 0, 0] = math.nan, math.inf, -math.inf, math.nan, math.nan
    Q[18], Q[30, 3, 5] = math.nan, math.inf                             # these see tokens
    o, z = run_attend(bt, Q, 0.2, starts, max_queries=most)
    for rows in (slice(0, 17), slice(40, 60)):
        assert bool((o[rows] == 0).all()) and bool((z[rows] == -math.inf).all())
    nan = torch.isnan(o).all(-1).cpu()
    assert torch.equal(nan, torch.isnan(o).any(-1).cpu()) and torch.equal(nan, torch.isnan(z).cpu())
    want = torch.zeros(60, 4, dtype=torch.bool)
    want[18], want[30, 3] = True, True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("most", [1, 5, 30])                            # one warp goes through several tiles, or the other kernel
def test_a_block_of_nan_shows_where_its_weight_is_nothing_too(most, x):
    """The last page, partly filled, holds NaN values 2^-200 in weight."""
    bt = Batch([70] * 130, heads=4, d=32, page=64, seed=6)
    for row in bt.table.tolist():
        bt.pool["k"][row[1]] = -64
        bt.pool["k_scale"][row[1]] = 2.0 ** -6
        bt.pool["v_scale"][row[1], 1] = math.nan
    rows = 30 if most == 30 else 1
    Q = torch.full((130 * rows, 4, 32), 5.0).to(x)
    starts = torch.arange(0, 131, dtype=torch.int32) * rows
    o, _ = run_attend(bt.cuda(), Q, 1.0, starts, max_queries=most)
    nan = torch.isnan(o).view(130, rows, 4, 32).cpu()
    want = torch.zeros_like(nan)
    want[:, -6:, 1] = True                                              # the last six rows see tokens 64 and on
    assert torch.equal(nan, want)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
def test_a_wait_that_runs_out_leaves_no_old_results(x):
    """Several items per CTA, items that CTAs share, and sequences of few rows, which are the other kernel's."""
    lens = [400, 300, 50, 200] * 20
    bt = Batch(lens, heads=2, d=64, page=32, seed=12).cuda()
    rows = [150, 40, 1, 30] * 20
    starts = torch.tensor([0] + rows).cumsum(0).to(torch.int32)
    Q = bt.randn(int(starts[-1]), 4, x)
    want, lse = run_attend(bt, Q, 0.2, starts, max_queries=150)
    try:
        tq.tq_selftest_kv8_timeout(True)
        o, z = run_attend(bt, Q, 0.2, starts, max_queries=150)
    finally:
        tq.tq_selftest_kv8_timeout(False)
    many = torch.tensor(rows).repeat_interleave(torch.tensor(rows)) > 1
    assert bool(torch.isnan(o[many]).all()) and bool(torch.isnan(z[many]).all())
    assert torch.equal(o[~many], want[~many]) and torch.equal(z[~many], lse[~many])
    assert bool(torch.isfinite(want).all())
    o, z = run_attend(bt, Q, 0.2, starts, max_queries=150)
    assert torch.equal(o, want) and torch.equal(z, lse)


@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,d", [(16, 96), (32, 32), (64, 64), (128, 128), (16, 128), (128, 96)])
def test_bounds_forget_tokens_that_were_taken_back(page, d, x, dtype):
    """Drafted tokens, large ones among them, are rejected (the lengths go back) and others appended: bounds are those of the codes that count."""
    lens = [0, 1, 5, page - 7, page // 2, page - 3, 2 * page - 9]
    n = len(lens)
    bt = Batch(lens, heads=3, d=d, page=page, dtype=dtype, seed=page + d, room=2).cuda()
    before = bt.tokens.clone()
    starts = torch.arange(0, n + 1, dtype=torch.int32) * 5
    check_append(bt, before, 1.9 * bt.randn(5 * n, 3, x), bt.randn(5 * n, 3, x), starts)
    check_append(bt, before + 2, bt.randn(n, 3, x), bt.randn(n, 3, x))                                   # one token each
    check_append(bt, before + 1, bt.randn(2 * n, 3, x), bt.randn(2 * n, 3, x), torch.arange(0, n + 1, dtype=torch.int32) * 2)
    check_append(bt, before, 30.0 * bt.randn(n, 3, x), bt.randn(n, 3, x))                                # scales grow
    check_append(bt, before, 0.1 * bt.randn(n, 3, x), bt.randn(n, 3, x))


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("g", [3, 20])
def test_attend_with_a_largest_number_of_rows_of_none(g, x):
    """The figure is wrong: it costs time, not results."""
    bt = Batch([90, 20, 64], d=64, page=32, dtype=E4M3, seed=17).cuda()
    starts = torch.tensor([0, 33, 34, 60], dtype=torch.int32)
    check_attend(bt, bt.randn(60, 2 * g, x), 0.15, starts, max_queries=0)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
def test_a_captured_chunk_follows_lengths_rows_and_pages(x):
    """Append and attention of both kinds captured once; replays see the lengths, the rows of each sequence and the table of their time."""
    bt = Batch([100, 20, 300], heads=2, d=64, page=32, seed=51, room=3).cuda()
    n = 90
    K, V, Q = (torch.zeros((n, h, 64), dtype=x, device=DEV) for h in (2, 2, 8))
    out, lse = torch.zeros_like(Q), torch.zeros((n, 8), device=DEV)
    starts, after = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    ws = workspace(tq.tq_kv8_attend_workspace_bytes(bt.cache, 3, n, 4, n))
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        tq.tq_kv8_append(bt.cache, bt.t, bt.n, K, V, starts=starts)
        tq.tq_kv8_attend(bt.cache, bt.t, after, Q, 0.2, out, ws, lse=lse, starts=starts, max_queries=n)
    for rows in ([60, 1, 20], [0, 30, 1], [1, 1, 1], [0, 0, 88]):
        total = sum(rows)
        s = torch.tensor([0] + rows).cumsum(0).to(torch.int32)
        k, v, q = bt.randn(n, 2, x), bt.randn(n, 2, x), bt.randn(n, 8, x)
        before = bt.tokens.clone()
        for dst, src in ((K, k), (V, v), (Q, q), (starts, s), (after, before + torch.tensor(rows, dtype=torch.int32)), (bt.n, before)):
            dst.copy_(src)
        out.fill_(7.0), lse.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ref.append(bt.pool, bt.table, before, k, v, s)
        bt.tokens = before + torch.tensor(rows, dtype=torch.int32)
        want, wl, t16, t32, tl = ref.attend(bt.pool, bt.table, bt.tokens, q, 0.2, s)
        tol = t16 if x == torch.bfloat16 else t32
        assert bool(((out.cpu().double() - want).abs() <= tol)[:total].all()) and bool(((lse.cpu().double() - wl).abs() <= tl)[:total].all())
        assert bool((out[total:] == 7.0).all()) and bool((lse[total:] == 7.0).all())


def test_calls_on_two_streams_at_once():
    """Each with a workspace of its own; results are those of calls made alone."""
    sets = []
    for seed in range(2):
        bt = Batch([900, 40, 333], heads=2, d=64, page=32, dtype=E4M3 if seed else I8, seed=60 + seed).cuda()
        starts = torch.tensor([0, 300, 301, 380], dtype=torch.int32, device=DEV)
        Q = bt.randn(380, 8, torch.bfloat16).to(DEV)
        ws = workspace(tq.tq_kv8_attend_workspace_bytes(bt.cache, 3, 380, 4, 300))
        want = torch.zeros_like(Q)
        tq.tq_kv8_attend(bt.cache, bt.t, bt.n, Q, 0.2, want, ws, starts=starts, max_queries=300)
        sets.append((bt, starts, Q, ws, want, [torch.zeros_like(Q) for _ in range(8)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(8):
        for bt, starts, Q, ws, _, outs, stream in sets:
            with torch.cuda.stream(stream):
                tq.tq_kv8_attend(bt.cache, bt.t, bt.n, Q, 0.2, outs[i], ws, starts=starts, max_queries=300)
    torch.cuda.synchronize()
    for _, _, _, _, want, outs, _ in sets:
        assert all(torch.equal(o, want) for o in outs)
