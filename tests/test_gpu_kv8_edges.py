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
