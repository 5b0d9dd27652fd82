"""Attention over pages of the 8-bit cache that differ widely in magnitude, against a plain form in 64 bits with an error bound of its own."""
import math

import pytest
import torch

from tests import kv8_reference as ref
from tests.test_gpu_kv8 import E4M3, I8, Batch, run_attend

pytestmark = pytest.mark.gpu


def bounded(bt, Q, scale, starts=None, lists=None):
    """(out, lse, bound of out's error, bound of lse's); rows of no sequence are NaN.

    In units of the largest product of a weight and a value scale that the row has, and nothing of the other pages:
    a score is off by (d + 16) 2^-24 of its sum of magnitudes and 2^-22 of itself (as in kv8_reference.attend, here token by token); the
    exponent's argument lies below 16 (half an ulp: 2^-21 ln 2) and exp2 is off by 2^-22, 2^-20 in all; the weight is rounded to fp16 (2^-11, two
    limbs: 2^-21), or where it is subnormal by 2^-25 absolutely, with the largest one at 2^2 at least (bf16, many queries), else 2^5;
    sums: 2^-24 a token, and as much for 64 more of the joined parts; the output's own rounding.  Errors of weights come in twice, with
    the values and with the sum; they are below 0.1, so 1.25 holds the second order."""
    n, hq, d = Q.shape
    T, heads = bt.page, bt.heads
    g, f32 = hq // heads, Q.dtype == torch.float32
    out = torch.full((n, hq, d), math.nan, dtype=torch.float64)
    lse = torch.full((n, hq), math.nan, dtype=torch.float64)
    tol, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    for r, b, seen in ref.visible_rows(bt.tokens, starts, bt.table.shape[0], n):
        for h in range(heads):
            pos = torch.arange(seen)
            if lists is not None:
                pages = [j for j in lists[r, h].tolist() if 0 <= j < bt.table.shape[1]]
                pos = (torch.tensor(pages, dtype=torch.long)[:, None] * T + torch.arange(T)).flatten()
                pos = pos[pos < seen]
            page = bt.table[b, pos // T]
            pos = pos[(page >= 0) & (page < bt.pool["k"].shape[0])]
            if not pos.numel():
                out[r, h * g:(h + 1) * g], lse[r, h * g:(h + 1) * g] = 0.0, -math.inf
                continue
            k, v = ref.gather(bt.pool, bt.table, b, h, pos, T)
            vs = bt.pool["v_scale"][bt.table[b, pos // T].long(), h].double()
            q = Q[r, h * g:(h + 1) * g].double()
            logit = scale * (q @ k.T)                                     # [g, tokens]
            z = torch.logsumexp(logit, 1, keepdim=True)
            w = torch.exp(logit - z)
            delta = (d + 16) * 2.0 ** -24 * abs(scale) * (q.abs() @ k.abs().T) + 2.0 ** -22 * logit.abs() + 2.0 ** -20
            assert float(delta.max()) < 0.1
            o, mag = w @ v, w @ v.abs()
            codes = (v.abs() / torch.where(vs > 0, vs, 1.0)[:, None]).sum(0)
            tiny = 2.0 ** (-30 if f32 else -27) * (w * vs).amax(1, keepdim=True) * codes
            rows = slice(h * g, (h + 1) * g)
            out[r, rows], lse[r, rows] = o, z[:, 0]
            tol[r, rows] = ((2.0 ** -23 if f32 else 2.0 ** -8) * o.abs() + ((2.0 ** -21 if f32 else 2.0 ** -11) + (pos.numel() + 64) * 2.0 ** -24) * mag + tiny
                            + 1.25 * ((w * delta) @ v.abs() + mag * (w * delta).sum(1, keepdim=True)) + 1e-37)
            tol_l[r, rows] = 1.25 * (w * delta).sum(1) + (pos.numel() + 64) * 2.0 ** -24 + 2.0 ** -22 * (z[:, 0].abs() + 8)
    return out, lse, tol, tol_l


def check(bt, Q, scale, starts=None, max_queries=1, lists=None):
    o, z = run_attend(bt, Q, scale, starts, max_queries, lists)
    out, lse, tol, tol_l = bounded(bt, Q, scale, starts, lists)
    o, z = o.cpu().double(), z.cpu().double()
    bad = ~((o - out).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[0].tolist(), float(o[bad][0]), float(out[bad][0]), float(tol[bad][0]))
    fin = torch.isfinite(lse)
    assert bool(((z - lse).abs() <= tol_l)[fin].all()), float(((z - lse).abs() - tol_l)[fin].max())
    assert bool((z[~fin] == lse[~fin]).all())


def scale_pages(bt, name, exponents, repeat=1):
    """Page j of every sequence times 2^exponents[j // repeat % n]: the scales alone change, exactly."""
    for row in bt.table:
        for j, p in enumerate(row.tolist()):
            if p >= 0:
                bt.pool[name][p] *= 2.0 ** exponents[j // repeat % len(exponents)]


def random_exponents(spread, n, seed):
    return torch.randint(-spread, spread + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()


ORDERS = {"down": [0, -25, -50, -75], "up": [-75, -50, -25, 0], "far_down": [-2, -61, -119], "far_up": [-119, -61, -2], "one_large": [60, 0, 3, -1],
          "spread_18": random_exponents(18, 9, 1), "spread_30": random_exponents(30, 9, 2), "spread_50": random_exponents(50, 9, 3),
          "spread_100": random_exponents(100, 9, 4)}


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("order", ORDERS)
def test_values_of_one_token_each(order, dtype, x):
    """More items than shares, so that one warp goes through several pages; and one sequence, whose pages are joined."""
    for lens, heads, page in (([200] * 130, 4, 64), ([600], 1, 16)):
        bt = Batch(lens, heads=heads, d=32, page=page, dtype=dtype, seed=page)
        scale_pages(bt, "v_scale", ORDERS[order], 64 // page)
        check(bt.cuda(), bt.randn(len(lens), heads, x), 0.2)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("large", [60, 90])
@pytest.mark.parametrize("at", [0, 2])
def test_a_large_page_without_weight_leaves_the_others_be(at, large, dtype, x):
    """Values 2^large above the others, with logits 160 below them: their weights are 2^-230."""
    bt = Batch([192] * 130, heads=4, d=32, page=64, dtype=dtype, seed=at)
    for row in bt.table.tolist():
        bt.pool["k"][row[at]] = torch.full((), -64.0).to(dtype)
        bt.pool["k_scale"][row[at]] = 2.0 ** -6
        bt.pool["v_scale"][row[at]] *= 2.0 ** large
    Q = torch.full((130, 8, 32), 5.0).to(x) + 0.25 * bt.randn(130, 8, x)
    check(bt.cuda(), Q.to(x), 1.0)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
def test_the_largest_values(x):
    """Averages of numbers near the largest that the type holds."""
    bt = Batch([100, 2000], heads=1, d=32, page=32, seed=3)
    bt.pool["v_scale"][bt.table[bt.table >= 0].long()] = 2.0 ** 120
    check(bt.cuda(), bt.randn(2, 2, x), 0.2)


# ---------------------------------------------------------------------------------------------------------------- many queries

@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("order", ORDERS)
def test_values_of_prompts(order, dtype, x):
    """Through the kernel of many queries, and through that of few (max_queries only chooses)."""
    starts = torch.tensor([0, 45, 90], dtype=torch.int32)
    for lens, page in (([400, 130], 16), ([700, 45], 128)):
        bt = Batch(lens, heads=1, d=32, page=page, dtype=dtype, seed=page + 1)
        scale_pages(bt, "v_scale", ORDERS[order])
        bt.cuda()
        Q = bt.randn(90, 1, x)
        for most in (45, 1):
            check(bt, Q, 0.2, starts, max_queries=most)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("large", [30, 60, 100])
@pytest.mark.parametrize("d", [32, 96, 128])
def test_rows_before_a_late_large_page_do_not_feel_it(d, large, dtype, x):
    """Finite values 2^large above the others in the last page of a chunk; the rows before it do not see that page."""
    bt = Batch([330], heads=1, d=d, page=32, dtype=dtype, seed=large)
    bt.pool["v_scale"][bt.table[0, 10]] *= 2.0 ** large
    bt.pool["k"][bt.table[0, 10], :, :, :16] = torch.full((), 96.0).to(dtype)       # keys too, in channels that queries leave at 0
    bt.pool["k"][bt.table[0, 10], :, :, 16:] = torch.zeros((), dtype=torch.int8).view(dtype) if dtype == I8 else torch.zeros(()).to(dtype)
    bt.pool["k_scale"][bt.table[0, 10]] *= 2.0 ** large
    Q = bt.randn(120, 2, x)
    Q[..., :16] = 0.0
    check(bt.cuda(), Q, 0.3, torch.tensor([0, 120], dtype=torch.int32), max_queries=120)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("spread", [18, 30, 50])
def test_keys_of_prompts(spread, dtype, x):
    """Keys of many magnitudes: the large ones in channels that queries leave at 0."""
    bt = Batch([500, 90], heads=2, d=64, page=16, dtype=dtype, seed=spread)
    for row in bt.table.tolist():
        for j, p in enumerate(row):
            if p >= 0 and j % 3 == 1:
                bt.pool["k"][p, :, :, 16:] = torch.zeros(()).to(dtype)
                bt.pool["k_scale"][p] *= 2.0 ** spread
            elif p >= 0 and j % 3 == 2:
                bt.pool["k_scale"][p] *= 2.0 ** -spread
    bt.cuda()
    Q = bt.randn(60, 4, x)
    Q[..., :16] = 0.0
    for most in (40, 1):
        check(bt, Q, 0.2, torch.tensor([0, 40, 60], dtype=torch.int32), max_queries=most)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
def test_the_largest_and_no_values_of_prompts(x):
    bt = Batch([100, 300], heads=1, d=32, page=32, seed=3)
    bt.pool["v_scale"][bt.table[bt.table >= 0].long()] = 2.0 ** 120
    bt.pool["v_scale"][bt.table[1, :5].long()] = 0.0                  # blocks of zeros before, and ones of no size behind
    bt.pool["v"][bt.table[1, :5].long()] = 0
    check(bt.cuda(), bt.randn(80, 2, x), 0.2, torch.tensor([0, 40, 80], dtype=torch.int32), max_queries=40)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("order", ["down", "spread_50"])
def test_one_sequence_in_hundreds_of_parts(order, x):
    bt = Batch([40_000], heads=1, d=32, page=128, seed=8)
    scale_pages(bt, "v_scale", ORDERS[order], 7)
    check(bt.cuda(), bt.randn(1, 2, x), 0.2)
    check(bt, bt.randn(20, 2, x), 0.2, torch.tensor([0, 20], dtype=torch.int32), max_queries=20)
    check(bt, bt.randn(3, 2, x), 0.2, torch.tensor([0, 3], dtype=torch.int32), max_queries=3)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("near", [None, 0, 1, 2, 5, 14, 16, 40])
def test_pages_beside_a_large_one_keep_their_bits(near, dtype, x):
    """One tile of 128 keys with a large last page, that early rows do not see, and pages 2^near below it, or of zeros (None), that they do;
    the others are smaller still."""
    bt = Batch([256], heads=1, d=32, page=16, dtype=dtype, seed=7)
    p = bt.table[0].tolist()
    for j in range(16):
        if j < 8 or 11 <= j < 14:
            bt.pool["v_scale"][p[j]] *= 2.0 ** -30
        elif j < 14:
            bt.pool["v_scale"][p[j]] *= 0.0 if near is None else 2.0 ** (30 - near)
        else:
            bt.pool["v_scale"][p[j]] *= 2.0 ** 30
    check(bt.cuda(), bt.randn(140, 2, x), 0.2, torch.tensor([0, 140], dtype=torch.int32), max_queries=140)
