"""Paged 8-bit KV cache on the GPU: tq_kv8_append, tq_kv8_attend and tq_kv8_select against their plain forms in 64 bits."""
import math

import pytest
import torch

import paper_2504_19874_b200 as tq
from tests import kv8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I8, E4M3 = torch.int8, torch.float8_e4m3fn


class Batch:
    """A cache and a page table over shuffled pages; lengths are tokens cached.  Slots behind the last token, and free pages, hold
    codes of any value (NaN among them) and scales of NaN."""

    def __init__(self, lens, heads=2, d=64, page=16, dtype=I8, seed=0, extra=3, room=0, spread=0.0):
        g = torch.Generator().manual_seed(seed)
        have = [-(-x // page) for x in lens]
        width = max(have + [1]) + room
        pages = sum(have) + len(lens) * room + extra
        order = torch.randperm(pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32)
        at = 0
        for b, x in enumerate(have):
            self.table[b, :x + room] = order[at:at + x + room]
            at += x + room
        raw = lambda: torch.randint(-128, 128, (pages, heads, page, d), generator=g, dtype=torch.int16).to(torch.int8)
        self.pool = {"k": raw().view(dtype), "v": raw().view(dtype), "k_scale": torch.full((pages, heads), math.nan),
                     "v_scale": torch.full((pages, heads), math.nan), "k_bounds": torch.zeros((pages, heads, 2, d), dtype=torch.int8)}
        self.tokens = torch.tensor(lens, dtype=torch.int32)
        n = sum(lens)
        x = [torch.randn((n, heads, d), generator=g) for _ in range(2)]
        if spread:                                             # blocks of very different magnitudes
            for y in x:
                y *= 2.0 ** torch.randint(-int(spread), int(spread) + 1, (n, heads, 1), generator=g)
        starts = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
        ref.append(self.pool, self.table, torch.zeros(len(lens), dtype=torch.int32), x[0], x[1], starts)
        self.heads, self.d, self.page, self.dtype, self.gen = heads, d, page, dtype, g

    def cuda(self):
        self.dev = {k: v.to(DEV) for k, v in self.pool.items()}
        self.cache = tq.Kv8Cache(self.dev["k"], self.dev["v"], self.dev["k_scale"], self.dev["v_scale"], self.dev["k_bounds"])
        self.t, self.n = self.table.to(DEV), self.tokens.to(DEV)
        return self

    def randn(self, rows, heads, dtype=torch.float32):
        return torch.randn((rows, heads, self.d), generator=self.gen).to(dtype)


def workspace(nbytes):
    return torch.full((max(256, nbytes),), 0x7F, dtype=torch.uint8, device=DEV)


def run_attend(bt, Q, scale, starts=None, max_queries=1, lists=None, out=None, lse=True):
    q = Q.to(DEV)
    o = torch.full_like(q, 7.0) if out is None else out
    z = torch.full(q.shape[:2], 7.0, device=DEV) if lse else None
    ws = workspace(tq.tq_kv8_attend_workspace_bytes(bt.cache, bt.table.shape[0], q.shape[0], q.shape[1] // bt.heads, max_queries,
                                                    0 if lists is None else lists.shape[2]))
    tq.tq_kv8_attend(bt.cache, bt.t, bt.n, q, scale, o, ws, lse=z, starts=None if starts is None else starts.to(DEV), max_queries=max_queries,
                     lists=None if lists is None else lists.to(DEV))
    return o, z


def check_attend(bt, Q, scale, starts=None, max_queries=1, lists=None):
    o, z = run_attend(bt, Q, scale, starts, max_queries, lists)
    out, lse, tol16, tol32, tol_l = ref.attend(bt.pool, bt.table, bt.tokens, Q, scale, starts, lists)
    rows = ~torch.isnan(lse)
    tol = tol16 if Q.dtype == torch.bfloat16 else tol32
    o, z = o.cpu().double(), z.cpu().double()
    assert bool(((o - out).abs() <= tol)[rows].all()), float(((o - out).abs() - tol)[rows].max())
    fin = torch.isfinite(lse)
    assert bool(((z - lse).abs() <= tol_l)[fin].all()), float(((z - lse).abs() - tol_l)[fin].max())
    assert bool((z[rows & ~fin] == lse[rows & ~fin]).all())
    assert bool((o[~rows] == 7.0).all()) and bool((z[~rows] == 7.0).all())
    return o, z


# ---------------------------------------------------------------------------------------------------------------- append

def check_append(bt, before, K, V, starts=None):
    tq.tq_kv8_append(bt.cache, bt.t, before.to(DEV), K.to(DEV), V.to(DEV), starts=None if starts is None else starts.to(DEV))
    ref.append(bt.pool, bt.table, before, K, V, starts)
    for name, want in bt.pool.items():
        got = bt.dev[name].cpu()
        if name in ("k", "v"):
            assert torch.equal(got.view(torch.int8), want.view(torch.int8)), name
        else:
            assert torch.equal(torch.nan_to_num(got.float(), nan=-3.0), torch.nan_to_num(want.float(), nan=-3.0)), name


@pytest.mark.parametrize("dtype", [I8, E4M3])
@pytest.mark.parametrize("page,d,x", [(16, 32, torch.float32), (32, 64, torch.bfloat16), (64, 96, torch.float32), (128, 128, torch.bfloat16),
                                      (16, 128, torch.bfloat16), (128, 32, torch.float32)])
def test_append_of_ragged_prompts_and_steps(dtype, page, d, x):
    lens = [0, 5, page, 2 * page - 1]
    bt = Batch(lens, heads=3, d=d, page=page, dtype=dtype, seed=page + d, room=4).cuda()
    new = [page + 3, 0, 1, 2 * page + 2]
    starts = torch.tensor([0] + new).cumsum(0).to(torch.int32)
    rows = int(starts[-1]) + 2                                       # two rows behind the last sequence
    before = bt.tokens.clone()
    check_append(bt, before, bt.randn(rows, 3, x), bt.randn(rows, 3, x), starts)
    before = before + torch.tensor(new, dtype=torch.int32)
    for step in range(3):                                            # one token each, the later ones larger: scales grow
        check_append(bt, before, bt.randn(4, 3, x) * 5.0 ** step, bt.randn(4, 3, x) * 3.0 ** step)
        before = before + 1


@pytest.mark.parametrize("dtype", [I8, E4M3])
def test_append_of_extreme_magnitudes(dtype):
    bt = Batch([3, 20, 0, 7, 16], heads=1, d=32, page=16, dtype=dtype, seed=5, room=2).cuda()
    K, V = bt.randn(5, 1), bt.randn(5, 1)
    K[0] *= 1e36
    K[1] *= 1e-42                                                    # subnormal inputs
    K[2], V[2] = 0.0, 0.0                                            # a block of zeros
    K[3, 0, 5], V[3, 0, 9] = math.inf, math.nan
    K[4] = torch.tensor([127.0, -127.0, 448.0, 0.5, 1.5, 2.5, -0.5, -0.0] * 4)
    V[4] = torch.finfo(torch.float32).max
    before = bt.tokens.clone()
    check_append(bt, before, K, V)
    check_append(bt, before + 1, bt.randn(5, 1), bt.randn(5, 1))     # behind zeros, behind NaN, behind the largest number
    check_append(bt, torch.tensor([16, 16, 16, 16, 32], dtype=torch.int32), bt.randn(5, 1), bt.randn(5, 1))   # a fresh page each


def test_append_drops_what_has_no_page_and_reads_any_strides():
    bt = Batch([4, 30, 9], heads=2, d=64, page=16, seed=3).cuda()
    bt.table[0, 0], bt.table[2, 0] = -1, 1 << 30
    bt.t.copy_(bt.table)
    starts = torch.tensor([0, 1, 8, 9], dtype=torch.int32)
    wide = torch.randn((9, 65, 5), generator=bt.gen)                 # channels are not contiguous: refused
    with pytest.raises(ValueError):
        tq.tq_kv8_append(bt.cache, bt.t, bt.n, wide.to(DEV)[:, :64].transpose(1, 2), wide.to(DEV)[:, :64].transpose(1, 2), starts=starts.to(DEV))
    K, V = torch.randn((9, 3, 65), generator=bt.gen), torch.randn((2, 9, 67), generator=bt.gen)
    k, v = K.to(DEV)[:, 1:, 1:], V.to(DEV).transpose(0, 1)[..., 2:66]    # rows off the 16-byte grid, heads outside
    tq.tq_kv8_append(bt.cache, bt.t, bt.n, k, v, starts=starts.to(DEV))
    ref.append(bt.pool, bt.table, bt.tokens, K[:, 1:, 1:], V.transpose(0, 1)[..., 2:66], starts)
    for name, want in bt.pool.items():
        assert torch.equal(torch.nan_to_num(bt.dev[name].cpu().float(), nan=-3.0), torch.nan_to_num(want.float(), nan=-3.0)), name


# ---------------------------------------------------------------------------------------------------------------- attend

@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype,page,d,g", [(I8, 16, 32, 1), (I8, 64, 128, 4), (E4M3, 32, 64, 8), (E4M3, 128, 96, 3), (I8, 32, 96, 7),
                                            (E4M3, 16, 128, 12), (I8, 128, 64, 16), (E4M3, 64, 32, 20)])
def test_attend_one_token_each(x, dtype, page, d, g):
    bt = Batch([1, 0, 15, 16, 17, 200, 64, 333], d=d, page=page, dtype=dtype, seed=page + d + g).cuda()
    check_attend(bt, bt.randn(8, 2 * g, x), 1.0 / math.sqrt(d))


@pytest.mark.parametrize("x,dtype", [(torch.bfloat16, E4M3), (torch.float32, I8)])
@pytest.mark.parametrize("g", [1, 3, 8])
def test_attend_several_tokens_each(x, dtype, g):
    bt = Batch([40, 3, 0, 129, 65, 1], d=64, page=32, dtype=dtype, seed=g).cuda()
    starts = torch.tensor([0, 4, 9, 11, 11, 14, 15], dtype=torch.int32)   # more rows than tokens, rows without tokens, no rows
    check_attend(bt, bt.randn(18, 2 * g, x), 0.2, starts, max_queries=5)


@pytest.mark.parametrize("x,dtype", [(torch.bfloat16, I8), (torch.bfloat16, E4M3), (torch.float32, I8), (torch.float32, E4M3)])
@pytest.mark.parametrize("d,g,page", [(128, 4, 64), (64, 1, 16), (96, 5, 32), (32, 16, 128)])
def test_attend_prompts(x, dtype, d, g, page):
    bt = Batch([300, 70, 1, 0, 257], heads=2, d=d, page=page, dtype=dtype, seed=d + g).cuda()
    starts = torch.tensor([0, 75, 145, 146, 148, 214], dtype=torch.int32)
    check_attend(bt, bt.randn(216, 2 * g, x), 1.0 / math.sqrt(d), starts, max_queries=75)


@pytest.mark.parametrize("most", [1, 5, 33, 1000, None])
def test_attend_with_a_wrong_largest_number_of_rows(most):
    """It chooses kernels; the results are the same to within their tolerances."""
    bt = Batch([90, 20, 64], d=64, page=32, dtype=E4M3, seed=17).cuda()
    starts = torch.tensor([0, 33, 34, 60], dtype=torch.int32)
    Q = bt.randn(60, 6, torch.bfloat16)
    if most is not None:
        check_attend(bt, Q, 0.15, starts, max_queries=most)
        return
    q, out = Q.to(DEV), torch.zeros((60, 6, 64), dtype=torch.bfloat16, device=DEV)
    tq.tq_kv8_attend(bt.cache, bt.t, bt.n, q, 0.15, out, workspace(tq.tq_kv8_attend_workspace_bytes(bt.cache, 3, 60, 3, 60)), starts=starts.to(DEV))
    assert torch.equal(out, run_attend(bt, Q, 0.15, starts, max_queries=60)[0])


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
def test_attend_blocks_of_very_different_magnitudes(x):
    bt = Batch([500, 90], d=64, page=16, dtype=I8, seed=4, spread=18).cuda()
    check_attend(bt, bt.randn(2, 4, x) * 2.0 ** -12, 1.0)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [-0.2, 0.0])
def test_attend_with_a_negative_scale_and_without_one(scale, x):
    bt = Batch([150, 40], d=64, page=32, dtype=I8, seed=23).cuda()
    check_attend(bt, bt.randn(2, 4, x), scale)
    check_attend(bt, bt.randn(45, 4, x), scale, torch.tensor([0, 40, 45], dtype=torch.int32), max_queries=40)


def test_attend_passes_over_pages_that_are_none():
    bt = Batch([100, 50], d=64, page=16, dtype=E4M3, seed=9).cuda()
    bt.table[0, 2], bt.table[0, 6], bt.table[1, :] = -1, 1 << 30, -5
    bt.t.copy_(bt.table)
    check_attend(bt, bt.randn(2, 4), 0.3)


@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
def test_attend_shows_nan_only_where_it_is_seen(x):
    bt = Batch([64, 64, 64], d=32, page=16, dtype=I8, seed=2).cuda()
    bt.dev["v_scale"][bt.table[0, 3].item(), 0] = math.nan              # seen by the last rows of sequence 0 only
    bt.dev["k_scale"][bt.table[1, 3].item(), 1] = math.nan
    starts = torch.tensor([0, 20, 40, 41], dtype=torch.int32)
    Q = bt.randn(41, 2, x)
    Q[40, 1, 3] = math.inf
    o, z = run_attend(bt, Q, 0.2, starts, max_queries=20)
    nan = torch.isnan(o).any(-1).cpu()
    want = torch.zeros(41, 2, dtype=torch.bool)
    want[4:20, 0], want[24:40, 1], want[40, 1] = True, True, True        # 64 - 19 + i tokens: beyond 48 from row 4 on
    assert torch.equal(nan, want)


def test_attend_strides_streams_and_captured_graphs():
    bt = Batch([77, 130], d=64, page=32, seed=6).cuda()
    Q = bt.randn(2, 4, torch.bfloat16)
    want, lse = run_attend(bt, Q, 0.25)
    big_q = torch.zeros((4, 9, 70), dtype=torch.bfloat16, device=DEV)
    q = big_q[::2, 1::2, 3:67]
    q.copy_(Q)
    big_o = torch.full((3, 5, 67), 3.0, dtype=torch.bfloat16, device=DEV)
    got, _ = run_attend(bt, q, 0.25, out=big_o[:2, :4, 1:65])
    assert torch.equal(got, want) and bool((big_o[2] == 3.0).all()) and bool((big_o[:, :, 0] == 3.0).all()) and bool((big_o[:, 4] == 3.0).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = run_attend(bt, Q, 0.25)
    side.synchronize()
    assert torch.equal(got, want)
    q, o = Q.to(DEV), torch.zeros_like(want)
    ws = workspace(tq.tq_kv8_attend_workspace_bytes(bt.cache, 2, 2, 2))
    graphs = []
    for _ in range(2):                                                  # two graphs that share the workspace, replayed in turn
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            tq.tq_kv8_attend(bt.cache, bt.t, bt.n, q, 0.25, o, ws)
        graphs.append(gr)
    for gr in graphs + graphs:
        o.zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
    bt.n[1] = 31                                                        # a captured call follows the lengths
    bt.tokens[1] = 31
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(o, run_attend(bt, Q, 0.25)[0]) and not torch.equal(o, want)


def test_attend_many_sequences_and_long_ones():
    lens = [(i * 37) % 150 for i in range(300)]
    lens[7], lens[250] = 9000, 5000
    bt = Batch(lens, heads=1, d=32, page=64, seed=8).cuda()
    Q = bt.randn(300, 2, torch.float32)
    check_attend(bt, Q, 0.3)


@pytest.mark.parametrize("lens,heads", [([20000, 9001, 5, 0, 3000], 2),              # few items, several units each: shares end with items
                                        ([(i * 61) % 90 + 180 for i in range(100)], 4)])   # as many items as CTAs: shares cross them
@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
def test_attend_work_laid_out_both_ways(lens, heads, x):
    bt = Batch(lens, heads=heads, d=32, page=128, seed=len(lens)).cuda()
    check_attend(bt, bt.randn(len(lens), 2 * heads, x), 0.2)


def test_attend_of_steps_and_prompts_in_one_batch_of_many():
    """600 sequences, most of them with one row: those go to one kernel, the few with 21 to the other."""
    lens = [(i * 13) % 60 + 30 for i in range(600)]
    bt = Batch(lens, heads=1, d=32, page=16, dtype=E4M3, seed=31).cuda()
    rows = [21 if i % 50 == 7 else (0 if i % 90 == 5 else 1) for i in range(600)]
    starts = torch.tensor([0] + rows).cumsum(0).to(torch.int32)
    check_attend(bt, bt.randn(int(starts[-1]) + 1, 1, torch.bfloat16), 0.2, starts, max_queries=21)


def test_attend_long_lists():
    bt = Batch([30000, 17000, 100], heads=2, d=32, page=128, seed=5).cuda()
    starts = torch.tensor([0, 3, 5, 6], dtype=torch.int32)
    Q = bt.randn(6, 4, torch.bfloat16)
    lists = ref.select(bt.pool, bt.table, bt.tokens, Q, 70, starts=starts)
    check_attend(bt, Q, 0.2, starts, max_queries=3, lists=lists)


# ---------------------------------------------------------------------------------------------------------------- select and lists

@pytest.mark.parametrize("x", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype,page,d,g,k", [(I8, 16, 32, 1, 3), (E4M3, 16, 64, 4, 8), (I8, 32, 96, 3, 2), (E4M3, 16, 128, 9, 12), (I8, 16, 128, 20, 5)])
def test_select_then_attend(x, dtype, page, d, g, k):
    bt = Batch([page * 21 + 3, 0, 5, page * 12, page * 40, page * k], d=d, page=page, dtype=dtype, seed=g + k).cuda()
    Q = bt.randn(6, 2 * g, x)
    Q[4, 0] = 0.0
    lists = torch.full((6, 2, k), -9, dtype=torch.int32, device=DEV)
    tq.tq_kv8_select(bt.cache, bt.t, bt.n, Q.to(DEV), lists, workspace(tq.tq_kv8_select_workspace_bytes(bt.cache, 6, bt.table.shape[1])))
    want = ref.select(bt.pool, bt.table, bt.tokens, Q, k)
    assert torch.equal(lists.cpu(), want)
    check_attend(bt, Q, 1.0 / math.sqrt(d), lists=want)


@pytest.mark.parametrize("first,last", [(0, 0), (2, 1), (0, 3)])
def test_select_of_equal_scores_takes_the_lowest_pages(first, last):
    bt = Batch([16 * 30, 16 * 700], d=32, page=16, seed=1, heads=1).cuda()
    bt.pool["k_bounds"].fill_(1)
    bt.pool["k_scale"].fill_(1.0)
    nan = bt.table[1, 500].item()
    bt.pool["k_scale"][nan] = math.nan                                  # a block with a NaN is always seen
    for name in ("k_bounds", "k_scale"):
        bt.dev[name].copy_(bt.pool[name])
    bt.table[0, 4] = -1                                                 # no page: the last choice
    bt.t.copy_(bt.table)
    starts = torch.tensor([0, 2, 5], dtype=torch.int32)
    Q = bt.randn(6, 3)
    Q[1], Q[2, 1] = math.nan, math.inf
    for k in (4, 29, 64):
        lists = torch.full((6, 1, k), -2, dtype=torch.int32, device=DEV)
        tq.tq_kv8_select(bt.cache, bt.t, bt.n, Q.to(DEV), lists, workspace(tq.tq_kv8_select_workspace_bytes(bt.cache, 6, bt.table.shape[1])),
                         starts=starts.to(DEV), first=first, last=last)
        assert torch.equal(lists.cpu(), ref.select(bt.pool, bt.table, bt.tokens, Q, k, first, last, starts))


def test_bounds_hold_every_logit():
    for dtype in (I8, E4M3):
        bt = Batch([16 * 9], d=64, page=16, dtype=dtype, seed=12, heads=1)
        hi, lo = bt.pool["k_bounds"][:, 0, 0].double(), bt.pool["k_bounds"][:, 0, 1].double()
        u = 1.0 if dtype == I8 else 4.0
        for j in range(9):
            p = int(bt.table[0, j])
            c = ref.values(bt.pool["k"][p, 0])
            assert bool((c <= u * hi[p]).all()) and bool((c >= u * lo[p]).all())


def test_attend_lists_of_any_kind():
    bt = Batch([100, 33, 0], d=64, page=16, dtype=E4M3, seed=14).cuda()
    starts = torch.tensor([0, 3, 4, 6], dtype=torch.int32)
    lists = torch.tensor([6, 0, -1, 3, 3, 900, -7, 2 ** 31 - 1], dtype=torch.int32).repeat(8, 2, 1)   # 3 counts twice, some are none
    lists[3, :, :] = -1
    check_attend(bt, bt.randn(8, 6, torch.bfloat16), 0.4, starts, max_queries=3, lists=lists)


def test_select_of_many_rows_takes_several_launches():
    """Keys of 64 MB at a time: 300 rows of one head and 65,536 pages are scored in two goes."""
    width, pages = 65536, 40
    g = torch.Generator().manual_seed(3)
    pool = {"k": torch.zeros((pages, 1, 16, 32), dtype=I8), "v": torch.zeros((pages, 1, 16, 32), dtype=I8), "k_scale": torch.ones((pages, 1)),
            "v_scale": torch.ones((pages, 1)), "k_bounds": torch.randint(-100, 100, (pages, 1, 2, 32), generator=g, dtype=torch.int16).to(I8)}
    table = torch.full((2, width), -1, dtype=torch.int32)
    table[:, :pages] = torch.randperm(pages, generator=g).to(torch.int32)
    tokens = torch.tensor([16 * 30, 16 * pages - 3], dtype=torch.int32)
    starts = torch.tensor([0, 140, 300], dtype=torch.int32)
    Q = torch.randn((300, 1, 32), generator=g)
    cache = tq.Kv8Cache(*(pool[x].to(DEV) for x in ("k", "v", "k_scale", "v_scale", "k_bounds")))
    nbytes = tq.tq_kv8_select_workspace_bytes(cache, 300, width)
    assert nbytes < 300 * width * 4
    lists = torch.full((300, 1, 7), -2, dtype=torch.int32, device=DEV)
    tq.tq_kv8_select(cache, table.to(DEV), tokens.to(DEV), Q.to(DEV), lists, workspace(nbytes), starts=starts.to(DEV))
    assert torch.equal(lists.cpu(), ref.select(pool, table[:, :pages], tokens, Q, 7, starts=starts))


def test_offsets_past_32_bits():
    """A pool whose keys alone take 5 GB, with the pages in use at its end."""
    pages, page, d = 310_000, 128, 128
    new = lambda *shape, dtype=I8: torch.empty(shape, dtype=dtype, device=DEV)
    cache = tq.Kv8Cache(new(pages, 1, page, d), new(pages, 1, page, d), new(pages, 1, dtype=torch.float32), new(pages, 1, dtype=torch.float32),
                        new(pages, 1, 2, d))
    bt = Batch([400, 130], heads=1, d=d, page=page, seed=21, extra=0)
    top = pages - 6
    for name in ("k", "v", "k_scale", "v_scale", "k_bounds"):
        getattr(cache, name)[top:].view(torch.uint8).copy_(bt.pool[name].view(torch.uint8).to(DEV))
    bt.cache, bt.t, bt.n = cache, (bt.table + top).masked_fill(bt.table < 0, -1).to(DEV), bt.tokens.to(DEV)
    check_attend(bt, bt.randn(2, 4, torch.bfloat16), 0.1)
    starts = torch.tensor([0, 30, 60], dtype=torch.int32)
    check_attend(bt, bt.randn(60, 4, torch.bfloat16), 0.1, starts, max_queries=30)
    lists = torch.zeros((2, 1, 2), dtype=torch.int32, device=DEV)
    Q = bt.randn(2, 4)
    tq.tq_kv8_select(cache, bt.t, bt.n, Q.to(DEV), lists, workspace(tq.tq_kv8_select_workspace_bytes(cache, 2, bt.table.shape[1])))
    assert torch.equal(lists.cpu(), ref.select(bt.pool, bt.table, bt.tokens, Q, 2))
    K, V = bt.randn(2, 1), bt.randn(2, 1)
    tq.tq_kv8_append(cache, bt.t, bt.n, K.to(DEV), V.to(DEV))
    ref.append(bt.pool, bt.table, bt.tokens, K, V)
    tq.tq_pages_copy(cache, torch.arange(top, pages, dtype=torch.int32, device=DEV), torch.arange(0, 6, dtype=torch.int32, device=DEV))
    for name in ("k", "v", "k_scale", "v_scale", "k_bounds"):
        want = torch.nan_to_num(bt.pool[name].float(), nan=-3.0)
        for got in (getattr(cache, name)[top:], getattr(cache, name)[:6]):
            assert torch.equal(torch.nan_to_num(got.cpu().float(), nan=-3.0), want), name


# ---------------------------------------------------------------------------------------------------------------- used together

@pytest.mark.parametrize("dtype", [I8, E4M3])
def test_a_prompt_and_ten_steps(dtype):
    """A prompt written and attended to, two sequences forked from it, ten tokens appended to each, dense and sparse attention."""
    heads, g, d, page, rows, pages = 2, 4, 64, 16, 4, 40
    gen = torch.Generator().manual_seed(0)
    cache = tq.Kv8Cache.empty(pages, heads, page, d, dtype=dtype, device=DEV)
    refs, table = torch.zeros(pages, dtype=torch.int32, device=DEV), torch.full((rows, 8), -1, dtype=torch.int32, device=DEV)
    tokens, spare = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = workspace(max(tq.tq_pages_workspace_bytes(pages, rows), tq.tq_kv8_attend_workspace_bytes(cache, rows, 64, g, 50),
                       tq.tq_kv8_select_workspace_bytes(cache, 64, 8)))
    K, V = (torch.randn((50, heads, d), generator=gen) for _ in range(2))
    Q = torch.randn((50, heads * g, d), generator=gen)
    nxt = torch.tensor([50, 0, 0, 0], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 50, 50, 50, 50], dtype=torch.int32, device=DEV)
    tq.tq_pages_extend(refs, table, tokens, nxt, page, spare, ws)
    tq.tq_kv8_append(cache, table, tokens, K.to(DEV), V.to(DEV), starts=starts)
    tokens.copy_(nxt)

    def check(Qr, starts, max_queries, lists=None):
        out = torch.zeros_like(Qr, device=DEV)
        lse = torch.zeros(Qr.shape[:2], device=DEV)
        tq.tq_kv8_attend(cache, table, tokens, Qr.to(DEV), 0.125, out, ws, lse=lse, starts=starts, max_queries=max_queries, lists=lists)
        pool = {"k": cache.k.cpu(), "v": cache.v.cpu(), "k_scale": cache.k_scale.cpu(), "v_scale": cache.v_scale.cpu(), "k_bounds": cache.k_bounds.cpu()}
        want, wl, _, tol, tol_l = ref.attend(pool, table.cpu(), tokens.cpu(), Qr, 0.125, None if starts is None else starts.cpu(),
                                             None if lists is None else lists.cpu())
        assert bool(((out.cpu().double() - want).abs() <= tol).all())
        fin = torch.isfinite(wl)
        assert bool(((lse.cpu().double() - wl).abs() <= tol_l)[fin].all())
        return pool

    check(Q, starts, 50)
    tq.tq_pages_fork(cache, refs, table, tokens, torch.tensor([0, 0], dtype=torch.int32, device=DEV), torch.tensor([2, 1], dtype=torch.int32, device=DEV), spare, ws)
    assert tokens.tolist() == [50, 50, 50, 0] and spare.item() == pages - 6
    one = torch.tensor([1, 1, 1, 0], dtype=torch.int32, device=DEV)
    starts = torch.tensor([0, 1, 2, 3, 3], dtype=torch.int32, device=DEV)
    for step in range(10):
        tq.tq_pages_extend(refs, table, tokens, tokens + one, page, spare, ws)
        k, v = torch.randn((3, heads, d), generator=gen), torch.randn((3, heads, d), generator=gen)
        tq.tq_kv8_append(cache, table, tokens, k.to(DEV), v.to(DEV), starts=starts)
        tokens += one
        q = torch.randn((3, heads * g, d), generator=gen)
        check(q, starts, 1)
        lists = torch.zeros((3, heads, 3), dtype=torch.int32, device=DEV)
        tq.tq_kv8_select(cache, table, tokens, q.to(DEV), lists, ws, starts=starts)
        pool = check(q, starts, 1, lists)
        assert torch.equal(lists.cpu(), ref.select(pool, table.cpu(), tokens.cpu(), q, 3, starts=starts.cpu()))
    before = [cache.k[table[b, :4].long()].clone() for b in range(3)]
    tq.tq_pages_free(refs, table, tokens, torch.tensor([0], dtype=torch.int32, device=DEV))
    tq.tq_pages_compact(cache, refs, table, spare, ws)
    assert int(table.max()) + 1 == pages - spare.item() == int((refs > 0).sum())
    for b in (1, 2):
        assert torch.equal(cache.k[table[b, :4].long()].view(torch.int8), before[b].view(torch.int8))
    check(torch.randn((3, heads * g, d), generator=gen), torch.tensor([0, 0, 1, 3, 3], dtype=torch.int32, device=DEV), 2)
