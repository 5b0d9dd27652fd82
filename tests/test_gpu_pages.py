"""Bookkeeping of cache pages on the GPU against a plain form: lists of pages and counts, one request after another."""
import pytest
import torch

import paper_2504_19874_b200 as tq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def workspace(pages, requests):
    return torch.full((tq.tq_pages_workspace_bytes(pages, requests),), 0x55, dtype=torch.uint8, device=DEV)


class State:
    def __init__(self, pages, rows, width, heads=2, page=16, d=32, seed=0, dtype=torch.int8, bounds=True):
        self.gen = torch.Generator().manual_seed(seed)
        self.cache = tq.Kv8Cache.empty(pages, heads, page, d, dtype=dtype, bounds=bounds, device=DEV)
        for t in self.arrays():
            t.copy_(torch.randint(-100, 100, t.shape, generator=self.gen).to(t.dtype))
        self.refs, self.table = [0] * pages, [[-1] * width for _ in range(rows)]
        self.tokens, self.page = [0] * rows, page
        self.d_refs, self.d_table, self.d_tokens, self.spare = ints(self.refs), ints(self.table), ints(self.tokens), ints([0])

    def arrays(self):
        c = self.cache
        return [t for t in (c.k.view(torch.int8), c.v.view(torch.int8), c.k_scale, c.v_scale, c.k_bounds) if t is not None]

    def check(self, spare=None):
        assert self.d_refs.tolist() == self.refs
        assert self.d_table.tolist() == self.table
        assert self.d_tokens.tolist() == self.tokens
        if spare is not None:
            assert self.spare.item() == spare

    # ---- plain forms
    def take(self):
        for p, r in enumerate(self.refs):
            if r == 0:
                self.refs[p] = 1
                return p
        return -1

    def extend(self, nxt):
        free, wanted = self.refs.count(0), 0
        for b, x in enumerate(nxt):
            for j in range(-(-self.tokens[b] // self.page), min(-(-x // self.page), len(self.table[b]))):
                self.table[b][j] = self.take()
                wanted += 1
        tq.tq_pages_extend(self.d_refs, self.d_table, self.d_tokens, ints(nxt), self.page, self.spare, workspace(len(self.refs), len(nxt)))
        self.check(free - wanted)
        self.tokens = list(nxt)
        self.d_tokens.copy_(ints(nxt))

    def free(self, seqs):
        for b in seqs:
            if 0 <= b < len(self.table):
                for j, p in enumerate(self.table[b]):
                    if p >= 0:
                        self.refs[p] -= 1
                    self.table[b][j] = -1
                self.tokens[b] = 0
        tq.tq_pages_free(self.d_refs, self.d_table, self.d_tokens, ints(seqs))
        self.check()

    def fork(self, parents, children):
        data = [t.clone() for t in self.arrays()]
        free, wanted, taken = self.refs.count(0), 0, []
        for p, c in zip(parents, children):
            full = self.tokens[p] // self.page
            row = [x if j < full else -1 for j, x in enumerate(self.table[p])]
            if self.tokens[p] % self.page and self.table[p][full] >= 0:
                wanted += 1
                row[full] = self.take()
                if row[full] >= 0:
                    for t in data:
                        t[row[full]] = t[self.table[p][full]]
            taken.append((c, row, self.tokens[p]))
        for c, row, n in taken:
            full = n // self.page
            for x in row[:full]:
                if x >= 0:
                    self.refs[x] += 1
            self.table[c], self.tokens[c] = row, n
        tq.tq_pages_fork(self.cache, self.d_refs, self.d_table, self.d_tokens, ints(parents), ints(children), self.spare,
                         workspace(len(self.refs), len(parents)))
        self.check(free - wanted)
        for got, want in zip(self.arrays(), data):
            assert torch.equal(got, want)

    def compact(self):
        data = [t.clone() for t in self.arrays()]
        live = sum(r > 0 for r in self.refs)
        src = [p for p, r in enumerate(self.refs) if r > 0 and p >= live]
        dst = [p for p, r in enumerate(self.refs) if r == 0 and p < live]
        to = dict(zip(src, dst))
        for s, t in to.items():
            self.refs[t], self.refs[s] = self.refs[s], 0
            for x in data:
                x[t] = x[s]
        self.table = [[to.get(x, x) for x in row] for row in self.table]
        tq.tq_pages_compact(self.cache, self.d_refs, self.d_table, self.spare, workspace(len(self.refs), 0))
        self.check(len(self.refs) - live)
        for got, want in zip(self.arrays(), data):
            assert torch.equal(got, want)


@pytest.mark.parametrize("pages,rows,width,bounds,dtype", [(40, 5, 7, True, torch.int8), (3000, 70, 40, True, torch.float8_e4m3fn),
                                                           (9001, 300, 30, False, torch.int8)])
def test_a_life_of_pages(pages, rows, width, bounds, dtype):
    st = State(pages, rows, width, seed=pages, dtype=dtype, bounds=bounds)
    rnd = lambda lo, hi, n: torch.randint(lo, hi, (n,), generator=st.gen).tolist()
    some = rows // 2
    top = 16 * min(width, max(1, pages // rows))
    st.extend(rnd(0, top + 1, some) + [0] * (rows - some))
    st.fork([0, 1, 0], [some, some + 1, some + 2])
    st.free([0, 0, rows + 5, -1, some + 1])                        # twice the same, and rows that are none
    st.extend([min(t + 17, 16 * width) if t else 0 for t in st.tokens])
    st.compact()
    st.free(list(range(0, rows, 3)))
    st.compact()
    st.compact()                                                   # nothing left to move
    st.extend([min(t + 1, 16 * width) if t else 0 for t in st.tokens])
    st.free(list(range(rows)))
    assert st.refs == [0] * pages
    st.compact()


def test_a_pool_that_is_too_small():
    st = State(6, 4, 5)
    st.extend([16, 33, 0, 0])
    st.fork([1], [2])
    st.extend([16, 33, 33 + 16 * 2, 40])                           # asks for 2 + 3 of one page: the rest is -1, spare -4
    assert st.spare.item() == -4 and st.table[3][:3] == [-1, -1, -1]
    st.fork([1], [0])                                              # no page for the copy
    assert st.table[0][2] == -1 and st.spare.item() == -1


def test_requests_beyond_the_tables_width_and_bad_rows():
    st = State(20, 3, 2)
    st.extend([100, 5, 0])                                         # two entries are all there are
    tq.tq_pages_fork(st.cache, st.d_refs, st.d_table, st.d_tokens, ints([0, 7, 1, -1]), ints([9, 2, 1, 2]), st.spare, workspace(20, 4))
    st.check(17)                                                   # rows outside the table, and a row onto itself: passed over


def test_copy():
    st = State(12, 1, 1, heads=3, page=128, d=96)
    data = [t.clone() for t in st.arrays()]
    src, dst = [3, 3, 7, 0, 99, 5], [1, 2, 11, 4, 6, -1]
    for s, t in zip(src, dst):
        if 0 <= s < 12 and 0 <= t < 12:
            for x in data:
                x[t] = x[s]
    tq.tq_pages_copy(st.cache, ints(src), ints(dst))
    for got, want in zip(st.arrays(), data):
        assert torch.equal(got, want)


def test_a_captured_step_follows_the_state():
    """Extension and release captured once and replayed: every replay sees the counts and lengths of its time."""
    pages, rows, width = 50, 4, 6
    refs, table, tokens, spare = ints([0] * pages), torch.full((rows, width), -1, dtype=torch.int32, device=DEV), ints([0] * rows), ints([0])
    nxt, gone, ws = ints([0] * rows), ints([3]), workspace(pages, rows)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            tq.tq_pages_free(refs, table, tokens, gone)
            tq.tq_pages_extend(refs, table, tokens, nxt, 16, spare, ws)
            tokens.copy_(nxt)
    free = pages
    for step, want in enumerate([[16, 1, 0, 33], [17, 2, 0, 5], [17, 50, 16, 0]]):
        nxt.copy_(ints(want))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        held = sum(-(-w // 16) for w in want)
        assert spare.item() == pages - held and int(refs.sum()) == held
        used = table[table >= 0]
        assert used.numel() == held == used.unique().numel()


@pytest.mark.parametrize("pages", [40, 9001])                          # one launch, and two
def test_extending_a_shortened_sequence_keeps_its_pages(pages):
    st = State(pages, 3, 12)
    st.extend([70, 33, 0])
    held = [list(r) for r in st.table]
    st.tokens = [40, 33, 0]                                            # 30 drafted tokens rejected: pages 3 and 4 of row 0 stay its own
    st.d_tokens.copy_(ints(st.tokens))
    ws = workspace(pages, 3)
    tq.tq_pages_extend(st.d_refs, st.d_table, st.d_tokens, ints([60, 33, 0]), 16, st.spare, ws)
    st.check(pages - 8)
    assert st.table == held
    tq.tq_pages_extend(st.d_refs, st.d_table, st.d_tokens, ints([100, 49, 16]), 16, st.spare, ws)
    st.table[0][5:7], st.table[1][3], st.table[2][0] = [8, 9], 10, 11
    for p in range(8, 12):
        st.refs[p] = 1
    st.check(pages - 12)
    st.tokens = [100, 49, 16]
    st.d_tokens.copy_(ints(st.tokens))
    st.free([0, 1, 2])
    assert st.refs == [0] * pages


def test_a_call_on_a_pool_that_was_too_small_made_again():
    st = State(6, 3, 8)
    st.extend([33, 0, 0])
    ws = workspace(6, 3)
    tq.tq_pages_extend(st.d_refs, st.d_table, st.d_tokens, ints([33, 40, 30]), 16, st.spare, ws)   # three more for row 1, two for row 2: 3 are left
    assert st.spare.item() == -2 and st.d_table[1:, :3].tolist() == [[3, 4, 5], [-1, -1, -1]]
    tq.tq_pages_free(st.d_refs, st.d_table, st.d_tokens, ints([0]))
    tq.tq_pages_extend(st.d_refs, st.d_table, st.d_tokens, ints([0, 40, 30]), 16, st.spare, ws)
    assert st.spare.item() == 1 and st.d_table[1:, :3].tolist() == [[3, 4, 5], [0, 1, -1]] and st.d_refs.tolist() == [1, 1, 0, 1, 1, 1]


def test_entries_of_free_pages_hold_none():
    st = State(30, 2, 4)
    st.d_table.fill_(7)                                                # numbers of a page that nobody has
    tq.tq_pages_extend(st.d_refs, st.d_table, st.d_tokens, ints([40, 20]), 16, st.spare, workspace(30, 2))
    assert st.d_table.tolist() == [[0, 1, 2, 7], [3, 4, 7, 7]] and st.spare.item() == 25
