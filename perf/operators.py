"""Cases of the paged 8-bit KV cache, one pass of which is timed.

A case is a dict of plain values; "op" says which of the paths below it takes:
  append    tq_kv8_append: new tokens of a batch of sequences quantised into their pages
  attend    tq_kv8_attend: attention of a batch of sequences over the whole of their caches
  sparse    tq_kv8_select and tq_kv8_attend: the k best pages for each query, and attention over those
  turnover  tq_pages_free of finished sequences and tq_pages_extend for what the others need next
  fork      tq_pages_free of dropped sequences and tq_pages_fork of the kept ones (beams, samples of one prompt)
  compact   tq_pages_compact: live pages of a thinned pool moved to its front

Sizes: "lens" and "news" are the shapes of the batch: cached tokens of each sequence (the new ones included) lie in
[len_lo, len_hi], new tokens in [new_lo, new_hi].  "code" is the cache's element type, "dtype" that of keys, values, queries
and outputs.  A block is one page of one head: it has one scale, the power of two that just holds its largest magnitude.
"""
import math

import torch

own = False

MOST = {"i8": 127.0, "e4m3": 448.0}                     # largest magnitude of a code
CODE = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
HOT = 8                                                 # channels of a head that are ten times the others


def listed():
    kv = {"heads": 8, "g": 4, "d": 128}
    return [
        # One decoding step of a server's batch: a token for each sequence, most of them inside a page.
        {"name": "append_step", "op": "append", **kv, "page": 64, "code": "i8", "dtype": "bf16", "seqs": 128, "len_lo": 1, "len_hi": 8192, "new_lo": 1, "new_hi": 1},
        # Prompts of several users written at once, some of them continued in the middle of a page.
        {"name": "append_prompts", "op": "append", **kv, "page": 32, "code": "e4m3", "dtype": "f32", "seqs": 6, "len_lo": 4096, "len_hi": 8192, "new_lo": 901, "new_hi": 4096},
        # One user's chat that has just begun: launches and host work count.
        {"name": "attend_one", "op": "attend", **kv, "page": 16, "code": "i8", "dtype": "bf16", "seqs": 1, "len_lo": 1000, "len_hi": 1000, "new_lo": 1, "new_hi": 1},
        # The layer of the framework's KV configuration: one sequence of 32,768 tokens.
        {"name": "attend_layer", "op": "attend", **kv, "page": 64, "code": "i8", "dtype": "bf16", "seqs": 1, "len_lo": 32768, "len_hi": 32768, "new_lo": 1, "new_hi": 1},
        # A server's ragged batch.
        {"name": "attend_batch", "op": "attend", **kv, "page": 64, "code": "e4m3", "dtype": "bf16", "seqs": 64, "len_lo": 1, "len_hi": 8192, "new_lo": 1, "new_hi": 1},
        # A few drafted tokens of each sequence checked at once, in 32 bits.
        {"name": "attend_draft", "op": "attend", "heads": 4, "g": 3, "d": 96, "page": 32, "code": "i8", "dtype": "f32", "seqs": 9, "len_lo": 5, "len_hi": 3001, "new_lo": 1, "new_hi": 5},
        # A chunk of a long prompt: its own tokens and those before it.
        {"name": "attend_chunk", "op": "attend", **kv, "page": 64, "code": "i8", "dtype": "bf16", "seqs": 1, "len_lo": 16384, "len_hi": 16384, "new_lo": 2048, "new_hi": 2048},
        # One very long context of which each query reads 64 pages.
        {"name": "sparse_one", "op": "sparse", **kv, "page": 64, "code": "i8", "dtype": "bf16", "seqs": 1, "len_lo": 131072, "len_hi": 131072, "new_lo": 1, "new_hi": 1, "k": 64},
        # A ragged batch, short sequences among them that have fewer pages than are asked for.
        {"name": "sparse_batch", "op": "sparse", **kv, "page": 32, "code": "e4m3", "dtype": "bf16", "seqs": 24, "len_lo": 300, "len_hi": 24000, "new_lo": 1, "new_hi": 1, "k": 48},
        # What a scheduler does between two steps: a few sequences end, the others get the pages that they need.
        {"name": "turnover", "op": "turnover", **kv, "page": 16, "code": "i8", "dtype": "bf16", "seqs": 256, "len_lo": 1, "len_hi": 4096, "new_lo": 1, "new_hi": 1},
        # Beams: each of 16 prompts goes on as four.
        {"name": "fork_beams", "op": "fork", **kv, "page": 64, "code": "i8", "dtype": "bf16", "seqs": 16, "len_lo": 100, "len_hi": 2000, "new_lo": 1, "new_hi": 1, "copies": 4},
        # A pool of which about half the sequences are gone.
        {"name": "compact_pool", "op": "compact", **kv, "page": 64, "code": "i8", "dtype": "bf16", "seqs": 96, "len_lo": 500, "len_hi": 4000, "new_lo": 1, "new_hi": 1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "sparse", "sparse", "sparse", "turnover", "fork", "compact"])
    c = {"op": op, "heads": rng.choice([1, 2, 3, 4, 8]), "g": rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]), "d": rng.choice([32, 64, 96, 128]),
         "page": rng.choice([16, 32, 64, 128]), "code": rng.choice(["i8", "e4m3"]), "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "attend" and rng.random() < 0.4:           # prompts and chunks
        c["seqs"] = rng.randint(1, 4)
        c["new_hi"] = _log(rng, 2, 2048)
        c["new_lo"] = rng.randint(0, c["new_hi"])
        c["len_lo"] = c["new_hi"] + _log(rng, 1, 1000)
        c["len_hi"] = c["len_lo"] + _log(rng, 1, 6000)
        while c["seqs"] * c["heads"] * c["g"] * c["new_hi"] * c["len_hi"] > 32 * 2048 * 12000:
            c["g"] = max(1, c["g"] // 2)
            c["heads"] = max(1, c["heads"] // 2)
            c["seqs"] = max(1, c["seqs"] - 1)
        return c
    c["seqs"] = _log(rng, 1, 128 if op != "turnover" else 256)
    top = _log(rng, 16, max(32, min(32768, 400_000 // c["seqs"])))
    c["len_hi"] = top
    c["len_lo"] = rng.randint(1, top)
    c["new_lo"] = c["new_hi"] = 1
    if op == "append" and rng.random() < 0.6:
        c["new_hi"] = _log(rng, 1, max(1, min(top, 24000 // c["seqs"])))
        c["new_lo"] = rng.randint(0, c["new_hi"])
    if op == "attend" and rng.random() < 0.3:
        c["new_hi"] = rng.randint(1, 6)
        c["new_lo"] = rng.randint(0, 1)
    if op == "sparse":
        c["k"] = rng.choice([2, 5, 8, 16, 33, 64])
        c["seqs"] = min(c["seqs"], 24)
        if rng.random() < 0.25:
            c["new_hi"] = rng.randint(1, 4)
    if op == "fork":
        c["seqs"] = min(c["seqs"], 32)
        c["copies"] = rng.randint(1, 4)
    if op in ("fork", "compact", "turnover"):
        c["len_hi"] = min(c["len_hi"], 3000)
        c["len_lo"] = min(c["len_lo"], c["len_hi"])
        c["seqs"] = min(c["seqs"], max(1, 300_000 // c["len_hi"]))
    return c


# ------------------------------------------------------------------------------------------------ what a program has in hand

def _lengths(case):
    """Cached tokens and new tokens of each sequence, from the case alone: a user's batch has these on the host too."""
    g = torch.Generator().manual_seed(case["len_hi"] * 31 + case["seqs"])
    n = case["seqs"]
    total = torch.randint(case["len_lo"], case["len_hi"] + 1, (n,), generator=g)
    new = torch.randint(case["new_lo"], case["new_hi"] + 1, (n,), generator=g)
    total[0], new[n - 1] = case["len_hi"], case["new_hi"]
    if n > 1 and case["new_hi"] > 1:
        total = torch.maximum(total, new)
    return total, torch.minimum(new, total)


def _values(gen, pages, heads, page, d):
    x = torch.randn((pages, heads, page, d), generator=gen, device="cuda")
    hot = torch.rand((heads, d), generator=gen, device="cuda").argsort(dim=1) < min(HOT, d // 4)
    return x * torch.where(hot, 10.0, 1.0)[None, :, None, :]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 11)
    cpu = torch.Generator().manual_seed(seed * 104729 + 5)
    heads, page, d, code, op = case["heads"], case["page"], case["d"], case["code"], case["op"]
    total, new = _lengths(case)
    n = case["seqs"]
    grow = 2 if op == "turnover" else 1
    rows = n * (1 + case["copies"]) if op == "fork" else n
    width = -(-(case["len_hi"] + grow * page) // page)
    have = -(-total // page)
    spare = n * max(2, case.get("copies", 0)) + 3
    pages = int(have.sum()) + spare
    order = torch.randperm(pages, generator=cpu).to(torch.int32)
    if op == "compact":                                    # the sequences before those that are left came and went
        pages = 2 * int(have.sum()) + spare
        order = torch.randperm(pages, generator=cpu).to(torch.int32)
    table = torch.full((rows, width), -1, dtype=torch.int32)
    at = torch.arange(width)[None, :] < have[:, None]
    table[:n][at] = order[:int(have.sum())]
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[table[table >= 0].long()] = 1
    tokens = torch.zeros(rows, dtype=torch.int32)
    tokens[:n] = total.to(torch.int32)

    s = {"case": dict(case), "table": table.cuda(), "tokens": tokens.cuda(), "refs": refs.cuda(), "longest": case["len_hi"]}
    held = torch.ones((pages, 1, page, 1), device="cuda")
    if op == "append":                                     # slots that the new tokens will take hold nothing yet
        slots = torch.arange(width * page).view(1, width, page) < (total - new)[:, None, None]
        held[table[at].long().cuda(), 0, :, 0] = slots.expand(n, width, page)[at].float().cuda()
    s["k_scale"], s["k"], s["k_bounds"] = _blocks(_values(gen, pages, heads, page, d) * held, code, held > 0)
    s["v_scale"], s["v"], _ = _blocks(_values(gen, pages, heads, page, d) * held, code, held > 0)
    s["scale"] = 1.0 / math.sqrt(d)
    starts = torch.zeros(n + 1, dtype=torch.int32)
    starts[1:] = new.cumsum(0)
    s["rows"] = int(starts[-1])
    s["starts"] = None if case["new_hi"] == 1 and case["new_lo"] == 1 else starts.cuda()
    dt = DTYPE[case["dtype"]]
    if op == "append":
        s["before"] = (total - new).to(torch.int32).cuda()
        s["K"], s["V"] = (_values(gen, s["rows"], heads, 1, d)[:, :, 0].to(dt) for _ in range(2))
    if op in ("attend", "sparse"):
        s["Q"] = torch.randn((s["rows"], heads * case["g"], d), generator=gen, device="cuda").to(dt)
        s["out"] = torch.empty_like(s["Q"])
        s["lse"] = torch.empty((s["rows"], heads * case["g"]), device="cuda")
    if op == "sparse":
        s["lists"] = torch.empty((s["rows"], heads, case["k"]), dtype=torch.int32, device="cuda")
    if op == "turnover":
        s["gone"] = torch.randperm(n, generator=cpu)[:max(1, n // 16)].to(torch.int32).cuda()
        s["next"] = s["tokens"] + torch.randint(0, page + 1, (n,), generator=cpu).to(torch.int32).cuda()
        s["next"][s["gone"].long()] = 0
    if op == "fork":
        s["parents"] = torch.arange(n, dtype=torch.int32).repeat_interleave(case["copies"]).cuda()
        s["children"] = (n + torch.randperm(n * case["copies"], generator=cpu)).to(torch.int32).cuda()
    if op in ("turnover", "fork", "compact"):
        s["spare"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        import paper_2504_19874_b200 as tq
        s["cache"] = tq.Kv8Cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["k_bounds"])
        sizes = {"attend": lambda: tq.tq_kv8_attend_workspace_bytes(s["cache"], n, s["rows"], case["g"], case["new_hi"], 0),
                 "sparse": lambda: max(tq.tq_kv8_attend_workspace_bytes(s["cache"], n, s["rows"], case["g"], case["new_hi"], case["k"]),
                                       tq.tq_kv8_select_workspace_bytes(s["cache"], s["rows"], width)),
                 "turnover": lambda: tq.tq_pages_workspace_bytes(pages, n), "fork": lambda: tq.tq_pages_workspace_bytes(pages, n * case["copies"]),
                 "compact": lambda: tq.tq_pages_workspace_bytes(pages, 0)}
        if op in sizes:
            s["workspace"] = torch.empty(max(256, sizes[op]()), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _exponent(a, most):
    """Least e >= -126 with a <= most * 2^e (a > 0, finite)."""
    m, e = torch.frexp(a)
    mm, me = math.frexp(most)
    return torch.clamp(e - me + (m > mm).to(e.dtype), min=-126)


def _power(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)          # its bits: pow() on a GPU need not be exact


def _round(x, code):
    return torch.round(x).to(torch.int8) if code == "i8" else x.to(torch.float8_e4m3fn)


def _bounds(codes, code, valid):
    """[..., 2, d] int8: upper and lower bound of the codes of each channel over the block's tokens, in steps of 1 (i8) or 4 (e4m3)."""
    c = codes.float()
    if code != "i8":
        c = c / 4
    hi, lo = torch.where(valid, c, -128.0), torch.where(valid, c, 127.0)
    return torch.stack([torch.ceil(hi.amax(-2)), torch.floor(lo.amin(-2))], dim=-2).to(torch.int8)


def _blocks(x, code, held):
    """Scales [...], codes [..., T, d] and bounds [..., 2, d] of blocks x [..., T, d]; slots that hold nothing bound nothing."""
    amax = x.abs().amax((-1, -2))
    scale = torch.where(amax > 0, _power(_exponent(amax, MOST[code])), 0.0)
    codes = _round(x * torch.where(scale > 0, 1.0 / scale, 0.0)[..., None, None], code)
    return scale, codes, _bounds(codes, code, held)


def _row_seq(s):
    """Sequence and place of each row of Q, K or V: [rows], [rows], and rows of each sequence [seqs]."""
    n = s["case"]["seqs"]
    r = torch.arange(s["rows"], device="cuda")
    if s["starts"] is None:
        return r, torch.zeros_like(r), torch.ones(n, dtype=torch.long, device="cuda")
    starts = s["starts"].long()
    seq = torch.searchsorted(starts, r, right=True) - 1
    return seq, r - starts[seq], starts[1:] - starts[:-1]


def _append(s):
    case = s["case"]
    page, code, most = case["page"], case["code"], MOST[case["code"]]
    seq, place, new = _row_seq(s)
    before = s["before"].long()
    # the pages that the new tokens fall on: page j of sequence b, j from before // page on
    span = (case["new_hi"] + page - 1) // page + 1
    logical = before[:, None] // page + torch.arange(span, device="cuda")[None, :]
    first, last = torch.maximum(logical * page, before[:, None]), torch.minimum((logical + 1) * page, (before + new)[:, None])
    touched = first < last                                                           # [seqs, span]
    ids = s["table"].long().gather(1, logical.clamp(max=s["table"].shape[1] - 1))
    slot = torch.arange(page, device="cuda") + logical[..., None] * page             # position of each slot [seqs, span, page]
    is_new = (slot >= first[..., None]) & (slot < last[..., None])
    is_old = slot < first[..., None]
    starts = torch.cumsum(new, 0) - new
    source = (starts[:, None, None] + slot - before[:, None, None]).clamp(0, max(s["rows"] - 1, 0))
    ids, is_new, is_old, source = ids[touched], is_new[touched], is_old[touched], source[touched]
    mask_new, mask_old = is_new[:, None, :, None], is_old[:, None, :, None]
    for x, codes, scales, bounds in ((s["K"], s["k"], s["k_scale"], s["k_bounds"]), (s["V"], s["v"], s["v_scale"], None)):
        fresh = torch.where(mask_new, x[source].float().transpose(1, 2), 0.0)        # [pages, heads, T, d]
        amax = fresh.abs().amax((-1, -2))
        old_scale = torch.where(is_old.any(1)[:, None], scales[ids], 0.0)
        scale = torch.maximum(torch.where(amax > 0, _power(_exponent(amax, most)), 0.0), old_scale)
        inv = torch.where(scale > 0, 1.0 / scale, 0.0)[..., None, None]
        have = codes[ids]
        kept = _round(have.float() * (old_scale[..., None, None] * inv), code)
        after = torch.where(mask_new, _round(fresh * inv, code).float(), torch.where(mask_old, kept.float(), have.float())).to(codes.dtype)
        codes.view(torch.int8)[ids] = after.view(torch.int8)
        scales[ids] = scale
        if bounds is not None:
            bounds[ids] = _bounds(after, code, mask_new | mask_old)
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "k_bounds": s["k_bounds"]}


def _softmax(x, seen):
    """Weights, their sum and the log of the sum of exponentials over the last axis; rows that see nothing have none."""
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    return p, total, (top + torch.log(total))[..., 0]


def _attend(s):
    case = s["case"]
    heads, g, d, page, n, most = case["heads"], case["g"], case["d"], case["page"], case["seqs"], case["new_hi"]
    seq, place, new = _row_seq(s)
    pages = -(-s["longest"] // page)
    ids = s["table"][:n, :pages].long()
    inside = torch.arange(pages * page, device="cuda")[None, :] < s["tokens"][:n, None]               # [seqs, tokens]

    def dense(codes, scales):
        at = ids.clamp(min=0)
        x = codes[at].float() * scales[at][..., None, None]                                           # [seqs, pages, heads, T, d]
        x = x.permute(0, 2, 1, 3, 4).reshape(n, heads, pages * page, d)
        return torch.where(inside[:, None, :, None], x, 0.0)

    q = torch.zeros((n, most, heads * g, d), device="cuda")
    q[seq, place] = s["Q"].float()
    q = q.view(n, most, heads, g, d).permute(0, 2, 1, 3, 4).reshape(n, heads, most * g, d)
    x = torch.matmul(q, dense(s["k"], s["k_scale"]).transpose(2, 3)) * s["scale"]
    visible = s["tokens"][:n, None] - (new[:, None] - 1 - torch.arange(most, device="cuda"))          # [seqs, most]
    seen = torch.arange(pages * page, device="cuda") < visible[..., None]                             # [seqs, most, tokens]
    seen = seen[:, None, :, None, :].expand(n, heads, most, g, pages * page).reshape(n, heads, most * g, pages * page)
    p, total, lse = _softmax(x, seen)
    del x, seen
    out = torch.matmul(p, dense(s["v"], s["v_scale"])) / torch.where(total > 0, total, 1.0)
    out = out.view(n, heads, most, g, d).permute(0, 2, 1, 3, 4).reshape(n, most, heads * g, d)
    lse = lse.view(n, heads, most, g).permute(0, 2, 1, 3).reshape(n, most, heads * g)
    return {"out": out[seq, place].to(s["Q"].dtype), "lse": lse[seq, place]}


def _select(s):
    """[rows, heads, k] page numbers.  Scores are sums of products of 8-bit integers and powers of two: 64 bits hold them exactly."""
    case = s["case"]
    heads, g, d, page, k = case["heads"], case["g"], case["d"], case["page"], case["k"]
    seq, place, new = _row_seq(s)
    visible = s["tokens"][seq] - (new[seq] - 1 - place)
    pages = -(-s["longest"] // page)
    q = s["Q"].double().view(s["rows"], heads, g, d)
    amax = q.abs().amax(-1, keepdim=True)
    qs = torch.where(amax > 0, _power(_exponent(amax.float(), 127.0)), 0.0).double()
    qi = torch.where(qs > 0, torch.round(q / qs), 0.0)
    ids = s["table"][seq, :pages].long().clamp(min=0)                                                 # [rows, pages]
    bounds = s["k_bounds"][ids].double().permute(0, 2, 3, 1, 4)                                       # [rows, heads, 2, pages, d]
    step = s["k_scale"][ids].double().transpose(1, 2) * (1.0 if case["code"] == "i8" else 4.0)        # [rows, heads, pages]
    score = torch.matmul(qi.clamp(min=0), bounds[:, :, 0].transpose(2, 3)) + torch.matmul(qi.clamp(max=0), bounds[:, :, 1].transpose(2, 3))
    score = (score * qs * step[:, :, None]).amax(2)                                                   # [rows, heads, pages]
    j = torch.arange(pages, device="cuda")
    count = -(-visible // page)[:, None, None]
    always = (j == 0) | (j == count - 1)
    score = torch.where(always, math.inf, score)
    score = torch.where(j < count, score, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :k]
    best = torch.where(best < count, best, pages)                                                     # pages behind the last one are none
    best = torch.sort(best, dim=-1)[0]
    best = torch.where(best < pages, best, -1).to(torch.int32)
    if best.shape[-1] < k:
        best = torch.cat([best, torch.full((*best.shape[:2], k - best.shape[-1]), -1, dtype=torch.int32, device="cuda")], dim=-1)
    return best


def _sparse(s):
    case = s["case"]
    heads, g, d, page, k, rows = case["heads"], case["g"], case["d"], case["page"], case["k"], s["rows"]
    lists = _select(s)
    seq, place, new = _row_seq(s)
    visible = s["tokens"][seq] - (new[seq] - 1 - place)
    at = lists.clamp(min=0).long()
    ids = s["table"].long()[seq[:, None, None], at].clamp(min=0)                                      # [rows, heads, k]
    pos = at[..., None] * page + torch.arange(page, device="cuda")
    seen = ((lists >= 0)[..., None] & (pos < visible[:, None, None, None])).reshape(rows, heads, 1, k * page)
    h = torch.arange(heads, device="cuda")[None, :, None]

    def dense(codes, scales):
        x = (codes.view(torch.int8)[ids, h].view(codes.dtype).float() * scales[ids, h][..., None, None]).reshape(rows, heads, k * page, d)
        return torch.where(seen[:, :, 0, :, None], x, 0.0)

    q = s["Q"].float().view(rows, heads, g, d)
    p, total, lse = _softmax(torch.matmul(q, dense(s["k"], s["k_scale"]).transpose(2, 3)) * s["scale"], seen)
    out = torch.matmul(p, dense(s["v"], s["v_scale"])) / torch.where(total > 0, total, 1.0)
    return {"lists": lists, "out": out.reshape(rows, heads * g, d).to(s["Q"].dtype), "lse": lse.reshape(rows, heads * g)}


def _free(refs, table, tokens, seqs):
    held = table[seqs.long()]
    gone = held[held >= 0].long()
    refs -= torch.zeros_like(refs).index_add_(0, gone, torch.ones_like(gone, dtype=torch.int32))
    table[seqs.long()] = -1
    tokens[seqs.long()] = 0


def _turnover(s):
    page = s["case"]["page"]
    refs, table, tokens = s["refs"].clone(), s["table"].clone(), s["tokens"].clone()
    _free(refs, table, tokens, s["gone"])
    have, need = -(-tokens // page), -(-s["next"] // page)
    j = torch.arange(table.shape[1], device="cuda")
    wanted = (j >= have[:, None]) & (j < need[:, None])
    free = torch.nonzero(refs == 0)[:, 0]
    got = free[:int(wanted.sum())]
    table[wanted] = got.to(torch.int32)
    refs[got] = 1
    return {"refs": refs, "table": table, "tokens": tokens, "spare": (free.numel() - wanted.sum()).to(torch.int32).view(1)}


def _pools(s):
    return [s["k"].view(torch.int8), s["v"].view(torch.int8), s["k_scale"], s["v_scale"], s["k_bounds"]]


def _fork(s):
    page = s["case"]["page"]
    refs, table, tokens = s["refs"], s["table"], s["tokens"]
    parents, children = s["parents"].long(), s["children"].long()
    _free(refs, table, tokens, children)
    length = tokens[parents]
    full, part = length // page, length % page > 0
    j = torch.arange(table.shape[1], device="cuda")
    rows = torch.where(j < full[:, None], table[parents], -1)
    shared = rows[rows >= 0].long()
    free = torch.nonzero(refs == 0)[:, 0]
    refs.index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    got = free[:int(part.sum())]
    refs[got] = 1
    source = table[parents[part], full[part].long()].long()
    rows[part.nonzero()[:, 0], full[part].long()] = got.to(torch.int32)
    table[children] = rows
    tokens[children] = length
    for p in _pools(s):
        p[got] = p[source]
    return {"refs": refs, "table": table, "tokens": tokens, "spare": (free.numel() - part.sum()).to(torch.int32).view(1),
            "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "k_bounds": s["k_bounds"]}


def _compact(s):
    refs, table = s["refs"].clone(), s["table"].clone()
    live = refs > 0
    count = live.sum()
    at = torch.arange(refs.numel(), device="cuda")
    source = torch.nonzero(live & (at >= count))[:, 0]          # live pages behind the front
    target = torch.nonzero(~live & (at < count))[:, 0]          # free ones in it, as many
    for p in _pools(s):
        p[target] = p[source]
    to = at.to(torch.int32)
    to[source] = target.to(torch.int32)
    table = torch.where(table >= 0, to[table.clamp(min=0).long()], table)
    refs[target] = refs[source]
    refs[source] = 0
    return {"refs": refs, "table": table, "spare": (refs.numel() - count).to(torch.int32).view(1),
            "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "k_bounds": s["k_bounds"]}


# ------------------------------------------------------------------------------------------------ the framework's calls

def _own(s):
    import paper_2504_19874_b200 as tq
    op = s["case"]["op"]
    cache, pool = s["cache"], {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "k_bounds": s["k_bounds"]}
    if op == "append":
        tq.tq_kv8_append(cache, s["table"], s["before"], s["K"], s["V"], starts=s["starts"])
        return pool
    if op == "attend":
        tq.tq_kv8_attend(cache, s["table"], s["tokens"], s["Q"], s["scale"], s["out"], s["workspace"], lse=s["lse"], starts=s["starts"], max_queries=s["case"]["new_hi"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "sparse":
        tq.tq_kv8_select(cache, s["table"], s["tokens"], s["Q"], s["lists"], s["workspace"], starts=s["starts"])
        tq.tq_kv8_attend(cache, s["table"], s["tokens"], s["Q"], s["scale"], s["out"], s["workspace"], lse=s["lse"], starts=s["starts"],
                         max_queries=s["case"]["new_hi"], lists=s["lists"])
        return {"lists": s["lists"], "out": s["out"], "lse": s["lse"]}
    if op == "turnover":
        refs, table, tokens = s["refs"].clone(), s["table"].clone(), s["tokens"].clone()
        tq.tq_pages_free(refs, table, tokens, s["gone"])
        tq.tq_pages_extend(refs, table, tokens, s["next"], s["case"]["page"], s["spare"], s["workspace"])
        return {"refs": refs, "table": table, "tokens": tokens, "spare": s["spare"]}
    if op == "fork":
        tq.tq_pages_free(s["refs"], s["table"], s["tokens"], s["children"])
        tq.tq_pages_fork(cache, s["refs"], s["table"], s["tokens"], s["parents"], s["children"], s["spare"], s["workspace"])
        return {"refs": s["refs"], "table": s["table"], "tokens": s["tokens"], "spare": s["spare"], **pool}
    refs, table = s["refs"].clone(), s["table"].clone()
    tq.tq_pages_compact(cache, refs, table, s["spare"], s["workspace"])
    return {"refs": refs, "table": table, "spare": s["spare"], **pool}


def run(s):
    if own:
        return _own(s)
    return {"append": _append, "attend": _attend, "sparse": _sparse, "turnover": _turnover, "fork": _fork, "compact": _compact}[s["case"]["op"]](s)


def work(case):
    total, new = _lengths(case)
    heads, g, d, page, n, op = case["heads"], case["g"], case["d"], case["page"], case["seqs"], case["op"]
    size = 4 if case["dtype"] == "f32" else 2
    rows, have = int(new.sum()), int((-(-total // page)).sum())
    block = heads * (2 * page * d + 8 + 2 * d)                    # a page in all arrays of the pool
    width = -(-(case["len_hi"] + (2 if op == "turnover" else 1) * page) // page)
    if op == "append":
        return {"bytes": rows * heads * d * 2 * (size + 1) + 4 * n * 2, "flops": rows * heads * d * 2 * 2}
    if op == "attend":
        seen = int(torch.clamp(new * total - new * (new - 1) // 2, min=0).sum())
        return {"bytes": int(total[new > 0].sum()) * heads * 2 * d + 2 * rows * heads * g * d * size + 4 * have, "flops": 4 * d * heads * g * seen}
    if op == "sparse":
        read = int(torch.minimum(total, torch.full_like(total, case["k"] * page)).sum()) * heads
        return {"bytes": have * heads * (2 * d + 4) + read * 2 * d + 2 * rows * heads * g * d * size + 4 * rows * heads * case["k"],
                "flops": 4 * d * g * read + 4 * d * g * have * heads}
    if op == "turnover":
        return {"bytes": 4 * (have + 3 * n) * 2, "flops": have}
    if op == "fork":
        part = int((total % page > 0).sum()) * case["copies"]
        return {"bytes": 2 * part * block + 4 * n * (1 + case["copies"]) * width, "flops": part}
    pages = 2 * have + n * 2 + 3
    moved = have - have * have // pages                           # live pages behind the front, when they lie anywhere
    return {"bytes": 2 * moved * block + 8 * pages + 8 * n * width, "flops": pages}


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits

def _exact_rows(s, lists=None):
    """out and lse, one sequence, query token and head after another, over the tokens that it sees in the order of the cache."""
    case = s["case"]
    heads, g, d, page = case["heads"], case["g"], case["d"], case["page"]
    _, new = _lengths(case)
    table, tokens = s["table"].cpu(), s["tokens"].cpu().tolist()
    out, lse, row = [], [], 0
    for b, m in enumerate(new.tolist()):
        ids = table[b, :-(-tokens[b] // page)].long().cuda()
        if m == 0 or ids.numel() == 0:
            out += [torch.zeros((m, heads * g, d), dtype=torch.float64, device="cuda")]
            lse += [torch.full((m, heads * g), -math.inf, dtype=torch.float64, device="cuda")]
            row += m
            continue
        o = torch.zeros((m, heads, g, d), dtype=torch.float64, device="cuda")
        z = torch.full((m, heads, g), -math.inf, dtype=torch.float64, device="cuda")
        for h in range(heads):
            k = (s["k"].view(torch.int8)[ids, h].view(s["k"].dtype).double() * s["k_scale"][ids, h].double()[:, None, None]).reshape(-1, d)
            v = (s["v"].view(torch.int8)[ids, h].view(s["v"].dtype).double() * s["v_scale"][ids, h].double()[:, None, None]).reshape(-1, d)
            k, v = k[:tokens[b]], v[:tokens[b]]
            q = s["Q"][row:row + m, h * g:(h + 1) * g].double()
            pos = torch.arange(tokens[b], device="cuda")
            ok = pos[None, :] < tokens[b] - (m - 1 - torch.arange(m, device="cuda"))[:, None]
            if lists is not None:
                listed_pages = lists[row:row + m, h].long()
                ok = ok & ((pos // page)[None, :, None] == listed_pages[:, None, :]).any(-1)
            logit = torch.einsum("mgd,td->mgt", q, k) / math.sqrt(d)
            logit = logit.masked_fill(~ok[:, None, :], -math.inf)
            z[:, h] = torch.logsumexp(logit, -1)
            o[:, h] = torch.einsum("mgt,td->mgd", torch.nan_to_num(torch.exp(logit - z[:, h, :, None])), v)
        out.append(o.reshape(m, heads * g, d))
        lse.append(z.reshape(m, heads * g))
        row += m
    return torch.cat(out), torch.cat(lse)


def _exact_lists(s):
    """Pages ranked by brute force: products of the integers channel by channel, ranks by counting what is better."""
    case = s["case"]
    heads, g, d, page, k = case["heads"], case["g"], case["d"], case["page"], case["k"]
    _, new = _lengths(case)
    tokens, row = s["tokens"].cpu().tolist(), 0
    lists = torch.full((s["rows"], heads, k), -1, dtype=torch.int32)
    for b, m in enumerate(new.tolist()):
        for i in range(m):
            seen = tokens[b] - (m - 1 - i)
            count = -(-seen // page) if seen > 0 else 0
            if count:
                ids = s["table"][b, :count].long()
                q = s["Q"][row].double().view(heads, g, 1, d)
                top = q.abs().amax(-1, keepdim=True)
                up = torch.clamp(torch.ceil(torch.log2(top / 127.0)), min=-126.0)
                unit = torch.where(top > 0, ((up.to(torch.int64) + 1023) << 52).view(torch.float64), 0.0)
                whole = torch.where(unit > 0, torch.round(q / unit), 0.0)
                hi, lo = s["k_bounds"][ids, :, 0].double().transpose(0, 1)[:, None], s["k_bounds"][ids, :, 1].double().transpose(0, 1)[:, None]
                best = torch.maximum(whole * hi, whole * lo).sum(-1)                                   # [heads, g, count]
                best = (best * unit[..., 0] * s["k_scale"][ids].double().t()[:, None]).amax(1).cpu()
                for h in range(heads):
                    ranked = sorted(range(count), key=lambda j: (0 if j in (0, count - 1) else 1, -float(best[h, j]) if j not in (0, count - 1) else 0.0, j))
                    chosen = sorted(ranked[:k])
                    lists[row, h, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
            row += 1
    return lists.cuda()


def exact(case, seed):
    if case["op"] not in ("attend", "sparse"):
        return None                                       # codes, scales and page numbers are exact by definition: nothing is computed further
    s = prepare(case, seed)
    if case["op"] == "attend":
        out, lse = _exact_rows(s)
        return {"out": out, "lse": lse}
    lists = _exact_lists(s)
    out, lse = _exact_rows(s, lists)
    return {"lists": lists, "out": out, "lse": lse}
