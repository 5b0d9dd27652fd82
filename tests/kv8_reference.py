"""Plain forms of the paged 8-bit KV cache in 64 bits, for the tests: one block, one row, one page at a time, on the CPU."""
import math

import torch

MOST = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def block_scale(amax: float, dtype) -> float:
    """Least 2^e, e >= -126, with amax <= most * 2^e; 0 for 0, NaN for what is not finite."""
    if not math.isfinite(amax):
        return math.nan
    if amax == 0:
        return 0.0
    e = max(-126, math.frexp(amax)[1] - 12)
    while amax > MOST[dtype] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def encode(x: torch.Tensor, dtype) -> torch.Tensor:
    """Codes of x (float64, already divided by the scale): nearest, ties to even."""
    if dtype == torch.int8:
        return torch.round(x).to(torch.int8)
    grid = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()       # all finite magnitudes, ascending
    a = x.abs()
    hi = torch.searchsorted(grid, a.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    down, up = a - grid[lo], grid[hi] - a
    take_lo = (down < up) | ((down == up) & (lo % 2 == 0))
    code = torch.where(take_lo, lo, hi).to(torch.uint8)
    code = torch.where(torch.signbit(x), code + 128, code)
    return code.view(torch.float8_e4m3fn)


def values(codes: torch.Tensor) -> torch.Tensor:
    return codes.float().double()


def bounds_of(codes: torch.Tensor) -> torch.Tensor:
    c = values(codes) / (1.0 if codes.dtype == torch.int8 else 4.0)
    return torch.stack([c.amax(0).ceil(), c.amin(0).floor()]).to(torch.int8)


def append(pool, table, tokens, K, V, starts=None):
    """pool: dict of CPU tensors k, v, k_scale, v_scale, k_bounds (or None), changed in place."""
    pages, heads, T, d = pool["k"].shape
    for b in range(table.shape[0]):
        r0, r1 = (b, b + 1) if starts is None else (int(starts[b]), int(starts[b + 1]))
        t = int(tokens[b])
        for lp in range(t // T, (t + r1 - r0 + T - 1) // T if r1 > r0 else 0):
            p0, p1 = max(0, t - lp * T), min(T, t + (r1 - r0) - lp * T)
            page = int(table[b, lp]) if lp < table.shape[1] else -1
            if not 0 <= page < pages:
                continue
            rows = slice(r0 + lp * T + p0 - t, r0 + lp * T + p1 - t)
            for h in range(heads):
                for x, codes, scales, bounds in ((K, pool["k"], pool["k_scale"], pool["k_bounds"]), (V, pool["v"], pool["v_scale"], None)):
                    block, new = codes[page, h], x[rows, h].double()
                    dt = codes.dtype
                    old = float(scales[page, h]) if p0 > 0 else 0.0
                    need = block_scale(float(new.abs().max()) if bool(torch.isfinite(new).all()) else math.inf, dt)
                    now = math.nan if math.isnan(old) or math.isnan(need) else max(old, need)
                    if math.isnan(now):
                        kept, fresh = block[:p0], torch.zeros_like(new)
                    else:
                        kept = encode(values(block[:p0]) * (old / now if now else 0.0), dt) if now != old else block[:p0]
                        fresh = new / now if now else torch.zeros_like(new) * new
                    after = torch.cat([kept.view(torch.int8), encode(fresh, dt).view(torch.int8)])
                    block.view(torch.int8)[:p1] = after
                    scales[page, h] = now
                    if bounds is not None:
                        bounds[page, h] = bounds_of(after.view(dt))


def visible_rows(tokens, starts, nseq, n):
    """(row, sequence, tokens that it sees) of every row that belongs to a sequence."""
    out = []
    for b in range(nseq):
        r0, r1 = (b, b + 1) if starts is None else (int(starts[b]), int(starts[b + 1]))
        out += [(r, b, max(0, int(tokens[b]) - (r1 - 1 - r))) for r in range(r0, min(r1, n))]
    return out


def gather(pool, table, b, h, positions, T):
    """Keys and values in 64 bits at the given positions of sequence b; positions on no page are left out."""
    page = table[b, (positions // T).long()].long()
    ok = (page >= 0) & (page < pool["k"].shape[0])
    page, slot = page[ok], (positions % T).long()[ok]
    k = values(pool["k"].view(torch.int8)[page, h, slot].view(pool["k"].dtype)) * pool["k_scale"][page, h].double()[:, None]
    v = values(pool["v"].view(torch.int8)[page, h, slot].view(pool["v"].dtype)) * pool["v_scale"][page, h].double()[:, None]
    return k, v


def attend(pool, table, tokens, Q, scale, starts=None, lists=None):
    """(out, lse, tolerance of out for bf16 and for fp32, tolerance of lse); rows of no sequence are NaN.

    The tolerances count the roundings that the call documents.  A score is a sum of d products in fp32: off by at most
    (d + 16) 2^-24 of the sum of magnitudes, the 16 for the scaling of q (fp32: two fp16 limbs, 2^-22) and of the score; with it
    2^-22 |logit| for the exponent's argument and exp2.  A weight is then off by that relative amount twice (its own and the
    sum's), and by its rounding to fp16 (2^-11) or to two limbs (2^-21); small weights are held to 2^-25 of 2^3 (bf16) or 2^6 each, with a value scale up
    to 2^4 below the largest one.  Sums of n weights: n 2^-24.  The output's own rounding: 2^-8 (bf16) or 2^-23."""
    n, hq, d = Q.shape
    T, heads = pool["k"].shape[2], pool["k"].shape[1]
    g = hq // heads
    out = torch.full((n, hq, d), math.nan, dtype=torch.float64)
    lse = torch.full((n, hq), math.nan, dtype=torch.float64)
    tol16, tol32, tol_l = torch.zeros_like(out), torch.zeros_like(out), torch.zeros_like(lse)
    for r, b, seen in visible_rows(tokens, starts, table.shape[0], n):
        seen = min(seen, table.shape[1] * T)
        for h in range(heads):
            pos = torch.arange(seen)
            if lists is not None:
                pages = [int(j) for j in lists[r, h] if 0 <= int(j) < table.shape[1]]
                pos = torch.cat([torch.arange(j * T, (j + 1) * T) for j in pages] + [torch.zeros(0, dtype=torch.long)])
                pos = pos[pos < seen].long()
            k, v = gather(pool, table, b, h, pos, T)
            for j in range(h * g, (h + 1) * g):
                q = Q[r, j].double()
                if k.shape[0] == 0:
                    out[r, j], lse[r, j] = 0.0, -math.inf
                    continue
                logit = scale * (k @ q)
                lse[r, j] = torch.logsumexp(logit, 0)
                w = torch.exp(logit - lse[r, j])
                out[r, j] = w @ v
                mag, top = w @ v.abs(), v.abs().max()
                delta = ((d + 16) * 2.0 ** -24 * abs(scale) * (k.abs() @ q.abs()) + 2.0 ** -22 * logit.abs()).max()
                tiny = k.shape[0] * 2.0 ** -31 * 16 * top
                common = (2 * delta + k.shape[0] * 2.0 ** -24) * mag + 1e-37
                tol16[r, j] = 2.0 ** -8 * out[r, j].abs() + 2.0 ** -11 * mag + 8 * tiny + common
                tol32[r, j] = 2.0 ** -23 * out[r, j].abs() + 2.0 ** -21 * mag + tiny * 2.0 ** -11 + common
                tol_l[r, j] = delta + k.shape[0] * 2.0 ** -24 + 2.0 ** -22 * (lse[r, j].abs() + 8)
    return out, lse, tol16, tol32, tol_l


def select(pool, table, tokens, Q, k, first=1, last=1, starts=None):
    """Lists [n, heads, k]; rows of no sequence are -2."""
    n, hq, d = Q.shape
    pages, heads, T, _ = pool["k"].shape
    g = hq // heads
    u = 1.0 if pool["k"].dtype == torch.int8 else 4.0
    lists = torch.full((n, heads, k), -2, dtype=torch.int32)
    for r, b, seen in visible_rows(tokens, starts, table.shape[0], n):
        count = -(-min(seen, table.shape[1] * T) // T)
        for h in range(heads):
            score = []
            for j in range(count):
                page = int(table[b, j])
                if j < first or j >= count - last:
                    score.append((2, 0.0))
                    continue
                if not 0 <= page < pages:
                    score.append((0, 0.0))
                    continue
                best = -math.inf
                for i in range(h * g, (h + 1) * g):
                    q = Q[r, i].double()
                    unit = block_scale(float(q.abs().max()), torch.int8) if bool(torch.isfinite(q).all()) else 0.0
                    qi = torch.round(q / unit) if unit else torch.zeros_like(q)
                    hi, lo = pool["k_bounds"][page, h].double()
                    best = max(best, float((qi.clamp(min=0) * hi + qi.clamp(max=0) * lo).sum()) * unit)
                s = float(pool["k_scale"][page, h])
                score.append((1, math.inf if math.isnan(s) else best * s * u))
            chosen = sorted(sorted(range(count), key=lambda j: (-score[j][0], -score[j][1], j))[:k])
            lists[r, h] = -1
            lists[r, h, :len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
    return lists
