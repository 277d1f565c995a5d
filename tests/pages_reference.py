"""Plain 64-bit forms of the operators on ragged batches and 8-bit pages, row by row, for the tests."""
import numpy as np
import torch


def attend_rows(q, k, v, scale, slopes=None, causal=True):
    """q [n, H, d], k, v [m, Hkv, d] in 64 bits; query i sees keys j <= i (causal) or all of them (n = 1).  Returns out, the weighted sum of |v| and the
    largest sum of |q k| times the scale per query: what the error bounds are made of."""
    n, H, d = q.shape
    G = H // k.shape[1]
    k, v = k.repeat_interleave(G, 1).transpose(0, 1), v.repeat_interleave(G, 1).transpose(0, 1)      # [H, m, d]
    q = q.transpose(0, 1)
    x = scale * (q @ k.transpose(1, 2))
    last = torch.arange(n, device=q.device) if causal else torch.full((n,), k.shape[1] - 1, device=q.device)
    j = torch.arange(k.shape[1], device=q.device)
    if slopes is not None:
        x = x - slopes.double()[:, None, None] * (last[:, None] - j)
    x = torch.where(j <= last[:, None], x, -torch.inf)
    p = torch.softmax(x, -1)
    size = (scale * (q.abs() @ k.abs().transpose(1, 2))).amax(-1)                                    # [H, n]
    return (p @ v).transpose(0, 1), (p @ v.abs()).transpose(0, 1), size.transpose(0, 1)


def bound(out, weighted, size, dtype, d, weights_rounded):
    """How far a kernel's output may be off.  Half a step of the output's type for its own rounding, and with `weights_rounded` half a step for that of
    every weight; the logits are sums of d binary32 products, 16 at a time (a step of 2^-23 each, plus four for scale, bias and exponent), and an error of a logit changes every weight
    by as much and their sum once more; the exponential and the rest of the binary32 arithmetic stay below 2^-18.  Binary16 outputs below 2^-14 are multiples of 2^-24."""
    half = torch.finfo(dtype).eps / 2
    logit = (d / 16 + 4) * 2.0 ** -23 * (size + 16)
    return half * out.abs() + (logit[..., None] * 2 + 2.0 ** -18 + (half if weights_rounded else 0)) * weighted + (2.0 ** -25 if dtype == torch.float16 else 0)


def power_of_two(top):
    """The smallest e >= -120 with top <= 127 * 2^e."""
    e = -120
    while top > 127 * 2.0 ** e:
        e += 1
    return e


def weight_floor(q, k, scale, slopes, unit):
    """What kf_pages_attend's weights may lose altogether, per query head of the one query [1, H, d].  A weight times the V scale of its page (`unit` [m, Hkv]) enters as
    two binary16 numbers that are multiples of 2^-24 and stand 2^7 above a reference, which lies at most 2^8 below and never above the largest of these
    products: it is off by at most half a multiple, 2^-32 of the reference, beside its relative error, and multiplies a code of at most 127."""
    n, H, d = q.shape
    G = H // k.shape[1]
    x = scale * (q.transpose(0, 1) @ k.repeat_interleave(G, 1).permute(1, 2, 0))[:, 0]               # [H, m]
    if slopes is not None:
        x = x - slopes.double()[:, None] * torch.arange(k.shape[0] - 1, -1, -1, device=q.device)
    top = (torch.softmax(x, -1) * unit.repeat_interleave(G, 1).T).amax(-1)
    return 2.0 ** -32 * 127 * k.shape[0] * top[None, :, None]


def write(cache, scale, table, length, rows, begin):
    """In place on numpy arrays: cache int8 [pages, Hkv, 2, page, d], scale fp32; rows [2, T, Hkv, d] in 64 bits."""
    page = cache.shape[3]
    for s in range(len(length)):
        at, todo = int(length[s]), list(range(begin[s], begin[s + 1]))
        if at < 0:
            continue
        while todo:
            r0 = at % page
            now, todo = todo[:page - r0], todo[page - r0:]
            slot, at = at // page, at + len(now)
            if slot >= table.shape[1] or not 0 <= table[s, slot] < cache.shape[0]:
                continue
            p = table[s, slot]
            for h in range(cache.shape[1]):
                for side in range(2):
                    x = rows[side, now, h]
                    old = float(scale[p, h, side])
                    if not np.isfinite(x).all() or (r0 and np.isnan(old)):
                        scale[p, h, side] = np.nan
                        cache[p, h, side, r0:r0 + len(now)] = 0
                        if not np.isfinite(x).all():
                            continue
                        cache[p, h, side, r0:r0 + len(now)] = 0
                        continue
                    new = 2.0 ** power_of_two(np.abs(x).max())
                    if r0:
                        new = max(new, old)
                        if new > old:
                            cache[p, h, side, :r0] = np.rint(cache[p, h, side, :r0] * (old / new))
                    scale[p, h, side] = new
                    cache[p, h, side, r0:r0 + len(now)] = np.rint(x / new)


def held(cache, scale, table, s, n):
    """Tokens 0 .. n - 1 of sequence s as the values their codes stand for: [2, n, Hkv, d] in 64 bits."""
    page = cache.shape[3]
    out = np.zeros((2, n, cache.shape[1], cache.shape[4]))
    for slot in range(-(-n // page)):
        p, m = table[s, slot], min(page, n - slot * page)
        out[:, slot * page:slot * page + m] = (cache[p].astype(np.float64) * scale[p].astype(np.float64)[..., None, None])[:, :, :m].transpose(1, 2, 0, 3)
    return out


def update(table, length, refs, parent, grow, page, cache, scale):
    """In place on numpy arrays (cache, scale with a leading dimension of layers); returns the pages that are missing."""
    S, W = table.shape
    pages, old, old_length = refs.shape[0], table.copy(), length.copy()
    for row in old:
        for p in row:
            if 0 <= p < pages:
                refs[p] -= 1
    rows, kept, missing = [], set(), 0
    for s in range(S):
        p = parent[s]
        n = int(old_length[p]) if 0 <= p < S else 0
        n = n if 0 <= n <= W * page else 0
        keeps = n % page > 0 and p not in kept
        if keeps:
            kept.add(p)
        row = [int(x) if 0 <= x < pages else -1 for x in old[p][:n // page + keeps]] if n else []
        for x in row:
            if x >= 0:
                refs[x] += 1
        rows.append(row)
        length[s] = n
    free = [p for p in range(pages) if refs[p] == 0]
    for s in range(S):
        n, row = int(length[s]), rows[s]
        need = -(-(n + max(0, int(grow[s]))) // page)
        missing += max(0, need - W)
        while len(row) < min(need, W):
            if free:
                x = free.pop(0)
                refs[x] = 1
                if len(row) < -(-n // page):                     # the copy of a page that is filled in part
                    source = int(old[parent[s]][len(row)])
                    if 0 <= source < pages:
                        cache[:, x, :, :, :n % page] = cache[:, source, :, :, :n % page]
                        scale[:, x] = scale[:, source]
                    else:
                        scale[:, x] = np.nan
            else:
                x = -1
                missing += 1
            row.append(x)
        table[s] = row + [-1] * (W - len(row))
    return missing
