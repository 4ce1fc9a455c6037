"""Plain implementations, in 64 bits on the CPU, of page tables, paged storing, packed prompts and decoding over pages."""
import numpy as np

import operator_refs as ref


def page_tables(table, held, fresh, free, page, tokens):
    """table [sequences, max_pages] in place.  Returns starts, positions, slots, last, taken."""
    width = table.shape[1]
    starts, last, taken = [0], [], 0
    positions, slots = np.full(tokens, -1, np.int64), np.full(tokens, -1, np.int64)
    for s in range(len(held)):
        h, row = min(max(int(held[s]), 0), width * page), starts[-1]
        rows = min(max(int(fresh[s]), 0), tokens - row)
        end = min(h + rows, width * page)
        for i in range(-(-h // page), -(-end // page)):
            table[s, i] = free[taken] if taken < len(free) else -1
            taken += 1
        for p in range(h, end):
            positions[row + p - h] = p
            if table[s, p // page] >= 0:
                slots[row + p - h] = table[s, p // page] * page + p % page
        starts.append(row + rows)
        last.append(end - 1)
    return np.array(starts), positions, slots, np.array(last), np.array([taken])


def set_mask(pattern, mode, l, c, h, n):
    """[n, n]: whether row i of a sequence attends position j, from the set's definition."""
    i, j = np.arange(n)[:, None], np.arange(n)[None]
    if pattern == ref.STRIDED:
        a1, a2 = i - j <= l, (i - j) % l == 0
    else:
        w = l - c * (1 + (h % (l // c) if pattern == ref.PER_HEAD else 0))
        a1, a2 = i // l == j // l, (j % l >= w) & (j % l < w + c)
    part = (ref.A1, ref.A2)[h % 2] if mode == ref.INTERLEAVED else mode
    return (j <= i) & (a1 if part == ref.A1 else a2 if part == ref.A2 else a1 | a2)


def packed(q, k, v, starts, l, c, pattern, mode, scale):
    """q [n, h, d], k and v [n, kv_h, d] float64.  Returns o [n, h, d], lse [h, n], and for each row what bounds the
    error: sum p |v|, the largest sum |q| |k| scale over its keys, and the number of keys.  Rows outside: NaN."""
    n, h, d = q.shape
    group = h // k.shape[1]
    o, lse = np.full((n, h, d), np.nan), np.full((h, n), np.nan)
    pv, qk, count = np.zeros((n, h, d)), np.zeros((n, h)), np.zeros((n, h))
    for a, b in zip(starts[:-1], starts[1:]):
        for j in range(h if b > a else 0):
            keep = set_mask(pattern, mode, l, c, j, b - a)
            x, kk, vv = q[a:b, j], k[a:b, j // group], v[a:b, j // group]
            s = np.where(keep, x @ kk.T * scale, -np.inf)
            top = s.max(axis=1)
            p = np.exp(s - np.where(np.isneginf(top), 0, top)[:, None])
            total = p.sum(axis=1)
            with np.errstate(divide="ignore"):
                lse[j, a:b] = np.where(np.isneginf(top), -np.inf, top + np.log(total))
            p /= np.where(total > 0, total, 1)[:, None]
            o[a:b, j], pv[a:b, j] = p @ vv, p @ np.abs(vv)
            qk[a:b, j] = np.where(keep, np.abs(x) @ np.abs(kk).T * scale, 0).max(axis=1)
            count[a:b, j] = keep.sum(axis=1)
    return o, lse, pv, qk, count


def gather(pages, table, capacity, page):
    """[b, kv_h, capacity, d] from pages [pages, kv_h, page, d]; positions without a page hold NaN."""
    b, (_, h, _, d) = len(table), pages.shape
    out = np.full((b, h, capacity, d), np.nan)
    for i in range(b):
        for at in range(0, capacity, page):
            p = table[i, at // page]
            if 0 <= p < len(pages):
                n = min(page, capacity - at)
                out[i, :, at:at + n] = pages[p, :, :n]
    return out


def bounds(o_ref, lse_ref, pv, qk, count, d, last, piece):
    """How far o and lse may be off.  A score is a sum of d products in fp32, off by e = (d + 8) 2^-24 sum |q||k| scale
    (products, sums, and its two scalings), and so is the log-sum-exp, plus 2^-22 of its size for the base-2 units and the
    logarithm, and count 2^-24 for the sum.  A weight is off by 2 e + 2^-20 relative (both ends of its difference;
    exponentials and rescaling) and the sum by count 2^-24; weights carry `piece`, outputs round by `last`."""
    e = (d + 8) * 2.0 ** -24 * qk
    size = np.abs(np.where(np.isfinite(lse_ref), lse_ref, 0.0))
    lse = e + 2.0 ** -22 * (size + 1) + count * 2.0 ** -24
    o = (2 * e + 2.0 ** -20 + 2 * count * 2.0 ** -24 + piece)[..., None] * pv + last * np.abs(o_ref)
    return o, lse
