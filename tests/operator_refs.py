"""Plain implementations, in 64 bits on the CPU, of the rotary positions, the 8-bit cache and its decoding step."""
from decimal import Decimal, getcontext

import numpy as np

STRIDED, FIXED, PER_HEAD = 0, 1, 2
A1, A2, MERGED, INTERLEAVED = 0, 1, 2, 3
PI = Decimal("3.14159265358979323846264338327950288419716939937510")


def turn_table(places, dims, base):
    """Angle of every pair of a token, as a fraction of a turn in [-1/2, 1/2], from 50 digits: [tokens, pairs]."""
    getcontext().prec = 50
    out = []
    for row in places:
        turns = []
        for p, s in zip(row, dims):
            for t in range(s // 2):
                x = Decimal(int(p)) * Decimal(base) ** (Decimal(-2 * t) / Decimal(s)) / (2 * PI)
                turns.append(float(x - x.to_integral_value()))
        out.append(turns)
    return np.array(out).reshape(len(out), sum(dims) // 2)


def pair_elements(dims, halves):
    first, second, at = [], [], 0
    for s in dims:
        t = np.arange(s // 2)
        first.append(at + (t if halves else 2 * t))
        second.append(at + (t + s // 2 if halves else 2 * t + 1))
        at += s
    return np.concatenate(first), np.concatenate(second)


def rotary(x, turns, dims, halves, inverse=False):
    """x [b, h, n, d] float64, turns [b or 1, n, pairs]: (y, |x0| + |x1| of each element's pair, 0 where none)."""
    m, p = pair_elements(dims, halves)
    c, s = np.cos(2 * np.pi * turns)[:, None], np.sin(2 * np.pi * turns)[:, None] * (-1 if inverse else 1)
    y, size = x.copy(), np.zeros_like(x)
    y[..., m] = x[..., m] * c - x[..., p] * s
    y[..., p] = x[..., m] * s + x[..., p] * c
    size[..., m] = size[..., p] = np.abs(x[..., m]) + np.abs(x[..., p])
    return y, size


def e4m3_values():
    """The value of every code."""
    v = []
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v.append((-1) ** (code >> 7) * (x if code & 127 != 127 else float("nan")))
    return np.array(v)


VALUES = e4m3_values()


def e4m3_encode(x):
    """Codes of float64 values of magnitude <= 448: nearest, ties to the even code; NaN and infinities 0x7f."""
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    up = np.searchsorted(VALUES[:127], a).clip(0, 126)
    lo = np.maximum(up - 1, 0)
    du, dl = VALUES[up] - a, a - VALUES[lo]
    code = np.where((dl < du) | ((dl == du) & (lo % 2 == 0)), lo, up)
    code = np.where(np.signbit(x), code | 128, code)
    return np.where(np.isfinite(x), code, 0x7F).astype(np.uint8)


def scale_exponent(top):
    """Least e in [-100, 120] with top <= 448 * 2^e."""
    e = -100
    while e < 120 and top > 448.0 * 2.0 ** e:
        e += 1
    return e


def store(codes, scales, x, start, counts, block):
    """x [b, h, n, d] float64 into codes [b, h, capacity, d] uint8 and scales [b, h, blocks], in place."""
    b, h, n, _ = x.shape
    capacity = codes.shape[2]
    for i in range(b):
        s = int(start[i])
        end = min(s + min(max(int(counts[i]), 0), n), capacity)
        if s < 0 or end <= s:
            continue
        for blk in range(s // block, (end - 1) // block + 1):
            r0, r1 = max(s, blk * block), min(end, (blk + 1) * block)
            for j in range(h):
                new = x[i, j, r0 - s:r1 - s]
                e = scale_exponent(np.abs(np.where(np.isfinite(new), new, 0.0)).max())
                if s > blk * block:
                    before = int(np.log2(scales[i, j, blk]))
                    e = max(e, before)
                    old = codes[i, j, blk * block:s]
                    if e > before:
                        codes[i, j, blk * block:s] = e4m3_encode(VALUES[old] * 2.0 ** (before - e))
                codes[i, j, r0:r1] = e4m3_encode(new * 2.0 ** -e)
                scales[i, j, blk] = 2.0 ** e


def attended(pattern, mode, l, c, h, pos):
    """The set of head h at pos, from its definition."""
    j = np.arange(pos + 1)
    if pattern == STRIDED:
        a1, a2 = pos - j <= l, (pos - j) % l == 0
    else:
        w = l - c * (1 + (h % (l // c) if pattern == PER_HEAD else 0))
        a1, a2 = j // l == pos // l, (j % l >= w) & (j % l < w + c)
    part = (A1, A2)[h % 2] if mode == INTERLEAVED else mode
    return np.nonzero(a1 if part == A1 else a2 if part == A2 else a1 | a2)[0]


def decode(q, k, v, positions, l, c, pattern, mode, scale):
    """q [b, h, d], k and v [b, kv_h, capacity, d] float64 (values).  Returns o, lse, and for each row what bounds
    the error: sum p |v|, the largest sum |q| |k| scale over its keys, and the number of keys."""
    b, h, d = q.shape
    group = h // k.shape[1]
    o, lse = np.zeros((b, h, d)), np.full((b, h), -np.inf)
    pv, qk, count = np.zeros((b, h, d)), np.zeros((b, h)), np.zeros((b, h))
    for i, pos in enumerate(positions):
        for j in range(h if pos >= 0 else 0):
            at = attended(pattern, mode, l, c, j, pos)
            if not len(at):
                continue
            kk, vv = k[i, j // group, at], v[i, j // group, at]
            s = kk @ q[i, j] * scale
            lse[i, j] = s.max() + np.log(np.exp(s - s.max()).sum())
            p = np.exp(s - lse[i, j])
            o[i, j], pv[i, j] = p @ vv, p @ np.abs(vv)
            qk[i, j], count[i, j] = (np.abs(kk) @ np.abs(q[i, j])).max() * scale, len(at)
    return o, lse, pv, qk, count
