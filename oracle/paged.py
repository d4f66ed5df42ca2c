"""The paged key/value cache in float64: quantising rows, what they stand for,
key bounds of pages, page selection and attention over a sequence's tokens.

Pools are numpy arrays: ``k``, ``v`` [pages][heads][page][head_dim] of values in
the format (bf16 values, or the numbers q of the 8-bit formats) and, for the
8-bit formats, ``k_exp``, ``v_exp`` [pages][heads][page] exponent codes; a
cached value is q * 2^(code - 127).
"""
from __future__ import annotations

import numpy as np

LIMIT = {"e4m3": 448.0, "int8": 127.0}
LEAST = -111
# What stands in for a number that would be rounded to 2^128, which no float32
# row holds: the next one towards zero, with the exponent that such rows have.
TOP = {"e4m3": 240.0, "int8": 63.0}


def round_e4m3(y):
    """Nearest e4m3 number (three bits behind the leading one, exponents from
    -6), ties to even; |y| <= 448."""
    y = np.asarray(y, np.float64)
    _, e = np.frexp(np.where(y == 0, 1.0, y))
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.rint(y / step) * step


def quantise(x, fmt):
    """Rows (last axis) of float32 values -> (q, codes); a row that is not finite:
    NaN (e4m3) or 0 (int8) with code 255."""
    x = np.asarray(x, np.float64)
    amax = np.abs(x).max(-1)
    bad = ~np.isfinite(amax)
    amax = np.where(bad, 0.0, amax)
    f, e = np.frexp(np.where(amax == 0, 1.0, amax) / LIMIT[fmt])
    e = np.where(f == 0.5, e - 1, e)           # an exact power of two
    # the quotient above is rounded: settle on the least e with amax <= limit 2^e
    e = np.where(amax <= LIMIT[fmt] * np.exp2(e - 1.0), e - 1, e)
    e = np.where(amax > LIMIT[fmt] * np.exp2(e * 1.0), e + 1, e)
    e = np.where(amax == 0, LEAST, np.maximum(e, LEAST))
    with np.errstate(invalid="ignore"):
        y = x * np.exp2(-e * 1.0)[..., None]
        q = round_e4m3(np.where(bad[..., None], 0.0, y)) if fmt == "e4m3" else np.rint(y)
    q = np.where(np.abs(q) * np.exp2(e * 1.0)[..., None] >= 2.0 ** 128, np.sign(q) * TOP[fmt], q)
    q = np.where(bad[..., None], np.nan if fmt == "e4m3" else 0.0, q)
    return q, np.where(bad, 255, e + 127).astype(np.int64)


def value(q, code):
    """q * 2^(code - 127); NaN for the code 255."""
    code = np.asarray(code)
    s = np.where(code == 255, np.nan, np.exp2(np.where(code == 255, 127, code) - 127.0))
    return np.asarray(q, np.float64) * s[..., None]


def tokens(pool, exp, table, n, page):
    """The first n tokens of the sequence with this page table:
    [n][heads][head_dim], and whether each lies in the pool."""
    j = np.arange(n)
    at, slot = np.asarray(table)[j // page], j % page
    ok = (at >= 0) & (at < pool.shape[0])
    at = np.where(ok, at, 0)
    x = pool[at, :, slot]
    return (np.asarray(x, np.float64) if exp is None else value(x, exp[at, :, slot])), ok


def bounds(keys):
    """Keys of a page [tokens][heads][head_dim] -> (int8 numbers [heads][2][head_dim], codes)."""
    k = np.asarray(keys, np.float64)
    both = np.concatenate((k.max(0), k.min(0)), -1)
    both = np.where(np.isfinite(k).all((0, 2))[:, None], both, np.nan)
    q, code = quantise(both, "int8")
    return q.reshape(k.shape[1], 2, k.shape[2]), code


def scores(q, bound, code):
    """Scores of one row's queries of a key head [group][head_dim] for pages
    with bounds [pages][2][head_dim] and exponent codes [pages]."""
    qq, qc = quantise(q, "int8")
    whole = np.maximum(qq, 0) @ bound[:, 0].T + np.minimum(qq, 0) @ bound[:, 1].T
    s = whole * np.exp2(code - 127.0) * np.exp2(qc - 127.0)[:, None]
    s = np.where((code == 255) | (qc == 255)[:, None], -np.inf, s)
    return s.max(0)


def select(score, n_select):
    """The n_select pages of the highest score, equal ones in order, ascending, -1 behind."""
    order = sorted(range(len(score)), key=lambda p: (-score[p], p))[:n_select]
    return sorted(order) + [-1] * (n_select - len(order))


def attention(q, k, v, look=None):
    """Rows q [rows][dh] over keys [n][dh], where `look` [rows][n] says so.
    Returns (o, a, d): the output, sum_j w_j |v_j| and the largest of
    sum_d |q_d k_d| / sqrt(dh) over the keys that count (what rounding errors scale with)."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    rows, n = q.shape[0], k.shape[0]
    o, a, d = np.zeros((rows, v.shape[1])), np.zeros((rows, v.shape[1])), np.zeros(rows)
    for i in range(rows):
        at = np.arange(n) if look is None else np.flatnonzero(look[i])
        if not at.size:
            continue
        s = k[at] @ q[i] / np.sqrt(q.shape[1])
        with np.errstate(invalid="ignore"):
            w = np.exp(s - s.max())
            w = w / w.sum()
        o[i], a[i] = w @ v[at], w @ np.abs(v[at])
        d[i] = (np.abs(k[at]) @ np.abs(q[i])).max() / np.sqrt(q.shape[1])
    return o, a, d
