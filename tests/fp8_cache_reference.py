"""The operators of the 8-bit key and value cache from their definitions, in 64 bits (NumPy), and how far the kernels may be off."""
import numpy as np
import torch

from fp8_reference import e4m3, to64

LEAST, MOST = -40, 40


def page_scale(amax):
    """The exponent of a page's scale for the largest magnitude written to it."""
    e = LEAST
    while e < MOST and amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def held(cache):
    """The cache as float64 codes and integer exponents: [k, v], [k, v]."""
    return [to64(cache.k), to64(cache.v)], [cache.k_scales.view(torch.uint8).cpu().numpy().astype(int) - 127,
                                            cache.v_scales.view(torch.uint8).cpu().numpy().astype(int) - 127]


def clamped(x, e):
    """Codes of values for the scale 2^e."""
    with np.errstate(invalid="ignore"):
        y = np.clip(np.where(np.isfinite(x), x, 0.0) * 2.0 ** -e, -448.0, 448.0)
    return np.where(np.isfinite(x), e4m3(y), np.nan)


def places(table, lengths, starts, rows, page):
    """(row, page's number, token of the page, whether the step begins the page) of every row that has a place, in order."""
    out = []
    for s, length in enumerate(lengths):
        a, b = (s, s + 1) if starts is None else (starts[s], starts[s + 1])
        for r in range(a, b):
            at = length - (b - r)
            if 0 <= at and at // page < table.shape[1]:
                out.append((r, table[s][at // page], at % page, at // page * page >= max(0, length - (b - a))))
    return out


def write(codes, exponents, x, table, lengths, starts, page):
    """Writes the rows x [row][head][dim] (float64) into codes and exponents, in place."""
    todo = {}
    for r, pid, t, begun in places(table, lengths, starts, x.shape[0], page):
        if 0 <= pid < codes.shape[0]:
            todo.setdefault(pid, ([], begun))[0].append((r, t))
    for pid, (tokens, begun) in todo.items():
        first = min(t for _, t in tokens)
        for h in range(codes.shape[1]):
            new = np.stack([x[r, h] for r, _ in tokens])
            e = page_scale(np.abs(np.where(np.isfinite(new), new, 0.0)).max())
            if not begun:
                e = max(e, exponents[pid, h])
                old = codes[pid, h, :first]
                codes[pid, h, :first] = np.where(np.isnan(old), np.nan, e4m3(np.where(np.isnan(old), 0.0, old) * 2.0 ** (exponents[pid, h] - e)))
            exponents[pid, h] = e
            for (_, t), v in zip(tokens, new):
                codes[pid, h, t] = clamped(v, e)


def sequence(codes, exponents, pages, length, page):
    """[head][token][dim] of one sequence; pages that are not there hold zeros."""
    out = np.zeros((codes.shape[1], length, codes.shape[3]))
    for i in range(0, length, page):
        n, pid = min(page, length - i), pages[i // page]
        if 0 <= pid < codes.shape[0]:
            out[:, i:i + n] = codes[pid, :, :n] * np.exp2(exponents[pid].astype(float))[:, None, None]
    return out


def attention(q, codes, exponents, table, lengths, starts, page, causal=True, window=0, scale=None):
    """(out, lse, slack of out, slack of lse) of the rows of sequences, others NaN.

    The slack: a query is two codes, off by 2^-17 of its row's largest value; scores add up at most dim + 32 terms of fp32, each
    step cutting off 2^-23 of the magnitudes' sum; 2^x is off by 2^-21 of itself, its argument rounded twice to 2^-24 of at most
    |s| + 64; a weight is two codes, off by 2^-8 of itself, or 2^-17 of the largest; sums of n weights and products
    lose 2^-23 of their magnitudes' sum a step, of which there are n / 32 + 64 (tokens of a tile add up inside the tensor cores);
    the result is rounded once, by 2^-8 of itself."""
    rows, heads, dim = q.shape
    kv = codes[0].shape[1]
    group = heads // kv
    scale = 1 / np.sqrt(dim) if scale is None else scale
    out, lse = np.full(q.shape, np.nan), np.full((rows, heads), np.nan)
    slack, slack_lse = np.zeros(q.shape), np.zeros((rows, heads))
    for s, length in enumerate(lengths):
        a, b = (s, s + 1) if starts is None else (starts[s], starts[s + 1])
        if a == b:
            continue
        total = min(length, table.shape[1] * page)
        k, v = (sequence(c, e, table[s], total, page) for c, e in zip(codes, exponents))
        position = np.arange(length - (b - a), length)[:, None]
        token = np.arange(total)[None, :]
        seen = np.ones((b - a, total), dtype=bool)
        if causal:
            seen &= token <= position
        if window:
            seen &= token > position - window
        some = seen.any(axis=1)
        count = seen.sum(axis=1)
        steps = (count / 32 + 64) * 2.0 ** -23
        for h in range(heads):
            kh, vh, qh = k[h // group], v[h // group], q[a:b, h]
            with np.errstate(invalid="ignore"):
                w = np.where(seen, scale * (qh @ kh.T), -np.inf)
            m = np.where(some, w.max(axis=1, initial=-np.inf), 0.0)
            p = np.exp(w - m[:, None])
            sums = p.sum(axis=1)
            with np.errstate(divide="ignore"):
                lse[a:b, h] = np.where(some, m + np.log(sums), -np.inf)
            p = p / np.where(some, sums, 1.0)[:, None]
            out[a:b, h] = p @ vh
            off = scale * (2.0 ** -17 * np.abs(qh).max(axis=1)[:, None] * np.abs(kh).sum(axis=1)[None, :] + (dim + 32) * 2.0 ** -23 * (np.abs(qh) @ np.abs(kh).T))
            off = np.where(seen, off, 0.0).max(axis=1, initial=0.0) + (np.where(seen, np.abs(w), 0.0).max(axis=1, initial=0.0) + 64) * 2.0 ** -22
            largest = np.where(seen, np.abs(vh).max(axis=1, initial=0.0)[None, :], 0.0).max(axis=1, initial=0.0)
            slack[a:b, h] = 2.0 ** -8 * np.abs(out[a:b, h]) + (2.0 ** -8 + 2 * off + 2 * steps)[:, None] * (p @ np.abs(vh)) + (2.0 ** -17 * largest + 2.0 ** -130)[:, None]
            slack_lse[a:b, h] = off + steps + 2.0 ** -22 * np.abs(np.where(some, lse[a:b, h], 0.0)) + 2.0 ** -21
    return out, lse, slack, slack_lse
