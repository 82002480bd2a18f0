"""CPU oracle for softmax attention on a paged key/value cache.  TEST INFRASTRUCTURE ONLY, like gr_oracle.py: plain float64 numpy, one sequence and one
head at a time, sharing no code with the library."""
import numpy as np


def rotate(x, positions, frequencies, interleaved):
    """x [tokens, heads, dim]: pair j of the first 2 * len(frequencies) features turned by positions * frequencies[j].  Angles in extended precision: a
    product of a position of 2^30 with a frequency keeps 2^-34 of a radian."""
    x = np.array(x, np.float64)
    r = 2 * len(frequencies)
    if r == 0:
        return x
    angle = np.asarray(positions, np.longdouble)[:, None] * np.asarray(frequencies, np.longdouble)[None, :]
    c, s = np.cos(angle).astype(np.float64)[:, None, :], np.sin(angle).astype(np.float64)[:, None, :]
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    first, second = x[..., a].copy(), x[..., b].copy()
    x[..., a] = first * c - second * s
    x[..., b] = first * s + second * c
    return x


def attend(q, k, v, scale, seen=None):
    """Causal attention of one sequence: q [m, Hq, dim], k and v [n, Hkv, dim]; row i sees keys 0..n-m+i, of those only where seen [n] is true.
    Returns the outputs and, for error bounds, sum w |v| [m, Hq, dim] and the largest scale * sum |q||k| of a row [m, Hq]."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    m, hq, dim = q.shape
    n, hkv = k.shape[0], k.shape[1]
    out, spread, size = np.zeros((m, hq, dim)), np.zeros((m, hq, dim)), np.zeros((m, hq))
    for h in range(hq):
        kh, vh = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
        for i in range(m):
            keys = np.arange(max(0, n - m + i + 1))
            if seen is not None:
                keys = keys[seen[keys]]
            if not len(keys):
                continue
            z = scale * (kh[keys] @ q[i, h])
            w = np.exp(z - z.max())
            w /= w.sum()
            out[i, h] = w @ vh[keys]
            spread[i, h] = w @ np.abs(vh[keys])
            size[i, h] = scale * (np.abs(kh[keys]) @ np.abs(q[i, h])).max()
    return out, spread, size


def page_rows(table_row, page_size, n_pages, n):
    """(page, slot) of tokens 0..n-1 of a sequence, and which of them lie in a page of the pool."""
    t = np.arange(n)
    page, slot = np.asarray(table_row)[t // page_size], t % page_size
    return page, slot, (page >= 0) & (page < n_pages)
