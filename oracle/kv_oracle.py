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


# codes of the quantised caches: bits of the fraction, exponent bias, and what a block's largest size over its scale may be (that itself included, or not)
FORMS = {"f8": (3, 7, 464.0, True), "f4": (1, 1, 7.0, False)}


def code_values(form):
    """Values of the codes without a sign, in their order; the last of f8, which is NaN, left out."""
    fraction, bias = FORMS[form][:2]
    count = 127 if form == "f8" else 8
    return np.array([(c & (1 << fraction) - 1) * 2.0 ** (1 - bias - fraction) if c >> fraction == 0 else (1 + (c & (1 << fraction) - 1) / 2.0 ** fraction) * 2.0 ** ((c >> fraction) - bias)
                     for c in range(count)])


def quantise(x, form, dtype):
    """x [..., dim] as a cache of an element type holds it: codes [..., dim] (0..255 or 0..15), scale bytes [..., dim / 32] and the values."""
    fraction, bias, limit, closed = FORMS[form]
    least = {("f8", True): -15, ("f8", False): -117, ("f4", True): -23, ("f4", False): -125}[form, dtype == "f16"]
    most = {("f8", True): 61440.0, ("f8", False): 240.0 * 2.0 ** 120, ("f4", True): 49152.0, ("f4", False): 1.5 * 2.0 ** 127}[form, dtype == "f16"]
    x = np.asarray(x, np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    broken = ~np.isfinite(blocks).all(-1)
    blocks = np.clip(np.where(np.isfinite(blocks), blocks, 0), -most, most)
    size = np.abs(blocks).max(-1)
    e = np.full(size.shape, least)
    for _ in range(300):                                # the least exponent at which the largest fits
        fits = size <= limit * 2.0 ** e if closed else size < limit * 2.0 ** e
        if fits.all():
            break
        e = np.where(fits, e, e + 1)
    y = blocks / 2.0 ** e[..., None]
    values = code_values(form)
    middle = (values[1:] + values[:-1]) / 2
    code = np.searchsorted(middle, np.abs(y))           # a middle stays with the lower code
    tie = (np.abs(y) == np.append(middle, np.inf)[code]) & (code % 2 == 1)
    code = code + tie
    sign = np.signbit(y)
    back = np.where(sign, -1.0, 1.0) * values[code] * 2.0 ** e[..., None]
    back = np.where(broken[..., None], np.nan, back)
    code = code + sign * (128 if form == "f8" else 8)
    return code.reshape(x.shape), np.where(broken, 255, e + 127), back.reshape(x.shape)


def stored_values(codes, scales, form):
    """Values of codes [..., dim] with scale bytes [..., dim / 32]."""
    values = code_values(form)
    if form == "f8":
        values = np.append(values, np.nan)
    half = len(values)
    y = np.where(codes >= half, -1.0, 1.0) * values[codes % half]
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return y * np.repeat(scale, 32, -1)


def unpack(pool, form):
    """Codes of the bytes of a pool."""
    if form == "f8":
        return pool.astype(np.int64)
    return np.stack([pool & 15, pool >> 4], -1).reshape(*pool.shape[:-1], -1).astype(np.int64)
