"""Oracle of the 4-bit cache, the attention over it, and of pages as a whole: plain numpy, 64-bit arithmetic, written from the
definitions alone.  (Test infrastructure; the product never imports it.)"""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
GROUP, SUB = 32, 16
NAN_SCALE = 255


def quantize(x):
    """Codes and scale exponents (uint8) of float64 rows [..., channels]; every group of 32 channels by itself."""
    g = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (-1, GROUP))
    top = np.abs(g).max(-1)
    finite = np.isfinite(top)
    exponents = np.arange(-125, 126)
    # the smallest power of two of which 7 times reach the largest magnitude; the largest there is, if none do
    reach = 7.0 * 2.0 ** exponents
    e = exponents[np.minimum(np.searchsorted(reach, np.where(finite, top, 0.0)), len(exponents) - 1)]
    y = np.where(finite[..., None], g, 0.0) / (2.0 ** e)[..., None]
    far = np.abs(np.abs(y)[..., None] - GRID)
    code = np.argmin(far, -1)                              # of two as near the first
    tie = (code < 7) & (np.take_along_axis(far, np.minimum(code + 1, 7)[..., None], -1)[..., 0] == far.min(-1))
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    code = np.where(finite[..., None], code + 8 * np.signbit(y), 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, e + 127, NAN_SCALE).astype(np.uint8)


def dequantize(code, scale):
    """float64 values of codes [..., channels] and scales [..., channels / 32]."""
    v = np.concatenate([GRID, -GRID])[code].reshape(code.shape[:-1] + (-1, GROUP))
    s = np.where(scale == NAN_SCALE, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (v * s[..., None]).reshape(code.shape)


def places(part, head, token, hd):
    """Byte offsets within a 16-token block, and shifts, of a token's codes [hd], and byte offsets of its scales [hd / 32]."""
    c, g = np.arange(hd), np.arange(hd // GROUP)
    if part == 0:
        return token * (hd // 2) + c // 2, 4 * (c % 2), 16 * hd + token * (hd // GROUP) + g
    per = hd // 16                                          # channels of a slice
    at = 8 * hd + (((token // 4) * 16 + c // per) * 4 + token % 4) * (per // 2) + c % per // 2
    return at, 4 * (c % 2), 16 * hd + hd // 2 + ((token // 4) * (hd // GROUP) + g) * 4 + token % 4


def _slot(pos, table, block):
    return int(table[pos // block]), pos % block


def store_token(pool, page, slot, k, v):
    """k, v float64 [heads, hd] into uint8 pool [pages][heads][block / 16][17 * hd]."""
    heads, hd = k.shape
    for part, x in enumerate((k, v)):
        code, scale = quantize(x)
        for h in range(heads):
            b = pool[page, h, slot // SUB]
            at, shift, scales = places(part, h, slot % SUB, hd)
            b[at[::2]] = code[h, ::2] << shift[::2] | code[h, 1::2] << shift[1::2]      # two channels a byte
            b[scales] = scale[h]


def load_token(pool, page, slot, hd):
    """(k, v) float64 [heads, hd]"""
    out = []
    for part in (0, 1):
        at, shift, scales = places(part, 0, slot % SUB, hd)
        b = pool[page, :, slot // SUB]
        out.append(dequantize((b[:, at] >> shift) & 15, b[:, scales]))
    return out


def load_keys(pool, table, keys, block, hd):
    """k, v float64 [keys, heads, hd] of a context, and whether each has a page."""
    heads = pool.shape[1]
    k, v, there = np.zeros((keys, heads, hd)), np.zeros((keys, heads, hd)), np.zeros(keys, dtype=bool)
    for j in range(keys):
        page, slot = _slot(j, table, block) if j // block < len(table) else (-1, 0)
        if 0 <= page < pool.shape[0]:
            there[j] = True
            k[j], v[j] = load_token(pool, page, slot, hd)
    return k, v, there


def attend(q, positions, k, v, there, scale, window):
    """Queries float64 [n, n_q, hd] of one context over its keys [keys, heads, hd].  Returns out, lse, and for every output the sum
    of |weight * v| (what errors are measured against) and, per row, the largest scale * sum |q| |k| of a seen key."""
    n, n_q, hd = q.shape
    group = n_q // k.shape[1] if k.shape[1] else 1
    out, lse = np.zeros((n, n_q, hd)), np.full((n, n_q), -np.inf)
    size, reach = np.zeros((n, n_q, hd)), np.zeros((n, n_q))
    j = np.arange(k.shape[0])
    for i in range(n):
        p = int(positions[i])
        seen = there & (j <= p) & (j > p - window if window else j >= 0)
        if not seen.any():
            continue
        for h in range(n_q):
            kk, vv = k[seen, h // group], v[seen, h // group]
            s = scale * (kk @ q[i, h])
            m = s.max()
            w = np.exp(s - m)
            lse[i, h] = m + np.log(w.sum())
            w /= w.sum()
            out[i, h] = w @ vv
            size[i, h] = w @ np.abs(vv)
            reach[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, lse, size, reach


def fork(tables, pages_copied, from_rows, to_rows, n_tok, new_pages, block):
    """Tables after the forks; appends (source page, new page, tokens) to `pages_copied`."""
    t = tables.copy()
    for a, b, n, new in zip(from_rows, to_rows, n_tok, new_pages):
        full, rest = n // block, n % block
        t[b] = -1
        t[b, :full] = tables[a, :full]
        if rest:
            t[b, full] = new
            pages_copied.append((int(tables[a, full]), int(new), int(rest)))
    return t


def compact(tables, num_pages):
    """(tables, live, moves [(from, to)], new number of every page)"""
    live = sorted({int(p) for p in tables.ravel() if 0 <= p < num_pages})
    n = len(live)
    free = [p for p in range(n) if p not in set(live)]
    moving = [p for p in live if p >= n]
    place = np.full(num_pages, -1, dtype=np.int32)
    place[live] = live
    place[moving] = free
    valid = (tables >= 0) & (tables < num_pages)
    return np.where(valid, place[np.clip(tables, 0, num_pages - 1)], -1).astype(np.int32), n, list(zip(moving, free)), place
