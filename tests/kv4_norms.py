"""Attention over the 4-bit cache held to norms, beside the limits per output of kv4_harness.attend_limits: outputs shrink with the
root of the number of keys, those limits do not, so over thousands of keys a run of values from a wrong place would pass them.
(Test infrastructure; not product code.)"""
import numpy as np

import gpu_harness as gh
import kv4_harness as kh
import oracle.kv4_oracle as kv4
from test_gpu_kv4 import Call


def store_keys(pool, table, block, hd, x):
    """kv4.store_token of all tokens x [n, 2, heads, hd] of a context at once, from slot 0 on."""
    code, scale = kv4.quantize(x)
    j = np.arange(len(x))
    for token in range(16):
        at = j[j % 16 == token]
        page, sub = np.asarray(table)[at // block], at % block // 16
        for part in (0, 1):
            codes, shift, scales = kv4.places(part, 0, token, hd)
            pool[page[:, None], :, sub[:, None], codes[None, ::2]] = (code[at, part][..., 0::2] | code[at, part][..., 1::2] << 4).transpose(0, 2, 1)
            pool[page[:, None], :, sub[:, None], scales[None]] = scale[at, part].transpose(0, 2, 1)


def load_keys(pool, table, keys, block, hd):
    """kv4.load_keys of a context at once."""
    j = np.arange(keys)
    entry = np.append(np.asarray(table), -1)[np.minimum(j // block, len(table))]
    there = (entry >= 0) & (entry < pool.shape[0])
    out = np.zeros((2, keys, pool.shape[1], hd))
    for token in range(16):
        at = j[there & (j % 16 == token)]
        if not len(at):
            continue
        b = pool[entry[at], :, at % block // 16]
        for part in (0, 1):
            codes, shift, scales = kv4.places(part, 0, token, hd)
            out[part, at] = kv4.dequantize((b[..., codes] >> shift.astype(np.uint8)) & 15, b[..., scales])
    return out[0], out[1], there


class Cache(kh.Cache):
    """kh.Cache for long contexts."""

    def __init__(self, rng, lens, n_kv, hd, block, slack=3):
        super().__init__(rng, [0] * len(lens), n_kv, hd, block)
        self.lens = list(lens)
        blocks = [-(-n // block) for n in lens]
        self.num_pages = sum(blocks) + slack
        self.pool = np.full((self.num_pages, n_kv, block // 16, 17 * hd), 0xFF, dtype=np.uint8)
        perm = rng.permutation(self.num_pages).astype(np.int32)
        self.tables = np.full((len(lens), max(blocks)), -1, dtype=np.int32)
        at = 0
        for s, (n, b) in enumerate(zip(lens, blocks)):
            self.tables[s, :b] = perm[at:at + b]
            at += b
            x = kh.f64(kh.rand_bf16(rng, (n, 2, n_kv, hd)))
            x[:, 0, :, hd // 3] *= 5
            store_keys(self.pool, self.tables[s], block, hd, x)

    def keys(self, s, n=None):
        return load_keys(self.pool, self.tables[s], self.lens[s] if n is None else n, self.block, self.hd)


def attend(q, positions, k, v, there, scale, window):
    """kv4.attend a head at a time, and the root of the sum of (weight * v)^2."""
    n, n_q, hd = q.shape
    group = n_q // k.shape[1]
    out, size, spread = (np.zeros((n, n_q, hd)) for _ in range(3))
    lse, reach = np.full((n, n_q), -np.inf), np.zeros((n, n_q))
    j, p = np.arange(len(k)), np.asarray(positions, dtype=np.int64)[:, None]
    seen = there & (j <= p) & ((j > p - window) if window else True)
    some = seen.any(1)
    if not some.any():
        return out, lse, size, reach, spread
    with np.errstate(divide="ignore", invalid="ignore"):
        for h in range(n_q):
            kk, vv = k[:, h // group], v[:, h // group]
            s = np.where(seen, scale * (q[:, h] @ kk.T), -np.inf)[some]
            m = s.max(1, keepdims=True)
            w = np.exp(s - m)
            lse[some, h] = (m + np.log(w.sum(1, keepdims=True)))[:, 0]
            w /= w.sum(1, keepdims=True)
            clean, bad = np.nan_to_num(vv), np.isnan(vv).astype(np.float64)
            out[some, h] = np.where(seen[some].astype(np.float64) @ bad > 0, np.nan, w @ clean)
            size[some, h], spread[some, h] = w @ np.abs(clean), np.sqrt(w ** 2 @ clean ** 2)
            reach[some, h] = np.where(seen, scale * (np.abs(q[:, h]) @ np.nan_to_num(np.abs(kk)).T), 0).max(1)[some]
    return out, lse, size, reach, spread


def rounding_step(x):
    """Half the distance of bf16 numbers at |x|."""
    return 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126))) - 8)


def worst_norm(out, want, spread, size, reach, hd, keys, weights_rounded=True):
    """The error's norm over what it may be, for outputs [rows, hd] of one head.

    The rounding of an output is off by up to 2^-8 of it, that of a weight to bf16 by up to 2^-8 of what the weight adds: if these are
    independent and even within their limits their squares have means of a third of the limits', so the error's norm is about
    2^-8 / sqrt(3) * sqrt(sum of y^2 + sum of (w v)^2), and less by some 0.7 since most numbers are not the smallest of their binade.
    Few rows, whose weights' roundings are shared by all channels, may have all of them near the limit: 4 / sqrt(rows) more, up to the
    limits themselves.  The fp32 sums add what attend_limits allows them without these two roundings."""
    fine = ~np.isnan(want)
    if not fine.any():
        return 0.0
    c = min(1.0, 3 ** -0.5 + 4 / np.sqrt(len(want)))
    rest = kh.attend_limits(size, reach, np.zeros(reach.shape), hd, keys)[0] - size * 2.0 ** -7 * 1.01
    limit = c * 2.0 ** -8 * np.sqrt((want[fine] ** 2).sum() + ((spread[fine] ** 2).sum() if weights_rounded else 0)) + np.sqrt((rest[fine] ** 2).sum())
    return np.sqrt(((out - want)[fine] ** 2).sum()) / max(limit, 1e-300)


class NormCall(Call):
    """A Call whose check goes by norms too: of every context and head, and of the whole."""

    def oracle(self):
        c, parts = self.cache, []
        for s in range(self.n_seq):
            a, b = self.cu[s], self.cu[s + 1]
            if a == b:
                continue
            keys = min(max(self.kv_lens[s], 0), c.tables.shape[1] * c.block)
            parts.append(attend(kh.f64(self.q[a:b]), self.positions[a:b], *load_keys(c.pool, c.tables[s], keys, c.block, c.hd), self.scale, self.window))
        self.answer = [np.concatenate(x) for x in zip(*parts)]
        return self.answer[:4]

    def check(self, flags=0, lse=True, weights_rounded=True):
        out = super().check(flags, lse)
        want, _, size, reach, spread = self.answer
        hd, keys = self.cache.hd, max(self.kv_lens)
        if not weights_rounded:
            # fp32 weights to 2^-17 or better (in two parts), sums in fp32, and one rounding
            soft = kh.attend_limits(size, reach, np.zeros(reach.shape), hd, keys)[0] - size * (2.0 ** -7 - 2.0 ** -17) * 1.01
            fine = ~np.isnan(want)
            err = np.abs(out - want) - rounding_step(np.abs(want) + soft) - soft
            assert err[fine].max() <= 0, f"{(err[fine] > 0).sum()} of {fine.sum()} outputs were not rounded once"
        pieces = [(slice(0, self.n), h) for h in range(self.n_q)] if len(out) == self.n_seq else \
                 [(slice(a, b), h) for a, b in zip(self.cu[:-1], self.cu[1:]) if b > a for h in range(self.n_q)]
        for rows, h in pieces + [(slice(0, self.n), slice(None))]:
            w, o, sp, sz = (x[rows, h].reshape(-1, hd) for x in (want, out, spread, size))
            got = worst_norm(o, w, sp, sz, reach[rows, h].reshape(-1), hd, keys, weights_rounded)
            assert got <= 1, f"rows {rows}, head {h}: an error of {got:.3g} of the limit in norm"
        return out
