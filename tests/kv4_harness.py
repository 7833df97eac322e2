"""Helpers of the tests of the 4-bit cache and of pages as a whole.  (Test infrastructure; not product code.)"""
import numpy as np

import gpu_harness as gh
import oracle.kv4_oracle as kv4
import synthetic as syn


def context(hc, n_q, n_kv, hd, block, n_layers=1, max_position=1 << 20):
    return hc.Context(gh.make_desc(hc, n_layers=n_layers, d_model=256, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=hd,
                                   block_size=block, max_position=max_position, rope_style=2))


def dev_u8(a):
    return gh.torch_mod().from_numpy(np.ascontiguousarray(a)).cuda()


def bits_of(t):
    torch = gh.torch_mod()
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def rand_bf16(rng, shape, scale=1.0):
    """bf16 bit patterns of N(0, scale^2)"""
    return syn.f32_to_bf16_bits(rng.standard_normal(shape, dtype=np.float32) * np.float32(scale))


def f64(bits):
    return syn.bf16_bits_to_f64(bits)


def cu_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


class Cache:
    """A 4-bit pool with random contents in the pages of `lens` contexts; every other byte is 0xFF, whose scales are NaN:
    whatever reads a slot that it should not see gives NaN."""

    def __init__(self, rng, lens, n_kv, hd, block, slack=3, stored=None):
        self.block, self.hd, self.lens = block, hd, list(lens)
        blocks = [-(-n // block) for n in lens]
        self.num_pages = sum(blocks) + slack
        self.pool = np.full((self.num_pages, n_kv, block // 16, 17 * hd), 0xFF, dtype=np.uint8)
        perm = rng.permutation(self.num_pages).astype(np.int32)
        self.tables = np.full((len(lens), max(max(blocks, default=0), 1)), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(blocks):
            self.tables[s, :n] = perm[at:at + n]
            at += n
        self.free = perm[at:]
        for s, n in enumerate(lens):
            x = f64(rand_bf16(rng, (n, 2, n_kv, hd)))
            x[:, 0, :, hd // 3] *= 5
            for j in range(n):
                page = self.tables[s, j // block]
                kv4.store_token(self.pool, page, j % block, x[j, 0], x[j, 1])

    def keys(self, s, n=None):
        return kv4.load_keys(self.pool, self.tables[s], self.lens[s] if n is None else n, self.block, self.hd)


def attend_limits(size, reach, lse, hd, keys):
    """How far outputs and sums may be off.  Keys and values are exact in bf16, and so are products of two bf16 in fp32.
    A score is a sum of hd products: off by at most hd * 2^-24 of the sum of their magnitudes (`reach`, scaled), the
    scaling and the exponent's argument by a few 2^-24 of it more, exp2 by 2^-22 or so: a weight by `weight` of itself.
    It is rounded to bf16 (2^-8 at most); a sum over the keys adds keys * 2^-24 of the sum of magnitudes (`size`); the
    division by the sum of weights, off by the same relative errors, and the rounding to bf16 (2^-8).
    Where all that is left of a sum is smaller than the smallest normal number, 2^-126, it may be zero: a weight when it
    is computed, rounded, scaled down with the running top and joined, 4 * 2^-126 a key of a value below 8 (they are N(0, 1))."""
    weight = (hd + 8) * 2.0 ** -24 * reach + 2.0 ** -20
    more = 2 * weight + 2 * (keys + 64) * 2.0 ** -24
    out = size * (2.0 ** -8 + 2.0 ** -8 + more[..., None]) * 1.01 + 4 * 8 * keys * 2.0 ** -126
    # the logarithm: the sum's relative error, and fp32 roundings of the results of the size of the top score
    log = weight + (keys + 64) * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -21 * np.maximum(reach, np.where(np.isfinite(lse), np.abs(lse), 0))
    return out, log
