"""The norms that attention over the 4-bit cache is held to: what they let pass and what they do not, with mistakes planted in the
oracle.  No GPU."""
import numpy as np
import pytest

import kv4_harness as kh
import kv4_norms as kn
import oracle.kv4_oracle as kv4


def bf16(x):
    step = 2 * kn.rounding_step(x)
    return np.round(x / step) * step


def rounded_attention(q, positions, k, v, there, scale):
    """The oracle's attention with weights rounded to bf16 for the product with the values, and the outputs."""
    out = np.zeros(q.shape)
    group = q.shape[1] // k.shape[1]
    for i, p in enumerate(positions):
        seen = there & (np.arange(len(k)) <= p)
        for h in range(q.shape[1]):
            s = scale * (k[seen, h // group] @ q[i, h])
            w = np.exp(s - s.max())
            out[i, h] = bf16((bf16(w) @ v[seen, h // group]) / w.sum())
    return out


@pytest.mark.parametrize("keys,queries", [(5000, 3), (700, 20), (40, 40)])
def test_norms_see_values_from_a_wrong_place(keys, queries):
    """Sixteen values, a whole run of the cache, from another place."""
    rng = np.random.default_rng([60, keys])
    hd, n_q, n_kv, scale = 64, 4, 2, 0.125
    cache = kn.Cache(rng, [keys], n_kv, hd, 16)
    k, v, there = cache.keys(0)
    q = kh.f64(kh.rand_bf16(rng, (queries, n_q, hd)))
    pos = np.arange(keys - queries, keys)
    want, lse, size, reach, spread = kn.attend(q, pos, k, v, there, scale, 0)
    limits = kh.attend_limits(size, reach, lse, hd, keys)[0]

    def worst(got):
        return max(kn.worst_norm(got[:, h], want[:, h], spread[:, h], size[:, h], reach[:, h], hd, keys) for h in range(n_q))
    right = rounded_attention(q, pos, k, v, there, scale)
    assert np.all(np.abs(right - want) <= limits) and worst(right) <= 0.85
    for at in range(0, keys - 32, max(32, (keys - 32) // 128 * 16)):
        wrong = v.copy()
        wrong[at + 16:at + 32] = v[at:at + 16]
        assert worst(rounded_attention(q, pos, k, wrong, there, scale)) > 1, at


def test_caches_and_attention_at_once_are_the_oracle_s():
    for hd, block in ((64, 16), (128, 32), (256, 64)):
        rng = np.random.default_rng([61, hd])
        slow = kh.Cache(rng, [50, 33], 2, hd, block)
        pool = np.full_like(slow.pool, 0xFF)
        for s, n in enumerate(slow.lens):
            k, v, there = slow.keys(s)
            kn.store_keys(pool, slow.tables[s], block, hd, np.stack([k, v], 1))
            for got, want in zip(kn.load_keys(slow.pool, slow.tables[s], n + 40, block, hd), kv4.load_keys(slow.pool, slow.tables[s], n + 40, block, hd)):
                assert np.array_equal(got, want, equal_nan=True)
            for got, want in zip(kn.load_keys(pool, slow.tables[s], n, block, hd), (k, v, there)):
                assert np.array_equal(got, want)
            q, pos = kh.f64(kh.rand_bf16(rng, (9, 4, hd))), np.array([3, -1, 1000, 5, 0, 20, 31, 32, 9])
            for window in (0, 4):
                for got, want in zip(kn.attend(q, pos, k, v, there, 0.1, window), kv4.attend(q, pos, k, v, there, 0.1, window)):
                    assert np.allclose(got, want, rtol=1e-12, atol=1e-15)
