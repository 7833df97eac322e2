"""GPU tests of how far single tokens' attention over the 4-bit cache is rounded: once, at the end."""
import numpy as np
import pytest

import kv4_norms as kn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hc():
    import paper_2410_05004_amd as m
    return m


@pytest.mark.parametrize("n_q,n_kv,hd,block", [(4, 4, 64, 16), (8, 2, 128, 16), (14, 2, 64, 32), (5, 5, 128, 64), (16, 2, 128, 32), (4, 2, 256, 16)])
@pytest.mark.parametrize("max_kv", [400, 100000])
def test_single_tokens_are_rounded_once(hc, n_q, n_kv, hd, block, max_kv):
    """Contexts of one key to several hundred, an empty place among them, with all keys in a workgroup and in shares."""
    rng = np.random.default_rng([40, n_q, hd])
    lens = [1, 2, 15, 16, 17, 1, 31, 33, 64, 129, 400]
    kv_lens = lens[:5] + [0] + lens[6:]
    call = kn.NormCall(hc, rng, kn.Cache(rng, lens, n_kv, hd, block), n_q, [1] * len(lens), kv_lens=kv_lens, max_kv=max_kv)
    assert (call.ws.numel() > 0) == (max_kv > 400)
    out = call.check(weights_rounded=False)
    assert np.all(out[5] == 0)


@pytest.mark.parametrize("window", [0, 37])
def test_few_rows_are_rounded_once(hc, window):
    """Two tokens of four heads a KV head, and one of eight: as many rows as the other half of a block takes."""
    rng = np.random.default_rng([41, window])
    for n_q, q_lens in ((8, [2, 1, 2, 0]), (16, [1, 1, 0, 1])):
        cache = kn.Cache(rng, [300, 1, 50, 20], 2, 128, 16)
        kn.NormCall(hc, rng, cache, n_q, q_lens, window=window, pad=8, extra_rows=2).check(weights_rounded=False)
