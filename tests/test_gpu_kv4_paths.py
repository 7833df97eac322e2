"""GPU tests of the attention over the 4-bit cache on every path of its launches, asserted by the library's own account of them: places
for tiles, shares of the keys under a window, workgroups that go over thousands of keys.  Held to norms as well (kv4_norms)."""
import itertools

import numpy as np
import pytest

import gpu_harness as gh
import kv4_harness as kh
import kv4_norms as kn
import oracle.kv4_oracle as kv4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hc():
    import paper_2410_05004_amd as m
    return m


@pytest.fixture(scope="module")
def torch():
    return gh.torch_mod()


SHAPES = [(4, 4, 64, 16), (8, 2, 128, 16), (14, 2, 64, 32), (5, 5, 128, 64), (6, 2, 128, 32)]
# rows of a workgroup (0: the many-row kernel's), whether there is a place for every tile, whether keys are shared
WAYS = {"few": (16, 0, 0), "few-flat": (16, 1, 0), "few-shared": (16, 0, 1), "few-flat-shared": (16, 1, 1),
        "two": (32, 0, 0), "two-flat": (32, 1, 0), "two-shared": (32, 0, 1), "two-flat-shared": (32, 1, 1),
        "many": (0, 0, 0), "many-flat": (0, 1, 0), "many-shared": (0, 0, 1), "many-flat-shared": (0, 1, 1)}


def sizes(hc, way, desc, n_seq, n, window=0):
    """Stated sizes (rows of no context behind the n, queries and keys of the longest context) that lead this way."""
    hd, group = desc.head_dim, desc.n_q_heads // desc.n_kv_heads
    tile = {64: 256, 128: 128, 256: 0}[hd]
    rows, flat, shared = WAYS[way]
    full, two = max(tile, 16) // group, max(1, 32 // group)
    for extra, max_q, max_kv in itertools.product((3, 40 * two, 7 * full, 20 * 1024 // desc.n_q_heads, 512 * tile // desc.n_q_heads),
                                                  (1, two, 2 * two + 1, 40, full, 2 * full), (1000, 4000, 20000, 1 << 20)):
        got = hc.diag_attend_kv4(desc, n_seq, n + extra, max_q, max_kv, window)
        if got[:2] == (rows or tile, flat) and (got[2] > 1) == bool(shared):
            return extra, max_q, max_kv
    raise AssertionError(f"no sizes lead to {way}")


def call_by(way, hc, rng, lens, q_lens, n_q, n_kv, hd, block, window=0, way_window=None, **more):
    """A call that goes this way whatever the contexts' sizes are (under `way_window`, if that is another than its own)."""
    desc = gh.make_desc(hc, n_layers=1, d_model=256, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=hd, block_size=block, rope_style=2)
    extra, max_q, max_kv = sizes(hc, way, desc, len(lens), sum(q_lens), window if way_window is None else way_window)
    return kn.NormCall(hc, rng, kn.Cache(rng, lens, n_kv, hd, block), n_q, q_lens, window=window, max_q=max_q, max_kv=max_kv,
                       extra_rows=extra, **more)


def spoil(call, groups=(), blocks=()):
    """NaN groups (part, context, head, key, group), and pages (context, block) that are none of the pool's."""
    c = call.cache
    for part, s, head, key, group in groups:
        page, slot = c.tables[s, key // c.block], key % c.block
        c.pool[page, head, slot // 16][kv4.places(part, head, slot % 16, c.hd)[2][group]] = 255
    for i, (s, b) in enumerate(blocks):
        c.tables[s, b] = (-1, c.num_pages, 1 << 30)[i % 3]
    call.pool.copy_(kh.dev_u8(c.pool))
    call.d["tab"].copy_(gh.to_dev_i32(c.tables))


# as many rows as this test has go another way than these
NOT_HERE = [("few-flat-shared", n_q) for n_q in (8, 14, 5, 6)] + [("two-flat-shared", 14)]


@pytest.mark.parametrize("way,n_q,n_kv,hd,block", [(way, *s) for s in SHAPES for way in WAYS if (way, s[0]) not in NOT_HERE])
def test_ways(hc, way, n_q, n_kv, hd, block):
    """Contexts of several tiles, of one, of a part of one, of none; then with NaN and without some pages."""
    rng = np.random.default_rng([50, n_q, hd])
    lens, q_lens = [50, 7, 620, 300, 20, 1], [50, 9, 600, 77, 0, 1]
    call = call_by(way, hc, rng, lens, q_lens, n_q, n_kv, hd, block, pad=8, q_extra=16)
    out = call.check()
    assert np.all(out[50:52] == 0)
    spoil(call, [(1, 2, n_kv - 1, 550, 1), (0, 2, 0, 615, 0), (1, 3, 0, 201, hd // 32 - 1), (1, 2, 0, 30, 0)], [(2, 400 // block), (3, 0)])
    out = call.check(flags=hc.HC_DEV_BAD_PAGE)
    assert np.isnan(out).any() and not np.isnan(out).all()


@pytest.mark.parametrize("way", ["two-flat", "two-flat-shared", "many-flat", "many-flat-shared"])
def test_places_for_tiles_in_a_graph(hc, torch, way):
    """Captured once; the lengths of the contexts, and with them their tiles, change between the replays."""
    rng = np.random.default_rng(51)
    call = call_by(way, hc, rng, [700, 90, 400], [300, 3, 40], 8, 2, 128, 16)
    call.check()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call.launch(stream=side.cuda_stream)
    for q_lens in ([300, 3, 40], [1, 90, 252], [0, 0, 343], [343, 0, 0]):
        call.cu = kh.cu_of(q_lens)
        call.positions[:343] = np.concatenate([np.arange(k - q, k) for q, k in zip(q_lens, call.kv_lens)])
        call.d["cu"].copy_(gh.to_dev_i32(call.cu))
        call.d["p"].copy_(gh.to_dev_i32(call.positions))
        call.out.fill_(99)
        call.lse.fill_(99)
        call.ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = call.out.clone(), call.lse.clone()
        call.check()
        assert torch.equal(call.out, got) and torch.equal(call.lse, got_lse)


# A wave looks 64 runs of 16 keys up at once: the tiles of the many-row kernel take 4 of them, those of the other 2 in each of 4 waves, so that
# lookups meet at every 1024th key and at every 4096th, 32 keys further for each wave.
@pytest.mark.parametrize("way,n_q,n_kv,hd,block,lens,q_lens,round", [
    ("many", 8, 2, 128, 16, [2100, 1100, 1024, 1025], [120, 33, 1, 2], 1024), ("many-flat", 2, 2, 64, 32, [3100, 1030], [300, 20], 1024),
    ("few", 8, 2, 128, 16, [8300, 4200, 4096, 4097, 4128], [1, 1, 1, 1, 1], 4096), ("few-flat", 2, 2, 64, 64, [8300, 4200], [40, 3], 4096),
    ("two", 4, 2, 64, 16, [8300, 4250], [30, 9], 4096), ("two-flat", 6, 2, 128, 32, [8300, 4200], [25, 1], 4096)])
@pytest.mark.parametrize("window", [0, 2 ** 31 - 1, 4500])
def test_more_keys_than_are_looked_up_at_once(hc, way, n_q, n_kv, hd, block, lens, q_lens, round, window):
    rng = np.random.default_rng([52, n_q, hd, round])
    call = call_by(way, hc, rng, lens, q_lens, n_q, n_kv, hd, block, window=window)
    call.check()
    # pages missing, and NaN, on both sides of where lookups meet
    blocks = [(s, k // block) for s, n in enumerate(lens) for k in (round - 1, round + 65, 2 * round, 2 * round - 65) if k < n - 100]
    groups = [(1, 0, 0, round - 80, 0), (1, 0, 1, 2 * round + 40, hd // 32 - 1), (1, 1, 0, round + 1, 1)]
    spoil(call, [g for g in groups if g[3] < lens[g[1]] and (g[1], g[3] // block) not in blocks], blocks)
    out = call.check(flags=hc.HC_DEV_BAD_PAGE)
    assert np.isnan(out).any() and not np.isnan(out).all()


SHARED = ["few-shared", "few-flat-shared", "two-shared", "two-flat-shared", "many-shared", "many-flat-shared"]


@pytest.mark.parametrize("way", SHARED)
@pytest.mark.parametrize("window", [9000, 2 ** 31 - 1])
@pytest.mark.parametrize("n_q,n_kv,hd,block", [(4, 2, 64, 16), (8, 2, 128, 32)])
def test_shares_of_a_window(hc, way, n_q, n_kv, hd, block, window):
    """The shares are of the keys that a window leaves."""
    rng = np.random.default_rng([53, hd, window])
    q_lens = [3, 1, 2, 0] if way == "few-shared" else [60, 9, 33, 0]
    call = call_by(way, hc, rng, [11000, 130, 9500, 20], q_lens, n_q, n_kv, hd, block, window=window, pad=8)
    call.check()
    spoil(call, [(1, 0, 1, 10990, 1)], [(0, 5000 // block), (2, 0)])
    call.check(flags=hc.HC_DEV_BAD_PAGE)


@pytest.mark.parametrize("way", SHARED)
@pytest.mark.parametrize("window", [1, 37, 2000])
@pytest.mark.parametrize("n_q,n_kv,hd,block", [(4, 2, 64, 16), (8, 2, 128, 32)])
def test_windows_that_leave_fewer_shares(hc, way, n_q, n_kv, hd, block, window):
    """Calls that would have shares without their window: fewer or none with it, the workspace being that of all keys."""
    rng = np.random.default_rng([56, hd, window])
    q_lens = [3, 1, 2, 0] if way == "few-shared" else [170, 9, 77, 0]
    call = call_by(way, hc, rng, [2600, 130, 2077, 20], q_lens, n_q, n_kv, hd, block, window=window, way_window=0, pad=8)
    assert call.ws.numel() > 0
    call.check()
    spoil(call, [(1, 0, 1, 2590, 1)], [(0, 1500 // block), (2, 0)])
    seen = any(p - window < end and p >= end - block for s, end in ((0, 1500 // block * block + block), (2, block))
               for p in call.positions[call.cu[s]:call.cu[s + 1]])
    call.check(flags=hc.HC_DEV_BAD_PAGE if seen else 0)


@pytest.mark.parametrize("way,n_q,n_kv,hd,lens,q_lens", [
    ("few-shared", 8, 2, 128, [20000, 5000], [1, 1]), ("few-shared", 4, 2, 64, [5000], [3]), ("two-shared", 8, 2, 128, [9000, 3000], [30, 4]),
    ("many-shared", 8, 2, 128, [9000, 500], [120, 32]), ("many-flat-shared", 4, 4, 64, [7000], [300])])
def test_long_contexts(hc, way, n_q, n_kv, hd, lens, q_lens):
    """Outputs of thousands of keys, a sixtieth of one value's size: norms tell what limits per output do not."""
    rng = np.random.default_rng([54, hd, lens[0]])
    call_by(way, hc, rng, lens, q_lens, n_q, n_kv, hd, 16).check()


@pytest.mark.parametrize("way", ["few-flat", "few-flat-shared", "few-shared"])
def test_256_channels(hc, way):
    rng = np.random.default_rng(55)
    call = call_by(way, hc, rng, [4500, 90, 300], [3, 1, 2] if way == "few-shared" else [40, 9, 77], 4, 2, 256, 16, window=0)
    call.check()
    spoil(call, [(1, 0, 1, 4100, 7), (1, 2, 0, 100, 0)], [(0, 255), (2, 3)])
    call.check(flags=hc.HC_DEV_BAD_PAGE)
