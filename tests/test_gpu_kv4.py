"""GPU tests of the 4-bit cache (rows in, rows out) and of the attention over it, against the 64-bit oracle.  Codes and scales have
to be the oracle's to the bit; attention is held to limits worked out from its roundings (kv4_harness.attend_limits)."""
import numpy as np
import pytest

import gpu_harness as gh
import kv4_harness as kh
import oracle.kv4_oracle as kv4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hc():
    import paper_2410_05004_amd as m
    return m


@pytest.fixture(scope="module")
def torch():
    return gh.torch_mod()


def special_rows(rng, n, n_kv, hd):
    """bf16 rows [n, 2, heads, hd]: ordinary values, and in the first rows groups at the edges of the format."""
    bits = kh.rand_bf16(rng, (n, 2, n_kv, hd))
    bits[:, 0, :, 5] = kh.rand_bf16(rng, (n, n_kv), 40)
    edge = [np.zeros(32), np.full(32, -0.0), np.array([7, -7, 6.97, 5, -5, 3.5, 2.5, 1.75, 1.25, .75, .25, -.25] + [0.1] * 20),
            np.full(32, 3.38e38), np.array([1e-38] * 16 + [2e-39] * 16), np.array([2.0 ** -126] * 32), np.array([2.0 ** -133] * 32)]
    for i, g in enumerate(edge[: n]):
        bits[i, i % 2, i % n_kv, 32:64] = kh.syn.f32_to_bf16_bits(g.astype(np.float32))
    if n > 9:
        bits[8, 0, 0, 3], bits[9, 1, n_kv - 1, hd - 1] = 0x7F80, 0xFFC1      # an infinity, a NaN
    return bits


@pytest.mark.parametrize("n_kv,hd,block,lens,starts", [
    (1, 64, 16, [1], [0]), (3, 64, 32, [37, 0, 5], [7, 0, 100]), (2, 128, 16, [50, 1, 16, 33], [3, 15, 16, 0]),
    (8, 128, 64, [70], [63]), (5, 128, 16, [1] * 40, list(range(40))), (2, 256, 16, [19, 30], [16, 1]), (1, 256, 128, [3], [126])])
def test_rows_in_and_out(hc, torch, n_kv, hd, block, lens, starts):
    rng = np.random.default_rng([1, n_kv, hd, block])
    n, n_seq, d_kv = sum(lens), len(lens), n_kv * hd
    blocks = [-(-(a + m) // block) for a, m in zip(starts, lens)]
    num_pages, width = sum(blocks) + 2, max(blocks) + 1
    perm = rng.permutation(num_pages).astype(np.int32)
    tables = np.full((n_seq, width), -1, dtype=np.int32)
    at = 0
    for s, b in enumerate(blocks):
        tables[s, :b] = perm[at:at + b]
        at += b
    pos = np.concatenate([a + rng.permutation(m) for a, m in zip(starts, lens)]).astype(np.int32)
    bits = special_rows(rng, n, n_kv, hd)
    want = rng.integers(0, 256, (num_pages, n_kv, block // 16, 17 * hd)).astype(np.uint8)
    pool = kh.dev_u8(want)
    ctx = kh.context(hc, n_kv, n_kv, hd, block)
    ctx.set_kv4_pool(0, pool, num_pages)
    assert hc.kv4_page_bytes(ctx.desc) * num_pages == pool.numel()
    s = gh.stream_handle()
    d_rows = gh.to_dev_bf16(bits.reshape(n, 2 * d_kv))
    d_pos, d_cu, d_tab = gh.to_dev_i32(pos), gh.to_dev_i32(kh.cu_of(lens)), gh.to_dev_i32(tables)
    ctx.quantize_kv(0, d_rows, d_pos, n, d_cu if n_seq > 1 else None, n_seq, d_tab, width, s)
    assert ctx.poll_device_error(s) == 0
    x, context = kh.f64(bits), np.repeat(np.arange(n_seq), lens)
    values = np.zeros((n, 2, n_kv, hd))
    for i in range(n):
        page, slot = tables[context[i], pos[i] // block], pos[i] % block
        kv4.store_token(want, page, slot, x[i, 0], x[i, 1])
        values[i] = kv4.load_token(want, page, slot, hd)
    assert np.array_equal(pool.cpu().numpy(), want)
    back = torch.zeros((n, 2 * d_kv), dtype=torch.bfloat16, device="cuda")
    ctx.dequantize_kv(0, back, d_pos, n, d_cu, n_seq, d_tab, width, s)
    got = kh.f64(kh.bits_of(back)).reshape(values.shape)
    assert np.array_equal(got, values, equal_nan=True)
    assert np.array_equal(np.signbit(got), np.signbit(values) | np.isnan(got) & np.signbit(got))
    ctx.destroy()


def test_every_bf16_value(hc, torch):
    """All finite patterns as the largest of a group, and beside a largest of 7."""
    bits = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    bits = bits[(bits & 0x7F80) != 0x7F80]
    n = len(bits) // 32
    rows = np.zeros((n, 2, 1, 64), dtype=np.uint16)
    rows[:, 0, 0, 0::2] = bits.reshape(n, 32)
    rows[:, 0, 0, 1] = bits[::32]
    rows[:, 1, 0] = np.repeat(bits.reshape(n, 32)[:, :2], 32, axis=1)
    rows[:, 1, 0, 9] = 0x40E0
    pool = torch.zeros((-(-n // 16), 1, 1, 17 * 64), dtype=torch.uint8, device="cuda")
    ctx = kh.context(hc, 1, 1, 64, 16)
    ctx.set_kv4_pool(0, pool, pool.shape[0])
    tab, pos = gh.to_dev_i32(np.arange(pool.shape[0])), gh.to_dev_i32(np.arange(n))
    ctx.quantize_kv(0, gh.to_dev_bf16(rows.reshape(n, 128)), pos, n, None, 1, tab, pool.shape[0], gh.stream_handle())
    back = torch.zeros((n, 128), dtype=torch.bfloat16, device="cuda")
    ctx.dequantize_kv(0, back, pos, n, None, 1, tab, pool.shape[0], gh.stream_handle())
    want = kv4.dequantize(*kv4.quantize(kh.f64(rows)))
    assert np.array_equal(kh.f64(kh.bits_of(back)), want.reshape(n, 128))
    ctx.destroy()


@pytest.mark.parametrize("n_kv,hd,block,n", [(2, 64, 16, 45), (3, 128, 32, 70), (1, 256, 64, 1)])
def test_pages_in(hc, torch, n_kv, hd, block, n):
    """bf16 pages to 4-bit pages, by tables of their own, from the middle of a page on."""
    rng = np.random.default_rng([2, hd])
    start, blocks = 5, -(-(n + 5) // block)
    t16, t4 = rng.permutation(blocks + 3)[:blocks].astype(np.int32), rng.permutation(blocks + 7)[:blocks].astype(np.int32)
    bits = special_rows(rng, n, n_kv, hd)
    src = gh.new_pool(blocks + 3, block, n_kv, hd)
    want = np.full((blocks + 7, n_kv, block // 16, 17 * hd), 0xA5, dtype=np.uint8)
    pool = kh.dev_u8(want)
    ctx = kh.context(hc, n_kv, n_kv, hd, block)
    ctx.set_kv_pool(0, src, blocks + 3)
    ctx.set_kv4_pool(0, pool, blocks + 7)
    pos = (start + rng.permutation(n)).astype(np.int32)
    s, d_pos = gh.stream_handle(), gh.to_dev_i32(pos)
    d16, d4 = gh.to_dev_i32(t16), gh.to_dev_i32(t4)
    ctx.scatter_kv(0, gh.to_dev_bf16(bits.reshape(n, -1)), d_pos, n, d16, blocks, s)
    ctx.quantize_kv_pages(0, d_pos, n, d16, blocks, d4, blocks, s)
    assert ctx.poll_device_error(s) == 0
    x = kh.f64(bits)
    for i in range(n):
        kv4.store_token(want, t4[pos[i] // block], pos[i] % block, x[i, 0], x[i, 1])
    assert np.array_equal(pool.cpu().numpy(), want)
    # a table that ends early, on either side
    for b16, b4 in ((blocks - 1, blocks), (blocks, blocks - 1)):
        ctx.quantize_kv_pages(0, d_pos, n, d16, b16, d4, b4, s)
        assert ctx.poll_device_error(s) == (hc.HC_DEV_BAD_POSITION if (pos // block == blocks - 1).any() else 0)
        assert np.array_equal(pool.cpu().numpy(), want)
    bad = t16.copy()
    bad[0] = blocks + 3
    ctx.quantize_kv_pages(0, d_pos, n, gh.to_dev_i32(bad), blocks, d4, blocks, s)
    assert ctx.poll_device_error(s) == (hc.HC_DEV_BAD_PAGE if (pos < block).any() else 0)
    assert np.array_equal(pool.cpu().numpy(), want)
    ctx.destroy()


def test_rows_without_a_place(hc, torch):
    """Bad positions and pages, and rows of no context, are skipped and flagged; their neighbours are stored."""
    n_kv, hd, block = 2, 128, 16
    rng = np.random.default_rng(3)
    tables = np.array([[4, -1, 2], [0, 9, 1]], dtype=np.int32)
    lens = [20, 8]                                         # 28 of 30 rows
    pos = np.concatenate([rng.permutation(48)[:20], rng.permutation(48)[:8], [3, 4]]).astype(np.int32)
    pos[0], pos[3], pos[21] = -1, 48, 1 << 20
    bits = kh.rand_bf16(rng, (30, 2, n_kv, hd))
    want = np.full((5, n_kv, 1, 17 * hd), 0x5A, dtype=np.uint8)
    pool = kh.dev_u8(want)
    ctx = kh.context(hc, n_kv, n_kv, hd, block)
    ctx.set_kv4_pool(0, pool, 5)
    s = gh.stream_handle()
    d_pos, d_cu, d_tab = gh.to_dev_i32(pos), gh.to_dev_i32(kh.cu_of(lens)), gh.to_dev_i32(tables)
    ctx.quantize_kv(0, gh.to_dev_bf16(bits.reshape(30, -1)), d_pos, 30, d_cu, 2, d_tab, 3, s)
    assert ctx.poll_device_error(s) == (hc.HC_DEV_BAD_POSITION | hc.HC_DEV_BAD_PAGE)
    x, good = kh.f64(bits), []
    for i in range(28):
        row = tables[0 if i < 20 else 1]
        if 0 <= pos[i] < 48 and 0 <= row[pos[i] // block] < 5:
            good.append(i)
            kv4.store_token(want, row[pos[i] // block], pos[i] % block, x[i, 0], x[i, 1])
    assert 5 < len(good) < 25
    assert np.array_equal(pool.cpu().numpy(), want)
    back = torch.full((30, 2 * n_kv * hd), 77.0, dtype=torch.bfloat16, device="cuda")
    ctx.dequantize_kv(0, back, d_pos, 30, d_cu, 2, d_tab, 3, s)
    assert ctx.poll_device_error(s) == (hc.HC_DEV_BAD_POSITION | hc.HC_DEV_BAD_PAGE)
    left = np.ones(30, dtype=bool)
    left[good] = False
    got = kh.f64(kh.bits_of(back))
    assert np.all(got[left] == 77) and np.array_equal(got[~left].reshape(-1, 2, n_kv, hd), kv4.dequantize(*kv4.quantize(x[~left])))
    ctx.destroy()


# ---- attention -----------------------------------------------------------------------------
class Call:
    """One call of the attention and the oracle's answer."""

    def __init__(self, hc, rng, cache, n_q, q_lens, positions=None, window=0, scale=None, pad=0, q_extra=0, extra_rows=0, max_q=None, max_kv=None,
                 kv_lens=None, layer_ctx=None, q_scale=1.0):
        torch = gh.torch_mod()
        self.hc, self.cache, self.n_q, self.window = hc, cache, n_q, window
        hd, n_seq = cache.hd, len(q_lens)
        self.n, self.rows = sum(q_lens), sum(q_lens) + extra_rows
        self.kv_lens = list(cache.lens if kv_lens is None else kv_lens)
        self.scale = float(np.float32(hd ** -0.5 if scale is None else scale))
        if positions is None:
            positions = np.concatenate([np.arange(k - q, k) for q, k in zip(q_lens, self.kv_lens)] or [np.zeros(0)])
        self.positions = np.concatenate([positions, np.full(extra_rows, 5)]).astype(np.int32)
        self.cu = kh.cu_of(q_lens)
        self.q = kh.rand_bf16(rng, (self.rows, n_q, hd), q_scale)
        width = n_q * hd
        big = np.full((self.rows, width + q_extra), 0x7FC1, dtype=np.uint16)
        big[:, :width] = self.q.reshape(self.rows, width)
        self.d_q, self.q_stride = gh.to_dev_bf16(big), width + q_extra
        self.out = torch.full((self.rows, width + pad), 99.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((self.rows, n_q), 99.0, dtype=torch.float32, device="cuda")
        self.ctx = layer_ctx or kh.context(hc, n_q, cache.pool.shape[1], hd, cache.block)
        self.pool = kh.dev_u8(cache.pool)
        self.d = dict(p=gh.to_dev_i32(self.positions), cu=gh.to_dev_i32(self.cu), kv=gh.to_dev_i32(self.kv_lens), tab=gh.to_dev_i32(cache.tables))
        self.n_seq, self.max_q, self.max_kv = n_seq, max(q_lens) if max_q is None else max_q, max(self.kv_lens) if max_kv is None else max_kv
        self.ctx.set_kv4_pool(0, self.pool, cache.num_pages)
        size = hc.attend_kv4_workspace(self.ctx.desc, n_seq, self.rows, self.max_q, self.max_kv)
        self.ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")

    def launch(self, lse=True, stream=None):
        self.ctx.attend_kv4(0, self.d_q, self.q_stride, self.d["p"], self.rows, self.d["cu"], self.d["kv"], self.n_seq, self.max_q, self.max_kv,
                            self.d["tab"], self.cache.tables.shape[1], self.scale, self.window, self.out, self.out.shape[1],
                            self.lse if lse else None, self.ws if self.ws.numel() else None, self.ws.numel(),
                            gh.stream_handle() if stream is None else stream)

    def oracle(self):
        c = self.cache
        parts = []
        for s in range(self.n_seq):
            a, b = self.cu[s], self.cu[s + 1]
            keys = min(max(self.kv_lens[s], 0), c.tables.shape[1] * c.block)
            parts.append(kv4.attend(kh.f64(self.q[a:b]), self.positions[a:b], *c.keys(s, keys), self.scale, self.window))
        return [np.concatenate(x) for x in zip(*parts)]

    def check(self, flags=0, lse=True):
        self.launch(lse)
        assert self.ctx.poll_device_error(gh.stream_handle()) == flags
        n, hd, width = self.n, self.cache.hd, self.n_q * self.cache.hd
        out = self.out.double().cpu().numpy()
        got_lse = self.lse.double().cpu().numpy()
        assert np.all(out[:, width:] == 99) and np.all(out[n:] == 99) and np.all(got_lse[n:] == 99), "written where nothing belongs"
        out = out[:n, :width].reshape(n, self.n_q, hd)
        want, want_lse, size, reach = self.oracle()
        tol, tol_lse = kh.attend_limits(size, reach, want_lse, hd, max(self.kv_lens))
        assert np.array_equal(np.isnan(out), np.isnan(want)), "NaN in other places than the oracle's"
        fine = ~np.isnan(want)
        err = np.abs(out - want)[fine] - tol[fine]
        assert not err.size or err.max() <= 0, f"{(err > 0).sum()} outputs too far off, by up to {err.max():.3g}"
        if lse:
            seen = np.isfinite(want_lse)
            assert np.array_equal(got_lse[:n][~seen], want_lse[~seen], equal_nan=True)
            bad = np.abs(got_lse[:n][seen] - want_lse[seen]) - tol_lse[seen]
            assert not bad.size or bad.max() <= 0, f"sums too far off, by up to {bad.max():.3g}"
        else:
            assert np.all(got_lse == 99)
        return out


LAYOUTS = [(4, 4, 64, 16), (8, 2, 128, 16), (14, 2, 64, 32), (5, 5, 128, 64), (16, 2, 128, 32), (4, 2, 256, 16), (34, 1, 64, 16)]


@pytest.mark.parametrize("n_q,n_kv,hd,block", LAYOUTS)
def test_single_tokens(hc, n_q, n_kv, hd, block):
    """A decoding step: contexts of one key to several hundred, an empty place among them."""
    rng = np.random.default_rng([10, n_q, hd])
    lens = [1, 2, 15, 16, 17, 0, 31, 33, 64, 129, 400]
    Call(hc, rng, kh.Cache(rng, lens, n_kv, hd, block), n_q, [1] * len(lens)).check()


@pytest.mark.parametrize("n_q,n_kv,hd,block", LAYOUTS)
@pytest.mark.parametrize("window", [0, 1, 37])
def test_prompts(hc, n_q, n_kv, hd, block, window):
    """Prompts on histories, ragged: one token, a few, more than the context has (the first then see nothing), none."""
    rng = np.random.default_rng([11, n_q, hd, window])
    lens, q_lens = [50, 7, 130, 300, 20], [50, 9, 1, 77, 0]
    out = Call(hc, rng, kh.Cache(rng, lens, n_kv, hd, block), n_q, q_lens, window=window, pad=8, q_extra=16, extra_rows=3).check()
    assert np.all(out[50:52] == 0)


@pytest.mark.parametrize("max_q,max_kv", [(1, 1), (500, 100000), (40, 5000)])
def test_hints_do_not_matter(hc, max_q, max_kv):
    rng = np.random.default_rng(12)
    Call(hc, rng, kh.Cache(rng, [700, 3, 90], 2, 64, 16), 4, [40, 3, 1], max_q=max_q, max_kv=max_kv).check()


def test_positions_in_any_order(hc):
    """Positions that repeat, lie beyond the keys or before the first, and a mask that leaves a row of one key."""
    rng = np.random.default_rng(13)
    pos = np.array([5, 2 ** 31 - 1, -1, 99, 0, 5, 100, 40, -2 ** 31, 63, 62, 64, 98, 1])
    for window in (0, 1, 20, 2 ** 31 - 1):
        out = Call(hc, rng, kh.Cache(rng, [100], 2, 128, 16), 4, [14], positions=pos, window=window).check()
        assert np.all(out[[2, 8]] == 0)
        assert np.all(out[1] == 0) == (0 < window < 2 ** 31 - 1)


def test_large_scores(hc):
    """Scores of hundreds: weights of one key, sums that would overflow without the running top."""
    rng = np.random.default_rng(14)
    Call(hc, rng, kh.Cache(rng, [333, 40], 2, 128, 16), 8, [20, 40], scale=3.0, q_scale=4.0).check()
    Call(hc, rng, kh.Cache(rng, [333], 2, 64, 16), 4, [1], scale=1e-30).check()


def test_without_sums(hc):
    rng = np.random.default_rng(15)
    Call(hc, rng, kh.Cache(rng, [333, 40], 2, 128, 16), 8, [1, 1]).check(lse=False)
    Call(hc, rng, kh.Cache(rng, [9000 // 8], 1, 64, 16), 8, [1], max_kv=100000).check(lse=False)


def test_pages_that_are_missing(hc):
    """Entries outside the pool, and key counts that the table has no room for: unseen, flagged, nothing read out of place.  Missing
    pages in front of a window are none of anybody's business."""
    rng = np.random.default_rng(16)
    cache = kh.Cache(rng, [100, 70], 2, 64, 16)
    cache.tables[0, 2], cache.tables[0, 5], cache.tables[1, 0] = -1, cache.num_pages, 1 << 30
    Call(hc, rng, cache, 4, [30, 1]).check(flags=hc.HC_DEV_BAD_PAGE)
    Call(hc, rng, cache, 4, [1, 1], window=4).check()
    cache = kh.Cache(rng, [112, 70], 2, 64, 16)
    Call(hc, rng, cache, 4, [3, 2], positions=np.array([111, 500, 60, 69, 3]), kv_lens=[2 ** 31 - 1, -5]).check(flags=hc.HC_DEV_BAD_POSITION)


@pytest.mark.parametrize("n_q,n_kv,hd,q_len", [(2, 2, 64, 1), (4, 2, 128, 1), (4, 2, 128, 40), (4, 1, 256, 40), (2, 2, 64, 40)])
def test_nan_where_it_is_seen(hc, n_q, n_kv, hd, q_len):
    """A key's or a value's group that is NaN: the rows that see it get NaN (of a value: in its channels), all others do not."""
    rng = np.random.default_rng([17, hd, q_len])
    cache = kh.Cache(rng, [100], n_kv, hd, 16)
    for part, head, key, group in ((1, n_kv - 1, 80, 1), (1, 0, 61, hd // 32 - 1), (0, 0, 95, 0)):
        page, slot = cache.tables[0, key // 16], key % 16
        cache.pool[page, head, 0][kv4.places(part, head, slot, hd)[2][group]] = 255
    for window in (0, 8):
        out = Call(hc, rng, cache, n_q, [q_len], window=window).check()
        assert np.isnan(out).any() and not np.isnan(out).all()


def test_far_pages(hc, torch):
    """Pages beyond 4 GiB into a pool."""
    n_q, n_kv, hd, block = 16, 8, 128, 16
    rng = np.random.default_rng(18)
    cache = kh.Cache(rng, [60, 33], n_kv, hd, block)
    far = 2 ** 32 // (n_kv * 17 * hd) + 1000
    pool = torch.empty((far + cache.num_pages, n_kv, 1, 17 * hd), dtype=torch.uint8, device="cuda")
    pool[far:] = kh.dev_u8(cache.pool)
    call = Call(hc, rng, cache, n_q, [20, 1])
    call.pool = pool
    call.ctx.set_kv4_pool(0, pool, far + cache.num_pages)
    call.d["tab"] = gh.to_dev_i32(np.where(cache.tables >= 0, cache.tables + far, -1))
    call.check()
    # and rows written and read there
    rows = kh.rand_bf16(rng, (60, 2 * n_kv * hd))
    d_rows, pos, tab = gh.to_dev_bf16(rows), gh.to_dev_i32(np.arange(60)), call.d["tab"]
    call.ctx.quantize_kv(0, d_rows, pos, 60, None, 1, tab, cache.tables.shape[1], gh.stream_handle())
    back = torch.zeros_like(d_rows)
    call.ctx.dequantize_kv(0, back, pos, 60, None, 1, tab, cache.tables.shape[1], gh.stream_handle())
    want = kv4.dequantize(*kv4.quantize(kh.f64(rows).reshape(60, 2, n_kv, hd)))
    assert np.array_equal(kh.f64(kh.bits_of(back)).reshape(want.shape), want)


@pytest.mark.parametrize("lens,q_lens", [([700, 90, 1, 300], [1, 1, 1, 1]), ([600], [600]), ([5000], [3])])
def test_same_result_every_time_and_in_a_graph(hc, torch, lens, q_lens):
    """Repeated calls, calls on another stream and replays of a captured one give the same bits; the graph has a workspace of its own."""
    rng = np.random.default_rng([19, len(lens)])
    call = Call(hc, rng, kh.Cache(rng, lens, 2, 64, 16), 4, q_lens)
    call.launch()
    torch.cuda.synchronize()
    want, want_lse = call.out.clone(), call.lse.clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    own, call.ws = call.ws, call.ws.clone()
    with torch.cuda.graph(graph, stream=side):
        call.launch(stream=side.cuda_stream)
    graph_ws, call.ws = call.ws, own
    for i in range(4):
        call.out.fill_(99)
        call.lse.fill_(99)
        torch.cuda.synchronize()
        if i % 2:
            graph.replay()
        else:
            call.launch(stream=side.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(call.out, want) and torch.equal(call.lse, want_lse)
        call.ws.fill_(255)
        graph_ws.fill_(255)
    # new lengths and positions on the device: the graph follows them
    call.kv_lens = [max(1, n - 20) for n in call.kv_lens]
    call.d["kv"].copy_(gh.to_dev_i32(call.kv_lens))
    call.d["p"].copy_(call.d["p"] - 20)
    call.positions = call.positions - 20
    graph.replay()
    torch.cuda.synchronize()
    got, got_lse = call.out.clone(), call.lse.clone()
    call.check()
    assert torch.equal(call.out, got) and torch.equal(call.lse, got_lse)


def test_two_at_once(hc, torch):
    """Two calls of one context on two streams, each with its workspace."""
    rng = np.random.default_rng(20)
    calls = [Call(hc, rng, kh.Cache(rng, [900, 80 + 50 * i], 2, 128, 16), 8, [1, 1]) for i in range(2)]
    want = []
    for c in calls:
        c.check()
        want.append((c.out.clone(), c.lse.clone()))
    ctx = calls[0].ctx
    calls[1].ctx = ctx
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for c, st in zip(calls, streams):
            ctx.set_kv4_pool(0, c.pool, c.cache.num_pages)
            c.launch(stream=st.cuda_stream)
    torch.cuda.synchronize()
    for c, (o, l) in zip(calls, want):
        assert torch.equal(c.out, o) and torch.equal(c.lse, l)


# ---- every way that sizes lead to: a workgroup of 16 rows, of 32, of 128 or 256, each with all of the keys or a share of them.  The sizes
# that a caller states are upper bounds; stated wider than they are, they lead small contexts there too.
WAYS = ["few", "few-flat", "few-shared", "few-halved", "two", "two-shared", "many", "many-shared"]
SHAPES = [(4, 4, 64, 16), (8, 2, 128, 16), (14, 2, 64, 32), (5, 5, 128, 64), (34, 1, 64, 16), (6, 2, 128, 32)]


def call_by(way, hc, rng, lens, q_lens, n_q, n_kv, hd, block, extra_rows=0, **more):
    group, tile = n_q // n_kv, 256 if hd == 64 else 128
    # empty contexts and rows of none, queries of the longest, keys of the longest
    full, two = tile // group, max(1, 32 // group)
    empty, padding, max_q, max_kv = {
        "few": (0, 0, 1, 1), "few-flat": (0, 0, 64, 300), "few-shared": (0, 0, 1, 4000), "few-halved": (-(-150 // n_kv), 0, 1, 4000),
        "two": (0, 20 * 1024 // n_q, two, 1270), "two-shared": (0, 0, two, 1 << 20),
        "many": (0, 512 * tile // n_q, full, 1000), "many-shared": (0, 7 * full, full, 1 << 20)}[way]
    none = [0] * empty
    return Call(hc, rng, kh.Cache(rng, lens + none, n_kv, hd, block), n_q, q_lens + none, max_q=more.pop("max_q", max_q), max_kv=max_kv,
                extra_rows=max(padding, extra_rows), **more)


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("n_q,n_kv,hd,block", SHAPES)
def test_ways(hc, way, n_q, n_kv, hd, block):
    rng = np.random.default_rng([21, n_q, hd])
    lens, q_lens = [50, 7, 130, 300, 20, 1], [50, 9, 1, 77, 0, 1]
    call = call_by(way, hc, rng, lens, q_lens, n_q, n_kv, hd, block, pad=8, q_extra=16, extra_rows=3)
    assert (call.ws.numel() > 0) == (way.endswith("shared") or way == "few-halved")
    out = call.check()
    assert np.all(out[50:52] == 0)


@pytest.mark.parametrize("window", [1, 37, 2 ** 31 - 1])
@pytest.mark.parametrize("n_q,n_kv,hd,block", SHAPES)
def test_windows_of_many_rows(hc, n_q, n_kv, hd, block, window):
    rng = np.random.default_rng([22, n_q, hd, window])
    call_by("many", hc, rng, [50, 7, 130, 500, 20], [50, 9, 1, 300, 0], n_q, n_kv, hd, block, window=window).check()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("n_q,n_kv,hd,block", [(2, 2, 64, 16), (4, 2, 128, 16)])
def test_ways_with_nan_and_missing_pages(hc, way, n_q, n_kv, hd, block):
    rng = np.random.default_rng([23, hd])
    call = call_by(way, hc, rng, [100, 300], [40, 200], n_q, n_kv, hd, block)
    cache = call.cache
    for part, s, head, key, group in ((1, 0, n_kv - 1, 80, 1), (1, 1, 0, 261, hd // 32 - 1), (0, 1, 0, 295, 0), (1, 1, 1, 101, 0)):
        page, slot = cache.tables[s, key // 16], key % 16
        cache.pool[page, head, 0][kv4.places(part, head, slot, hd)[2][group]] = 255
    call.pool.copy_(kh.dev_u8(cache.pool))
    out = call.check()
    assert np.isnan(out).any() and not np.isnan(out).all()
    cache.tables[0, 2], cache.tables[1, 15], cache.tables[1, 0] = -1, cache.num_pages, 1 << 30
    call.d["tab"].copy_(gh.to_dev_i32(cache.tables))
    call.check(flags=hc.HC_DEV_BAD_PAGE)


@pytest.mark.parametrize("way", WAYS)
def test_ways_with_positions_in_any_order(hc, way):
    rng = np.random.default_rng(24)
    pos = np.concatenate([[5, 2 ** 31 - 1, -1, 299, 0, 5, 300, 40, -2 ** 31, 63, 62, 64, 298, 1], rng.integers(-5, 320, 186)])
    for scale, q_scale in ((None, 1.0), (3.0, 4.0)):
        out = call_by(way, hc, rng, [300], [200], 4, 2, 128, 16, positions=pos, scale=scale, q_scale=q_scale).check()
        assert np.all(out[[2, 8]] == 0)


@pytest.mark.parametrize("way", WAYS)
def test_ways_in_a_graph(hc, torch, way):
    rng = np.random.default_rng(25)
    call = call_by(way, hc, rng, [700, 90], [300, 3], 8, 2, 128, 16)
    call.check()
    want = call.out.clone()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call.launch(stream=side.cuda_stream)
    for _ in range(3):
        call.out.fill_(99)
        call.ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(call.out, want)


@pytest.mark.parametrize("way", WAYS)
def test_queries_that_are_not_finite(hc, torch, way):
    """An infinity or a NaN among a query's channels: that row and head is NaN, all others are what they were."""
    rng = np.random.default_rng(26)
    call = call_by(way, hc, rng, [100, 300], [40, 70], 8, 2, 128, 16)
    call.check()
    want, want_lse = call.out.clone(), call.lse.clone()
    width = 8 * 128
    bad = [(3, 1, 0x7F80), (39, 7, 0x7FC0), (40, 0, 0xFF80), (80, 4, 0xFFC1), (109, 5, 0x7F80)]
    for row, head, bits in bad:
        call.d_q.view(torch.int16)[row, head * 128 + 11] = bits - 65536 if bits >= 32768 else bits
    call.launch()
    out, lse = call.out[:, :width].reshape(-1, 8, 128), call.lse
    for row, head, _ in bad:
        assert torch.isnan(out[row, head]).all() and torch.isnan(lse[row, head])
        out[row, head], lse[row, head] = want[:, :width].reshape(-1, 8, 128)[row, head], want_lse[row, head]
    assert torch.equal(call.out, want) and torch.equal(call.lse, want_lse)


@pytest.mark.parametrize("n_seq,longest", [(65, 40), (1000, 200), (5000, 64), (4097, 0)])
def test_many_contexts(hc, n_seq, longest):
    """Mostly single tokens, places without any, and a prompt among them: every context finds its tiles."""
    rng = np.random.default_rng([27, n_seq])
    q_lens = rng.integers(0, 3, n_seq)
    q_lens[n_seq // 3] = longest
    q_lens[-1] = 5
    lens = q_lens + rng.integers(0, 4, n_seq)
    Call(hc, rng, kh.Cache(rng, lens.tolist(), 1, 64, 16), 4, q_lens.tolist()).check()


def test_more_contexts_than_one_dimension_has_places(hc):
    """A place a context, up to four queries: 40000 of them, the last ones beyond 32768."""
    rng = np.random.default_rng(28)
    q_lens = rng.integers(0, 5, 40000) * (rng.random(40000) < 0.2)
    q_lens[[0, 32767, 32768, 39999]] = [1, 2, 3, 4]
    lens = q_lens + rng.integers(0, 2, 40000) * (q_lens > 0)
    Call(hc, rng, kh.Cache(rng, lens.tolist(), 1, 64, 16), 4, q_lens.tolist()).check()


@pytest.mark.parametrize("way", ["few", "few-flat", "few-shared", "few-halved", "many", "many-shared"])
@pytest.mark.parametrize("n_q,n_kv", [(4, 2), (3, 3), (20, 1)])
def test_ways_of_256_channels(hc, way, n_q, n_kv):
    """Heads that take the same rows to a workgroup whatever their number: whole, with shares joined by four groups or by sixteen."""
    rng = np.random.default_rng([29, n_q])
    lens, q_lens = [50, 7, 130, 300, 20, 1], [50, 9, 1, 77, 0, 1]
    call = call_by(way, hc, rng, lens, q_lens, n_q, n_kv, 256, 16, pad=8, q_extra=16, extra_rows=3)
    call.check()
    cache = call.cache
    for part, s, head, key, group in ((1, 0, n_kv - 1, 30, 7), (0, 3, 0, 295, 3), (1, 3, 0, 261, 0)):
        page, slot = cache.tables[s, key // 16], key % 16
        cache.pool[page, head, 0][kv4.places(part, head, slot, 256)[2][group]] = 255
    cache.tables[2, 3] = -1
    call.pool.copy_(kh.dev_u8(cache.pool))
    call.d["tab"].copy_(gh.to_dev_i32(cache.tables))
    out = call.check(flags=hc.HC_DEV_BAD_PAGE)
    assert np.isnan(out).any() and not np.isnan(out).all()
