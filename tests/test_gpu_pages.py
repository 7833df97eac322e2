"""GPU tests of forking contexts and compacting a cache, against the oracle: bytes, so everything has to be equal."""
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


class Pools:
    """Pools of random bytes, as the device and the host have them."""

    def __init__(self, hc, rng, which, layers, num_pages, n_kv, hd, block):
        self.hc, self.which, self.block, self.num_pages = hc, which, block, num_pages
        self.ctx = kh.context(hc, n_kv, n_kv, hd, block, n_layers=layers)
        self.kv, self.kv4, self.d_kv, self.d_kv4 = [], [], [], []
        for l in range(layers):
            if which & hc.HC_POOL_KV:
                self.kv.append(rng.integers(0, 1 << 16, (num_pages, 2, block, n_kv, hd)).astype(np.uint16))
                self.d_kv.append(gh.to_dev_bf16(self.kv[-1]))
                self.ctx.set_kv_pool(l, self.d_kv[-1], num_pages)
            if which & hc.HC_POOL_KV4:
                self.kv4.append(rng.integers(0, 256, (num_pages, n_kv, block // 16, 17 * hd)).astype(np.uint8))
                self.d_kv4.append(kh.dev_u8(self.kv4[-1]))
                self.ctx.set_kv4_pool(l, self.d_kv4[-1], num_pages)

    def copy(self, src, dst, tokens=None):
        """A page, or of it the tokens in use, in every pool."""
        for p in self.kv:
            p[dst, :, :tokens] = p[src, :, :tokens]
        for p in self.kv4:
            n = None if tokens is None else -(-tokens // 16)
            p[dst, :, :n] = p[src, :, :n]

    def check(self):
        for d, p in zip(self.d_kv, self.kv):
            assert np.array_equal(kh.bits_of(d), p)
        for d, p in zip(self.d_kv4, self.kv4):
            assert np.array_equal(d.cpu().numpy(), p)


@pytest.mark.parametrize("which", [1, 2, 3])
@pytest.mark.parametrize("layers,n_kv,hd,block,forks", [(1, 1, 64, 16, 1), (3, 2, 128, 32, 7), (2, 3, 64, 64, 70), (65, 1, 64, 16, 5), (2, 1, 256, 16, 3)])
def test_fork(hc, torch, which, layers, n_kv, hd, block, forks):
    rng = np.random.default_rng([30, which, layers, forks])
    parents, width = 3, 5
    num_pages = parents * width + forks + 4
    perm = rng.permutation(num_pages).astype(np.int32)
    tables = np.full((parents + forks + 1, width), -7, dtype=np.int32)
    tables[:parents] = perm[: parents * width].reshape(parents, width)
    pools = Pools(hc, rng, which, layers, num_pages, n_kv, hd, block)
    src = rng.integers(0, parents, forks).astype(np.int32)
    dst = (parents + rng.permutation(forks)).astype(np.int32)
    n_tok = rng.integers(0, width * block + 1, forks).astype(np.int32)
    n_tok[0] = width * block - 1
    n_tok[1:4] = [0, width * block, block][: len(n_tok[1:4])]
    new = np.where(n_tok % block, perm[parents * width: parents * width + forks], -1).astype(np.int32)
    d_tab, s = gh.to_dev_i32(tables), gh.stream_handle()
    pools.ctx.fork_pages(which, d_tab, len(tables), width, src, dst, n_tok, new, s)
    assert pools.ctx.poll_device_error(s) == 0
    copied = []
    want = kv4.fork(tables, copied, src, dst, n_tok, new, block)
    for a, b, n in copied:
        pools.copy(a, b, n)
    assert np.array_equal(d_tab.cpu().numpy(), want)
    pools.check()
    pools.ctx.destroy()


def test_fork_without_a_page_to_copy(hc):
    """Sources whose last page is missing, or is the new page: -1 and a flag; the other forks of the call are made."""
    rng = np.random.default_rng(31)
    pools = Pools(hc, rng, 3, 2, 12, 1, 64, 16)
    tables = np.array([[0, 1, -1, 3], [4, 50, 6, 7]] + [[-9] * 4] * 5, dtype=np.int32)
    d_tab, s = gh.to_dev_i32(tables), gh.stream_handle()
    args = ([0, 1, 0, 1, 0], [2, 3, 4, 5, 6], [40, 20, 20, 33, 16], [8, 9, 10, 6, -1])
    pools.ctx.fork_pages(3, d_tab, 7, 4, *args, s)
    assert pools.ctx.poll_device_error(s) == hc.HC_DEV_BAD_PAGE
    pools.copy(1, 10, 4)
    assert d_tab.cpu().numpy().tolist() == tables[:2].tolist() + [[0, 1, -1, -1], [4, -1, -1, -1], [0, 10, -1, -1], [4, 50, -1, -1], [0, -1, -1, -1]]
    pools.check()
    pools.ctx.fork_pages(3, d_tab, 7, 4, [], [], [], [], s)
    pools.ctx.destroy()


def check_compact(hc, torch, pools, tables, flags=0, in_place=False, times=1):
    d_in = gh.to_dev_i32(tables)
    d_out = d_in if in_place else gh.to_dev_i32(np.full(tables.shape, 55))
    plan = torch.full((2 + 2 * pools.num_pages,), 1234567, dtype=torch.int32, device="cuda")
    s = gh.stream_handle()
    for _ in range(times):
        pools.ctx.compact_pages(pools.which, d_in, d_out, tables.shape[0], tables.shape[1], plan, s)
    assert pools.ctx.poll_device_error(s) == flags
    want, live, moves, place = kv4.compact(tables, pools.num_pages)
    for a, b in moves:
        pools.copy(a, b)
    got = plan.cpu().numpy()
    assert (got[0], got[1]) == (live, len(moves))
    assert np.array_equal(got[2:2 + pools.num_pages], place)
    assert got[2 + pools.num_pages:][: 2 * len(moves)].reshape(-1, 2).tolist() == [list(m) for m in moves]
    assert np.all(got[2 + pools.num_pages + 2 * len(moves):] == 1234567)
    assert np.array_equal(d_out.cpu().numpy(), want)
    if not in_place:
        assert np.array_equal(d_in.cpu().numpy(), tables)
    pools.check()
    return want


def some_tables(rng, rows, width, num_pages, live):
    """`live` pages, each named once at least, some more often, among entries of -1."""
    t = np.full(rows * width, -1, dtype=np.int32)
    named = rng.permutation(num_pages)[:live]
    at = rng.permutation(rows * width)
    t[at[:live]] = named
    again = at[live: live + live // 3]
    t[again] = named[: len(again)]
    return t.reshape(rows, width)


@pytest.mark.parametrize("which,layers,n_kv,hd,block", [(1, 2, 2, 64, 16), (2, 3, 1, 128, 32), (3, 2, 1, 64, 16), (2, 130, 1, 64, 16), (3, 66, 1, 64, 16)])
@pytest.mark.parametrize("num_pages,live", [(1, 1), (33, 20), (64, 63), (97, 1), (40, 40)])
def test_compact(hc, torch, which, layers, n_kv, hd, block, num_pages, live):
    rng = np.random.default_rng([32, which, num_pages, layers])
    pools = Pools(hc, rng, which, layers, num_pages, n_kv, hd, block)
    tables = some_tables(rng, 5, num_pages // 2 + 1, num_pages, live)
    after = check_compact(hc, torch, pools, tables, times=2)          # from the old tables it can be done again
    # what is compact stays as it is, and is done in place
    assert np.array_equal(check_compact(hc, torch, pools, after, in_place=True), after)
    pools.ctx.destroy()


def test_compact_nothing_and_bad_entries(hc, torch):
    rng = np.random.default_rng(33)
    pools = Pools(hc, rng, 2, 1, 20, 1, 64, 16)
    check_compact(hc, torch, pools, np.full((3, 4), -1, dtype=np.int32))
    check_compact(hc, torch, pools, np.zeros((0, 4), dtype=np.int32))
    check_compact(hc, torch, pools, np.array([[5, 20, -3], [2 ** 31 - 1, -2 ** 31, 17]], dtype=np.int32), flags=hc.HC_DEV_BAD_PAGE, in_place=True)
    pools.ctx.destroy()


@pytest.mark.parametrize("num_pages,live", [(32768, 20000), (40000, 39999), (100003, 61234), (1 << 20, 700001)])
def test_compact_many_pages(hc, torch, num_pages, live):
    """Plans of many pages; the pages themselves, of one head of 64 in 16 tokens, are checked by a mark in each."""
    rng = np.random.default_rng([34, num_pages])
    pool = torch.zeros((num_pages, 1, 1, 17 * 64), dtype=torch.uint8, device="cuda")
    ids = torch.arange(num_pages, dtype=torch.int32, device="cuda")
    mark = pool.view(num_pages, -1)
    for at in (0, 512, 1084):
        mark[:, at:at + 4] = ids.view(torch.uint8).view(num_pages, 4)
    ctx = kh.context(hc, 1, 1, 64, 16)
    ctx.set_kv4_pool(0, pool, num_pages)
    tables = some_tables(rng, 7, live // 5 + 1, num_pages, live)
    d_tab, plan = gh.to_dev_i32(tables), torch.zeros((2 + 2 * num_pages,), dtype=torch.int32, device="cuda")
    ctx.compact_pages(hc.HC_POOL_KV4, d_tab, d_tab, *tables.shape, plan, gh.stream_handle())
    assert ctx.poll_device_error(gh.stream_handle()) == 0
    seen = np.zeros(num_pages, dtype=bool)
    seen[tables[tables >= 0]] = True
    named = np.nonzero(seen)[0]
    place = np.full(num_pages, -1, dtype=np.int32)
    place[named] = named
    moving = named[named >= live]
    place[moving] = np.nonzero(~seen[:live])[0]
    got = plan.cpu().numpy()
    assert got[0] == live and got[1] == len(moving) and np.array_equal(got[2:2 + num_pages], place)
    assert np.array_equal(d_tab.cpu().numpy(), np.where(tables >= 0, place[np.maximum(tables, 0)], -1))
    for at in (0, 512, 1084):
        now = mark[:, at:at + 4].contiguous().view(torch.int32)[:, 0].cpu().numpy()
        assert np.array_equal(now[place[named]], named)
    ctx.destroy()


def test_pages_in_a_graph(hc, torch):
    """A fork and a compaction captured once and replayed on other tables, between other work."""
    rng = np.random.default_rng(35)
    pools = Pools(hc, rng, 3, 2, 30, 2, 64, 16)
    tables = some_tables(rng, 4, 9, 30, 14)
    tables[2:] = -1
    d_tab, out = gh.to_dev_i32(tables), gh.to_dev_i32(np.zeros_like(tables))
    plan = torch.zeros((62,), dtype=torch.int32, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        pools.ctx.compact_pages(3, d_tab, out, 4, 9, plan, side.cuda_stream)
        pools.ctx.fork_pages(3, out, 4, 9, [0], [3], [33], [29], side.cuda_stream)
    for i in range(3):
        tables = some_tables(np.random.default_rng([36, i]), 4, 9, 30, 12 + i)
        tables[0, :3] = [29 - i, 3, 28 - i]
        tables[3] = -1
        d_tab.copy_(gh.to_dev_i32(tables))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert pools.ctx.poll_device_error(gh.stream_handle()) == 0
        want, live, moves, place = kv4.compact(tables, 30)
        for a, b in moves:
            pools.copy(a, b)
        copied = []
        want = kv4.fork(want, copied, [0], [3], [33], [29], 16)
        for a, b, n in copied:
            pools.copy(a, b, n)
        assert np.array_equal(out.cpu().numpy(), want)
        pools.check()


def test_a_cache_in_use(hc, torch):
    """The operators together, as a serving program has them: a layer's context restored into bf16 pages, taken over into 4 bits,
    attended to, forked, both continued by a token of their own, the parent ended, the cache compacted, attended to again."""
    rng = np.random.default_rng(37)
    n_q, n_kv, hd, block, n = 8, 2, 128, 16, 75
    d_kv, width, num_pages = n_kv * hd, 8, 24
    desc = gh.make_desc(hc, n_layers=1, d_model=256, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=hd, block_size=block, max_position=256)
    ctx, s = hc.Context(desc), gh.stream_handle()
    case = gh.LayerCase(rng, 256, n_kv, hd, n)
    d_w, d_g, d_x = gh.to_dev_bf16(case.wkv_bits), gh.to_dev_bf16(case.gamma_bits), gh.to_dev_bf16(case.x_bits)
    pool, pool4 = gh.new_pool(num_pages, block, n_kv, hd), torch.full((num_pages, n_kv, 1, 17 * hd), 255, dtype=torch.uint8, device="cuda")
    ctx.set_layer_weights(0, d_w, d_g, s)
    ctx.set_kv_pool(0, pool, num_pages)
    ctx.set_kv4_pool(0, pool4, num_pages)
    tables = np.full((2, width), -1, dtype=np.int32)
    tables[0, :5] = [20, 3, 17, 9, 22]
    d_tab, pos = gh.to_dev_i32(tables), gh.to_dev_i32(np.arange(n))
    ctx.restore_kv(0, d_x, pos, n, d_tab, width, s)
    ctx.quantize_kv_pages(0, pos, n, d_tab, width, d_tab, width, s)
    # the oracle goes on from the bf16 rows as they were restored
    rows = torch.zeros((n, 2 * d_kv), dtype=torch.bfloat16, device="cuda")
    ctx.gather_kv(0, rows, pos, n, d_tab, width, s)
    kv = kv4.dequantize(*kv4.quantize(kh.f64(kh.bits_of(rows)).reshape(n, 2, n_kv, hd)))

    def attend(d_tables, q_bits, lens, contexts):
        m = len(q_bits)
        size = hc.attend_kv4_workspace(desc, m, m, 1, max(lens))
        ws = torch.empty((max(size, 16),), dtype=torch.uint8, device="cuda")
        out, lse = torch.zeros((m, n_q * hd), dtype=torch.bfloat16, device="cuda"), torch.zeros((m, n_q), device="cuda")
        d_q = gh.to_dev_bf16(q_bits.reshape(m, -1))
        ctx.attend_kv4(0, d_q, n_q * hd, gh.to_dev_i32(np.array(lens) - 1), m, gh.to_dev_i32(np.arange(m + 1)), gh.to_dev_i32(lens), m, 1,
                       max(lens), d_tables, width, hd ** -0.5, 0, out, n_q * hd, lse, ws, ws.numel(), s)
        assert ctx.poll_device_error(s) == 0
        got, got_lse = out.double().cpu().numpy().reshape(m, n_q, hd), lse.double().cpu().numpy()
        for i, x in enumerate(contexts):
            want, want_lse, size, reach = kv4.attend(kh.f64(q_bits[i:i + 1]), [lens[i] - 1], x[:, 0], x[:, 1], np.ones(len(x), dtype=bool),
                                                     float(np.float32(hd ** -0.5)), 0)
            tol, tol_lse = kh.attend_limits(size, reach, want_lse, hd, lens[i])
            assert np.all(np.abs(got[i] - want[0]) <= tol[0]) and np.all(np.abs(got_lse[i] - want_lse[0]) <= tol_lse[0])
        return out

    q = kh.rand_bf16(rng, (2, n_q, hd))
    attend(d_tab, q[:1], [n], [kv])
    ctx.fork_pages(hc.HC_POOL_KV | hc.HC_POOL_KV4, d_tab, 2, width, [0], [1], [n], [11], s)
    assert d_tab.cpu().numpy()[1].tolist() == [20, 3, 17, 9, 11, -1, -1, -1]
    new = kh.rand_bf16(rng, (2, 2, n_kv, hd))
    ctx.quantize_kv(0, gh.to_dev_bf16(new.reshape(2, -1)), gh.to_dev_i32([n, n]), 2, gh.to_dev_i32([0, 1, 2]), 2, d_tab, width, s)
    values = kv4.dequantize(*kv4.quantize(kh.f64(new)))
    both = [np.concatenate([kv, values[i:i + 1]]) for i in range(2)]
    out = attend(d_tab, q, [n + 1, n + 1], both)
    # the parent ends: what it alone had is freed
    plan = torch.zeros((2 + 2 * num_pages,), dtype=torch.int32, device="cuda")
    child = d_tab[1:].contiguous()
    ctx.compact_pages(hc.HC_POOL_KV | hc.HC_POOL_KV4, child, child, 1, width, plan, s)
    assert ctx.poll_device_error(s) == 0
    assert plan[0].item() == 5 and sorted(child.cpu().numpy()[0, :5].tolist()) == [0, 1, 2, 3, 4]
    again = attend(child, q[1:], [n + 1], both[1:])
    assert torch.equal(again[0], out[1])
    ctx.destroy()


def test_compact_many_pages_in_a_graph(hc, torch):
    """A plan whose bits need more LDS than a launch has by itself, captured; the replays find less and less to do."""
    num_pages, live = 300000, 1000
    rng = np.random.default_rng(38)
    pool = torch.zeros((num_pages, 1, 1, 17 * 64), dtype=torch.uint8, device="cuda")
    ctx = kh.context(hc, 1, 1, 64, 16)
    ctx.set_kv4_pool(0, pool, num_pages)
    d_tab, plan = torch.zeros((10, 100), dtype=torch.int32, device="cuda"), torch.zeros((2 + 2 * num_pages,), dtype=torch.int32, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        ctx.compact_pages(hc.HC_POOL_KV4, d_tab, d_tab, 10, 100, plan, side.cuda_stream)
    for i in range(3):
        named = rng.permutation(num_pages)[:live].astype(np.int32)
        marks = torch.from_numpy(rng.integers(0, 256, (live, 17 * 64)).astype(np.uint8)).cuda()
        pool.view(num_pages, -1)[torch.from_numpy(named).cuda().long()] = marks
        d_tab.copy_(gh.to_dev_i32(named.reshape(10, 100)))
        for again in range(2):
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert ctx.poll_device_error(gh.stream_handle()) == 0
            assert plan[:2].tolist() == [live, 0 if again else int((named >= live).sum())]
            now = d_tab.cpu().numpy().reshape(-1)
            assert sorted(now.tolist()) == list(range(live)) and np.array_equal(now[named < live], named[named < live])
            assert torch.equal(pool.view(num_pages, -1)[d_tab.view(-1).long()], marks)
    ctx.destroy()
