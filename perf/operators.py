"""The cache operators that performance is measured on beside the restoration, and the ranges they stand for:
a KV cache held in 4 bits, attention over it, forking contexts and compacting the pages of a cache.

`run` computes an operator in plain torch, in 32 bits and rounded once at the end, or, where `own` is set, with
the library's entry points.  Head layouts are those of this repository's workloads, and three generic ones.
Values: keys and values N(0, 1) with two of a head's key channels five times as large, queries N(0, 1), pages a random
permutation of a pool 25 % larger than needed.

The 4-bit cache: 32 neighbouring channels of a row share a scale, a power of two s, the smallest with
max|x| <= 7 s; codes are the 4-bit floats 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign.  Of 16 tokens a head's block holds
the codes of K by token, those of V with the four tokens of a quarter side by side for every 16th of the
channels, and the scales of both in the same orders.
"""
import random

import numpy as np
import torch

own = False

GROUP = 32                 # channels that share a scale
SUB = 16                   # tokens of a block of the 4-bit cache

# (query heads, KV heads, head dim)
LAYOUTS = {
    "4x64": (4, 4, 64),
    "32x128": (32, 32, 128),
    "32-8x128": (32, 8, 128),
    "40x128": (40, 40, 128),
    "56x128": (56, 56, 128),
    "64-8x128": (64, 8, 128),
    "14-2x64": (14, 2, 64),
    "16-8x256": (16, 8, 256),
    "12-4x128": (12, 4, 128),
}


def listed():
    return [
        # the keys and values of a decoding step of 64 contexts go into the 4-bit cache, and come back
        dict(name="cache-step", op="cache", layout="32-8x128", source="rows", contexts=64, tokens=64, history=2000, block=16),
        # a turn's rows of a multi-head model, starting inside a page
        dict(name="cache-turn", op="cache", layout="40x128", source="rows", contexts=1, tokens=2501, history=1003, block=16),
        # a long context, as it stands restored in bf16 pages, becomes a 4-bit one
        dict(name="cache-context", op="cache", layout="64-8x128", source="pages", contexts=1, tokens=32768, history=0, block=16),
        # one token of a single short conversation: nothing but launch and latency
        dict(name="attend-one", op="attend", layout="32-8x128", contexts=1, idle=0, q=1, kv=1037, window=0, block=16),
        # a decoding step of a full batch with uneven contexts, two of its places empty
        dict(name="attend-batch", op="attend", layout="32-8x128", contexts=64, idle=2, q=1, kv=8192, window=0, block=16),
        # one token of a single very long context
        dict(name="attend-long", op="attend", layout="64-8x128", contexts=1, idle=0, q=1, kv=131072, window=0, block=16),
        # a user's next turn on a restored history
        dict(name="attend-turn", op="attend", layout="32-8x128", contexts=1, idle=0, q=501, kv=8692, window=0, block=16),
        # prompts of several requests of a multi-head model on histories of their own
        dict(name="attend-prompts", op="attend", layout="40x128", contexts=8, idle=0, q=2048, kv=4096, window=0, block=16),
        # eight samples from one prompt: 32 layers of bf16 pages
        dict(name="fork-samples", op="fork", layout="32-8x128", pool="kv", layers=32, forks=8, kv=1003, block=16),
        # many contexts of a 4-bit cache forked at once
        dict(name="fork-many", op="fork", layout="64-8x128", pool="kv4", layers=80, forks=64, kv=2037, block=16),
        # a small 4-bit cache after a few of its contexts have ended
        dict(name="compact-small", op="compact", layout="32-8x128", pool="kv4", layers=8, pages=500, live=290, contexts=5, block=16),
        # bf16 pages of 32 layers, 2048 tokens more or less to a context, a third of the pages free
        dict(name="compact-large", op="compact", layout="32-8x128", pool="kv", layers=32, pages=2048, live=1361, contexts=11, block=16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["cache"] * 3 + ["attend"] * 6 + ["fork", "compact"] * 2)
    layout = rng.choice(list(LAYOUTS))
    nq, nkv, hd = LAYOUTS[layout]
    block = rng.choice([16, 16, 32, 64])
    if op == "cache":
        most = 2 ** 25 // (nkv * hd)
        tokens = _log_int(rng, 1, most)
        source = rng.choice(["rows", "rows", "pages"])
        contexts = 1 if source == "pages" else _log_int(rng, 1, min(64, tokens))
        return dict(op=op, layout=layout, source=source, contexts=contexts, tokens=tokens, history=rng.randrange(2048), block=block)
    if op == "attend":
        contexts = _log_int(rng, 1, 64)
        q = rng.choice([1, 1, 1, rng.randrange(2, 9), _log_int(rng, 16, 2048), _log_int(rng, 16, 2048)])
        most = min(131072, 2 ** 22 * 128 // (contexts * nkv * hd), 2 ** 31 * 128 // (contexts * nq * q * hd))
        q = min(q, most)
        return dict(op=op, layout=layout, contexts=contexts, idle=rng.choice([0, 0, contexts // 8]), q=q, kv=max(q, _log_int(rng, 1, most)),
                    window=rng.choice([0, 0, 0, _log_int(rng, 1, 4096)]), block=block)
    pool = rng.choice(["kv", "kv4"])
    layers = rng.choice([1, 4, 8, 32, 80])
    page = layers * nkv * hd * block * (4 if pool == "kv" else 2)   # values as bytes, more or less
    if op == "fork":
        most = max(2, min(64, 2 ** 30 // (4 * page)))
        forks = _log_int(rng, 1, most)
        blocks = max(1, int(2 ** 31 / 1.3 / page - forks) // max(1, forks // 8))
        return dict(op=op, layout=layout, pool=pool, layers=layers, forks=forks, kv=_log_int(rng, 1, min(8192, blocks * block)), block=block)
    pages = _log_int(rng, 8, max(8, min(16384, 2 ** 31 // page)))
    live = rng.randrange(1, pages + 1)
    return dict(op=op, layout=layout, pool=pool, layers=layers, pages=pages, live=live, contexts=_log_int(rng, 1, min(64, live)), block=block)


def _shares(key, n, total):
    """`n` uneven numbers of at least 1 that add up to `total`."""
    r = random.Random(key)
    part = [r.uniform(0.25, 2.0) for _ in range(n)]
    got = [1 + int((total - n) * p / sum(part)) for p in part]
    got[-1] += total - sum(got)
    return got


def lengths(case):
    """(queries, keys) of every context of an attention case: the first has the most, idle ones at the end none."""
    r = random.Random("%d-%d-%d" % (case["contexts"], case["q"], case["kv"]))
    qs, kvs = [], []
    for i in range(case["contexts"]):
        q = case["q"] if i == 0 or case["q"] == 1 else r.randint(max(1, case["q"] // 4), case["q"])
        kv = case["kv"] if i == 0 else r.randint(max(q, case["kv"] // 4), case["kv"])
        qs.append(q)
        kvs.append(kv)
    for i in range(case["contexts"] - case["idle"], case["contexts"]):
        qs[i], kvs[i] = 1, 0
    return qs, kvs


def _blocks(tokens, block):
    return -(-tokens // block)


# ---- inputs --------------------------------------------------------------------------------
class _Inputs:
    """Tensors made on the GPU from one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.bfloat16)

    def keys_values(self, n, nkv, hd):
        """bf16 [n, 2, KV heads, head dim]"""
        x = self.normal((n, 2, nkv, hd))
        x[:, 0, :, hd // 3] *= 5
        x[:, 0, :, hd - 7] *= 5
        return x

    def permutation(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _tables(inp, blocks, num_pages):
    """int32 [contexts, most blocks], -1 behind a context's last block."""
    perm = inp.permutation(num_pages).to(torch.int32)
    count = torch.tensor(blocks, device="cuda")
    width = max(max(blocks), 1)
    at = torch.arange(width, device="cuda")
    first = (count.cumsum(0) - count)[:, None]
    return torch.where(at < count[:, None], perm[(first + at).clamp(max=num_pages - 1)], -1).contiguous()


def _library(case, layers):
    """A context of the library with the case's head layout."""
    import paper_2410_05004_amd as hc
    nq, nkv, hd = LAYOUTS[case["layout"]]
    desc = hc.ModelDesc(layers, 256, nq, nkv, hd, case["block"], 1 << 20, 2, 1e4, 1e-5, hc.HC_NORM_RMS)
    return hc, desc, hc.Context(desc)


def prepare(case, seed):
    inp = _Inputs(seed)
    nq, nkv, hd = LAYOUTS[case["layout"]]
    block = case["block"]
    s = dict(case, nq=nq, nkv=nkv, hd=hd)
    if case["op"] == "cache":
        n, contexts = case["tokens"], case["contexts"]
        part = _shares("%d-%d" % (n, contexts), contexts, n)
        blocks = [_blocks(case["history"] + p, block) for p in part]
        num_pages = sum(blocks) * 5 // 4 + 1
        s["table"] = _tables(inp, blocks, num_pages)
        s["context"] = torch.repeat_interleave(torch.arange(contexts, device="cuda"), torch.tensor(part, device="cuda"))
        s["cu"] = _ints([0] + list(np.cumsum(part)))
        s["positions"] = (torch.arange(n, device="cuda") - s["cu"].long()[s["context"]] + case["history"]).to(torch.int32)
        s["pool"] = torch.zeros((num_pages, nkv, block // SUB, 17 * hd), dtype=torch.uint8, device="cuda")
        rows = inp.keys_values(n, nkv, hd)
        if case["source"] == "rows":
            s["rows"] = rows.view(n, 2 * nkv * hd)
        else:
            s["source_table"] = _tables(inp, blocks, num_pages)
            s["source_pool"] = torch.zeros((num_pages, 2, block, nkv, hd), dtype=torch.bfloat16, device="cuda")
            pos = s["positions"].long()
            s["source_pool"][s["source_table"][0][pos // block].long(), :, pos % block] = rows
        if own:
            hc, _, s["ctx"] = _library(case, 1)
            s["ctx"].set_kv4_pool(0, s["pool"], num_pages)
            if case["source"] == "pages":
                s["ctx"].set_kv_pool(0, s["source_pool"], num_pages)
        return s
    if case["op"] == "attend":
        qs, kvs = lengths(case)
        blocks = [_blocks(k, block) for k in kvs]
        num_pages = sum(blocks) * 5 // 4 + 1
        s["table"] = _tables(inp, blocks, num_pages)
        s["q_lens"], s["kv_lens"], s["cu"] = _ints(qs), _ints(kvs), _ints([0] + list(np.cumsum(qs)))
        s["context"] = torch.repeat_interleave(torch.arange(len(qs), device="cuda"), torch.tensor(qs, device="cuda"))
        n = sum(qs)
        s["n"], s["most_q"], s["most_kv"] = n, max(qs), max(kvs)
        at = torch.arange(n, device="cuda") - s["cu"].long()[s["context"]]
        s["positions"] = (s["kv_lens"] - s["q_lens"])[s["context"]].add(at).to(torch.int32)   # -1 in an empty place
        s["query"] = inp.normal((n, nq, hd))
        s["scale"] = hd ** -0.5
        s["pool"] = torch.empty((num_pages, nkv, block // SUB, 17 * hd), dtype=torch.uint8, device="cuda")
        step = max(1, 2 ** 26 // (block * nkv * hd))
        for at in range(0, num_pages, step):
            m = min(step, num_pages - at)
            k, v = inp.keys_values(m * block, nkv, hd).view(m, block // SUB, SUB, 2, nkv, hd).permute(3, 0, 4, 1, 2, 5)
            s["pool"][at:at + m] = _pack(*_codes(k.float()), *_codes(v.float()))
        if own:
            hc, desc, s["ctx"] = _library(case, 1)
            s["ctx"].set_kv4_pool(0, s["pool"], num_pages)
            size = hc.attend_kv4_workspace(desc, len(qs), n, s["most_q"], s["most_kv"])
            s["workspace"] = torch.empty((size,), dtype=torch.uint8, device="cuda")
        return s
    layers = case["layers"]
    kv4 = case["pool"] == "kv4"
    page = (nkv, block // SUB, 17 * hd) if kv4 else (2, block, nkv, hd)
    if case["op"] == "fork":
        # an eighth of the forks, one at least, are parents: every fork at a length of its own
        parents, forks = max(1, case["forks"] // 8), case["forks"]
        r = random.Random("%d-%d" % (forks, case["kv"]))
        own_len = [case["kv"] if i == 0 else r.randint(max(1, case["kv"] // 2), case["kv"]) for i in range(parents)]
        blocks = [_blocks(n, block) for n in own_len]
        num_pages = (sum(blocks) + forks) * 5 // 4 + 1
        perm = inp.permutation(num_pages).to(torch.int32)
        first = np.cumsum([0] + blocks)
        s["table"] = torch.full((parents + forks, max(blocks) + 1), -1, dtype=torch.int32, device="cuda")
        for i in range(parents):
            s["table"][i, :blocks[i]] = perm[first[i]:first[i + 1]]
        s["h_from"] = np.array([i % parents for i in range(forks)], dtype=np.int32)
        s["h_to"] = np.arange(parents, parents + forks, dtype=np.int32)
        s["h_len"] = np.array([own_len[i % parents] if i < parents else r.randint(max(1, own_len[i % parents] // 2), own_len[i % parents]) for i in range(forks)], dtype=np.int32)
        s["h_page"] = perm[first[-1]:first[-1] + forks].cpu().numpy()
        s["from"], s["to"], s["len"], s["page"] = (torch.from_numpy(s["h_" + k]).cuda().long() for k in ("from", "to", "len", "page"))
    else:
        num_pages, live, contexts = case["pages"], case["live"], case["contexts"]
        moves = _moves(case)
        low, high = inp.permutation(live), live + inp.permutation(num_pages - live)
        named = torch.cat([low[:live - moves], high[:moves]])
        named = named[inp.permutation(live)].to(torch.int32)
        part = _shares("%d-%d" % (live, contexts), contexts, live)
        # the last row is a context forked from the first: it shares half of its pages
        s["table"] = torch.full((contexts + 1, max(part) + 3), -1, dtype=torch.int32, device="cuda")
        for i, f in enumerate(np.cumsum([0] + part[:-1])):
            s["table"][i, :part[i]] = named[f:f + part[i]]
        s["table"][contexts, :part[0] // 2] = s["table"][0, :part[0] // 2]
        s["new_table"] = torch.empty_like(s["table"])
        s["plan"] = torch.zeros((2 + 2 * num_pages,), dtype=torch.int32, device="cuda")
    s["pages"] = num_pages
    if kv4:
        s["pool"] = torch.randint(0, 250, (layers, num_pages) + page, generator=inp.g, device="cuda", dtype=torch.uint8)
    else:
        s["pool"] = inp.normal((layers, num_pages) + page)
    if own:
        s["hc"], _, s["ctx"] = _library(case, layers)
        for l in range(layers):
            (s["ctx"].set_kv4_pool if kv4 else s["ctx"].set_kv_pool)(l, s["pool"][l], num_pages)
    return s


def _moves(case):
    """Live pages that lie behind the place of the last one of a compact cache: as many as by chance."""
    live, pages = case["live"], case["pages"]
    return min(pages - live, round(live * (pages - live) / pages))


# ---- the 4-bit format ----------------------------------------------------------------------
def _codes(x):
    """Codes (uint8, one each) and scales (uint8 exponents) of 32-bit rows."""
    g = x.unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e - 3 + (m > 0.875), -125).clamp(-125, 125)
    y = torch.ldexp(g, -e[..., None]).abs()
    c = (y > 0.25).to(torch.uint8)
    c += y >= 0.75
    c += y > 1.25
    c += y >= 1.75
    c += y > 2.5
    c += y >= 3.5
    c += y > 5
    c += torch.signbit(g).to(torch.uint8) * 8
    fine = torch.isfinite(top)
    return torch.where(fine[..., None], c, 0).flatten(-2), torch.where(fine, e + 127, 255).to(torch.uint8)


def _nibbles(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _pack(kc, ks, vc, vs):
    """Blocks uint8 [..., 17 * head dim] of codes and scales [..., 16 tokens, channels]."""
    k, v = _nibbles(kc), _nibbles(vc)
    v = v.unflatten(-2, (4, 4)).unflatten(-1, (16, -1)).transpose(-3, -2)      # [quarter, 16th, token, bytes]
    vs = vs.unflatten(-2, (4, 4)).transpose(-2, -1)                            # [quarter, group, token]
    return torch.cat([k.flatten(-2), v.flatten(-4), ks.flatten(-2), vs.flatten(-3)], -1)


def _parts(pool, hd):
    """Views of a pool: codes of K [..., token, bytes] and of V [..., quarter, 16th, token, bytes], their scales."""
    k, v, ks, vs = pool.split([8 * hd, 8 * hd, hd // 2, hd // 2], -1)
    return k.unflatten(-1, (SUB, -1)), v.unflatten(-1, (4, 16, 4, -1)), ks.unflatten(-1, (SUB, -1)), vs.unflatten(-1, (4, -1, 4))


def _values(codes, scales):
    """32-bit rows of packed codes [..., channels / 2] and scales [..., channels / 32]."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=c.device)
    s = torch.where(scales == 255, float("nan"), (scales.int() << 23).view(torch.float32))
    return table[c.int()].unflatten(-1, (-1, GROUP)).mul_(s[..., None]).flatten(-2)


# ---- passes --------------------------------------------------------------------------------
def run(s):
    if own:
        return {"cache": _own_cache, "attend": _own_attend, "fork": _own_fork, "compact": _own_compact}[s["op"]](s)
    return {"cache": _plain_cache, "attend": _plain_attend, "fork": _plain_fork, "compact": _plain_compact}[s["op"]](s)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _own_cache(s):
    n, stream, table = s["tokens"], _stream(), s["table"]
    if s["source"] == "rows":
        s["ctx"].quantize_kv(0, s["rows"], s["positions"], n, s["cu"], s["contexts"], table, table.shape[1], stream)
    else:
        s["ctx"].quantize_kv_pages(0, s["positions"], n, s["source_table"], table.shape[1], table, table.shape[1], stream)
    out = torch.empty((n, 2 * s["nkv"] * s["hd"]), dtype=torch.bfloat16, device="cuda")
    s["ctx"].dequantize_kv(0, out, s["positions"], n, s["cu"], s["contexts"], table, table.shape[1], stream)
    return out


def _plain_cache(s):
    n, nkv, hd, block = s["tokens"], s["nkv"], s["hd"], s["block"]
    pos = s["positions"].long()
    page, slot = s["table"][s["context"], pos // block].long(), pos % block
    if s["source"] == "rows":
        x = s["rows"].view(n, 2, nkv, hd)
    else:
        x = s["source_pool"][s["source_table"][0][pos // block].long(), :, slot]
    codes, scales = _codes(x.float())
    codes = _nibbles(codes)
    k, v, ks, vs = _parts(s["pool"], hd)
    sub, token = slot // SUB, slot % SUB
    quarter, at = token // 4, token % 4
    k[page, :, sub, token] = codes[:, 0]
    v[page, :, sub, quarter, :, at] = codes[:, 1].unflatten(-1, (16, -1))
    ks[page, :, sub, token] = scales[:, 0]
    vs[page, :, sub, quarter, :, at] = scales[:, 1]
    k = _values(k[page, :, sub, token], ks[page, :, sub, token])
    v = _values(v[page, :, sub, quarter, :, at].flatten(-2), vs[page, :, sub, quarter, :, at])
    return torch.stack([k, v], 1).view(n, 2 * nkv * hd).to(torch.bfloat16)


def _own_attend(s):
    out = torch.empty_like(s["query"])
    lse = torch.empty(s["query"].shape[:2], dtype=torch.float32, device="cuda")
    width = s["nq"] * s["hd"]
    s["ctx"].attend_kv4(0, s["query"], width, s["positions"], s["n"], s["cu"], s["kv_lens"], s["contexts"], s["most_q"], s["most_kv"],
                        s["table"], s["table"].shape[1], s["scale"], s["window"], out, width, lse, s["workspace"], s["workspace"].numel(), _stream())
    return out, lse


def _plain_attend(s):
    nq, nkv, hd, n = s["nq"], s["nkv"], s["hd"], s["contexts"]
    g, most_q = nq // nkv, s["most_q"]
    # every context's keys and values, [contexts, KV heads, keys, channels]
    blocks = s["pool"][s["table"].clamp(min=0).long()].transpose(1, 2).flatten(2, 3)
    k, v, ks, vs = _parts(blocks, hd)
    k = _values(k, ks).flatten(2, 3)
    v = _values(v.transpose(-3, -2).flatten(-2), vs.transpose(-2, -1)).flatten(2, 4)
    # its queries, [contexts, KV heads, query heads of one * queries, channels]
    at = s["cu"][:-1, None].long() + torch.arange(most_q, device="cuda")
    at = at.clamp(max=s["n"] - 1)
    q = s["query"].float()[at].view(n, most_q, nkv, g, hd).permute(0, 2, 3, 1, 4).flatten(2, 3)
    p = s["positions"][at]
    j = torch.arange(k.shape[2], device="cuda", dtype=torch.int32)
    seen = (j <= p[..., None]) & (j < s["kv_lens"][:, None, None])
    if s["window"]:
        seen &= j > p[..., None] - s["window"]
    seen = seen[:, None].repeat(1, 1, g, 1)
    w = (q @ k.transpose(2, 3)).mul_(s["scale"]).masked_fill_(~seen, float("-inf"))
    top = w.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    w = w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    out = (w @ v).div_(torch.where(total > 0, total, 1.0))
    lse = (total.log() + top)[..., 0]
    # back to the queries' own order
    row = torch.arange(s["n"], device="cuda") - s["cu"].long()[s["context"]]
    out = out.unflatten(2, (g, most_q))[s["context"], :, :, row]
    lse = lse.unflatten(2, (g, most_q))[s["context"], :, :, row]
    return out.reshape(s["n"], nq, hd).to(torch.bfloat16), lse.reshape(s["n"], nq)


def _own_fork(s):
    t = s["table"]
    s["ctx"].fork_pages(s["hc"].HC_POOL_KV4 if s["pool"].dtype == torch.uint8 else s["hc"].HC_POOL_KV, t, t.shape[0], t.shape[1],
                        s["h_from"], s["h_to"], s["h_len"], s["h_page"], _stream())
    return t, s["pool"]


def _plain_fork(s):
    t, pool, block = s["table"], s["pool"], s["block"]
    whole, rest = s["len"] // block, s["len"] % block
    b = torch.arange(t.shape[1], device="cuda")
    parent = t[s["from"]]
    child = torch.where(b < whole[:, None], parent, -1)
    child = torch.where((b == whole[:, None]) & (rest > 0)[:, None], s["page"][:, None].int(), child)
    t[s["to"]] = child
    # of a part-filled page the slots in use (of a 4-bit one, its 16-token blocks in use) are copied
    last = parent.gather(1, whole[:, None])[:, 0].clamp(min=0).long()
    if pool.dtype == torch.uint8:
        used = (torch.arange(block // SUB, device="cuda") * SUB < rest[:, None])[:, None, :, None]
    else:
        used = (torch.arange(block, device="cuda") < rest[:, None])[:, None, :, None, None]
    pool[:, s["page"]] = torch.where(used, pool[:, last], pool[:, s["page"]])
    return t, pool


def _own_compact(s):
    t = s["table"]
    s["ctx"].compact_pages(s["hc"].HC_POOL_KV4 if s["pool"].dtype == torch.uint8 else s["hc"].HC_POOL_KV, t, s["new_table"], t.shape[0], t.shape[1],
                           s["plan"], _stream())
    return s["new_table"], s["plan"][:2 + s["pages"]], s["pool"]


def _plain_compact(s):
    t, pool, n = s["table"], s["pool"], s["pages"]
    named = torch.zeros((n + 1,), dtype=torch.int32, device="cuda")
    named.scatter_(0, torch.where(t >= 0, t, n).flatten().long(), 1)
    named = named[:n] > 0
    live = named.sum()
    p = torch.arange(n, device="cuda")
    hole, mover = (~named & (p < live)).nonzero()[:, 0], (named & (p >= live)).nonzero()[:, 0]
    place = torch.where(named, p, -1)
    place[mover] = hole
    pool[:, hole] = pool[:, mover]
    s["new_table"].copy_(torch.where(t >= 0, place[t.clamp(min=0).long()], -1))
    s["plan"][0], s["plan"][1] = live, len(hole)
    s["plan"][2:2 + n] = place
    return s["new_table"], s["plan"][:2 + n], pool


# ---- what a pass cannot do without -----------------------------------------------------------
def work(case):
    nq, nkv, hd = LAYOUTS[case["layout"]]
    block = case["block"]
    if case["op"] == "cache":              # rows read, codes written, codes read, rows written
        values = case["tokens"] * 2 * nkv * hd
        return {"bytes": values * (2 + 17 / 32) * 2, "flops": 0}
    if case["op"] == "attend":
        qs, kvs = lengths(case)
        n = sum(qs)
        pairs = keys = 0
        for q, kv in zip(qs, kvs):
            first = kv - q                 # keys before the first query
            w = case["window"] or kv
            if kv:
                pairs += sum(min(w, first + i + 1) for i in range(q))
                keys += min(kv, w + q - 1)
        return {"bytes": keys * nkv * 17 * hd // 16 + n * nq * (4 * hd + 4), "flops": 4 * hd * nq * pairs}
    page = nkv * (block // SUB * 17 * hd if case["pool"] == "kv4" else 4 * block * hd)
    if case["op"] == "fork":               # half a page each, more or less, and the tables' rows
        return {"bytes": case["layers"] * case["forks"] * page + 8 * case["forks"] * _blocks(case["kv"], block), "flops": 0}
    return {"bytes": 2 * _moves(case) * case["layers"] * page + 8 * case["live"] + 4 * case["pages"], "flops": 0}


# ---- the same in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    """What `run` returns: nearest codes found by trying all of them, attention in 64 bits context by context,
    pages moved one at a time."""
    s = prepare(case, seed)
    nq, nkv, hd = LAYOUTS[case["layout"]]
    block = case["block"]
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    if case["op"] == "cache":
        pos = s["positions"].long()
        if case["source"] == "rows":
            x = s["rows"]
        else:
            x = s["source_pool"][s["source_table"][0][pos // block].long(), :, pos % block].reshape(case["tokens"], -1)
        out = []
        for part in x.split(max(1, 2 ** 24 // x.shape[1])):
            g = part.double().view(-1, GROUP)
            s_exp = torch.ceil(torch.log2(g.abs().amax(1) / 7)).clamp(-125, 125)
            s_exp = torch.where(g.abs().amax(1) > 7 * 2.0 ** s_exp, s_exp + 1, s_exp)      # where the logarithm's rounding fell short
            s_exp = torch.where(g.abs().amax(1) <= 3.5 * 2.0 ** s_exp, s_exp - 1, s_exp).clamp(-125, 125)
            y = g / (2.0 ** s_exp)[:, None]
            # the last of the grid's values that is no further than the one before; of two as near, that with an even code
            mid = (grid[1:] + grid[:-1]) / 2
            code = torch.bucketize(y.abs(), mid)
            tie = (y.abs()[..., None] == mid).any(-1)
            code = torch.where(tie & (code % 2 == 1), code + 1, code)
            out.append((grid[code] * y.sign() * (2.0 ** s_exp)[:, None]).view(part.shape))
        return torch.cat(out)
    if case["op"] == "attend":
        qs, kvs = lengths(case)
        out, lse = torch.zeros((s["n"], nq, hd), dtype=torch.float64, device="cuda"), torch.full((s["n"], nq), float("-inf"), dtype=torch.float64, device="cuda")
        signed = torch.cat([grid, -grid])
        row = 0
        for i, (q, kv) in enumerate(zip(qs, kvs)):
            if kv:
                b = s["pool"][s["table"][i, :_blocks(kv, block)].long()].transpose(0, 1).reshape(nkv, -1, 17 * hd).long()
                k = torch.stack([b[..., :8 * hd] % 16, b[..., :8 * hd] // 16], -1).view(nkv, -1, hd)
                v = torch.stack([b[..., 8 * hd:16 * hd] % 16, b[..., 8 * hd:16 * hd] // 16], -1)
                v = v.view(nkv, -1, 4, 16, 4, hd // 16).permute(0, 1, 2, 4, 3, 5).reshape(nkv, -1, hd)
                ks = b[..., 16 * hd:16 * hd + hd // 2].reshape(nkv, -1, hd // GROUP)
                vs = b[..., 16 * hd + hd // 2:].view(nkv, -1, 4, hd // GROUP, 4).transpose(3, 4).reshape(nkv, -1, hd // GROUP)
                k, v = (signed[c] * (2.0 ** (e.double() - 127)).repeat_interleave(GROUP, 2) for c, e in ((k, ks), (v, vs)))
                pos = torch.arange(kv - q, kv, device="cuda")[:, None]
                at = torch.arange(kv, device="cuda")
                seen = (at <= pos) & (at > pos - (case["window"] or kv + 1))
                for h in range(nq):
                    w = s["query"][row:row + q, h].double() @ k[h * nkv // nq, :kv].t() * s["scale"]
                    w = torch.where(seen, w, float("-inf"))
                    lse[row:row + q, h] = w.logsumexp(1)
                    out[row:row + q, h] = (w - lse[row:row + q, h, None]).exp() @ v[h * nkv // nq, :kv]
            row += q
        return out, lse
    t = s["table"].cpu().numpy().copy()
    pool = s["pool"]
    if case["op"] == "fork":
        for a, b, n, new in zip(s["h_from"], s["h_to"], s["h_len"], s["h_page"]):
            full, rest = int(n) // block, int(n) % block
            t[b] = -1
            t[b, :full] = t[a, :full]
            if rest:
                t[b, full] = new
                if case["pool"] == "kv4":
                    pool[:, new, :, :-(-rest // SUB)] = pool[:, t[a, full], :, :-(-rest // SUB)]
                else:
                    pool[:, new, :, :rest] = pool[:, t[a, full], :, :rest]
        return t, pool
    live = sorted(set(t[t >= 0].tolist()))
    holes = sorted(set(range(len(live))) - set(live))
    plan = np.full(2 + case["pages"], -1, dtype=np.int32)
    plan[0], plan[1] = len(live), len(holes)
    plan[2 + np.array(live)] = live
    for a, b in zip(live[len(live) - len(holes):], holes):
        plan[2 + a] = b
        pool[:, b] = pool[:, a]
    return np.where(t >= 0, plan[2 + np.maximum(t, 0)], -1), plan, pool
