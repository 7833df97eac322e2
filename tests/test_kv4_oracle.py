"""The oracle of the 4-bit cache against its definition, and the host side of the cache's entry points; no GPU."""
import os
import shutil
import subprocess

import numpy as np
import pytest

import oracle.kv4_oracle as kv4
import synthetic as syn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_codes_are_nearest_and_scales_smallest():
    """Every bf16 pattern of both signs, in groups: no value is further than half a step from its code, halving the scale would put
    the largest out of reach, and ties go to the even code."""
    bits = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    bits = bits[(bits & 0x7F80) != 0x7F80]
    rng = np.random.default_rng(5)
    x = syn.bf16_bits_to_f64(rng.permutation(bits)[: len(bits) // 32 * 32]).reshape(-1, 32)
    x = np.concatenate([x, np.repeat(syn.bf16_bits_to_f64(bits)[:, None], 32, 1)])
    code, e = kv4.quantize(x)
    s = 2.0 ** (e[:, :1].astype(np.float64) - 127)
    top = np.abs(x).max(1, keepdims=True)
    y = kv4.dequantize(code, e)
    step = np.array([.5, .5, .5, .5, 1, 1, 2, 2])
    near = np.abs(x) / s
    lower = np.abs(kv4.GRID[code & 7] - near)
    inside = top <= 7 * 2.0 ** 125
    assert np.all((lower <= step[code & 7] / 2) | ~inside)
    assert np.all((top > 3.5 * s) | (e[:, :1] == 2))
    assert np.all((top <= 7 * s) | (e[:, :1] == 252))
    assert np.all(np.signbit(y) == np.signbit(x))
    assert np.array_equal(syn.bf16_bits_to_f64(syn.f32_to_bf16_bits(y.astype(np.float32))), y), "values are exact in bf16"


@pytest.mark.parametrize("value,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5, 6), (7, 7), (0.26, 1)])
def test_ties(value, code):
    x = np.zeros((1, 32))
    x[0, 0], x[0, 5] = 7, -value
    c, e = kv4.quantize(x)
    assert e[0, 0] == 127 and c[0, 0] == 7 and c[0, 5] == code + 8


def test_groups_that_are_not_finite():
    x = np.ones((3, 64))
    x[0, 3], x[1, 40] = np.inf, np.nan
    c, e = kv4.quantize(x)
    assert e.tolist() == [[255, e[2, 0]], [e[2, 0], 255], [e[2, 0], e[2, 0]]]
    y = kv4.dequantize(c, e)
    assert np.isnan(y[0, :32]).all() and np.isfinite(y[0, 32:]).all() and np.isnan(y[1, 32:]).all()


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_places_fill_a_block(hd):
    """Codes and scales of 16 tokens take every nibble and byte of a block once."""
    seen = np.zeros((17 * hd, 2), dtype=int)
    for part in (0, 1):
        for t in range(16):
            at, shift, scales = kv4.places(part, 0, t, hd)
            np.add.at(seen, (at, shift // 4), 1)
            seen[scales] += 1
    assert np.all(seen == 1)


def test_store_and_load(hd=64):
    rng = np.random.default_rng(1)
    pool = rng.integers(0, 256, (3, 2, 2, 17 * hd)).astype(np.uint8)
    x = syn.bf16_bits_to_f64(syn.f32_to_bf16_bits(rng.standard_normal((2, 2, hd), dtype=np.float32)))
    kv4.store_token(pool, 1, 21, x[0], x[1])
    k, v = kv4.load_token(pool, 1, 21, hd)
    assert np.array_equal(k, kv4.dequantize(*kv4.quantize(x[0]))) and np.array_equal(v, kv4.dequantize(*kv4.quantize(x[1])))


def test_oracle_attention_is_softmax():
    rng = np.random.default_rng(2)
    k, v, q = rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((3, 4, 8))
    out, lse, _, _ = kv4.attend(q, [8, 4, -1], k, v, np.ones(9, dtype=bool), 0.5, 0)
    w = np.exp(0.5 * k[:5, 1] @ q[1, 2])
    assert np.allclose(out[1, 2], w @ v[:5, 1] / w.sum()) and np.isclose(lse[1, 2], np.log(w.sum()))
    assert np.all(out[2] == 0) and np.all(np.isinf(lse[2]))
    one, _, _, _ = kv4.attend(q, [8, 4, -1], k, v, np.ones(9, dtype=bool), 0.5, 1)
    assert np.allclose(one[1, 3], v[4, 1])


def test_oracle_compaction():
    t = np.array([[7, 2, -1], [9, 2, 0], [12, -1, -1]], dtype=np.int32)
    tables, live, moves, place = kv4.compact(t, 10)
    assert live == 4 and moves == [(7, 1), (9, 3)]
    assert tables.tolist() == [[1, 2, -1], [3, 2, 0], [-1, -1, -1]]
    assert place.tolist() == [0, -1, 2, -1, -1, -1, -1, 1, -1, 3]


def test_sizes_and_refusals_without_a_context():
    import paper_2410_05004_amd as hc

    def desc(**over):
        kw = dict(n_layers=2, d_model=256, n_q_heads=8, n_kv_heads=2, head_dim=128, block_size=32, max_position=128, rope_style=2,
                  rope_theta=1e4, rms_eps=1e-5, norm_kind=0)
        kw.update(over)
        return hc.ModelDesc(*kw.values())
    assert hc.kv4_page_bytes(desc()) == 2 * 2 * 17 * 128
    for over in (dict(head_dim=192), dict(block_size=8), dict(n_layers=0)):
        with pytest.raises(hc.HCacheError) as e:
            hc.kv4_page_bytes(desc(**over))
        assert e.value.status == hc.HC_EINVAL
        with pytest.raises(hc.HCacheError):
            hc.attend_kv4_workspace(desc(**over), 1, 1, 1, 1)
    with pytest.raises(hc.HCacheError):
        hc.attend_kv4_workspace(desc(), 1, -1, 1, 1)
    assert hc.attend_kv4_workspace(desc(), 0, 0, 0, 0) == 0
    assert hc.attend_kv4_workspace(desc(), 1, 1, 1, 16) == 0
    for sizes in ((1, 1, 1, 131072), (64, 64, 1, 8192), (3, 40, 20, 100000)):
        assert hc.attend_kv4_workspace(desc(), *sizes) % (8 * sizes[1] * 130 * 4) == 0
    for name in ("hc_set_kv4_pool", "hc_quantize_kv", "hc_quantize_kv_pages", "hc_dequantize_kv", "hc_attend_kv4", "hc_fork_pages",
                 "hc_compact_pages"):
        fn = getattr(hc.lib, name)
        args = [None] + [0.0 if "float" in str(t) else 0 if "int" in str(t) or "long" in str(t) else None for t in fn.argtypes[1:]]
        assert fn(*args) == hc.HC_EINVAL, name


def test_refusals_on_the_host(tmp_path):
    """Every refusal of the cache's entry points, on a context whose device pointers are never followed."""
    cc = next((c for c in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc") if c and os.path.exists(c)), None)
    if cc is None:
        pytest.skip("hipcc not found")
    import paper_2410_05004_amd as hc
    exe = str(tmp_path / "cache_refusals")
    lib = os.path.dirname(hc.lib_path())
    r = subprocess.run([cc, "-x", "hip", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                        "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2410_05004_amd", "csrc"),
                        os.path.join(ROOT, "tests", "cache_refusals.cpp"), "-o", exe, "-L", lib, "-lhcache", f"-Wl,-rpath,{lib}"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "refusals ok" in run.stdout, run.stdout + run.stderr
