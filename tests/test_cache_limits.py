"""Sizes at the limits of the entry points of the 4-bit cache and of pages as a whole, without a GPU."""
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

import oracle.kv4_oracle as kv4
import synthetic as syn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_limits_on_the_host(tmp_path):
    """Sizes whose products pass 32 bits are refused, on contexts whose device pointers are never followed."""
    cc = next((c for c in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc") if c and os.path.exists(c)), None)
    if cc is None:
        pytest.skip("hipcc not found")
    import paper_2410_05004_amd as hc
    exe = str(tmp_path / "cache_limits")
    lib = os.path.dirname(hc.lib_path())
    r = subprocess.run([cc, "-x", "hip", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                        "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2410_05004_amd", "csrc"),
                        os.path.join(ROOT, "tests", "cache_limits.cpp"), "-o", exe, "-L", lib, "-lhcache", f"-Wl,-rpath,{lib}"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "limits ok" in run.stdout, run.stdout + run.stderr


@pytest.mark.parametrize("n_q,n_kv,hd", [(32, 8, 128), (64, 8, 128), (40, 40, 128), (14, 2, 64), (4, 4, 64), (34, 1, 64), (16, 8, 256), (600, 600, 64)])
def test_one_workspace_for_all_batches(n_q, n_kv, hd):
    """A workspace of the bound of the largest batch serves every smaller one, although these may need more than the largest itself."""
    import paper_2410_05004_amd as hc
    desc = hc.ModelDesc(1, 256, n_q, n_kv, hd, 16, 4096, 2, 1e4, 1e-5, 0)
    rng = random.Random(n_q + hd)

    def size(hi):
        return rng.choice([hi, rng.randint(0, hi), int(hi ** rng.random())])
    for _ in range(60):
        most_q, most_kv = size(2 ** 31 // n_q // 64), size(2 ** 20)
        bound = hc.attend_kv4_workspace_bound(desc, most_q, most_kv)
        assert bound <= 36 << 20
        assert hc.attend_kv4_workspace_bound(desc, size(most_q), size(most_kv)) <= bound
        for _ in range(60):
            total_q = size(most_q)
            n_seq, max_q = size(min(65535, max(total_q, 1))), size(max(total_q, 1))
            assert hc.attend_kv4_workspace(desc, n_seq, total_q, max_q, size(most_kv)) <= bound
    if (n_q, n_kv) == (32, 8):
        assert hc.attend_kv4_workspace(desc, 64, 64, 1, 8192) > hc.attend_kv4_workspace(desc, 256, 256, 1, 8192)
        assert hc.attend_kv4_workspace_bound(desc, 256, 8192) >= hc.attend_kv4_workspace(desc, 64, 64, 1, 8192)
    assert hc.attend_kv4_workspace_bound(desc, 0, 1 << 20) == hc.attend_kv4_workspace_bound(desc, 1 << 10, 0) == 0
    for args in ((-1, 1), (1, -1)):
        with pytest.raises(hc.HCacheError) as e:
            hc.attend_kv4_workspace_bound(desc, *args)
        assert e.value.status == hc.HC_EINVAL


def test_where_the_scale_ends():
    """Every finite bf16 value as a group's largest: at most half a step from its code up to 7 * 2^125, 6 * 2^125 beyond; the smallest
    scale that reaches it, or 2^-125."""
    bits = np.arange(1, 0x7F80, dtype=np.uint16)
    top = syn.bf16_bits_to_f64(bits)
    x = np.zeros((len(top), 32))
    x[:, 0], x[:, 1] = top, -0.7 * top
    code, scale = kv4.quantize(x)
    got, s = kv4.dequantize(code, scale), 2.0 ** (scale[:, 0].astype(np.float64) - 127)
    ends = top > 7 * 2.0 ** 125
    assert 10 < ends.sum() < 128
    assert np.all(got[ends, 0] == 6 * 2.0 ** 125) and np.all(s[ends] == 2.0 ** 125)
    for c in (0, 1):
        y, far = np.abs(x[~ends, c]) / s[~ends], np.abs(got[~ends, c] - x[~ends, c]) / s[~ends]
        step = np.select([y < 2, y < 4], [0.5, 1], 2)
        assert np.all(far <= step / 2)
    assert np.all((top <= 7 * s) | ends) and np.all((top > 3.5 * s) | (s == 2.0 ** -125))
