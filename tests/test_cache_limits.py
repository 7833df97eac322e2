"""Sizes at the limits of the entry points of the 4-bit cache and of pages as a whole, without a GPU."""
import os
import shutil
import subprocess

import pytest

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
