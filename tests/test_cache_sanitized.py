"""The host side of the cache's entry points (argument checks, the lists of forks and pools, launch plans) under AddressSanitizer and
UndefinedBehaviorSanitizer: the programs of refusals and limits, compiled together with the library's sources and with the
sanitizers on the HOST side only, run here, where there is no GPU."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2410_05004_amd", "csrc")


def test_cache_entry_points_under_sanitizers(tmp_path):
    cc = next((c for c in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc") if c and os.path.exists(c)), None)
    if cc is None:
        pytest.skip("hipcc not found")
    import torch
    if torch.cuda.is_available():
        pytest.skip("sanitizer builds run on GPU-less hosts only")
    from paper_2410_05004_amd.build import SOURCES
    sanitize = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize=function,vptr"]
    base = [cc, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-pthread", "-Xclang", "-target-feature", "-Xclang",
            "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"), "-I", CSRC, *sanitize]

    def compile_one(path):
        out = str(tmp_path / (os.path.basename(path) + ".o"))
        res = subprocess.run([*base, "-c", path, "-o", out], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-3000:]
        return out
    programs = ["cache_refusals", "cache_limits"]
    with ThreadPoolExecutor(max_workers=8) as pool:
        objects = list(pool.map(compile_one, [os.path.join(CSRC, s) for s in SOURCES] + [os.path.join(ROOT, "tests", p + ".cpp") for p in programs]))
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0 abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    for program, main in zip(programs, objects[len(SOURCES):]):
        exe = str(tmp_path / program)
        res = subprocess.run([cc, "--offload-arch=gfx950", "-pthread", *sanitize, *objects[: len(SOURCES)], main, "-o", exe], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-3000:]
        run = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
        print(run.stdout[-500:], run.stderr[-3000:])
        assert run.returncode == 0 and " ok" in run.stdout
        assert "Sanitizer" not in run.stderr and "runtime error" not in run.stderr, "a sanitizer reported a finding"
