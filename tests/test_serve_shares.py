"""The cache attention's kernels as their sources have them: the functions that deal the work out, run on the host, and the register that the
copies of their rings write (no GPU needed)."""
import os
import re
import subprocess

from paper_2603_02170_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_02170_amd", "csrc")


def test_every_unit_is_dealt_once_by_the_kernels_own_functions(tmp_path):
    exe = str(tmp_path / "serve_shares")
    cmd = [build.hipcc_path(), "-x", "hip", "--cuda-host-only", "-O1", "-std=c++17", "-I", CSRC, os.path.join(ROOT, "tests", "serve_shares.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


def test_only_the_rings_copies_use_m0(tmp_path):
    """ring_copy writes m0 without the compiler's knowledge (a clobber of it is not honoured): nothing else of a kernel with a ring may use it."""
    out = str(tmp_path / "serve.s")
    cmd = [build.hipcc_path(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "--cuda-device-only", "-S",
           os.path.join(CSRC, "serve_api.hip"), "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    rings = set()
    kernel, inside = None, False
    for line in open(out):
        label = re.match(r"(_ZN4sage\w+):", line)
        kernel = label.group(1) if label else kernel
        inside = "ASMSTART" in line or inside and "ASMEND" not in line
        if re.search(r"\bm0\b", line.split(";")[0]):
            assert inside, (kernel, line)
            rings.add(kernel)
    assert len(rings) == 12 and all("cache_attend_kernel" in k or "cache_wide_kernel" in k for k in rings), rings
