"""The kernels of the cache held in 8 bits as they are built: registers, scratch and LDS that their occupancy counts on."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2603_02170_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_02170_amd", "csrc")


@pytest.fixture(scope="module")
def assembly():
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "serve8.s")
        cmd = [build.hipcc_path(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "--cuda-device-only", "-S",
               os.path.join(CSRC, "serve8_api.hip"), "-o", out]
        res = subprocess.run(cmd, capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-2000:]
        return open(out).read()


@pytest.fixture(scope="module")
def kernels(assembly):
    assert not re.search(r"\bv_pk_(fma|mul|add)_f32\b", assembly)
    info = {}
    for block in assembly.split(".amdhsa_kernel ")[1:]:
        get = lambda key: int(re.search(key + r"\s+(\d+)", block).group(1))  # noqa: E731
        info[block.split("\n")[0].strip()] = dict(vgpr=get(r"\.amdhsa_next_free_vgpr"), scratch=get(r"\.amdhsa_private_segment_fixed_size"),
                                                  lds=get(r"\.amdhsa_group_segment_fixed_size"))
    return info


def _pick(kernels, stem, *bits):
    hits = [v for k, v in kernels.items() if stem in k and all(b in k for b in bits)]
    assert hits, (stem, bits)
    return hits


def test_two_workgroups_of_the_attention_of_few_rows_share_a_cu(kernels):
    for bits in ("ELi1EEEv", "ELi2EEEv"):
        for k in _pick(kernels, "cache8_attend_kernel", bits):
            assert k["vgpr"] <= 256 and k["scratch"] == 0 and 2 * k["lds"] <= 160 * 1024, k
    for bits in ("ELi3EEEv", "ELi4EEEv"):              # (one)
        for k in _pick(kernels, "cache8_attend_kernel", "ILi128", bits):
            assert k["vgpr"] <= 512 and k["scratch"] <= 64, k


def test_the_attention_of_many_rows_fits_a_cu(kernels):
    for stem in ("cache8_chunk_kernel", "cache8_wide_kernel"):
        for k in _pick(kernels, stem):
            assert k["vgpr"] <= 256 and k["lds"] <= 160 * 1024, (stem, k)
    for k in _pick(kernels, "cache8_chunk_kernel") + _pick(kernels, "cache8_wide_kernel", "ILi128E"):
        assert k["scratch"] == 0, k
    for k in _pick(kernels, "cache8_wide_kernel", "ILi64E"):           # two workgroups of eight waves
        assert k["vgpr"] <= 128 and 2 * k["lds"] <= 160 * 1024, k


def test_the_others_keep_their_registers(kernels):
    for stem in ("cache8_append_kernel", "cache8_read_kernel", "cache8_unpack_kernel", "cache8_join"):
        for k in _pick(kernels, stem):
            assert k["scratch"] == 0 and k["vgpr"] <= 128, (stem, k)


def test_only_the_rings_copies_use_m0(assembly):
    """The copies of the ring write m0 without the compiler's knowledge: nothing else of a kernel with a ring may use it."""
    rings, kernel, inside = set(), None, False
    for line in assembly.splitlines():
        label = re.match(r"(_ZN4sage\w+):", line)
        kernel = label.group(1) if label else kernel
        inside = "ASMSTART" in line or inside and "ASMEND" not in line
        if re.search(r"\bm0\b", line.split(";")[0]):
            assert inside, (kernel, line)
            rings.add(kernel)
    assert len(rings) == 2 and all("cache8_wide_kernel" in k for k in rings), rings


def test_what_is_spilled_does_not_grow(kernels):
    """Of heads of 64 the kernel whose keys are unpacked beforehand holds 128 registers for two workgroups a CU, and 29 words of a lane in scratch."""
    for k in _pick(kernels, "cache8_wide_kernel", "ILi64E"):
        assert k["scratch"] <= 116, k
    for k in _pick(kernels, "cache8_short_kernel"):
        assert k["scratch"] == 0 and k["vgpr"] <= 256 and 2 * k["lds"] <= 160 * 1024, k
