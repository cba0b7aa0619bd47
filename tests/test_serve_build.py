"""The kernels of sagebwd_serve.h as they are built: registers, scratch and LDS that their occupancy counts on, no packed FP32 instruction, and the
arithmetic of how work is dealt out, gone through on the host."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2603_02170_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_02170_amd", "csrc")


@pytest.fixture(scope="module")
def kernels():
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "serve.s")
        cmd = [build.hipcc_path(), "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "--cuda-device-only", "-S",
               os.path.join(CSRC, "serve_api.hip"), "-o", out]
        res = subprocess.run(cmd, capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-2000:]
        text = open(out).read()
    assert not re.search(r"\bv_pk_(fma|mul|add)_f32\b", text)
    info = {}
    for block in text.split(".amdhsa_kernel ")[1:]:
        get = lambda key: int(re.search(key + r"\s+(\d+)", block).group(1))  # noqa: E731
        info[block.split("\n")[0].strip()] = dict(vgpr=get(r"\.amdhsa_next_free_vgpr"), scratch=get(r"\.amdhsa_private_segment_fixed_size"),
                                                  lds=get(r"\.amdhsa_group_segment_fixed_size"))
    return info


def _pick(kernels, stem, *bits):
    hits = [v for k, v in kernels.items() if stem in k and all(b in k for b in bits)]
    assert hits, (stem, bits)
    return hits


def test_two_workgroups_of_the_attention_of_few_rows_share_a_cu(kernels):
    for k in _pick(kernels, "cache_attend_kernel"):
        assert k["vgpr"] <= 256 and 2 * k["lds"] <= 160 * 1024, k
    for d in ("ILi64E", "ILi128E"):
        for k in _pick(kernels, "cache_attend_kernel", d, "ELi1EEEv"):
            assert k["scratch"] == 0 and k["vgpr"] <= (168 if d == "ILi64E" else 208), k
    # two tiles of queries, groups of 32 at d = 128: some registers parked
    for k in _pick(kernels, "cache_attend_kernel", "ELi2EEEv"):
        assert k["scratch"] <= 192, k


def test_the_attention_of_many_rows_keeps_its_operands_in_registers(kernels):
    for k in _pick(kernels, "cache_chunk_kernel"):
        assert k["scratch"] == 0 and k["vgpr"] <= 256 and k["lds"] <= 160 * 1024, k
    for k in _pick(kernels, "cache_wide_kernel", "ILi128E"):
        assert k["scratch"] == 0 and k["vgpr"] <= 256 and k["lds"] <= 160 * 1024, k
    for k in _pick(kernels, "cache_wide_kernel", "ILi64E"):           # two workgroups of eight waves
        assert k["scratch"] <= 64 and k["vgpr"] <= 128 and 2 * k["lds"] <= 160 * 1024, k


def test_the_others_fill_a_cu(kernels):
    for stem in ("cache_append_kernel", "cache_read_kernel", "cache_unpack_kernel", "rotary_kernel", "cache_join_kernel", "cache_plan", "cache_trim"):
        for k in _pick(kernels, stem):
            assert k["scratch"] == 0 and k["vgpr"] <= 72, (stem, k)


def _shares(total, workgroups):
    """AttendShares, in Python: what begin() and owner() return is asserted against the dealing itself."""
    n = min(workgroups, total)
    each, more = total // n, total % n
    begin = lambda w: each * w + min(w, more)  # noqa: E731

    def owner(unit):
        big = (each + 1) * more
        return unit // (each + 1) if unit < big else more + (unit - big) // each
    return n, begin, owner


@pytest.mark.parametrize("cost", [2, 6])
def test_every_unit_is_dealt_once_and_every_divided_item_joined_once(cost):
    """How items (of u units and `cost` in front) are cut into shares, and which border leaves word for the joining launch."""
    import random
    rng = random.Random(cost)
    cut = lambda offset: max(0, offset - cost)  # noqa: E731
    for trial in range(300):
        items = [rng.choice([1, 1, 2, rng.randint(1, 9), rng.randint(1, 200)]) for _ in range(rng.randint(1, 40))]
        starts = [sum(items[:i]) + cost * i for i in range(len(items) + 1)]
        total = starts[-1]
        n, begin, owner = _shares(total, rng.choice([1, 3, 8, 256, 512]))
        assert begin(0) == 0 and begin(n) == total and all(begin(w) < begin(w + 1) for w in range(n))
        parts, joins = {}, {}
        for w in range(n):
            b, e = begin(w), begin(w + 1)
            i = max(k for k in range(len(items)) if starts[k] <= b)
            x, j0 = starts[i], cut(b - starts[i])
            if cut(e - x) <= j0:
                continue
            if j0 > 0 and cut(begin(w - 1) - x) == 0:
                joins[i] = (w, owner(x + items[i] + cost - 1) - w + 2)
            while i < len(items) and cut(e - x) > j0:
                j1 = min(items[i], cut(e - x))
                parts.setdefault(i, []).append((w, j0, j1))
                if j1 < items[i]:
                    break
                x += items[i] + cost
                i, j0 = i + 1, 0
        for i, u in enumerate(items):
            assert [p[1] for p in parts[i]] == [0] + [p[2] for p in parts[i]][:-1] and parts[i][-1][2] == u
            if len(parts[i]) > 1:
                ws = [p[0] for p in parts[i]]
                assert ws == list(range(ws[0], ws[0] + len(ws)))                 # neighbours, in the order of the keys
                assert joins[i] == (ws[1], len(ws))
            else:
                assert i not in joins


def test_the_rows_of_a_head_are_taken_from_both_ends():
    for tiles in range(1, 40):
        at = [tiles - 1 - p // 2 if p % 2 else p // 2 for p in range(tiles)]
        assert sorted(at) == list(range(tiles))


def test_the_attention_of_up_to_128_rows_fits_a_cu(kernels):
    for k in _pick(kernels, "cache_span_kernel"):
        assert k["vgpr"] <= 256 and k["lds"] <= 160 * 1024 and k["scratch"] <= 96, k
    for k in _pick(kernels, "cache_span_kernel", "ELi4EEEv") + _pick(kernels, "cache_span_kernel", "ILi64E"):
        assert k["scratch"] == 0, k
