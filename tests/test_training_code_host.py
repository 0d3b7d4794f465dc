"""What the host's choices of grids count on, read from the built code of the training operators: how many workgroups a CU holds, by registers and LDS."""
import os
import re
import subprocess

import pytest

from gpu_code import LLVM, code_objects, resources
from paper_2405_01248_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    out = {}
    for o in code_objects(tmp_path_factory.mktemp("co")):
        out.update(resources(o))
        notes = subprocess.run([os.path.join(LLVM, "llvm-readelf"), "--notes", o], check=True, capture_output=True, text=True).stdout
        for kernel in re.split(r"\n\s+- \.agpr_count", notes)[1:]:
            name = re.search(r"\.symbol:\s*(\S+)", kernel)[1].strip("'").removesuffix(".kd")
            out[name]["lds"] = int(re.search(r"\.group_segment_fixed_size:\s*(\d+)", kernel)[1])
    return out


def _workgroups_a_cu(vgprs, threads):
    """By registers: 512 a lane of each of the four SIMDs, handed out in eights, eight waves a SIMD at most."""
    return min(8, 512 // ((vgprs + 7) // 8 * 8)) * 4 // (threads // 64)


def test_layernorm_backward_runs_as_many_workgroups_at_once_as_its_grid_has(kernels):
    # workgroups a CU that the grid is sized by, for lanes of a row and groups of columns a lane
    wanted = {(16, 1): 3, (32, 1): 3, (64, 1): 3, (64, 2): 2, (256, 1): 4, (512, 1): 2, (1024, 1): 1}
    seen = 0
    for name, r in kernels.items():
        m = re.search(r"norm_bwd_kernelI\w+?Li(\d+)ELi(\d+)EE", name)
        if not m:
            continue
        lanes, groups = int(m[1]), int(m[2])
        seen += 1
        assert r["private_segment_fixed_size"] == 0, name
        assert _workgroups_a_cu(r["vgpr_count"], max(256, lanes)) >= wanted[lanes, groups], (name, r)
    assert seen == 3 * len(wanted), seen


def _lds_a_cu(bytes_of_lds):
    """160 KB, handed out in steps of 1280 bytes."""
    return 160 * 1024 // ((bytes_of_lds + 1279) // 1280 * 1280)


def test_relbias_workgroups_a_cu(kernels):
    """By registers as many as the rules take at most; the LDS without the bias is what they add the bias to.  Bytes of the bias and of the sums by distance: nine floats
    an entry, 4 * 376 of them with 32 buckets to 128 distances of both directions, 4 * 628 with 64 to 256."""
    wanted = {  # pattern: (threads, LDS by width, workgroups a CU by registers)
        r"rel_bwd_few_(?:dq|dkv|both)_bf16_kernelILi(\d+)": (256, {64: 1024 * 64 + 2096, 96: 1024 * 96 + 2096}, {64: 2, 96: 1}),
        r"rel_bwd_dq_bf16_kernelILi(\d+)": (256, {64: 512 * 64 + 1072, 96: 512 * 96 + 1072}, {64: 3, 96: 2}),
        r"rel_bwd_dkv_bf16_kernelILi(\d+)ELi\d+ELi3E": (256, {64: 768 * 64 + 1024}, {64: 3}),
        r"rel_fwd_bf16_kernelILi(\d+)": (256, {64: 512 * 64, 96: 512 * 96}, {64: 4, 96: 3}),
    }
    for pattern, (threads, lds, workgroups) in wanted.items():
        found = [(int(m[1]), r, n) for n, r in kernels.items() if (m := re.search(pattern, n))]
        assert found, pattern
        for width, r, name in found:
            assert r["lds"] <= lds[width] <= r["lds"] + 1100, (name, r)
            assert _workgroups_a_cu(r["vgpr_count"], threads) >= workgroups[width], (name, r)
    small, large = 9 * 4 * 376, 9 * 4 * 628
    assert _lds_a_cu(1024 * 64 + 2096 + small) == 2 and _lds_a_cu(1024 * 64 + 2096 + large) == 1
    assert _lds_a_cu(512 * 64 + 1072 + small) == 3 and _lds_a_cu(512 * 64 + 1072 + large) == 2


def test_what_the_relative_bias_leaves_in_scratch(kernels):
    """Nothing, but for the three waves a SIMD of dK / dV and the wide heads of the kernel that has all keys: no more than their comments say."""
    known = {r"rel_bwd_dkv_bf16_kernelILi64ELi4ELi3E": (5, 24), r"rel_bwd_dkv_bf16_kernelILi64ELi3ELi3E": (2, 12), r"rel_bwd_short_bf16_kernelILi96E": (23, 96)}
    seen = 0
    for name, r in kernels.items():
        if not re.search(r"rel_(fwd|bwd|join|dtable)", name):
            continue
        seen += 1
        registers, scratch = next((v for k, v in known.items() if re.search(k, name)), (0, 0))
        assert r["vgpr_spill_count"] <= registers and r["private_segment_fixed_size"] <= scratch, (name, r)
    assert seen > 50, seen
