"""What the host's choices of grids count on, read from the built code of the training operators: how many workgroups the registers of a CU hold."""
import os
import re

import pytest

from gpu_code import code_objects, resources
from paper_2405_01248_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    out = {}
    for o in code_objects(tmp_path_factory.mktemp("co")):
        out.update(resources(o))
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
