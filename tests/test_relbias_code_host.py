"""The attention with a relative position bias copies its tiles to LDS by instructions that the compiler's hazard tables know nothing of.  In the built
code every such copy brings the wait states itself that a buffer load needs behind a vector instruction that wrote one of its scalar registers (five), and sets
M0 right before; and what the kernels of many tokens keep for their loops stays in registers."""
import os

import pytest

from gpu_code import code_objects, listings, resources
from paper_2405_01248_amd import build

WAIT_STATES = 5


@pytest.fixture(scope="module")
def objects(tmp_path_factory):
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    return [o for o in code_objects(tmp_path_factory.mktemp("co")) if any("rel_fwd" in n for n in resources(o))]


def test_every_copy_to_lds_brings_its_wait_states(objects):
    copies = 0
    for o in objects:
        for name, lines in listings(o, lambda n: "rel_" in n and "bf16" in n):
            states, m0 = 0, False
            for line in lines:
                if line.startswith("buffer_load") and line.endswith("lds"):
                    copies += 1
                    assert m0 and states >= WAIT_STATES, (name, line)
                    m0 = False
                if line.startswith("s_mov_b32 m0,"):
                    states, m0 = 1, True
                elif line.startswith("s_nop"):
                    states += 1 + int(line.split()[1])
                elif line.startswith("v_"):
                    states = 0
                else:
                    states += 1
    assert copies > 50, copies


def test_no_packed_fp32_and_no_scratch_in_the_loops_over_many_tokens(objects):
    for o in objects:
        for name, r in resources(o).items():
            if "rel_fwd_bf16" in name or "rel_bwd_dq_bf16" in name:
                assert r["private_segment_fixed_size"] == 0 and r["vgpr_spill_count"] == 0, (name, r)
        for name, lines in listings(o, lambda n: "rel_" in n):
            assert not any(line.startswith(("v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32")) for line in lines), name
