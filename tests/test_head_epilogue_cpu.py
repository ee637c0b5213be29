"""A rule of csrc/tli_head.cu that no run can show to be kept: the loads from tensor memory and the barrier of the epilogue are instructions
that a whole warp has to take together, so behind what one lane does alone (an arrival, a store) the warp meets again."""
import os
import re

from rows_on_cpu import CSRC


def epilogue():
    src = open(os.path.join(CSRC, "tli_head.cu")).read()
    body = src[src.index("tli_head_gemm_kernel(const __grid_constant__"):src.index("// ---- rows and targets ----")]
    return [re.sub(r"//.*", "", line).strip() for line in body[body.index("slab_put ="):].splitlines()]


def test_the_warp_meets_behind_one_lane():
    lines, alone = epilogue(), 0
    for i, line in enumerate(lines):
        if not line.startswith("if (lane == 0)"):
            continue
        end = i
        if line.endswith("{"):
            depth = 1
            while depth:
                end += 1
                depth += lines[end].count("{") - lines[end].count("}")
        alone += 1
        assert lines[end + 1] in ("__syncwarp();", "}") and "__syncwarp();" in lines[end + 1:end + 3], (line, lines[end + 1])
    assert alone == 7                                                        # a slab free, a sum there and read, three stores, the last copies


def test_stores_by_one_lane_stand_before_a_commit():
    lines = epilogue()
    stores = [i for i, line in enumerate(lines) if line.startswith("if (store)")]
    assert len(stores) == 3 and all(lines[i + 1].startswith("if (lane == 0)") and "commit_group" in lines[i + 1] for i in stores)
