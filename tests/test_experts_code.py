"""The experts' kernel as compiled: what its loads into LDS rely on."""
import os
import re

import pytest

from paper_2304_09049_amd.build import CSRC
from test_kernel_code import compile_listing


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    text = compile_listing(tmp_path_factory.mktemp("experts"), os.path.join(CSRC, "dg_experts_kernel.hip"))
    found = re.findall(r"^(\S*14experts_kernelILb\dELi\d\S+):(.*?)^\.Lfunc_end", text, re.M | re.S)
    assert len(found) == 6
    return found


def test_a_stage_reads_its_scales_before_others_may_come_to_their_place(kernels):
    """Two places of scales, four stages each: of five stages the last has the second place, and the next tile's first scales are asked for, into the first,
    with three stages in flight, while the fourth is multiplied."""
    for name, code in kernels:
        stage = code[code.rindex("s_barrier"):]                      # (the last one is the main loop's)
        loads, reads = stage.index("buffer_load"), [m.start() for m in re.finditer("ds_read_u8", stage)]
        assert len(reads) == 4 and max(reads) < loads, name
        assert "lgkmcnt(0)" in stage[max(reads):loads], name


def test_nothing_is_being_read_at_a_barrier(kernels):
    """Behind it every wavefront's loads go to the place of the stage before."""
    for name, code in kernels:
        at = [m.start() for m in re.finditer(r"\ts_barrier", code)]
        for a in at:
            before = code[:a].rsplit("s_waitcnt", 1)
            assert "lgkmcnt(0)" in before[1].split("\n")[0] and "ds_read" not in before[1], name
