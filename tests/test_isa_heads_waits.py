"""The grouped-head attention kernels (CPU only, on the assembly of this build's own source): on every path, nothing touches the destination of an
LDS read in inline assembly before a wait has covered it."""
import pytest

from paper_2508_15881_amd import build as b
from test_isa_tree_waits import parse, touched_too_early


@pytest.mark.parametrize("source,part,instances", [("heads_ranges.hip", "heads_ranges_kernel", 6), ("heads_prompts.hip", "heads_prompts_kernel", 4)])
def test_no_read_is_used_before_its_wait(source, part, instances):
    kernels = parse(b.device_assembly(source), part)
    assert len(kernels) == instances
    for name, (insts, labels) in kernels.items():
        assert sum(in_asm and t.startswith("ds_read") for t, in_asm in insts) >= 16, name
        assert touched_too_early(insts, labels) is None, name
