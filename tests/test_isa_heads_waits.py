"""The grouped-head attention kernels (CPU only, on the assembly of this build's own source): they read LDS in inline assembly, and those for
prompts multiply there and keep their accumulators in registers of their choice, so what the compiler otherwise guarantees is checked on every path."""
import re

import pytest

import test_isa_tree_results as results
from paper_2508_15881_amd import build as b
from test_isa_tree_waits import parse, touched_too_early

INSTANCES = {"heads_ranges": 4, "heads_prompts": 8}


@pytest.fixture(scope="module")
def assembly():
    return {s: b.device_assembly(s + ".hip") for s in INSTANCES}


@pytest.mark.parametrize("source", INSTANCES)
def test_no_read_is_used_before_its_wait(assembly, source):
    kernels = parse(assembly[source], source + "_kernel")
    assert len(kernels) == INSTANCES[source]
    for name, (insts, labels) in kernels.items():
        assert sum(in_asm and t.startswith("ds_read") for t, in_asm in insts) >= 16, name
        assert touched_too_early(insts, labels) is None, name


def test_matrix_instructions_have_their_wait_states(assembly):
    for name, (insts, labels) in parse(assembly["heads_prompts"], "heads_prompts_kernel").items():
        assert sum(in_asm and t.startswith("v_mfma") for t, in_asm in insts) >= 24, name
        assert all(in_asm for t, in_asm in insts if t.startswith("v_mfma")), name
        assert results.touched_too_early(insts, labels) is None, name
        assert results.written_too_late(insts, labels) is None, name


def test_the_accumulation_registers_are_the_kernels_own(assembly):
    """No instruction of the compiler's touches v192 to v255, and there are no accumulation registers."""
    mine = {("v", k) for k in range(192, 256)}
    for name, (insts, _) in parse(assembly["heads_prompts"], "heads_prompts_kernel").items():
        theirs = [t for t, in_asm in insts if not in_asm and results.registers(t) & mine]
        assert not theirs, (name, theirs[0])
        assert not any(kind == "a" for t, _ in insts for kind, _ in results.registers(t)), name


def test_nothing_of_the_prompt_kernels_is_kept_in_scratch_memory(assembly):
    """A reload in the loop waits for the tiles that are on their way."""
    sizes = re.findall(r"\.name:\s+(\S*heads_prompts_kernel\S*).*?\.private_segment_fixed_size:\s+(\d+)", assembly["heads_prompts"], flags=re.S)
    assert len(sizes) == INSTANCES["heads_prompts"] and all(int(v) == 0 for _, v in sizes), sizes
