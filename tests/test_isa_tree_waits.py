"""The drafted tokens' attention kernels read LDS from inline assembly: no instruction touches such a read before its wait, and
nothing is kept in scratch memory (CPU only)."""
import re

from paper_2508_15881_amd import build as b
from test_isa_lds_waits import _kernels, check_kernel


def test_tree_kernels():
    asm = b.device_assembly("tree_mfma.hip")
    kernels = {n: i for n, i in _kernels(asm).items() if "tree_mfma_kernel" in n}
    assert len(kernels) >= 4, sorted(kernels)
    for name, insts in kernels.items():
        assert sum(in_asm and t.startswith("ds_read") for t, in_asm in insts) >= 16, name
        bad = check_kernel(insts)
        assert not bad, (name, bad[0])
    sizes = re.findall(r"\.name:\s+(\S*tree_mfma_kernel\S*).*?\.private_segment_fixed_size:\s+(\d+)", asm, flags=re.S)
    assert len({n for n, _ in sizes}) == len(kernels) and all(int(v) == 0 for _, v in sizes), sizes
