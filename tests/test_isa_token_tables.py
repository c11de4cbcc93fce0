"""tpla_commit_drafts may write its lengths over those it reads (CPU only, on the assembly of this build's own source): no wave stores
before all of the workgroup's have read."""
import re

from paper_2508_15881_amd import build as b


def test_lengths_are_read_by_all_waves_before_one_writes():
    asm = b.device_assembly("token_tables.hip")
    m = re.search(r"^(_ZN4tpla\w*commit_drafts_kernel\w*):(.*?)^\.Lfunc_end", asm, re.M | re.S)
    lines = [x.split(";")[0].strip() for x in m.group(2).splitlines()]
    barrier = next(i for i, x in enumerate(lines) if x.startswith("s_barrier"))
    store = next(i for i, x in enumerate(lines) if x.startswith(("global_store", "flat_store", "buffer_store")))
    assert barrier < store
