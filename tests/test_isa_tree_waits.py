"""The drafted tokens' attention kernels (CPU only, on the assembly of this build's own source): they read LDS, multiply and keep their
accumulators in inline assembly, so what the compiler otherwise guarantees is checked here on every path through a kernel."""
import re

import pytest

from paper_2508_15881_amd import build as b
from test_isa_lds_waits import _LGKM_OP, _vgprs

MAX_COUNT = 15          # the most that an s_waitcnt can leave in flight


def parse(asm, part):
    """name -> (instructions as (text, inside inline assembly?), label -> index)."""
    out, cur, labels, in_asm = {}, None, None, False
    for line in asm.splitlines():
        m = re.match(r"^(_ZN4tpla\w*%s\w*):" % part, line)
        if m:
            cur, labels, in_asm = [], {}, False
            out[m.group(1)] = (cur, labels)
            continue
        if cur is None:
            continue
        t = line.strip()
        m = re.match(r"^(\.LBB\w+):", t)
        if m:
            labels[m.group(1)] = len(cur)
        elif t.startswith(";;#ASMSTART") or t.startswith(";;#ASMEND"):
            in_asm = t.startswith(";;#ASMSTART")
        elif t.startswith(".Lfunc_end"):
            cur = None
        else:
            t = t.split(";")[0].strip()
            if t and not t.startswith(".") and not t.endswith(":"):
                cur.append((t, in_asm))
    return out


def touched_too_early(insts, labels):
    """Follows every path with the LDS reads in flight, oldest first, as the counter sees them; returns the first instruction that
    touches the destination of an assembly read that no wait has covered."""
    seen, todo = set(), [(0, ())]
    while todo:
        i, flight = todo.pop()
        while i < len(insts):
            t, in_asm = insts[i]
            mnem = t.split()[0]
            if mnem == "s_endpgm":
                break
            if mnem == "s_branch" or mnem.startswith("s_cbranch"):
                target = (labels[t.split()[1]], flight)
                if target not in seen:
                    seen.add(target)
                    todo.append(target)
                if mnem == "s_branch":
                    break
                i += 1
                continue
            if mnem == "s_waitcnt":
                m = re.search(r"lgkmcnt\((\d+)\)", t)
                if m:
                    n = int(m.group(1))
                    flight = flight[len(flight) - n:] if 0 < n < len(flight) else flight if n else ()
                elif "vmcnt" not in t and "expcnt" not in t:
                    flight = ()
                i += 1
                continue
            unsafe = set().union(*flight) if flight else set()
            if unsafe and _vgprs(t[len(mnem):]) & unsafe:
                return i, t
            if _LGKM_OP.match(mnem):
                dest = frozenset(_vgprs(t[len(mnem):].split(",")[0])) if in_asm and mnem.startswith("ds_read") else frozenset()
                flight = flight + (dest,)
                while flight and not flight[0]:
                    flight = flight[1:]             # an old operation without a destination of ours says nothing more
            i += 1
    return None


def test_the_walk_sees_paths():
    read, use, wait = ("ds_read_b128 v[4:7], v1", True), ("v_add_f32 v9, v4, v5", False), ("s_waitcnt lgkmcnt(0)", True)
    end = ("s_endpgm", False)
    skip = [read, ("s_cbranch_scc1 .LBB0_1", False), wait, use, end]
    assert touched_too_early(skip, {".LBB0_1": 3}) == (3, use[0])          # the branch jumps over the wait
    assert touched_too_early([read, wait, ("s_cbranch_scc1 .LBB0_1", False), use, end], {".LBB0_1": 3}) is None
    # laid out in between, but on a path of its own
    assert touched_too_early([read, ("s_branch .LBB0_2", False), use, end, wait, use, end], {".LBB0_1": 2, ".LBB0_2": 4}) is None
    # a loop whose last read is used a turn later without a wait
    assert touched_too_early([use, read, ("s_cbranch_scc1 .LBB0_0", False), wait, end], {".LBB0_0": 0}) == (0, use[0])


@pytest.fixture(scope="module")
def assembly():
    return b.device_assembly("tree_mfma.hip")


def test_no_path_touches_an_lds_read_before_its_wait(assembly):
    kernels = parse(assembly, "tree")
    assert len(kernels) >= 8, sorted(kernels)
    for name, (insts, labels) in kernels.items():
        assert sum(in_asm and t.startswith("ds_read") for t, in_asm in insts) >= 16, name
        assert touched_too_early(insts, labels) is None, name


def test_the_accumulation_registers_are_the_kernels_own(assembly):
    """No instruction of the compiler's reads or writes one."""
    for name, (insts, _) in parse(assembly, "tree_mfma_kernel").items():
        theirs = [t for t, in_asm in insts if not in_asm and (re.search(r"\ba(\d+|\[\d+:\d+\])", t) or "accvgpr" in t)]
        assert not theirs, (name, theirs[0])


def test_ordinary_writes_are_two_wait_states_ahead_of_matrix_reads(assembly):
    for name, (insts, _) in parse(assembly, "tree_mfma_kernel").items():
        for k, (t, _) in enumerate(insts):
            if not t.startswith("v_mfma"):
                continue
            reads = set()
            for part in t.split(None, 1)[1].split(", ")[1:]:
                m = re.fullmatch(r"v\[(\d+):(\d+)\]", part.strip())
                reads |= set(range(int(m.group(1)), int(m.group(2)) + 1)) if m else set()
            states = 0                               # each instruction in between is at least one
            for u, _ in reversed(insts[max(0, k - 3):k]):
                if states >= 2:
                    break
                if u.startswith("v_") and not u.startswith("v_mfma"):
                    m = re.match(r"\S+ v(?:\[(\d+):(\d+)\]|(\d+))", u)
                    w = set(range(int(m.group(1)), int(m.group(2)) + 1)) if m and m.group(1) else {int(m.group(3))} if m else set()
                    assert not (w & reads), (name, u, t)
                states += 1 + (int(u.split()[1]) if u.startswith("s_nop") else 0)


def test_nothing_is_kept_in_scratch_memory(assembly):
    """A reload in the loop waits for the tiles that are on their way."""
    sizes = re.findall(r"\.name:\s+(\S*tree\w+kernel\S*).*?\.private_segment_fixed_size:\s+(\d+)", assembly, flags=re.S)
    assert {n for n, _ in sizes} == set(parse(assembly, "tree")) and all(int(v) == 0 for _, v in sizes), sizes
