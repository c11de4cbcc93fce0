"""The drafted tokens' attention kernel multiplies in inline assembly (CPU only, on the assembly of this build's own source): the compiler
does not know how long a result is on its way, so that nothing touches one too early is checked here on every path through the kernel."""
import re

import pytest

from paper_2508_15881_amd import build as b
from test_isa_tree_waits import parse

STATES = 11             # wait states between a 16x16x32 matrix instruction and an ordinary one that touches its result

_N = r"(0x[0-9a-f]+|\d+)"
_REG = re.compile(r"\b([va])(?:\[%s(?::%s)?\]|(\d+))" % (_N, _N))


def registers(text):
    """v7, v[4:7], a[0x40:0x43], a[0x40]."""
    out = set()
    for kind, lo, hi, one in _REG.findall(text):
        first = int(lo or one, 0)
        out |= {(kind, k) for k in range(first, int(hi, 0) + 1 if hi else first + 1)}
    return frozenset(out)


def walk(insts, labels, touches, gives):
    """Follows every path with what is on its way (register -> wait states left, an instruction is at least one); returns the first instruction that
    touches such a register.  gives: the registers that an instruction puts on their way, and for how many states."""
    seen, todo = set(), [(0, frozenset())]
    while todo:
        i, start = todo.pop()
        pending = dict(start)
        while i < len(insts):
            t, in_asm = insts[i]
            mnem = t.split()[0]
            if mnem == "s_endpgm":
                break
            if pending and any(r in pending for r in touches(t)):
                return i, t
            passed = 1 + (int(t.split()[1], 0) if mnem == "s_nop" else 0)
            pending = {r: n - passed for r, n in pending.items() if n > passed}
            new, states = gives(t, in_asm)
            pending.update({r: states for r in new})
            if mnem == "s_branch" or mnem.startswith("s_cbranch"):
                target = (labels[t.split()[1]], frozenset(pending.items()))
                if target not in seen:
                    seen.add(target)
                    todo.append(target)
                if mnem == "s_branch":
                    break
            i += 1
    return None


def matrix_parts(t):
    return [registers(x) for x in t.split(None, 1)[1].split(", ")] if t.startswith("v_mfma") else None


def touched_too_early(insts, labels):
    """Results of assembly matrix instructions.  Another that adds to the very same registers may follow at once."""
    def touches(t):
        parts = matrix_parts(t)
        if parts is None:
            return registers(t)
        return (parts[1] | parts[2]) if parts[3] == parts[0] else parts[0] | parts[1] | parts[2] | parts[3]

    return walk(insts, labels, touches, lambda t, in_asm: (matrix_parts(t)[0], STATES) if in_asm and t.startswith("v_mfma") else ((), 0))


def written_too_late(insts, labels):
    """Operands of assembly matrix instructions, written by ordinary ones: two states.  (The registers of loads are the waits' business.)"""
    def gives(t, in_asm):
        return (registers(t.split(None, 1)[1].split(", ")[0]), 2) if t.startswith("v_") and not t.startswith(("v_mfma", "v_cmp", "v_read", "v_nop")) else ((), 0)

    return walk(insts, labels, lambda t: frozenset().union(*matrix_parts(t)[1:]) if t.startswith("v_mfma") else (), gives)


MM, END = ("v_mfma_f32_16x16x32_bf16 v[0:3], v[10:13], v[20:23], v[0:3]", True), ("s_endpgm", False)
OUT = ("v_mfma_f32_16x16x32_bf16 a[0:3], v[10:13], v[20:23], a[0:3]", True)
FAR = ("v_mfma_f32_16x16x32_bf16 a[0x40:0x43], v[10:13], v[20:23], a[0x40:0x43]", True)


@pytest.mark.parametrize("between,use,fails", [
    ([], "v_max_f32_e32 v9, v3, v8", True), ([("s_nop 9", True)], "v_max_f32_e32 v9, v3, v8", True), ([("s_nop 10", True)], "v_max_f32_e32 v9, v3, v8", False),
    ([("v_add_u32_e32 v7, 1, v7", False)] * 10, "v_mov_b32_e32 v2, 0", True), ([("v_add_u32_e32 v7, 1, v7", False)] * 11, "v_mov_b32_e32 v2, 0", False),
    ([], "v_mov_b32_e32 v4, 0", False), ([MM], "v_mov_b32_e32 v4, 0", False), ([("s_nop 15", True), MM], "v_mov_b32_e32 v0, v4", True),
    ([], "v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[20:23], v[4:7]", True), ([], "v_mfma_f32_16x16x32_bf16 v[0:3], v[10:13], v[20:23], 0", True),
    ([], "global_store_dwordx4 v[30:31], v[0:3], off", True), ([OUT, ("s_nop 10", True)], "v_accvgpr_read_b32 v9, a2", False),
    ([("s_nop 15", True), OUT, ("s_nop 5", True)], "v_accvgpr_read_b32 v9, a2", True), ([("s_nop 15", True), FAR, ("s_nop 5", True)], "v_accvgpr_read_b32 v9, a[0x42]", True), ([("s_nop 15", True), OUT], "v_accvgpr_write_b32 a0, v9", True),
])
def test_the_walk_counts_states(between, use, fails):
    insts = [MM] + between + [(use, False), END]
    found = touched_too_early(insts, {})
    assert found == ((len(insts) - 2, use) if fails else None)


def test_the_walk_sees_paths():
    use, nop, add = ("v_max_f32_e32 v9, v3, v8", False), ("s_nop 15", True), ("v_add_u32_e32 v7, 1, v7", False)
    assert touched_too_early([MM, ("s_cbranch_scc1 .LBB0_1", False), nop, use, END], {".LBB0_1": 3}) == (3, use[0])      # the branch jumps over the wait
    assert touched_too_early([MM, nop, ("s_cbranch_scc1 .LBB0_1", False), use, END], {".LBB0_1": 3}) is None
    assert touched_too_early([add, use, MM, ("s_cbranch_scc1 .LBB0_0", False), nop, END], {".LBB0_0": 0}) == (1, use[0])  # used a turn later
    assert touched_too_early([nop, use, MM, ("s_cbranch_scc1 .LBB0_0", False), nop, END], {".LBB0_0": 0}) is None
    # a matrix instruction of the compiler's has the compiler's waits
    assert touched_too_early([(MM[0], False), use, END], {}) is None


@pytest.mark.parametrize("between,fails", [([], True), (["s_nop 0"], True), (["s_nop 1"], False), (["v_add_u32_e32 v7, 1, v7"] * 2, False)])
@pytest.mark.parametrize("write", ["v_cvt_pk_bf16_f32 v20, v4, v5", "v_mov_b32_e32 v11, 0", "v_accvgpr_write_b32 a[2], 0", "v_mul_f32 v3, v3, v4"])
def test_the_walk_counts_states_behind_writes(write, between, fails):
    product = OUT[0] if "accvgpr" in write else MM[0]
    insts = [(write, False)] + [(t, False) for t in between] + [(product, True), END]
    assert (written_too_late(insts, {}) is not None) == fails
    assert (written_too_late([("s_cbranch_scc1 .LBB0_2", False)] + insts, {".LBB0_2": 1 + len(between) + 1}) is not None) == fails


@pytest.fixture(scope="module")
def kernels():
    return parse(b.device_assembly("tree_mfma.hip"), "tree_mfma_kernel")


def test_no_path_touches_a_result_on_its_way(kernels):
    assert len(kernels) == 7, sorted(kernels)
    for name, (insts, labels) in kernels.items():
        assert sum(in_asm and t.startswith("v_mfma") for t, in_asm in insts) >= 16, name
        assert touched_too_early(insts, labels) is None, name


def test_no_path_multiplies_what_was_just_written(kernels):
    for name, (insts, labels) in kernels.items():
        assert written_too_late(insts, labels) is None, name


def test_a_use_that_is_moved_up_is_found(kernels):
    """Planted in a copy of the listing, behind matrix instructions all over the kernel."""
    for name, (insts, labels) in kernels.items():
        at = [i for i, (t, in_asm) in enumerate(insts) if in_asm and t.startswith("v_mfma")]
        for i in at[::max(1, len(at) // 6)]:
            kind, n = sorted(registers(insts[i][0].split(None, 1)[1].split(", ")[0]))[0]
            use = ("v_accvgpr_read_b32 v255, a%d" if kind == "a" else "v_mov_b32_e32 v255, v%d") % n
            moved = {k: v + (v > i) for k, v in labels.items()}
            assert touched_too_early(insts[:i + 1] + [(use, False)] + insts[i + 1:], moved) is not None, (name, insts[i][0])
