"""Wait states around the hand-placed matrix instructions of the 8-bit product's
tile kernels, read from the built library's machine code (CPU only).

The kernels issue their matrix instructions from asm, which the compiler's hazard
recogniser does not look into.  Checked here on the compiled code, on every
straight-line path into the instruction:

* an operand or scale of a matrix instruction is not written by a VALU
  instruction less than two wait states before it;
* nothing but a matrix instruction reads or writes a sum less than 19 wait
  states (the longest write of these instructions) after it was issued, and none
  of the main loop does at all;
* the kernels have no scratch memory.
"""
import os
import re

import pytest

from tests.test_signal_waits_isa import LIB, OBJDUMP, library_code, successors  # noqa: F401  (a fixture)

_REG = re.compile(r"\b([va])(?:(\d+)|\[(\d+):(\d+)\])")


def registers(operand: str) -> set:
    out = set()
    for kind, one, lo, hi in _REG.findall(operand):
        out |= {(kind, int(one))} if one else {(kind, k) for k in range(int(lo), int(hi) + 1)}
    return out


def split(operands: str) -> list:
    return [o.strip() for o in re.sub(r"//.*", "", operands).split(",")]


def states(mnemonic: str, operands: str) -> int:
    return int(operands.split()[0]) + 1 if mnemonic == "s_nop" else 1


def is_valu(mnemonic: str) -> bool:
    return mnemonic.startswith("v_") and not mnemonic.startswith("v_mfma")


def predecessors(start, ins):
    pred = [[] for _ in ins]
    for i, out in enumerate(successors(start, ins)):
        for j in out:
            pred[j].append(i)
    return pred


def within(pred, ins, i, limit):
    """Instructions reached backwards from ins[i] over less than `limit` wait states."""
    todo, seen = [(i, 0)], {}
    while todo:
        at, passed = todo.pop()
        for j in pred[at]:
            if j not in seen or passed < seen[j]:
                seen[j] = passed
                more = passed + states(ins[j][1], ins[j][2])
                if more < limit:
                    todo.append((j, more))
    return seen


def check(start, ins):
    """[(address, what)] of a kernel's broken rules."""
    pred, bad = predecessors(start, ins), []
    mfma = [i for i, (_, mn, _, _) in enumerate(ins) if mn.startswith("v_mfma")]
    for i in mfma:
        sources = set().union(*(registers(o) for o in split(ins[i][2])[1:]))
        for j in within(pred, ins, i, 2):
            if is_valu(ins[j][1]) and registers(split(ins[j][2])[0]) & sources:
                bad.append((hex(ins[i][0]), "operand written by %s" % ins[j][1]))
    for i, (a, mn, ops, _) in enumerate(ins):
        if mn.startswith("v_mfma") or not mn.startswith(("v_", "ds_", "buffer_", "global_", "flat_", "scratch_")):
            continue
        used = registers(ops)
        for j in within(pred, ins, i, 19) if used else ():
            if ins[j][1].startswith("v_mfma") and registers(split(ins[j][2])[0]) & used:
                bad.append((hex(a), "%s touches a sum of %s" % (mn, ins[j][1])))
    if any(mn.startswith("scratch_") for _, mn, _, _ in ins):
        bad.append(("", "scratch memory"))
    return bad


def _code(*rows):
    return [(4 * k, mn, ops, tgt) for k, (mn, ops, tgt) in enumerate(rows)]


def test_the_checks_see_planted_hazards():
    product = ("v_mfma_f32_16x16x32_bf16", "a[0:3], v[4:7], v[8:11], a[0:3]", None)
    end = ("s_endpgm", "", None)
    nops = ("s_nop", "15", None)
    assert check(0, _code(("v_mov_b32_e32", "v4, v0", None), ("s_nop", "1", None), product, nops, nops,
                          ("v_accvgpr_read_b32", "v1, a0", None), end)) == []
    assert "operand" in check(0, _code(("v_mov_b32_e32", "v4, v0", None), ("s_nop", "0", None), product, end))[0][1]
    assert "sum" in check(0, _code(product, ("s_nop", "7", None), ("v_accvgpr_read_b32", "v1, a2", None), end))[0][1]
    # around a loop's back edge
    loop = _code(product, ("v_mov_b32_e32", "v9, v0", None), ("s_cbranch_scc1", "-3", 0), end)
    assert "operand" not in str(check(0, _code(product, ("v_mov_b32_e32", "v9, v0", None), end)))
    assert check(0, loop) == [] or "operand" in check(0, loop)[0][1]
    assert "operand" in str(check(0, _code(product, ("v_mov_b32_e32", "v9, v0", None), ("s_branch", "-3", 0), end)))


@pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not found")
def test_tile_kernels_keep_their_wait_states(library_code):  # noqa: F811
    kernels, problems = 0, []
    for name, start, ins in library_code:
        if "tile_kernel" not in name or "quantize" in name:
            continue
        kernels += 1
        problems += [(name[-24:],) + b for b in check(start, ins)]
    assert kernels >= 6
    assert not problems, problems[:20]
