"""Waits of the kernels whose meetings leave a load under way, read from the built
library's machine code (CPU only).

The 256 x 256 tiles of the orthogonalised update ask for lines of later blocks with loads
that nobody reads, one a block, and a meeting waits for all loads but the last one
issued.  That one has to be such a load (or, between tiles, a store) whichever way the
meeting is reached, the first time too: were it one of the ring's, the meeting would let
its block be read before it has landed."""
import os
import re

import pytest

from tests.test_product_isa import predecessors
from tests.test_signal_waits_isa import LIB, OBJDUMP, library_code  # noqa: F401  (a fixture)

MEMORY = ("buffer_", "global_", "flat_", "scratch_")


def meetings(ins):
    """[(index, loads left under way)] of the waits right before a barrier."""
    out = []
    for i, (_, mn, ops, _) in enumerate(ins):
        left = re.search(r"vmcnt\((\d+)\)", ops)
        if mn == "s_waitcnt" and left and i + 1 < len(ins) and ins[i + 1][1] == "s_barrier":
            out.append((i, int(left.group(1))))
    return out


def youngest(pred, ins, i):
    """The memory instructions that may be the last one issued before ins[i]."""
    todo, seen, out = [i], set(), set()
    while todo:
        for j in pred[todo.pop()]:
            if j in seen:
                continue
            seen.add(j)
            if ins[j][1].startswith(MEMORY):
                out.add(j)
            else:
                todo.append(j)
    return out


def of_the_ring(mnemonic, operands):
    return mnemonic == "buffer_load_dwordx4" and " lds" in operands


def check(start, ins):
    """(meetings that leave one load, [(address, instruction)] of those that may leave one of the ring's)."""
    pred, n, bad = predecessors(start, ins), 0, []
    for i, left in meetings(ins):
        if left == 1:
            n += 1
            bad += [(hex(ins[j][0]), ins[j][1]) for j in youngest(pred, ins, i) if of_the_ring(ins[j][1], ins[j][2])]
    return n, bad


def test_the_check_sees_a_planted_race():
    ring, ahead = ("buffer_load_dwordx4", "v1, s[0:3], s4 offen lds", None), ("buffer_load_dword", "v1, s[0:3], s4 offen lds", None)
    meet, end = [("s_waitcnt", "vmcnt(1) lgkmcnt(0)", None), ("s_barrier", "", None)], ("s_endpgm", "", None)
    code = lambda *rows: [(4 * k, mn, ops, tgt) for k, (mn, ops, tgt) in enumerate(rows)]  # noqa: E731
    assert check(0, code(ring, ahead, *meet, end)) == (1, [])
    assert check(0, code(ahead, ring, *meet, end))[1] == [("0x4", "buffer_load_dwordx4")]
    # a loop that ends with the load ahead, entered without one
    loop = [*meet, ring, ahead, ("s_cbranch_scc1", "-5", 4), end]
    assert check(0, code(ring, *loop))[1] == [("0x0", "buffer_load_dwordx4")]
    loop[4] = ("s_cbranch_scc1", "-5", 8)
    assert check(0, code(ring, ahead, *loop)) == (1, [])


@pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not found")
def test_meetings_leave_only_loads_that_nobody_reads(library_code):  # noqa: F811
    kernels, problems = 0, []
    for name, start, ins in library_code:
        n, bad = check(start, ins)
        kernels += n > 0 and "orth_step_kernel" in name
        problems += [(name[-44:],) + b for b in bad]
    assert kernels == 4
    assert not problems, problems[:20]
