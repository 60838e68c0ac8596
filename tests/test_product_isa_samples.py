"""The wait-state checks of the 8-bit product's kernels on further planted hazards,
and which kernels they look at (CPU only)."""
import os
import re

import pytest

from tests.test_product_isa import _code, check
from tests.test_signal_waits_isa import LIB, OBJDUMP, library_code  # noqa: F401  (a fixture)

PRODUCT = ("v_mfma_f32_16x16x32_bf16", "a[0:3], v[4:7], v[8:11], a[0:3]", None)
OPERAND = ("v_mov_b32_e32", "v9, v0", None)
END = ("s_endpgm", "", None)


def loop(*between):
    """A product at address 0, what follows it, and a conditional branch back to it."""
    return _code(PRODUCT, *between, ("s_cbranch_scc1", "-3", 0), END)


def test_a_conditional_back_edge():
    """The branch is one wait state: an operand written right before it is one short."""
    bad = check(0, loop(OPERAND))
    assert len(bad) == 1 and bad[0] == (hex(0), "operand written by v_mov_b32_e32")
    assert check(0, loop(OPERAND, ("s_nop", "0", None))) == []
    # on the way out of the loop nothing multiplies any more
    assert check(0, _code(PRODUCT, ("s_cbranch_scc1", "-1", 0), OPERAND, END)) == []


def test_a_sum_around_a_back_edge():
    """A sum read at the head of a loop whose product is its last instruction."""
    head = ("v_accvgpr_read_b32", "v1, a2", None)
    bad = check(0, _code(head, ("s_nop", "15", None), PRODUCT, ("s_cbranch_scc1", "-4", 0), END))
    assert [b for b in bad if b[0] == hex(0)] == [(hex(0), "v_accvgpr_read_b32 touches a sum of v_mfma_f32_16x16x32_bf16")]
    assert check(0, _code(head, PRODUCT, ("s_nop", "15", None), ("s_nop", "1", None), ("s_cbranch_scc1", "-5", 0), END)) == []


_INSTANCE = re.compile(r"11tile_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELb([01])EE")


@pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not found")
def test_every_tile_kernel_is_looked_at(library_code):  # noqa: F811
    """Sizes of a wave's part, stages of the ring, and results in 32 bits or not, each for
    dense products, row groups and depth groups."""
    shapes = {(2, 2, 2, w) for w in (0, 1)} | {(2, 2, 4, w) for w in (0, 1)} | {(4, 4, 2, w) for w in (0, 1)}
    shapes |= {(4, 4, 4, 0), (8, 4, 2, 1), (8, 8, 2, 0)}
    want = {(a, b, s, mode, w) for a, b, s, w in shapes for mode in (0, 1, 2)}
    seen = []
    for name, start, ins in library_code:
        if "tile_kernel" in name and "quantize" not in name:
            a, b, s, mode, w = map(int, _INSTANCE.search(name).groups())
            seen.append((a, b, s, mode, w))
            # a block's products of a wave, each in four quarters with operands in bf16
            assert sum(mn.startswith("v_mfma") for _, mn, _, _ in ins) >= a * b * (4 if w else 1)
    assert sorted(seen) == sorted(want) and len(want) == 27
