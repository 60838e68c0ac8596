"""Wait states around the hand-placed matrix instructions of the orthogonalised update's
kernels for operands of two values, read from the built library's machine code (CPU only)."""
import os
import re

import pytest

from tests.test_product_isa import check
from tests.test_signal_waits_isa import LIB, OBJDUMP, library_code  # noqa: F401  (a fixture)


@pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not found")
def test_fine_kernels_keep_their_wait_states(library_code):  # noqa: F811
    kernels, problems = 0, []
    for name, start, ins in library_code:
        if "orth_fine_kernel" not in name:
            continue
        kernels += 1
        wm, wn = map(int, re.search(r"orth_fine_kernelILi(\d+)ELi(\d+)E", name).groups())
        assert sum(mn == "v_mfma_f32_16x16x32_f16" for _, mn, _, _ in ins) >= 2 * wm * wn  # a block's
        problems += [(name[-40:],) + b for b in check(start, ins)]
    assert kernels == 12
    assert not problems, problems[:20]
