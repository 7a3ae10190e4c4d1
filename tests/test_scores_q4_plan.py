"""How many workgroups of the four-bit scores a compute unit runs: what the launch counts on against what the compiler made (no GPU).

A workgroup is eight waves, two on each SIMD of 512 registers: two of them need kernels of 128 registers at most."""
import os
import re

import pytest

from test_scratch_memory import LLVM, compiled


@pytest.mark.skipif(not os.path.exists(LLVM + "clang-offload-bundler"), reason="needs ROCm's LLVM tools")
def test_registers_are_what_the_launch_counts_on(pqlib_path, tmp_path):
    from paper_2408_09992_amd import build
    obj = os.path.join(build.OBJ, "scores_q4.o")
    if not os.path.exists(obj):
        pytest.skip("the library was built elsewhere")
    with open(os.path.join(build.CSRC, "scores_q4.hip")) as f:
        one = set(re.findall(r"per_cu = SETS == (\d) \|\| fixed", f.read()))
    found = 0
    for kernel, (scratch, registers) in compiled(obj, tmp_path).items():
        k = re.search(r"24default_scores_q4_kernelILi(\d)ELi(\d)E", kernel)
        assert scratch == 0, kernel
        if k:
            found += 1
            assert (registers > 128) == (k[2] in one), (kernel, registers)
    assert found == 35
