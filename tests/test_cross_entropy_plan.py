"""How many workgroups of the loss by sub-ids a compute unit runs: what the plan counts on against what the compiler made (no GPU).

A workgroup is 16 waves, four on each SIMD of 512 registers: two of them need kernels of 64 registers at most."""
import ctypes
import os
import re

import pytest

from test_scratch_memory import LLVM, compiled

CUS = 256


@pytest.fixture(scope="module")
def shares(pqlib_path):
    L = ctypes.CDLL(pqlib_path)

    def of(N, B, m, b, u16=False):
        f = getattr(L, "pq_cross_entropy_u16_workspace_bytes" if u16 else "pq_cross_entropy_workspace_bytes")
        f.argtypes, f.restype = [ctypes.c_longlong] + [ctypes.c_int] * 3, ctypes.c_size_t
        return max(1, (f(N, B, m, b) - 16) // (8 * B))
    return of


@pytest.mark.parametrize("N,B,m,b,u16", [(1_280_000, 1, 16, 256, False), (1_280_000, 2, 16, 256, False), (1_280_000, 1, 32, 256, False), (1_280_000, 2, 32, 256, False),
                                         (1_280_000, 2, 8, 1024, True), (1_280_000, 1, 16, 512, True), (300_000, 64, 16, 256, False)])
def test_long_rows_are_one_round_of_workgroups(shares, N, B, m, b, u16):
    groups = (B + 3) // 4 if B >= 3 else 1
    assert CUS / 2 < groups * shares(N, B, m, b, u16) <= CUS


@pytest.mark.skipif(not os.path.exists(LLVM + "clang-offload-bundler"), reason="needs ROCm's LLVM tools")
def test_registers_are_what_the_plan_counts_on(pqlib_path, tmp_path):
    from paper_2408_09992_amd import build
    obj = os.path.join(build.OBJ, "cross_entropy.o")
    if not os.path.exists(obj):
        pytest.skip("the library was built elsewhere")
    found = {}
    for kernel, (scratch, registers) in compiled(obj, tmp_path).items():
        k = re.search(r"20cross_entropy_kernelILi(\d+)E([ht])Li(\d+)E", kernel)
        assert scratch == 0, kernel
        if k:
            found[int(k[1]), 1 if k[2] == "h" else 2, int(k[3])] = registers
    assert len(found) == 32
    for (m, code_bytes, Q), registers in found.items():
        if (m, code_bytes) not in ((16, 1), (16, 2), (8, 2), (32, 1)):
            assert registers <= 64, (m, code_bytes, Q, registers)
