"""The plans of the log-probabilities: what a workgroup keeps in LDS against what there is (no GPU)."""
import os
import re
import shutil
import subprocess

import pytest

from test_scratch_memory import LLVM

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2408_09992_amd", "csrc")

MAIN = r"""
#include <stdio.h>
#include "cross_entropy.hpp"
using namespace pqk::head;
using namespace pqk::head::subids;
int main() {                                         // every table that the call takes: entries of a query, queries at once, bytes of LDS
    for (int code_bytes = 1; code_bytes <= 2; ++code_bytes)
        for (int m = 1; m <= 128; ++m)
            for (int b = code_bytes == 1 ? 256 : 1; b <= (code_bytes == 1 ? 256 : 65536) && m * b <= 36864; b += m * b < 9000 ? 97 : 1)
                for (int B : {1, 2, 3}) {
                    Plan p;
                    if (check_shape(50000, B, m, b, code_bytes) || !plan_loss(p, 50000, B, m, b, code_bytes, kListedBytes)) continue;
                    const size_t need = (size_t)m * entries_of(b, code_bytes) * 4 * p.Q + (size_t)kWaves * p.Q * sizeof(float4) + p.Q * sizeof(int);
                    if (p.lds > kMaxLds || p.lds < need) printf("m %d b %d B %d: %zu bytes of LDS, %zu needed\n", m, b, B, p.lds, need);
                }
    puts("done");
}
"""


@pytest.mark.skipif(not shutil.which("hipcc"), reason="needs hipcc")
def test_tables_sums_and_counts_fit_lds(tmp_path):
    (tmp_path / "main.hip").write_text(MAIN)
    subprocess.run(["hipcc", "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(tmp_path / "main.hip"), "-c", "-o",
                    str(tmp_path / "main.o")], check=True, capture_output=True)
    (tmp_path / "error.cpp").write_text("#include <hip/hip_runtime_api.h>\nnamespace pqk { int record_hip_error(hipError_t) { return 0; } }\n")
    subprocess.run(["hipcc", "-O1", str(tmp_path / "main.o"), str(tmp_path / "error.cpp"), "-o", str(tmp_path / "main")], check=True, capture_output=True)
    out = subprocess.run([str(tmp_path / "main")], check=True, capture_output=True, text=True).stdout
    assert out == "done\n"


@pytest.mark.skipif(not os.path.exists(LLVM + "clang-offload-bundler"), reason="needs ROCm's LLVM tools")
def test_nothing_lies_in_lds_that_the_plan_does_not_count(pqlib_path, tmp_path):
    # (static LDS comes on top of what a launch asks for: 16 bytes of it beside a table that fills the rest made HIP refuse the launch)
    from paper_2408_09992_amd import build
    obj = os.path.join(build.OBJ, "log_probs.o")
    if not os.path.exists(obj):
        pytest.skip("the library was built elsewhere")
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.run([LLVM + "llvm-objcopy", "--dump-section", ".hip_fatbin=" + fat, obj, str(tmp_path / "rest.o")], check=True)
    subprocess.run([LLVM + "clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", "--input=" + fat, "--output=" + code], check=True)
    notes = subprocess.run([LLVM + "llvm-readelf", "--notes", code], check=True, capture_output=True, text=True).stdout
    found = {}
    for kernel in notes.split("- .agpr_count")[1:]:
        name = re.search(r"\.name: +(\S+)", kernel).group(1)
        if "log_probs_kernel" in name:
            found[name] = int(re.search(r"\.group_segment_fixed_size: +(\d+)", kernel).group(1))
    assert len(found) == 32 and not {k: v for k, v in found.items() if v}


def test_no_workspace_is_larger_than_its_lists(pqlib_path):
    # the lists' 2 GiB, or what 4096 items take (8192 where a list keeps more than 512); of positions whose items come in pieces 16 KB more, and 64 MiB of sums or a piece's
    import ctypes
    L = ctypes.CDLL(pqlib_path)
    sizes = []
    for name, rest in (("pq_log_probs", (8, 256)), ("pq_log_probs_u16", (8, 1000)), ("pq_default_log_probs", (64, 1)), ("pq_default_log_probs", (512, 0)), ("pq_default_log_probs", (512, 1))):
        f = getattr(L, name + "_workspace_bytes")
        f.argtypes, f.restype = [ctypes.c_longlong] + [ctypes.c_int] * 4, ctypes.c_size_t
        sizes.append((name, lambda N, B, K, f=f, rest=rest: f(N, B, *rest, K)))
    for N in (1, 1000, 4097, 12_000, 16_384, 16_385, 50_000, 300_000, 1_271_638, 28_457_277, 2 ** 30, 2 ** 31 - 1):
        for B in (1, 64, 65, 128, 129, 1024, 8192, 16_384, 30_000, 60_000, 65_535):
            for K in (1, 10, 100, 512):
                if K > N:
                    continue
                for name, size in sizes:
                    keep = K + 16 if "default" in name else K
                    lists = max(2 ** 31, 8 * B * (4096 if keep <= 512 else 8192))
                    assert 0 < size(N, B, K) <= lists + B * (16_384 + 64) + 2 ** 27, (name, N, B, K, size(N, B, K))
    for name, size in sizes:                                     # in one piece nothing is kept between pieces
        assert size(4000, 2000, 10) < 8 * 2000 * 4096 + 2 ** 23
