"""The choice of a kernel for the rows of pods_logp_chunk (csrc/row_plan.cuh), compiled for the host: every device, whole or a part of
one, gets a plan that it can run."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2504_13818_b200.csrc import build as cuda_build

ROW_EACH, ROWS_WARP, ROWS_PIPE = range(3)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    at = tmp_path_factory.mktemp("row_plan")
    (at / "plan.cpp").write_text("""#include "row_plan.cuh"
extern "C" void plan(int64_t T, int64_t nvec, int sms, int* out) {
    const pods_logp::RowPlan p = pods_logp::plan_rows(T, nvec, sms);
    out[0] = p.kernel; out[1] = p.batch; out[2] = p.warps; out[3] = p.cluster;
}
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.dirname(cuda_build.__file__), str(at / "plan.cpp"), "-o",
                    str(at / "plan.so")], check=True)
    lib = C.CDLL(str(at / "plan.so"))
    lib.plan.argtypes = [C.c_int64, C.c_int64, C.c_int, C.c_void_p]

    def ask(T, V, esize, sms=148):
        out = (C.c_int * 4)()
        lib.plan(T, V // (16 // esize), sms, out)
        return tuple(out)
    return ask


@pytest.mark.parametrize("sms", list(range(1, 33)) + [36, 70, 74, 132, 146, 148, 160])
def test_devices_and_parts_of_them(plan, sms):
    for T in (1, 5, 8 * sms, 8 * sms + 1, 3000, 1 << 24):
        for V in (1, 7, 1000, 8192, 8200, 32768, 40000, 151936, 524288):
            for esize in (2, 4):
                kernel, batch, warps, cluster = plan(T, V, esize, sms)
                if kernel == ROWS_PIPE:
                    assert cluster in (1, 2, 4, 8) and cluster <= sms and warps in (4, 16), (T, V, esize)
                    assert cluster < 4 or 16 + cluster <= sms
                elif kernel == ROWS_WARP:
                    assert 1 <= batch <= 8 and V * esize <= 1024 * 16 + 15
                else:
                    assert kernel == ROW_EACH and T <= 8 * sms and V * esize <= 4096 * 16 + 15


def test_the_sizes_tested_on_the_gpu_reach_every_kernel(plan):
    """On 148 SMs; a limit that moves has to take the sizes of these tests along."""
    from test_gpu_logp_many_rows import SHAPES
    seen = set()
    for name, dtype, T, V, _ in SHAPES:
        kernel, batch, warps, cluster = plan(T, V, 4 if dtype == "fp32" else 2)
        got = "rows" if kernel == ROWS_WARP else "pipe%d" % warps if kernel == ROWS_PIPE else "row"
        assert name == got + (" x%d" % cluster if cluster > 1 else ""), (T, V, dtype)
        seen.add((name, dtype) if kernel == ROWS_WARP else name)
        if kernel == ROWS_WARP:
            seen.add("batch of 1" if batch == 1 else "batch of 8" if batch == 8 else "batch between")
        elif T > 32 * 148 // cluster:
            seen.add("more rows than a look at the mask, " + ("one CTA" if cluster == 1 else "a cluster"))
    assert seen >= {("rows", "bf16"), ("rows", "fp16"), ("rows", "fp32"), "batch of 1", "batch of 8", "batch between", "pipe4", "pipe16", "pipe16 x2",
                    "pipe16 x4", "pipe16 x8", "more rows than a look at the mask, one CTA", "more rows than a look at the mask, a cluster"}
