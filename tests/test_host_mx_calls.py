"""Host-side checks of the microscaled and expert calls that need no GPU: sizes and refusals."""
import ctypes

import pytest

from paper_2607_00501_b200 import _build, qmm


@pytest.fixture(scope="module")
def L():
    _build.build()
    return qmm.lib()


@pytest.fixture(scope="module")
def a():
    buf = (ctypes.c_char * 4096)()
    a.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


def test_type_of_the_experts_rows(L, a):
    args = qmm.MxMoeArgs(4, 64, 64, 8, 2, 32, 0, a, 64, a, a, a, a, a, None, None, None, None, None, a, 64)
    need = L.qmm_mx_moe_workspace_bytes(ctypes.byref(args))
    args.rows_f32 = 1
    wide = L.qmm_mx_moe_workspace_bytes(ctypes.byref(args))
    assert wide == need + 4 * 2 * 64 * 2                                           # T * topk rows of H, two bytes more each
    assert L.qmm_mx_moe(ctypes.byref(args), a, need, None) == 4
    args.rows_f32 = 2
    assert L.qmm_mx_moe_workspace_bytes(ctypes.byref(args)) == 0 and "rows_f32" in qmm.last_error()


@pytest.mark.parametrize("query", ["qmm_mx_linear_workspace_bytes", "qmm_mx_gemm_workspace_bytes"])
def test_workspace_sizes_do_not_fall_with_the_batch(L, query):
    """A workspace sized for the largest batch serves every smaller one."""
    for fmt in (32, 16):
        for N, K in ((2048, 8192), (512, 16384), (8192, 8192), (130, 5000), (128256, 2048), (2048, 2048)):
            sizes = [getattr(L, query)(fmt, M, N, K) for M in [*range(0, 300), 512, 1000, 4096]]
            assert all(a <= b for a, b in zip(sizes, sizes[1:])), (fmt, N, K)


def test_a_call_asks_for_no_more_workspace_than_it_uses(L, a):
    """64 rows of 2048 x 8192 share nothing, one row does: the header is enough for the first.  (Without a GPU the call goes on to the device check.)"""
    assert L.qmm_mx_gemm(32, a, 1, a, 2048, 8192, None, None, 0, a, 2048, a, 1024, None) == 4
    assert L.qmm_mx_gemm(32, a, 128, a, 2048, 8192, None, None, 0, a, 2048, a, 1023, None) == 4


def test_workspace_sizes_without_weight_rows(L):
    """N = 0 is refused like any other argument out of range (in a process of its own: it once ended in a division by zero)."""
    import subprocess
    import sys
    code = ("from paper_2607_00501_b200 import qmm\n"
            "for q in (qmm.mx_gemm_workspace_bytes, qmm.mx_linear_workspace_bytes):\n"
            "    for M in (0, 1, 200):\n"
            "        assert q(32, M, 0, 8192) == 0 and 'N must be positive' in qmm.last_error()\n")
    assert subprocess.run([sys.executable, "-c", code]).returncode == 0


def test_index_arrays_of_the_experts_calls_are_aligned(L, a):
    """Misaligned index arrays and status words are refused on the host (a kernel would fault on them)."""
    good = [a, a, a, a]
    for i in range(4):
        bad = [p + 2 * (i == j) for j, p in enumerate(good)]
        assert L.qmm_mx_quantize_experts(32, 0, a, 64, 4, 2, 8, 64, *bad, None, a, None) == 3, i
    for off, units, status in ((a + 2, a, None), (a, a + 1, None), (a, a, a + 2)):
        assert L.qmm_mx_experts_gate_up(32, a, 4, 2, 8, off, units, a, a, 64, 64, None, None, None, None, a, status, None) == 3
        assert L.qmm_mx_experts_gemm(32, a, 4, 2, 8, off, units, a, 64, 64, None, None, 0, a, 64, status, None) == 3
