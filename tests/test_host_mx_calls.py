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
