"""Host-side checks of the microscaled and expert-sort entry points that need no GPU: size queries, refusals before
anything is launched, and the 64-bit reference against hand-made values."""
import ctypes

import numpy as np
import pytest

from paper_2607_00501_b200 import _build, qmm
from tests import mxref


@pytest.fixture(scope="module")
def L():
    _build.build()
    return qmm.lib()


@pytest.fixture(scope="module")
def a():
    buf = (ctypes.c_char * 4096)()
    a.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


def test_sizes(L):
    assert qmm.mx_bytes(32, 128, 256) == 16384 + 1024 and qmm.mx_bytes(16, 128, 256) == 16384 + 2048
    assert qmm.mx_bytes(32, 129, 257) == 4 * qmm.mx_bytes(32, 1, 1)
    assert qmm.mx_bytes(32, 0, 256) == 0 and qmm.mx_bytes(8, 128, 256) == 0 and qmm.mx_bytes(32, -1, 256) == 0 and qmm.mx_bytes(16, 1, 0) == 0
    assert qmm.mx_linear_workspace_bytes(32, 130, 64, 512) == 1024 + qmm.mx_bytes(32, 130, 512)
    assert qmm.mx_gemm_workspace_bytes(32, 1, 64, 512) == 1024 and qmm.mx_gemm_workspace_bytes(32, 1, 2048, 8192) > 1024       # partial sums
    # any routing fits: rows spread over the experts so that as many units as possible are begun
    for T, topk, E in ((1, 1, 1), (4, 8, 128), (100, 3, 2), (4096, 8, 128), (129, 1, 1)):
        P, u = T * topk, 17408
        most = max(sum(-(-c // 128) for c in counts) for counts in
                   ([1] * min(E, P) + [], [P - min(E, P) + 1] + [1] * (min(E, P) - 1), [129] * min(E, P // 129), [P]) if sum(counts) <= P)
        assert qmm.mx_experts_bytes(32, T, topk, E, 256) >= most * u
    assert L.qmm_expert_sort_workspace_bytes(16384, 8, 128) == 0 and L.qmm_expert_sort_workspace_bytes(16385, 8, 128) > 0
    assert L.qmm_expert_sort_workspace_bytes(1, 33, 128) == 0 and L.qmm_expert_sort_workspace_bytes(-1, 1, 1) == 0


def test_refusals_of_the_microscaled_calls(L, a):
    assert L.qmm_mx_quantize(4, 0, a, 256, 1, 256, None, a, None) == 1 and "format" in qmm.last_error()
    assert L.qmm_mx_quantize(32, 3, a, 256, 1, 256, None, a, None) == 1
    assert L.qmm_mx_quantize(32, 0, a, 255, 1, 256, None, a, None) == 2
    assert L.qmm_mx_quantize(32, 0, a + 1, 256, 1, 256, None, a, None) == 3
    assert L.qmm_mx_quantize(32, 2, a + 2, 256, 1, 256, None, a, None) == 3
    assert L.qmm_mx_quantize(32, 0, a, 256, 1, 256, None, a + 8, None) == 3
    assert L.qmm_mx_quantize(32, 0, a, 256, 1, 256, a, a, None) == 1 and "tensor scale" in qmm.last_error()
    assert L.qmm_mx_quantize(16, 0, a, 256, 1, 256, a + 2, a, None) == 3
    assert L.qmm_mx_quantize(32, 0, None, 256, 1, 256, None, a, None) == 1
    assert L.qmm_mx_quantize(32, 0, a, 256, -1, 256, None, a, None) == 1
    assert L.qmm_mx_quantize(32, 0, a, 256, 1, 0, None, a, None) == 1
    assert L.qmm_mx_quantize(32, 0, a, 1 << 21, 1, 1 << 21, None, a, None) == 5
    assert L.qmm_mx_quantize(32, 0, None, 0, 0, 256, None, None, None) == 0           # no rows: nothing is touched
    assert L.qmm_mx_dequantize(32, a, 1, 256, None, 0, a, 100, None) == 2
    assert L.qmm_mx_dequantize(32, a + 4, 1, 256, None, 0, a, 256, None) == 3
    assert L.qmm_mx_pack(32, None, a, 1, 256, a, None) == 1
    assert L.qmm_mx_pack(32, a, a, 1, 256, a + 8, None) == 3
    assert L.qmm_mx_gemm(32, a, 1, a, 0, 256, None, None, 0, a, 256, a, 4096, None) == 1
    assert L.qmm_mx_gemm(32, a, 1, a, 64, 256, None, None, 0, a, 63, a, 4096, None) == 2
    assert L.qmm_mx_gemm(32, a, 1, a, 64, 256, None, None, 0, a, 64, a, 1023, None) == 4
    assert L.qmm_mx_gemm(32, a, 1, a, 64, 256, None, None, 0, a, 64, a + 16, 8192, None) == 3
    assert L.qmm_mx_gemm(32, a, 1, a, 64, 256, None, None, 0, a, 64, None, 0, None) == 4
    assert L.qmm_mx_gemm(32, a, 1, a + 8, 64, 256, None, None, 0, a, 64, a, 4096, None) == 3
    assert L.qmm_mx_gemm(32, a, 1, a, 64, 256, a, None, 0, a, 64, a, 4096, None) == 1
    assert L.qmm_mx_gemm(32, None, 0, None, 64, 256, None, None, 0, None, 64, None, 0, None) == 0
    assert L.qmm_mx_linear(32, 0, a, 256, 1, a, 64, 256, None, None, a, 64, a, 256, None) == 4
    assert L.qmm_mx_linear(32, 0, a, 255, 1, a, 64, 256, None, None, a, 64, a, 1 << 20, None) == 2


def test_refusals_of_the_expert_calls(L, a):
    assert L.qmm_expert_sort(a, 4, 2, 0, a, a, a, a, None, 0, None) == 1
    assert L.qmm_expert_sort(a, 4, 33, 8, a, a, a, a, None, 0, None) == 5
    assert L.qmm_expert_sort(a, 4, 2, 1025, a, a, a, a, None, 0, None) == 5
    assert L.qmm_expert_sort(a, 1 << 22, 2, 8, a, a, a, a, None, 0, None) == 5
    assert L.qmm_expert_sort(None, 4, 2, 8, a, a, a, a, None, 0, None) == 1
    assert L.qmm_expert_sort(a, 4, 2, 8, a, a, None, a, None, 0, None) == 1
    assert L.qmm_expert_sort(a + 2, 4, 2, 8, a, a, a, a, None, 0, None) == 3
    assert L.qmm_expert_sort(a, 131073, 1, 8, a, a, a, a, None, 0, None) == 4
    assert L.qmm_expert_gather(0, a, 63, 4, 2, 64, a, a, None, a, 64, None) == 2
    assert L.qmm_expert_gather(0, a, 64, 4, 2, 0, a, a, None, a, 64, None) == 1
    assert L.qmm_expert_gather(9, a, 64, 4, 2, 64, a, a, None, a, 64, None) == 1
    assert L.qmm_expert_gather(0, a, 64, 4, 2, 64, None, a, None, a, 64, None) == 1
    assert L.qmm_expert_gather(0, None, 64, 0, 2, 64, None, None, None, None, 64, None) == 0
    assert L.qmm_expert_combine(0, a, 64, 4, 2, 64, None, None, a, 64, None) == 1
    assert L.qmm_expert_combine(2, a + 2, 64, 4, 2, 64, a, None, a, 64, None) == 3
    assert L.qmm_expert_combine_grad(0, a, 64, a, 64, 4, 2, 64, a, a, None, a, 64, a, None) == 1
    assert L.qmm_expert_combine_grad(0, a, 64, a, 64, 4, 2, 64, a, a, a, a, 60, a, None) == 2
    assert L.qmm_mx_quantize_experts(32, 0, a, 64, 4, 2, 8, 64, a, a, None, a, None, a, None) == 1
    assert L.qmm_mx_experts_gate_up(32, a, 4, 2, 8, a, a, a, None, 64, 64, None, None, None, None, a, None, None) == 1
    assert L.qmm_mx_experts_gemm(32, a, 4, 2, 8, a, a, a, 64, 64, None, None, 0, a, 60, None, None) == 2
    args = qmm.MxMoeArgs(4, 64, 64, 8, 2, 32, 0, a, 64, a, a, a, a, a, None, None, None, None, None, a, 64)
    need = L.qmm_mx_moe_workspace_bytes(ctypes.byref(args))
    assert need > 0
    assert L.qmm_mx_moe(ctypes.byref(args), a, need - 1, None) == 4
    args.ldo = 60
    assert L.qmm_mx_moe(ctypes.byref(args), a, need, None) == 2
    args.ldo, args.h_scale = 64, a
    assert L.qmm_mx_moe(ctypes.byref(args), a, need, None) == 1
    args.h_scale, args.topk = None, 40
    assert L.qmm_mx_moe_workspace_bytes(ctypes.byref(args)) == 0


def test_reference_on_hand_made_values():
    x = np.zeros((1, 32))
    x[0, :8] = [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25]
    codes, scale = mxref.quantize(x, 32)
    assert scale[0, 0] == 127 and list(codes[0, 0, :8]) == [7, 6, 6, 4, 4, 2, 2, 0]     # ties to the even code
    codes, scale = mxref.quantize(-x * 2.0**-5, 32)
    assert scale[0, 0] == 122 and list(codes[0, 0, :8]) == [15, 14, 14, 12, 12, 10, 10, 8]
    x[0, 0] = 7.9
    assert mxref.quantize(x, 32)[0][0, 0, 0] == 7                                          # saturates
    codes, scale = mxref.quantize(np.array([[3.0] * 16]), 16, 0.5)
    assert scale[0, 0] == 0x38 and (codes == 7).all()                                      # 3 / (6 * 0.5) = 1.0 = e4m3 0x38
    assert mxref.values(codes, scale, 16, 16, 0.5)[0, 0] == 3.0
    assert mxref.quantize(np.array([[np.inf] + [1.0] * 15]), 16)[1][0, 0] == 127
    rng = np.random.default_rng(0)
    c, s = rng.integers(0, 16, (130, 17, 16)), rng.integers(0, 127, (130, 17))
    got_c, got_s = mxref.unpack(mxref.pack(c, s, 16), 16, 130, 272)
    assert np.array_equal(got_c[:, :272], c.reshape(130, -1)) and np.array_equal(got_s[:, :17], s)
    order, place, offsets, units = mxref.sort(np.array([[2, 0], [-1, 2], [0, 5]]), 3)
    assert list(order) == [1, 4, 0, 3, -1, -1] and list(place) == [2, 0, -1, 3, 1, -1] and list(offsets) == [0, 2, 2, 4] and list(units) == [0, 1, 1, 2]
