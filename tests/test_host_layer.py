"""Host-side checks of the router, the norm with 8-bit rows and the adapters that need no GPU: sizes and refusals, of the C entries and of the binding."""
import ctypes
import importlib.machinery
import importlib.util
import os
import subprocess
import sysconfig

import pytest
import torch

from paper_2607_00501_b200 import _build, qmm
from tests.test_host_binding import Tensor


@pytest.fixture(scope="module")
def L():
    _build.build()
    return qmm.lib()


@pytest.fixture(scope="module")
def a():
    buf = (ctypes.c_char * 4096)()
    a.keep = buf
    return (ctypes.addressof(buf) + 255) & ~255


def test_refusals_of_the_router(L, a):
    def route(dtype=0, logits=a, ld=64, T=4, E=64, topk=8, scores=0, bias=None, groups=1, top=1, group_top=1, renorm=1, scale=1.0, idx=a, w=a):
        return L.qmm_expert_route(dtype, logits, ld, T, E, topk, scores, bias, groups, top, group_top, renorm, scale, idx, w, None)
    assert route(dtype=3) == 1 and route(logits=None) == 1 and route(idx=None) == 1 and route(w=None) == 1
    assert route(ld=63) == 2 and route(logits=a + 1) == 3 and route(dtype=2, logits=a + 2) == 3
    assert route(idx=a + 2) == 3 and route(w=a + 1) == 3 and route(bias=a + 2) == 3
    assert route(T=-1) == 1 and route(E=0) == 1 and route(topk=0) == 1 and route(topk=65) == 5 and route(E=4, topk=8) == 1 and "topk" in qmm.last_error()
    assert route(E=1025, ld=1025) == 5 and route(topk=33) == 5
    assert route(scores=2) == 1 and route(scale=float("nan")) == 1 and route(scale=float("inf")) == 1
    assert route(groups=0) == 1 and route(groups=3) == 1 and route(groups=64) == 1 and route(groups=8, top=9) == 1 and route(top=0) == 1 and route(group_top=3) == 1
    assert route(T=0, logits=None, idx=None, w=None) == 0

    def grad(dtype=0, dw=a, logits=a, ld=64, idx=a, T=4, E=64, topk=8, scores=0, renorm=1, scale=1.0, out=a, ldo=64):
        return L.qmm_expert_route_grad(dtype, dw, logits, ld, idx, T, E, topk, scores, renorm, scale, out, ldo, None)
    assert grad(dw=None) == 1 and grad(idx=None) == 1 and grad(out=None) == 1 and grad(dtype=7) == 1 and grad(scores=-1) == 1
    assert grad(ldo=60) == 2 and grad(out=a + 1) == 3 and grad(dw=a + 2) == 3 and grad(topk=65) == 5
    assert grad(T=0, dw=None, logits=None, idx=None, out=None) == 0


def test_refusals_of_the_norm(L, a):
    def norm(dtype=0, x=a, ldx=64, r=None, ldr=64, w=a, eps=1e-6, rows=2, K=64, h=None, ldh=64, y=a, ldy=64, fmt=0, codes=None, ldc=64, scales=None):
        return L.qmm_rms_norm(dtype, x, ldx, r, ldr, w, eps, rows, K, h, ldh, y, ldy, fmt, codes, ldc, scales, None)
    assert norm(dtype=4) == 1 and norm(x=None) == 1 and norm(y=None) == 1 and "codes" in qmm.last_error()
    assert norm(eps=0.0) == 1 and norm(eps=-1.0) == 1 and norm(eps=float("inf")) == 1 and norm(rows=-1) == 1 and norm(K=0) == 1 and norm(K=32769, ldx=32769, ldy=32769) == 5
    assert norm(ldx=63) == 2 and norm(r=a, ldr=10) == 2 and norm(h=a, ldh=1) == 2 and norm(ldy=0) == 2 and norm(y=None, codes=a, ldc=63, scales=a) == 2
    assert norm(x=a + 1) == 3 and norm(w=a + 1) == 3 and norm(dtype=2, w=a + 2) == 3 and norm(y=None, codes=a, scales=a + 2) == 3
    assert norm(y=None, codes=a, scales=None) == 1 and norm(codes=a, scales=a, fmt=2) == 1
    assert norm(rows=0, x=None, y=None) == 0

    def grad(dtype=0, dy=a, h=a, ldh=64, w=a, eps=1e-6, rows=2, K=64, dh=None, dx=a, lddx=64, dw=a, ws=a, nb=1 << 20):
        return L.qmm_rms_norm_grad(dtype, dy, 64, h, ldh, w, eps, rows, K, dh, 64, dx, lddx, dw, ws, nb, None)
    assert grad(dx=None, dw=None) == 1 and grad(dy=None) == 1 and grad(h=None) == 1 and grad(eps=0.0) == 1
    assert grad(lddx=1) == 2 and grad(dw=a + 2) == 3 and grad(ws=None) == 4 and grad(nb=511) == 4 and grad(ws=a + 8) == 3
    assert grad(rows=0, dy=None, h=None, dx=a, dw=None) == 0
    assert qmm.rms_norm_grad_workspace_bytes(2, 64) == 512 and qmm.rms_norm_grad_workspace_bytes(-1, 64) == 0 and qmm.rms_norm_grad_workspace_bytes(1, 0) == 0
    sizes = [qmm.rms_norm_grad_workspace_bytes(r, 1000) for r in (*range(0, 700), 5000, 100000)]
    assert all(x <= y for x, y in zip(sizes, sizes[1:]))

    assert L.qmm_rows_quantize(0, a, 64, 2, 64, 5, a, 64, a, None) == 1 and L.qmm_rows_quantize(0, a, 64, 2, 64, 0, None, 64, a, None) == 1
    assert L.qmm_rows_quantize(0, a, 64, 2, 64, 0, a, 10, a, None) == 2 and L.qmm_rows_quantize(2, a + 2, 64, 2, 64, 0, a, 64, a, None) == 3
    assert L.qmm_rows_quantize(0, None, 64, 0, 64, 0, None, 64, None, None) == 0
    assert L.qmm_rows_dequantize(1, a, 64, a, 2, 64, 9, a, 64, None) == 1 and L.qmm_rows_dequantize(1, a, 64, a, 2, 64, 0, a, 63, None) == 2
    assert L.qmm_rows_dequantize(1, a, 64, None, 2, 64, 0, a, 64, None) == 1 and L.qmm_rows_dequantize(3, a, 64, a, 2, 64, 0, a, 64, None) == 1


def test_rows_without_a_workspace(L, a):
    """The wrapper's bound is the library's: beyond it the workspace holds the blocks' parts, and a forward pass without one is refused."""
    most = qmm.LORA_ROWS_WITHOUT_WORKSPACE
    sizes = [qmm.lora_workspace_bytes(T, 1, 128) for T in range(2 * most)]
    jumps = [T for T in range(2 * most - 1) if sizes[T + 1] - sizes[T] > 1 << 20]
    assert jumps == [most]
    q = qmm.LoraArgs(T=most + 1, n=1, r=128, K=64, N=32, X=a, ldx=64, idx=a, A=a, B=a, Y=a, ldy=32)
    assert L.qmm_lora(ctypes.byref(q), None, 0, None) == 4


def test_refusals_of_the_adapters(L, a):
    base = dict(T=600, n=4, r=16, dtype=0, K=64, N=32, X=a, ldx=64, idx=a, A=a, B=a, S=a, Y0=a, ldy0=32, Y=a, ldy=32, dY=a, lddy=32, dX0=a, lddx0=64, dX=a, lddx=64, dA=a, dB=a)
    need = qmm.lora_workspace_bytes(600, 4, 16)

    def call(which, ws=a, nb=need, **kw):
        return getattr(L, which)(ctypes.byref(qmm.LoraArgs(**{**base, **kw})), ws, nb, None)
    for which in ("qmm_lora", "qmm_lora_grad"):
        assert L.qmm_lora(None, a, need, None) == 1
        for kw, status in ((dict(T=-1), 1), (dict(n=0), 1), (dict(n=1025), 5), (dict(r=12), 5), (dict(r=256), 5), (dict(r=0), 5), (dict(dtype=2), 1), (dict(K=0), 1), (dict(N=-3), 1),
                           (dict(K=1 << 21, ldx=1 << 21, lddx=1 << 21, lddx0=1 << 21), 5), (dict(idx=None), 1), (dict(A=None), 1), (dict(B=None), 1), (dict(idx=a + 2), 3),
                           (dict(scale=a + 1), 3), (dict(A=a + 1), 3), (dict(order=a), 1), (dict(order=a, offsets=a), 1), (dict(order=a, offsets=a + 1, units=a), 3), (dict(S=a + 4), 3),
                           (dict(ldx=63), 2), (dict(X=None), 1), (dict(x_scale=a, x_format=7), 1), (dict(x_scale=a + 2), 3), (dict(ws=None), 4), (dict(nb=need - 1), 4), (dict(ws=a + 16), 3)):
            assert call(which, **kw) == status, (which, kw, qmm.last_error())
    assert call("qmm_lora", Y=None) == 1 and call("qmm_lora", ldy=31) == 2 and call("qmm_lora", Y0=a + 1) == 3
    assert call("qmm_lora", T=0, X=None, idx=None, A=None, B=None, Y=None) == 0
    assert call("qmm_lora_grad", dX=None, dA=None, dB=None) == 1 and call("qmm_lora_grad", dA=a + 4) == 3 and call("qmm_lora_grad", dB=a + 8) == 3
    assert call("qmm_lora_grad", dY=None) == 1 and call("qmm_lora_grad", S=None) == 1 and "forward" in qmm.last_error() and call("qmm_lora_grad", lddx=60) == 2
    assert L.qmm_lora_workspace_bytes(4, 4, 12) == 0 and L.qmm_lora_workspace_bytes(-4, 4, 16) == 0
    sizes = [qmm.lora_workspace_bytes(T, 64, 32) for T in (*range(0, 600), 5000, 200000)]
    assert all(x <= y for x, y in zip(sizes, sizes[1:]))
    with pytest.raises(qmm.QmmError):
        qmm.lora_workspace_bytes(4, 4, 12)


# ---------------------------------------------------- the extension, over a stand-in for the library

STUB = r"""
#include "qmm.h"
int calls = 0;
qmm_lora_args last;
static qmm_status called(void) { ++calls; return QMM_OK; }
qmm_status qmm_expert_route(qmm_dtype d, const void* l, int64_t ld, int32_t T, int32_t E, int32_t k, qmm_scores s, const float* b, int32_t g, int32_t t, int32_t gt, int32_t r, float c,
                            int32_t* i, float* w, void* st) { return called(); }
qmm_status qmm_expert_route_grad(qmm_dtype d, const float* w, const void* l, int64_t ld, const int32_t* i, int32_t T, int32_t E, int32_t k, qmm_scores s, int32_t r, float c, void* o,
                                 int64_t lo, void* st) { return called(); }
qmm_status qmm_rms_norm(qmm_dtype d, const void* x, int64_t lx, const void* r, int64_t lr, const void* w, float e, int64_t rows, int64_t K, void* h, int64_t lh, void* y, int64_t ly,
                        qmm_row_format f, void* c, int64_t lc, float* s, void* st) { return called(); }
qmm_status qmm_rms_norm_grad(qmm_dtype d, const void* dy, int64_t l, const void* h, int64_t lh, const void* w, float e, int64_t rows, int64_t K, const void* dh, int64_t ldh, void* dx,
                             int64_t ldx, float* dw, void* ws, size_t nb, void* st) { return called(); }
qmm_status qmm_rows_quantize(qmm_dtype d, const void* x, int64_t l, int64_t r, int64_t K, qmm_row_format f, void* c, int64_t lc, float* s, void* st) { return called(); }
qmm_status qmm_rows_dequantize(qmm_row_format f, const void* c, int64_t lc, const float* s, int64_t r, int64_t K, qmm_dtype d, void* o, int64_t lo, void* st) { return called(); }
qmm_status qmm_lora(const qmm_lora_args* q, void* ws, size_t nb, void* st) { last = *q; return called(); }
qmm_status qmm_lora_grad(const qmm_lora_args* q, void* ws, size_t nb, void* st) { last = *q; return called(); }
"""


@pytest.fixture(scope="module")
def ext(tmp_path_factory):
    at = tmp_path_factory.mktemp("layer_ext")
    (at / "stub.c").write_text(STUB)
    so = str(at / ("_qmm_layer_py" + sysconfig.get_config_var("EXT_SUFFIX")))
    include = os.path.join(os.path.dirname(_build.HERE), "include")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-I", include, os.path.join(_build.CSRC, "qmm_layer_py.c"), str(at / "stub.c"), "-o", so],
                   check=True)
    saved = torch._C._cuda_getDeviceCount, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    torch._C._cuda_getDeviceCount, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream = lambda: 2, lambda: 0, lambda d: 0
    try:
        loader = importlib.machinery.ExtensionFileLoader("_qmm_layer_py", so)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_qmm_layer_py", loader))
        loader.exec_module(module)
    finally:
        torch._C._cuda_getDeviceCount, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream = saved
    module.counter = ctypes.c_int.in_dll(ctypes.CDLL(so), "calls")
    module.last = qmm.LoraArgs.in_dll(ctypes.CDLL(so), "last")
    return module


F16, F32, I32, U8, E4 = torch.float16, torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn


def good(other=0):
    """Arguments of each call that pass."""
    t = lambda *s, dtype=F16: Tensor(*s, dtype=dtype, device=other)  # noqa: E731
    plan = (4096, 8192, 12288, other)
    return {
        "expert_route": [t(6, 16), 4, 1, t(16, dtype=F32), 2, 1, 1, 1, 1.0, t(6, 4, dtype=I32), t(6, 4, dtype=F32)],
        "expert_route_grad": [t(6, 4, dtype=F32), t(6, 16), t(6, 4, dtype=I32), 4, 0, 1, 1.0, t(6, 16)],
        "rms_norm": [t(6, 32), t(32), 1e-6, t(6, 32), t(6, 32), t(6, 32), t(6, 32, dtype=E4), t(6, dtype=F32)],
        "rms_norm_grad": [t(6, 32), t(6, 32), t(32), 1e-6, t(6, 32), t(6, 32), t(32, dtype=F32), t(9999, dtype=U8)],
        "rows_quantize": [t(6, 32), t(6, 32, dtype=torch.int8), t(6, dtype=F32)],
        "rows_dequantize": [t(6, 32, dtype=E4), t(6, dtype=F32), t(6, 32, dtype=F32)],
        "lora": [t(6, 32), None, t(6, dtype=I32), t(3, 8, 32), t(3, 24, 8), t(3, dtype=F32), *plan, t(6, 8, dtype=F32), t(6, 24), t(6, 24), t(9999, dtype=U8)],
        "lora_grad": [t(6, 32, dtype=E4), t(6, dtype=F32), t(6, dtype=I32), t(3, 8, 32), t(3, 24, 8), t(3, dtype=F32), *plan, t(6, 8, dtype=F32), t(6, 24), t(6, 32), t(6, 32),
                      t(3, 8, 32, dtype=F32), t(3, 24, 8, dtype=F32), t(9999, dtype=U8)],
    }


@pytest.mark.parametrize("name", list(good()))
def test_the_extension_passes_good_calls_and_refuses_others(ext, name):
    before = ext.counter.value
    args = good()[name]
    assert getattr(ext, name)(*args) == 0 and ext.counter.value == before + 1
    with pytest.raises(TypeError):
        getattr(ext, name)(*args[:-1])
    for i, v in enumerate(args):
        if not isinstance(v, Tensor):
            continue
        odd = [Tensor(*v.shape, dtype=torch.float64, device=0), Tensor(*v.shape, dtype=v.dtype, device=1), Tensor(*v.shape, dtype=v.dtype, device=-1)]
        if v.dtype != U8:                                   # (a workspace may be any size here: the library looks)
            odd.append(Tensor(*v.shape[:-1], v.shape[-1] + 1, dtype=v.dtype, device=0))
        for w in odd:
            if name == "rows_quantize" and i == 0 and w.dtype == v.dtype and w.device == 0 and w.shape == v.shape:
                continue
            with pytest.raises(AssertionError):
                getattr(ext, name)(*[w if k == i else u for k, u in enumerate(args)])
    with pytest.raises(AssertionError):                     # everything on a GPU that is not the current one
        getattr(ext, name)(*good(1)[name])
    assert ext.counter.value == before + 1


def test_the_extension_fills_the_adapters_arguments(ext):
    ext.lora(*good()["lora"])
    q = ext.last
    assert (q.T, q.n, q.r, q.dtype, q.K, q.N, q.ldx, q.ldy0, q.ldy) == (6, 3, 8, 0, 32, 24, 32, 24, 24) and (q.order, q.offsets, q.units) == (4096, 8192, 12288) and not q.x_scale
    args = good()["lora"]
    args[0], args[1] = Tensor(6, 32, dtype=torch.int8), Tensor(6, dtype=F32)
    args[6:9] = [0, 0, 0]
    args[10] = args[11] = None
    ext.lora(*args)
    q = ext.last
    assert q.x_scale and q.x_format == 1 and not q.order and not q.S and not q.Y0
    args[1] = None                                          # codes without their scales
    with pytest.raises(AssertionError):
        ext.lora(*args)
    args = good()["lora"]
    args[0] = None
    with pytest.raises(AssertionError):
        ext.lora(*args)
