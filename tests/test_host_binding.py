"""The binding without a GPU: the extension's checks and calls, on a stand-in for libqmm and for the tensors.

The extension is compiled together with C functions of the library's names that record their call and, where told, wait; the
tensors are objects with the attributes that it reads."""
import importlib.machinery
import importlib.util
import os
import subprocess
import sys
import sysconfig
import threading
import time

import pytest
import torch

from paper_2607_00501_b200 import _build

STUB = r"""
#include <unistd.h>
#include "qmm.h"
int calls = 0, naps_us = 0;
static qmm_status called(void) { __atomic_add_fetch(&calls, 1, __ATOMIC_SEQ_CST); if (naps_us) usleep(naps_us); return QMM_OK; }
size_t qmm_mx_bytes(qmm_mx_format fmt, int64_t rows, int64_t K) { return (size_t)((rows + 127) / 128 * ((K + 255) / 256) * (16384 + 32768 / (int)fmt)); }
qmm_status qmm_mx_quantize(qmm_mx_format f, qmm_dtype d, const void* x, int64_t l, int64_t r, int64_t K, const float* t, void* p, void* s) { return called(); }
qmm_status qmm_mx_dequantize(qmm_mx_format f, const void* p, int64_t r, int64_t K, const float* t, qmm_dtype d, void* o, int64_t l, void* s) { return called(); }
qmm_status qmm_mx_linear(qmm_mx_format f, qmm_dtype d, const void* X, int64_t l, int64_t M, const void* w, int64_t N, int64_t K, const float* xs, const float* ws, void* Y,
                         int64_t ly, void* k, size_t kb, void* s) { return called(); }
qmm_status qmm_expert_sort(const int32_t* i, int32_t T, int32_t k, int32_t E, int32_t* o, int32_t* p, int32_t* f, int32_t* u, void* w, size_t b, void* s) { return called(); }
qmm_status qmm_expert_gather(qmm_dtype d, const void* x, int64_t l, int32_t T, int32_t k, int64_t H, const int32_t* o, const int32_t* p, const float* w, void* xs, int64_t lx,
                             void* s) { return called(); }
qmm_status qmm_expert_combine(qmm_dtype d, const void* y, int64_t l, int32_t T, int32_t k, int64_t H, const int32_t* p, const float* w, void* o, int64_t lo, void* s) { return called(); }
qmm_status qmm_expert_combine_grad(qmm_dtype d, const void* dy, int64_t l, const void* y, int64_t ly, int32_t T, int32_t k, int64_t H, const int32_t* o, const int32_t* p,
                                   const float* w, void* dys, int64_t ld, float* dw, void* s) { return called(); }
"""


class Tensor:
    """What the extension reads of a CUDA tensor."""

    def __init__(self, *shape, dtype=torch.float16, device=0):
        self.shape, self.dtype, self.is_cuda, self.device = tuple(shape), dtype, True, device

    def stride(self):
        return tuple(self.shape[1:]) + (1,)

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 4096

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device


@pytest.fixture(scope="module")
def ext(tmp_path_factory):
    """The extension over the stand-in; device 0 of two is current, streams are handle 0."""
    import ctypes
    at = tmp_path_factory.mktemp("binding")
    (at / "stub.c").write_text(STUB)
    so = str(at / ("_qmm_py" + sysconfig.get_config_var("EXT_SUFFIX")))
    root = os.path.dirname(_build.HERE)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-I", os.path.join(root, "include"), os.path.join(_build.CSRC, "qmm_py.c"),
                    str(at / "stub.c"), "-o", so], check=True)
    kept = {n: getattr(torch._C, n) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice", "_cuda_getDeviceCount")}
    torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice, torch._C._cuda_getDeviceCount = (lambda device: 0), (lambda: 0), (lambda: 2)
    try:
        loader = importlib.machinery.ExtensionFileLoader("_qmm_py", so)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_qmm_py", loader))
        loader.exec_module(module)
    finally:
        for n, f in kept.items():
            setattr(torch._C, n, f)
        sys.modules.pop("_qmm_py", None)
    lib = ctypes.CDLL(so)
    module_calls = lambda: ctypes.c_int.in_dll(lib, "calls").value                 # noqa: E731
    naps = ctypes.c_int.in_dll(lib, "naps_us")
    return module, module_calls, naps


def every_call(device=lambda i: 0):
    """(name, arguments) of a good call of every entry; device(i) places its i-th tensor.  The plan's arrays are addresses."""
    u8, f32, i32 = torch.uint8, torch.float32, torch.int32
    T, k, H = 4, 2, 64
    calls = [
        ("mx_quantize", [32, (5, 256), ((17408,), u8), None]),
        ("mx_quantize", [16, (5, 256), ((18432,), u8), ((1,), f32)]),
        ("mx_dequantize", [16, ((18432,), u8), (5, 256), ((1,), f32)]),
        ("mx_linear", [16, (5, 256), ((18432,), u8), 100, (5, 100), ((1,), f32), ((1,), f32), ((4096,), u8)]),
        ("expert_sort", [((T, k), i32), 8, 4096, 4096, 4096, 4096, 0, 0, 0]),
        ("expert_gather", [(T, H), T, k, 4096, 4096, 0, ((T, k), f32), (T * k, H)]),
        ("expert_combine", [(T * k, H), T, k, 4096, 0, ((T, k), f32), (T, H)]),
        ("expert_combine_grad", [(T, H), (T * k, H), T, k, 4096, 4096, 0, ((T, k), f32), (T * k, H), ((T, k), f32)]),
    ]
    out = []
    for name, args in calls:
        made, i = [], 0
        for a in args:
            if isinstance(a, tuple):
                shape, dtype = a if isinstance(a[0], tuple) else (a, torch.float16)
                made.append(Tensor(*shape, dtype=dtype, device=device(i)))
                i += 1
            else:
                made.append(a)
        out.append((name, made, i))
    return out


def test_good_calls_reach_the_library(ext):
    module, calls, _ = ext
    for name, args, _ in every_call():
        before = calls()
        assert getattr(module, name)(*args) == 0 and calls() == before + 1


def test_tensors_of_another_gpu_are_refused(ext):
    """A kernel runs on the current device: a tensor of another one, or tensors of two, never reach the library."""
    module, calls, _ = ext
    for n, (name, _, tensors) in enumerate(every_call()):
        for odd in [None, *range(tensors)]:
            args = every_call(lambda i: 1 if odd is None or i == odd else 0)[n][1]
            before = calls()
            with pytest.raises(AssertionError, match="device"):
                getattr(module, name)(*args)
            assert calls() == before


def test_wrappers_refuse_tensors_of_another_gpu(monkeypatch):
    """The same for the calls that go through ctypes (over a stand-in whose launches are only counted)."""
    from types import SimpleNamespace

    from paper_2607_00501_b200 import qmm
    _build.build()
    real, launched = qmm.lib(), []

    class Lib:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith(("_bytes", "_error")) else lambda *a: launched.append(name) or 0
    monkeypatch.setattr(qmm, "lib", Lib)
    monkeypatch.setattr(qmm, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(qmm, "_one_gpu", False)
    T, k, E, H = 4, 2, 8, 256
    u8, i32, f32 = torch.uint8, torch.int32, torch.float32
    unit, rows = qmm.mx_bytes(16, 1, 256), qmm.mx_experts_bytes(16, T, k, E, H)
    plan = SimpleNamespace(T=T, topk=k, E=E, ptrs=(4096,) * 4, buf=None)
    wrappers = [
        lambda t: qmm.mx_pack(16, t(5, 128, dtype=u8), t(5, 16, dtype=u8), H, out=t(unit, dtype=u8)),
        lambda t: qmm.mx_gemm(16, t(unit, dtype=u8), 5, t(unit, dtype=u8), 100, H, Y=t(5, 100), a_scale=t(1, dtype=f32), w_scale=t(1, dtype=f32), ws=t(1024, dtype=u8)),
        lambda t: qmm.mx_quantize_experts(16, t(T, H), t(T, k, dtype=i32), plan, out=t(rows, dtype=u8), tensor_scale=t(1, dtype=f32)),
        lambda t: qmm.mx_experts_gate_up(16, t(rows, dtype=u8), plan, t(E * unit, dtype=u8), t(E * unit, dtype=u8), 100, H, h=t(rows, dtype=u8), a_scale=t(1, dtype=f32),
                                         gate_scale=t(E, dtype=f32), up_scale=t(E, dtype=f32), h_scale=t(1, dtype=f32)),
        lambda t: qmm.mx_experts_gemm(16, t(rows, dtype=u8), plan, t(E * unit, dtype=u8), 100, H, Y=t(T * k, 100), a_scale=t(1, dtype=f32), w_scale=t(E, dtype=f32)),
        lambda t: qmm.mx_moe_run(qmm.mx_moe_args(16, t(T, H), t(T, k, dtype=i32), t(T, k, dtype=f32), t(E * unit, dtype=u8), t(E * unit, dtype=u8), t(2 * E * unit, dtype=u8), 100, E,
                                                 t(T, H), x_scale=t(1, dtype=f32), gate_scale=t(E, dtype=f32)), t(1 << 20, dtype=u8)),
    ]
    for call in wrappers:
        made = []
        call(lambda *shape, dtype=torch.float16: made.append(Tensor(*shape, dtype=dtype)) or made[-1])
        count = len(made)
        assert len(launched) == 1
        for odd in range(count):
            i = iter(range(count))
            with pytest.raises(AssertionError, match="device"):
                call(lambda *shape, dtype=torch.float16: Tensor(*shape, dtype=dtype, device=int(next(i) == odd)))
        assert len(launched) == 1
        launched.clear()


def test_arguments_of_a_layer_may_be_built_anywhere(monkeypatch):
    """mx_moe_args only wants its tensors together; the run is where the current device counts."""
    from paper_2607_00501_b200 import qmm
    _build.build()
    monkeypatch.setattr(qmm, "_one_gpu", False)
    now = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    u8, i32, f32 = torch.uint8, torch.int32, torch.float32
    t = lambda *shape, dtype=torch.float16: Tensor(*shape, dtype=dtype, device=1)  # noqa: E731
    w = t(8 * qmm.mx_bytes(32, 256, 256), dtype=u8)
    args = qmm.mx_moe_args(32, t(4, 256), t(4, 2, dtype=i32), t(4, 2, dtype=f32), w, w, w, 128, 8, t(4, 256))
    real, launched = qmm.lib(), []

    class Lib:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith(("_bytes", "_error")) else lambda *a: launched.append(name) or 0
    monkeypatch.setattr(qmm, "lib", Lib)
    monkeypatch.setattr(qmm, "_stream", lambda: 0)
    with pytest.raises(AssertionError, match="device"):
        qmm.mx_moe_run(args, t(1 << 20, dtype=u8))
    now[0] = 1
    qmm.mx_moe_run(args, t(1 << 20, dtype=u8))
    assert launched == ["qmm_mx_moe"]


def test_host_memory_is_refused_by_the_wrappers(monkeypatch):
    """Index arrays, workspaces and status words in host memory never reach a kernel (over the same stand-in)."""
    from types import SimpleNamespace

    from paper_2607_00501_b200 import qmm
    _build.build()
    real, launched = qmm.lib(), []

    class Lib:
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith(("_bytes", "_error")) else lambda *a: launched.append(name) or 0
    monkeypatch.setattr(qmm, "lib", Lib)
    monkeypatch.setattr(qmm, "_stream", lambda: 0)
    monkeypatch.setattr(qmm, "_one_gpu", True)
    T, k, E, H, u8, i32 = 4, 2, 8, 256, torch.uint8, torch.int32
    unit, rows = qmm.mx_bytes(32, 1, 256), qmm.mx_experts_bytes(32, T, k, E, H)
    plan = SimpleNamespace(T=T, topk=k, E=E, ptrs=(4096,) * 4, buf=None)
    w = Tensor(E * unit, dtype=u8)

    def host(t, contiguous=True):
        t.is_cuda, t.is_contiguous = not contiguous, lambda: contiguous
        return t
    calls = [lambda idx: qmm.mx_quantize_experts(32, Tensor(T, H), idx, plan, out=Tensor(rows, dtype=u8)),
             lambda ws: qmm.mx_gemm(32, Tensor(unit, dtype=u8), 5, Tensor(unit, dtype=u8), 100, H, Y=Tensor(5, 100), ws=ws),
             lambda ws: qmm.mx_moe_run(qmm.MxMoeArgs(), ws),
             lambda word: qmm.mx_experts_gate_up(32, Tensor(rows, dtype=u8), plan, w, w, 100, H, h=Tensor(rows, dtype=u8), status=word),
             lambda word: qmm.mx_experts_gemm(32, Tensor(rows, dtype=u8), plan, w, 100, H, Y=Tensor(T * k, 100), status=word)]
    good = [lambda: Tensor(T, k, dtype=i32), lambda: Tensor(4096, dtype=u8), lambda: Tensor(4096, dtype=u8), lambda: Tensor(1, dtype=i32), lambda: Tensor(1, dtype=i32)]
    for call, make in zip(calls, good):
        call(make())
        for bad in (host(make()), host(make(), contiguous=False)):
            with pytest.raises(AssertionError):
                call(bad)
        assert len(launched) == 1
        launched.clear()
    for call in calls[3:]:
        with pytest.raises(AssertionError):
            call(Tensor(2, dtype=u8))                                              # not a whole word


def test_plan_of_another_gpu_is_refused(ext, monkeypatch):
    """The plan's arrays go through the extension as addresses, with their device beside them."""
    from paper_2607_00501_b200 import qmm
    module, calls, _ = ext
    monkeypatch.setattr(qmm, "_ext", module)
    plan = qmm.ExpertPlan.__new__(qmm.ExpertPlan)
    plan.T, plan.topk, plan.E, plan.ptrs, plan.ws_ptr, plan.ws_bytes = 4, 2, 8, (4096,) * 4, 0, 0
    x, ys, w, idx = Tensor(4, 64), Tensor(8, 64), Tensor(4, 2, dtype=torch.float32), Tensor(4, 2, dtype=torch.int32)
    for call in (lambda: qmm.expert_sort(idx, 8, out=plan), lambda: qmm.expert_gather(x, plan, out=ys), lambda: qmm.expert_combine(ys, plan, out=x),
                 lambda: qmm.expert_gather_grad(ys, plan, out=x), lambda: qmm.expert_combine_grad(x, ys, plan, w, dys=ys, dw=w)):
        plan.device, before = 0, calls()
        call()
        assert calls() == before + 1
        plan.device = 1
        with pytest.raises(AssertionError, match="device"):
            call()
        assert calls() == before + 1


def test_cpu_tensors_are_refused(ext):
    module, calls, _ = ext
    before = calls()
    for n, (name, _, tensors) in enumerate(every_call()):
        for odd in range(tensors):
            with pytest.raises(AssertionError):
                getattr(module, name)(*every_call(lambda i: -1 if i == odd else 0)[n][1])
    assert calls() == before


def test_calls_let_other_threads_run(ext):
    """While a call waits in the library (a launch queue may be full), other Python threads go on."""
    module, _, naps = ext
    naps.value = 200000
    try:
        for name, args, _ in every_call():
            ticks, stop = [0], threading.Event()

            def tick():
                while not stop.is_set():
                    ticks[0] += 1
                    time.sleep(0.001)
            t = threading.Thread(target=tick)
            t.start()
            time.sleep(0.02)
            before = ticks[0]
            assert getattr(module, name)(*args) == 0
            during = ticks[0] - before
            stop.set()
            t.join()
            assert during >= 10, "%s: %d ticks in 200 ms" % (name, during)
    finally:
        naps.value = 0


def test_sizes_past_32_bits_are_refused(ext):
    """Token counts are 32-bit in the library: larger ones are refused, not cut."""
    module, calls, _ = ext
    before = calls()
    with pytest.raises(AssertionError):
        module.expert_sort(Tensor(2**32 + 4, 2, dtype=torch.int32), 8, 4096, 4096, 4096, 4096, 0, 0, 0)
    with pytest.raises(AssertionError):
        module.expert_sort(Tensor(4, 2, dtype=torch.int32), 2**32 + 8, 4096, 4096, 4096, 4096, 0, 0, 0)
    with pytest.raises(AssertionError):
        module.expert_gather(Tensor(2**32 + 4, 8), 2**32 + 4, 1, 4096, 4096, 0, None, Tensor(2**32 + 4, 8))
    with pytest.raises(AssertionError):
        module.mx_quantize(2**32 + 32, Tensor(5, 256), Tensor(17408, dtype=torch.uint8), None)
    assert calls() == before
    with pytest.raises(AssertionError):
        module.mx_quantize(10**30, Tensor(5, 256), Tensor(17408, dtype=torch.uint8), None)
    from paper_2607_00501_b200 import qmm
    _build.build()
    for T, k, E in ((2**32 + 4, 2, 8), (4, 2**32 + 2, 8), (4, 2, 2**32 + 8)):
        with pytest.raises(AssertionError):
            qmm.ExpertPlan(T, k, E, device="cpu")
        with pytest.raises(AssertionError):
            qmm.mx_experts_bytes(32, T, k, E, 256)
    with pytest.raises(AssertionError):
        qmm.mx_moe_args(32, Tensor(2**32 + 4, 256), Tensor(2**32 + 4, 2, dtype=torch.int32), Tensor(2**32 + 4, 2, dtype=torch.float32), None, None, None, 128, 8,
                        Tensor(2**32 + 4, 256))
    assert calls() == before


OLDER_CALLS = r"""
import os, sys
sys.path.insert(0, sys.argv[1])
from paper_2607_00501_b200 import _build, qmm
assert os.path.dirname(_build.HERE) == sys.argv[1]
def run(*a, **k):
    raise RuntimeError("no compiler on this machine")
_build.subprocess.run = run
assert qmm.version() > 0 and qmm.packed_bytes(qmm.Q4, 128, 256) > 0 and qmm.mx_bytes(32, 128, 256) > 0
try:
    qmm.mx_quantize(32, None, out=None if len(sys.argv) < 3 else sys.argv[2])
except RuntimeError as e:
    assert "no compiler" in str(e)
else:
    raise SystemExit("the extension came from nowhere")
"""


def shipped(tmp_path, foreign):
    """A copy of the package with its library and without the extension (foreign: with one of another interpreter)."""
    import shutil
    _build.build()
    to = tmp_path / os.path.basename(_build.HERE)
    to.mkdir()
    for f in os.listdir(_build.HERE):
        if f.endswith(".py") or f == "libqmm.so":
            shutil.copy(os.path.join(_build.HERE, f), to / f)
    if foreign:
        (to / "_qmm_py.cpython-38-x86_64-linux-gnu.so").write_bytes(b"built for another interpreter")
    return str(tmp_path)


@pytest.mark.parametrize("foreign", [False, True])
def test_calls_without_the_extension_need_no_compiler(tmp_path, foreign):
    """A machine with the built library alone serves every call that does not go through the extension."""
    at = shipped(tmp_path, foreign)
    r = subprocess.run([sys.executable, "-c", OLDER_CALLS, at, "x"], cwd=at, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_extension_is_named_for_its_interpreter(tmp_path):
    """An extension of one CPython is not loaded by another; the module's place and name are the import system's."""
    assert _build.EXT.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    _build.build()
    from paper_2607_00501_b200 import qmm
    assert os.path.samefile(qmm._native().__file__, _build.EXT)
