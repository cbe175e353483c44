"""The products leave the calling thread's CUDA context as it is, also where that is not the one that the runtime makes by itself."""
import os
import re
import subprocess
import sys

import pytest

from tests.test_operator_sources import body, code

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import ctypes as C
import numpy as np
from paper_2508_05700_b200 import mfet as m

cu = C.CDLL("libcuda.so.1")
def ok(rc):
    assert rc == 0, rc
ok(cu.cuInit(0))
dev, ctx = C.c_int(), C.c_void_p()
ok(cu.cuDeviceGet(C.byref(dev), 0))
ok(cu.cuCtxCreate_v2(C.byref(ctx), 0, dev))

def check():
    now = C.c_void_p()
    ok(cu.cuCtxGetCurrent(C.byref(now)))
    assert now.value == ctx.value, "another context is current"

def memory(values):
    p = C.c_uint64()
    ok(cu.cuMemAlloc_v2(C.byref(p), C.c_size_t(values.nbytes)))
    ok(cu.cuMemcpyHtoD_v2(p, values.ctypes.data_as(C.c_void_p), C.c_size_t(values.nbytes)))
    return p.value

def values(p, shape):
    out = np.empty(shape, np.float16)
    ok(cu.cuMemcpyDtoH_v2(out.ctypes.data_as(C.c_void_p), C.c_uint64(p), C.c_size_t(out.nbytes)))
    return out.astype(np.float64)

def some(rows, cols, value):
    return memory(np.full((rows, cols), value, np.float16))

rows, n, k = 300, 128, 256
x, wg, wu, h, status = some(rows, k, 1.0), some(n, k, 1 / 64), some(n, k, 1 / 128), some(rows, n, 7.0), memory(np.zeros(1, np.uint32))
m.mfet_gated_linear(x, m.F16, k, rows, wg, k, wu, k, n, k, m.ACT_NONE, h, n, None, 0, status)
check()
assert (values(h, (rows, n)) == 8.0).all()
g = some(rows, k, 1.0)
out, ws = some(rows, k, 7.0), some(1, m.mfet_orthogonalize_bytes(rows, k) // 2 + 1, 0.0)
m.mfet_orthogonalize(g, m.F16, k, rows, k, [1.0, 0.0, 0.0], 1, 277.1281292110204, out, m.F16, k, ws, m.mfet_orthogonalize_bytes(rows, k), status)
check()
assert (values(out, (rows, k)) == 1.0).all()  # 1 / sqrt(300 * 256), scaled back, rounded to fp16
codes, scales = some(1, m.mfet_mx4_code_bytes(n, k), 0.0), some(1, m.mfet_mx4_scale_bytes(n, k), 0.0)
m.mfet_mx4_quantize(x, m.F16, k, n, k, codes, scales)
y, s2 = some(rows, n, 7.0), some(1, m.mfet_mx4_linear_bytes(rows, k), 0.0)
m.mfet_mx4_linear(x, m.F16, k, rows, codes, scales, n, k, None, m.ACT_NONE, y, m.F16, n, s2, m.mfet_mx4_linear_bytes(rows, k), status)
check()
assert (values(y, (rows, n)) == 256.0).all()
st = np.empty(1, np.uint32)
ok(cu.cuMemcpyDtoH_v2(st.ctypes.data_as(C.c_void_p), C.c_uint64(status), C.c_size_t(4)))
assert st[0] == 0
print("same context")
"""


def test_a_context_is_bound_where_there_is_none_alone():
    """A launch into another context than its pointers' would read outside its memory, so this much is read from the source."""
    b = body(code("tensor.cuh"), "encode_tiled")
    assert re.search(r"if \(current\(&context\) != CUDA_SUCCESS \|\| !context\) \{[^{}]*cudaSetDevice\(", b)
    assert b.count("cudaSetDevice(") == 1
    for name in ("mx4.cu", "gemm16.cuh", "gated.cu", "ortho.cu", "norm.cu"):
        assert "cudaSetDevice(" not in code(name)


@pytest.mark.gpu
def test_calls_in_a_context_of_the_callers_own():
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "same context" in r.stdout, r.stdout[-3000:]


@pytest.mark.gpu
def test_a_thread_without_a_context():
    """Its first call is a product."""
    import threading

    import torch
    from paper_2508_05700_b200 import mfet as m
    x, w = torch.ones(300, 256, dtype=torch.float16, device="cuda"), torch.full((128, 256), 1 / 64, dtype=torch.float16, device="cuda")
    h = torch.zeros(300, 128, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    errors = []

    def work():
        try:
            m.mfet_gated_linear(x, m.F16, 256, 300, w, 256, w, 256, 128, 256, m.ACT_NONE, h, 128, None, 0)
        except Exception as e:  # handed to the test's own thread
            errors.append(e)
    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not errors and bool((h == 16.0).all())
