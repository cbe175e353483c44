"""The clipping, row and matrix calls on the bounds-checked build: their tests again in a child process, with no access reported outside its
array (the report is printed by the kernel; calls with a status word set MFET_DEV_BOUNDS in it as well, which the tests would see)."""
import os
import re
import subprocess
import sys

import pytest

from tests.test_operator_sources import code

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TESTS = ["tests/test_gpu_rows.py", "tests/test_gpu_grad_clip.py", "tests/test_gpu_clip_calls.py", "tests/test_gpu_mx4.py",
         "tests/test_gpu_mx4_calls.py", "tests/test_gpu_mxfp4_tables.py", "tests/test_gpu_example.py"]


def test_every_kernel_of_these_calls_has_checks():
    for name, kernels in (("rows.cu", ["rows_write_kernel", "rows_read_kernel"]), ("gradclip.cu", ["piece_squares", "piece_scale"]),
                          ("mx4.cu", ["mx4_quantize_kernel", "mx4_few_kernel", "mx4_gemm_kernel"])):
        text = code(name)
        for k in kernels:
            head = re.search(r"\b%s\((?=const|RowsParams)" % k, text).start()  # the definition
            start = text.index("{", head)
            end = text.index("\n}\n", start)
            assert "MFET_INSIDE" in text[start:end], (name, k)


@pytest.mark.gpu
def test_no_access_outside_on_the_bounds_checked_build():
    from paper_2508_05700_b200 import build
    lib = build.build(checked=True)
    env = dict(os.environ, MFET_LIBRARY=lib)
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-s", "-m", "gpu", "-p", "no:cacheprovider"] + TESTS +
                       ["-k", "not costs_one_pass"], cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=1500)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:]
    assert "index out of bounds" not in r.stdout, [l for l in r.stdout.splitlines() if "out of bounds" in l][:10]
