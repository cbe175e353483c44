"""The layer norm, gated block and orthogonalising calls on the bounds-checked build: their tests again in a child process, with no access reported
outside its array."""
import os
import re
import subprocess
import sys

import pytest

from tests.test_operator_sources import code

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TESTS = ["tests/test_gpu_layer_norm.py", "tests/test_gpu_gated.py", "tests/test_gpu_orthogonalize.py", "tests/test_gpu_block_example.py",
         "tests/test_gpu_mx4_edges.py"]


def test_every_kernel_of_these_calls_has_checks():
    for name in ("norm.cu", "gated.cu", "ortho.cu", "gemm16.cuh"):
        text = code(name)
        found = [m.end() for m in re.finditer(r"__global__ void[^;{]*?\b\w+_kernel\(const", text)]
        for at in found:
            start = text.index("{", at)
            body = text[start:text.index("\n}\n", start)]
            inside = "MFET_INSIDE" in body or "eight<" in body or "eight_of<" in body
            assert inside, (name, text[at - 40:at])
        assert found or name == "gated.cu"


@pytest.mark.gpu
def test_no_access_outside_on_the_bounds_checked_build():
    from paper_2508_05700_b200 import build
    lib = build.build(checked=True)
    env = dict(os.environ, MFET_LIBRARY=lib)
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-s", "-m", "gpu", "-p", "no:cacheprovider"] + TESTS, cwd=ROOT, env=env,
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=1500)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:]
    assert "index out of bounds" not in r.stdout, [l for l in r.stdout.splitlines() if "out of bounds" in l][:10]
