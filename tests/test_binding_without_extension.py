"""The binding on a Python for which the extension of the frequent calls was not built: the same calls, through ctypes."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIDE = "import sys; sys.modules['paper_2508_05700_b200._fastcall'] = None; import pytest; sys.exit(pytest.main(sys.argv[1:]))"


def run(*args):
    r = subprocess.run([sys.executable, "-c", HIDE, "-x", "-q", "-p", "no:cacheprovider"] + list(args), cwd=ROOT, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=900)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:]


def test_arguments_and_refusals_are_the_same():
    run("tests/test_operator_arguments.py", "tests/test_abi.py")


def test_a_build_without_a_compiler_leaves_no_extension(tmp_path, monkeypatch):
    from paper_2508_05700_b200 import build
    target = tmp_path / "_fastcall.so"
    target.write_bytes(b"of an older source")
    monkeypatch.setattr(build, "FASTCALL", str(target))
    for compiler in ("false", str(tmp_path / "none")):
        monkeypatch.setenv("CC", compiler)
        assert build.build_fastcall(force=True) is None and not target.exists()


@pytest.mark.gpu
def test_results_are_the_same():
    run("-m", "gpu", "tests/test_gpu_rows.py", "tests/test_gpu_mx4.py", "tests/test_gpu_grad_clip.py", "-k",
        "another_stream or two_streams or counts or nan_blocks or in_place or plain_tables")
