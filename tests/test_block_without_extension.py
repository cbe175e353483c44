"""The layer norm, gated block and orthogonalising calls on a Python for which the extension of the frequent calls was not built."""
import pytest

from tests.test_binding_without_extension import run


def test_arguments_and_refusals_are_the_same():
    run("tests/test_block_arguments.py")


@pytest.mark.gpu
def test_results_are_the_same():
    run("-m", "gpu", "tests/test_gpu_layer_norm.py", "tests/test_gpu_gated.py", "tests/test_gpu_orthogonalize.py", "-k", "captured or other_streams")
