"""Both gradients of the gated block in one launch, in fp16."""
import pytest

from tests.test_gpu_gated import Block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k,act,pad,shift", [(8192, 1024, 896, "silu", 0, 0), (5000, 1500, 700, "gelu", 3, 1), (19000, 700, 260, "none", 0, 0),
                                                 (12000, 130, 2000, "sigmoid", 8, 0)])
def test_both_gradients_in_one_launch(m, n, k, act, pad, shift):
    """More tiles of 256 x 256 than the GPU takes at a time, of products of different lengths."""
    b = Block(m, n, k, "f16", act, pad, shift, seed=m)
    b.backward()
    b.check_backward()
