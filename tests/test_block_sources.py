"""Rules of the layer norm, gated block and orthogonalising kernels that no run on a GPU can show: read from the sources (no GPU needed)."""
import re

from tests.test_operator_sources import body, code


def test_shared_memory_of_another_block_is_touched_between_cluster_barriers():
    for name, kernel, first, last in (("gemm16.cuh", "gemm16_kernel", "peer_load(", "peer_load("), ("ortho.cu", "ortho_small_kernel", "ld.shared::cluster", "peer_load(")):
        text = code(name)
        b = body(text, kernel) if name == "gemm16.cuh" else text[text.index("ortho_small_kernel(const"):]
        b = b[b.index("{"):]
        assert b.index("cluster_sync()") < b.index(first), kernel
        assert re.search(r"cluster(_or_block)?_sync\(", b[b.rindex(last):]), kernel


def test_the_product_ends_with_nothing_under_way():
    """After a wait that ran out: copies and products are waited for once all roles have ended, and only then is the tensor memory freed."""
    b = body(code("gemm16.cuh"), "gemm16_kernel")
    joined = b.index("__syncthreads();", b.index("if (warp >= 2) {"))
    copies, products = b.rindex("bar_wait(full("), b.rindex("commit<CTAS>(drained")
    assert joined < copies and joined < products
    assert b.index("bar_wait(drained", products) < b.index("__syncthreads();", max(copies, products)) < b.index("tcgen05.dealloc")


def test_every_wait_has_a_limit():
    for name in ("tensor.cuh", "gemm16.cuh", "ortho.cu"):
        text = code(name)
        for f in re.findall(r"mbarrier\.(?:try|test)_wait", text):
            assert name == "tensor.cuh"
    for f in ("bar_wait", "bar_sleep"):
        assert "kStallNs" in body(code("tensor.cuh"), f)


def test_no_copy_goes_to_several_blocks():
    for name in ("tensor.cuh", "gemm16.cuh", "gated.cu", "ortho.cu", "norm.cu", "mx4.cu"):
        for line in code(name).splitlines():
            assert not ("cp.async.bulk" in line and "multicast" in line)
