"""How many clusters of a kernel run at a time decides its grid, its form and the parts of its sum: the answer that is kept is that kernel's own."""
import re

from tests.test_operator_sources import code


def test_clusters_at_a_time_are_kept_for_each_kernel():
    """A table in a function template over the kernel's type would be one table: all forms of the product have the same type."""
    text = code("gemm16.cuh")
    assert re.search(r"template <auto Kernel>\s*int64_t clusters_at_once\(uint32_t members, uint32_t smem\)", text)
    calls = re.findall(r"clusters_at_once<gemm16_kernel<([^>]*)>>\([^;]*?, G::smem\)", text)
    assert len(calls) == 3 == text.count("clusters_at_once<")
    for at in re.finditer(r"clusters_at_once<gemm16_kernel<([^>]*)>>", text):  # G is that kernel's shape
        assert text.rindex("using G = Shape<%s>;" % at.group(1), 0, at.start()) > text.rindex("template <", 0, at.start())
