"""Rules of the kernels of the clipping, row and matrix calls that no run on a GPU can show: read from the sources (no GPU needed)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_05700_b200", "csrc")


def code(name):
    """A source file without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)


def body(text, name):
    """The braces of the function `name`, its last definition."""
    at = [m.start() for m in re.finditer(r"\b%s\(" % name, text)][-1]
    start = text.index("{", text.index(")", at))
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[start:i + 1]
    raise AssertionError(name)


def test_a_cluster_has_started_before_its_shared_memory_is_written():
    """Memory of another block of the cluster exists once that block runs: a barrier comes ahead of the first access and one behind the last."""
    found = 0
    for name in sorted(os.listdir(CSRC)):
        text = code(name) if name.endswith((".cu", ".cuh")) else ""
        for kernel in re.findall(r"__cluster_dims__[^{;]*?(\w+)\(const", text, flags=re.S):
            b = body(text, kernel)
            first, last = b.index("shared::cluster"), b.rindex("st.shared::cluster")
            waits = [m.start() for m in re.finditer(r"barrier\.cluster\.wait", b)]
            assert waits and waits[0] < first, kernel
            assert waits[-1] > last, kernel
            found += 1
    assert found == 1


def test_gradients_are_not_read_through_the_read_only_path():
    """Clipping in place writes what the same kernel has read, which that path does not allow for."""
    text = code("gradclip.cu")
    assert "ld.global.nc" not in text and "__ldg(" not in text


def test_the_product_ends_with_nothing_under_way():
    """When a wait of the product has run out in one role, the other roles may have ended before: copies and products are waited for once all roles
    have, and only then is the tensor memory freed."""
    b = body(code("mx4.cu"), "mx4_gemm_kernel")
    last_role = b.index("cp.async.bulk.wait_group.read 0;")
    joined = b.index("__syncthreads();", last_role)
    copies, products = b.rindex("bar_wait(full("), b.rindex("mma_commit(drained)")
    assert joined < copies and joined < products
    assert b.index("bar_wait(drained", products) < b.index("__syncthreads();", max(copies, products)) < b.index("tcgen05.dealloc")


def test_no_line_of_the_l2_cache_is_kept_beyond_a_call():
    """A line that is marked to leave last stays in the way of the next kernels when the second pass does not read it."""
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh")):
            assert "evict_last" not in code(name), name
