"""What the one-launch update does after a wait that ran out, read from its source (no GPU run may stall)."""
import re

from tests.test_operator_sources import code


def kernel():
    text = code("ortho.cu")
    b = text[text.index("ortho_small_kernel(const"):]
    return b[b.index("{"):b.index("\n}\n")]


def test_a_wait_that_ran_out_is_noticed():
    b = kernel()
    assert re.search(r"auto done = \[&\]\(\) \{\s*ok = __all_sync\(kAllLanes, ok && bar_wait\(bar, phase, &dead\)\);", b)
    assert b.count("bar_wait(") == 2  # that one, and the last one


def test_no_products_are_issued_and_no_operands_written_after_it():
    b = kernel()
    loop = b[b.index("for (int step = 0;"):]
    loop = loop[:loop.index("mma_commit(drained)")]
    assert len(re.findall(r"if \(warp == 0 && ok\) \{\s*if \(elect_one\(\)\) \{\s*issues = true;", loop)) == loop.count("mma_commit(bar)") == 3
    # every store to shared memory in the steps stands in a loop that `ok` ends
    stores = [m.start() for m in re.finditer(r"put_words\(|\*reinterpret_cast<(?:uint4|float4)\*>\(smem", loop)]
    assert len(stores) == 8
    for at in stores:
        head = max(loop.rfind("ok && c <", 0, at), loop.rfind("if (!ok ||", 0, at))
        assert head > loop.rfind("done();", 0, at) and head > loop.rfind("cluster_sync();", 0, at)


def test_every_block_comes_to_every_barrier():
    b = kernel()
    loop = b[b.index("for (int step = 0;"):b.index("mma_commit(drained)")]
    assert "return" not in loop
    for m in re.finditer(r"cluster_sync\(\);|ready\(\);", loop):  # not inside anything that `ok` decides
        depth, guarded = 0, False
        for line in reversed(loop[:m.start()].splitlines()):
            depth += line.count("}") - line.count("{")
            if depth < 0:
                guarded |= "ok" in re.findall(r"\w+", line)
                depth = 0
        assert not guarded


def test_tensor_memory_is_freed_when_nothing_is_under_way():
    b = kernel()
    last = b.rindex("mma_commit(drained)")
    assert b.rindex("__syncthreads();", 0, last) > b.rindex("done();")  # `dead` is final
    assert re.search(r"if \(issues\) \{\s*mma_commit\(drained\);\s*bar_wait\(drained, 0, &none\);", b)
    assert last < b.index("cluster_or_block_sync(", last) < b.index("tcgen05.dealloc")
