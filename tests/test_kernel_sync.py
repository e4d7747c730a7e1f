"""Orders between threads that no run can be trusted to show broken, read from the kernels' source (CPU only)."""
import re

from test_kernel_source import source


def body(src, head):
    """The text from a function's head to the end of its outermost braces."""
    at = src.index(head)
    depth, i = 0, src.index("{", at)
    for j in range(i, len(src)):
        depth += {"{": 1, "}": -1}.get(src[j], 0)
        if depth == 0:
            return src[at: j + 1]
    raise AssertionError(head)


def test_group_flags_are_ordered_between_lanes():
    """A token's lanes write the flags of their own groups and read those of all: a __syncwarp (shuffles order no memory)
    stands between each write and the reads that follow it, and between reads and the next write."""
    kernel = body(source("route_topk.cu"), "topk_lists_kernel(")
    write = kernel.index("kept[g] = ")
    call = kernel.index("settle_groups(")
    assert "__syncwarp();" in kernel[write: call]
    assert "__syncwarp();" in kernel[call: kernel.index("kept[", call)]
    settle = body(source("route_topk.cu"), "bool settle_groups(")
    read, write = settle.index("kept[g]"), settle.index("kept[g_of] = ")
    assert read < write and re.search(r"__syncwarp\(m8\);", settle[read: write])
