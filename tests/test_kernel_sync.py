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


def test_the_four_bit_products_turns_are_told_apart():
    """A wait on a parity returns at once while the turn before the awaited one is still open.  A set of scale warps waits
    for the codes of its own pairs of stages alone, so for each stage k the codes of stage k - kStages, which the other set
    may have waited for, must be known to have arrived: their MMAs lie at or before the last stage three pairs back
    (waited for before the pair is written), or stage k - kStages is waited for by itself."""
    src = source("linear_mx4.cu")
    wide, mid, small = map(int, re.search(r"kStages = TN > 128 \? (\d+) : TN > 64 \? (\d+) : (\d+);", src).groups())
    places, group = int(re.search(r"kPlaces = (\d+);", src).group(1)), int(re.search(r"kGroup = (\d+);", src).group(1))
    assert "if (last2 >= 0) ok = all_wait(empty + last2 % S::kStages, last2 / S::kStages & 1);" in src and places == 3
    waits = re.search(r"if \(S::kStages < 2 \* S::kPlaces && brings_codes\)\s*"
                      r"for \(int k = max\(j, last2 \+ 1 \+ S::kStages\); ok && k < j \+ n; \+\+k\)\s*"
                      r"ok = all_wait\(empty \+ k % S::kStages, \(k / S::kStages - 1\) & 1\);.*?"
                      r"if \(brings_codes\)\s*for \(int k = j; ok && k < j \+ n; \+\+k\) "
                      r"ok = all_wait\(codes \+ k % S::kStages, k / S::kStages & 1\);", src, re.S)
    for stages in (wide, mid, small):
        own_wait = waits is not None and stages < 2 * places
        for nkb in range(1, 14):
            last, j = [], 0  # of the pairs so far
            for _ in range(12):  # tiles
                for kb in range(0, nkb, group):
                    n_group = min(group, nkb - kb)
                    for i in range(0, n_group, 2):
                        n = min(2, n_group - i)
                        through = last[-places] if len(last) >= places else -1  # MMAs known to be through
                        for k in range(j, j + n):
                            if k >= stages:
                                assert k - stages <= through or own_wait, (stages, nkb, k)
                                # the turn before that, of the barrier that tells it
                                assert k - 2 * stages <= through, (stages, nkb, k)
                        j += n
                        last.append(j - 1)
