"""Rules of the instruction set that no run can be trusted to show broken, read from the kernels' source (CPU only)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2107_02103_gb300", "csrc")


def source(name):
    """The file without its comments."""
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_register_moves_by_whole_warpgroups():
    """setmaxnreg: all warps of a warpgroup execute the same one, so each stands first in a branch on a warp number
    that begins a warpgroup, and every role has one."""
    src = source("linear_i8.cu")
    heads = re.findall(r"(?:if \((warp >= [\w:]+)\)|else) \{\s*if constexpr \(S::kWide\) "
                       r"asm volatile\(\"setmaxnreg\.\w+\.sync\.aligned\.u32 %0;\" ::\"n\"\((\w+)\)\);", src)
    assert heads == [("warp >= S::kMmaWarp", "kMmaRegs"), ("warp >= kEpiWarps", "kLoadRegs"), ("", "kEpiRegs")]
    assert src.count("setmaxnreg") == 3
    assert "kEpiWarps % 4 == 0 && kLoadWarps % 4 == 0 && kThreads % 128 == 0" in src
