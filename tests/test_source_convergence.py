"""tcgen05.ld, .st and .wait are .sync.aligned: all lanes of a warp execute them together.  In the prompt attention's softmax
role, a branch that some lanes take alone is followed by a point where the warp is whole again (__syncwarp, a vote or a wait
by the whole warp) before the next such instruction, and no lane leaves a loop's body by itself.  What single lanes do inside
the loops is predicated instead."""
import os
import re

from paper_2404_14469_b200 import build

DIVERGE = r"if \((?:mine|lane [=<>!]=?|f_their)"
CONVERGE = r"__syncwarp\(|__any_sync\(|__all_sync\(|mbar_wait_warp\("
ALIGNED = r"tmem_(?:ld32|ld16|st16|wait_ld|wait_st|dealloc)\("


def _softmax_role():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "snapkv_prefill.cu")).read())
    kernel = text[text.index("prefill_kernel(const"):text.index("cudaError_t launch_prefill")]
    return kernel[kernel.index("const int t = warp >> 2"):]


def test_no_lane_leaves_alone():
    assert not re.search(r"if \((?:!mine|!?\(?lane\b)[^;{]*\)\s*(?:continue|break|return)", _softmax_role())


def test_the_warp_is_whole_in_front_of_aligned_instructions():
    events = [(m.lastgroup, m.group()) for m in
              re.finditer(f"(?P<diverge>{DIVERGE})|(?P<converge>{CONVERGE})|(?P<aligned>{ALIGNED})", _softmax_role())]
    kinds = [k for k, _ in events]
    assert "diverge" in kinds and kinds.count("aligned") >= 12
    apart = False
    for kind, what in events:
        if kind == "aligned":
            assert not apart, what
        apart = kind == "diverge" or (apart and kind != "converge")
    # and nothing of the kind in the loop that writes the results, whose next round begins with an aligned wait
    loop = _softmax_role()
    loop = loop[loop.index("const bool there"):loop.index("bar_of(t))")]
    assert not re.search(DIVERGE, loop) and "st_global_32" in loop
