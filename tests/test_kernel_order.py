"""The order of waits and barriers in kernels whose roles wait for one another, read from their sources: what such an order prevents is
a rare meeting of events (a wait that runs out for one warp and not for another, a kernel that starts early beside this one) that no test on a
GPU brings about safely."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_06412_b200", "csrc")


def _kernel(file, name):
    """The body of a kernel, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())
    at = text.index("{", text.index(name + "("))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i + 1]
    raise AssertionError("no end of " + name)


def test_epilogue_warps_of_the_adapters_enter_their_loop_together():
    """Each of the four warps has its own result of the bounded wait for t; the loop over features begins with barriers of all four."""
    body = _kernel("gemm_adapters_tc.cu", "gemm_adapters_tc_kernel")
    loop = [m.start() for m in re.finditer(r"for \(; j < n2 && ok; \+\+j\)", body)][-1]   # the first one is the multiplying warp's
    last_wait = body.rindex("mbar_wait(t_done", 0, loop)
    between = body[last_wait:loop]
    assert re.search(r"\bok = epilogue_warps_agree\(ok\);", between), "a warp whose wait ran out leaves the others at the loop's first barrier"
    assert not re.search(r"\bok =(?! epilogue_warps_agree)", between[between.index("epilogue_warps_agree"):]), "and its result stays agreed on"
    turn = body[loop:]
    assert turn.index("ok = epilogue_warps_agree(ok);") < turn.index("if (!ok) break;")


def test_adapters_hold_their_tensor_memory_before_the_next_kernel_may_start():
    """A kernel launched early may take tensor memory in its first instructions and then wait for this grid's end: if a CTA of this grid had
    still to get its own, neither would go on."""
    body = _kernel("gemm_adapters_tc.cu", "gemm_adapters_tc_kernel")
    assert body.index("griddep_wait()") < body.index("tc_alloc(") < body.index("griddep_launch()") and body.count("griddep_launch()") == 1
