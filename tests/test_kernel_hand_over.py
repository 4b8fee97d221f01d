"""How a warp hands an accumulator over to the MMAs of another CTA, which no result shows (no GPU needed)."""
import os
import re

from tests.test_kernel_sources import CSRC, _code


def body(code, name):
    """The text between the braces of a function."""
    found = re.search(r"\b%s\s*\([^;{]*\)\s*\{" % name, code)
    assert found, name
    at = found.end() - 1
    depth = 0
    for i in range(at, len(code)):
        depth += (code[i] == "{") - (code[i] == "}")
        if depth == 0:
            return code[at:i]


def test_reads_of_tensor_memory_are_ordered_before_the_arrival():
    """The arrival is relaxed, so every path to it has the fence for tensor memory, and all of the warp's lanes."""
    code = _code(os.path.join(CSRC, "mxf4_pair.cu"))
    hand_over = body(code, "hand_over")
    assert re.search(r"\btc_fence_before\(\);\s*__syncwarp\(\);\s*if \(lane == 0\) mbar_arrive_cluster_relaxed\(", hand_over)
    epilogue = body(code, "mx_pair_epilogue")
    assert "mbar_arrive" not in epilogue and epilogue.count("hand_over(") >= 2


def test_nothing_is_handed_over_behind_the_last_tile():
    """Nobody waits for that arrival, and the CTA that it goes to may have ended when it gets there."""
    epilogue = body(_code(os.path.join(CSRC, "mxf4_pair.cu")), "mx_pair_epilogue")
    assert re.search(r"const bool last = ch\.t \+ w\.stride >= p\.tiles;", epilogue)
    assert re.search(r"bool handed = last \|\| ", epilogue)  # the loop over chunks hands over only what is not
    assert re.search(r"if \(handed && !last\) hand_over\(", epilogue)
    assert re.search(r"if \(!handed && [^{]*\{\s*hand_over\(", epilogue)
    assert epilogue.count("hand_over(") == 2
