"""The order of a kernel's set-up, which no result shows (no GPU needed)."""
import glob
import os
import re

from tests.test_kernel_sources import CSRC, _code


def test_tensor_memory_is_taken_before_the_next_kernel_may_start():
    """A CTA that has let its successors start waits for no tensor memory: they keep theirs until it has ended."""
    kernels = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        code = _code(path)
        for body in re.split(r"\b__global__\b", code)[1:]:
            body = body[:body.find("\n}\n")]
            took = re.search(r"\btmem_alloc(_pair)?\(", body)
            started = re.search(r"\bpdl_(trigger|begin)\(", body)
            if took:
                kernels += 1
                assert started and took.start() < body.find("__syncthreads()", took.start()) < started.start(), path
    assert kernels >= 5
