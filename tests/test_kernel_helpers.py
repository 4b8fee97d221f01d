"""Device functions that nothing calls (no GPU needed)."""
import glob
import os
import re

from tests.test_kernel_sources import CSRC, _code


def test_every_device_function_is_called():
    files = {p: _code(p) for p in sorted(glob.glob(os.path.join(CSRC, "*.cu*")))}
    everything = "\n".join(files.values())
    names = [n for code in files.values() for n in re.findall(r"\bSVL_DEVINL\s+[\w:<>*&\s]*?\b(\w+)\s*\(", code)]
    assert len(names) > 50
    unused = [n for n in names if len(re.findall(r"\b%s\b" % n, everything)) < 2]
    assert not unused
