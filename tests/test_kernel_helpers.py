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


def test_only_kernels_take_tensor_memory():
    """It is taken by two functions, which kernels call themselves: the order in a kernel's set-up is then seen in its own text."""
    calls = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu*"))):
        code = _code(path)
        for m in re.finditer(r"tcgen05\.alloc", code):
            name = re.findall(r"\bSVL_DEVINL\s+void\s+(\w+)\(", code[:m.start()])[-1]
            assert name in ("tmem_alloc", "tmem_alloc_pair"), path
        kernels = [b[:b.find("\n}\n")] for b in re.split(r"\b__global__\b", code)[1:]]
        uses = r"(?<!void )\btmem_alloc(?:_pair)?\("
        assert len(re.findall(uses, code)) == sum(len(re.findall(uses, b)) for b in kernels), path
        calls += len(re.findall(uses, code))
    assert calls >= 5
