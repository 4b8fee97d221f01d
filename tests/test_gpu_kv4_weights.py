"""How exactly the 4-bit cache's attention holds its weights: rows of V that nearly cancel, so that the output's own
rounding does not cover theirs."""
import numpy as np
import pytest
import torch

import tests.test_gpu_kv4 as kv4_tests
from paper_2607_20357_gb300 import svl
from tests import kv4_reference as R

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)


def bound(ref, spread, size, n):
    """Weights times scales are kept as two bf16 numbers of 8 bits. Up to four columns: the upper cut off (what is left is
    under 2^-7 of the product), the lower rounded (2^-8 of that): 2^-15. More: both of the weight rounded (2^-8, then 2^-8
    of what is left: 2^-16), and of the product with the scale (2^-8, then 2^-8 of the rest and of the weight's lower
    number, under 2^-7 together: 2^-15). Then n float32 additions, scores in float32 (2^-16 of their terms), and the
    output's rounding."""
    weights = 2.0 ** -15 + 2.0 ** -16 + n * 2.0 ** -24 + 2.0 ** -16 * (1 + size)
    return 2.0 ** -8 * np.abs(ref) + weights * spread * (1 + 2.0 ** -8)


@pytest.mark.parametrize("heads,kv,dh", [(2, 2, 64), (3, 1, 64), (16, 2, 64), (2, 2, 128), (4, 1, 128), (7, 1, 128)])
@pytest.mark.parametrize("n", [2, 6, 40, 200])
@pytest.mark.parametrize("room", [0, 13_000])
def test_rows_that_nearly_cancel(heads, kv, dh, n, room):
    g = torch.Generator().manual_seed(141)
    k = torch.randn(n, kv, dh, generator=g)
    k[1::2] = k[::2] + 0.1 * torch.randn(n // 2, kv, dh, generator=g)
    # whole numbers of a group's scale, so that a row and its negative are both held as they are
    v = torch.randint(-7, 8, (n, kv, dh // 32, 32), generator=g).float()
    v[..., 0] = -8.0
    v *= torch.exp2(torch.randint(-3, 4, (n, kv, dh // 32, 1), generator=g).float()) * 1.3125
    v[1::2] = -v[::2]
    k, v = (t.reshape(n, -1).to(torch.bfloat16) for t in (k, v))
    desc = svl.Kv4Desc(1, kv, dh, max(n + 3, room))
    cache = kv4_tests.new_cache(desc)
    kv4_tests.write(desc, cache, k.cuda(), v.cuda(), [n], None)
    kk, vv = (R.quantised(t.view(n, kv, dh)) for t in (k, v))
    np.testing.assert_array_equal(vv[1::2], -vv[::2])
    q = torch.randn(1, heads * dh, generator=g).to(torch.bfloat16)
    got = kv4_tests._attend(desc, cache, q, [n - 1], 1, heads, 0, 0, 0.02).reshape(heads, dh)
    qq = q.double().numpy().reshape(heads, dh)
    for h in range(heads):
        ref, spread, size = R.attention(qq[h], kk[:, h * kv // heads], vv[:, h * kv // heads], np.float32(0.02))
        err = np.abs(got[h] - ref)
        assert (err <= bound(ref, spread, size, n)).all(), (h, (err / bound(ref, spread, size, n)).max())
