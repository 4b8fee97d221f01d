"""Attention over the 4-bit cache with queries at both ends of bf16's range: scores of ordinary size stay finite and
right however large or small the queries are that they come from."""
import numpy as np
import pytest
import torch

import tests.test_gpu_kv4 as kv4_tests
from paper_2607_20357_gb300 import svl
from tests import kv4_reference as R

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

BF16 = torch.bfloat16
SHAPES = [(2, 2, 64, 1), (3, 1, 64, 1), (16, 2, 64, 1), (2, 2, 128, 1), (6, 2, 128, 1), (8, 1, 128, 1), (28, 4, 128, 3)]


def _check(heads, kv, dh, rows, q, power, scale):
    """300 and 40 rows of V of ordinary size and K of 2^power, in a cache that a cluster and one that all CTAs walk."""
    counts = [300, 40]
    x = kv4_tests.rows_of(91, sum(counts), 2 * kv * dh).float()
    k, v = (x[:, :kv * dh] * 2.0 ** power).to(BF16), x[:, kv * dh:].to(BF16)
    kk, vv = (R.quantised(t.view(-1, kv, dh)) for t in (k, v))
    for max_len in (305, 13_000):
        desc = svl.Kv4Desc(2, kv, dh, max_len)
        cache = kv4_tests.new_cache(desc)
        kv4_tests.write(desc, cache, k.cuda(), v.cuda(), counts, None)
        kv4_tests._check_attention(desc, cache, q, [c - rows for c in counts], rows, heads, 0, 0,
                                   lambda b, j: (kk[j + counts[0] * b], vv[j + counts[0] * b]), scale)


def _queries(heads, dh, rows):
    """Elements under 2 (a standard normal's, cut off)."""
    g = torch.Generator().manual_seed(92)
    return torch.randn(2 * rows, heads * dh, generator=g).clamp(-1.9, 1.9)


@pytest.mark.parametrize("heads,kv,dh,rows", SHAPES)
@pytest.mark.parametrize("power,scale", [(117, 1.0), (118, 1.0), (121, None), (125, None), (127, -(2.0 ** -6)),
                                         (100, 2.0 ** 20), (-100, None), (-120, 1.0)])
def test_queries_of_any_size(heads, kv, dh, rows, power, scale):
    """Keys small or large enough to undo the queries' size (and the scale's, where it has one)."""
    q = (_queries(heads, dh, rows) * 2.0 ** power).to(BF16)
    assert bool(torch.isfinite(q.float()).all())
    undo = -power - (20 if scale and scale > 1 else 0)
    _check(heads, kv, dh, rows, q, max(undo, -121), scale)


@pytest.mark.parametrize("heads,kv,dh,rows", SHAPES)
def test_a_huge_query_beside_ordinary_and_tiny_ones(heads, kv, dh, rows):
    """One head's queries at the end of the range, its neighbours' not: each against the same keys of 2^-121."""
    q = _queries(heads, dh, rows).view(2 * rows, heads, dh)
    q[:, 0] *= 2.0 ** 126
    q[:, 1::3] *= 2.0 ** 119
    q[:, 2::3] *= 2.0 ** -110
    q = q.view(2 * rows, -1).to(BF16)
    _check(heads, kv, dh, rows, q, -121, None)


def test_the_largest_query_that_there_is():
    q = torch.full((2, 4 * 128), torch.finfo(BF16).max, dtype=BF16)
    q[:, ::2] *= -1
    _check(4, 4, 128, 1, q, -121, None)


def test_the_sign_of_a_scale_that_needs_two_factors():
    """A negative scale prefers the keys that a positive one shuns."""
    desc = svl.Kv4Desc(1, 1, 64, 40)
    k = torch.zeros(2, 64)
    k[0, 0], k[1, 0] = 2.0 ** -110, -(2.0 ** -110)
    v = torch.zeros(2, 64)
    v[0], v[1] = 1.0, 2.0
    cache = kv4_tests.new_cache(desc)
    kv4_tests.write(desc, cache, k.to(BF16).cuda(), v.to(BF16).cuda(), [2], None)
    q = torch.zeros(1, 64)
    q[0, 0] = 2.0 ** 125
    for scale, want in ((1.0, 1.0), (-1.0, 2.0)):
        got = kv4_tests._attend(desc, cache, q.to(BF16), [1], 1, 1, 0, 0, scale)
        np.testing.assert_array_equal(got, np.full((1, 64), want))
