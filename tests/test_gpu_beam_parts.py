"""Beam selection where a row's parts are shorter than a chunk for every warp of a block, and just around that."""
import pytest
import torch

from tests.test_gpu_beam import check, random_case

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)


@pytest.mark.parametrize("V", [4095, 4097, 4608, 5000, 8193, 9000, 12289, 20481])
@pytest.mark.parametrize("S,W,take", [(1, 1, 32), (2, 3, 32), (40, 16, 7)])
def test_vocabularies_around_the_parts_edges(V, S, W, take):
    x, c = random_case(131 + V, S, W, V)
    check(x, c, None, 5, take)
    # the best ones all at the end, in the last part's last warp
    x[..., -take:] += 50
    check(x, c, None, V - 1, take, ld=V + 1)
