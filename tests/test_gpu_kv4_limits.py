"""Limits that the calls of one beam search share: the reordering takes every cache that the other calls do."""
import pytest
import torch

from paper_2607_20357_gb300 import svl

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)


@pytest.mark.parametrize("layers,slots,beams,kv,length", [(33, 4096, 2, 1, 20), (70_000, 4, 4, 2, 20), (3, 65535, 1, 1, 40)])
def test_reorder_of_more_layers_and_samples_than_a_grid_is_high(layers, slots, beams, kv, length):
    desc = svl.Kv4Desc(slots, kv, 64, length)
    per = svl.svl_kv4_cache_size(desc) // slots
    assert layers * (slots // beams) > 65535
    # every slot of every layer holds 16-byte words of its own number
    number = torch.arange(layers * slots, device="cuda", dtype=torch.int64).view(-1, 1)
    old = torch.cat((number, -1 - number), 1)[:, None].expand(-1, per // 16, -1).contiguous()
    cache = old.clone()
    g = torch.Generator().manual_seed(121)
    parent = torch.randint(0, beams, (slots,), generator=g, dtype=torch.int32).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = torch.full((slots,), length, dtype=torch.int32, device="cuda")
    svl.svl_kv4_reorder(desc, cache, layers, beams, parent, None, lens, status)
    at = torch.arange(slots, device="cuda") // beams * beams + parent.long()
    assert torch.equal(cache.view(layers, slots, -1), old.view(layers, slots, -1)[:, at])
    assert int(status) == 0
