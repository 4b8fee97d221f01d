"""Limits that the calls of one beam search share: how many slots a model's calls take, and that the reordering takes
every cache that the other calls do."""
import pytest
import torch

import tests.test_gpu_kv4_model as model_tests
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


def test_slots_that_a_decode_step_does_not_take_are_refused_by_the_prefill():
    case = model_tests._case(model_tests.MHA, 123, [10], [5], gates=False)
    m, b = case.model, case.b
    P = 1 << 20

    def prefill(B, beams):  # (a workspace that is too small: nothing is launched whatever the answer)
        with pytest.raises(svl.SvlError) as e:
            svl.svl_gated_prefill_kv4(m.handle, B, 15, P, P, P, b["layer_gate"], b["group_gate"], 0, P, P, 64, beams, P,
                                      P, 64)
        return e.value.code
    assert prefill(4096, 1) == prefill(256, 16) == 7
    assert prefill(4097, 1) == prefill(257, 16) == prefill(1024, 16) == prefill(1, 4097) == 3
    size = svl.svl_decode_kv4_workspace_size
    assert size(m.handle, 4096, 64) > 0
    assert size(m.handle, 4097, 64) == 0
    with pytest.raises(svl.SvlError) as e:
        svl.svl_decode_step_kv4(m.handle, 4097, P, P, 64, P, P, P, 0, 0, P, P, P, 1 << 40)
    assert e.value.code == 3
    case.close()
