"""Beam search and the room that its cache has: a search that does not fit is refused, one that just fits is right."""
import pytest
import torch

import tests.test_gpu_kv4_model as model_tests
from paper_2607_20357_gb300 import svl

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)


def _short(case, max_seq):
    """A model of the case's weights for sequences of up to max_seq positions."""
    return svl.GatedPrefill(case.dims, case.w, max_seq=max_seq)


def test_a_search_without_room_is_refused():
    """Prompts of 80 and 45 rows in a model of 85 positions: six tokens feed five rows, up to position 84; a seventh
    token would need a position that there is not. The longest search that fits is what a longer model gives."""
    case = model_tests._case(model_tests.GQA, 101, [64, 33], [16, 12], gates=False)
    m = _short(case, 85)
    want = case.model.beam_search(case.b, 3, 6)
    got = m.beam_search(case.b, 3, 6)
    for name in ("tokens", "scores", "finished", "cache_len"):
        assert torch.equal(got[name], want[name]), name
    assert got["cache_len"].tolist() == [85] * 3 + [50] * 3
    assert svl.svl_get_device_status(m.handle) == 0
    for steps in (7, 400):
        with pytest.raises(ValueError, match="max_seq"):
            m.beam_search(case.b, 3, steps)
    assert svl.svl_get_device_status(m.handle) == 0
    m.close()
    # a prompt longer than the model: refused whatever the steps
    m = _short(case, 79)
    with pytest.raises(ValueError, match="max_seq"):
        m.beam_search(case.b, 3, 1)
    assert svl.svl_get_device_status(m.handle) == 0
    m.close()
    # a prompt that fills it: one token, for which no row is fed
    m = _short(case, 80)
    one = m.beam_search(case.b, 3, 1)
    assert torch.equal(one["tokens"], case.model.beam_search(case.b, 3, 1)["tokens"])
    assert one["cache_len"].tolist() == [80] * 3 + [45] * 3
    m.close()
    case.close()


def test_room_is_counted_after_the_selection():
    """Visual tokens that the selection drops need no room: 64 of which 10 are kept, with 16 of text."""
    case = model_tests._case(model_tests.MHA, 103, [64], [16], gates=False)
    case.b["keep_count"].fill_(10)
    m = _short(case, 30)
    got, want = m.beam_search(case.b, 2, 5), case.model.beam_search(case.b, 2, 5)
    assert torch.equal(got["tokens"], want["tokens"]) and torch.equal(got["scores"], want["scores"])
    assert got["cache_len"].tolist() == [30] * 2
    assert svl.svl_get_device_status(m.handle) == 0
    m.close()
    case.close()
