"""A whole beam search beside one put together without the library's reordering and back-tracking: every beam keeps its
ids as a list, the slots' caches are copied whole in torch, and the selection is checked against its definition in 64
bits. The prompts' last tiles fill up and new ones begin behind them on the way."""
import numpy as np
import pytest
import torch

import tests.test_gpu_kv4_model as model_tests
from paper_2607_20357_gb300 import svl
from tests import kv4_reference as R

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

# The same rows take the same steps in the same slots, so logits should not differ at all; a summed log-probability of
# 40 tokens near 7 each is rounded to float32 some 120 times: 120 * 2^-24 * 280 = 2e-3 at the very worst, a tenth of
# that as errors of either sign add up.
TOL = 1e-3


class Slots:
    """The prompts in slots of a cache of the search's own size, and single decode steps."""

    def __init__(self, case, beams, steps, window, sinks):
        self.case, self.beams, self.window, self.sinks = case, beams, window, sinks
        B, d = case.b["B"], case.dims
        out = case.model.run(case.b, stages=("select", "pack"))
        lens = out["cu_seqlens"][1:] - out["cu_seqlens"][:-1]
        self.max_len = int(lens.max()) + steps - 1
        desc, cache, self.len, out, _ = model_tests._prefill(case, self.max_len, beams)
        self.slots = cache.view(d.n_layers, B, beams, -1)
        self.slots.copy_(self.slots[:, :, :1].clone().expand_as(self.slots))  # every beam has its sample's prompt
        self.cache, self.first = cache, out["logits"]
        self.gates = [case.b[n].repeat_interleave(beams, 0).contiguous() for n in ("layer_gate", "group_gate")]
        n = B * beams
        size = svl.svl_decode_kv4_workspace_size(case.model.handle, n, self.max_len)
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        self.logits = torch.empty(n, d.vocab, device="cuda")

    def step(self, tokens):
        svl.svl_decode_step_kv4(self.case.model.handle, self.len.numel(), model_tests._i32(tokens), self.cache,
                                self.max_len, self.len, *self.gates, self.window, self.sinks, self.logits, None, self.ws,
                                self.ws.numel())
        return self.logits

    def take_over(self, parents):
        at = torch.tensor(parents, device="cuda")
        for s in range(at.shape[0]):
            self.slots[:, s] = self.slots[:, s][:, at[s]].clone()


def _select(logits, scores, finished, eos, take):
    """svl_beam_select's answer, which has to be the definition's wherever scores lie farther apart than they round."""
    S, W = scores.shape
    dev = torch.as_tensor(logits).cuda().contiguous()
    V = dev.shape[-1]
    out = [torch.empty(S, take, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32, torch.uint8)]
    ws = torch.empty(max(svl.svl_beam_select_workspace_size(S, W, V, take), 256), dtype=torch.uint8, device="cuda")
    fin = None if finished is None else torch.as_tensor(finished).cuda()
    svl.svl_beam_select(S, W, V, take, dev, V, torch.as_tensor(scores).cuda(), fin, eos, *out, ws, ws.numel())
    got = [x.cpu().numpy() for x in out]
    x = dev.cpu().numpy().reshape(S, W, V)
    for s in range(S):
        want = R.beam_select(x[s], scores[s], None if finished is None else finished[s], eos, take + 1)
        near = np.diff([float(c[0]) for c in want]) > -1e-4
        if not near.any():
            assert [(int(p), int(t)) for p, t in zip(got[1][s], got[2][s])] == [(p, t) for _, p, t, _ in want[:take]]
        np.testing.assert_allclose(got[0][s], [c[0] for c in want[:take]], rtol=0, atol=1e-4)
    return got


def _search(case, beams, steps, eos, window, sinks):
    at = Slots(case, beams, steps, window, sinks)
    B = case.b["B"]
    got = _select(at.first.cpu(), np.zeros((B, 1), np.float32), None, eos, beams)
    ids = [[[int(t)] for t in row] for row in got[2]]
    moved = 0
    for _ in range(1, steps):
        logits = at.step([ids[s][w][-1] for s in range(B) for w in range(beams)])
        got = _select(logits, got[0], got[3], eos, beams)
        at.take_over(got[1].tolist())
        ids = [[ids[s][p] + [int(t)] for p, t in zip(got[1][s], got[2][s])] for s in range(B)]
        moved += int((got[1] != np.arange(beams)).sum())
    return ids, got[0], got[3], moved


def _own_scores(case, tokens, steps, eos, window, sinks):
    """Summed log-probabilities of each beam's ids, fed into slots that are never moved (up to its eos)."""
    at = Slots(case, tokens.shape[1], steps, window, sinks)
    logits, total, live = at.first.repeat_interleave(tokens.shape[1], 0), 0.0, 1.0
    for t in range(steps):
        tok = tokens[:, :, t].reshape(-1)
        total = total + live * torch.log_softmax(logits.double(), -1).gather(1, tok.long()[:, None])[:, 0]
        live = live * (tok != eos).double()
        if t + 1 < steps:
            logits = at.step(tok.tolist())
    return total.view(tokens.shape[:2]).cpu().numpy()


CASES = [(model_tests.MHA, 4, 0, 0), (model_tests.GQA, 3, 0, 0), (model_tests.GQA, 5, 8, 2), (model_tests.MHA, 4, 8, 0)]


@pytest.mark.parametrize("dims,beams,window,sinks", CASES, ids=["mha", "gqa", "gqa_window", "mha_window"])
def test_search_equals_one_put_together(dims, beams, window, sinks):
    """40 tokens behind prompts of 80 and 45 rows: positions 79 to 118 and 44 to 83, across tiles at 96 and at 64."""
    steps = 40
    case = model_tests._case(dims, 111, [64, 33], [16, 12])
    ids, scores, finished, moved = _search(case, beams, steps, -1, window, sinks)
    assert moved > 0
    got = case.model.beam_search(case.b, beams, steps, window=window, sinks=sinks)
    assert got["tokens"].tolist() == ids
    np.testing.assert_allclose(got["scores"].cpu().numpy(), scores, rtol=0, atol=TOL)
    assert not finished.any() and not got["finished"].any()
    own = _own_scores(case, got["tokens"], steps, -1, window, sinks)
    np.testing.assert_allclose(got["scores"].cpu().numpy(), own, rtol=0, atol=TOL)
    assert svl.svl_get_device_status(case.model.handle) == 0
    case.close()


@pytest.mark.parametrize("dims,beams", [(model_tests.MHA, 4), (model_tests.GQA, 3)], ids=["mha", "gqa"])
def test_search_with_an_end(dims, beams):
    """The second best first id as eos: the beam that takes it at once stands in the search from its first step on."""
    steps = 12
    case = model_tests._case(dims, 113, [64, 20], [16, 5], gates=False)
    eos = int(case.model.run(case.b)["logits"][0].topk(2).indices[1])
    ids, scores, finished, _ = _search(case, beams, steps, eos, 0, 0)
    got = case.model.beam_search(case.b, beams, steps, eos=eos)
    assert got["tokens"].tolist() == ids
    np.testing.assert_array_equal(got["finished"].cpu().numpy(), finished)
    np.testing.assert_allclose(got["scores"].cpu().numpy(), scores, rtol=0, atol=TOL)
    own = _own_scores(case, got["tokens"], steps, eos, 0, 0)
    np.testing.assert_allclose(got["scores"].cpu().numpy(), own, rtol=0, atol=TOL)
    assert finished[0].any()
    for s in range(2):
        for w in range(beams):
            ends = [t for t, v in enumerate(ids[s][w]) if v == eos]
            assert bool(finished[s, w]) == bool(ends)
            assert not ends or ends == list(range(ends[0], steps))
    case.close()


def test_a_search_whose_beams_do_not_move_is_found_out(monkeypatch):
    """The check of scores above misses its mark without the reordering after the first step."""
    dims, beams, steps, window = model_tests.MHA, 4, 12, 8
    case = model_tests._case(dims, 115, [64, 33], [16, 12])
    reorder, select, parents = svl.svl_kv4_reorder, svl.svl_beam_select, []

    def selected(*args, **kw):
        select(*args, **kw)
        parents.append(args[10])

    def once(desc, cache, n_layers, W, parent, start_from, *rest, **kw):
        if start_from is None:  # (the prompt's hand-over)
            reorder(desc, cache, n_layers, W, parent, start_from, *rest, **kw)

    monkeypatch.setattr(svl, "svl_beam_select", selected)
    good = case.model.beam_search(case.b, beams, steps, window=window)
    moves = [p.cpu().numpy() for p in parents[1:]]
    assert any((p != np.arange(beams)).any() for p in moves[:-1])
    monkeypatch.setattr(svl, "svl_kv4_reorder", once)
    bad = case.model.beam_search(case.b, beams, steps, window=window)
    monkeypatch.undo()
    for got, right in ((good, True), (bad, False)):
        own = _own_scores(case, got["tokens"], steps, -1, window, 0)
        assert (np.abs(got["scores"].cpu().numpy() - own).max() <= TOL) == right
    case.close()
