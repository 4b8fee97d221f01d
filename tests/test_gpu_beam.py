"""Beam selection against its plain definition: scores within the rounding of their float32 operations, parents, ids
and finished flags equal."""
import numpy as np
import pytest
import torch

from paper_2607_20357_gb300 import svl
from tests import kv4_reference as R

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

INF = float("inf")


def select(logits, scores, finished, eos, take, ld=None, stream=None):
    """logits [S, W, V] float32 on the CPU."""
    S, W, V = logits.shape
    ld = ld or V
    dev = torch.full((S * W, ld), 1e30, device="cuda")
    dev[:, :V] = logits.view(S * W, V).cuda()
    sc = torch.as_tensor(scores, dtype=torch.float32).cuda()
    fin = None if finished is None else torch.as_tensor(finished, dtype=torch.uint8).cuda()
    out = [torch.full((S, take), -5, dtype=d, device="cuda") for d in (torch.float32, torch.int32, torch.int32)]
    out.append(torch.full((S, take), 77, dtype=torch.uint8, device="cuda"))
    ws = torch.empty(max(svl.svl_beam_select_workspace_size(S, W, V, take), 256), dtype=torch.uint8, device="cuda")
    svl.svl_beam_select(S, W, V, take, dev, ld, sc, fin, eos, *out, ws, ws.numel(), stream)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in out]


def check(logits, scores, finished, eos, take, ld=None):
    got = select(logits, scores, finished, eos, take, ld)
    x, c = logits.numpy(), np.asarray(scores, np.float32)
    for s in range(x.shape[0]):
        want = R.beam_select(x[s], c[s], None if finished is None else np.asarray(finished)[s], eos, take)
        for i, name in ((1, "parent"), (2, "token"), (3, "finished")):
            np.testing.assert_array_equal(got[i][s], [w[i] for w in want], err_msg=f"{name} of sample {s}")
        ref = np.array([w[0] for w in want], np.float32)
        np.testing.assert_array_equal(np.isneginf(got[0][s]), np.isneginf(ref))
        fine = np.isfinite(ref)
        # three roundings (lse, offset, sum) of numbers no larger than these, each 2^-24 of them, and lse's own error
        size = np.abs(x[s][np.isfinite(x[s])]).max(initial=0.0) + np.abs(c[s][np.isfinite(c[s])]).max(initial=0.0) + 20
        assert np.abs(got[0][s][fine].astype(np.float64) - ref[fine]).max(initial=0.0) <= 8 * 2.0 ** -24 * size
    return got


def random_case(seed, S, W, V, std=2.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(S, W, V, generator=g) * std, -10 * torch.rand(S, W, generator=g)


@pytest.mark.parametrize("S,W,V,take", [
    (1, 1, 1, 1), (1, 1, 5, 5), (3, 2, 7, 7), (2, 4, 33, 32), (1, 4, 32000, 4), (5, 3, 32003, 6), (2, 16, 1000, 32),
    (2, 8, 152064, 16), (70, 5, 999, 10), (1, 1, 152064, 32), (4, 2, 4096, 1), (2, 3, 8191, 3),
])
def test_random(S, W, V, take):
    x, c = random_case(S * 1000 + V, S, W, V)
    check(x, c, None, -1, take)
    check(x, c, None, min(2, V - 1), take, ld=V + 3)


def test_finished_beams_stand_for_themselves():
    x, c = random_case(1, 6, 4, 500)
    fin = np.zeros((6, 4), np.uint8)
    fin[0, 1] = fin[1, :3] = fin[2, :] = 1
    fin[3, 0] = 200  # any byte but 0
    c[1, 0] = 3.0
    c[2, 1] = -INF
    got = check(x, c, fin, 7, 8)
    # all four finished: four entries, then no continuations
    assert np.isneginf(got[0][2]).sum() == 5 and (got[3][2] == 1).all()


def test_first_step_expands_the_first_beam_alone():
    x, c = random_case(2, 3, 5, 1000)
    x[:] = x[:, :1]
    c[:] = -INF
    c[:, 0] = 0
    got = check(x, c, None, -1, 10)
    assert (got[1] == 0).all()


def test_equal_logits_and_equal_beams():
    """Ties: the lower beam, then the lower id."""
    x = torch.zeros(3, 3, 40000)
    x[1, :, 100:200] = 5.0
    x[2] = torch.randint(0, 3, (1, 40000), generator=torch.Generator().manual_seed(3)).float()
    check(x, np.zeros((3, 3), np.float32), None, 3, 32)
    # a tie that a whole block of equal values makes late in the row
    y = torch.full((1, 2, 30000), -1.0)
    y[..., 20000:] = 1.0
    check(y, np.zeros((1, 2), np.float32), None, -1, 32)
    # -0 and 0 are equal
    z = torch.zeros(1, 1, 3000)
    z[..., ::2] = -0.0
    check(z, np.zeros((1, 1), np.float32), None, -1, 8)


def test_ascending_descending_and_peaked_rows():
    """The best ones all in one place: at the end, at the start, in one thread's share."""
    V = 50000
    x = torch.empty(4, 1, V)
    x[0, 0] = torch.arange(V) / V
    x[1, 0] = -torch.arange(V) / V
    x[2] = -3
    x[2, 0, ::512] = torch.linspace(1, 2, len(range(0, V, 512)))
    x[3] = -3
    x[3, 0, 31000:31064] = torch.linspace(2, 1, 64)
    check(x, np.zeros((4, 1), np.float32), None, -1, 32)


def test_masked_logits():
    """-inf and the lowest float for ids that are not allowed; rows with too few or none that are."""
    low = torch.finfo(torch.float32).min
    x, c = random_case(4, 5, 3, 3001)
    x[0, :, 10:] = -INF
    x[1, :, 3:] = low
    x[2, 1] = -INF                       # this beam offers nothing
    x[3] = -INF                          # none does
    x[4, :, 2:] = -INF
    check(x, c, None, 1, 8)


def test_nan_and_infinite_logits():
    x, c = random_case(5, 4, 3, 2048)
    x[0, 1, 77] = float("nan")
    x[1, 2, 5] = INF
    x[2, 0, 9] = -float("nan")
    c[3, 1] = float("nan")
    got = check(x, c, None, -1, 6)
    assert not (got[1][0] == 1).any() and not (got[1][1] == 2).any() and not (got[1][3] == 1).any()


def test_large_and_equal_scores():
    """Scores so large that the logits vanish in them: the order within a beam stays that of the logits."""
    x, c = random_case(6, 2, 4, 700)
    c[0] = torch.tensor([-1e9, 0.0, -1e9, -1e9])
    c[1] = -1e30
    check(x, c, None, -1, 8)


def test_another_stream():
    x, c = random_case(7, 2, 4, 32000)
    a = select(x, c, None, 2, 8)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = select(x, c, None, 2, 8)
    for p, q in zip(a, b):
        np.testing.assert_array_equal(p, q)
