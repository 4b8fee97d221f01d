"""The 4-bit cache's attention and the model calls over it at their edges: values that are not finite in sight and in
queries, eight heads per KV head under gates, prompts that the cache has no room for, both ways to cut a call's work."""
import numpy as np
import pytest
import torch

import tests.test_gpu_kv4 as kv4_tests
import tests.test_gpu_kv4_model as model_tests
from paper_2607_20357_gb300 import svl, synth
from tests import kv4_reference as R

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

BF16 = torch.bfloat16
GQA8 = synth.reduced(model_tests.TINY.dims, n_layers=2, d_model=2048, n_heads=16, n_kv_heads=2, n_groups=2, c_vis=2048)


# One, three and eight columns; row `at` holds a V that is not a number in its second group, in a tile that every column
# sees whole, in the last one and in one far from the row that takes all the weight.
@pytest.mark.parametrize("n,at", [(40, 7), (40, 37), (4000, 7), (4000, 2000), (4000, 3995)])
@pytest.mark.parametrize("heads,kv,dh", [(2, 2, 64), (3, 1, 64), (16, 2, 64), (2, 2, 128), (6, 2, 128), (8, 1, 128)])
def test_a_nan_in_sight_shows_though_its_weight_is_zero(heads, kv, dh, n, at):
    """0 * NaN is a NaN, as in the formula; the other groups are the row of weight 1."""
    desc = svl.Kv4Desc(1, kv, dh, n + 5)
    k = torch.zeros(n, kv, dh)
    k[5, :, 0] = 8.0
    v = kv4_tests.rows_of(61, n, kv * dh).view(n, kv, dh)
    clean = v.clone()
    v[at, :, 40] = float("nan")
    cache = kv4_tests.new_cache(desc)
    kv4_tests.write(desc, cache, k.to(BF16).view(n, -1).cuda(), v.view(n, -1).cuda(), [n], None)
    q = torch.zeros(1, heads, dh)
    q[:, :, 0] = 400.0  # scores of 3,200 and 0: weights of 1 and e^-3200
    got = kv4_tests._attend(desc, cache, q.to(BF16).view(1, -1), [n - 1], 1, heads, 0, 0, 1.0)
    got = got.reshape(heads, dh // 32, 32)
    nan = np.isnan(got)
    assert nan[:, 1].all() and nan.sum() == heads * 32
    want = R.as_bf16(R.quantised(clean[5])).double().numpy().reshape(kv, dh // 32, 32)
    for h in range(heads):
        for g in range(dh // 32):
            if g != 1:
                np.testing.assert_array_equal(got[h, g], want[h * kv // heads, g])


@pytest.mark.parametrize("heads,kv,rows", [(4, 4, 1), (4, 4, 2), (8, 2, 1), (8, 2, 2), (28, 4, 3)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite_spoils_its_head_alone(heads, kv, rows, bad):
    dh, counts = 128, [3000, 45]
    desc = svl.Kv4Desc(2, kv, dh, 3000)
    cache, _ = kv4_tests._filled(62, desc, counts)
    starts = [c - rows for c in counts]
    q = kv4_tests.rows_of(63, 2 * rows, heads * dh)
    clean = kv4_tests._attend(desc, cache, q, starts, rows, heads, 0, 0, 0.088)
    assert np.isfinite(clean).all()
    r, h = 2 * rows - 1, heads - 2
    for row in (0, r):
        dirty = q.clone()
        dirty[row, h * dh + 77] = bad
        got = kv4_tests._attend(desc, cache, dirty, starts, rows, heads, 0, 0, 0.088).reshape(-1, heads, dh)
        want = clean.reshape(-1, heads, dh).copy()
        want[row, h] = np.nan
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("heads,kv", [(3, 3), (4, 1), (16, 2)])
def test_a_query_of_zeros_averages(heads, kv):
    desc = svl.Kv4Desc(2, kv, 64, 333)
    cache, look = kv4_tests._filled(64, desc, [333, 12])
    kv4_tests._check_attention(desc, cache, torch.zeros(2, heads * 64, dtype=BF16), [332, 11], 1, heads, 100, 7, look)


@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 5)])
def test_decode_step_with_eight_heads_per_kv_head(window, sinks):
    model_tests.test_decode_step_equals_its_parts(GQA8, window, sinks, svl.SVL_GEMM_BF16)


def test_a_prompt_that_the_cache_has_no_room_for():
    """The rows that have a place are stored and the logits are the whole prompt's; the slot cannot go on."""
    dims, short = model_tests.GQA, 45
    case = model_tests._case(dims, 65, [64, 20], [16, 9], gates=False)
    m, b = case.model, case.b
    desc, cache, cache_len, out, _ = model_tests._prefill(case, 120, 1)
    lens = cache_len.tolist()
    assert lens[0] > short > lens[1]
    assert svl.svl_get_device_status(m.handle) == 0
    want = out["logits"].cpu().numpy()
    desc2, cache2, cache_len2, out2, _ = model_tests._prefill(case, short, 1)
    assert svl.svl_get_device_status(m.handle) == svl.SVL_DEV_BAD_INDEX
    assert cache_len2.tolist() == lens
    np.testing.assert_array_equal(out2["logits"].cpu().numpy(), want)
    per, per2 = svl.svl_kv4_cache_size(desc), svl.svl_kv4_cache_size(desc2)
    counts = [short, lens[1]]
    for l in range(dims.n_layers):
        one = kv4_tests.read(desc, cache[l * per:], counts, [0, 0])
        two = kv4_tests.read(desc2, cache2[l * per2:], counts, [0, 0])
        for x, y in zip(one, two):
            kv4_tests.same(y, x)
            assert bool(torch.isfinite(x.float()).all())
    dws = torch.empty(svl.svl_decode_kv4_workspace_size(m.handle, 2, short), dtype=torch.uint8, device="cuda")
    nxt = torch.empty(2, dtype=torch.int32, device="cuda")
    logits = torch.empty(2, dims.vocab, device="cuda")
    svl.svl_decode_step_kv4(m.handle, 2, kv4_tests.i32([1, 2]), cache2, short, cache_len2, b["layer_gate"],
                            b["group_gate"], 0, 0, logits, nxt, dws, dws.numel())
    assert svl.svl_get_device_status(m.handle) == svl.SVL_DEV_BAD_INDEX
    assert cache_len2.tolist() == [lens[0], lens[1] + 1]
    assert int(nxt[0]) == -1 and int(nxt[1]) >= 0
    case.close()


# The same sizes as the other file's, in a cache with room for far more positions and with many slots: how a call's work
# is cut depends on both.
@pytest.mark.parametrize("heads,kv,dh,rows,starts,window,sinks", kv4_tests.test_attention.pytestmark[0].args[1])
def test_attention_in_a_cache_with_room_for_more(heads, kv, dh, rows, starts, window, sinks):
    desc = svl.Kv4Desc(len(starts), kv, dh, 13_000)
    cache, look = kv4_tests._filled(71, desc, [max(0, s + rows) for s in starts])
    q = kv4_tests.rows_of(72, len(starts) * rows, heads * dh + 8)
    kv4_tests._check_attention(desc, cache, q, starts, rows, heads, window, sinks, look)


@pytest.mark.parametrize("slots,heads,kv,dh,rows,window,sinks", [
    (40, 8, 4, 64, 3, 70, 5), (40, 4, 4, 128, 1, 40, 37), (13, 7, 1, 64, 1, 0, 0), (3, 12, 4, 128, 1, 0, 0),
    (8, 4, 4, 64, 1, 0, 0), (19, 8, 2, 128, 2, 0, 0), (38, 4, 2, 64, 1, 64, 1), (75, 2, 2, 128, 1, 0, 0),
    (152, 1, 1, 64, 1, 0, 0), (153, 1, 1, 64, 2, 0, 0), (7, 40, 2, 64, 16, 100, 0),
])
def test_attention_of_many_and_few_items(slots, heads, kv, dh, rows, window, sinks):
    rng = np.random.default_rng(slots)
    starts = rng.integers(-2, 300, slots).tolist()
    starts[0] = 400
    desc = svl.Kv4Desc(slots, kv, dh, 420)
    cache, look = kv4_tests._filled(73, desc, [max(0, s + rows) for s in starts])
    q = kv4_tests.rows_of(74, slots * rows, heads * dh)
    kv4_tests._check_attention(desc, cache, q, starts, rows, heads, window, sinks, look)


def test_beam_search_over_many_items_under_gates():
    dims = synth.reduced(model_tests.TINY.dims, n_layers=2, d_model=512, n_heads=8, n_kv_heads=8, n_groups=8, c_vis=512)
    model_tests.test_beam_search_scores_are_its_tokens_log_probabilities(dims, 16, 0)


def test_one_item_per_cluster_gives_the_same_bits_every_time():
    desc = svl.Kv4Desc(2, 4, 128, 4000)
    cache, _ = kv4_tests._filled(75, desc, [4000, 77])
    q = kv4_tests.rows_of(76, 2, 28 * 128)
    first = kv4_tests._attend(desc, cache, q, [3999, 76], 1, 28, 0, 0, 0.088)
    for _ in range(5):
        np.testing.assert_array_equal(first, kv4_tests._attend(desc, cache, q, [3999, 76], 1, 28, 0, 0, 0.088))


@pytest.mark.parametrize("kv,dh", [(1, 64), (3, 64), (1, 128), (5, 128)])
def test_one_row_per_slot_equals_rows_by_offsets(kv, dh):
    """Values of every kind, written both ways into caches that hold the same before: the same bytes."""
    n, cols = 60, kv * dh
    desc = svl.Kv4Desc(n, kv, dh, 70)
    x = kv4_tests.rows_of(77, n, 2 * cols + 16).float()
    x[1] = 0.0
    x[2], x[3] = 3.0, -3.0
    x[4, ::2], x[4, 1::2] = 5.0, -5.0
    x[5] = torch.arange(2 * cols + 16) % 33 - 16.0
    x[6, ::7] = float("nan")
    x[7, ::40], x[8, 3::50] = float("inf"), -float("inf")
    x[9], x[10] = x[9] * 2.0 ** -126, x[10] * 2.0 ** -122
    x[11] = 3e38
    x[12:20] = torch.randint(-255, 256, x[12:20].shape, generator=torch.Generator().manual_seed(78)).float()
    xd = x.to(BF16).cuda()
    k, v = xd[:, 8:8 + cols], xd[:, 16 + cols:]
    starts = [(7 * i) % 70 for i in range(n)]
    starts[20:24] = [-1, -70, 70, 2 ** 31 - 1]
    caches, status = [], []
    for row_off in (None, "ragged"):
        g = torch.Generator(device="cuda").manual_seed(79)
        cache = torch.randint(0, 256, (svl.svl_kv4_cache_size(desc),), dtype=torch.uint8, device="cuda", generator=g)
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        kv4_tests.write(desc, cache, k, v, [1] * n, starts, st, row_off)
        caches.append(cache)
        status.append(int(st))
    assert torch.equal(*caches)
    assert status == [svl.SVL_DEV_BAD_INDEX] * 2


def test_rows_without_a_place_are_reported_under_gates():
    """The first group is off in every layer; a prompt longer than the cache still shows."""
    dims = model_tests.GQA
    case = model_tests._case(dims, 81, [64], [16], gates=False)
    case.b["group_gate"][:, :, 0] = 0
    _, _, cache_len, _, _ = model_tests._prefill(case, 45, 1)
    assert cache_len.tolist()[0] > 45
    assert svl.svl_get_device_status(case.model.handle) == svl.SVL_DEV_BAD_INDEX
    case.close()
