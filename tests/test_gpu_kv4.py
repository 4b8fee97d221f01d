"""The 4-bit KV cache: quantising rows into it, reading them back, attention over it and the reordering of its slots,
against plain 64-bit definitions."""
import numpy as np
import pytest
import torch

from paper_2607_20357_gb300 import svl
from tests import kv4_reference as R

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

BF16 = torch.bfloat16


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def new_cache(desc, byte=0xFF):
    """A cache full of a byte: 0xFF makes every scale a NaN."""
    n = svl.svl_kv4_cache_size(desc)
    assert n == desc.n_slots * desc.n_kv_heads * -(-desc.max_len // 32) * 36 * desc.d_head
    return torch.full((n,), byte, dtype=torch.uint8, device="cuda")


def rows_of(seed, n, cols):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, cols, generator=g) * torch.exp(torch.randn(cols, generator=g))
    return x.to(BF16)


def offsets(counts):
    return np.concatenate(([0], np.cumsum(counts))).tolist()


def write(desc, cache, k, v, counts, starts, status=None, row_off="ragged"):
    n = k.shape[0]
    svl.svl_kv4_write(desc, cache, k, k.stride(0), v, v.stride(0), n, i32(offsets(counts)) if row_off else None,
                      None if starts is None else i32(starts), status)


def read(desc, cache, counts, starts, fill=7.0, row_off="ragged"):
    n, cols = sum(counts), desc.n_kv_heads * desc.d_head
    k, v = (torch.full((max(n, 1), cols), fill, dtype=BF16, device="cuda") for _ in range(2))
    svl.svl_kv4_read(desc, cache, n, i32(offsets(counts)) if row_off else None,
                     None if starts is None else i32(starts), k, cols, v, cols)
    return k[:n].cpu(), v[:n].cpu()


def expected(x, desc):
    q = R.quantised(x.view(x.shape[0], desc.n_kv_heads, desc.d_head))
    return R.as_bf16(q.reshape(x.shape))


def same(got, want):
    np.testing.assert_array_equal(got.float().numpy(), want.float().numpy())


# ------------------------------------------------------------------ write and read
@pytest.mark.parametrize("kv,dh,counts,starts", [
    (1, 64, [1], [0]), (4, 128, [1], [31]), (2, 64, [0, 5, 0, 33, 1], [0, 3, 7, 31, 64]),
    (4, 128, [100, 32, 31, 65], [0, 32, 1, 30]), (3, 64, [7] * 9, [0, 1, 2, 3, 15, 16, 17, 31, 63]),
    (32, 128, [40, 3], [0, 90]), (5, 128, [64], [32]),
])
def test_rows_come_back_as_quantised(kv, dh, counts, starts):
    desc = svl.Kv4Desc(len(counts), kv, dh, 130)
    n, cols = sum(counts), kv * dh
    wide = rows_of(1, n, 2 * cols + 24)  # K and V as columns of wider rows
    wd = wide.cuda()
    cache = new_cache(desc)
    write(desc, cache, wd[:, 8:8 + cols], wd[:, 16 + cols:16 + 2 * cols], counts, starts)
    k, v = read(desc, cache, counts, starts)
    same(k, expected(wide[:, 8:8 + cols], desc))
    same(v, expected(wide[:, 16 + cols:16 + 2 * cols], desc))


def test_one_row_per_slot_and_no_start():
    desc = svl.Kv4Desc(6, 2, 128, 40)
    x = rows_of(2, 6, 512)
    xd = x.cuda()
    cache = new_cache(desc)
    write(desc, cache, xd[:, :256], xd[:, 256:], [1] * 6, [0, 5, 31, 32, 39, 16], row_off=None)
    k, v = read(desc, cache, [1] * 6, [0, 5, 31, 32, 39, 16], row_off=None)
    same(k, expected(x[:, :256], desc))
    same(v, expected(x[:, 256:], desc))
    write(desc, cache, xd[:, 256:], xd[:, :256], [1] * 6, None, row_off=None)
    k, v = read(desc, cache, [1] * 6, None, row_off=None)
    same(k, expected(x[:, 256:], desc))
    same(v, expected(x[:, :256], desc))


@pytest.mark.parametrize("dh", [64, 128])
def test_rows_written_one_by_one_equal_rows_written_at_once(dh):
    """Neighbouring positions share words of the V codes: the later write leaves the earlier one's as they were."""
    desc = svl.Kv4Desc(2, 3, dh, 96)
    n, cols = 70, 3 * dh
    x = rows_of(3, 2 * n, 2 * cols)
    xd = x.cuda()
    a, b = new_cache(desc, 0), new_cache(desc, 0)
    write(desc, a, xd[:, :cols], xd[:, cols:], [n, n], [5, 0])
    for i in list(range(1, n, 2)) + list(range(0, n, 2)):
        pair = xd[[i, n + i]]
        write(desc, b, pair[:, :cols], pair[:, cols:], [1, 1], [5 + i, i], row_off=None)
    assert torch.equal(a, b)
    c = new_cache(desc, 0)
    cut = 37
    parts = torch.cat((xd[:cut], xd[n:n + 11])), torch.cat((xd[cut:n], xd[n + 11:]))
    for p, counts, starts in zip(parts, ([cut, 11], [n - cut, n - 11]), ([5, 0], [5 + cut, 11])):
        write(desc, c, p[:, :cols], p[:, cols:], counts, starts)
    assert torch.equal(a, c)


def test_groups_of_every_kind():
    """Zeros, one value, both signs alike, ties between codes, tiny, huge and non-finite values."""
    desc = svl.Kv4Desc(1, 1, 128, 64)
    rows = torch.zeros(40, 128)
    rows[1] = 3.0
    rows[2] = -3.0
    rows[3, ::2], rows[3, 1::2] = 5.0, -5.0                              # +e and -e: e is the positive one
    rows[4] = torch.arange(128) % 33 - 16.0                              # x / s = k + 1/2 for the odd ones
    rows[5] = (torch.arange(128) % 17 - 8.0) / 2
    rows[6, 7], rows[6, 40] = 1e-38, -1e-40                              # held as zeros
    rows[7] = 3e38
    rows[8] = torch.linspace(-3e38, 3e38, 128)
    rows[9] = torch.linspace(-1e-36, 1e-36, 128)
    rows[10, 3], rows[10, 100] = float("inf"), -float("inf")
    rows[11, 64] = float("nan")
    rows[12, 0] = 2.0 ** -123
    rows[13, 0], rows[13, 1] = 2.0 ** -120, -2.0 ** -130
    g = torch.Generator().manual_seed(4)
    for i in range(14, 40):                                             # small integers: many exact ties
        rows[i] = torch.randint(-255, 256, (128,), generator=g).float() * 2.0 ** (i - 20)
    x = rows.to(BF16)
    xd = x.cuda()
    cache = new_cache(desc)
    write(desc, cache, xd, xd, [40], [3])
    k, v = read(desc, cache, [40], [3])
    same(k, expected(x, desc))
    same(v, expected(x, desc))


def test_rows_without_a_place_are_not_stored():
    desc = svl.Kv4Desc(3, 2, 64, 50)  # not whole tiles
    x = rows_of(5, 12, 256).cuda()
    cache, before = new_cache(desc, 3), new_cache(desc, 3)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    write(desc, cache, x[:, :128], x[:, 128:], [4, 4, 4], [-2, -9, 10], status)
    assert int(status) == 0  # idle slots are no fault
    k, v = read(desc, cache, [4, 4, 4], [-2, -9, 10])
    want = expected(x[:, :128].cpu(), desc)
    want[:2] = 0
    want[4:8] = 0
    same(k, want)
    write(desc, cache, x[:, :128], x[:, 128:], [4, 4, 4], [48, 50, 2 ** 31 - 2], status)
    assert int(status) == svl.SVL_DEV_BAD_INDEX
    k, v = read(desc, cache, [4, 4, 4], [48, 50, 2 ** 31 - 2])
    want = expected(x[:, 128:].cpu(), desc)
    want[2:] = 0
    same(v, want)
    # nothing but the rows that have a place changed
    cache2 = new_cache(desc, 3)
    write(desc, cache2, x[:2, :128], x[:2, 128:], [0, 2, 0], [0, 0, 0])  # reach slot 1 alone
    rest = torch.cat((cache2[:len(before) // 3], cache2[2 * len(before) // 3:]))
    assert bool((rest == 3).all())
    # rows past row_off's end are left alone, on both ways
    off = i32([0, 1, 1, 2])
    k2 = torch.full((12, 128), 9.0, dtype=BF16, device="cuda")
    svl.svl_kv4_read(desc, cache, 12, off, i32([0, 0, 10]), k2, 128, k2.clone(), 128)
    assert bool((k2[2:] == 9).all())


def test_a_cache_past_32_bits_of_bytes():
    """One slot of 4.8 GB: its last positions, written, read and attended to."""
    desc = svl.Kv4Desc(1, 32, 128, 1_040_000)
    cache = torch.empty(svl.svl_kv4_cache_size(desc), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 2 ** 32
    n, at = 70, 1_039_900
    x = rows_of(6, n, 2 * 4096)
    xd = x.cuda()
    write(desc, cache, xd[:, :4096], xd[:, 4096:], [n], [at])
    write(desc, cache, xd[:9, :4096], xd[:9, 4096:], [9], [0])
    k, v = read(desc, cache, [n], [at])
    same(k, expected(x[:, :4096], desc))
    same(v, expected(x[:, 4096:], desc))
    q = rows_of(7, 1, 4096)
    kk, vv = ({0: R.quantised(t.view(n, 32, 128))} for t in (x[:, :4096], x[:, 4096:]))
    _check_attention(desc, cache, q, [at + n - 1], 1, 32, 50, 5,
                     lambda b, j: (kk[0][np.where(j < 9, j, j - at)], vv[0][np.where(j < 9, j, j - at)]))


# ------------------------------------------------------------------ attention
def _attend(desc, cache, q, starts, rows, heads, window, sinks, scale, stream=None, fill=7.0):
    ws = torch.empty(svl.svl_kv4_attention_workspace_size(desc, heads, rows), dtype=torch.uint8, device="cuda")
    qd = q.cuda()
    out = torch.full((q.shape[0], heads * desc.d_head + 16), fill, dtype=BF16, device="cuda")
    svl.svl_kv4_attention(desc, cache, heads, rows, qd, qd.stride(0), i32(starts), window, sinks, scale, out,
                          out.stride(0), ws, ws.numel(), stream)
    torch.cuda.synchronize()
    assert bool((out[:, heads * desc.d_head:] == fill).all())
    return out[:, :heads * desc.d_head].cpu().double().numpy()


def _check_attention(desc, cache, q, starts, rows, heads, window, sinks, look, scale=None):
    dh, grp = desc.d_head, heads // desc.n_kv_heads
    scale = scale or dh ** -0.5
    got = _attend(desc, cache, q, starts, rows, heads, window, sinks, scale).reshape(-1, heads, dh)
    qq = q.double().numpy()[:, :heads * dh].reshape(-1, heads, dh)
    for b, start in enumerate(starts):
        for r in range(rows):
            j = R.visible(start + r, desc.max_len, window, sinks)
            k, v = look(b, j) if len(j) else (np.zeros((0, desc.n_kv_heads, dh)),) * 2
            for h in range(heads):
                ref, spread, size = R.attention(qq[b * rows + r, h], k[:, h // grp], v[:, h // grp], np.float32(scale))
                err = np.abs(got[b * rows + r, h] - ref)
                assert (err <= R.attention_bound(ref, spread, size)).all(), (b, r, h, err.max())


def _filled(seed, desc, counts):
    """A cache whose slots hold rows 0 .. counts[b] - 1, NaN scales elsewhere, and how to look its rows up."""
    n, cols = sum(counts), desc.n_kv_heads * desc.d_head
    x = rows_of(seed, n, 2 * cols)
    xd = x.cuda()
    cache = new_cache(desc)
    write(desc, cache, xd[:, :cols], xd[:, cols:], counts, None)
    off = offsets(counts)
    kk, vv = (R.quantised(t.view(n, desc.n_kv_heads, desc.d_head)) for t in (x[:, :cols], x[:, cols:]))
    return cache, lambda b, j: (kk[off[b] + j], vv[off[b] + j])


@pytest.mark.parametrize("heads,kv,dh,rows,starts,window,sinks", [
    (1, 1, 64, 1, [0], 0, 0),                                        # one position
    (4, 4, 64, 1, [0, 1, 30, 31, 32, 33, 63, 64], 0, 0),             # tile edges
    (32, 32, 128, 1, [250, 5, 449], 0, 0),
    (28, 4, 128, 1, [1900], 0, 0),
    (28, 4, 128, 3, [100, -3, -1, -2, 333], 0, 0),                   # idle slots, rows that see nothing
    (12, 1, 64, 1, [700, 20], 0, 0),                                 # twelve heads share the KV head
    (40, 8, 128, 2, [64, 95], 0, 0),
    (4, 4, 128, 16, [0, 50, 500], 0, 0),                             # sixteen rows
    (12, 1, 128, 5, [40], 0, 0),                                     # sixty columns
    (8, 2, 128, 1, [600, 31, 0], 1, 0),                              # a window of the row itself
    (8, 2, 128, 1, [600, 31, 0], 1, 1),
    (8, 8, 64, 1, [999, 64, 3], 64, 4),
    (8, 8, 64, 4, [999, 64, 3], 33, 37),                             # sinks past a tile, window across tiles
    (28, 4, 128, 3, [2000, 700, 63], 1024, 4),
    (4, 2, 64, 2, [300, 10], 5000, 3),                               # a window that holds everything
    (4, 2, 64, 2, [300, 10], 40, 5000),                              # sinks that hold everything
    (7, 7, 128, 1, [5000, 100, 2], 0, 0),
])
def test_attention(heads, kv, dh, rows, starts, window, sinks):
    desc = svl.Kv4Desc(len(starts), kv, dh, max(starts) + rows + 3)
    cache, look = _filled(11, desc, [max(0, s + rows) for s in starts])
    q = rows_of(12, len(starts) * rows, heads * dh + 8)
    _check_attention(desc, cache, q, starts, rows, heads, window, sinks, look)


def test_attention_scores_far_apart_and_all_alike():
    """Large scores (one weight near 1), the same key everywhere (weights alike), a scale of zero, a negative one."""
    desc = svl.Kv4Desc(2, 2, 128, 400)
    cache, look = _filled(13, desc, [390, 77])
    q = rows_of(14, 2, 4 * 128)
    for scale in (3.0, 1e-30, -0.2):
        _check_attention(desc, cache, q, [389, 76], 1, 4, 0, 0, look, scale)
    x = rows_of(15, 1, 2 * 256).repeat(390, 1)
    v = rows_of(16, 390, 256)
    c2 = new_cache(desc)
    write(desc, c2, x[:, :256].contiguous().cuda(), v.cuda(), [390, 0], None)
    kk, vv = R.quantised(x[:, :256].view(390, 2, 128)), R.quantised(v.view(390, 2, 128))
    _check_attention(desc, c2, q, [389, -1], 1, 4, 0, 0, lambda b, j: (kk[j], vv[j]))


@pytest.mark.parametrize("power", [-100, -30, 30, 100])
def test_attention_values_of_any_size(power):
    """V (and K against a scale that undoes it) near both ends of bf16's range."""
    desc = svl.Kv4Desc(1, 2, 64, 100)
    x = rows_of(17, 90, 256).float()
    k, v = (x[:, :128] * 2.0 ** (power // 2)).to(BF16), (x[:, 128:] * 2.0 ** power).to(BF16)
    v[40:50] = (v[40:50].float() * 2.0 ** -20).to(BF16)
    cache = new_cache(desc)
    write(desc, cache, k.cuda(), v.cuda(), [90], None)
    kk, vv = R.quantised(k.view(90, 2, 64)), R.quantised(v.view(90, 2, 64))
    _check_attention(desc, cache, rows_of(18, 1, 256), [89], 1, 4, 0, 0, lambda b, j: (kk[j], vv[j]),
                     0.125 * 2.0 ** -(power // 2))


def test_attention_small_weights_add_up():
    """One row takes nearly all the weight and its value is zero: the output is what thousands of small weights add."""
    n = 8000
    desc = svl.Kv4Desc(1, 1, 128, n)
    g = torch.Generator().manual_seed(19)
    k = torch.zeros(n, 128)
    k[:, 0] = torch.randn(n, generator=g) * 0.01
    k[0, 0] = 1.0
    v = torch.randn(n, 128, generator=g)
    v[0] = 0
    k, v = k.to(BF16), v.to(BF16)
    cache = new_cache(desc)
    write(desc, cache, k.cuda(), v.cuda(), [n], None)
    kk, vv = R.quantised(k.view(n, 1, 128)), R.quantised(v.view(n, 1, 128))
    q = torch.zeros(1, 128)
    q[0, 0] = 16.0
    _check_attention(desc, cache, q.to(BF16), [n - 1], 1, 1, 0, 0, lambda b, j: (kk[j], vv[j]), 1.0)


def test_what_is_not_visible_does_not_count():
    """NaNs and infinities at positions outside the window, behind the row and in idle slots; NaNs in sight do show:
    of K in the whole row, of V in its group's dimensions."""
    desc = svl.Kv4Desc(2, 2, 64, 300)
    n, cols = 290, 128
    x = rows_of(20, 2 * n, 2 * cols)
    bad = x.clone()
    bad[4:150, ::3] = float("nan")          # slot 0: between the sinks and every row's window
    bad[201:n, 5::7] = float("inf")         # behind its last row
    bad[n:] = float("nan")                  # slot 1 is idle
    xd = bad.cuda()
    cache = new_cache(desc)
    write(desc, cache, xd[:, :cols], xd[:, cols:], [n, n], None)
    kk, vv = (R.quantised(t.view(2 * n, 2, 64)) for t in (x[:, :cols], x[:, cols:]))
    q = rows_of(21, 4, 4 * 64)
    _check_attention(desc, cache, q, [199, -2], 2, 4, 49, 4, lambda b, j: (kk[j], vv[j]))
    # row 0 sees position 199, row 1 position 200 as well: its V has a NaN in the second group of head 1
    one = x[200:201].clone()
    one[0, cols + 64 + 40] = float("nan")
    od = one.cuda()
    write(desc, cache, od[:, :cols], od[:, cols:], [1, 0], [200, 0])
    got = _attend(desc, cache, q, [199, -2], 2, 4, 49, 4, 0.125).reshape(4, 4, 64)
    nan = np.isnan(got)
    want = np.zeros_like(nan)
    want[1, 2:, 32:] = True
    np.testing.assert_array_equal(nan, want)
    one[0, 3] = float("inf")  # and its K one in head 0
    write(desc, cache, one.cuda()[:, :cols], one.cuda()[:, cols:], [1, 0], [200, 0])
    got = _attend(desc, cache, q, [199, -2], 2, 4, 49, 4, 0.125).reshape(4, 4, 64)
    want[1, :2] = True
    np.testing.assert_array_equal(np.isnan(got), want)


def test_rows_past_the_cache_give_zeros():
    desc = svl.Kv4Desc(2, 2, 64, 40)
    cache, look = _filled(22, desc, [40, 40])
    _check_attention(desc, cache, rows_of(23, 6, 256), [38, 2 ** 31 - 2], 3, 4, 0, 0, look)


def test_many_slots_and_another_stream():
    """More slots than the GPU has SMs, ragged, on a stream of their own with nothing waited for in between."""
    slots = 400
    rng = np.random.default_rng(24)
    starts = rng.integers(-1, 120, slots).tolist()
    desc = svl.Kv4Desc(slots, 2, 64, 130)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        cache, look = _filled(25, desc, [p + 1 for p in starts])
        _check_attention(desc, cache, rows_of(26, slots, 256), starts, 1, 4, 0, 0, look)


def test_results_do_not_change_from_call_to_call():
    desc = svl.Kv4Desc(3, 4, 128, 5000)
    cache, _ = _filled(27, desc, [5000, 77, 2500])
    q = rows_of(28, 3, 28 * 128)
    first = _attend(desc, cache, q, [4999, 76, 2499], 1, 28, 0, 0, 0.088)
    for _ in range(5):
        np.testing.assert_array_equal(first, _attend(desc, cache, q, [4999, 76, 2499], 1, 28, 0, 0, 0.088))


def test_graph_capture():
    """A decode step's calls in a CUDA graph, replayed at growing positions."""
    desc = svl.Kv4Desc(2, 2, 64, 64)
    x = rows_of(29, 2, 512).cuda()
    cache = new_cache(desc)
    start = i32([0, 0])
    out = torch.empty(2, 256, dtype=BF16, device="cuda")
    ws = torch.empty(svl.svl_kv4_attention_workspace_size(desc, 4, 1), dtype=torch.uint8, device="cuda")

    def step():
        svl.svl_kv4_write(desc, cache, x[:, :128], 512, x[:, 128:], 512, 2, None, start, None)
        svl.svl_kv4_attention(desc, cache, 4, 1, x[:, 256:], 512, start, 0, 0, 0.125, out, 256, ws, ws.numel())
        start.add_(1)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(20):
        g.replay()
    torch.cuda.synchronize()
    assert start.tolist() == [21, 21]
    # every position holds the same row: the output is that row's V
    want = expected(x[:, 128:256].cpu().contiguous(), desc).float().view(2, 2, 1, 64).expand(2, 2, 2, 64).reshape(2, 256)
    np.testing.assert_allclose(out.cpu().float().numpy(), want.numpy(), rtol=2.0 ** -7, atol=1e-6)


# ------------------------------------------------------------------ reorder
@pytest.mark.parametrize("beams,layers,parents,first,lens", [
    (1, 1, [[0], [0]], None, [10, 10]),
    (2, 1, [[1, 0]], None, [40, 70]),                                     # a swap, beams of different length
    (4, 3, [[1, 2, 3, 0], [0, 0, 0, 0], [3, 3, 1, 1]], [0, 33, 64], [96] * 12),
    (5, 2, [[4, 3, 2, 1, 0], [2, 2, 2, 0, 1]], [31, 32], [100, 1, 64, 65, 32] * 2),
    (16, 2, [[15 - i for i in range(16)]], [10], [80] * 16),
    (3, 2, [[0, 1, 2]], None, [96] * 3),                                  # nothing moves
    (3, 1, [[1, 1, 1]], None, [0, 0, 0]),                                 # nothing is held
])
@pytest.mark.parametrize("dh", [64, 128])
def test_reorder(beams, layers, parents, first, lens, dh):
    samples, kv, tiles = len(parents), 3, 4
    desc = svl.Kv4Desc(samples * beams, kv, dh, 100)
    g = torch.Generator().manual_seed(31)
    size = svl.svl_kv4_cache_size(desc)
    old = torch.randint(0, 256, (layers * size,), generator=g, dtype=torch.uint8)
    cache = old.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    svl.svl_kv4_reorder(desc, cache, layers, beams, i32(parents), None if first is None else i32(first), i32(lens), status)
    want = old.clone().view(layers, samples * beams, kv, tiles, 36 * dh)
    src = old.view_as(want)
    for s in range(samples):
        for w in range(beams):
            p = s * beams + parents[s][w]
            lo, hi = (first[s] if first else 0) // 32, -(-lens[p] // 32)
            want[:, s * beams + w, :, lo:hi] = src[:, p, :, lo:hi]
    assert int(status) == 0
    assert torch.equal(cache.cpu().view_as(want), want)


def test_reorder_reports_a_parent_out_of_range():
    desc = svl.Kv4Desc(4, 1, 64, 32)
    old = torch.randint(0, 256, (svl.svl_kv4_cache_size(desc),), dtype=torch.uint8).cuda()
    cache = old.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    svl.svl_kv4_reorder(desc, cache, 1, 4, i32([1, 4, -1, 0]), None, i32([32] * 4), status)
    assert int(status) == svl.SVL_DEV_BAD_INDEX
    o, c = old.view(4, -1), cache.view(4, -1)
    assert torch.equal(c, o[[1, 1, 2, 0]])
