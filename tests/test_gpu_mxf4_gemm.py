"""Products of MXFP4 matrices against 64-bit sums of what the operands hold, and a gated MLP in 4 bits."""
import numpy as np
import pytest
import torch

from paper_2607_20357_gb300 import svl
from tests import mxf4_reference as R

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


def operand(seed, rows, cols, ld=None, low=125, high=129):
    """Random codes and scales on the GPU (bytes low..high - 1; rows that do not exist have NaN scales) and their values."""
    g = np.random.default_rng(seed)
    blocks = -(-cols // 32)
    code = g.integers(0, 16, (rows, blocks * 32)).astype(np.uint8)
    code[:, cols:] = 0
    byte = g.integers(low, high, (rows, blocks)).astype(np.uint8)
    held = np.full((rows, ld or R.held_bytes(cols)), 0x77, np.uint8)
    held[:, :blocks * 16] = R.packed(code)
    scales = R.laid_out(byte, cols, 0xFF)
    return torch.from_numpy(held).cuda(), torch.from_numpy(scales).cuda(), R.values(code, byte)[:, :cols]


def product(a, sa, b, sb, m, n, k, kept, ld_c=None, **kw):
    ld_c = ld_c or n
    out = torch.full((m, ld_c), 7.0, dtype=kept, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    svl.svl_gemm_mxf4(a, a.shape[1], sa, b, b.shape[1], sb, m, n, k, out, ld_c,
                      svl.SVL_OUT_F32 if kept == F32 else svl.SVL_OUT_BF16, status=status, **kw)
    assert status.item() == 0
    return out


def whole(m, n, factor, residual, kept):
    """A power of two per row and small whole numbers to add: with the codes' values every sum is exact in 32 bits."""
    g = torch.Generator().manual_seed(m + n)
    f = torch.ldexp(torch.ones(m), torch.randint(-2, 3, (m,), generator=g)) if factor else None
    r = torch.randint(-64, 65, (m, n), generator=g).to(kept) if residual else None
    return f, r


# (M, N, K, bytes between rows of A and of B (None: dense), ld_c)
SHAPES = [
    (1, 1, 32, None, None, None), (5, 9, 1, None, None, None), (130, 40, 7, None, None, None), (1, 8, 8, None, None, None),
    (3, 5, 40, 48, 64, 9), (1, 128, 64, None, None, None),
    (2, 129, 96, None, 80, 130), (16, 128, 128, None, None, None), (17, 200, 160, None, None, 203),
    (1, 4096, 4096, None, None, None), (5, 300, 1000, 512, 528, None), (31, 1000, 256, None, None, None),
    (33, 127, 288, None, None, 128), (48, 260, 512, 272, None, None), (64, 4096, 2048, None, None, None),
    (65, 130, 544, None, None, None), (96, 384, 768, None, None, None), (127, 512, 1024, None, None, 520),
    (128, 128, 1088, None, None, None), (129, 640, 480, None, 256, 644), (200, 256, 11008, None, None, None),
    (255, 383, 320, None, None, None), (256, 1024, 2080, None, None, None), (257, 129, 640, 336, None, 136),
    (300, 3584, 1024, None, None, None), (384, 896, 2400, None, None, None), (513, 2050, 264, None, None, 2051),
    (700, 5000, 1152, None, None, None), (1025, 4224, 512, None, None, None), (2000, 7, 4096, None, None, None),
    (2600, 4096, 1312, None, None, None), (8, 32000, 4096, None, None, None), (1, 3584, 18944, None, None, None),
    (40, 77, 18944, None, None, 80), (24, 300, 2000, None, None, None), (50, 640, 12288, None, None, 645),
    (100, 640, 6000, None, None, None), (128, 300, 18944, None, None, None), (70, 20000, 320, None, None, None),
    (16, 20000, 512, None, None, None), (130, 700, 4128, None, None, 703), (300, 3584, 4352, None, None, None),
    (520, 1300, 8192, None, None, None), (129, 20000, 96, None, None, None), (200, 39000, 288, None, None, None),
    (250, 25000, 416, None, None, 25001), (300, 20100, 1040, None, None, 20104), (330, 21000, 128, None, None, None),
    (384, 700, 8192, None, None, None), (290, 1100, 12288, None, None, None), (160, 1000, 18944, None, None, 1001), (1100, 129, 640, None, None, 136), (1100, 2052, 256, None, None, 2056),
]


@pytest.mark.parametrize("m,n,k,ld_a,ld_b,ld_c", SHAPES)
@pytest.mark.parametrize("kept,factor,residual", [(F32, False, False), (F32, True, True), (BF16, False, True),
                                                  (BF16, True, False), (BF16, True, True)])
def test_exact_sums(m, n, k, ld_a, ld_b, ld_c, kept, factor, residual):
    """Sums of multiples of 2^-5 under 2^18 leave nothing to round before the result's own type."""
    a, sa, va = operand(m + k, m, k, ld_a, 125, 128)
    b, sb, vb = operand(n + k + 1, n, k, ld_b, 126, 129)
    f, r = whole(m, n, factor, residual, kept)
    assert np.sqrt((va ** 2).sum(1).max() * (vb ** 2).sum(1).max()) < 2 ** 18  # bounds any sum of magnitudes
    ld_r = n + 3 if ld_c else n
    rr = None
    if residual:
        rr = torch.full((m, ld_r), float("nan"), dtype=kept)
        rr[:, :n] = r
        rr = rr.cuda()
    out = product(a, sa, b, sb, m, n, k, kept, ld_c, row_factor=None if f is None else f.cuda(), residual=rr,
                  ld_residual=ld_r if residual else 0)
    want = torch.from_numpy(va).cuda() @ torch.from_numpy(vb).cuda().t()
    if factor:
        want = want * f.double().cuda()[:, None]
    if residual:
        want = want + r.double().cuda()
    assert (out[:, n:] == 7).all()
    # (exact in 32 bits, so its rounding to bf16 is the only one)
    assert torch.equal(out[:, :n], want.float().to(kept))


@pytest.mark.parametrize("m,n,k", [(1, 300, 4096), (40, 513, 2176), (300, 700, 8192), (600, 1300, 1024)])
@pytest.mark.parametrize("kept", [F32, BF16])
def test_scales_far_apart(m, n, k, kept):
    """Scales from 2^-20 to 2^20. Each of the K additions is off by at most 2^-23 (a truncation) of the sum of
    magnitudes, whatever their order; then the factor, the residual and the result round by half a step each."""
    a, sa, va = operand(m, m, k, None, 107, 148)
    b, sb, vb = operand(n, n, k, None, 107, 148)
    g = torch.Generator().manual_seed(k)
    f, r = torch.rand(m, generator=g) + 0.5, torch.randn(m, n, generator=g).to(kept)
    out = product(a, sa, b, sb, m, n, k, kept, row_factor=f.cuda(), residual=r.cuda(), ld_residual=n).double().cpu()
    va, vb = torch.from_numpy(va), torch.from_numpy(vb)
    p, mag = (va @ vb.t()) * f.double()[:, None], (va.abs() @ vb.abs().t()) * f.double()[:, None]
    want = p + r.double()
    tol = mag * (k + 2) * 2.0 ** -23 + (want.abs() + mag * k * 2.0 ** -23) * torch.finfo(kept).eps / 2 + r.double().abs() * 2.0 ** -24
    assert ((out - want).abs() <= tol).all()


@pytest.mark.parametrize("m,n,k", [(3, 200, 512), (150, 200, 4096), (520, 900, 512)])
def test_nan_blocks_stay_in_their_row_and_column(m, n, k):
    a, sa, va = operand(1, m, k, None, 126, 128)
    b, sb, vb = operand(2, n, k, None, 126, 128)
    i, j = m - 1, n // 2
    sa[R.scale_at(m, k)[i, k // 32 - 1]] = 255
    sb[R.scale_at(n, k)[j, 0]] = 255
    out = product(a, sa, b, sb, m, n, k, F32).cpu()
    want = torch.from_numpy(va @ vb.T).float()
    want[i], want[:, j] = float("nan"), float("nan")
    assert torch.equal(out.isnan(), want.isnan())
    assert torch.equal(out.nan_to_num(), want.nan_to_num())


def test_results_that_overflow():
    """Sums past float32 become infinities, of their own sign."""
    m, n, k = 2, 130, 64
    a = torch.full((m, 32), 0x77, dtype=U8, device="cuda")       # 6 everywhere
    a[1] = 0xFF                                                  # -6
    b = torch.full((n, 32), 0x77, dtype=U8, device="cuda")
    s = [torch.full((svl.svl_mxf4_scale_size(r, k),), 254, dtype=U8, device="cuda") for r in (m, n)]
    out = product(a, s[0], b, s[1], m, n, k, F32)
    assert (out[0] == float("inf")).all() and (out[1] == -float("inf")).all()


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (100, 640, 512), (600, 1000, 1024)])
@pytest.mark.parametrize("kept", [F32, BF16])
def test_residual_in_place(m, n, k, kept):
    a, sa, va = operand(5, m, k, None, 125, 128)
    b, sb, vb = operand(6, n, k, None, 126, 129)
    _, r = whole(m, n, False, True, kept)
    c = r.cuda()
    svl.svl_gemm_mxf4(a, k // 2, sa, b, k // 2, sb, m, n, k, c, n, svl.SVL_OUT_F32 if kept == F32 else svl.SVL_OUT_BF16,
                      residual=c, ld_residual=n)
    assert torch.equal(c.cpu(), (torch.from_numpy(va @ vb.T) + r.double()).float().to(kept))


@pytest.mark.parametrize("m,n,k", [(1, 4096, 8192), (300, 3584, 4096), (2500, 2304, 1024)])
def test_same_bits_again(m, n, k):
    """Scales far apart make sums depend on their order; the order does not change, nor with what runs beside it."""
    a, sa, _ = operand(1, m, k, None, 107, 148)
    b, sb, _ = operand(2, n, k, None, 107, 148)
    first = product(a, sa, b, sb, m, n, k, F32)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    outs = [torch.empty(m, n, device="cuda") for _ in range(12)]
    for i, o in enumerate(outs):
        svl.svl_gemm_mxf4(a, a.shape[1], sa, b, b.shape[1], sb, m, n, k, o, n, svl.SVL_OUT_F32,
                          stream=streams[i % 3].cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)


class Layer:
    """A gated MLP with its weights in 4 bits and every buffer of a forward."""

    def __init__(self, rows, width, inner):
        g = torch.Generator(device="cuda").manual_seed(rows + width)
        self.rows, self.width, self.inner = rows, width, inner
        self.x = torch.randn(rows, width, device="cuda", generator=g).to(BF16)
        self.gain = (1 + 0.2 * torch.randn(width, device="cuda", generator=g)).to(BF16)
        self.gate_up = self.held(torch.randn(2 * inner, width, device="cuda", generator=g).to(BF16) * 0.03)
        self.down = self.held(torch.randn(width, inner, device="cuda", generator=g).to(BF16) * 0.03)
        self.a, self.h = self.room(rows, width), self.room(rows, inner)
        self.inv_rms = torch.empty(rows, device="cuda")
        self.both = torch.empty(rows, 2 * inner, dtype=BF16, device="cuda")
        self.out = torch.empty(rows, width, dtype=BF16, device="cuda")

    @staticmethod
    def room(rows, cols):
        return (torch.zeros(rows, R.held_bytes(cols), dtype=U8, device="cuda"),
                torch.zeros(svl.svl_mxf4_scale_size(rows, cols), dtype=U8, device="cuda"))

    def held(self, w):
        c, s = self.room(*w.shape)
        svl.svl_quantize_rows_mxf4(w.contiguous(), w.shape[0], w.shape[1], w.shape[1], c, c.shape[1], s)
        return c, s

    def forward(self):
        (a, sa), (h, sh), (w1, s1), (w2, s2) = self.a, self.h, self.gate_up, self.down
        rows, width, inner = self.rows, self.width, self.inner
        svl.svl_quantize_rows_mxf4(self.x, rows, width, width, a, a.shape[1], sa, gain=self.gain, eps=1e-5,
                                   inv_rms=self.inv_rms)
        svl.svl_gemm_mxf4(a, a.shape[1], sa, w1, w1.shape[1], s1, rows, 2 * inner, width, self.both, 2 * inner,
                          svl.SVL_OUT_BF16, row_factor=self.inv_rms)
        svl.svl_swiglu_rows_mxf4(self.both, 2 * inner, self.both[:, inner:], 2 * inner, rows, inner, h, h.shape[1], sh)
        svl.svl_gemm_mxf4(h, h.shape[1], sh, w2, w2.shape[1], s2, rows, width, inner, self.out, width, svl.SVL_OUT_BF16,
                          residual=self.x, ld_residual=width)

    @staticmethod
    def values(held, rows, cols):
        c, s = held[0].cpu().numpy(), held[1].cpu().numpy()
        code = np.stack((c & 15, c >> 4), -1).reshape(rows, -1)
        return R.values(code, s[R.scale_at(rows, cols)])[:, :cols]

    def check(self):
        """Each step from what the one before it left."""
        x, gain = self.x.cpu().double().numpy(), self.gain.cpu().double().numpy()
        rows, width, inner = self.rows, self.width, self.inner
        code, byte = R.quantised(x * gain)
        a = self.values(self.a, rows, width)
        np.testing.assert_array_equal(a, R.values(code, byte)[:, :width])
        inv = 1 / np.sqrt((x ** 2).mean(1) + 1e-5)
        assert (np.abs(self.inv_rms.cpu().double().numpy() / inv - 1) <= 32 * 2.0 ** -24).all()
        f = self.inv_rms.cpu().double().numpy()[:, None]
        w1, w2 = self.values(self.gate_up, 2 * inner, width), self.values(self.down, width, inner)
        both = self.both.cpu().double().numpy()
        mag = np.abs(a) @ np.abs(w1).T * f
        err = mag * (width + 1) * 2.0 ** -23
        assert (np.abs(both - a @ w1.T * f) <= err + (np.abs(both) + err) * 2.0 ** -8).all()
        gate, up = both[:, :inner], both[:, inner:]
        want = gate / (1 + np.exp(-gate)) * up
        h = self.values(self.h, rows, inner)
        top = np.repeat(np.abs(R.blocks(want)).max(-1), 32, 1)[:, :inner]
        # a code is off by half a step, at most 1 of the 3 to 6 that the largest magnitude has
        assert (np.abs(h - want) <= top / 3 * (1 + 2.0 ** -20) + 2.0 ** -128).all()
        mag, out = np.abs(h) @ np.abs(w2).T, self.out.cpu().double().numpy()
        err = mag * (inner + 1) * 2.0 ** -23
        assert (np.abs(out - (h @ w2.T + x)) <= err + (np.abs(out) + err) * 2.0 ** -8 + np.abs(x) * 2.0 ** -23).all()


@pytest.mark.parametrize("rows,width,inner", [(1, 256, 512), (7, 512, 1376), (150, 264, 680), (300, 1024, 2752)])
def test_gated_mlp(rows, width, inner):
    layer = Layer(rows, width, inner)
    layer.forward()
    layer.check()


def test_gated_mlp_in_a_graph():
    """Captured once, replayed with other rows."""
    layer = Layer(20, 512, 1376)
    layer.forward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward()
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        layer.x.copy_(torch.randn(20, 512, device="cuda", generator=g).to(BF16) * 3)
        graph.replay()
        torch.cuda.synchronize()
        layer.check()
