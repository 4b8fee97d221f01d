"""MXFP4 rows: quantising them (with a gain, 1/rms, as the result of SwiGLU) and reading them back, against plain 64-bit
definitions."""
import numpy as np
import pytest
import torch

from paper_2607_20357_gb300 import svl
from tests import mxf4_reference as R

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

BF16, U8 = torch.bfloat16, torch.uint8

# (rows, cols, elements between source rows, bytes between code rows)
SHAPES = [(1, 8, 8, 16), (1, 32, 32, 16), (3, 40, 48, 48), (1, 4096, 4096, 2048), (2, 1000, 1000, 512),
          (31, 128, 128, 64), (33, 136, 144, 96), (129, 264, 520, 160), (130, 4096, 4096, 2048), (257, 72, 72, 48),
          (5, 18944, 18944, 9472), (700, 1024, 1032, 528), (2049, 64, 64, 32),
          (25001, 256, 256, 128), (70001, 40, 40, 32), (19500, 264, 264, 144)]


def rows_of(seed, rows, cols, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(cols, generator=g))
    return x.to(BF16)


def strided(x, ld, fill=float("nan")):
    """The rows of x on the GPU, `ld` elements apart, NaNs between them."""
    out = torch.full((x.shape[0], ld), fill, dtype=x.dtype)
    out[:, :x.shape[1]] = x
    return out.cuda()


class Held:
    """Codes and scales full of a byte, and what they hold after a call."""

    def __init__(self, rows, cols, ld, fill=0xEE):
        self.rows, self.cols, self.ld, self.fill = rows, cols, ld, fill
        self.codes = torch.full((rows, ld), fill, dtype=U8, device="cuda")
        self.scales = torch.full((svl.svl_mxf4_scale_size(rows, cols),), fill, dtype=U8, device="cuda")

    def check(self, code, byte):
        """Everything in memory, what the call must leave alone with it."""
        want = np.full((self.rows, self.ld), self.fill, np.uint8)
        want[:, :R.held_bytes(self.cols)] = R.packed(code)
        np.testing.assert_array_equal(self.codes.cpu().numpy(), want)
        np.testing.assert_array_equal(self.scales.cpu().numpy(), R.laid_out(byte, self.cols, self.fill))


def quantise(x, ld=None, ld_codes=None, gain=None, eps=0.0, inv_rms=None):
    rows, cols = x.shape
    ld = ld or cols
    h = Held(rows, cols, ld_codes or R.held_bytes(cols))
    svl.svl_quantize_rows_mxf4(strided(x, ld), rows, cols, ld, h.codes, h.ld, h.scales, gain=gain, eps=eps,
                               inv_rms=inv_rms)
    return h


@pytest.mark.parametrize("rows,cols,ld,ld_codes", SHAPES)
@pytest.mark.parametrize("gain", [False, True])
def test_quantised_rows(rows, cols, ld, ld_codes, gain):
    x = rows_of(rows + cols, rows, cols)
    g = rows_of(7, 1, cols, 0.3)[0] if gain else None
    h = quantise(x, ld, ld_codes, None if g is None else g.cuda())
    want = x.double() * g.double() if gain else x.double()  # (two bf16 factors: exact in 32 bits too)
    h.check(*R.quantised(want.numpy()))


@pytest.mark.parametrize("rows,cols,ld,ld_codes", SHAPES)
@pytest.mark.parametrize("gain", [False, True])
def test_rows_with_their_rms(rows, cols, ld, ld_codes, gain):
    x = rows_of(rows + cols + 1, rows, cols)
    g = rows_of(8, 1, cols, 0.3)[0] if gain else None
    inv = torch.full((rows + 1,), -7.0, device="cuda")
    h = quantise(x, ld, ld_codes, None if g is None else g.cuda(), 1e-5, inv)
    h.check(*R.quantised((x.double() * g.double() if gain else x.double()).numpy()))
    got = inv.cpu().double().numpy()
    want = 1 / np.sqrt((x.double().numpy() ** 2).mean(-1) + 1e-5)
    # Each of a thread's four sums takes 4 of the 16 squares of a step of at least 512 columns (one rounding each), then
    # 2 + 5 + 8 sums join them: half their relative error after the root, and the roundings of the mean, the sum with
    # eps, the root and the quotient.
    tol = (0.5 * (4 * -(-cols // 512) + 15 + 2) + 2) * 2.0 ** -24
    assert got[rows] == -7 and (np.abs(got[:rows] / want - 1) <= tol).all()


def test_rms_of_a_row_of_zeros():
    inv = torch.empty(2, device="cuda")
    quantise(torch.zeros(2, 64, dtype=BF16), eps=0.25, inv_rms=inv)
    assert (inv == 2).all()


def special_rows():
    rows = [np.zeros(32), np.full(32, -0.0)]
    for e in (-126, -100, -3, 0, 5, 100, 120):   # every tie of the grid, and its neighbours, at several scales
        grid = np.array([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5])
        row = np.concatenate((grid, grid * (1 + 2 ** -7), grid * (1 - 2 ** -7), -grid))
        rows.append(np.minimum(np.abs(row), 6) * np.sign(row) * 2.0 ** e)
    for top in (6.0, 6.0 * (1 + 2 ** -7), 4.0, 4.0 * (1 - 2 ** -7), 3.0, 3.0 * (1 + 2 ** -7)):  # where the exponent changes
        rows.append(np.linspace(-top, top, 32))
    tiny = np.zeros(32)
    tiny[3], tiny[7] = 2.0 ** -133, -3 * 2.0 ** -133          # bf16's smallest
    rows.append(tiny)
    rows.append(np.linspace(-1, 1, 32) * 2.0 ** -126)
    rows.append(np.linspace(-1, 1, 32) * float(torch.finfo(BF16).max))
    return torch.from_numpy(np.stack(rows)).to(BF16)


def test_special_values():
    x = special_rows()
    quantise(x).check(*R.quantised(x.double().numpy()))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_blocks_that_are_not_finite(bad):
    x = rows_of(3, 4, 200)
    x[0, 0] = x[1, 31] = x[2, 100] = x[3, 199] = bad
    h = quantise(x)
    code, byte = R.quantised(x.double().numpy())
    assert (byte == 255).sum() == 4
    h.check(code, byte)
    out = torch.empty(4, 200, dtype=BF16, device="cuda")
    svl.svl_dequantize_rows_mxf4(h.codes, h.ld, h.scales, 4, 200, out, 200)
    got = out.cpu().double().numpy()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(R.values(code, byte)[:, :200]))


def test_gain_beyond_float32():
    """Products that overflow make a block NaN, ones that underflow round as float32 does."""
    x = torch.full((1, 64), 2.0 ** 100, dtype=BF16)
    g = torch.full((64,), 1.0, dtype=BF16)
    g[0], g[32:] = 2.0 ** 100, 2.0 ** -100
    h = quantise(x, gain=g.cuda())
    want = (x.float() * g.float()).double().numpy()
    h.check(*R.quantised(want))


# ------------------------------------------------------------------ reading back
@pytest.mark.parametrize("rows,cols,ld,ld_codes", SHAPES)
def test_read_back(rows, cols, ld, ld_codes):
    g = np.random.default_rng(rows * cols)
    blocks = -(-cols // 32)
    code = g.integers(0, 16, (rows, blocks * 32)).astype(np.uint8)
    byte = g.integers(0, 256, (rows, blocks)).astype(np.uint8)
    byte[0, 0] = 0
    codes = np.full((rows, ld_codes), 0xEE, np.uint8)
    codes[:, :blocks * 16] = R.packed(code)
    out = torch.full((rows, ld), 7.0, dtype=BF16, device="cuda")
    svl.svl_dequantize_rows_mxf4(torch.from_numpy(codes).cuda(), ld_codes,
                                 torch.from_numpy(R.laid_out(byte, cols, 0xFF)).cuda(), rows, cols, out, ld)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(R.values(code, byte)[:, :cols]).to(BF16)
    got = out.cpu()
    assert (got[:, cols:] == 7).all()
    np.testing.assert_array_equal(got[:, :cols].float().numpy(), want.float().numpy())


# ------------------------------------------------------------------ SwiGLU
@pytest.mark.parametrize("rows,cols,ld,ld_codes", SHAPES)
def test_swiglu(rows, cols, ld, ld_codes):
    gate, up = rows_of(rows + 11, rows, cols, 0.5) * 2, rows_of(cols + 12, rows, cols, 0.5)
    h = Held(rows, cols, ld_codes)
    both = torch.full((rows, 2 * ld), float("nan"), dtype=BF16)
    both[:, :cols], both[:, ld:ld + cols] = gate, up
    both = both.cuda()
    svl.svl_swiglu_rows_mxf4(both, 2 * ld, both[:, ld:], 2 * ld, rows, cols, h.codes, ld_codes, h.scales)
    g, u = gate.double().numpy(), up.double().numpy()
    x = R.blocks(g / (1 + np.exp(-g)) * u)
    # float32, as derived: the power of two within two ulp, what its second factor leaves out 2^-23, the reciprocal one
    # ulp, and six roundings of half an ulp (that factor, its product, the sum with one, two products, and once to spare)
    err = (2.0 ** -22 + 2.0 ** -23 + 2.0 ** -23 + 6 * 2.0 ** -24) * np.abs(x) + np.abs(R.blocks(u)) * 2.0 ** -149 + 2.0 ** -149
    codes, scales = h.codes.cpu().numpy(), h.scales.cpu().numpy()
    byte = scales[R.scale_at(rows, cols)].astype(np.int64)
    top = np.abs(x).max(-1)
    low, high = (R.scale_exponents(top * (1 + s * 2.0 ** -20)) + 127 for s in (-1, 1))
    assert ((byte >= low) & (byte <= high)).all()
    code = np.stack((codes[:, :R.held_bytes(cols)] & 15, codes[:, :R.held_bytes(cols)] >> 4), -1).reshape(x.shape)
    s = np.ldexp(1.0, byte - 127)[..., None]
    got = R.VALUES[code] * s
    a = np.abs(x) / s
    half = np.where(a <= 2, 0.25, np.where(a <= 4, 0.5, 1.0)) * s   # (at 2 and 4 the wider side is exact)
    assert (np.abs(got - x) <= half + err).all()
    assert (codes[:, R.held_bytes(cols):] == h.fill).all()
    pad = code.reshape(rows, -1)[:, cols:]
    assert (pad % 8 == 0).all()


def test_swiglu_far_out():
    """Gates whose exponential overflows give zeros, infinite ones NaN blocks."""
    gate = torch.zeros(1, 64, dtype=BF16)
    gate[0, 0], gate[0, 1], gate[0, 2], gate[0, 33] = -1e30, 1e4, -90, float("inf")
    up = torch.ones(1, 64, dtype=BF16)
    h = Held(1, 64, 32)
    svl.svl_swiglu_rows_mxf4(gate.cuda(), 64, up.cuda(), 64, 1, 64, h.codes, 32, h.scales)
    want = torch.zeros(1, 64, dtype=torch.float64)
    want[0, 1], want[0, 33] = gate[0, 1].double(), float("inf")
    code, byte = R.quantised(want.numpy())
    got = h.codes.cpu().numpy()
    got = np.stack((got & 15, got >> 4), -1).reshape(1, 64)
    np.testing.assert_array_equal(got % 8, code % 8)
    np.testing.assert_array_equal(h.scales.cpu().numpy()[R.scale_at(1, 64)], byte)
