"""Products with several tiles a CTA pair and so short a K that a tile's sums are ready before the results of the one before
have left: every result of many calls, each with operands of its own."""
import pytest
import torch

from paper_2607_20357_gb300 import svl

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8
GRID = [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]


def operand(g, rows, cols, low):
    """Random codes and scales (bytes low to low + 2) of [rows, cols], cols a multiple of 64, and their values."""
    codes = torch.randint(0, 256, (rows, cols // 2), dtype=U8, device="cuda", generator=g)
    byte = torch.randint(low, low + 3, (rows, cols // 32), dtype=U8, device="cuda", generator=g)
    rt, kt = -(-rows // 128), -(-cols // 128)
    scales = torch.zeros(rt * 128, kt * 4, dtype=U8, device="cuda")
    scales[:rows, :cols // 32] = byte
    scales = scales.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).contiguous()
    grid = torch.tensor(GRID, device="cuda")
    values = torch.stack((grid[(codes & 15).long()], grid[(codes >> 4).long()]), -1).view(rows, cols // 32, 32)
    return codes, scales, (values * torch.ldexp(torch.ones((), device="cuda"), byte.int() - 127)[..., None]).view(rows, cols)


# rows of A, rows of B: tiles of 256 (four chunks a warp in float32, two in bf16; ends of 8, 128 and 96 columns) and of 128
@pytest.mark.parametrize("m,n", [(2048, 8192), (1300, 16392), (20000, 384), (9000, 2400), (60000, 128), (60000, 64)])
@pytest.mark.parametrize("k", [64, 256])
@pytest.mark.parametrize("kept", [F32, BF16])
@pytest.mark.parametrize("factor,beside", [(False, False), (True, False), (False, True)])
def test_every_result_of_many_calls(m, n, k, kept, factor, beside):
    """Sums of multiples of 2^-5 under 72 * 256 (and a power of two per row) are exact in 32 bits, here and there."""
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    kind = svl.SVL_OUT_F32 if kept == F32 else svl.SVL_OUT_BF16
    other = torch.cuda.Stream()
    traffic = torch.empty(2, 1 << 27, dtype=U8, device="cuda")
    outs = [torch.empty(m, n, dtype=kept, device="cuda") for _ in range(4)]
    f = None
    for _ in range(50):
        sets = [(operand(g, m, k, 125), operand(g, n, k, 126)) for _ in outs]
        if factor:
            f = torch.ldexp(torch.ones(m, device="cuda"), torch.randint(-2, 3, (m,), device="cuda", generator=g))
        torch.cuda.synchronize()
        if beside:
            with torch.cuda.stream(other):
                for _ in range(8):
                    traffic[0].copy_(traffic[1])
        for out, ((a, sa, _), (b, sb, _)) in zip(outs, sets):
            svl.svl_gemm_mxf4(a, k // 2, sa, b, k // 2, sb, m, n, k, out, n, kind, row_factor=f)
        for out, ((_, _, va), (_, _, vb)) in zip(outs, sets):
            want = va @ vb.t()
            if factor:
                want *= f[:, None]
            assert torch.equal(out, want.to(kept))
    torch.cuda.synchronize()
