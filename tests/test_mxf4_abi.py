"""Sizes and refusals of the MXFP4 entry points (no GPU needed): nothing is launched and no pointer below is followed."""
import numpy as np
import pytest
import torch

from paper_2607_20357_gb300 import svl
from tests import mxf4_reference as R

INVALID, UNSUPPORTED = 1, 3
P = 1 << 20  # an aligned address that nothing reads
NAN, INF = float("nan"), float("inf")


def code(fn, *args, **kw):
    with pytest.raises(svl.SvlError) as e:
        fn(*args, stream=0, **kw)
    return e.value.code


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (128, 128), (129, 128), (128, 129), (5403, 4096), (7, 18944)])
def test_scale_size(svl_lib, rows, cols):
    assert svl.svl_mxf4_scale_size(rows, cols) == R.scale_bytes(rows, cols)


def test_scale_size_of_nothing(svl_lib):
    for rows, cols in ((0, 32), (-1, 32), (1, 0), (1, -8), (1, (1 << 30) + 1), (1 << 60, 1 << 20)):
        assert svl.svl_mxf4_scale_size(rows, cols) == 0
    assert svl.svl_mxf4_scale_size(1 << 20, 1 << 30) == (1 << 50) // 32


def test_layout_of_the_reference():
    """Every block of a matrix has a byte of its own, and whole tiles have no others."""
    for rows, cols in ((128, 128), (256, 384), (130, 100)):
        at = R.scale_at(rows, cols)
        assert len(np.unique(at)) == at.size and at.max() < R.scale_bytes(rows, cols)
    assert R.scale_at(256, 384).size == R.scale_bytes(256, 384)
    at = R.scale_at(200, 300)
    assert (at[0, 1], at[1, 0], at[32, 0], at[128, 0], at[0, 4]) == (1, 16, 4, 1536, 512)


def test_rounding_of_the_reference():
    x = np.array([0, 0.25, 0.26, 0.5, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.1, 6])
    np.testing.assert_array_equal(R.nearest(x), [0, 0, 1, 1, 2, 2, 4, 4, 6, 6, 7, 7])
    assert R.scale_exponents(np.array([6.0]))[0] == 0 and R.scale_exponents(np.array([6.000001]))[0] == 1
    assert R.scale_exponents(np.array([3.0]))[0] == -1 and R.scale_exponents(np.array([0.0]))[0] == -127


def test_quantise(svl_lib):
    def call(src=P, rows=4, cols=64, ld=64, dst=P, ld_dst=32, scale=P, **kw):
        return code(svl.svl_quantize_rows_mxf4, src, rows, cols, ld, dst, ld_dst, scale, **kw)
    assert call(src=None) == INVALID
    assert call(src=P + 8) == INVALID
    assert call(rows=-1) == INVALID
    assert call(cols=0) == INVALID
    assert call(cols=60) == INVALID
    assert call(ld=56) == INVALID
    assert call(ld=68) == INVALID
    assert call(dst=None) == INVALID
    assert call(dst=P + 8) == INVALID
    assert call(ld_dst=16) == INVALID
    assert call(ld_dst=40) == INVALID
    assert call(cols=72, ld=72, ld_dst=32) == INVALID  # a third block's bytes
    assert call(scale=None) == INVALID
    assert call(scale=P + 4) == INVALID
    assert call(gain=P + 2) == INVALID
    assert call(inv_rms=P + 2) == INVALID
    for eps in (-1e-5, NAN, INF):
        assert call(inv_rms=P, eps=eps) == INVALID
    assert call(cols=(1 << 30) + 8, ld=1 << 31, ld_dst=1 << 31) == UNSUPPORTED
    assert call(rows=1 << 60, cols=1 << 20, ld=1 << 20, ld_dst=1 << 20) == UNSUPPORTED
    before = svl.svl_launch_count()
    svl.svl_quantize_rows_mxf4(P, 0, 64, 64, P, 32, P, stream=0)
    assert svl.svl_launch_count() == before


def test_swiglu(svl_lib):
    def call(gate=P, ld_gate=128, up=P + 128, ld_up=128, rows=4, cols=64, dst=P, ld_dst=32, scale=P):
        return code(svl.svl_swiglu_rows_mxf4, gate, ld_gate, up, ld_up, rows, cols, dst, ld_dst, scale)
    assert call(gate=None) == INVALID
    assert call(up=None) == INVALID
    assert call(up=P + 2) == INVALID
    assert call(ld_gate=63) == INVALID
    assert call(ld_up=60) == INVALID
    assert call(rows=-1) == INVALID
    assert call(cols=4) == INVALID
    assert call(ld_dst=24) == INVALID
    assert call(scale=None) == INVALID
    before = svl.svl_launch_count()
    svl.svl_swiglu_rows_mxf4(P, 128, P, 128, 0, 64, P, 32, P, stream=0)
    assert svl.svl_launch_count() == before


def test_dequantise(svl_lib):
    def call(src=P, ld=32, scale=P, rows=4, cols=64, dst=P, ld_dst=64):
        return code(svl.svl_dequantize_rows_mxf4, src, ld, scale, rows, cols, dst, ld_dst)
    assert call(src=None) == INVALID
    assert call(src=P + 4) == INVALID
    assert call(ld=31) == INVALID
    assert call(ld=24) == INVALID
    assert call(scale=None) == INVALID
    assert call(rows=-1) == INVALID
    assert call(cols=12) == INVALID
    assert call(dst=None) == INVALID
    assert call(dst=P + 2) == INVALID
    assert call(ld_dst=60) == INVALID
    before = svl.svl_launch_count()
    svl.svl_dequantize_rows_mxf4(P, 32, P, 0, 64, P, 64, stream=0)
    assert svl.svl_launch_count() == before


def test_product(svl_lib):
    def call(a=P, ld_a=32, sa=P, b=P, ld_b=32, sb=P, m=4, n=8, k=64, c=P, ld_c=8, t=svl.SVL_OUT_F32, **kw):
        return code(svl.svl_gemm_mxf4, a, ld_a, sa, b, ld_b, sb, m, n, k, c, ld_c, t, **kw)
    for name in ("a", "sa", "b", "sb"):
        assert call(**{name: None}) == INVALID
        assert call(**{name: P + 8}) == INVALID
    assert call(m=-1) == INVALID
    assert call(n=0) == INVALID
    assert call(k=0) == INVALID
    assert call(k=-32) == INVALID
    assert call(k=65) == INVALID             # rows of three blocks
    assert call(ld_a=24) == INVALID
    assert call(ld_b=40) == INVALID
    assert call(c=None) == INVALID
    assert call(c=P + 2) == INVALID
    assert call(c=P + 1, t=svl.SVL_OUT_BF16) == INVALID
    assert call(ld_c=7) == INVALID
    assert call(t=2) == INVALID
    assert call(residual=P, ld_residual=7) == INVALID
    assert call(residual=P + 2, ld_residual=8) == INVALID
    assert call(row_factor=P + 1) == INVALID
    assert call(status=P + 2) == INVALID
    assert call(k=(1 << 30) + 32, ld_a=1 << 30, ld_b=1 << 30) == UNSUPPORTED
    before = svl.svl_launch_count()
    svl.svl_gemm_mxf4(P, 32, P, P, 32, P, 0, 8, 64, P, 8, svl.SVL_OUT_F32, stream=0)
    assert svl.svl_launch_count() == before


def test_arguments_of_other_types(svl_lib):
    """Tensors and plain ints go as they are, addresses and other integers are converted, alone or beside them."""
    x = torch.zeros(4096, dtype=torch.uint8)  # (a CPU tensor: nothing is launched for no rows)
    at = x.data_ptr()
    assert at % 16 == 0
    for p in (x, at):
        for i in (int, np.int32, np.int64):
            svl.svl_dequantize_rows_mxf4(p, i(32), x, i(0), i(64), x, i(64), stream=0)
            svl.svl_quantize_rows_mxf4(p, i(0), 64, i(64), at, 32, x, gain=p, inv_rms=x, eps=np.float32(1e-5), stream=0)
            svl.svl_swiglu_rows_mxf4(x, i(64), p, 64, i(0), 64, x, 32, p, stream=0)
            svl.svl_gemm_mxf4(p, 32, x, p, i(32), x, i(0), 8, i(64), x, 8, svl.SVL_OUT_BF16, row_factor=x, residual=p,
                              ld_residual=i(8), status=x, stream=0)
    assert code(svl.svl_gemm_mxf4, x, np.int64(24), x, x, 32, x, 4, 8, 64, x, 8, 0) == INVALID


def test_empty_tensors(svl_lib):
    """No rows: the tensors that hold them are empty, their addresses null."""
    none, b = torch.empty(0, 32, dtype=torch.uint8), torch.zeros(4096, dtype=torch.uint8)
    assert none.data_ptr() == 0 and svl.svl_mxf4_scale_size(0, 64) == 0
    before = svl.svl_launch_count()
    svl.svl_quantize_rows_mxf4(none, 0, 64, 64, none, 32, none, stream=0, gain=b, inv_rms=none)
    svl.svl_swiglu_rows_mxf4(none, 128, none, 128, 0, 64, none, 32, none, stream=0)
    svl.svl_dequantize_rows_mxf4(none, 32, none, 0, 64, none, 64, stream=0)
    svl.svl_gemm_mxf4(none, 32, none, b, 32, b, 0, 8, 64, none, 8, svl.SVL_OUT_BF16, stream=0, row_factor=none)
    assert svl.svl_launch_count() == before
    assert code(svl.svl_gemm_mxf4, none, 32, none, none, 32, b, 0, 8, 64, none, 8, 0) == INVALID  # no weight
    assert code(svl.svl_quantize_rows_mxf4, none, 0, 64, 64, none, 16, none) == INVALID
    assert code(svl.svl_dequantize_rows_mxf4, none, 32, none, 1, 64, none, 64) == INVALID
