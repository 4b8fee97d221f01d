"""MXFP4 calls that the documentation allows and nothing else makes: results at any address, offsets past 32 bits, several
host threads, other streams, graphs beside each other."""
import os
import subprocess
import sys
import threading

import numpy as np
import pytest
import torch

from paper_2607_20357_gb300 import svl
from tests import mxf4_reference as R
from tests.test_gpu_mxf4_gemm import BF16, F32, U8, operand, product, whole

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)


def held(x):
    rows, cols = x.shape
    c = torch.zeros(rows, R.held_bytes(cols), dtype=U8, device="cuda")
    s = torch.zeros(svl.svl_mxf4_scale_size(rows, cols), dtype=U8, device="cuda")
    svl.svl_quantize_rows_mxf4(x, rows, cols, x.stride(0), c, c.shape[1], s)
    return c, s


@pytest.mark.parametrize("m,n,k", [(1, 640, 512), (20, 640, 4096), (60, 640, 8192), (100, 384, 8192), (200, 640, 1024),
                                   (300, 512, 12288), (1030, 1024, 512)])
@pytest.mark.parametrize("kept", [F32, BF16])
@pytest.mark.parametrize("shift_c,shift_r", [(1, 0), (0, 3), (2, 2)])
def test_results_at_any_address(m, n, k, kept, shift_c, shift_r):
    """C and the residual start `shift` elements behind an aligned address."""
    a, sa, va = operand(m, m, k, None, 125, 128)
    b, sb, vb = operand(n, n, k, None, 126, 129)
    _, r = whole(m, n, False, True, kept)
    c = torch.full((m * n + 8,), 7.0, dtype=kept, device="cuda")
    rr = torch.full((m * n + 8,), float("nan"), dtype=kept, device="cuda")
    rr[shift_r:shift_r + m * n] = r.cuda().view(-1)
    svl.svl_gemm_mxf4(a, k // 2, sa, b, k // 2, sb, m, n, k, c[shift_c:], n,
                      svl.SVL_OUT_F32 if kept == F32 else svl.SVL_OUT_BF16, residual=rr[shift_r:], ld_residual=n)
    want = (torch.from_numpy(va).cuda() @ torch.from_numpy(vb).cuda().t() + r.double().cuda()).float().to(kept)
    assert torch.equal(c[shift_c:shift_c + m * n].view(m, n), want)
    assert (c[:shift_c] == 7).all() and (c[shift_c + m * n:] == 7).all()


@pytest.mark.parametrize("m", [2, 100, 300])
def test_residual_of_other_rows_apart(m):
    """C and the residual with strides of their own, columns between them left alone."""
    n, k = 256, 512
    a, sa, va = operand(1, m, k, None, 125, 128)
    b, sb, vb = operand(2, n, k, None, 126, 129)
    _, r = whole(m, n, False, True, BF16)
    rr = torch.full((m, n + 24), float("nan"), dtype=BF16, device="cuda")
    rr[:, :n] = r.cuda()
    out = product(a, sa, b, sb, m, n, k, BF16, ld_c=n + 8, residual=rr, ld_residual=n + 24)
    want = (torch.from_numpy(va) @ torch.from_numpy(vb).t() + r.double()).float().to(BF16)
    assert torch.equal(out[:, :n].cpu(), want) and (out[:, n:] == 7).all()


def test_rows_past_32_bits():
    """More than 2^32 values: the last rows are those of a call of their own."""
    rows, cols = 65540, 65600
    src = torch.empty(rows, cols, dtype=BF16, device="cuda")
    for r in range(0, rows, 8192):
        src[r:r + 8192].normal_()
    gain = torch.rand(cols, device="cuda").to(BF16)
    codes = torch.zeros(rows, R.held_bytes(cols), dtype=U8, device="cuda")
    scales = torch.zeros(svl.svl_mxf4_scale_size(rows, cols), dtype=U8, device="cuda")
    inv = torch.empty(rows, device="cuda")
    svl.svl_quantize_rows_mxf4(src, rows, cols, cols, codes, codes.shape[1], scales, gain=gain, eps=1e-5, inv_rms=inv)
    first = rows // 128 * 128
    last = src[first:].contiguous()
    n = rows - first
    c2 = torch.zeros(n, R.held_bytes(cols), dtype=U8, device="cuda")
    s2 = torch.zeros(svl.svl_mxf4_scale_size(n, cols), dtype=U8, device="cuda")
    inv2 = torch.empty(n, device="cuda")
    svl.svl_quantize_rows_mxf4(last, n, cols, cols, c2, c2.shape[1], s2, gain=gain, eps=1e-5, inv_rms=inv2)
    assert torch.equal(codes[first:], c2) and torch.equal(scales[-s2.numel():], s2)
    # groups of other sizes add in another order: a thread's four sums take 4 of a step's 16 squares, 129 steps of 512
    # columns at most, 17 more sums join them and make the mean, half of that after the root, and two roundings more
    tol = 2 * (0.5 * (4 * 129 + 17) + 2) * 2.0 ** -24
    assert torch.allclose(inv[first:], inv2, rtol=tol, atol=0)
    out = src.zero_()
    svl.svl_dequantize_rows_mxf4(codes, codes.shape[1], scales, rows, cols, out, cols)
    back = torch.empty(n, cols, dtype=BF16, device="cuda")
    svl.svl_dequantize_rows_mxf4(c2, c2.shape[1], s2, n, cols, back, cols)
    assert torch.equal(out[first:], back)


@pytest.mark.parametrize("m,n", [(65600, 65664), (65600, 65601)])
def test_product_past_32_bits(m, n):
    """More than 2^32 results, by tensor stores and by plain ones."""
    k = 64
    a, sa, va = operand(1, m, k, None, 125, 128)
    b, sb, vb = operand(2, n, k, None, 126, 129)
    out = torch.full((m, n), 7.0, dtype=BF16, device="cuda")
    svl.svl_gemm_mxf4(a, k // 2, sa, b, k // 2, sb, m, n, k, out, n, svl.SVL_OUT_BF16)
    wb = torch.from_numpy(vb).float().cuda()
    for r in (0, 255, 32768, 65400, m - 1):
        assert torch.equal(out[r].float(), (wb @ torch.from_numpy(va[r]).float().cuda()).to(BF16).float())
    assert torch.equal(out[:, n - 1].float(), (torch.from_numpy(va).float().cuda() @ wb[n - 1]).to(BF16).float())


def test_threads_at_once():
    """Host threads with products of different kinds, each on a stream of its own."""
    shapes = [(1, 4096, 4096), (48, 1024, 8192), (100, 640, 8192), (300, 512, 12288), (700, 1024, 1024), (1500, 2048, 512)]
    inputs, wants = [], []
    for i, (m, n, k) in enumerate(shapes):
        a, b = operand(i, m, k, None, 125, 128), operand(i + 50, n, k, None, 126, 129)
        inputs.append((a, b))
        wants.append(product(a[0], a[1], b[0], b[1], m, n, k, F32).clone())
    torch.cuda.synchronize()
    bad = []

    def work(i):
        m, n, k = shapes[i]
        (a, sa, _), (b, sb, _) = inputs[i]
        stream = torch.cuda.Stream()
        out = torch.empty(m, n, device="cuda")
        torch.cuda.current_stream().synchronize()
        for _ in range(40):
            svl.svl_gemm_mxf4(a, a.shape[1], sa, b, b.shape[1], sb, m, n, k, out, n, svl.SVL_OUT_F32,
                              stream=stream.cuda_stream)
        stream.synchronize()
        if not torch.equal(out, wants[i]):
            bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(shapes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_graphs_beside_each_other():
    """Two captured chains of calls, replayed on two streams at once."""
    def chain(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn(64, 1024, device="cuda", generator=g).to(BF16)
        w = held(torch.randn(2048, 1024, device="cuda", generator=g).to(BF16))
        c = torch.zeros(64, 512, dtype=U8, device="cuda")
        s = torch.zeros(svl.svl_mxf4_scale_size(64, 1024), dtype=U8, device="cuda")
        out = torch.empty(64, 2048, device="cuda")

        def run():
            svl.svl_quantize_rows_mxf4(x, 64, 1024, 1024, c, 512, s)
            svl.svl_gemm_mxf4(c, 512, s, w[0], 512, w[1], 64, 2048, 1024, out, 2048, svl.SVL_OUT_F32)
        return run, out

    chains = [chain(1), chain(2)]
    wants, graphs = [], []
    for run, out in chains:
        run()
        torch.cuda.synchronize()
        wants.append(out.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append(graph)
        out.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for (_, out), want in zip(chains, wants):
        assert torch.equal(out, want)


FIRST = """
import torch
from paper_2607_20357_gb300 import svl
BF16, U8 = torch.bfloat16, torch.uint8
m, n, k = %d, 512, %d
x, w = torch.randn(m, k, device="cuda").to(BF16), torch.randn(n, k, device="cuda").to(BF16)
held = [(torch.zeros(r, k // 2, dtype=U8, device="cuda"),
         torch.zeros(svl.svl_mxf4_scale_size(r, k), dtype=U8, device="cuda")) for r in (m, n)]
out = torch.zeros(m, n, device="cuda")

def run():
    for src, (c, s) in zip((x, w), held):
        svl.svl_quantize_rows_mxf4(src, src.shape[0], k, k, c, k // 2, s)
    (a, sa), (b, sb) = held
    svl.svl_gemm_mxf4(a, k // 2, sa, b, k // 2, sb, m, n, k, out, n, svl.SVL_OUT_F32)

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run()
graph.replay()
torch.cuda.synchronize()
first = out.clone()
out.zero_()
run()
assert torch.equal(out, first) and out.abs().max() > 0
"""


@pytest.mark.parametrize("m,k", [(3, 4096), (60, 12288), (300, 1024), (300, 16384)])
def test_a_process_whose_first_call_is_captured(m, k):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST % (m, k)], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr


def test_the_same_matrix_twice():
    """A matrix times itself, and results that do not change when they are computed over."""
    a, s, v = operand(3, 200, 320, None, 126, 128)
    first = product(a, s, a, s, 200, 200, 320, F32)
    assert torch.equal(first, first.t()) and torch.equal(first.cpu(), torch.from_numpy(v @ v.T).float())


def test_rows_beside_each_other():
    """Matrices whose rows alternate in memory: each call leaves the other's alone."""
    g = np.random.default_rng(5)
    x = torch.from_numpy(g.standard_normal((2, 33, 96))).to(BF16)
    both = torch.full((33, 2, 48), 0xEE, dtype=U8, device="cuda")
    scales = [torch.full((512,), 0xEE, dtype=U8, device="cuda") for _ in range(2)]
    for i in range(2):
        svl.svl_quantize_rows_mxf4(x[i].contiguous().cuda(), 33, 96, 96, both[:, i], 96, scales[i])
    for i in range(2):
        code, byte = R.quantised(x[i].double().numpy())
        np.testing.assert_array_equal(both[:, i].cpu().numpy(), R.packed(code))
        np.testing.assert_array_equal(scales[i].cpu().numpy(), R.laid_out(byte, 96, 0xEE))


@pytest.mark.parametrize("m,k", [(1, 512), (12, 4096), (60, 2560), (128, 256)])
def test_kernels_that_take_all_tensor_memory_behind_a_product(m, k):
    """Products of few rows leave room on their SMs, where CTAs of the next kernel may start before they have ended."""
    from tests.test_gpu_fp8 import TINY, Case, synth
    case = Case(synth.reduced(TINY.dims, n_layers=1), TINY, seed=5, max_seq=256)
    n = 19456  # a tile for every SM
    a, sa, va = operand(1, m, k, None, 125, 128)
    b, sb, vb = operand(2, n, k, None, 126, 129)
    out, other = torch.empty(m, n, device="cuda"), torch.empty(300, 4096, device="cuda")
    codes = torch.full((4096, 128), 0x38, dtype=U8, device="cuda")  # ones
    ones = torch.ones(4096, device="cuda")

    def run():
        for _ in range(20):
            svl.svl_gemm_mxf4(a, k // 2, sa, b, k // 2, sb, m, n, k, out, n, svl.SVL_OUT_F32)
            svl.svl_gemm_e4m3(case.model.handle, codes, ones, codes, ones, 300, 4096, 128, other)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    out.zero_()
    other.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, (torch.from_numpy(va).cuda() @ torch.from_numpy(vb).cuda().t()).float())
    assert (other == 128).all()
