"""The 4-bit cache's attention called from several host threads at once, each with its own sizes, stream, workspace and
buffers: what one call sets up on the host does not reach another's."""
import threading

import numpy as np
import pytest
import torch

import tests.test_gpu_kv4 as kv4_tests
from paper_2607_20357_gb300 import svl

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)


# (heads, KV heads, rows): two to four columns of an item share one kernel, five to eight another; few items go to clusters
@pytest.mark.parametrize("calls,max_len", [
    ([(8, 1, 1), (5, 1, 1), (6, 1, 1)], 200), ([(4, 1, 1), (2, 1, 1), (3, 1, 1)], 200),
    ([(8, 1, 1), (5, 1, 1), (6, 1, 1)], 13_000), ([(4, 1, 1), (2, 1, 1), (3, 1, 1)], 13_000),
])
def test_calls_of_different_sizes_from_several_threads(calls, max_len):
    jobs = []
    for i, (heads, kv, rows) in enumerate(calls):
        desc = svl.Kv4Desc(1, kv, 128, max_len)
        cache, _ = kv4_tests._filled(95 + i, desc, [60])
        q = kv4_tests.rows_of(99, rows, heads * 128)
        want = kv4_tests._attend(desc, cache, q, [60 - rows], rows, heads, 0, 0, 0.088)
        ws = torch.empty(svl.svl_kv4_attention_workspace_size(desc, heads, rows), dtype=torch.uint8, device="cuda")
        out = torch.zeros(rows, heads * 128, dtype=torch.bfloat16, device="cuda")
        jobs.append((desc, cache, heads, rows, q.cuda(), kv4_tests.i32([60 - rows]), out, ws, want))
    torch.cuda.synchronize()
    failed, gate = [], threading.Barrier(len(jobs))

    def work(desc, cache, heads, rows, q, start, out, ws, want):
        stream = torch.cuda.Stream()
        gate.wait()
        try:
            for _ in range(4000):
                svl.svl_kv4_attention(desc, cache, heads, rows, q, q.stride(0), start, 0, 0, 0.088, out, out.stride(0),
                                      ws, ws.numel(), stream)
        except Exception as e:  # (a thread's exception would not reach the test)
            failed.append(e)
        stream.synchronize()

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for j in jobs:
        np.testing.assert_array_equal(j[6].cpu().double().numpy(), j[-1])
