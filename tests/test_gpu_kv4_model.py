"""The gated prefill, decode step and beam search over a 4-bit KV cache, against the same layers put together from the
library's single stages and operators (each of which has tests of its own)."""
import numpy as np
import pytest
import torch

from paper_2607_20357_gb300 import svl, synth
from tests.gpu_common import BAR, Case, rel_err
from tests.kv4_reference import as_bf16, quantised

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

TINY = synth.WORKLOADS["tiny"]
MHA = synth.reduced(TINY.dims, n_layers=3, n_prefix=1)
GQA = synth.reduced(TINY.dims, n_layers=2, d_model=1024, n_heads=8, n_kv_heads=4, n_groups=4, c_vis=1024)
BF16 = torch.bfloat16


def _case(dims, seed, n_vis, s_text, gemm_format=svl.SVL_GEMM_BF16, gates=True):
    case = Case(dims, TINY, seed=seed, batch=None, max_seq=512, gemm_format=gemm_format, std=0.05)
    b = synth.make_batch(TINY, seed, n_vis_list=n_vis, s_text_list=s_text, keep_list=[-1] * len(n_vis),
                         budget_list=[1.0] * len(n_vis), dims=dims)
    B = len(n_vis)
    g = torch.Generator().manual_seed(seed)
    b["group_gate"] = torch.ones(B, dims.n_layers, dims.n_groups, dtype=torch.uint8)
    b["layer_gate"] = torch.ones(B, dims.n_layers, dtype=torch.uint8)
    if gates:
        b["group_gate"] = (torch.rand(B, dims.n_layers, dims.n_groups, generator=g) < 0.7).to(torch.uint8)
        b["layer_gate"][0, dims.n_layers - 1] = 0
    case.b = {k: (v.cuda() if isinstance(v, torch.Tensor) else v) for k, v in b.items()}
    return case


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _prefill(case, max_len, beams):
    """The prompt's cache (every byte 0xFF before), lengths, logits and packed batch."""
    m, d, b = case.model, case.dims, case.b
    B = b["B"]
    nv, nt = int(b["vis"].shape[0]), int(b["text_ids"].shape[0])
    out = m.run(b, stages=("select", "pack"))
    X = out["X"].clone()
    desc = svl.Kv4Desc(B * beams, d.n_kv_heads, d.d_head, max_len)
    cache = torch.full((d.n_layers * svl.svl_kv4_cache_size(desc),), 0xFF, dtype=torch.uint8, device="cuda")
    cache_len = torch.full((B * beams,), -7, dtype=torch.int32, device="cuda")
    ws, wsb = m.workspace(B, nv, nt, "cuda", ("prefill",))
    svl.svl_gated_prefill_kv4(m.handle, B, nv + nt, out["X"], out["cu_seqlens"], out["pos"], b["layer_gate"],
                              b["group_gate"], svl.SVL_LOGITS_LAST, out["logits"], cache, max_len, beams, cache_len, ws,
                              wsb)
    return desc, cache, cache_len, out, X


@pytest.mark.parametrize("dims", [MHA, GQA], ids=["mha", "gqa"])
def test_prefill_stores_the_quantised_rows(dims):
    """Layer 0's cache holds what the QKV stage gives for the active groups; the logits are the plain prefill's."""
    case = _case(dims, 41, [64, 40, 7], [16, 9, 30])
    m, b = case.model, case.b
    B, beams = b["B"], 2
    desc, cache, cache_len, out, X = _prefill(case, 120, beams)
    lens = np.diff(out["cu_seqlens"].cpu().numpy())
    np.testing.assert_array_equal(cache_len.cpu().numpy(), np.repeat(lens, beams))
    t_cap, kvc = X.shape[0], dims.n_kv_heads * dims.d_head
    q = torch.zeros(t_cap, dims.d_model, dtype=BF16, device="cuda")
    k = torch.zeros(t_cap, kvc, dtype=BF16, device="cuda")
    vt = torch.zeros(kvc, (t_cap + 7) // 8 * 8, dtype=BF16, device="cuda")
    nv, nt = int(b["vis"].shape[0]), int(b["text_ids"].shape[0])
    ws, wsb = m.workspace(B, nv, nt, "cuda", ("prefill",))
    svl.svl_layer_stage(m.handle, svl.SVL_LAYER_QKV, 0, B, t_cap, X, out["cu_seqlens"], out["pos"], b["layer_gate"],
                        b["group_gate"], q=q, k=k, vt=vt, workspace=ws, workspace_bytes=wsb)
    total = int(lens.sum())
    ko, vo = (torch.empty(total, kvc, dtype=BF16, device="cuda") for _ in range(2))
    off = [0]
    for n in lens:
        off += [off[-1] + int(n), off[-1] + int(n)]
    svl.svl_kv4_read(desc, cache, total, _i32(off), None, ko, kvc, vo, kvc)
    gate = b["group_gate"].cpu()[:, 0] * b["layer_gate"].cpu()[:, :1]
    if dims.n_prefix > 0:
        gate = torch.ones_like(gate)
    shape = (total, dims.n_kv_heads, dims.d_head)
    wk, wv = (as_bf16(quantised(x[:total].cpu().reshape(shape))).float().numpy() for x in (k, vt.t().contiguous()))
    ko, vo = (x.cpu().float().numpy().reshape(shape) for x in (ko, vo))
    r = 0
    for s, n in enumerate(lens):
        for h in range(dims.n_kv_heads):
            on = bool(gate[s, h * dims.n_groups // dims.n_kv_heads])
            for got, want in ((ko, wk), (vo, wv)):
                if on:
                    np.testing.assert_array_equal(got[r:r + n, h], want[r:r + n, h])
                else:
                    assert np.isnan(got[r:r + n, h]).all()  # never written
        r += n
    plain = m.run(b, stages=("select", "pack", "prefill"))
    np.testing.assert_array_equal(out["logits"].cpu().numpy(), plain["logits"].cpu().numpy())
    assert svl.svl_get_device_status(m.handle) == 0
    case.close()


@pytest.mark.parametrize("dims,window,sinks,fmt", [
    (MHA, 0, 0, svl.SVL_GEMM_BF16), (GQA, 0, 0, svl.SVL_GEMM_BF16), (GQA, 40, 3, svl.SVL_GEMM_BF16),
    (MHA, 33, 33, svl.SVL_GEMM_BF16), (GQA, 0, 0, svl.SVL_GEMM_E4M3),
], ids=["mha", "gqa", "gqa_window", "mha_window", "gqa_e4m3"])
def test_decode_step_equals_its_parts(dims, window, sinks, fmt):
    """Three steps, each beside one put together from the layer stages and the cache's operators on a copy of the cache;
    the final norm and LM head in torch. Logits to the repository's bar for one bf16 forward."""
    case = _case(dims, 43, [64, 40], [16, 30], fmt)
    m, b = case.model, case.b
    B, L, dh, kvc = b["B"], dims.n_layers, dims.d_head, dims.n_kv_heads * dims.d_head
    desc, cache, cache_len, _, _ = _prefill(case, 96, 1)
    mine = cache.clone()
    per = svl.svl_kv4_cache_size(desc)
    dws = torch.empty(svl.svl_decode_kv4_workspace_size(m.handle, B, 96), dtype=torch.uint8, device="cuda")
    aws = torch.empty(svl.svl_kv4_attention_workspace_size(desc, dims.n_heads, 1), dtype=torch.uint8, device="cuda")
    ws, wsb = m.workspace(B, B, B, "cuda", ("prefill",))
    logits = torch.empty(B, dims.vocab, device="cuda")
    nxt = torch.empty(B, dtype=torch.int32, device="cuda")
    w = case.w
    cu = _i32(list(range(B + 1)))
    for t in range(3):
        tok = _i32([(17 * t + 5 * i + 3) % dims.vocab for i in range(B)])
        start = cache_len.clone()
        svl.svl_decode_step_kv4(m.handle, B, tok, cache, 96, cache_len, b["layer_gate"], b["group_gate"], window, sinks,
                                logits, nxt, dws, dws.numel())
        assert cache_len.tolist() == (start + 1).tolist()
        X = w["embed"][tok.long()].contiguous()
        for l in range(L):
            q, ao = (torch.zeros(B, dims.d_model, dtype=BF16, device="cuda") for _ in range(2))
            k, v = (torch.zeros(B, kvc, dtype=BF16, device="cuda") for _ in range(2))
            vt = torch.zeros(kvc, 8, dtype=BF16, device="cuda")
            h = torch.zeros(B, dims.d_ffn, dtype=BF16, device="cuda")

            def stage(s):
                svl.svl_layer_stage(m.handle, s, l, B, B, X, cu, start, b["layer_gate"], b["group_gate"], q=q, k=k,
                                    vt=vt, ao=ao, h=h, workspace=ws, workspace_bytes=wsb)
            stage(svl.SVL_LAYER_QKV)
            v.copy_(vt.t()[:B])
            layer = mine[l * per:(l + 1) * per]
            svl.svl_kv4_write(desc, layer, k, kvc, v, kvc, B, None, start, None)
            # (groups that are off have no rows in the cache: their outputs are whatever and never read)
            svl.svl_kv4_attention(desc, layer, dims.n_heads, 1, q, dims.d_model, start, window, sinks, dh ** -0.5, ao,
                                  dims.d_model, aws, aws.numel())
            stage(svl.SVL_LAYER_OPROJ)
            stage(svl.SVL_LAYER_GATEUP)
            stage(svl.SVL_LAYER_DOWN)
        x = X.double()
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + dims.rms_eps) * w["final_norm"].double()
        want = (y.to(BF16).double() @ w["lm_head"].double().t()).cpu().numpy()
        got = logits.cpu().double().numpy()
        for i in range(B):
            assert rel_err(got[i], want[i]) < BAR, (t, i, rel_err(got[i], want[i]))
        assert nxt.tolist() == logits.argmax(-1).tolist()
    assert svl.svl_get_device_status(m.handle) == 0
    case.close()


def test_decode_step_with_a_full_cache():
    case = _case(MHA, 45, [40, 20], [10, 6], gates=False)
    m, b = case.model, case.b
    _, cache, cache_len, out, _ = _prefill(case, 51, 1)
    assert cache_len.tolist() == [50, 26]
    dws = torch.empty(svl.svl_decode_kv4_workspace_size(m.handle, 2, 51), dtype=torch.uint8, device="cuda")
    logits = torch.empty(2, MHA.vocab, device="cuda")
    nxt = torch.empty(2, dtype=torch.int32, device="cuda")
    for t, status in ((0, 0), (1, svl.SVL_DEV_BAD_INDEX)):
        svl.svl_decode_step_kv4(m.handle, 2, _i32([1, 2]), cache, 51, cache_len, b["layer_gate"], b["group_gate"], 0, 0,
                                logits, nxt, dws, dws.numel())
        assert svl.svl_get_device_status(m.handle) == status
        assert cache_len.tolist() == [51, 27 + t]
        assert bool(torch.isfinite(logits).all())
    assert int(nxt[0]) == -1 and int(nxt[1]) >= 0
    case.close()


@pytest.mark.parametrize("dims,beams,window", [(MHA, 4, 0), (GQA, 3, 40), (MHA, 1, 0)])
def test_beam_search_scores_are_its_tokens_log_probabilities(dims, beams, window):
    """Each returned beam, fed token by token into a cache that is never reordered: the sum of its tokens' log
    probabilities is its score. Every step's logits agree within 2^-8 of the largest (one bf16 rounding of the final
    state), so a step's log probability within twice that."""
    steps, sinks = 7, 2 if window else 0
    case = _case(dims, 47, [64, 33], [16, 12])
    m, b = case.model, case.b
    got = m.beam_search(b, beams, steps, eos=-1, window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert svl.svl_get_device_status(m.handle) == 0
    B, S = b["B"], b["B"] * beams
    tokens, scores = got["tokens"], got["scores"].cpu().double().numpy()
    assert tokens.shape == (B, beams, steps) and bool((np.diff(scores, axis=1) <= 0).all())
    assert len({tuple(r) for r in tokens[0].tolist()}) == beams
    desc, cache, cache_len, out, _ = _prefill(case, 128, beams)
    svl.svl_kv4_reorder(desc, cache, dims.n_layers, beams, _i32([0] * S), None, cache_len, None)
    lg, gg = b["layer_gate"].repeat_interleave(beams, 0), b["group_gate"].repeat_interleave(beams, 0)
    dws = torch.empty(svl.svl_decode_kv4_workspace_size(m.handle, S, 128), dtype=torch.uint8, device="cuda")
    logits = out["logits"].repeat_interleave(beams, 0).contiguous()
    total, slack = np.zeros(S), 0.0
    for t in range(steps):
        tok = tokens[:, :, t].reshape(-1).contiguous()
        p = torch.log_softmax(logits.double(), -1).gather(1, tok.long()[:, None])
        total += p[:, 0].cpu().numpy()
        slack += 2 * 2.0 ** -8 * float(logits.abs().max())
        svl.svl_decode_step_kv4(m.handle, S, tok, cache, 128, cache_len, lg, gg, window, sinks, logits, None, dws,
                                dws.numel())
    np.testing.assert_allclose(scores.reshape(-1), total, rtol=0, atol=slack)
    case.close()


def test_beam_search_greedy_first_token_and_eos():
    """The best first tokens are the prompt's best ids; a beam that meets eos stays as it is."""
    case = _case(MHA, 49, [64, 20], [16, 5], gates=False)
    m, b = case.model, case.b
    one = m.beam_search(b, 4, 1)
    plain = m.run(b)
    top = torch.log_softmax(plain["logits"].double(), -1).topk(4, -1)
    assert one["tokens"][:, :, 0].tolist() == top.indices.tolist()
    np.testing.assert_allclose(one["scores"].cpu().numpy(), top.values.cpu().numpy(), rtol=1e-5)
    eos = int(top.indices[0, 1])
    out = m.beam_search(b, 4, 6, eos=eos)
    t, fin, sc = out["tokens"].cpu(), out["finished"].cpu(), out["scores"].cpu()
    assert int(fin.sum()) > 0
    for s in range(2):
        for w in range(4):
            ends = (t[s, w] == eos).nonzero().flatten().tolist()
            assert bool(fin[s, w]) == bool(ends)
            if ends:
                assert ends == list(range(ends[0], 6))
    # the one that took eos at once is worth that one token
    at = [w for w in range(4) if t[0, w].tolist() == [eos] * 6]
    if at:
        assert abs(float(sc[0, at[0]]) - float(top.values[0, 1])) < 1e-4
    assert svl.svl_get_device_status(m.handle) == 0
    case.close()


def test_model_refusals():
    case = _case(MHA, 51, [10], [5], gates=False)
    m, b = case.model, case.b
    P = 1 << 20

    def code(fn, *args):
        with pytest.raises(svl.SvlError) as e:
            fn(*args)
        return e.value.code
    h, lg, gg = m.handle, b["layer_gate"], b["group_gate"]
    pre, dec = svl.svl_gated_prefill_kv4, svl.svl_decode_step_kv4
    assert code(pre, h, 1, 15, P, P, P, lg, gg, 0, P, None, 64, 1, P, P, 1 << 40) == 1
    assert code(pre, h, 1, 15, P, P, P, lg, gg, 0, P, P, 513, 1, P, P, 1 << 40) == 1       # longer than max_seq
    assert code(pre, h, 1, 15, P, P, P, lg, gg, 0, P, P, 64, 0, P, P, 1 << 40) == 1
    assert code(pre, h, 1, 15, P, P, P, lg, gg, 0, P, P, 64, 1, None, P, 1 << 40) == 1
    assert code(pre, h, 1, 15, P, P, P, lg, gg, 0, P, P, 64, 1, P, P, 64) == 7
    assert code(dec, h, 1, P, P + 8, 64, P, lg, gg, 0, 0, P, P, P, 1 << 40) == 1
    assert code(dec, h, 1, P, P, 64, P, lg, gg, -1, 0, P, P, P, 1 << 40) == 1
    assert code(dec, h, 1, P, P, 64, P, lg, gg, 0, -1, P, P, P, 1 << 40) == 1
    assert code(dec, h, 1, P, P, 64, P, lg, gg, 0, 0, None, P, P, 1 << 40) == 1
    assert code(dec, h, 1, P, P, 64, P, lg, gg, 0, 0, P, P, P, 64) == 7
    assert svl.svl_decode_kv4_workspace_size(h, 0, 64) == 0
    with pytest.raises(ValueError):
        m.beam_search(b, 0, 3)
    case.close()
