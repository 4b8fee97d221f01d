"""The 4-bit KV cache, attention over it and beam selection in 64 bits, written from their definitions alone."""
import numpy as np
import torch


def quantised(x):
    """[..., d_head] bf16 values as float64 values that the cache stands for (before their rounding to bf16)."""
    g = x.double().numpy().reshape(x.shape[:-1] + (-1, 32))
    big = np.abs(g).max(-1, keepdims=True)
    e = np.where((g == big).any(-1, keepdims=True), big, -big)
    s = e / -8.0
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        n = np.clip(np.rint(g / s), -8, 7)  # rint: half to even
        out = np.where(big < 2.0 ** -123, 0.0, s * n)
    out = np.where(np.isfinite(g).all(-1, keepdims=True), out, np.nan)
    return out.reshape(x.shape)


def as_bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)


def visible(pos, max_len, window, sinks):
    """Positions that a row at `pos` sees."""
    if pos < 0 or pos >= max_len:
        return np.zeros(0, np.int64)
    j = np.arange(pos + 1)
    return j[(j > pos - window) | (j < sinks)] if window else j


def attention(q, k, v, scale):
    """One query row of one head over the visible rows k, v [n, d_head] (float64): the output, and the spread
    sum_j p_j |v_j| and largest sum_d |q_d k_jd| that the error bound needs."""
    if len(k) == 0:
        return np.zeros(v.shape[-1]), np.zeros(v.shape[-1]), 0.0
    x = scale * (k @ q)
    p = np.exp(x - x.max())
    p /= p.sum()
    return p @ v, p @ np.abs(v), float(abs(scale) * (np.abs(k) @ np.abs(q)).max())


def attention_bound(ref, spread, size):
    """Largest error of a bf16 output whose softmax weights and weights times scale are rounded to 11 bits each
    (2^-11 of every term twice, so 2^-10 of their sum), whose scores are sums in float32 (relative error of a weight
    at most some 2^-17 of the score's terms) and which is rounded to bf16 once (8 bits: 2^-8)."""
    return 2.0 ** -8 * np.abs(ref) + (2.0 ** -10 + 2.0 ** -16 * (1 + size)) * spread * (1 + 2.0 ** -8) + 1e-37


def beam_select(logits, scores, finished, eos, take):
    """[W, V] float32 logits of one sample: the best `take` as (score, parent, token, finished), the score as the
    definition rounds it (float32) with lse from 64 bits."""
    rows = []
    for w in range(logits.shape[0]):
        if finished is not None and finished[w]:
            rows.append([(scores[w], w, eos)])
            continue
        x = logits[w].astype(np.float64)
        if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all():
            rows.append([(np.float32(-np.inf), w, t) for t in range(take)])
            continue
        lse = np.float32(x.max() + np.log(np.exp(x - x.max()).sum()))
        with np.errstate(invalid="ignore"):
            off = np.float32(scores[w] - lse)
            order = np.lexsort((np.arange(len(x)), -x))[:take]
            rows.append([(np.float32(logits[w, t] + off), w, int(t)) for t in order])
    flat = [(np.float32(-np.inf) if np.isnan(c) else c, w, t, i) for r in rows for i, (c, w, t) in enumerate(r)]
    for w, r in enumerate(rows):
        flat += [(np.float32(-np.inf), w, eos, i) for i in range(len(r), take)]
    flat.sort(key=lambda c: (-c[0], c[1], c[3]))
    return [(c, w, t, bool((finished is not None and finished[w]) or t == eos)) for c, w, t, _ in flat[:take]]
