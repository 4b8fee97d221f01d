"""Performance cases of the 4-bit KV cache and of beam search: writing rows into the cache and reading them back,
attention over it (sliding window, first tokens that stay visible), beam selection, and the reordering of the cache's
slots after it.

``run`` has two forms. With ``own`` it makes the calls a program makes of the framework's binding; without, it computes
the same with elementary torch operations in 32 bits. A case holds its sizes; ``shape`` seeds what decides the amount of
work (ragged lengths, parents), so that ``work`` knows it without the data.

The cache of one layer is [slots][kv heads][tiles] of tiles of 32 positions, 36 * d_head bytes each, J = d_head / 32
groups of 32 dimensions per row:

    codes of K   [32 rows][4 t][J j] words of 8 nibbles: dimensions 32 j + 8 t + 0..7
    codes of V   [2 strips][2 quads][8 g][4 t][J j] words: rows 16 strip + 8 quad + 2 t (low half) and + 1 (high half),
                 dimensions 32 j + 4 g + 0..3
    scales of K  [32 rows][J] bf16
    scales of V  [16 row pairs][J][2] bf16

A nibble n of a group with scale s stands for s * (n - 8); s = e / -8 with e the group's element of largest magnitude
(the positive one of two alike), and 0 where |e| is under 2^-123.
"""
import math
import random

import torch

own = False

BF16, F32, F64, I32, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8
TILE = 32


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one decode step of 16 running requests: each slot's new row goes into the cache (the smallest write)
        dict(name="append_batch", kind="write", slots=16, kv=32, dh=128, fused=96, rows_lo=1, rows_hi=1, at_lo=250,
             at_hi=450, shape=1),
        # the prompts of a batch of 16, packed one after the other
        dict(name="write_prompts", kind="write", slots=16, kv=32, dh=128, fused=96, rows_lo=150, rows_hi=640, at_lo=0,
             at_hi=0, shape=2),
        # a few rows of a small model's cache, for a look at what it holds
        dict(name="read_few", kind="read", slots=3, kv=4, dh=64, rows_lo=5, rows_hi=90, at_lo=0, at_hi=40, shape=3),
        # the caches of eight long requests as bf16, to hand them on to a process without the 4-bit form
        dict(name="read_long", kind="read", slots=8, kv=4, dh=128, rows_lo=2000, rows_hi=8000, at_lo=0, at_hi=64,
             shape=4),
        # one token more for a single request of 1,900 rows, seven heads per KV head: latency
        dict(name="attend_one", kind="attend", slots=1, heads=28, kv=4, dh=128, rows=1, at_lo=1900, at_hi=1900, idle=0,
             window=0, sinks=0, shape=5),
        # one token more for each of 16 running requests
        dict(name="attend_batch", kind="attend", slots=16, heads=32, kv=32, dh=128, rows=1, at_lo=250, at_hi=450, idle=0,
             window=0, sinks=0, shape=6),
        # long contexts, a batch of eight
        dict(name="attend_long", kind="attend", slots=8, heads=32, kv=32, dh=128, rows=1, at_lo=4000, at_hi=16000,
             idle=0, window=0, sinks=0, shape=7),
        # three drafted tokens per request over the last 1,024 rows and the first four
        dict(name="attend_window", kind="attend", slots=8, heads=28, kv=4, dh=128, rows=3, at_lo=8000, at_hi=30000,
             idle=1, window=1024, sinks=4, shape=8),
        # one request with four beams
        dict(name="beam_one", kind="beam", samples=1, beams=4, vocab=32000, take=4, done=0.0, shape=9),
        # 32 requests with eight beams, a large vocabulary, twice as many candidates as beams, some beams finished
        dict(name="beam_batch", kind="beam", samples=32, beams=8, vocab=152064, take=16, done=0.1, shape=10),
        # a step of a beam search: what grew behind the shared prompts moves
        dict(name="reorder_step", kind="reorder", samples=4, beams=4, layers=4, kv=32, dh=128, at_lo=250, at_hi=450,
             grown_lo=1, grown_hi=64, shape=11),
        # beams that share nothing: whole slots move (the largest call)
        dict(name="reorder_whole", kind="reorder", samples=8, beams=4, layers=4, kv=32, dh=128, at_lo=0, at_hi=0,
             grown_lo=300, grown_hi=640, shape=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "read", "attend", "attend", "attend", "beam", "beam", "reorder"])
    shape = rng.randrange(1 << 30)
    kv, group, dh = rng.choice([(4, 1, 64), (4, 7, 128), (32, 1, 128), (40, 1, 128), (8, 4, 128), (2, 5, 64), (1, 12, 64)])
    if kind in ("write", "read"):
        slots = _log(rng, 1, 64)
        most = max(1, min(8000, int(1.2e6 / (slots * kv * dh / 128))))
        hi = _log(rng, 1, most)
        c = dict(kind=kind, slots=slots, kv=kv, dh=dh, rows_lo=max(1, hi // rng.choice([1, 2, 4])), rows_hi=hi, at_lo=0,
                 at_hi=rng.choice([0, 31, 500]), shape=shape)
        if kind == "write":
            c["fused"] = kv * (group + 2)
        return c
    if kind == "attend":
        slots = _log(rng, 1, 64)
        most = max(16, min(60000, int(2.4e6 / (slots * kv * dh / 128))))
        hi = _log(rng, 16, most)
        window = rng.choice([0, 0, 0, 33, 256, 1024, 4096])
        return dict(kind=kind, slots=slots, heads=kv * group, kv=kv, dh=dh, rows=rng.choice([1, 1, 1, 2, 3, 5, 8]),
                    at_lo=max(0, hi // rng.choice([1, 2, 8])), at_hi=hi, idle=rng.choice([0, 0, 1]), window=window,
                    sinks=rng.choice([0, 4, 37]) if window else 0, shape=shape)
    if kind == "beam":
        vocab = rng.choice([1000, 32000, 32003, 152064, 50001])
        beams = rng.choice([1, 2, 3, 4, 5, 8, 16])
        samples = _log(rng, 1, max(1, min(64, int(3.8e7 / (vocab * beams)))))
        return dict(kind=kind, samples=samples, beams=beams, vocab=vocab, take=beams * rng.choice([1, 1, 2]),
                    done=rng.choice([0.0, 0.0, 0.2]), shape=shape)
    beams = rng.choice([2, 3, 4, 5, 8])
    samples, layers = _log(rng, 1, 16), rng.choice([1, 2, 4])
    most = max(1, min(700, int(1.9e6 / (samples * beams * layers * kv * dh / 128))))
    hi = _log(rng, 1, most)
    return dict(kind=kind, samples=samples, beams=beams, layers=layers, kv=kv, dh=dh, at_lo=0,
                at_hi=rng.choice([0, 31, 200]), grown_lo=max(1, hi // rng.choice([1, 2, 4])), grown_hi=hi, shape=shape)


def _sizes(case):
    """What the case's `shape` decides: per slot (write, read, attend) or per sample (reorder) a start and a count."""
    rng = random.Random(case["shape"])
    if case["kind"] in ("write", "read"):
        return [(rng.randint(case["at_lo"], case["at_hi"]), rng.randint(case["rows_lo"], case["rows_hi"]))
                for _ in range(case["slots"])]
    if case["kind"] == "attend":
        got = [(rng.randint(case["at_lo"], case["at_hi"]), case["rows"]) for _ in range(case["slots"])]
        return [(-case["rows"], r) if i and i <= case["idle"] else (p, r) for i, (p, r) in enumerate(got)]
    if case["kind"] == "reorder":
        return [(rng.randint(case["at_lo"], case["at_hi"]), rng.randint(case["grown_lo"], case["grown_hi"]))
                for _ in range(case["samples"])]
    return []


def _parents(case):
    """The survivors of a sample keep their slots, each other beam takes over one of them (so that a pass repeated on
    the same state changes nothing)."""
    rng = random.Random(case["shape"] + 1)
    out = []
    for _ in range(case["samples"]):
        w = case["beams"]
        alive = sorted(rng.sample(range(w), rng.randint(1, max(1, w - 1))))
        out.append([i if i in alive else rng.choice(alive) for i in range(w)])
    return out


def _visible(pos, window, sinks):
    if pos < 0:
        return 0
    return pos + 1 if not window else min(pos + 1, window + min(sinks, max(0, pos + 1 - window)))


def work(case):
    kind = case["kind"]
    if kind == "beam":
        n = case["samples"] * case["beams"] * case["vocab"]
        return {"bytes": 4.0 * n + 13.0 * case["samples"] * case["take"], "flops": 4.0 * n}
    per = case["kv"] * (case["dh"] + case["dh"] // 8)  # cache bytes of one position
    row = case["kv"] * case["dh"] * 4                  # its K and V in bf16
    sizes = _sizes(case)
    if kind == "write":  # rows in, cache written, rows out
        n = sum(r for _, r in sizes)
        return {"bytes": float(n * (2 * row + per)), "flops": 8.0 * n * case["kv"] * case["dh"] * 2}
    if kind == "read":
        n = sum(r for _, r in sizes)
        return {"bytes": float(n * (row + per)), "flops": 2.0 * n * case["kv"] * case["dh"] * 2}
    if kind == "reorder":  # sources read, moved rows written, and all of them read back
        b = 0.0
        for (_, grown), p in zip(sizes, _parents(case)):
            moved = [i for i in range(case["beams"]) if p[i] != i]
            b += grown * case["layers"] * (per * (len({p[i] for i in moved}) + len(moved)) + row * case["beams"])
        return {"bytes": b, "flops": 2.0 * sum(g for _, g in sizes) * case["layers"] * case["beams"] * case["kv"] * case["dh"] * 2}
    b = f = 0.0
    for start, rows in sizes:
        last = start + rows - 1
        if last >= 0:
            # the union over the slot's rows: the last row's, and what earlier rows' windows reach further back
            reach = _visible(last, case["window"], case["sinks"])
            if case["window"]:
                reach = min(last + 1, reach + rows - 1)
            b += reach * per
        f += sum(_visible(start + r, case["window"], case["sinks"]) for r in range(rows)) * case["heads"] * case["dh"] * 4.0
    return {"bytes": b + case["slots"] * case["rows"] * case["heads"] * case["dh"] * 4.0, "flops": f}


# ------------------------------------------------------------------ inputs
def _quantise(x):
    """Codes 0..15 and bf16 scales of [..., dh] values, in groups of 32."""
    g = x.float().unflatten(-1, (-1, 32))
    hi, lo = g.amax(-1, keepdim=True), g.amin(-1, keepdim=True)
    e = torch.where(hi >= -lo, hi, lo)
    s = torch.where(torch.isfinite(e), e / -8, torch.full_like(e, math.nan))
    s = torch.where(s.abs() < 2.0 ** -126, torch.zeros_like(s), s).to(BF16)
    f = s.float()
    n = torch.round(g / torch.where(f == 0, torch.ones_like(f), f)).clamp(-8, 7) + 8
    n = torch.where(torch.isfinite(f) & (f != 0), n, torch.full_like(n, 8.0))
    return n.to(U8).flatten(-2), s.squeeze(-1)


def _bytes(n):
    return n[..., 0::2] | (n[..., 1::2] << 4)


def _nibbles(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _to_tiles(k, v):
    """[..., 32 T, dh] values as tiles [..., T, 36 dh]."""
    dh = k.shape[-1]
    J = dh // 32
    (nk, sk), (nv, sv) = _quantise(k.unflatten(-2, (-1, TILE))), _quantise(v.unflatten(-2, (-1, TILE)))
    kb = _bytes(nk.unflatten(-1, (J, 4, 8)).movedim(-2, -3)).flatten(-4)
    vb = nv.unflatten(-1, (J, 8, 4)).unflatten(-4, (2, 2, 4, 2))  # strip quad t half J g i
    vb = _bytes(torch.einsum("...sqthjgi->...sqgtjhi", vb)).flatten(-7)
    svp = sv.unflatten(-2, (16, 2)).transpose(-1, -2)
    return torch.cat((kb, vb, sk.contiguous().view(U8).flatten(-2), svp.contiguous().view(U8).flatten(-3)), -1)


def _places(cache, slot, pos):
    """The bytes that rows `pos` of slots `slot` (index tensors of one shape) have in the cache, as views and indices: codes of
    K [.., heads, dh / 2] and of V [.., heads, 8 g, J, 2], scales of K [.., heads, 2 J] and of V [.., heads, J, 2]."""
    dh = cache.shape[-1] // 36
    J, tile, p, every = dh // 32, pos // TILE, pos % TILE, slice(None)
    return ((cache[..., :16 * dh].unflatten(-1, (TILE, dh // 2)), (slot, every, tile, p)),
            (cache[..., 16 * dh:32 * dh].unflatten(-1, (2, 2, 8, 4, J, 2, 2)),
             (slot, every, tile, p // 16, p % 16 // 8, every, p % 8 // 2, every, p % 2)),
            (cache[..., 32 * dh:34 * dh].unflatten(-1, (TILE, 2 * J)), (slot, every, tile, p)),
            (cache[..., 34 * dh:].unflatten(-1, (16, J, 2, 2)), (slot, every, tile, p // 2, every, p % 2)))


def _rows_at(cache, slot, pos):
    """K and V [.., heads, dh] in 32 bits that the cache holds at rows `pos` of slots `slot`."""
    nk, nv, sk, sv = (view[at].contiguous() for view, at in _places(cache, slot, pos))
    dh = cache.shape[-1] // 36
    nk = _nibbles(nk.unflatten(-1, (4, dh // 32, 4))).movedim(-3, -2).float() - 8     # J t 8
    nv = _nibbles(nv).movedim(-3, -2).float() - 8                                     # J g 4
    sk, sv = sk.view(BF16).float(), sv.view(BF16).squeeze(-1).float()
    return (nk * sk[..., None, None]).flatten(-3), (nv * sv[..., None, None]).flatten(-3)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _rows(g, shape, dh):
    """Keys or values as layers make them: some channels larger than the rest, rows of different size."""
    x = torch.randn(shape + (dh,), device="cuda", generator=g, dtype=F32)
    channel = torch.exp(0.5 * torch.randn(dh, device="cuda", generator=g))
    row = torch.exp(0.2 * torch.randn(shape + (1,), device="cuda", generator=g))
    return (x * channel * row).to(BF16)


def _cache(g, slots, kv, tiles, dh):
    out = torch.empty(slots, kv, tiles, 36 * dh, dtype=U8, device="cuda")
    for i in range(slots):
        out[i] = _to_tiles(_rows(g, (kv, tiles * TILE), dh), _rows(g, (kv, tiles * TILE), dh))
    return out


def _i32(v):
    return torch.tensor(v, dtype=I32, device="cuda")


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _row_index(starts, counts):
    """Slot and position of every packed row."""
    slot = [torch.full((n,), i, dtype=torch.int64) for i, n in enumerate(counts)]
    pos = [torch.arange(s, s + n, dtype=torch.int64) for s, n in zip(starts, counts)]
    return torch.cat(slot).cuda(), torch.cat(pos).cuda()


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    st = {"case": dict(case)}
    if kind == "beam":
        S, W, V = case["samples"], case["beams"], case["vocab"]
        x = torch.randn(S * W, V, device="cuda", generator=g, dtype=F32)
        st["logits"] = x * (1.5 + torch.rand(S * W, 1, device="cuda", generator=g)) + 2
        st["scores"] = -torch.rand(S, W, device="cuda", generator=g).mul(12).sort(-1).values
        st["finished"] = (torch.rand(S, W, device="cuda", generator=g) < case["done"]).to(U8)
        st["eos"] = 2
        K = case["take"]
        st["out"] = (torch.empty(S, K, device="cuda"), torch.empty(S, K, dtype=I32, device="cuda"),
                     torch.empty(S, K, dtype=I32, device="cuda"), torch.empty(S, K, dtype=U8, device="cuda"))
        return st
    kv, dh = case["kv"], case["dh"]
    sizes = _sizes(case)
    if kind == "reorder":
        W, layers = case["beams"], case["layers"]
        starts = [s for s, _ in sizes for _ in range(W)] * layers
        counts = [n for _, n in sizes for _ in range(W)] * layers
        slots = case["samples"] * W
        st["parents"] = _i32(_parents(case))
        st["from"] = _i32([s for s, _ in sizes])
        st["len"] = _i32([s + n for s, n in sizes for _ in range(W)])
        all_slots = slots * layers
    else:
        starts, counts = [s for s, _ in sizes], [n for _, n in sizes]
        slots = all_slots = case["slots"]
    max_len = max(s + n for s, n in zip(starts, counts))
    max_len = max(max_len, 1) + 7
    tiles = -(-max_len // TILE)
    st.update(slots=slots, all_slots=all_slots, max_len=max_len, tiles=tiles, start=_i32(starts))
    if kind == "write":
        st["cache"] = torch.zeros(slots, kv, tiles, 36 * dh, dtype=U8, device="cuda")
    else:
        st["cache"] = _cache(g, all_slots, kv, tiles, dh)
    if kind == "attend":
        n = case["slots"] * case["rows"]
        st["q"] = (torch.randn(n, case["heads"] * dh, device="cuda", generator=g) * 0.7).to(BF16)
        st["scale"] = 1.0 / math.sqrt(dh)
        st["out"] = torch.empty(n, case["heads"] * dh, dtype=BF16, device="cuda")
        return st
    total = sum(counts)
    st["total"] = total
    st["row_off"] = _i32(_offsets(counts))
    st["slot"], st["pos"] = _row_index(starts, counts)
    st["k_out"] = torch.empty(total, kv * dh, dtype=BF16, device="cuda")
    st["v_out"] = torch.empty(total, kv * dh, dtype=BF16, device="cuda")
    if kind == "write":
        # K and V are columns of the rows that the fused projection wrote
        fused = _rows(g, (total, case["fused"]), dh).flatten(1)
        st["ld"] = case["fused"] * dh
        st["k"], st["v"] = fused[:, -2 * kv * dh:-kv * dh], fused[:, -kv * dh:]
    return st


# ------------------------------------------------------------------ the plain forms
def _plain_read(st):
    k, v = _rows_at(st["cache"], st["slot"], st["pos"])
    return k.flatten(1).to(BF16), v.flatten(1).to(BF16)


def _plain_write(st):
    case = st["case"]
    J = case["dh"] // 32
    (nk, sk), (nv, sv) = (_quantise(st[n].unflatten(1, (case["kv"], case["dh"]))) for n in ("k", "v"))
    new = (_bytes(nk.unflatten(-1, (J, 4, 8)).movedim(-2, -3)).flatten(-3), _bytes(nv.unflatten(-1, (J, 8, 4))).movedim(-3, -2),
           sk.contiguous().view(U8), sv.contiguous().view(U8).unflatten(-1, (J, 2)))
    for (view, at), x in zip(_places(st["cache"], st["slot"], st["pos"]), new):
        view[at] = x
    return _plain_read(st)


def _plain_attend(st):
    case = st["case"]
    S, R, A, kv, dh = case["slots"], case["rows"], case["heads"], case["kv"], case["dh"]
    start = st["start"].long()[:, None]
    # the rows that any of a slot's queries may see: all up to the last one, or the first ones and the window's
    if case["window"]:
        near = torch.arange(case["window"] + R - 1, device="cuda") + (start - case["window"] + 1).clamp(min=case["sinks"])
        j = torch.cat((torch.arange(case["sinks"], device="cuda").expand(S, -1), near), 1)
    else:
        j = torch.arange(case["at_hi"] + R, device="cuda").expand(S, -1)
    slot = torch.arange(S, device="cuda")[:, None].expand_as(j)
    k, v = (x.movedim(1, 2) for x in _rows_at(st["cache"], slot, j.clamp(max=st["max_len"] - 1)))  # slot kv rows dh
    q = st["q"].float().view(S, R, kv, A // kv, dh).permute(0, 2, 1, 3, 4).flatten(2, 3)            # slot kv (row head) dh
    pos = (start + torch.arange(R, device="cuda"))[..., None]
    see = j[:, None] <= pos
    if case["window"]:
        see &= (j[:, None] > pos - case["window"]) | (j[:, None] < case["sinks"])
    see = see[:, None, :, None].expand(S, 1, R, A // kv, -1).flatten(2, 3)
    x = torch.matmul(q, k.transpose(-1, -2)) * st["scale"]
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return o.unflatten(2, (R, A // kv)).permute(0, 2, 1, 3, 4).reshape(S * R, A * dh).to(BF16)


def _plain_beam(st):
    case = st["case"]
    S, W, V, K = case["samples"], case["beams"], case["vocab"], case["take"]
    x = st["logits"].view(S, W, V)
    m = x.amax(-1, keepdim=True)
    lse = (m + torch.log(torch.exp(x - m).sum(-1, keepdim=True)))
    alive = torch.isfinite(lse)
    x = torch.where(alive, x + 0.0, torch.zeros_like(x))
    # the best of each beam: larger logits first, of equal ones the lower id
    bits = x.view(I32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32) + torch.arange(V - 1, -1, -1, device="cuda")
    token = V - 1 - (torch.topk(key, K, -1).values & 0xFFFFFFFF)
    cand = x.gather(-1, token) + torch.where(alive, st["scores"][..., None] - lse, torch.full_like(lse, -math.inf))
    cand = torch.where(torch.isnan(cand), torch.full_like(cand, -math.inf), cand)
    # a finished beam stands for itself alone
    done = st["finished"][..., None] != 0
    keep = torch.full_like(cand, -math.inf)
    keep[..., 0] = torch.where(torch.isnan(st["scores"]), torch.full_like(st["scores"], -math.inf), st["scores"])
    cand = torch.where(done, keep, cand)
    token = torch.where(done, torch.full_like(token, st["eos"]), token)
    best, at = torch.sort(cand.flatten(1), dim=-1, descending=True, stable=True)
    at = at[:, :K]
    token, parent = token.flatten(1).gather(1, at), at // K
    finished = (st["finished"].gather(1, parent) != 0) | (token == st["eos"])
    return best[:, :K].contiguous(), parent.to(I32), token.to(I32), finished.to(U8)


def _plain_reorder(st):
    case = st["case"]
    layers, S, W = case["layers"], case["samples"], case["beams"]
    c = st["cache"].view((layers, S, W) + st["cache"].shape[1:])
    par = st["parents"].long()
    sample = torch.arange(S, device="cuda")[:, None]
    tile = torch.arange(st["tiles"], device="cuda")
    moved = (tile >= (st["from"] // TILE)[:, None, None]) & (tile * TILE < st["len"].view(S, W).gather(1, par)[..., None])
    c.copy_(torch.where(moved[None, :, :, None, :, None], c[:, sample, par], c))
    return _plain_read(st)


# ------------------------------------------------------------------ the framework's calls
def _plan(st):
    """What a program keeps between calls: the cache's description, a workspace."""
    from paper_2607_20357_gb300 import svl
    case = st["case"]
    plan = {"svl": svl}
    if case["kind"] == "beam":
        size = svl.svl_beam_select_workspace_size(case["samples"], case["beams"], case["vocab"], case["take"])
    else:
        plan["desc"] = svl.Kv4Desc(st["slots"], case["kv"], case["dh"], st["max_len"])
        plan["all"] = svl.Kv4Desc(st["all_slots"], case["kv"], case["dh"], st["max_len"])
        size = svl.svl_kv4_attention_workspace_size(plan["desc"], case["heads"], case["rows"]) if case["kind"] == "attend" else 0
    plan["ws"] = torch.empty(max(size, 256), dtype=U8, device="cuda")
    st["plan"] = plan
    return plan


def _run_own(st):
    case, plan = st["case"], st.get("plan") or _plan(st)
    svl, kind = plan["svl"], case["kind"]
    if kind == "beam":
        scores, parent, token, finished = st["out"]
        svl.svl_beam_select(case["samples"], case["beams"], case["vocab"], case["take"], st["logits"], case["vocab"],
                            st["scores"], st["finished"], st["eos"], scores, parent, token, finished, plan["ws"],
                            plan["ws"].numel())
        return st["out"]
    if kind == "attend":
        ld = case["heads"] * case["dh"]
        svl.svl_kv4_attention(plan["desc"], st["cache"], case["heads"], case["rows"], st["q"], ld, st["start"],
                              case["window"], case["sinks"], st["scale"], st["out"], ld, plan["ws"], plan["ws"].numel())
        return st["out"]
    if kind == "write":
        svl.svl_kv4_write(plan["desc"], st["cache"], st["k"], st["ld"], st["v"], st["ld"], st["total"], st["row_off"],
                          st["start"], None)
    elif kind == "reorder":
        svl.svl_kv4_reorder(plan["desc"], st["cache"], case["layers"], case["beams"], st["parents"], st["from"],
                            st["len"], None)
    ld = case["kv"] * case["dh"]
    svl.svl_kv4_read(plan["all"], st["cache"], st["total"], st["row_off"], st["start"], st["k_out"], ld, st["v_out"], ld)
    return st["k_out"], st["v_out"]


def run(state):
    if own:
        return _run_own(state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend, "beam": _plain_beam,
            "reorder": _plain_reorder}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ 64 bits, from the definitions
def _peek(cache, slot, pos, dh):
    """K and V [heads, positions, dh] of one slot in 64 bits, each element looked up at its place in the tile."""
    c = cache[slot]  # heads tiles bytes
    d = torch.arange(dh, device="cuda")
    J = dh // 32
    p, tile = pos % TILE, pos // TILE

    def scale(at):
        b = c[:, tile[:, None], at].to(torch.int64) | (c[:, tile[:, None], at + 1].to(torch.int64) << 8)
        return (b << 16).to(I32).view(F32).double()  # a bf16 number is the upper half of a float

    p = p[:, None]
    at_k = p * (dh // 2) + (((d % 32) // 8) * J + d // 32) * 4 + (d % 8) // 2
    at_v = 16 * dh + ((((p // 16) * 2 + (p % 16) // 8) * 8 + (d % 32) // 4) * 4 + (p % 8) // 2) * J * 4 + (d // 32) * 4 \
        + (p % 2) * 2 + (d % 4) // 2
    n_k, n_v = c[:, tile[:, None], at_k], c[:, tile[:, None], at_v]
    odd = (d % 2).to(U8) * 4
    s_k = scale(32 * dh + (p * J + d // 32) * 2)
    s_v = scale(34 * dh + (((p // 2) * J + d // 32) * 2 + p % 2) * 2)
    return ((n_k >> odd) & 15).double().sub(8) * s_k, ((n_v >> odd) & 15).double().sub(8) * s_v


def _exact_quantised(x):
    """[rows, columns] as what the cache holds of it."""
    g = x.double().view(x.shape[0], -1, 32)
    at = g.abs().argmax(-1, keepdim=True)
    e = g.gather(-1, at).abs()
    e = torch.where((g == e).any(-1, keepdim=True), e, -e)
    s = torch.where(e.abs() < 2.0 ** -123, torch.zeros_like(e), (e / -8).to(BF16).double())
    n = torch.clamp(torch.round(g / torch.where(s == 0, torch.ones_like(s), s)), -8, 7)
    return (s * n).view(x.shape)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "beam":
        S, W, V, K = case["samples"], case["beams"], case["vocab"], case["take"]
        x = st["logits"].double().view(S, W, V)
        score = st["scores"].double()[..., None]
        cand = score + torch.log_softmax(x, -1)
        done = st["finished"].view(S, W, 1) != 0
        only = torch.full_like(cand, -math.inf)
        only[..., st["eos"]] = score[..., 0]
        cand = torch.where(done, only, cand).flatten(1)
        return torch.topk(cand, K, -1).values, None, None, None
    if kind == "write":
        return _exact_quantised(st["k"].contiguous()), _exact_quantised(st["v"].contiguous())
    dh = case["dh"]
    if kind == "attend":
        S, R, A, kv = case["slots"], case["rows"], case["heads"], case["kv"]
        out = torch.zeros(S, R, A, dh, dtype=F64, device="cuda")
        q = st["q"].double().view(S, R, A, dh)
        for b, start in enumerate(st["start"].tolist()):
            for r in range(R):
                at = start + r
                if at < 0:
                    continue
                pos = torch.arange(at + 1, device="cuda")
                if case["window"]:
                    pos = pos[(pos > at - case["window"]) | (pos < case["sinks"])]
                k, v = _peek(st["cache"], b, pos, dh)
                x = torch.einsum("hgd,hpd->hgp", q[b, r].view(kv, A // kv, dh), k) / math.sqrt(dh)
                out[b, r] = torch.einsum("hgp,hpd->hgd", torch.softmax(x, -1), v).reshape(A, dh)
        return out.view(S * R, A * dh)
    k_all, v_all = [], []
    off = st["row_off"].tolist()
    for i, start in enumerate(st["start"].tolist()):
        src = torch.arange(start, start + off[i + 1] - off[i], device="cuda")
        slot = i
        if kind == "reorder":
            w = case["beams"]
            slot = i - i % w + _parents(case)[(i // w) % case["samples"]][i % w]
        k, v = _peek(st["cache"], slot, src, dh)
        k_all.append(k.transpose(0, 1).flatten(1))
        v_all.append(v.transpose(0, 1).flatten(1))
    return torch.cat(k_all), torch.cat(v_all)
