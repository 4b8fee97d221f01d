"""Performance cases of 4-bit floating point with a scale for every 32 values (MXFP4): quantising rows, with or without a
norm's gain and the rows' 1/rms, reading them back, SwiGLU with the quantisation of its result, and the product of two such
matrices with a factor per row and a residual, from single tokens to whole prefill batches.

``run`` has two forms. With ``own`` it makes the calls a program makes of the framework's binding; without, it computes the
same with elementary torch operations in 32 bits.

A matrix [rows, cols] is held as codes and scales. Codes: a row is ceil(cols / 32) * 16 bytes, two values to a byte, the
earlier one in the low nibble, zeros behind the row's end. A code is sign, two bits of exponent, one of mantissa: 0, 0.5, 1,
1.5, 2, 3, 4, 6. Scales: a byte b for every 32 values of a row stands for 2^(b - 127) (255: NaN); 128 rows by 4 blocks make
512 bytes, [ceil(rows / 128)][ceil(cols / 128)][row % 32][row % 128 / 32][block % 4].

The exponent of a block is the smallest (from -127 up) at which its largest magnitude is at most 6; codes are rounded to
the nearest, ties to the even code.
"""
import math

import torch

own = False

BF16, F32, F64, I32, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # the normalised row of a single token on its way into a projection (the smallest call)
        dict(name="quantise_token", kind="quantise", rows=1, cols=4096, gain=True, rms=True),
        # the rows of 16 prompts with half of their visual tokens, before QKV or gate/up
        dict(name="quantise_prefill", kind="quantise", rows=5403, cols=4096, gain=True, rms=True),
        # weights quantised as a model is loaded
        dict(name="quantise_weights", kind="quantise", rows=18944, cols=3584, gain=False, rms=False),
        # a few rows with a ragged end, for a look at what they became
        dict(name="read_few", kind="read", rows=37, cols=1000),
        # weights handed on to a process without the 4-bit form
        dict(name="read_weights", kind="read", rows=11008, cols=4096),
        # the hidden rows of 16 running requests
        dict(name="swiglu_batch", kind="swiglu", rows=16, cols=11008),
        # the hidden rows of a prefill
        dict(name="swiglu_prefill", kind="swiglu", rows=5403, cols=11008),
        # an output projection for a single token: latency
        dict(name="product_token", kind="product", m=1, n=4096, k=4096, factor=False, residual=True, f32=False),
        # logits of eight requests
        dict(name="product_logits", kind="product", m=8, n=32000, k=4096, factor=True, residual=False, f32=True),
        # a prompt of 300 rows through a down projection
        dict(name="product_prompt", kind="product", m=300, n=3584, k=18944, factor=False, residual=True, f32=False),
        # gate and up of a full batch of 16 prompts (the largest call)
        dict(name="product_gate_up", kind="product", m=10240, n=22016, k=4096, factor=True, residual=False, f32=False),
        # the down projection of half of that batch, added to the residual stream
        dict(name="product_down", kind="product", m=5403, n=4096, k=11008, factor=False, residual=True, f32=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quantise", "quantise", "read", "swiglu", "product", "product", "product", "product"])
    width = rng.choice([256, 1024, 3584, 4096, 5120, 11008, 13824, 18944, 8 * _log(rng, 1, 2400)])
    if kind != "product":
        rows = _log(rng, 1, min(20000, int(6.4e7 / width)))
        c = dict(kind=kind, rows=rows, cols=width)
        if kind == "quantise":
            c.update(gain=rng.random() < 0.5, rms=rng.random() < 0.5)
        return c
    n = rng.choice([256, 1000, 3584, 4096, 4608, 5120, 11008, 12288, 22016, 32000, _log(rng, 1, 30000)])
    m = _log(rng, 1, max(1, min(10240, int(9e11 / (n * width)))))
    return dict(kind=kind, m=m, n=n, k=width, factor=rng.random() < 0.5, residual=rng.random() < 0.5,
                f32=rng.random() < 0.3)


def work(case):
    if case["kind"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        out = (4 if case["f32"] else 2) * m * n * (2 if case["residual"] else 1)
        return {"bytes": 17 / 32 * (m + n) * k + out + (4 * m if case["factor"] else 0), "flops": 2.0 * m * n * k}
    v = case["rows"] * case["cols"]
    held = 17 / 32 * v
    if case["kind"] == "read":
        return {"bytes": held + 2 * v, "flops": 1.0 * v}
    # rows in, codes out, and back
    return {"bytes": (4 if case["kind"] == "swiglu" else 2) * v + 2 * held + 2 * v,
            "flops": (8.0 if case["kind"] == "swiglu" else 3.0 + (2 if case["rms"] else 0)) * v}


# ------------------------------------------------------------------ plain quantisation
def _quantise(x):
    """Codes 0..15 [rows, 32 blocks] and scale bytes [rows, blocks] of [rows, cols] values in 32 bits."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    if cols % 32:
        x = torch.cat((x, torch.zeros(rows, blocks * 32 - cols, device=x.device, dtype=x.dtype)), 1)
    x = x.view(rows, blocks, 32)
    top = x.abs().amax(-1)
    bits = top.view(I32)
    byte = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x400000)).clamp(min=0)
    good = torch.isfinite(top)
    byte = torch.where(good, byte, torch.full_like(byte, 255))
    q = x * ((254 - byte.clamp(max=253)) << 23).view(F32)[..., None]
    a = torch.where(good[..., None], q.abs(), torch.zeros_like(q))
    code = (a > 0.25).to(U8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5
    code += (torch.signbit(q) & good[..., None]).to(U8) << 3
    return code.view(rows, blocks * 32), byte.to(U8)


def _pack(code):
    return code[:, 0::2] | (code[:, 1::2] << 4)


def _tiled(byte):
    """Scale bytes [rows, blocks] in their order in memory."""
    rows, blocks = byte.shape
    rt, kt = -(-rows // 128), -(-blocks // 4)
    out = torch.zeros(rt * 128, kt * 4, dtype=U8, device=byte.device)
    out[:rows, :blocks] = byte
    return out.view(rt, 4, 32, kt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _values(codes, scales, rows, cols):
    """[rows, cols] in 32 bits that codes and scales stand for."""
    rt, kt = -(-rows // 128), -(-cols // 128)
    byte = scales.view(rt, kt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, kt * 4)[:rows, :-(-cols // 32)].to(I32)
    s = torch.where(byte == 0, torch.full_like(byte, 0x400000), byte << 23).view(F32)
    s = torch.where(byte == 255, torch.full_like(s, math.nan), s)
    code = torch.stack((codes & 15, codes >> 4), -1).view(rows, -1, 32).to(I32)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    return (grid[code] * s[..., None]).view(rows, -1)[:, :cols]


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _rows(g, rows, cols, size=1.0):
    """Rows as layers make them: some channels far larger than the rest, rows of different size."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    x *= torch.exp(0.6 * torch.randn(cols, device="cuda", generator=g))
    x *= size * torch.exp(0.3 * torch.randn(rows, 1, device="cuda", generator=g))
    return x.to(BF16)


def _held(x):
    code, byte = _quantise(x.float())
    return _pack(code), _tiled(byte)


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    st = {"case": dict(case)}
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        st["a"], st["a_scale"] = _held(_rows(g, m, k))
        st["b"], st["b_scale"] = _held(_rows(g, n, k, 0.02))
        st["factor"] = torch.rand(m, device="cuda", generator=g) + 0.5 if case["factor"] else None
        kept = F32 if case["f32"] else BF16
        st["residual"] = torch.randn(m, n, device="cuda", generator=g).to(kept) if case["residual"] else None
        st["out"] = torch.empty(m, n, dtype=kept, device="cuda")
        return st
    rows, cols = case["rows"], case["cols"]
    width, tiles = -(-cols // 32) * 16, -(-rows // 128) * -(-cols // 128)
    st["out"] = torch.empty(rows, cols, dtype=BF16, device="cuda")
    if kind == "read":
        st["codes"], st["scales"] = _held(_rows(g, rows, cols, 0.02))
        return st
    st["codes"] = torch.zeros(rows, width, dtype=U8, device="cuda")
    st["scales"] = torch.zeros(tiles * 512, dtype=U8, device="cuda")
    if kind == "swiglu":
        # gate and up are the two halves of the rows that one product wrote
        st["both"] = _rows(g, rows, 2 * cols, 1.5)
        return st
    st["src"] = _rows(g, rows, cols)
    st["gain"] = (1 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(BF16) if case["gain"] else None
    st["inv_rms"] = torch.empty(rows, device="cuda") if case["rms"] else None
    return st


# ------------------------------------------------------------------ the plain forms
def _plain_product(st):
    case = st["case"]
    c = torch.matmul(_values(st["a"], st["a_scale"], case["m"], case["k"]),
                     _values(st["b"], st["b_scale"], case["n"], case["k"]).t())
    if case["factor"]:
        c = c * st["factor"][:, None]
    if case["residual"]:
        c = c + st["residual"].float()
    return c.to(st["out"].dtype)


def _plain(st):
    case = st["case"]
    rows, cols = case["rows"], case["cols"]
    inv_rms = None
    if case["kind"] != "read":
        if case["kind"] == "swiglu":
            gate, up = st["both"][:, :cols].float(), st["both"][:, cols:].float()
            x = gate / (1 + torch.exp(-gate)) * up
        else:
            x = st["src"].float()
            if case["rms"]:
                inv_rms = 1 / torch.sqrt((x * x).sum(-1) / cols + 1e-5)
            if case["gain"]:
                x = x * st["gain"].float()
        code, byte = _quantise(x)
        st["codes"].copy_(_pack(code))
        st["scales"].copy_(_tiled(byte))
    out = _values(st["codes"], st["scales"], rows, cols).to(BF16)
    return out if inv_rms is None else (out, inv_rms)


# ------------------------------------------------------------------ the framework's calls
def _run_own(st):
    from paper_2607_20357_gb300 import svl
    case, out = st["case"], st["out"]
    if case["kind"] == "product":
        n, held = case["n"], st["a"].shape[1]
        svl.svl_gemm_mxf4(st["a"], held, st["a_scale"], st["b"], held, st["b_scale"], case["m"], n, case["k"], out, n,
                          svl.SVL_OUT_F32 if case["f32"] else svl.SVL_OUT_BF16, row_factor=st["factor"],
                          residual=st["residual"], ld_residual=n)
        return out
    rows, cols = case["rows"], case["cols"]
    codes, held, scales = st["codes"], st["codes"].shape[1], st["scales"]
    if case["kind"] == "swiglu":
        svl.svl_swiglu_rows_mxf4(st["both"], 2 * cols, st["both"][:, cols:], 2 * cols, rows, cols, codes, held, scales)
    elif case["kind"] == "quantise":
        svl.svl_quantize_rows_mxf4(st["src"], rows, cols, cols, codes, held, scales, gain=st["gain"], eps=1e-5,
                                   inv_rms=st["inv_rms"])
    svl.svl_dequantize_rows_mxf4(codes, held, scales, rows, cols, out, cols)
    return (out, st["inv_rms"]) if case.get("rms") else out


def run(state):
    if own:
        return _run_own(state)
    return _plain_product(state) if state["case"]["kind"] == "product" else _plain(state)


# ------------------------------------------------------------------ 64 bits, from the definitions
def _look_up(codes, scales, rows, cols):
    """Each value looked up at its place."""
    d = torch.arange(cols, device="cuda")
    out = torch.empty(rows, cols, dtype=F64, device="cuda")
    for r0 in range(0, rows, 4096):
        r = torch.arange(r0, min(rows, r0 + 4096), device="cuda")[:, None]
        n = ((codes[r, d // 2] >> ((d % 2) * 4).to(U8)) & 15).to(torch.int64)
        at = ((r // 128) * (-(-cols // 128)) + d // 128) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + d % 128 // 32
        b = scales[at].to(torch.int64)
        e, f = (n >> 1) & 3, (n & 1).double()
        size = torch.where(e == 0, f * 0.5, torch.ldexp(1 + 0.5 * f, (e - 1).double()))
        value = torch.where(n >= 8, -size, size) * torch.pow(2.0, b.double() - 127)
        out[r0:r0 + 4096] = torch.where(b == 255, torch.full_like(value, math.nan), value)
    return out


def _exact_held(x):
    """[rows, cols] in 64 bits as what is held of it."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    m, k = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(m <= 0.75, k - 3, k - 2).clamp(min=-127)
    s = torch.pow(2.0, e.double())
    a = (x / s).abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.sign(x) * torch.round(a / step) * step * s).view(rows, -1)[:, :cols]


def exact(case, seed):
    st, kind = prepare(case, seed), case["kind"]
    if kind == "product":
        c = _look_up(st["a"], st["a_scale"], case["m"], case["k"]) @ _look_up(st["b"], st["b_scale"], case["n"], case["k"]).t()
        if case["factor"]:
            c *= st["factor"].double()[:, None]
        if case["residual"]:
            c += st["residual"].double()
        return c
    rows, cols = case["rows"], case["cols"]
    if kind == "read":
        return _look_up(st["codes"], st["scales"], rows, cols)
    if kind == "swiglu":
        gate, up = st["both"][:, :cols].double(), st["both"][:, cols:].double()
        return _exact_held(gate * torch.sigmoid(gate) * up)
    x = st["src"].double()
    inv_rms = torch.rsqrt((x ** 2).mean(-1) + 1e-5)
    held = _exact_held(x * st["gain"].double() if case["gain"] else x)
    return (held, inv_rms) if case["rms"] else held
