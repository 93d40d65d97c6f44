"""Performance cases of the 8-bit operators: block-scaled products, the quantisation that feeds them, and the norms
around a block.

What a program asks of the library when a transformer block's projections run on 8-bit operands: activations and
weights as e4m3 values with one power-of-two scale per block of 128 along K (activations: 1 x 128, weights: 128 x
128), the projections with the epilogues of the step (store, GELU, gated residual) and the one that hands its result
on in 8 bits, and the row pass between two blocks: norm of the block's output, gated and scaled residual update,
norm and modulation of the next block's input. Shapes follow the measured workloads: width 1024, ratio-4 MLP, 4096
and 32768 tokens, late cached steps of a few hundred rows, single rows; and generic odd ones.

All inputs are drawn on the GPU from the case's seed. The plain forms are elementary float32 operations; exact() is
written from the definitions in float64.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128
EPILOGUES = {"store": 0, "gelu": 1, "resid": 2, "gelu_fp8": 3}
NORMS = {"none": 0, "layer": 1, "rms": 2}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


def listed():
    return [
        # One token through a first MLP projection: nothing but latency and the weights' way from HBM.
        dict(name="gemm_one_row", kind="gemm", M=1, N=4096, K=1024, epi="gelu_fp8", gate=False),
        # The second MLP projection of the last cached steps at 16^3 (820 active tokens), gated residual.
        dict(name="gemm_late_resid", kind="gemm", M=820, N=1024, K=4096, epi="resid", gate=True),
        # Keys and values of the active tokens of a cached 32^3 step.
        dict(name="gemm_cached32_kv", kind="gemm", M=9831, N=2048, K=1024, epi="store", gate=False),
        # The MLP of a full 32^3 step: the first projection, handed on in 8 bits, ...
        dict(name="gemm_full32_fc1", kind="gemm", M=32768, N=4096, K=1024, epi="gelu_fp8", gate=False),
        # ... and the second one, added to the float32 residual rows.
        dict(name="gemm_full32_fc2", kind="gemm", M=32768, N=1024, K=4096, epi="resid", gate=True),
        # Sizes that fit no tile: ragged rows, columns and a last K block of 16.
        dict(name="gemm_odd", kind="gemm", M=1237, N=1328, K=1424, epi="gelu", gate=False),
        # The attention output of a cached 32^3 step, quantised for its output projection.
        dict(name="quant_cached32", kind="quant", rows=9831, K=1024, dtype="bf16", block_rows=1),
        # A layer's first MLP weight as it is loaded.
        dict(name="quant_weight", kind="quant", rows=4096, K=1024, dtype="f32", block_rows=128),
        # Between two blocks of the last cached steps at 16^3: norms on both sides, 8-bit rows for the next product.
        dict(name="norm_late", kind="norm", rows=820, d=1024, dtype="bf16", out="fp8", post="layer", pre="layer",
             batch=1, weights=False),
        # The same over all rows of a full 32^3 step, with learned RMS norms.
        dict(name="norm_full32", kind="norm", rows=32768, d=1024, dtype="bf16", out="fp8", post="rms", pre="rms",
             batch=1, weights=True),
        # Four samples at their own times (own gates and modulation), odd width, float32 block output.
        dict(name="norm_odd_b4", kind="norm", rows=4999, d=1320, dtype="f32", out="bf16", post="rms", pre="layer",
             batch=4, weights=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["gemm", "gemm", "gemm", "gemm", "quant", "norm", "norm"])
    if kind == "gemm":
        n, k = 16 * _log(rng, 8, 512), 16 * _log(rng, 8, 512)
        m = _log(rng, 1, max(2, min(32768, (1 << 37) // (n * k))))
        epi = rng.choice(sorted(EPILOGUES))
        return dict(kind=kind, M=m, N=n, K=k, epi=epi, gate=epi == "resid" and rng.random() < 0.7)
    if kind == "quant":
        return dict(kind=kind, rows=_log(rng, 1, 32768), K=8 * _log(rng, 16, 512), dtype=rng.choice(["f32", "bf16"]),
                    block_rows=rng.choice([1, 1, 128]))
    return dict(kind=kind, rows=_log(rng, 8, 32768), d=8 * _log(rng, 16, 512), dtype=rng.choice(["f32", "bf16", "bf16"]),
                out=rng.choice(["f32", "bf16", "fp8", "fp8"]), post=rng.choice(["none", "layer", "rms"]),
                pre=rng.choice(["layer", "rms"]), batch=rng.randint(1, 8), weights=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ shared inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV) * scale


def _blocks(k):
    return (k + BLOCK - 1) // BLOCK


def _scale_buffer(rows, k):
    """Scale bytes of `rows` rows or row blocks; row strides are multiples of 4."""
    return torch.full((rows, (_blocks(k) + 3) // 4 * 4), 127, dtype=torch.uint8, device=DEV)


def _scales(buf, k):
    """The scales that a buffer holds, as the values that they stand for."""
    return buf.view(torch.float8_e8m0fnu)[:, :_blocks(k)]


def _offsets(case):
    """Rows of each sample: ragged, as quotas leave them."""
    b, n = case["batch"], case["rows"]
    return [n * (i * (i + 3)) // (b * (b + 3)) for i in range(b + 1)]


def _quantise(x, block_rows):
    """(e4m3 values [R][K], scale exponents int32 [ceil(R / block_rows)][ceil(K / 128)]) of float32 rows: the smallest
    power of two 2^e, e in [-126, 127], with |x| <= 448 * 2^e over the block; x / 2^e rounded to nearest even."""
    r, k = x.shape
    rb, kb = (r + block_rows - 1) // block_rows, _blocks(k)
    p = torch.nn.functional.pad(x, (0, kb * BLOCK - k, 0, rb * block_rows - r)).view(rb, block_rows, kb, BLOCK)
    amax = p.abs().amax(dim=(1, 3))
    m, e = torch.frexp(amax)                       # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(amax == 0, -126, e).clamp(-126, 127).to(torch.int32)
    inv = ((127 - e) << 23).view(torch.float32)    # 2^-e
    q = (p * inv[:, None, :, None]).reshape(rb * block_rows, kb * BLOCK)[:r, :k]
    return q.to(torch.float8_e4m3fn).contiguous(), e


def _expand(e, rows, k, block_rows):
    """2^e for each element."""
    s = ((e + 127) << 23).view(torch.float32)
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :k]


def _gelu(x):
    u = 0.7978845608028654 * (x + 0.044715 * x * x * x)
    return x / (1.0 + torch.exp(-2.0 * u))


# ------------------------------------------------------------------------------------------------------ prepare

def prepare(case, seed):
    g = _gen(seed)
    return {"gemm": _prepare_gemm, "quant": _prepare_quant, "norm": _prepare_norm}[case["kind"]](case, g)


def _gemm_inputs(case, g):
    """Float32 operands before their quantisation, and the rest of the call."""
    m, n, k = case["M"], case["N"], case["K"]
    if case["epi"] == "resid":       # the rows that a GELU leaves
        a = _gelu(_randn(g, m, k, scale=0.64))
    else:                            # normed and modulated rows
        a = _randn(g, m, k) * (1.0 + _randn(g, k, scale=0.2)) + _randn(g, k, scale=0.2)
    out = dict(w=_randn(g, n, k, scale=0.02), a=a, bias=_randn(g, n, scale=0.02))
    if case["epi"] == "resid":
        out["h"] = _randn(g, m, n)
        out["gate"] = _randn(g, n, scale=0.5) if case["gate"] else None
    return out


def _prepare_gemm(case, g):
    s = _gemm_inputs(case, g)
    m, n, k = case["M"], case["N"], case["K"]
    out = dict(case=case, bias=s["bias"], gate=s.get("gate"), h=s.get("h"))
    for name, x, br in (("a", s["a"], 1), ("w", s["w"], BLOCK)):
        q, e = _quantise(x, br)
        buf = _scale_buffer(e.shape[0], k)
        buf[:, :e.shape[1]] = (e + 127).to(torch.uint8)
        out[name], out[name + "_scale"] = q, buf
    if case["epi"] == "gelu_fp8":
        out["out"] = torch.empty(m, n, dtype=TYPES["fp8"], device=DEV)
        out["out_scale"] = _scale_buffer(m, n)
    elif case["epi"] != "resid":
        out["out"] = torch.empty(m, n, dtype=TYPES["bf16"], device=DEV)
    return out


def _quant_input(case, g):
    if case["block_rows"] == 1:      # attention output: channels of different size
        x = _randn(g, case["rows"], case["K"], scale=0.3) * (1.0 + _randn(g, case["K"], scale=0.5).abs())
    else:
        x = _randn(g, case["rows"], case["K"], scale=0.02)
    return x.to(TYPES[case["dtype"]])


def _prepare_quant(case, g):
    r, k, br = case["rows"], case["K"], case["block_rows"]
    return dict(case=case, x=_quant_input(case, g), q=torch.empty(r, k, dtype=TYPES["fp8"], device=DEV),
                scale=_scale_buffer((r + br - 1) // br, k))


def _norm_inputs(case, g):
    r, d, b = case["rows"], case["d"], case["batch"]
    s = dict(h=_randn(g, r, d), y=_randn(g, r, d, scale=0.4).to(TYPES[case["dtype"]]), gate=_randn(g, b, d, scale=0.5),
             shift=_randn(g, b, d, scale=0.2), scale=_randn(g, b, d, scale=0.2))
    if case["weights"]:
        s.update(post_w=1.0 + _randn(g, d, scale=0.1), pre_w=1.0 + _randn(g, d, scale=0.1))
    return s


def _prepare_norm(case, g):
    r, d = case["rows"], case["d"]
    s = _norm_inputs(case, g)
    s.update(case=case, off=_offsets(case), out=torch.empty(r, d, dtype=TYPES[case["out"]], device=DEV))
    if case["out"] == "fp8":
        s["out_scale"] = _scale_buffer(r, d)
    return s


RESID_SCALE = 0.7071067811865476


# ---------------------------------------------------------------------------------------------------------- run

def run(s):
    return {"gemm": _run_gemm, "quant": _run_quant, "norm": _run_norm}[s["case"]["kind"]](s)


def _run_gemm(s):
    case, n = s["case"], s["case"]["N"]
    epi = case["epi"]
    if own:
        from paper_2511_22533_amd import f3c
        f3c.op_gemm_fp8(EPILOGUES[epi], s["a"], s["a_scale"], s["w"], s["w_scale"], s["bias"], out=s.get("out"),
                        out_scale=s.get("out_scale"), resid=s["h"], gate=s["gate"])
        if epi == "resid":
            return s["h"]
        return s["out"] if epi != "gelu_fp8" else {"q": s["out"], "scale": _scales(s["out_scale"], n)}
    m, k = case["M"], case["K"]
    kb = _blocks(k)
    a = s["a"].float() * _expand(s["a_scale"][:, :kb].int() - 127, m, k, 1)
    w = s["w"].float() * _expand(s["w_scale"][:, :kb].int() - 127, n, k, BLOCK)
    v = a @ w.t() + s["bias"]
    if epi == "resid":
        s["h"] += v if s["gate"] is None else s["gate"] * v
        return s["h"]
    if epi == "store":
        return v.to(TYPES["bf16"])
    v = _gelu(v)
    if epi == "gelu":
        return v.to(TYPES["bf16"])
    q, e = _quantise(v, 1)
    return {"q": q, "scale": (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)}


def _run_quant(s):
    case = s["case"]
    if own:
        from paper_2511_22533_amd import f3c
        f3c.op_quant_fp8(f3c.F3C_BF16 if case["dtype"] == "bf16" else f3c.F3C_F32, s["x"], s["q"], s["scale"],
                         block_rows=case["block_rows"])
        return {"q": s["q"], "scale": _scales(s["scale"], case["K"])}
    q, e = _quantise(s["x"].float(), case["block_rows"])
    return {"q": q, "scale": (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)}


def _norm(x, kind, eps):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    return x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + eps)


def _run_norm(s):
    case = s["case"]
    if own:
        from paper_2511_22533_amd import f3c
        codes = {"f32": f3c.F3C_F32, "bf16": f3c.F3C_BF16, "fp8": f3c.F3C_FP8}
        f3c.op_resid_norm(codes[case["dtype"]], codes[case["out"]], s["h"], y=s["y"], off=s["off"], out=s["out"],
                          out_scale=s.get("out_scale"), post=NORMS[case["post"]], pre=NORMS[case["pre"]],
                          post_w=s.get("post_w") if case["post"] != "none" else None, pre_w=s.get("pre_w"),
                          gate=s["gate"], resid_scale=RESID_SCALE, shift=s["shift"], scale=s["scale"])
        out = {"h": s["h"], "out": s["out"]}
        return dict(out, scale=_scales(s["out_scale"], case["d"])) if case["out"] == "fp8" else out
    rows = torch.tensor([b - a for a, b in zip(s["off"], s["off"][1:])], device=DEV)
    each = lambda v: v.repeat_interleave(rows, 0, output_size=case["rows"])  # noqa: E731
    p = _norm(s["y"].float(), case["post"], 1e-6)
    if case["weights"] and case["post"] != "none":
        p = p * s["post_w"]
    s["h"] += RESID_SCALE * (each(s["gate"]) * p)
    u = _norm(s["h"], case["pre"], 1e-6)
    if case["weights"]:
        u = u * s["pre_w"]
    u = u * (1.0 + each(s["scale"])) + each(s["shift"])
    if case["out"] != "fp8":
        return {"h": s["h"], "out": u.to(TYPES[case["out"]])}
    q, e = _quantise(u, 1)
    return {"h": s["h"], "out": q, "scale": (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)}


# --------------------------------------------------------------------------------------------------------- work

def work(case):
    if case["kind"] == "gemm":
        m, n, k = case["M"], case["N"], case["K"]
        b = m * (k + _blocks(k)) + n * k + _blocks(n) * _blocks(k) + 4 * n
        b += {"store": 2 * m * n, "gelu": 2 * m * n, "resid": 8 * m * n, "gelu_fp8": m * (n + _blocks(n))}[case["epi"]]
        return {"bytes": b, "flops": 2 * m * n * k}
    size = {"f32": 4, "bf16": 2, "fp8": 1}
    if case["kind"] == "quant":
        r, k = case["rows"], case["K"]
        return {"bytes": r * k * (size[case["dtype"]] + 1), "flops": 3 * r * k}
    r, d = case["rows"], case["d"]
    return {"bytes": r * d * (size[case["dtype"]] + 8 + size[case["out"]]), "flops": 16 * r * d}


# -------------------------------------------------------------------------------------------------------- exact

def _pow2(e):
    """2^e in float64 for whole e in -1022..1023 (pow() need not be exact, and values lie on rounding borders)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_quantise(x, block_rows):
    """Values and scales of the definition, for float64 rows."""
    r, k = x.shape
    rb, kb = -(-r // block_rows), -(-k // BLOCK)
    big = torch.zeros(rb * block_rows, kb * BLOCK, dtype=torch.float64, device=x.device)
    big[:r, :k] = x
    big = big.view(rb, block_rows, kb, BLOCK)
    ratio = big.abs().amax(dim=(1, 3)) / 448.0
    m, e = torch.frexp(ratio)
    e = torch.where(m == 0.5, e - 1, e).clamp(-126, 127)          # 2^e >= ratio, the smallest such
    e = torch.where(ratio == 0, torch.full_like(e, -126), e)
    y = big * _pow2(-e)[:, None, :, None]
    m, ex = torch.frexp(y.abs())
    step = _pow2((ex - 1).clamp(min=-6) - 3)
    q = (torch.round(y / step) * step).reshape(rb * block_rows, kb * BLOCK)[:r, :k]
    return q, _pow2(e)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "gemm":
        a, w = s["a"].double(), s["w"].double()
        for x, b, br in ((a, s["a_scale"], 1), (w, s["w_scale"], BLOCK)):
            k = _pow2(b.int() - 127)
            rows, cols = torch.arange(x.shape[0], device=DEV) // br, torch.arange(x.shape[1], device=DEV) // BLOCK
            x *= k[rows][:, cols]
        v = torch.matmul(a, w.t()) + s["bias"].double()
        if case["epi"] == "resid":
            return s["h"].double() + (v if s["gate"] is None else v * s["gate"].double())
        if case["epi"] == "store":
            return v
        v = 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
        if case["epi"] == "gelu":
            return v
        q, scale = _exact_quantise(v, 1)
        return {"q": q, "scale": scale}
    if case["kind"] == "quant":
        q, scale = _exact_quantise(s["x"].double(), case["block_rows"])
        return {"q": q, "scale": scale}
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and k in ("h", "y", "gate", "shift", "scale", "post_w",
                                                                             "pre_w")}
    h, u = d["h"], torch.empty_like(d["h"])

    def normed(x, kind, weight):
        if kind == "none":
            return x
        if kind == "layer":
            x = (x - x.mean(1, keepdim=True)) * torch.rsqrt(x.var(1, unbiased=False, keepdim=True) + 1e-6)
        else:
            x = x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6)
        return x if weight is None else x * weight

    for b, (lo, hi) in enumerate(zip(s["off"], s["off"][1:])):
        h[lo:hi] += RESID_SCALE * d["gate"][b] * normed(d["y"][lo:hi], case["post"], d.get("post_w"))
        u[lo:hi] = normed(h[lo:hi], case["pre"], d.get("pre_w")) * (1.0 + d["scale"][b]) + d["shift"][b]
    if case["out"] != "fp8":
        return {"h": h, "out": u}
    q, scale = _exact_quantise(u, 1)
    return {"h": h, "out": q, "scale": scale}
