"""Performance cases of a transformer block on 8-bit integers with its keys and values held in 8 bits: the
quantisation of rows, integer products with a scale for each token and channel, the cache that keys and values are
appended to, and attention over it.

What a program asks of the library when it holds the keys and values of a trajectory or a sequence in 8 bits: rows and
weights as whole numbers with a float32 scale each, projections of them with the epilogues of the step (store, GELU,
gated residual), pages of 64 tokens as e4m3 values with one power-of-two scale for each page and head, and queries that
attend over the pages of their sample: one new token, a chunk of them, or all active tokens of a step. Shapes follow the
measured workloads: width 1024, 16 heads of 64, ratio-4 MLP, 1374 condition tokens, 32768 tokens of which 9831 are
active; and generic ones with shared key heads.

All inputs are drawn on the GPU from the case's seed. The plain forms are elementary float32 operations; exact() is
written from the definitions in float64.
"""
import math

import torch

own = False

DEV = "cuda"
PAGE = 64
EPILOGUES = {"store": 0, "gelu": 1, "resid": 2}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
F8 = torch.float8_e4m3fn


def listed():
    return [
        # The attention output of a cached 32^3 step, quantised for its output projection.
        dict(name="quant_cached32", kind="quant", rows=9831, K=1024, dtype="bf16"),
        # A second MLP weight as it is loaded, a scale for each output channel; a width that fills no wave evenly.
        dict(name="quant_weight", kind="quant", rows=1320, K=5288, dtype="f32"),
        # One token through a first MLP projection: nothing but latency and the weights' way from HBM.
        dict(name="gemm_one_row", kind="gemm", M=1, N=4096, K=1024, epi="gelu", gate=False),
        # Sizes that fit no tile, into gated residual rows: ragged rows, columns and a last K tile of 16.
        dict(name="gemm_odd_resid", kind="gemm", M=1237, N=1328, K=1424, epi="resid", gate=True),
        # The first MLP projection of a full 32^3 step.
        dict(name="gemm_full32_fc1", kind="gemm", M=32768, N=4096, K=1024, epi="gelu", gate=False),
        # Keys and values of four samples' condition tokens into empty caches.
        dict(name="append_cond_b4", kind="append", dtype="bf16", batch=4, kv_heads=16, hd=64, len=0, new=1374),
        # One new token of each of 32 sequences, at ragged places of their last pages.
        dict(name="append_one_token", kind="append", dtype="bf16", batch=32, kv_heads=8, hd=128, len=4096, new=1),
        # One query over one sample's condition tokens: latency.
        dict(name="attn_one_token", kind="attn", batch=1, heads=16, kv_heads=16, hd=64, len=1374, nq=1, causal=False),
        # The newest token of each of 32 sequences, four query heads to a key head: the cache's way from HBM.
        dict(name="attn_decode_b32", kind="attn", batch=32, heads=32, kv_heads=8, hd=128, len=16384, nq=1, causal=True),
        # Chunks of new tokens behind what three sequences hold already, ragged ends.
        dict(name="attn_chunk_b3", kind="attn", batch=3, heads=16, kv_heads=4, hd=128, len=5003, nq=1021, causal=True),
        # Cross-attention of a full 32^3 step.
        dict(name="attn_cross32", kind="attn", batch=1, heads=16, kv_heads=16, hd=64, len=1374, nq=32768, causal=False),
        # The active tokens of a cached 32^3 step over the cached keys and values of all tokens.
        dict(name="attn_active32", kind="attn", batch=1, heads=16, kv_heads=16, hd=64, len=32768, nq=9831, causal=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quant", "gemm", "gemm", "gemm", "append", "append", "attn", "attn", "attn", "attn"])
    if kind == "quant":
        return dict(kind=kind, rows=_log(rng, 1, 32768), K=8 * _log(rng, 4, 1024), dtype=rng.choice(["f32", "bf16"]))
    if kind == "gemm":
        n, k = 16 * _log(rng, 8, 512), 16 * _log(rng, 8, 512)
        m = _log(rng, 1, max(2, min(32768, (1 << 37) // (n * k))))
        epi = rng.choice(sorted(EPILOGUES))
        return dict(kind=kind, M=m, N=n, K=k, epi=epi, gate=epi == "resid" and rng.random() < 0.7)
    hd, kv = rng.choice([32, 64, 64, 128]), rng.choice([1, 2, 4, 5, 8, 16])
    batch, wide = _log(rng, 1, 32), kv * hd
    if kind == "append":
        most = (1 << 28) // (batch * wide)
        return dict(kind=kind, dtype=rng.choice(["f32", "bf16", "bf16"]), batch=batch, kv_heads=kv, hd=hd,
                    len=rng.choice([0, _log(rng, 1, min(8192, most))]),
                    new=rng.choice([1, _log(rng, 2, min(4096, most))]))
    group, n = rng.choice([1, 1, 2, 4, 7]), _log(rng, 1, min(32768, (1 << 29) // (batch * wide)))
    # neither more scores nor more query values than the larger listed cases have
    most = min(8192, (1 << 31) // (batch * n * kv * group), (1 << 26) // (batch * wide * group))
    nq = 1 if rng.random() < 0.4 or most < 3 else _log(rng, 2, most)
    return dict(kind=kind, batch=batch, heads=kv * group, kv_heads=kv, hd=hd, len=n, nq=nq, causal=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ shared inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV) * scale


def _quantise_rows(x):
    """(whole numbers int8, scales float32) of rows: amax / 127 rounded to float32, at least 2^-126; the nearest whole
    number of x / scale, ties to even. In 64 bits: quotients lie next to borders."""
    amax = x.abs().amax(dim=1).double()
    s = (amax / torch.full_like(amax, 127.0)).float().clamp(min=2.0 ** -126)
    return torch.round(x.double() / s.double()[:, None]).to(torch.int8), s


def _exponent(amax):
    """The smallest e in [-126, 127] with amax <= 448 * 2^e, int32."""
    m, e = torch.frexp(amax)                       # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.where(amax == 0, -126, e).clamp(-126, 127).to(torch.int32)


def _pow2_f32(e):
    return ((e + 127) << 23).view(torch.float32)


def _byte(e):
    return (e + 127).to(torch.uint8)


def _slot(t):
    """Where a page's values hold token t (0..63) of the page: the order in which the matrix cores take them."""
    return 16 * ((t // 4) % 4) + 4 * (t // 16) + t % 4


def _lens(case):
    """Tokens that each sample's cache holds: ragged, the first one all of them."""
    b, n = case["batch"], case["len"]
    return [n - 5 * n * i // (8 * b) for i in range(b)]


def _new(case, key):
    """Row offsets of each sample's new tokens or queries: ragged, but for single ones."""
    off = [0]
    for i in range(case["batch"]):
        off.append(off[-1] + case[key] - case[key] * i // (2 * case["batch"]))
    return off


def _table(g, pages):
    """Pages of each sample, int32 [B][most], drawn from one pool without order; and the pool's size. Entries behind a
    sample's last page name no page (-1)."""
    most, n = max(pages), sum(pages) + 3
    order = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    count = torch.tensor(pages, device=DEV)
    at = (torch.cumsum(count, 0) - count)[:, None] + torch.arange(most, device=DEV)
    used = torch.arange(most, device=DEV) < count[:, None]
    return torch.where(used, order[at.clamp(max=n - 1)], -1).to(torch.int32).contiguous(), n


def _pool(g, n_pages, heads, hd, transposed, chunk=2048):
    """Quantised pages and their scale bytes: K [n][heads][64][hd], V [n][heads][hd][64]; channels of different size and
    mean, pages of different size."""
    shape = (hd, PAGE) if transposed else (PAGE, hd)
    size, mean = 0.5 + _randn(g, heads, hd, scale=0.3).abs(), _randn(g, heads, hd, scale=0.3)
    size, mean = (t[:, :, None] if transposed else t[:, None, :] for t in (size, mean))
    q = torch.empty(n_pages, heads, *shape, dtype=F8, device=DEV)
    scale = torch.empty(n_pages, heads, dtype=torch.uint8, device=DEV)
    for i in range(0, n_pages, chunk):
        m = min(chunk, n_pages - i)
        x = (_randn(g, m, heads, *shape) * size + mean) * torch.exp2(torch.rand(m, heads, 1, 1, generator=g, device=DEV))
        e = _exponent(x.abs().amax(dim=(2, 3)))
        q[i:i + m] = (x * _pow2_f32(-e)[:, :, None, None]).to(F8)
        scale[i:i + m] = _byte(e)
    return q, scale


# ------------------------------------------------------------------------------------------------------ prepare

def prepare(case, seed):
    g = _gen(seed)
    make = {"quant": _prepare_quant, "gemm": _prepare_gemm, "append": _prepare_append, "attn": _prepare_attn}
    return dict(make[case["kind"]](case, g), case=case)


def _prepare_quant(case, g):
    r, k = case["rows"], case["K"]
    x = _randn(g, r, k, scale=0.3) * (1.0 + _randn(g, k, scale=0.5).abs())
    return dict(x=x.to(TYPES[case["dtype"]]), q=torch.empty(r, k, dtype=torch.int8, device=DEV),
                scale=torch.empty(r, dtype=torch.float32, device=DEV))


def _gelu(x):
    u = 0.7978845608028654 * (x + 0.044715 * x * x * x)
    return x / (1.0 + torch.exp(-2.0 * u))


def _prepare_gemm(case, g):
    m, n, k = case["M"], case["N"], case["K"]
    if case["epi"] == "resid":       # the rows that a GELU leaves
        a = _gelu(_randn(g, m, k, scale=0.64))
    else:                            # normed and modulated rows
        a = _randn(g, m, k) * (1.0 + _randn(g, k, scale=0.2)) + _randn(g, k, scale=0.2)
    s = dict(bias=_randn(g, n, scale=0.02))
    s["a"], s["a_scale"] = _quantise_rows(a)
    s["w"], s["w_scale"] = _quantise_rows(_randn(g, n, k, scale=0.02))
    if case["epi"] == "resid":
        s["h"] = _randn(g, m, n)
        s["gate"] = _randn(g, n, scale=0.5) if case["gate"] else None
    else:
        s["out"] = torch.empty(m, n, dtype=TYPES["bf16"], device=DEV)
    return s


def _prepare_append(case, g):
    lens, off = _lens(case), _new(case, "new")
    held = [(n + b - a + PAGE - 1) // PAGE for n, a, b in zip(lens, off, off[1:])]
    table, n_pages = _table(g, held)
    h, hd, t = case["kv_heads"], case["hd"], TYPES[case["dtype"]]
    k, k_scale = _pool(g, n_pages, h, hd, False)
    v, v_scale = _pool(g, n_pages, h, hd, True)
    rows = lambda: (_randn(g, off[-1], h * hd) * (0.5 + _randn(g, h * hd, scale=0.7).abs())).to(t)  # noqa: E731
    return dict(cache=(k, v, k_scale, v_scale, table), lens=lens, off=off, k=rows(), v=rows())


def _prepare_attn(case, g):
    lens, off = _lens(case), _new(case, "nq")
    table, n_pages = _table(g, [(n + PAGE - 1) // PAGE for n in lens])
    h, hd = case["kv_heads"], case["hd"]
    k, k_scale = _pool(g, n_pages, h, hd, False)
    v, v_scale = _pool(g, n_pages, h, hd, True)
    # what a page holds behind a sample's last token was never written: NaN here
    t = torch.arange(PAGE, device=DEV)
    n = torch.tensor(lens, device=DEV)
    last = table[torch.arange(len(lens), device=DEV), (n - 1) // PAGE].long()
    empty = torch.arange(PAGE, device=DEV) > ((n - 1) % PAGE)[:, None]
    k[last] = torch.where(empty[:, None, :, None], math.nan, k[last].float()).to(F8)
    by_slot = torch.empty_like(empty)
    by_slot[:, _slot(t)] = empty
    v[last] = torch.where(by_slot[:, None, None, :], math.nan, v[last].float()).to(F8)
    q = _randn(g, off[-1], case["heads"] * hd, scale=1.3).to(TYPES["bf16"])
    return dict(cache=(k, v, k_scale, v_scale, table), lens=lens, off=off, q=q, o=torch.empty_like(q))


# ---------------------------------------------------------------------------------------------------------- run

def run(s):
    return {"quant": _run_quant, "gemm": _run_gemm, "append": _run_append, "attn": _run_attn}[s["case"]["kind"]](s)


def _run_quant(s):
    if own:
        from paper_2511_22533_amd import f3c
        f3c.op_quant_i8(f3c.F3C_BF16 if s["case"]["dtype"] == "bf16" else f3c.F3C_F32, s["x"], s["q"], s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    q, scale = _quantise_rows(s["x"].float())
    return {"q": q, "scale": scale}


def _run_gemm(s):
    epi = s["case"]["epi"]
    if own:
        from paper_2511_22533_amd import f3c
        f3c.op_gemm_i8(EPILOGUES[epi], s["a"], s["a_scale"], s["w"], s["w_scale"], s["bias"], out=s.get("out"),
                       resid=s.get("h"), gate=s.get("gate"))
        return s["h"] if epi == "resid" else s["out"]
    v = (s["a"].float() @ s["w"].float().t()) * s["w_scale"] * s["a_scale"][:, None] + s["bias"]
    if epi == "resid":
        s["h"] += v if s["gate"] is None else s["gate"] * v
        return s["h"]
    return (_gelu(v) if epi == "gelu" else v).to(TYPES["bf16"])


def _cache(s):
    k, v, k_scale, v_scale, _ = s["cache"]
    e8 = torch.float8_e8m0fnu
    return {"k": k, "v": v, "k_scale": k_scale.view(e8), "v_scale": v_scale.view(e8)}


def _run_append(s):
    case = s["case"]
    if own:
        from paper_2511_22533_amd import f3c
        f3c.op_cache8_append(f3c.F3C_BF16 if case["dtype"] == "bf16" else f3c.F3C_F32, f3c.Cache8(*s["cache"]),
                             s["lens"], s["off"], s["k"], s["v"])
        return _cache(s)
    h, hd, table = case["kv_heads"], case["hd"], s["cache"][4].long()
    lens, off = torch.tensor(s["lens"], device=DEV), torch.tensor(s["off"], device=DEV)
    row = torch.arange(s["off"][-1], device=DEV)
    sample = torch.searchsorted(off, row, right=True) - 1
    pos = lens[sample] + row - off[sample]
    page, slot = table[sample, pos // PAGE], pos % PAGE
    # pages that hold tokens of before, one at most for a sample, and how many each
    begun = torch.tensor([b for b, n in enumerate(s["lens"]) if n % PAGE], dtype=torch.long, device=DEV)
    part = (lens % PAGE)[begun, None]
    old = table[begun, lens[begun] // PAGE]
    for x, pool, scale, transposed in ((s["k"], s["cache"][0], s["cache"][2], False),
                                       (s["v"], s["cache"][1], s["cache"][3], True)):
        x = x.float().view(-1, h, hd)
        amax = torch.zeros(pool.shape[0], h, device=DEV)
        amax.scatter_reduce_(0, page[:, None].expand(-1, h), x.abs().amax(dim=2), "amax")
        e = _exponent(amax)
        was = scale[old].int() - 127
        e[old] = torch.maximum(e[old], was)
        t = torch.arange(PAGE, device=DEV)
        keep = torch.empty(old.shape[0], PAGE, dtype=torch.bool, device=DEV)
        keep[:, _slot(t) if transposed else t] = t < part
        held = pool[old].float()
        moved = (held * _pow2_f32(was - e[old])[:, :, None, None]).to(F8).float()
        shape = (-1, 1, 1, PAGE) if transposed else (-1, 1, PAGE, 1)
        pool[old] = torch.where(keep.view(shape), moved, held).to(F8)
        q = (x * _pow2_f32(-e[page])[:, :, None]).to(F8).view(torch.uint8)
        if transposed:
            pool.view(torch.uint8)[page, :, :, _slot(slot)] = q
        else:
            pool.view(torch.uint8)[page, :, slot] = q
        scale[page] = _byte(e[page])
    return _cache(s)


def _run_attn(s):
    case = s["case"]
    if own:
        from paper_2511_22533_amd import f3c
        f3c.op_cache8_attention(f3c.Cache8(*s["cache"]), case["heads"], s["off"], s["lens"], s["q"], s["o"],
                                causal=case["causal"])
        return s["o"]
    k, v, k_scale, v_scale, table = s["cache"]
    b, kv, hd, heads = case["batch"], case["kv_heads"], case["hd"], case["heads"]
    grp, nq, n = heads // kv, case["nq"], table.shape[1] * PAGE
    lens, off = torch.tensor(s["lens"], device=DEV), torch.tensor(s["off"], device=DEV)
    rows = off[1:] - off[:-1]
    at = table.clamp(min=0).long()
    seen = torch.arange(n, device=DEV) < lens[:, None]
    # keys [B][kv][hd][n], values [B][kv][n][hd]; what no token has written counts as 0
    keys = (k[at].float() * _pow2_f32(k_scale[at].int() - 127)[..., None, None]).permute(0, 2, 4, 1, 3)
    keys = torch.where(seen[:, None, None, :], keys.reshape(b, kv, hd, n), 0.0)
    t = _slot(torch.arange(PAGE, device=DEV))
    vals = (v[at].float() * _pow2_f32(v_scale[at].int() - 127)[..., None, None])[..., t].permute(0, 2, 1, 4, 3)
    vals = torch.where(seen[:, None, :, None], vals.reshape(b, kv, n, hd), 0.0)
    i = torch.arange(nq, device=DEV)
    src = (off[:-1, None] + i).clamp(max=s["off"][-1] - 1)
    q = s["q"].float()[src].view(b, nq, kv, grp, hd).permute(0, 2, 3, 1, 4).reshape(b, kv, grp * nq, hd)
    p = torch.matmul(q, keys)
    p *= 1.0 / math.sqrt(hd)
    most = lens[:, None] - rows[:, None] + 1 + i if case["causal"] else lens[:, None].expand(b, nq)
    masked = torch.arange(n, device=DEV) >= torch.minimum(most, lens[:, None])[:, :, None]
    p.view(b, kv, grp, nq, n).masked_fill_(masked[:, None, None], -math.inf)
    top = p.amax(dim=3, keepdim=True)
    p -= torch.where(top == -math.inf, 0.0, top)
    p.exp_()
    total = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p, vals) / torch.where(total == 0, 1.0, total)
    o = o.view(b, kv, grp, nq, hd).permute(0, 3, 1, 2, 4).reshape(b, nq, heads * hd)
    return o[i < rows[:, None]].to(TYPES["bf16"])


# --------------------------------------------------------------------------------------------------------- work

def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["kind"] == "quant":
        r, k = case["rows"], case["K"]
        return {"bytes": r * k * (size[case["dtype"]] + 1) + 4 * r, "flops": 3 * r * k}
    if case["kind"] == "gemm":
        m, n, k = case["M"], case["N"], case["K"]
        return {"bytes": m * k + n * k + 4 * (m + 2 * n) + m * n * (8 if case["epi"] == "resid" else 2),
                "flops": 2 * m * n * k}
    h, hd, lens = case["kv_heads"], case["hd"], _lens(case)
    if case["kind"] == "append":
        n = _new(case, "new")[-1] * h * hd * 2
        return {"bytes": n * (size[case["dtype"]] + 1), "flops": 3 * n}
    off = _new(case, "nq")
    pairs = 0
    for n, rows in zip(lens, (y - x for x, y in zip(off, off[1:]))):
        most = min(rows, n)
        pairs += most * (2 * n - most + 1) // 2 if case["causal"] else rows * n
    return {"bytes": 2 * sum(lens) * h * hd + 4 * off[-1] * case["heads"] * hd,
            "flops": 4 * pairs * case["heads"] * hd}


# -------------------------------------------------------------------------------------------------------- exact

def _pow2(e):
    """2^e in float64 for whole e in -1022..1023 (pow() need not be exact, and values lie on rounding borders)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e4m3(y):
    """float64 values rounded to e4m3, as float64."""
    _, ex = torch.frexp(y.abs())
    step = _pow2((ex - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step




def exact(case, seed):
    s = prepare(case, seed)
    return {"quant": _exact_quant, "gemm": _exact_gemm, "append": _exact_append, "attn": _exact_attn}[case["kind"]](s)


def _exact_quant(s):
    x = s["x"].double()
    scale = torch.maximum(x.max(1).values, -x.min(1).values) / torch.tensor(127.0, dtype=torch.float64, device=DEV)
    scale = scale.clamp(min=2.0 ** -126)
    q = x / scale.float().double().view(-1, 1)
    lo = torch.floor(q)
    up = (q - lo > 0.5) | ((q - lo == 0.5) & (lo % 2 != 0))
    return {"q": (lo + up).to(torch.int8), "scale": scale}


def _exact_gemm(s):
    a = s["a"].double() * s["a_scale"].double().view(-1, 1)
    w = s["w"].double() * s["w_scale"].double().view(-1, 1)
    v = torch.matmul(a, w.t()).add_(s["bias"].double())
    if s["case"]["epi"] == "resid":
        return s["h"].double() + (v if s["gate"] is None else v * s["gate"].double())
    if s["case"]["epi"] == "gelu":
        v = 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    return v


def _exact_append(s):
    case, (k, v, k_scale, v_scale, table) = s["case"], s["cache"]
    h, hd, table = case["kv_heads"], case["hd"], table.tolist()
    if case["batch"] * case["new"] * h > 400000:
        return None
    out = {"k": k.double(), "v": v.double(), "k_scale": _pow2(k_scale.int() - 127), "v_scale": _pow2(v_scale.int() - 127)}
    for name in ("k", "v"):
        pool, scale, src = out[name], out[name + "_scale"], s[name].double().view(-1, h, hd)
        for b, n in enumerate(s["lens"]):
            lo, hi = s["off"][b], s["off"][b + 1]
            while lo < hi:
                page, at = table[b][n // PAGE], n % PAGE
                m = min(PAGE - at, hi - lo)
                idx = torch.arange(PAGE, device=DEV)
                idx = _slot(idx) if name == "v" else idx
                tile = pool[page].transpose(1, 2)[:, idx] if name == "v" else pool[page][:, idx]   # [h][token][hd]
                fresh = src[lo:lo + m].transpose(0, 1)
                # (over all heads at once: the exponent as the smallest whole number at or above log2, on exact borders)
                ratio = fresh.abs().amax(dim=(1, 2)) / 448.0
                mant, e = torch.frexp(ratio)
                e = torch.where(ratio == 0, torch.full_like(e, -126), torch.where(mant == 0.5, e - 1, e)).clamp(-126, 127)
                if at:
                    was = torch.frexp(scale[page])[1] - 1
                    e = torch.maximum(e, was.to(e.dtype))
                    tile[:, :at] = _e4m3(tile[:, :at] * _pow2(was - e)[:, None, None])
                tile[:, at:at + m] = _e4m3(fresh * _pow2(-e)[:, None, None])
                if name == "v":
                    pool[page][:, :, idx] = tile.transpose(1, 2)
                else:
                    pool[page] = tile
                scale[page] = _pow2(e)
                lo, n = lo + m, n + m
    return out


def _exact_attn(s):
    case, (k, v, k_scale, v_scale, table) = s["case"], s["cache"]
    kv, hd, heads = case["kv_heads"], case["hd"], case["heads"]
    if case["batch"] * heads > 2048:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    order = [16 * (t // 4 % 4) + 4 * (t // 16) + t % 4 for t in range(PAGE)]
    for b, n in enumerate(s["lens"]):
        lo, hi = s["off"][b], s["off"][b + 1]
        pages = table[b, :(n + PAGE - 1) // PAGE].long()
        for g in range(kv):
            key = k[pages, g].double() * _pow2(k_scale[pages, g].int() - 127)[:, None, None]
            val = v[pages, g].double() * _pow2(v_scale[pages, g].int() - 127)[:, None, None]
            key = key.reshape(-1, hd)[:n]
            val = val[:, :, order].transpose(1, 2).reshape(-1, hd)[:n]
            for c in range(g * (heads // kv), (g + 1) * (heads // kv)):
                cols = slice(c * hd, (c + 1) * hd)
                z = torch.matmul(s["q"][lo:hi, cols].double(), key.t()) / math.sqrt(hd)
                if case["causal"]:
                    i = torch.arange(hi - lo, device=DEV)[:, None]
                    z = torch.where(torch.arange(n, device=DEV) <= n - (hi - lo) + i, z, -math.inf)
                out[lo:hi, cols] = torch.nan_to_num(torch.softmax(z, dim=1)) @ val
    return out
