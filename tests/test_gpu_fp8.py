"""GPU parity of the 8-bit operators, through the C ABI, against the float64 oracle (oracle/fp8.py).

* quantisation bit for bit: codes and scale bytes, rows and weights, ragged blocks, strides, zeros, NaN, infinities and
  values down to the smallest subnormal;
* products against float64 on the same quantised operands, each output within what the matrix core's sums can be off
  (below) and one rounding of the output; an output row's bits do not depend on the number of rows;
* the pass between two blocks, every pair of norms and each type; and a whole MLP sublayer of the three together.
"""
import numpy as np
import pytest

from helpers import say, to_dev
from oracle import fp8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    from paper_2511_22533_amd import f3c
    f3c.lib()
    return t


@pytest.fixture(scope="module")
def f3c(torch):
    from paper_2511_22533_amd import f3c as m
    return m


def _rows(torch, rows, cols, dtype, pad=0, fill=0):
    """A [rows][cols] view with row stride cols + pad (of a buffer filled with `fill`, one row longer)."""
    buf = torch.full((rows + 1, cols + pad), fill, dtype=torch.float32, device="cuda").to(dtype)
    return buf, buf[:rows, :cols]


def _u8(torch, a, pad=0):
    """uint8 array on the GPU, row stride its length + pad; the padding holds 0xff (NaN as value and as scale)."""
    buf = torch.full((a.shape[0], a.shape[1] + pad), 255, dtype=torch.uint8, device="cuda")
    buf[:, :a.shape[1]] = to_dev(a)
    return buf[:, :a.shape[1]]


def _scale_dev(torch, f3c, a, cols):
    """Scale bytes with the row stride that the operators ask for, 0xff in its padding."""
    buf = torch.full((a.shape[0], f3c.fp8_scale_stride(cols)), 255, dtype=torch.uint8, device="cuda")
    buf[:, :a.shape[1]] = to_dev(a)
    return buf


# ------------------------------------------------------------------------------------------------- quantisation

def _quant_input(rows, K, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, K)) * np.exp(rng.uniform(-12, 12, size=(rows, 1)))
    x = x.astype(np.float32)
    x[:, :: 17] = 0.0
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K,br,pad", [(1, 8, 1, 0), (1, 1024, 1, 0), (3, 128, 1, 8), (5, 136, 1, 24),
                                           (67, 520, 1, 0), (9, 4096, 1, 0), (1000, 1000, 1, 8), (1, 8, 128, 0), (128, 128, 128, 0),
                                           (129, 136, 128, 8), (300, 1000, 128, 16), (1024, 512, 128, 0)])
def test_quant_bit_exact(torch, f3c, dtype, rows, K, br, pad):
    say("quant", dtype, rows, K, br, pad)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    _, x = _rows(torch, rows, K, t, pad)
    x.copy_(to_dev(_quant_input(rows, K, rows + K)))
    want_q, want_s = fp8.quantise(x.float().cpu().numpy(), br)
    qbuf, q = _rows(torch, rows, K, torch.float32, pad, 7)
    qbuf = qbuf.to(torch.uint8)
    q = qbuf[:rows, :K]
    scale = torch.full(((rows + br - 1) // br + 1, f3c.fp8_scale_stride(K)), 77, dtype=torch.uint8, device="cuda")
    f3c.op_quant_fp8(f3c.F3C_F32 if dtype == "f32" else f3c.F3C_BF16, x, q, scale[:-1], block_rows=br)
    torch.cuda.synchronize()
    assert np.array_equal(scale.cpu().numpy()[:-1, :want_s.shape[1]], want_s)
    assert np.array_equal(q.cpu().numpy(), want_q)
    # what lies behind the rows, the columns and the scales is left alone
    assert bool((qbuf[rows:] == 7).all()) and bool((qbuf[:, K:] == 7).all())
    assert bool((scale[-1] == 77).all()) and bool((scale[:, want_s.shape[1]:] == 77).all())


@pytest.mark.parametrize("br", [1, 128])
def test_quant_extreme_values(torch, f3c, br):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((256, 512)).astype(np.float32)
    x[0, :128] = 0.0
    x[1, 3], x[1, 200], x[2, 5] = np.nan, np.inf, -np.inf
    x[3, :128] = np.nan
    x[4] = 3.4e38
    x[5] = 2.0 ** -149
    x[6] *= np.float32(1e-38)
    x[7, :8] = [448, -448, 449, 1e-3, 2.0 ** -10, 2.0 ** -9, -0.0, 0.0]
    x[8, 128:256] = 1.75 * 2.0 ** np.arange(-60, 68)
    x[9] = 1.0 + np.arange(512) / 4096
    x[10:140] *= np.float32(1e-30)
    codes, scale = fp8.quantise(x, br)
    d = to_dev(x)
    q = torch.empty(256, 512, dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.empty(256 // br, 4, dtype=torch.float8_e8m0fnu, device="cuda")
    say("quant extremes", br)
    f3c.op_quant_fp8(f3c.F3C_F32, d, q, s, block_rows=br)
    got = q.view(torch.uint8).cpu().numpy()
    bad = ~np.isfinite(x)
    assert np.array_equal(s.view(torch.uint8).cpu().numpy(), scale)
    assert np.array_equal(got[~bad], codes[~bad])
    assert np.all((got[bad] & 0x7F) == 0x7F)


# ------------------------------------------------------------------------------------------------------ products

def _operands(M, N, K, seed, spread=2.0):
    """Quantised operands whose blocks differ in size by powers of two, and their float64 values."""
    rng = np.random.default_rng(seed)
    kb = -(-K // 128)
    a = rng.standard_normal((M, K)) * np.repeat(2.0 ** rng.uniform(-spread, spread, (M, kb)), 128, 1)[:, :K]
    w = rng.standard_normal((N, K)) * np.repeat(2.0 ** rng.uniform(-spread, spread, (1, kb)), 128, 1)[:, :K]
    w /= np.sqrt(K)
    (aq, ascl), (wq, wscl) = fp8.quantise(a, 1), fp8.quantise(w, 128)
    bias = rng.standard_normal(N).astype(np.float32)
    return aq, ascl, wq, wscl, bias


def _sum_bound(a, w):
    """How far the matrix core's sum of a row of products can be off: of 8 products each loses less than 2^-13 of the
    largest, and each of the K / 8 additions to the float32 accumulator less than 2^-23 of the sum so far."""
    K = a.shape[1]
    A, W = np.abs(a), np.abs(w)
    tot, lost = np.zeros((A.shape[0], W.shape[0])), np.zeros((A.shape[0], W.shape[0]))
    for k in range(0, K, 8):
        p = [np.outer(A[:, i], W[:, i]) for i in range(k, k + 8)]
        lost += 8 * 2.0 ** -13 * np.maximum.reduce(p)
        tot += sum(p)
    return lost + (K / 8 + 2) * 2.0 ** -23 * tot


def _gemm(torch, f3c, epi, aq, ascl, wq, wscl, bias, M=None, pads=(0, 0, 0), resid=None, gate=None):
    K, N = aq.shape[1], wq.shape[0]
    M = aq.shape[0] if M is None else M
    A, W = _u8(torch, aq[:M], pads[0]), _u8(torch, wq, pads[1])
    sa, sw = _scale_dev(torch, f3c, ascl[:M], K), _scale_dev(torch, f3c, wscl, K)
    b = None if bias is None else to_dev(bias)
    if epi == 2:
        buf = torch.full((M + 1, N + pads[2]), 5.0, device="cuda")
        buf[:M, :N] = to_dev(resid[:M])
        f3c.op_gemm_fp8(2, A, sa, W, sw, b, resid=buf[:M, :N], gate=None if gate is None else to_dev(gate))
        out = buf
        left = 5.0
    else:
        t = torch.uint8 if epi == 3 else torch.bfloat16
        out = torch.full((M + 1, N + pads[2]), 5, device="cuda").to(t)
        so = torch.full((M + 1, f3c.fp8_scale_stride(N)), 9, dtype=torch.uint8, device="cuda") if epi == 3 else None
        f3c.op_gemm_fp8(epi, A, sa, W, sw, b, out=out[:M, :N], out_scale=so[:M] if epi == 3 else None)
        left = 5
    torch.cuda.synchronize()
    assert bool((out[M:] == left).all()) and bool((out[:, N:] == left).all())      # nothing behind rows and columns
    if epi == 3:
        nb = -(-N // 128)
        assert bool((so[M:] == 9).all()) and bool((so[:, nb:] == 9).all())
        return out[:M, :N].cpu().numpy(), so[:M, :nb].cpu().numpy()
    return out[:M, :N].float().cpu().numpy()


def _check_gemm(torch, f3c, epi, ops, pads=(0, 0, 0), gated=True, with_bias=True):
    aq, ascl, wq, wscl, bias = ops
    M, N = aq.shape[0], wq.shape[0]
    a, w = fp8.dequantise(aq, ascl, 1), fp8.dequantise(wq, wscl, 128)
    bias = bias if with_bias else None
    v = fp8.linear(a, w, bias)
    tol = _sum_bound(a, w) + 2.0 ** -23 * np.abs(v)
    rng = np.random.default_rng(M + N)
    if epi == 2:
        h = rng.standard_normal((M, N)).astype(np.float32)
        gate = rng.standard_normal(N).astype(np.float32) if gated else None
        got = _gemm(torch, f3c, 2, aq, ascl, wq, wscl, bias, pads=pads, resid=h, gate=gate)
        g = 1.0 if gate is None else gate
        want = h + g * v
        tol = np.abs(g) * tol + 2.0 ** -22 * (np.abs(h) + np.abs(g * v))
    elif epi == 0:
        got, want = _gemm(torch, f3c, 0, aq, ascl, wq, wscl, bias, pads=pads), v
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    else:
        # the slope of GELU is at most 1.13; its float32 evaluation is off by a few roundings, relative, with the
        # exponent's argument (at most 2 |u| log2 e, |u| < |v| (0.8 + 0.036 v^2)) rounded before the power is taken
        want = fp8.gelu(v)
        u = np.abs(v) * (0.8 + 0.036 * v * v)
        tol = 1.13 * tol + 2.0 ** -24 * (8 + 12 * u) * np.abs(want) + 1e-30
        got = _gemm(torch, f3c, epi, aq, ascl, wq, wscl, bias, pads=pads)
        if epi == 1:
            tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
        else:
            codes, scale = got
            wide = np.pad(np.abs(want), ((0, 0), (0, -N % 128))).reshape(M, -1, 128)
            far = np.pad(tol, ((0, 0), (0, -N % 128))).reshape(M, -1, 128)
            lo = [[fp8.block_exponent(x) for x in r] for r in np.maximum(wide - far, 0).max(axis=2)]
            hi = [[fp8.block_exponent(x) for x in r] for r in (wide + far).max(axis=2)]
            e = scale.astype(int) - 127
            assert np.all(e >= lo) and np.all(e <= hi)
            got = fp8.dequantise(codes, scale, 1)
            # half a step of e4m3, or of its subnormals, at the scale that was chosen
            tol = tol + np.maximum(2.0 ** -4 * (np.abs(want) + tol), 2.0 ** -10 * fp8.scales(scale, M, N, 1))
    err = np.abs(got - want)
    assert np.all(err <= tol), (epi, M, N, aq.shape[1], float(np.max(err / tol)))


SHAPES = [(1, 16, 16), (1, 128, 128), (1, 1024, 1024), (3, 144, 144), (17, 16, 2064), (33, 272, 400), (64, 128, 640),
          (70, 1040, 272), (130, 256, 1424), (257, 400, 512), (300, 512, 4096)]


@pytest.mark.parametrize("epi", [0, 1, 2, 3])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_against_float64(torch, f3c, epi, M, N, K):
    say("gemm_fp8", epi, M, N, K)
    _check_gemm(torch, f3c, epi, _operands(M, N, K, M + N + K))


@pytest.mark.parametrize("epi", [0, 1, 2, 3])
def test_gemm_strides_and_absent_operands(torch, f3c, epi):
    say("gemm_fp8 strides", epi)
    _check_gemm(torch, f3c, epi, _operands(77, 208, 336, 4), pads=(48, 16, 16), gated=False, with_bias=False)


@pytest.mark.parametrize("epi", [0, 2])
def test_gemm_scales_far_apart(torch, f3c, epi):
    """Blocks of very different size: each K block's scale is applied to its own products."""
    say("gemm_fp8 scales", epi)
    _check_gemm(torch, f3c, epi, _operands(40, 144, 1280, 6, spread=18.0))


@pytest.mark.parametrize("M,N,K", [(1, 128, 4112), (40, 144, 4240), (200, 272, 4112), (700, 528, 4112),
                                   (1, 128, 2064), (64, 1024, 4096), (300, 512, 2432), (2000, 1024, 4096)])
def test_gemm_residual_of_long_sums_is_exact(torch, f3c, M, N, K):
    """Beyond K = 2048 (4096 with a gate) the residual epilogue's products are exact and its sums float32: each of the
    K / 16 additions to the accumulator (and those within an instruction, 16 at a time) is off by 2^-23 at most of the
    sum of magnitudes."""
    say("gemm_fp8 wide", M, N, K)
    aq, ascl, wq, wscl, bias = _operands(M, N, K, 12)
    ascl[M // 2, 3], ascl[0, 1] = 255, 0                 # a NaN scale, and the smallest
    a, w = fp8.dequantise(aq, ascl, 1), fp8.dequantise(wq, wscl, 128)
    a[M // 2] = 0.0
    v, tot = fp8.linear(a, w, bias), np.abs(a) @ np.abs(w).T + np.abs(bias)
    h = np.random.default_rng(1).standard_normal((M, N)).astype(np.float32)
    got = _gemm(torch, f3c, 2, aq, ascl, wq, wscl, bias, resid=h)
    ok = np.arange(M) != M // 2
    assert np.isnan(got[M // 2]).all()
    tol = (K / 16 + 16) * 2.0 ** -23 * tot + 2.0 ** -22 * (np.abs(h) + np.abs(v))
    assert np.all(np.abs(got - (h + v))[ok] <= tol[ok])
    # and in the mean far below what 8-bit sums give (1e-5 of v)
    if M > 1:
        assert np.linalg.norm((got - h - v)[ok]) <= 2e-6 * np.linalg.norm(v[ok])


def test_gemm_bad_rows_stay_alone(torch, f3c):
    aq, ascl, wq, wscl, bias = _operands(50, 144, 400, 8)
    good = _gemm(torch, f3c, 0, aq, ascl, wq, wscl, bias)
    aq2, ascl2, wq2 = aq.copy(), ascl.copy(), wq.copy()
    aq2[7, 33], ascl2[20, 1], wq2[100, 399] = 0x7F, 255, 0xFF          # NaN value, NaN scale, NaN weight
    say("gemm_fp8 NaN")
    got = _gemm(torch, f3c, 0, aq2, ascl2, wq2, wscl, bias)
    bad = np.zeros_like(good, bool)
    bad[7], bad[20], bad[:, 100] = True, True, True
    assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], good[~bad])
    # a NaN in front of the quantising epilogue: NaN there, and its block's scale from the other values
    codes, scale = _gemm(torch, f3c, 3, aq, ascl, wq2, wscl, bias)
    assert np.all((codes[:, 100] & 0x7F) == 0x7F)
    rest = np.delete(codes, 100, axis=1)
    assert not np.any((rest & 0x7F) == 0x7F) and scale.max() < 160


@pytest.mark.parametrize("N,K", [(1024, 1024), (1024, 4096), (4096, 1024), (400, 1424), (512, 4112)])
def test_gemm_rows_do_not_depend_on_their_number(torch, f3c, N, K):
    """Other row counts take other kernels and tiles; each output is the same sum in the same order."""
    rng = np.random.default_rng(N + K)
    top = 5000
    a = rng.standard_normal((top, K)) * np.repeat(2.0 ** rng.uniform(-6, 6, (top, -(-K // 128))), 128, 1)[:, :K]
    A = torch.empty(top, K, dtype=torch.uint8, device="cuda")
    sa = torch.empty(top, f3c.fp8_scale_stride(K), dtype=torch.uint8, device="cuda")
    f3c.op_quant_fp8(f3c.F3C_F32, to_dev(a.astype(np.float32)), A, sa)
    w = to_dev((rng.standard_normal((N, K)) / 32).astype(np.float32))
    W = torch.empty(N, K, dtype=torch.uint8, device="cuda")
    sw = torch.empty(-(-N // 128), f3c.fp8_scale_stride(K), dtype=torch.uint8, device="cuda")
    f3c.op_quant_fp8(f3c.F3C_F32, w, W, sw, block_rows=128)
    bias, gate = to_dev(rng.standard_normal(N).astype(np.float32)), to_dev(rng.standard_normal(N).astype(np.float32))

    def run(epi, m):
        o = torch.zeros(m, N, device="cuda") if epi == 2 else torch.zeros(m, N, device="cuda").to(
            torch.uint8 if epi == 3 else torch.bfloat16)
        so = torch.zeros(m, f3c.fp8_scale_stride(N), dtype=torch.uint8, device="cuda")
        say("gemm_fp8 rows", epi, m, N, K)
        if epi == 2:
            f3c.op_gemm_fp8(2, A[:m], sa[:m], W, sw, bias, resid=o, gate=gate)
        else:
            f3c.op_gemm_fp8(epi, A[:m], sa[:m], W, sw, bias, out=o, out_scale=so if epi == 3 else None)
        return o, so

    for epi in (2,) if K > 4096 else (0, 1, 2, 3):
        whole = run(epi, top)
        for m in (1, 2, 16, 17, 33, 64, 100, 129, 300, 700, 1500, 2500, 4000):
            for x, y in zip(run(epi, m), whole):
                assert torch.equal(x, y[:m]), (epi, m)


# ------------------------------------------------------------------------------------- the pass between two blocks

def _check_norm(torch, f3c, dtype, out_dtype, post, pre, off, d, rows=None, weights=True, mods=True, shared=False,
                have_y=True, have_out=True, pad=0, seed=0):
    rng = np.random.default_rng(seed + d)
    B, R = len(off) - 1, rows or off[-1] + 1
    ty = {0: torch.float32, 1: torch.bfloat16}[dtype]
    to = {0: torch.float32, 1: torch.bfloat16, 2: torch.uint8}[out_dtype]
    f = lambda *s, scale=1.0: (rng.standard_normal(s) * scale).astype(np.float32)  # noqa: E731
    hbuf, h = _rows(torch, R, d, torch.float32, pad)
    h.copy_(to_dev(f(R, d) + 0.5))
    _, y = _rows(torch, R, d, ty, pad)
    y.copy_(to_dev(f(R, d, scale=0.3)))
    nb = 1 if shared else B
    gate, shift, scale = (f(nb, d, scale=0.5) for _ in range(3))
    pw, qw = f(d), f(d)
    dev = lambda a: to_dev(a[0] if shared else a)  # noqa: E731
    h0 = h.cpu().numpy()
    _, out = _rows(torch, R, d, torch.float32, pad, 3)
    obuf = torch.full((R + 1, d + pad), 3, device="cuda").to(to)
    out = obuf[:R, :d]
    so = torch.full((R, f3c.fp8_scale_stride(d)), 9, dtype=torch.uint8, device="cuda")
    kw = dict(y=y if have_y else None, off=off, out=out if have_out else None,
              out_scale=so if out_dtype == 2 and have_out else None, post=post, pre=pre, resid_scale=0.7, eps=1e-5)
    if weights:
        kw.update(post_w=to_dev(pw), pre_w=to_dev(qw))
    if mods:
        kw.update(gate=dev(gate), shift=dev(shift), scale=dev(scale))
    say("resid_norm", dtype, out_dtype, post, pre, off, d, pad)
    f3c.op_resid_norm(dtype, out_dtype, h, **kw)
    torch.cuda.synchronize()
    kinds = ("none", "layer", "rms")
    each = (lambda a: np.repeat(a, B, 0) if shared else a)
    full = dict(post=kinds[post], pre=kinds[pre], resid_scale=np.float64(np.float32(0.7)),
                eps=np.float64(np.float32(1e-5)))
    if weights:
        full.update(post_w=pw.astype(np.float64), pre_w=qw.astype(np.float64))
    if mods:
        full.update(gate=each(gate).astype(np.float64), shift=each(shift).astype(np.float64),
                    scale=each(scale).astype(np.float64))
    wh, wu = fp8.resid_norm(h0, y.float().cpu().numpy() if have_y else None, off, **full)
    # Statistics are sums of d terms in float32 (each lane adds its d / 64 in turn: n = d / 64 + 6 additions), the rest
    # a dozen roundings. A value's error is relative to the row's largest, through the mean and through 1 / sqrt.
    n, eps32 = d / 64 + 6, 2.0 ** -24
    gh = h.cpu().numpy()
    inside = np.zeros(R, bool)
    inside[off[0]:off[-1]] = True
    if have_y:
        tol = (n + 16) * eps32 * (np.abs(wh) + np.abs(wh - h0).max(axis=1, keepdims=True) + np.abs(h0))
        assert np.all(np.abs(gh - wh)[inside] <= tol[inside])
    else:
        assert np.array_equal(gh, h0)
    assert np.array_equal(gh[~inside], h0[~inside]) and bool((hbuf[:, d:] == 0).all())
    raw = obuf.cpu()
    if not have_out:
        assert bool((raw == 3).all())
        return
    got = raw[:R, :d].float().numpy() if out_dtype != 2 else None
    assert bool((raw[R:] == 3).all()) and bool((raw[:, d:] == 3).all()) and bool((raw[:R][~inside] == 3).all())
    # the error of h, divided by the row's deviation, adds to the norm's own
    sd = np.ones((R, 1)) if pre == 0 else np.maximum(
        np.sqrt(((wh - (wh.mean(1, keepdims=True) if pre == 1 else 0)) ** 2).mean(1, keepdims=True)), 1e-3)
    factor = (np.abs(qw) if weights else 1.0) * np.ones((R, d))
    add = np.zeros((R, d))
    if mods:
        for b, (lo, hi) in enumerate(zip(off, off[1:])):
            factor[lo:hi] *= np.abs(1.0 + each(scale)[b])
            add[lo:hi] = np.abs(each(shift)[b])
    rowmax = np.abs(wh).max(axis=1, keepdims=True) + np.abs(h0).max(axis=1, keepdims=True) + \
        np.abs(wh - h0).max(axis=1, keepdims=True)
    tol = 4 * (n + 16) * eps32 * (factor * rowmax / sd * (1 + rowmax / sd) + add)
    if out_dtype == 1:
        tol = tol + 2.0 ** -8 * (np.abs(wu) + tol)
    if out_dtype == 2:
        s = so.cpu().numpy()
        nb = -(-d // 128)
        assert np.all(s[~inside] == 9) and np.all(s[:, nb:] == 9)
        s, codes = s[:, :nb], raw[:R, :d].numpy()
        wide = np.pad(np.abs(wu), ((0, 0), (0, -d % 128))).reshape(R, -1, 128)
        far = np.pad(tol, ((0, 0), (0, -d % 128))).reshape(R, -1, 128)
        lo = np.array([[fp8.block_exponent(x) for x in r] for r in np.maximum(wide - far, 0).max(axis=2)])
        hi = np.array([[fp8.block_exponent(x) for x in r] for r in (wide + far).max(axis=2)])
        e = s.astype(int) - 127
        assert np.all((e >= lo)[inside]) and np.all((e <= hi)[inside])
        got = fp8.dequantise(codes, s, 1)
        tol = tol + np.maximum(2.0 ** -4 * (np.abs(wu) + tol), 2.0 ** -10 * fp8.scales(s, R, d, 1))
    err = np.abs(got - wu)[inside]
    assert np.all(err <= tol[inside]), float(np.max(err / tol[inside]))


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("pre", [0, 1, 2])
@pytest.mark.parametrize("dtype,out_dtype", [(0, 0), (1, 1), (1, 2)])
def test_resid_norm_norms_and_types(torch, f3c, post, pre, dtype, out_dtype):
    _check_norm(torch, f3c, dtype, out_dtype, post, pre, [0, 37], 1024)
    _check_norm(torch, f3c, dtype, out_dtype, post, pre, [0, 5, 5, 20], 328, pad=8)


@pytest.mark.parametrize("d", [8, 64, 120, 128, 136, 512, 520, 1000, 1024, 1032, 2048, 2056, 4096, 4104, 8192])
@pytest.mark.parametrize("out_dtype", [0, 1, 2])
def test_resid_norm_widths(torch, f3c, d, out_dtype):
    _check_norm(torch, f3c, out_dtype % 2, out_dtype, 2, 1, [1, 2, 9], d)


def test_resid_norm_options(torch, f3c):
    for kw in (dict(weights=False), dict(mods=False), dict(weights=False, mods=False), dict(shared=True),
               dict(have_y=False), dict(have_out=False), dict(pad=16)):
        _check_norm(torch, f3c, 1, 2, 1, 2, [2, 2, 30, 31, 60], 640, rows=64, **kw)
        _check_norm(torch, f3c, 0, 0, 2, 1, [0, 1], 1024, **kw)


def test_resid_norm_many_rows_and_samples(torch, f3c):
    rng = np.random.default_rng(3)
    off = [0] + [int(v) for v in np.sort(rng.integers(0, 3000, 63))] + [3000]
    _check_norm(torch, f3c, 1, 2, 2, 1, off, 256)
    _check_norm(torch, f3c, 1, 1, 1, 1, [0, 5000], 128)


def test_resid_norm_equal_and_huge_rows(torch, f3c):
    """A row of equal values (no variance), one of zeros, and a block whose NaN stays in its row."""
    h = np.zeros((4, 256), np.float32)
    h[0] = 3.0
    h[2], h[3] = np.arange(256), 1e15
    h[2, 9] = np.nan
    d = to_dev(h)
    out = torch.empty(4, 256, device="cuda")
    f3c.op_resid_norm(f3c.F3C_F32, f3c.F3C_F32, d, out=out, pre=f3c.F3C_NORM_LAYER)
    got = out.cpu().numpy()
    assert np.all(got[[0, 1, 3]] == 0.0) and np.isnan(got[2]).all()
    f3c.op_resid_norm(f3c.F3C_F32, f3c.F3C_F32, d, out=out, pre=f3c.F3C_NORM_RMS)
    got = out.cpu().numpy()
    assert np.allclose(got[[0, 3]], 1.0, rtol=1e-6) and np.all(got[1] == 0.0) and np.isnan(got[2]).all()


# -------------------------------------------------------------------------------------------------------- together

class Sublayer:
    """An MLP sublayer with norms on both sides, as a program runs it: four calls, three of them products or passes
    over what the one before left."""

    def __init__(self, torch, f3c, rows, d, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s, scale=1.0: torch.randn(*s, generator=g, device="cuda") * scale  # noqa: E731
        self.f3c, self.rows, self.d = f3c, rows, d
        self.h0, self.mod = r(rows, d), [r(d, scale=0.3) for _ in range(5)]
        self.w1, self.w2 = r(4 * d, d, scale=0.03), r(d, 4 * d, scale=0.03)
        self.b1, self.b2 = r(4 * d, scale=0.1), r(d, scale=0.1)
        u8 = lambda a, b: torch.zeros(a, b, dtype=torch.uint8, device="cuda")  # noqa: E731
        st = f3c.fp8_scale_stride
        self.q1, self.s1 = u8(4 * d, d), u8((4 * d + 127) // 128, st(d))
        self.q2, self.s2 = u8(d, 4 * d), u8((d + 127) // 128, st(4 * d))
        f3c.op_quant_fp8(f3c.F3C_F32, self.w1, self.q1, self.s1, block_rows=128)
        f3c.op_quant_fp8(f3c.F3C_F32, self.w2, self.q2, self.s2, block_rows=128)
        self.h = torch.empty_like(self.h0)
        self.u, self.us = u8(rows, d), u8(rows, st(d))
        self.hid, self.hs = u8(rows, 4 * d), u8(rows, st(4 * d))
        self.y = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
        self.out = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")

    def run(self):
        f, (shift, scale, gate, shift2, scale2) = self.f3c, self.mod
        self.h.copy_(self.h0)
        f.op_resid_norm(f.F3C_BF16, f.F3C_FP8, self.h, out=self.u, out_scale=self.us, shift=shift, scale=scale)
        f.op_gemm_fp8(3, self.u, self.us, self.q1, self.s1, self.b1, out=self.hid, out_scale=self.hs)
        f.op_gemm_fp8(0, self.hid, self.hs, self.q2, self.s2, self.b2, out=self.y)
        f.op_resid_norm(f.F3C_BF16, f.F3C_BF16, self.h, y=self.y, out=self.out, post=f.F3C_NORM_RMS, gate=gate,
                        shift=shift2, scale=scale2)


@pytest.mark.parametrize("rows,d", [(1, 128), (300, 256)])
def test_sublayer_of_the_three(torch, f3c, rows, d):
    """Each stage against the oracle's stage on the library's own input to it."""
    say("sublayer", rows, d)
    s = Sublayer(torch, f3c, rows, d, 5)
    s.run()
    torch.cuda.synchronize()
    n = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    by = lambda t, cols: t.cpu().numpy()[:, :-(-cols // 128)]  # noqa: E731
    shift, scale, gate, shift2, scale2 = (n(m)[None] for m in s.mod)
    _, u = fp8.resid_norm(n(s.h0), shift=shift, scale=scale)
    got = fp8.dequantise(s.u.cpu().numpy(), by(s.us, d))
    assert np.all(np.abs(got - u) <= 2.0 ** -4 * np.abs(u) + 2.0 ** -10 * fp8.scales(by(s.us, d), rows, d) + 1e-4)
    w1 = fp8.dequantise(s.q1.cpu().numpy(), by(s.s1, d), 128)
    step = 2.0 ** -10 * fp8.scales(by(s.s1, d), 4 * d, d, 128)
    assert np.all(np.abs(w1 - n(s.w1)) <= 2.0 ** -4 * np.abs(n(s.w1)) + step)
    v = fp8.gelu(fp8.linear(got, w1, n(s.b1)))
    tol = 1.13 * _sum_bound(got, w1) + 1e-5 * (1 + np.abs(v))
    hid = fp8.dequantise(s.hid.cpu().numpy(), by(s.hs, 4 * d))
    step = 2.0 ** -10 * fp8.scales(by(s.hs, 4 * d), rows, 4 * d)
    assert np.all(np.abs(hid - v) <= 2.0 ** -4 * np.abs(v) + step + 1.1 * tol)
    w2 = fp8.dequantise(s.q2.cpu().numpy(), by(s.s2, 4 * d), 128)
    y = fp8.linear(hid, w2, n(s.b2))
    tol = _sum_bound(hid, w2) + 1e-5 * (1 + np.abs(y))
    assert np.all(np.abs(n(s.y) - y) <= 2.0 ** -8 * np.abs(y) + 1.1 * tol)
    h, u2 = fp8.resid_norm(n(s.h0), n(s.y), post="rms", gate=gate, shift=shift2, scale=scale2)
    assert np.allclose(n(s.h), h, rtol=1e-5, atol=1e-5)
    assert np.all(np.abs(n(s.out) - u2) <= 2.0 ** -8 * np.abs(u2) + 1e-4)


def test_graph_replays_and_streams(torch, f3c):
    """A captured sublayer replays bit for bit between eager runs of another one; two streams at once do not meet."""
    a, b = Sublayer(torch, f3c, 200, 256, 1), Sublayer(torch, f3c, 333, 256, 2)
    outs = lambda s: [t.clone() for t in (s.h, s.u, s.us, s.hid, s.hs, s.y, s.out)]  # noqa: E731
    a.run()
    b.run()
    torch.cuda.synchronize()
    want_a, want_b = outs(a), outs(b)
    side = torch.cuda.Stream()
    say("graph")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for _ in range(3):
        for t in (a.h, a.u, a.us, a.hid, a.hs, a.y, a.out):
            t.zero_()
        graph.replay()
        with torch.cuda.stream(side):
            b.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs(a), want_a))
        assert all(torch.equal(x, y) for x, y in zip(outs(b), want_b))
        b.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs(b), want_b))


# ------------------------------------------------------------------------------------------------------- far corners

def test_gemm_infinities_before_the_quantising_epilogue(torch, f3c):
    """An infinite sum becomes NaN and does not count for its block's scale."""
    for M, N, K in ((3, 144, 272), (300, 272, 272), (2000, 2048, 272)):       # small and large tiles
        aq, ascl, wq, wscl, bias = _operands(M, N, K, 21)
        low, inf = bias.copy(), bias.copy()
        low[[5, 100]], inf[[5, 100]] = -1e30, (np.inf, np.nan)              # GELU of -1e30 is -0
        say("gemm_fp8 inf", M, N, K)
        q0, s0 = _gemm(torch, f3c, 3, aq, ascl, wq, wscl, low)
        q1, s1 = _gemm(torch, f3c, 3, aq, ascl, wq, wscl, inf)
        assert np.array_equal(s0, s1) and np.all((q1[:, [5, 100]] & 0x7F) == 0x7F)
        assert np.array_equal(np.delete(q0, [5, 100], 1), np.delete(q1, [5, 100], 1))
        assert np.all((q0[:, [5, 100]] & 0x7F) == 0)


def test_no_rows(torch, f3c):
    e = lambda *s, t=torch.uint8: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    f3c.op_quant_fp8(f3c.F3C_BF16, e(0, 256, t=torch.bfloat16), e(0, 256), e(0, 4))
    f3c.op_gemm_fp8(0, e(0, 256), e(0, 4), e(128, 256), e(1, 4), out=e(0, 128, t=torch.bfloat16))
    f3c.op_resid_norm(f3c.F3C_F32, f3c.F3C_F32, e(0, 64, t=torch.float32), out=e(0, 64, t=torch.float32))
    h = torch.ones(5, 64, device="cuda")
    f3c.op_resid_norm(f3c.F3C_F32, f3c.F3C_F32, h, y=h.clone(), off=[2, 2, 2], out=e(5, 64, t=torch.float32))
    torch.cuda.synchronize()
    assert bool((h == 1).all())


def test_rows_far_apart_and_offsets_beyond_32_bits(torch, f3c):
    """Row strides up to the limit, and rows that start beyond 4 GiB, give the bits of packed rows."""
    rng = np.random.default_rng(31)
    M, N, K = 260, 48, 144
    aq, ascl, wq, wscl, bias = _operands(M, N, K, 30)
    want = _gemm(torch, f3c, 0, aq, ascl, wq, wscl, bias)
    ld = (1 << 22) - 16
    A, W = (torch.empty(n, ld, dtype=torch.uint8, device="cuda")[:, :K] for n in (M, N))
    A.copy_(to_dev(aq))
    W.copy_(to_dev(wq))
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    sa, sw = _scale_dev(torch, f3c, ascl, K), _scale_dev(torch, f3c, wscl, K)
    say("gemm_fp8 strides", ld)
    f3c.op_gemm_fp8(0, A, sa, W, sw, to_dev(bias), out=out)
    assert np.array_equal(out.float().cpu().numpy(), want)
    # 5 GiB of rows; the last ones hold the values
    R, ld = 1_100_000, 5120
    A = torch.zeros(R, ld, dtype=torch.uint8, device="cuda")[:, :K]
    sa = torch.full((R, 4), 127, dtype=torch.uint8, device="cuda")
    A[R - M:], sa[R - M:] = to_dev(aq), _scale_dev(torch, f3c, ascl, K)
    W = to_dev(wq)
    out = torch.zeros(R, N, dtype=torch.bfloat16, device="cuda")
    h = torch.zeros(R, 1040, device="cuda")[:, :N]                           # 4.6 GB of residual rows
    say("gemm_fp8 far", R, ld)
    f3c.op_gemm_fp8(0, A, sa, W, sw, to_dev(bias), out=out)
    f3c.op_gemm_fp8(2, A, sa, W, sw, to_dev(bias), resid=h)
    assert np.array_equal(out[R - M:].float().cpu().numpy(), want)
    assert torch.equal(h[R - M:].to(torch.bfloat16), out[R - M:])
    del A, out, h
    x = torch.zeros(R, 1040, device="cuda")
    x[R - 3:] = to_dev(rng.standard_normal((3, 1040)).astype(np.float32))
    q, s = torch.empty(R, 1040, dtype=torch.uint8, device="cuda"), torch.empty(R, 12, dtype=torch.uint8, device="cuda")
    say("quant far", R)
    f3c.op_quant_fp8(f3c.F3C_F32, x, q, s)
    wq_, ws_ = fp8.quantise(x[R - 3:].cpu().numpy())
    assert np.array_equal(q[R - 3:].cpu().numpy(), wq_) and np.array_equal(s[R - 3:, :9].cpu().numpy(), ws_)
    o = torch.empty(R, 1040, device="cuda")
    few = torch.empty(3, 1040, device="cuda")
    say("resid_norm far", R)
    f3c.op_resid_norm(f3c.F3C_F32, f3c.F3C_F32, x, y=x, out=o, post=f3c.F3C_NORM_RMS)
    last = x[R - 3:].clone()
    f3c.op_resid_norm(f3c.F3C_F32, f3c.F3C_F32, last, out=few)
    assert torch.equal(o[R - 3:], few)
    # weights, the second row block beyond 4 GiB
    w = torch.zeros(130, 8_400_000, device="cuda")[:, :264]
    w.copy_(to_dev(rng.standard_normal((130, 264)).astype(np.float32)))
    q, s = torch.empty(130, 264, dtype=torch.uint8, device="cuda"), torch.empty(2, 4, dtype=torch.uint8, device="cuda")
    f3c.op_quant_fp8(f3c.F3C_F32, w, q, s, block_rows=128)
    wq_, ws_ = fp8.quantise(w.cpu().numpy(), 128)
    assert np.array_equal(q.cpu().numpy(), wq_) and np.array_equal(s[:, :3].cpu().numpy(), ws_)


def test_calls_on_a_named_stream_and_float8_types(torch, f3c):
    a = Sublayer(torch, f3c, 70, 256, 9)
    a.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    out, so = torch.zeros(70, 1024, dtype=f8, device="cuda"), torch.zeros(70, 8, dtype=e8, device="cuda")
    torch.cuda.synchronize()
    f3c.op_gemm_fp8(3, a.u.view(f8), a.us.view(e8), a.q1.view(f8), a.s1.view(e8), a.b1, out=out, out_scale=so,
                    stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(out.view(torch.uint8), a.hid) and torch.equal(so.view(torch.uint8), a.hs)


def _tile(name, M, N, K, epi):
    """Index of the tile that the library takes (choose_tiles in k_gemm8.hip, with the table as it stands there)."""
    import math
    import os
    import re
    from paper_2511_22533_amd import build
    with open(os.path.join(build.CSRC, "k_gemm8.hip")) as f:
        body = f.read()
    body = body[body.index(name + "[] = {"):]
    best = None
    for i, row in enumerate(re.findall(r"\{([-\d., ]+)\}", body[:body.index("};")])):
        bm, bn, per_cu, fixed, k, k_round, k_group, k_load, rnd, group, *load_epi = (float(x) for x in row.split(","))
        if epi == 3 and bn < 128:
            continue
        load = math.ceil(M / bm) * math.ceil(N / bn) / 256.0
        rounds, groups, kt = math.ceil(load / per_cu), math.ceil(load), math.ceil(K / 128)
        t = fixed + kt * (k + k_round * rounds + k_group * groups + k_load * load) + rnd * rounds + group * groups
        t += load_epi[(0, 1, 2, 3)[epi]] * load
        if best is None or t < best[0]:
            best = (t, i)
    return best[1]


@pytest.mark.parametrize("table,epi,shapes,tiles", [
    ("kTile8Cost", 0, [(4096, 1024), (1024, 1024), (3600, 144)], 9),
    ("kTile8Cost", 1, [(4096, 1024), (1024, 1024), (3600, 144)], 9),
    ("kTile8Cost", 2, [(4096, 1024), (1024, 1024), (1024, 2048)], 9),
    ("kTile8Cost", 3, [(4096, 1024), (1024, 1024)], 7),
    ("kTile8WideCost", 2, [(2048, 4112), (512, 4112)], 5)])
def test_gemm_tiles_agree_bit_for_bit(torch, f3c, table, epi, shapes, tiles):
    """Row counts that take each of the tiles (asserted) agree on the rows they share, the largest run's."""
    g = torch.Generator(device="cuda").manual_seed(3)
    top, crossed = 16000, set()
    for N, K in shapes:
        bytes_ = lambda r, c: torch.randint(0, 256, (r, c), generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
        code = lambda r, c: (lambda b: torch.where((b & 0x7F) == 0x7F, b - 1, b))(bytes_(r, c))  # noqa: E731
        A, W = code(top, K), code(N, K)
        sa = 120 + bytes_(top, f3c.fp8_scale_stride(K)) % 12
        sw = 110 + bytes_(-(-N // 128), f3c.fp8_scale_stride(K)) % 12
        bias = torch.randn(N, generator=g, device="cuda")

        def run(m):
            say("gemm_fp8 tiles", table, epi, m, N, K, _tile(table, m, N, K, epi))
            so = torch.zeros(m, f3c.fp8_scale_stride(N), dtype=torch.uint8, device="cuda")
            if epi == 2:
                o = torch.ones(m, N, device="cuda")
                f3c.op_gemm_fp8(2, A[:m], sa[:m], W, sw, bias, resid=o)
            else:
                o = torch.zeros(m, N, dtype=torch.uint8 if epi == 3 else torch.bfloat16, device="cuda")
                f3c.op_gemm_fp8(epi, A[:m], sa[:m], W, sw, bias, out=o, out_scale=so if epi == 3 else None)
            return o, so

        whole = run(top)
        seen = {_tile(table, top, N, K, epi)}
        for m in (1, 40, 70, 100, 130, 200, 260, 400, 520, 700, 900, 1300, 1700, 2500, 3300, 4000, 4500, 6000, 8000, 12000):
            t = _tile(table, m, N, K, epi)
            if t in seen:
                continue
            seen.add(t)
            for x, y in zip(run(m), whole):
                assert torch.equal(x, y[:m]), (m, N, K, t)
        crossed |= seen
    assert len(crossed) >= tiles, crossed


# ------------------------------------------------------------------------------------------- accuracy of the products

def _residual(torch, f3c, aq, ascl, wq, wscl, gate=None, h=None):
    """The residual epilogue without a bias, on zeros where h is not given: gate * v with no rounding behind it."""
    h = np.zeros((aq.shape[0], wq.shape[0]), np.float32) if h is None else h
    return _gemm(torch, f3c, 2, aq, ascl, wq, wscl, None, resid=h, gate=gate)


def _rel(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


@pytest.mark.parametrize("rows", ["normal", "gelu"])
@pytest.mark.parametrize("K", [128, 1024, 2048])
def test_gemm_8_bit_sums_are_as_exact_as_stated(torch, f3c, rows, K):
    """In the 2-norm 1.5e-5 of v on normal operands and 2.1e-5 behind a GELU, under half as much again allowed: one bit
    less kept of each product would double the error. Epilogue 3 hands on what epilogue 1 rounds to bf16: held to the same
    sums by the tests against float64."""
    rng = np.random.default_rng(K)
    a = rng.standard_normal((300, K))
    a = fp8.gelu(0.64 * a) if rows == "gelu" else a
    (aq, ascl), (wq, wscl) = fp8.quantise(a, 1), fp8.quantise(0.02 * rng.standard_normal((256, K)), 128)
    say("gemm_fp8 accuracy", rows, K)
    got = _residual(torch, f3c, aq, ascl, wq, wscl)
    assert _rel(got, fp8.linear(fp8.dequantise(aq, ascl), fp8.dequantise(wq, wscl, 128))) <= (
        3e-5 if rows == "gelu" else 2e-5)


@pytest.mark.parametrize("K", [512, 2048, 2064, 4096, 4112])
def test_gemm_gate_of_ones_is_no_gate(torch, f3c, K):
    """The same bits, and with them the same accuracy."""
    aq, ascl, wq, wscl, _ = _operands(70, 144, K, K)
    h = np.random.default_rng(2).standard_normal((70, 144)).astype(np.float32)
    say("gemm_fp8 gate of ones", K)
    one, none = (_residual(torch, f3c, aq, ascl, wq, wscl, gate=g, h=h) for g in (np.ones(144, np.float32), None))
    assert np.array_equal(one, none)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 128, 2064), (1, 128, 4112), (1, 1024, 4096), (40, 144, 2064), (300, 512, 4096),
                                   (200, 272, 4112), (1500, 1024, 4096)])
def test_gemm_residual_of_long_sums_with_gates(torch, f3c, gated, M, N, K):
    """Beyond K = 2048 products are exact and sums float32, whatever the gate's size: each of K / 16 additions to the
    accumulator and of those within an instruction is off by 2^-23 of the sum of magnitudes at most, and in the 2-norm,
    where they do not all fall to one side, by 2^-23 times the root of their number of the sum itself."""
    aq, ascl, wq, wscl, _ = _operands(M, N, K, M + K, spread=0.0)
    rng = np.random.default_rng(N)
    gate = (rng.standard_normal(N) * np.exp2(rng.uniform(-4, 4, N))).astype(np.float32) if gated else None
    a, w = fp8.dequantise(aq, ascl), fp8.dequantise(wq, wscl, 128)
    g = 1.0 if gate is None else gate.astype(np.float64)
    want, tot = g * fp8.linear(a, w), np.abs(g) * (np.abs(a) @ np.abs(w).T)
    say("gemm_fp8 long sums", M, N, K, gated)
    got = _residual(torch, f3c, aq, ascl, wq, wscl, gate=gate)
    assert np.all(np.abs(got - want) <= (K / 16 + 16) * 2.0 ** -23 * tot + 2.0 ** -22 * np.abs(want))
    assert _rel(got, want) <= np.sqrt(K / 16 + 16) * 2.0 ** -23 + 2.0 ** -23


@pytest.mark.parametrize("K", [272, 2064])
def test_gemm_scales_at_their_ends(torch, f3c, K):
    """A product knows its blocks' scales by their product alone: every pair of bytes that multiply to 1 gives the bits
    of unit scales, from 2^-127 to 2^127."""
    aq, _, wq, _, _ = _operands(40, 144, K, 3)
    kb = -(-K // 128)
    same = lambda e, n: np.full((n, kb), e, np.uint8)  # noqa: E731
    want = _residual(torch, f3c, aq, same(127, 40), wq, same(127, 2))
    assert np.isfinite(want).all() and np.abs(want).max() > 0
    for e in (0, 1, 7, 8, 64, 119, 135, 200, 246, 247, 253, 254):
        say("gemm_fp8 scale bytes", K, e)
        assert np.array_equal(_residual(torch, f3c, aq, same(e, 40), wq, same(254 - e, 2)), want), e


@pytest.mark.parametrize("K", [272, 2064])
def test_gemm_single_products_at_any_scales(torch, f3c, K):
    """Rows with one value that is not zero, under any two scale bytes: its products have at most 8 significant bits, so
    that each is exact wherever float32 holds it, but for what lies below 2^-80."""
    rng = np.random.default_rng(K)
    M, N, kb = 3000, 144, -(-K // 128)
    aq, ascl = np.zeros((M, K), np.uint8), rng.integers(0, 255, (M, kb), dtype=np.uint8)
    code = lambda n: (rng.integers(0, 127, n) | rng.integers(0, 2, n) << 7).astype(np.uint8)  # noqa: E731
    aq[np.arange(M), rng.integers(0, K, M)] = code(M)
    aq[:200][aq[:200] != 0] = 0x7E                         # the largest value beside the smallest weights
    wq, wscl = code(N * K).reshape(N, K), rng.integers(0, 255, (2, kb), dtype=np.uint8)
    wq[::3] = wq[::3] & 0x80 | 1
    want = fp8.linear(fp8.dequantise(aq, ascl), fp8.dequantise(wq, wscl, 128))
    say("gemm_fp8 single products", K)
    got = _residual(torch, f3c, aq, ascl, wq, wscl)
    held = np.abs(want) < 2.0 ** 128
    assert np.all(np.abs(got - want)[held] <= np.where(np.abs(want) < 2.0 ** -80, 2.0 ** -80, 0.0)[held])
    assert held.mean() > 0.5 and (np.abs(want[held]) > 2.0 ** 100).any()


@pytest.mark.parametrize("d", [512, 520, 1024, 1320, 2048, 2056, 4096, 4608, 8192])
def test_resid_norm_rows_do_not_depend_on_their_number(torch, f3c, d):
    """Of many rows a wave works off several in turn; each has the bits of a call of its own few, in every count of waves
    per row."""
    g = torch.Generator(device="cuda").manual_seed(d)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    rows, off = 20000, [0, 7000, 7001, 20000]
    h0, y, mod = r(rows, d), r(rows, d).to(torch.bfloat16), [r(3, d) for _ in range(3)]
    w = [r(d), r(d)]

    def run(lo, hi, off, b):
        h, out = h0[lo:hi].clone(), torch.zeros(hi - lo, d, dtype=torch.uint8, device="cuda")
        so = torch.zeros(hi - lo, f3c.fp8_scale_stride(d), dtype=torch.uint8, device="cuda")
        say("resid_norm rows", d, lo, hi)
        f3c.op_resid_norm(f3c.F3C_BF16, f3c.F3C_FP8, h, y=y[lo:hi], off=off, out=out, out_scale=so, post=f3c.F3C_NORM_RMS,
                          pre=f3c.F3C_NORM_LAYER, post_w=w[0], pre_w=w[1], gate=mod[0][b], shift=mod[1][b], scale=mod[2][b])
        return h, out, so

    many = run(0, rows, off, slice(0, 3))
    for lo, hi, b in ((0, 5, 0), (6990, 7000, 0), (7000, 7001, 1), (7001, 7100, 2), (13000, 13001, 2), (19990, 20000, 2)):
        for x, z in zip(run(lo, hi, None, slice(b, b + 1)), many):
            assert torch.equal(x, z[lo:hi]), (lo, hi)


@pytest.mark.parametrize("K", [400, 2064])
def test_gemm_bad_scales_stay_alone(torch, f3c, K):
    """A NaN scale of a row is NaN in its row, one of a block of weights in the block's columns, on either path."""
    aq, ascl, wq, wscl, _ = _operands(50, 272, K, 8)
    good = _residual(torch, f3c, aq, ascl, wq, wscl)
    ascl[20, 1], wscl[1, 3] = 255, 255
    aq[:, 128 * 3:] = 0                                  # (0 times NaN is NaN as well)
    say("gemm_fp8 NaN scales", K)
    got = _residual(torch, f3c, aq, ascl, wq, wscl)
    bad = np.zeros(good.shape, bool)
    bad[20], bad[:, 128:256] = True, True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    wscl[1, 3] = 127
    again = _residual(torch, f3c, aq, ascl, wq, wscl)
    assert np.array_equal(got[~bad], again[~bad])
