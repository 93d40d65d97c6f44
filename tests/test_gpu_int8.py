"""GPU parity of the integer rows and products, through the C ABI, against the float64 oracle (oracle/int8.py).

* quantisation bit for bit: whole numbers and scales, ties, quotients next to borders, bad rows, strides;
* products: the sums are exact, so an output is off by the roundings behind the sum alone; an output row's bits do not
  depend on the number of rows; sums up to the ends of 32 bits.
"""
import numpy as np
import pytest

from helpers import say, to_dev
from oracle import fp8, int8

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


def _view(torch, a, pad, fill, dtype=None):
    """a as rows with `pad` columns and one row more in their buffer, which hold `fill`."""
    t = to_dev(a)
    buf = torch.full((a.shape[0] + 1, a.shape[1] + pad), fill, device="cuda").to(dtype or t.dtype)
    buf[:a.shape[0], :a.shape[1]] = t
    return buf, buf[:a.shape[0], :a.shape[1]]


# ------------------------------------------------------------------------------------------------- quantisation

def _check_quant(torch, f3c, x, pad=0):
    """x: a float32 or bfloat16 tensor [R][K] on the GPU."""
    R, K = x.shape
    want_q, want_s = int8.quantise(x.float().cpu().numpy())
    qbuf, q = _view(torch, np.zeros((R, K), np.int8), pad, 7)
    s = torch.full((R + 1,), 77.0, device="cuda")
    f3c.op_quant_i8(f3c.F3C_F32 if x.dtype == torch.float32 else f3c.F3C_BF16, x, q, s[:R])
    torch.cuda.synchronize()
    assert np.array_equal(s[:R].cpu().numpy(), want_s, equal_nan=True)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert bool((qbuf[R:] == 7).all()) and bool((qbuf[:, K:] == 7).all()) and float(s[R]) == 77.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K,pad", [(1, 8, 0), (1, 1024, 0), (3, 128, 8), (5, 136, 24), (67, 520, 0), (9, 2056, 0),
                                        (1000, 1000, 8), (17, 4096, 16), (3, 8192, 0), (2, 8200, 0), (2, 20488, 8)])
def test_quant_bit_exact(torch, f3c, dtype, rows, K, pad):
    say("quant_i8", dtype, rows, K, pad)
    rng = np.random.default_rng(rows + K)
    x = (rng.standard_normal((rows, K)) * np.exp(rng.uniform(-80, 80, size=(rows, 1)))).astype(np.float32)
    x[:, :: 17] = 0.0
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    _check_quant(torch, f3c, _view(torch, x, pad, 0, t)[1], pad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [120, 128, 256, 264, 512, 1024, 1032, 1600, 2048, 4096, 4104])
def test_quant_at_the_borders_of_its_forms(torch, f3c, dtype, K):
    say("quant_i8 forms", dtype, K)
    rng = np.random.default_rng(K)
    x = rng.standard_normal((37, K)).astype(np.float32)
    x[5, K - 1], x[6, K - 1], x[7], x[8, 0] = 100.0, np.nan, 0.0, -np.inf
    _check_quant(torch, f3c, _view(torch, x, 8, 0, torch.float32 if dtype == "f32" else torch.bfloat16)[1], 8)


@pytest.mark.parametrize("K", [64, 512, 8448])
def test_quant_borders(torch, f3c, K):
    """Quotients at half steps and next to them: rows whose largest value is 127 of a scale, the rest at (n + 1/2) times
    the scale, moved by single units of the last place."""
    rng = np.random.default_rng(K)
    s = np.exp(rng.uniform(-60, 60, 400)).astype(np.float32)
    s[:40] = 2.0 ** rng.integers(-100, 100, 40)          # exact ties
    n = rng.integers(-127, 127, (400, K))
    x = ((n + 0.5) * s[:, None].astype(np.float64)).astype(np.float32)
    step = rng.integers(-2, 3, x.shape)
    x = np.where(step < 0, np.nextafter(x, np.float32(-3e38)), np.where(step > 1, np.nextafter(x, np.float32(3e38)), x))
    x[:, 0] = (127.0 * s).astype(np.float32)
    say("quant_i8 borders", K)
    _check_quant(torch, f3c, to_dev(x))


def test_quant_extremes(torch, f3c):
    x = np.random.default_rng(5).standard_normal((16, 256)).astype(np.float32)
    x[0] = 0.0
    x[1, 3], x[2, 255], x[3, 0] = np.nan, np.inf, -np.inf
    x[4] = 3.4028234e38
    x[5] = 2.0 ** -149
    x[6] = np.float32(2.0 ** -126) * np.arange(256)
    x[7] *= np.float32(1e-38)
    x[8] = -x[8]
    x[9, 1:] = -0.0
    say("quant_i8 extremes")
    _check_quant(torch, f3c, to_dev(x))
    _check_quant(torch, f3c, to_dev(x).bfloat16())


# ------------------------------------------------------------------------------------------------------ products

def _operands(M, N, K, seed):
    rng = np.random.default_rng(seed)
    a, w = (rng.integers(-127, 128, s).astype(np.int8) for s in ((M, K), (N, K)))
    sa = np.exp(rng.uniform(-6, 0, M)).astype(np.float32)
    sw = (np.exp(rng.uniform(-6, 0, N)) / np.sqrt(K) / 100).astype(np.float32)
    return a, sa, w, sw, rng.standard_normal(N).astype(np.float32)


def _check_gemm(torch, f3c, epi, ops, pads=(0, 0, 0), gated=True, with_bias=True):
    a, sa, w, sw, bias = ops
    bias = bias if with_bias else None
    (M, K), N = a.shape, w.shape[0]
    p, v = int8.linear(a, sa, w, sw), int8.linear(a, sa, w, sw, bias)
    # the sum in float32, two products, the bias: a rounding each
    tol = 2.0 ** -24 * (3.01 * np.abs(p) + np.abs(v))
    A, W = _view(torch, a, pads[0], 99)[1], _view(torch, w, pads[1], 99)[1]
    dev = [to_dev(sa), W, to_dev(sw), None if bias is None else to_dev(bias)]
    if epi == 2:
        rng = np.random.default_rng(M + N)
        h = rng.standard_normal((M, N)).astype(np.float32)
        gate = rng.standard_normal(N).astype(np.float32) if gated else None
        buf, out = _view(torch, h, pads[2], 5.0)
        f3c.op_gemm_i8(2, A, *dev, resid=out, gate=None if gate is None else to_dev(gate))
        g = 1.0 if gate is None else gate
        want = h + g * v
        tol = np.abs(g) * tol + 2.0 ** -24 * 1.01 * (np.abs(g * v) + np.abs(want))
    else:
        buf, out = _view(torch, np.zeros((M, N), np.float32), pads[2], 5.0, torch.bfloat16)
        f3c.op_gemm_i8(epi, A, *dev, out=out)
        want = v
        if epi == 1:
            # the slope of GELU is at most 1.13; its float32 evaluation is off by a few roundings, relative, with the
            # exponent's argument (at most 2 |u| log2 e, |u| < |v| (0.8 + 0.036 v^2)) rounded before the power is taken
            want = fp8.gelu(v)
            tol = 1.13 * tol + 2.0 ** -24 * (8 + 12 * np.abs(v) * (0.8 + 0.036 * v * v)) * np.abs(want) + 1e-30
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    torch.cuda.synchronize()
    assert bool((buf[M:] == 5).all()) and bool((buf[:, N:] == 5).all())            # nothing behind rows and columns
    err = np.abs(out.float().cpu().numpy() - want)
    assert np.all(err <= tol + 1e-37), (epi, M, N, K, float(np.max(err / (tol + 1e-37))))


SHAPES = [(1, 16, 16), (1, 128, 128), (1, 1024, 1024), (3, 144, 144), (17, 16, 2064), (33, 272, 400), (64, 128, 640),
          (70, 1040, 272), (130, 256, 1424), (257, 400, 512), (300, 512, 4096), (1, 4096, 4096), (5, 80, 8208),
          (1000, 2064, 144), (3000, 1024, 1024), (2500, 4096, 512)]


@pytest.mark.parametrize("epi", [0, 1, 2])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gemm_against_float64(torch, f3c, epi, M, N, K):
    say("gemm_i8", epi, M, N, K)
    _check_gemm(torch, f3c, epi, _operands(M, N, K, M + N + K))


@pytest.mark.parametrize("epi", [0, 1, 2])
@pytest.mark.parametrize("M", [1, 77])
def test_gemm_strides_and_absent_operands(torch, f3c, epi, M):
    say("gemm_i8 strides", epi, M)
    _check_gemm(torch, f3c, epi, _operands(M, 208, 336, 4), pads=(48, 16, 16), gated=False, with_bias=False)


@pytest.mark.parametrize("M,N,K,low", [(1, 16, 133120, -127), (40, 80, 133120, -127), (40, 16, 131056, -128),
                                       (300, 144, 131056, -128)])
def test_gemm_sums_to_the_ends_of_32_bits(torch, f3c, M, N, K, low):
    say("gemm_i8 ends", M, N, K)
    a, w = np.full((M, K), low, np.int8), np.full((N, K), low, np.int8)
    w[1::2] = 127
    ones = lambda n: np.ones(n, np.float32)  # noqa: E731
    _check_gemm(torch, f3c, 2, (a, ones(M) / 64, w, ones(N) / 2 ** 20, ones(N)), gated=False)


def test_gemm_bad_rows_stay_alone(torch, f3c):
    a, sa, w, sw, bias = _operands(50, 144, 400, 8)
    sa[7], sw[100] = np.nan, np.inf
    say("gemm_i8 NaN")
    out = torch.zeros(50, 144, dtype=torch.bfloat16, device="cuda")
    f3c.op_gemm_i8(0, to_dev(a), to_dev(sa), to_dev(w), to_dev(sw), to_dev(bias), out=out)
    got, good = out.float().cpu().numpy(), int8.linear(a, sa, w, sw, bias)
    bad = np.zeros(got.shape, bool)
    bad[7], bad[:, 100] = True, True
    assert np.isnan(got[7]).all() and not np.isfinite(got[:, 100]).any() and np.isfinite(got[~bad]).all()
    assert np.all(np.abs(got - good)[~bad] <= 2.0 ** -7 * np.abs(good)[~bad] + 1e-6)


@pytest.mark.parametrize("N,K", [(1024, 1024), (1024, 4096), (4096, 1024), (400, 1424), (512, 4112)])
def test_gemm_rows_do_not_depend_on_their_number(torch, f3c, N, K):
    """Other row counts take other kernels and tiles; sums are exact and what follows them is the same."""
    g = torch.Generator(device="cuda").manual_seed(N + K)
    top = 9000
    A = torch.randint(-127, 128, (top, K), generator=g, device="cuda", dtype=torch.int8)
    W = torch.randint(-127, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = (torch.rand(n, generator=g, device="cuda") / K / 10 for n in (top, N))
    sa *= K
    bias, gate = (torch.randn(N, generator=g, device="cuda") for _ in range(2))

    def run(epi, m):
        say("gemm_i8 rows", epi, m, N, K)
        if epi == 2:
            o = torch.zeros(m, N, device="cuda")
            f3c.op_gemm_i8(2, A[:m], sa[:m], W, sw, bias, resid=o, gate=gate)
        else:
            o = torch.zeros(m, N, device="cuda", dtype=torch.bfloat16)
            f3c.op_gemm_i8(epi, A[:m], sa[:m], W, sw, bias, out=o)
        return o

    for epi in (0, 1, 2):
        whole = run(epi, top)
        for m in (1, 2, 8, 16, 17, 33, 64, 100, 129, 300, 700, 1500, 2500, 4000, 6000):
            assert torch.equal(run(epi, m), whole[:m]), (epi, m)


def test_gemm_far_rows(torch, f3c):
    """Rows of A and of the output beyond 2^31 bytes."""
    M, N, K, lda = 700, 128, 256, (1 << 22) - 16
    A = torch.zeros(M, lda, dtype=torch.int8, device="cuda")[:, :K]
    a, sa, w, sw, bias = _operands(M, N, K, 3)
    A.copy_(to_dev(a))
    out = torch.zeros(M, 1 << 21, dtype=torch.bfloat16, device="cuda")[:, :N]
    say("gemm_i8 far")
    f3c.op_gemm_i8(0, A, to_dev(sa), to_dev(w), to_dev(sw), to_dev(bias), out=out)
    want = int8.linear(a, sa, w, sw, bias)
    assert np.all(np.abs(out.float().cpu().numpy() - want) <= 2.0 ** -7 * np.abs(want) + 1e-6)


@pytest.mark.parametrize("M,N", [(700, 512), (5, 528)])
def test_gemm_far_rows_of_each_kernel(torch, f3c, M, N):
    """As above where tiles are taken, and of the weights where rows are few."""
    K, ld = 256, (1 << 22) - 16
    few = M < 16
    far = torch.zeros(N if few else M, ld, dtype=torch.int8, device="cuda")[:, :K]
    a, sa, w, sw, bias = _operands(M, N, K, 3)
    far.copy_(to_dev(w if few else a))
    out = torch.zeros(M, 1 << 21, dtype=torch.bfloat16, device="cuda")[:, :N]
    say("gemm_i8 far rows", M, N)
    f3c.op_gemm_i8(0, *((to_dev(a), to_dev(sa), far, to_dev(sw)) if few else (far, to_dev(sa), to_dev(w), to_dev(sw))),
                   to_dev(bias), out=out)
    want = int8.linear(a, sa, w, sw, bias)
    assert np.all(np.abs(out.float().cpu().numpy() - want) <= 2.0 ** -7 * np.abs(want) + 1e-6)


def test_quantised_product_chain_and_graph(torch, f3c):
    """Rows through quantisation, an MLP's two products and the residual, eagerly, on another stream and from a graph
    replayed with new inputs between eager work."""
    rng = np.random.default_rng(2)
    M, D, F = 90, 256, 1024
    f = lambda *s, scale=1.0: to_dev((rng.standard_normal(s) * scale).astype(np.float32))  # noqa: E731
    w1, w2, b1, b2 = f(F, D, scale=0.06), f(D, F, scale=0.03), f(F, scale=0.1), f(D, scale=0.1)
    e = lambda *s, t=torch.int8: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    q1, q2, s1, s2 = e(F, D), e(D, F), e(F, t=torch.float32), e(D, t=torch.float32)
    f3c.op_quant_i8(f3c.F3C_F32, w1, q1, s1)
    f3c.op_quant_i8(f3c.F3C_F32, w2, q2, s2)
    x, h = f(M, D), f(M, D)
    h0 = h.clone()
    xq, xs, y, yq, ys = e(M, D), e(M, t=torch.float32), e(M, F, t=torch.bfloat16), e(M, F), e(M, t=torch.float32)

    def step():
        f3c.op_quant_i8(f3c.F3C_F32, x, xq, xs)
        f3c.op_gemm_i8(1, xq, xs, q1, s1, b1, out=y)
        f3c.op_quant_i8(f3c.F3C_BF16, y, yq, ys)
        f3c.op_gemm_i8(2, yq, ys, q2, s2, b2, resid=h)

    say("int8 chain")
    step()
    a, asc = int8.quantise(x.cpu().numpy())
    v = fp8.gelu(int8.linear(a, asc, q1.cpu().numpy(), s1.cpu().numpy(), b1.cpu().numpy()))
    got = y.float().cpu().numpy()
    assert np.all(np.abs(got - v) <= 2.0 ** -8 * np.abs(v) + 1e-5)
    b, bs = int8.quantise(got)
    assert np.array_equal(b, yq.cpu().numpy()) and np.array_equal(bs, ys.cpu().numpy())
    want = h0.cpu().numpy() + int8.linear(b, bs, q2.cpu().numpy(), s2.cpu().numpy(), b2.cpu().numpy())
    assert np.all(np.abs(h.cpu().numpy() - want) <= 2.0 ** -21 * (np.abs(want) + 4))
    first = h.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h.copy_(h0)
        step()
    side.synchronize()
    assert torch.equal(h, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        x.copy_(f(M, D))
        h.copy_(h0)
        graph.replay()
        torch.cuda.synchronize()
        replayed = h.clone()
        h.copy_(h0)
        step()
        assert torch.equal(h, replayed), seed
