"""Pins of the 8-bit oracle (CPU): the e4m3 code, the scale rule, quantisation by brute force, the operators."""
import math

import numpy as np
import pytest

from oracle import fp8


def test_codes_are_e4m3():
    assert fp8.VALUES[0x7E] == 448.0 and fp8.VALUES[0x38] == 1.0 and fp8.VALUES[1] == 2.0 ** -9
    assert np.isnan(fp8.decode([0x7F, 0xFF])).all() and fp8.decode([0xC0])[0] == -2.0
    assert np.all(np.diff(fp8.VALUES) > 0)
    torch = pytest.importorskip("torch")
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(got, fp8.decode(np.arange(256)), equal_nan=True)


def test_rounding_is_to_nearest_even_of_brute_force():
    rng = np.random.default_rng(0)
    mids = (fp8.VALUES[1:] + fp8.VALUES[:-1]) / 2
    x = np.concatenate([fp8.VALUES, mids, np.nextafter(mids, 0), np.nextafter(mids, 999), rng.uniform(0, 448, 500)])
    x = x[x <= 448.0]
    for v, c in zip(x, fp8.encode(x)):
        d = np.abs(fp8.VALUES - v)
        best = np.flatnonzero(d == d.min())
        assert c in best and (len(best) == 1 or c % 2 == 0)
    assert np.array_equal(fp8.encode(-x), fp8.encode(x) | 0x80)
    torch = pytest.importorskip("torch")
    f = x.astype(np.float32)
    assert np.array_equal(torch.from_numpy(f).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), fp8.encode(f))


@pytest.mark.parametrize("amax,e", [(448.0, 0), (np.nextafter(448.0, 999), 1), (224.0, -1), (1.0, -8), (1.75, -8),
                                    (1.76, -7), (0.0, -126), (2.0 ** -140, -126), (3.4e38, 120)])
def test_scale_is_the_smallest_power_that_holds_the_block(amax, e):
    assert fp8.block_exponent(amax) == e
    assert amax <= 448.0 * 2.0 ** e
    assert e == -126 or amax > 448.0 * 2.0 ** (e - 1)


def test_quantise_ragged_blocks_and_bad_values():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((130, 200))
    x[3, 5], x[4, 6], x[5, :128] = np.nan, np.inf, 0.0
    for br in (1, 128):
        codes, scale = fp8.quantise(x, br)
        assert scale.shape == (-(-130 // br), 2)
        back = fp8.dequantise(codes, scale, br)
        ok = np.isfinite(x)
        assert np.isnan(back[~ok]).all()
        s = fp8.scales(scale, 130, 200, br)
        assert np.all(np.abs(back - x)[ok] <= np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10)[ok])
    assert scale.max() < 127           # the infinity did not count
    assert fp8.quantise(np.zeros((1, 8)))[1][0, 0] == 1


def test_operators_by_scalar_loops():
    rng = np.random.default_rng(2)
    a, w, b = rng.standard_normal((3, 5)), rng.standard_normal((4, 5)), rng.standard_normal(4)
    v = fp8.linear(a, w, b)
    for i in range(3):
        for j in range(4):
            assert math.isclose(v[i, j], sum(a[i, k] * w[j, k] for k in range(5)) + b[j], rel_tol=1e-12, abs_tol=1e-12)
    h, y = rng.standard_normal((6, 8)), rng.standard_normal((6, 8))
    pw, qw = rng.standard_normal(8), rng.standard_normal(8)
    g, sh, sc = (rng.standard_normal((2, 8)) for _ in range(3))
    for post in ("none", "layer", "rms"):
        for pre in ("none", "layer", "rms"):
            h2, u = fp8.resid_norm(h, y, [1, 3, 5], post, pre, pw, qw, g, 0.5, sh, sc, 1e-3)

            def one(x, kind):
                m = sum(x) / 8 if kind == "layer" else 0.0
                r = math.sqrt(sum((t - m) ** 2 for t in x) / 8 + 1e-3) if kind != "none" else 1.0
                return [(t - m) / r for t in x]

            for row, b in ((1, 0), (2, 0), (3, 1), (4, 1)):
                p = one(list(y[row]), post)
                hn = [h[row, c] + 0.5 * g[b, c] * p[c] * pw[c] for c in range(8)]
                q = one(hn, pre)
                assert np.allclose(h2[row], hn, rtol=1e-12, atol=1e-13)
                assert np.allclose(u[row], [q[c] * qw[c] * (1 + sc[b, c]) + sh[b, c] for c in range(8)], rtol=1e-11,
                                   atol=1e-12)
            assert np.array_equal(h2[[0, 5]], h[[0, 5]])
