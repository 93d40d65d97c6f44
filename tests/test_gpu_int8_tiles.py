"""Integer products on the matrix tiles (GPU), which calls of few outputs do not reach: a case for each tile, named by the
cost model's table as it stands in the source (a case that another choice would take elsewhere fails by name).

Ragged rows, columns and K, strides, no bias, no gate, bad scales, sums at the ends of 32 bits.
"""
import math
import os
import re

import pytest

from helpers import say, to_dev
from test_gpu_int8 import _check_gemm, _operands


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


TILES = [(256, 256), (192, 256), (128, 256), (128, 128), (64, 128), (32, 128), (64, 64), (32, 64), (128, 128)]

# epilogue, tile, rows, columns, K
CASES = [(0, 0, 4872, 2464, 400), (1, 0, 9927, 1168, 848), (2, 0, 9972, 1168, 1504), (0, 1, 10971, 672, 80),
         (1, 1, 11442, 656, 592), (2, 1, 11131, 656, 144), (0, 2, 8342, 400, 144), (1, 2, 9351, 400, 144),
         (2, 2, 9351, 400, 144), (0, 3, 10950, 544, 80), (1, 3, 11217, 336, 96), (2, 3, 10022, 592, 112),
         (0, 4, 5497, 144, 544), (1, 4, 4188, 208, 304), (2, 4, 161, 5520, 528), (0, 5, 133, 5456, 80),
         (1, 5, 133, 5456, 80), (2, 5, 35, 5232, 96), (0, 6, 67, 5472, 80), (1, 6, 33, 4144, 176), (2, 6, 2744, 144, 96),
         (0, 7, 33, 4144, 176), (1, 7, 35, 4112, 400), (2, 7, 33, 4144, 176), (0, 8, 11050, 144, 80),
         (1, 8, 11050, 144, 80), (2, 8, 11121, 144, 144)]
# tile, rows, columns of sums as long as 32 bits hold, into the residual
LONG = [(0, 3462, 3104), (1, 2818, 2832), (2, 2306, 1680), (3, 3604, 4384), (4, 961, 1040), (5, 771, 1232), (6, 613, 784),
        (7, 289, 416), (8, 1352, 1424)]


def tile(M: int, N: int, K: int, epi: int):
    """Index into TILES of what the library's integer products take, None for the kernel of few outputs."""
    groups = lambda r, c: math.ceil(M / r) * math.ceil(N / c)  # noqa: E731
    if M <= 16 or groups(32, 16) <= 256 or (groups(32, 32) <= 256 and groups(32, 32) * K <= 1 << 20):
        return None
    from paper_2511_22533_amd import build
    with open(os.path.join(build.CSRC, "k_gemm8.hip")) as f:
        text = f.read()
    body = text[text.index("kTile8Cost[] = {"):]
    rows = [[float(x) for x in r.split(",")] for r in re.findall(r"\{([-\d., ]+)\}", body[:body.index("};")])]
    assert [(r[0], r[1]) for r in rows] == TILES
    cost = []
    for bm, bn, per_cu, fixed, k, k_round, k_group, k_load, rnd, group, store, gelu, resid, _ in rows:
        load = math.ceil(M / bm) * math.ceil(N / bn) / 256.0
        rounds = math.ceil(load / per_cu)
        cost.append(fixed + math.ceil(K / 128) * (k + k_round * rounds + k_group * math.ceil(load) + k_load * load) +
                    rnd * rounds + group * math.ceil(load) + (store, gelu, resid)[epi] * load)
    return cost.index(min(cost))


def test_cases_reach_every_tile():
    """(No GPU.) Each case takes the tile that it is named for, each tile all three epilogues."""
    assert [tile(m, n, k, epi) for epi, _, m, n, k in CASES] == [t for _, t, *_ in CASES]
    assert {(epi, t) for epi, t, *_ in CASES} == {(e, t) for e in range(3) for t in range(len(TILES))}
    assert [tile(m, n, 133120, 2) for _, m, n in LONG] == list(range(len(TILES)))
    assert [tile(m, n, 131056, 2) for _, m, n in LONG] == list(range(len(TILES)))


@pytest.mark.gpu
@pytest.mark.parametrize("epi,t,M,N,K", CASES)
def test_strides_and_absent_operands(torch, f3c, epi, t, M, N, K):
    """No bias and no gate, a bias without a gate, and (into the residual) a gate without a bias."""
    say("gemm_i8 tiles", epi, TILES[t], M, N, K)
    ops = _operands(M, N, K, t)
    _check_gemm(torch, f3c, epi, ops, pads=(48, 16, 16), gated=False, with_bias=False)
    _check_gemm(torch, f3c, epi, ops, gated=False)
    if epi == 2:
        _check_gemm(torch, f3c, epi, ops, pads=(16, 48, 4), with_bias=False)


@pytest.mark.gpu
@pytest.mark.parametrize("K,low", [(133120, -127), (131056, -128)])
@pytest.mark.parametrize("t,M,N", LONG)
def test_sums_to_the_ends_of_32_bits(torch, f3c, t, M, N, K, low):
    """Rows of one value each: every sum is K times a product of two, to the ends of 32 bits."""
    say("gemm_i8 long", TILES[t], M, N, K)
    a = torch.full((M,), low, dtype=torch.int8, device="cuda")
    w = torch.full((N,), low, dtype=torch.int8, device="cuda")
    a[::3], w[1::2], w[::7] = 127, 127, 1
    sums = K * a.double()[:, None] * w.double()
    assert float(sums.abs().max()) == K * low * low < 2 ** 31
    h = torch.randn(M, N, device="cuda")
    sa, sw = torch.rand(M, device="cuda") / 64, torch.rand(N, device="cuda") / 2 ** 20
    v = sa.double()[:, None] * (sw.double() * sums)
    want = h.double() + v
    # the sum in float32, two products, the residual: a rounding each
    tol = 2.0 ** -24 * (3.01 * v.abs() + 1.01 * want.abs())
    f3c.op_gemm_i8(2, a[:, None].expand(M, K).contiguous(), sa, w[:, None].expand(N, K).contiguous(), sw, resid=h)
    assert bool(((h.double() - want).abs() <= tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("epi,t,M,N,K", [c for c in CASES if c[0] != 1])
def test_bad_scales_stay_alone(torch, f3c, epi, t, M, N, K):
    """Scales that are NaN or infinite spoil their rows and columns, the last among them; all else is the same, bit for bit."""
    say("gemm_i8 bad scales", epi, TILES[t], M, N, K)
    a, sa, w, sw, bias = (to_dev(x) for x in _operands(M, N, K, t))
    h = torch.randn(M, N, device="cuda")

    def run(sa, sw):
        if epi == 2:
            out = h.clone()
            f3c.op_gemm_i8(2, a, sa, w, sw, bias, resid=out)
        else:
            out = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
            f3c.op_gemm_i8(0, a, sa, w, sw, bias, out=out)
        return out

    good = run(sa, sw)
    rows, cols = [5, M - 1], [0, N // 2, N - 1]
    sa, sw = sa.clone(), sw.clone()
    sa[rows[0]], sa[rows[1]] = float("nan"), float("inf")
    sw[cols[0]], sw[cols[1]], sw[cols[2]] = float("nan"), float("inf"), float("-inf")
    got = run(sa, sw)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[rows], bad[:, cols] = True, True
    assert bool(good.isfinite().all()) and bool(got[rows[0]].isnan().all()) and bool(got[:, cols[0]].isnan().all())
    assert not bool(got[bad].isfinite().any()) and torch.equal(got[~bad], good[~bad])
