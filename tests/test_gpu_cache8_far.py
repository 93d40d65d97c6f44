"""Attention over the 8-bit cache with scores far from zero (GPU): what a row's largest score is must get the whole
probability, whatever its size, and a call must end.

A key's columns all hold one value and a query's too, so that every score is an exact float32 number: equal keys tie
exactly, and other keys lie a sixteenth of the score below. A row's output is then the plain mean of V over the keys of
its largest score; a query of zeros sees all its keys alike.
"""
import numpy as np
import pytest

from helpers import say, to_dev
from oracle import cache8

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


def _pool(torch, f3c, gen, lens, heads, hd, low, high):
    """(cache, K values float64 [sample][head][token], V the same with columns). K: e4m3 codes of 1 to 15/8 with a scale of
    2^low to 2^high a page, of both signs; V random; NaN behind the last token."""
    rng = np.random.default_rng(hd + sum(lens))
    need = [-(-n // 64) for n in lens]
    order = torch.from_numpy(rng.permutation(sum(need))).cuda()
    pages = sum(need)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n].int()
        at += n
    rand = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen, device="cuda")  # noqa: E731
    code = (0x38 + rand(0, 8, pages, heads, 64) + 0x80 * rand(0, 2, pages, heads, 64)).to(torch.uint8)
    k = code[..., None].expand(-1, -1, -1, hd).contiguous()
    v = torch.randn(pages, heads, 64, hd, generator=gen, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    ks = (127 + rand(low, high + 1, pages, heads)).to(torch.uint8)
    vs = torch.full((pages, heads), 127, dtype=torch.uint8, device="cuda")
    f8 = lambda x: x.view(torch.float8_e4m3fn).double()  # noqa: E731
    kval, vval = f8(code) * torch.exp2(ks.double() - 127)[..., None], f8(v)
    keys = [kval[table[b, :n].long()].transpose(0, 1).reshape(heads, -1)[:, :lens[b]] for b, n in enumerate(need)]
    vals = [vval[table[b, :n].long()].transpose(0, 1).reshape(heads, -1, hd)[:, :lens[b]] for b, n in enumerate(need)]
    for b, n in enumerate(lens):
        if n % 64:
            k[table[b, n // 64], :, n % 64:] = v[table[b, n // 64], :, n % 64:] = 0x7F
    vt = torch.empty(pages, heads, hd, 64, dtype=torch.uint8, device="cuda")
    vt[..., torch.from_numpy(cache8.SLOTS).cuda()] = v.transpose(2, 3)
    return f3c.Cache8(k, vt, ks, vs, table), keys, vals


def _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, qs, prescaled=False):
    """qs: a query's value is drawn from these, with a sign; every eighth query is zeros.

    Tolerance: ties have one probability p, so that a row is p sum(v) / (n p). In float32 its n sums are off by at most
    n 2^-24 mean|v| each; a sum of probabilities that are not the rounded ones of the product (16 rows a workgroup) is
    that of p = 1, exact; joins of parts multiply by 2^0 or by what is below e^-40 (gaps of a sixteenth of a score of
    2^10 or more); 1 / n and its product 2^-23; the rounding to bf16 2^-8. Zeros queries: p = 1 for all keys."""
    gen = torch.Generator(device="cuda").manual_seed(hd * 7 + nq[0])
    pool, keys, vals = _pool(torch, f3c, gen, lens, kv, hd, low, high)
    off = [1]
    for n in nq:
        off.append(off[-1] + n)
    R = off[-1] + 1
    val = torch.tensor(qs, dtype=torch.float64, device="cuda")[
        torch.randint(0, len(qs), (R, heads), generator=gen, device="cuda")]
    val = val * (1 - 2 * torch.randint(0, 2, (R, heads), generator=gen, device="cuda"))
    val[::8] = 0.0
    q = val[..., None].expand(-1, -1, hd).reshape(R, heads * hd).bfloat16().contiguous()
    assert torch.equal(q.double().view(R, heads, hd)[..., 0], val)
    o = torch.full_like(q, 5.0)
    say("far scores", hd, kv, heads, nq, lens, causal, low, high, qs)
    f3c.op_cache8_attention(pool, heads, off, lens, q, o, causal=causal, q_prescaled=prescaled)
    torch.cuda.synchronize()
    assert bool((o[:1] == 5).all()) and bool((o[off[-1]:] == 5).all())
    for b, held in enumerate(lens):
        if not nq[b]:
            continue
        got = o[off[b]:off[b + 1]].double().view(nq[b], heads, hd)
        see = torch.ones(nq[b], held, dtype=torch.bool, device="cuda")
        if causal:
            last = held - nq[b] + torch.arange(nq[b], device="cuda")
            see = torch.arange(held, device="cuda")[None] <= last[:, None]
        for h in range(heads):
            g = h // (heads // kv)
            s = (val[off[b]:off[b + 1], h, None] * keys[b][g][None]).masked_fill(~see, float("-inf"))
            top = (s == s.amax(1, keepdim=True)) & see
            n = top.sum(1, keepdim=True).clamp(min=1)
            p = top.double() / n
            want, mag = p @ vals[b][g], p @ vals[b][g].abs()
            tol = (n * 2.0 ** -24 + 2.0 ** -22) * mag + 1e-15 * vals[b][g].abs().max()
            tol = tol + 2.0 ** -8 * (want.abs() + tol)
            err = (got[:, h] - want).abs()
            assert bool((err <= tol).all()), (b, h, int((~(err <= tol)).any(1).nonzero()[0]), float(err.nan_to_num(9.0).max()))


FAR = [(20, 22), (27, 29), (31, 34), (10, 40)]     # exponents of K's scales; the softmax sees scores 2^6 to 2^11 times as large


@pytest.mark.parametrize("low,high", FAR)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_far_scores_in_one_masked_page(torch, f3c, hd, causal, low, high):
    """Fewer tokens than a page holds: 128 rows a workgroup (and 16)."""
    for kv, heads, nq, lens in ((8, 16, [2000], [63]), (2, 14, [1500, 1500], [41, 63]), (1, 1, [40], [50])):
        _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, [8.0, 13.0, 120.0])
