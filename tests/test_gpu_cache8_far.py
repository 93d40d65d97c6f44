"""Attention over the 8-bit cache with scores far from zero (GPU): what a row's largest score is must get the whole
probability, whatever its size, and a call must end.

A key's columns all hold one value and a query's too, so that every score is an exact float32 number: equal keys tie
exactly, and other keys lie a sixteenth of the score below. Where scores are large a row's output is the plain mean of V over
the keys of its largest one; a query of zeros sees all its keys alike.
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


def _pool(torch, f3c, gen, lens, heads, hd, low, high, v_exp=0, gone=(), signs=2):
    """(cache, K values float64 [sample][head][token], V the same with columns, whether a token is there [sample][token]).
    K: e4m3 codes of 1 to 15/8 with a scale of 2^low to 2^high a page, of both signs (or signs 1); V random, times 2^v_exp; NaN behind
    the last token. gone: (sample, page) that is none."""
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
    code = (0x38 + rand(0, 8, pages, heads, 64) + 0x80 * rand(0, signs, pages, heads, 64)).to(torch.uint8)
    k = code[..., None].expand(-1, -1, -1, hd).contiguous()
    v = torch.randn(pages, heads, 64, hd, generator=gen, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)
    ks = (127 + rand(low, high + 1, pages, heads)).to(torch.uint8)
    vs = torch.full((pages, heads), 127 + v_exp, dtype=torch.uint8, device="cuda")
    f8 = lambda x: x.view(torch.float8_e4m3fn).double()  # noqa: E731
    kval, vval = f8(code) * torch.exp2(ks.double() - 127)[..., None], f8(v) * 2.0 ** v_exp
    keys = [kval[table[b, :n].long()].transpose(0, 1).reshape(heads, -1)[:, :lens[b]] for b, n in enumerate(need)]
    vals = [vval[table[b, :n].long()].transpose(0, 1).reshape(heads, -1, hd)[:, :lens[b]] for b, n in enumerate(need)]
    for b, n in enumerate(lens):
        if n % 64:
            k[table[b, n // 64], :, n % 64:] = v[table[b, n // 64], :, n % 64:] = 0x7F
    vt = torch.empty(pages, heads, hd, 64, dtype=torch.uint8, device="cuda")
    vt[..., torch.from_numpy(cache8.SLOTS).cuda()] = v.transpose(2, 3)
    there = [torch.ones(n, dtype=torch.bool, device="cuda") for n in lens]
    for b, page in gone:
        table[b, page] = -1
        there[b][64 * page:64 * page + 64] = False
    return f3c.Cache8(k, vt, ks, vs, table), keys, vals, there


def _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, qs, v_exp=0, gone=(), workspace=None, signs=2):
    """qs: a query's value is drawn from these, with a sign; every eighth query is zeros.

    Tolerance: scores are exact but for their scale, 3 roundings of 2^-24; other keys lie 2^-4 of the score below, so that
    they count (above e^-30) where it is below 480 alone: e^ds is 1 within 2^-13.4 there. Probabilities are rounded to bf16
    in the product with V, by 2^-8 at most: p(1 + d) in place of p, in the product alone or in the sum too, puts a mean o
    of v off by 2^-8 (mean|v| + |o|) at most (equal keys as well, where the reference moves between them). Those scores,
    exponentials, their references' moves: 2^-12 of mean|v|; float32 sums of n terms: n 2^-24. A key below 2^-102 of the
    largest may count as none (exponentials end at 2^-126, taken against a reference within 2^24 of the largest): n of
    them lose n 2^-102 max|v|. Then o is rounded to bf16, 2^-8."""
    gen = torch.Generator(device="cuda").manual_seed(hd * 7 + nq[0])
    pool, keys, vals, there = _pool(torch, f3c, gen, lens, kv, hd, low, high, v_exp, gone, signs)
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
    f3c.op_cache8_attention(pool, heads, off, lens, q, o, causal=causal, workspace=workspace)
    torch.cuda.synchronize()
    assert bool((o[:1] == 5).all()) and bool((o[off[-1]:] == 5).all())
    for b, held in enumerate(lens):
        if not nq[b]:
            continue
        got = o[off[b]:off[b + 1]].double().view(nq[b], heads, hd)
        see = there[b][None].expand(nq[b], held)
        if causal:
            last = held - nq[b] + torch.arange(nq[b], device="cuda")
            see = see & (torch.arange(held, device="cuda")[None] <= last[:, None])
        for h in range(heads):
            g = h // (heads // kv)
            s = (val[off[b]:off[b + 1], h, None] * keys[b][g][None] * hd ** 0.5).masked_fill(~see, float("-inf"))
            n = see.sum(1, keepdim=True)
            p = torch.softmax(s, 1).nan_to_num(nan=0.0)
            want, mag = p @ vals[b][g], p @ vals[b][g].abs()
            tol = (2.0 ** -8 + 2.0 ** -12 + n * 2.0 ** -24) * mag + 2.0 ** -8 * want.abs()
            tol = tol + n * 2.0 ** -102 * vals[b][g].abs().max()
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


# head width, K/V heads, heads, queries, tokens, causal: every form of the kernel that calls take (16, 128 and 256 rows a
# workgroup, one and two groups of waves, pages whole and split), then rows enough for each form again under a mask
FORMS = [(32, 1, 1, [37], [98], True), (32, 1, 1, [32], [3741], True), (32, 1, 4, [4017, 1340], [92, 47], False),
         (32, 2, 8, [2528, 843], [1612, 807], False), (32, 2, 8, [2091, 698], [130, 66], False),
         (32, 2, 8, [667, 223], [6761, 3381], True), (32, 8, 56, [616], [2385], False),
         (32, 2, 14, [3254, 1085], [906, 454], False), (32, 1, 2, [2590, 864], [8147, 4074], False),
         (64, 1, 1, [34], [94], True), (64, 1, 1, [34], [2292], False), (64, 4, 4, [3022, 1008], [91, 46], False),
         (64, 1, 4, [2140], [4746], True), (64, 4, 28, [713], [389], False), (64, 1, 7, [445, 149], [5003, 2502], False),
         (64, 8, 32, [3350], [129], False), (64, 8, 32, [783, 262], [3050, 1540], False),
         (64, 8, 32, [1522, 508], [260, 131], False), (64, 4, 28, [882, 295], [1104, 553], False),
         (128, 1, 1, [32], [104], False), (128, 1, 1, [40], [1273], True), (128, 8, 16, [608, 203], [90, 46], False),
         (128, 8, 56, [67, 23], [1875, 938], False), (128, 2, 8, [1327, 443], [582, 292], False),
         (128, 4, 4, [1032], [2379], False),
         (32, 2, 14, [3254, 1085], [906, 454], True), (64, 4, 28, [882, 295], [1104, 553], True),
         (128, 2, 8, [1327, 443], [582, 292], True)]


@pytest.mark.parametrize("low,high", FAR + [(90, 99)])
@pytest.mark.parametrize("hd,kv,heads,nq,lens,causal", FORMS)
def test_far_scores_in_whole_pages(torch, f3c, hd, kv, heads, nq, lens, causal, low, high):
    """References that begin far out, and (exponents of 10 to 40) that get there from page to page; values up to 2^99."""
    _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, [8.0, 13.0, 120.0])
    pages = -(-lens[0] // 64)
    gone = [(0, p) for p in {0, pages // 2, pages - 1}]
    _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, [1.0, 96.0], 97 if low == 10 else 0, gone)


# calls in one piece of more than 64 pages, which are looked up 64 at a time
DEEP = [(32, 8, 32, [2055], [4419], False), (32, 8, 56, [456], [8462], True), (32, 8, 16, [2101], [8461], False),
        (64, 8, 56, [1217], [4407], True), (64, 8, 56, [300], [8584], False), (64, 8, 32, [3138], [4668], False),
        (64, 2, 14, [2395], [8439], True), (128, 8, 32, [1037], [4423], False), (128, 4, 28, [344], [8412], True)]


@pytest.mark.parametrize("low,high", FAR)
@pytest.mark.parametrize("hd,kv,heads,nq,lens,causal", DEEP)
def test_far_scores_over_many_pages(torch, f3c, hd, kv, heads, nq, lens, causal, low, high):
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, [8.0, 13.0, 120.0], workspace=none)
    _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, [1.0, 96.0], gone=[(0, 63), (0, 64), (0, 66)],
           workspace=none)


@pytest.mark.parametrize("hd,kv,heads,nq,lens,causal", FORMS + DEEP)
def test_far_scores_of_one_sign(torch, f3c, hd, kv, heads, nq, lens, causal):
    """Keys of one sign: half of the queries see negative scores alone, whose references come nearer from page to page, and
    references on both sides of those that whole pages keep to (2^12)."""
    for low, high in ((10, 40), (14, 18), (-6, 6), (0, 20)):
        _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, [8.0, 13.0, 120.0], signs=1)
    for low, high in ((14, 18), (0, 20)):
        _check(torch, f3c, hd, kv, heads, nq, lens, causal, low, high, [8.0, 13.0, 120.0],
               workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
