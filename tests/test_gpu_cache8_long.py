"""Single tokens over long caches (GPU), in one piece: a wave looks its pages up 64 at a time, and takes more than 64 from
32768 tokens on where a workgroup has eight waves (up to 256 workgroups), from 16384 where it has four.
"""
import pytest

from helpers import say
from oracle import cache8
from test_gpu_cache8 import _tokens

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


# head width, K/V heads, heads, queries, tokens, waves a workgroup
LONG = [(32, 1, 1, [1], [33000], 8), (64, 2, 4, [1], [40000], 8), (128, 1, 2, [3, 1], [33300, 70001], 8),
        (32, 8, 8, [1] * 33, [17000 + 3 * i for i in range(33)], 4),
        (64, 5, 10, [1] * 64, [500 * i + 9 for i in range(64)], 4), (128, 8, 8, [1] * 36, [20000 - 64 * i for i in range(36)], 4)]


@pytest.mark.parametrize("hd,kv,heads,nq,lens,waves", LONG)
def test_pages_behind_a_waves_64th(torch, f3c, hd, kv, heads, nq, lens, waves):
    """Samples share a few hundred pages but their last (NaN behind its last token); pages that are none at the end of a wave's
    first 64, at the beginning of its next, around both, and a whole 64 of another's.

    Tolerance: a score is a float32 sum of hd products, at most hd + 2 roundings of 2^-24 of the largest sum of |q k|, twice
    that where its maximum is subtracted; probabilities are rounded to bf16 (2^-8) for the product with V, not for
    their sum; a lane's own sum has n / 64 / waves * 16 terms, at most 2^12 here, so that sums add less than 2^-12; the
    result is rounded to bf16."""
    gen = torch.Generator(device="cuda").manual_seed(hd + len(lens))
    B, most, share = len(lens), max(-(-n // 64) for n in lens), 300
    pages = share + B
    table = torch.randint(0, share, (B, most), generator=gen, device="cuda", dtype=torch.int32)
    code = lambda: torch.randn(pages, kv, 64, hd, generator=gen, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)  # noqa: E731
    scale = lambda: torch.randint(126, 129, (pages, kv), generator=gen, device="cuda").to(torch.uint8)  # noqa: E731
    k, v = code(), code()
    for b, n in enumerate(lens):
        table[b, (n - 1) // 64] = share + b
        k[share + b, :, (n - 1) % 64 + 1:] = v[share + b, :, (n - 1) % 64 + 1:] = 0x7F
        table[b, -(-n // 64):] = -1
    vt = torch.empty(pages, kv, hd, 64, dtype=torch.uint8, device="cuda")
    vt[..., torch.from_numpy(cache8.SLOTS).cuda()] = v.transpose(2, 3)
    pool = f3c.Cache8(k, vt, scale(), scale(), table.contiguous())
    off = [1]
    for n in nq:
        off.append(off[-1] + n)
    q = (torch.randn(off[-1] + 1, heads * hd, generator=gen, device="cuda") * 1.5).bfloat16()
    of = lambda wave, at: wave + at * waves                                # noqa: E731  (page `at` of a wave's)
    none = [of(0, 63), of(1, 64), of(2, 63), of(2, 64), of(3, 62), of(3, 63), of(3, 64), of(3, 65)]
    none += [of(waves - 1, i) for i in range(64)]
    for gone in ((), none, [of(0, 64 + i) for i in range(30)]):
        for b, n in enumerate(lens):
            for p in gone:
                if p < -(-n // 64):
                    pool.table[b, p] = (-1, pages, 2 ** 31 - 1)[p % 3]
        o = torch.full_like(q, 5.0)
        say("long", hd, kv, heads, nq[:3], lens[:3], waves, len(gone))
        f3c.op_cache8_attention(pool, heads, off, lens, q, o, causal=True,
                                workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert bool((o[:1] == 5).all()) and bool((o[off[-1]:] == 5).all())
        for b, held in enumerate(lens):
            rows = slice(off[b], off[b + 1])
            last = held - nq[b] + torch.arange(nq[b], device="cuda")
            for g in range(kv):
                key, val, there = _tokens(torch, pool, b, held, g)
                assert bool(key.isfinite().all()) and bool(val.isfinite().all())
                see = there[None] & (torch.arange(held, device="cuda")[None] <= last[:, None])
                for h in range(g * (heads // kv), (g + 1) * (heads // kv)):
                    x, got = (t[rows, h * hd:(h + 1) * hd].double() for t in (q, o))
                    p = torch.softmax((x @ key.t() / hd ** 0.5).masked_fill(~see, float("-inf")), 1).nan_to_num(nan=0.0)
                    want, mag = p @ val, p @ val.abs()
                    top = ((x.abs() @ key.abs().t()) / hd ** 0.5).masked_fill(~see, 0.0).amax(1, keepdim=True)
                    tol = (2.0 ** -8 + 2.0 ** -12 + 6 * (hd + 2) * 2.0 ** -24 * top) * mag
                    tol = tol + 2.0 ** -8 * (want.abs() + tol)
                    assert bool(((got - want).abs() <= tol).all()), (b, h, float(((got - want).abs() / tol).max()))
