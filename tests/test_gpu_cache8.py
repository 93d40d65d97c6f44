"""GPU parity of the 8-bit cache of keys and values, through the C ABI, against the float64 oracle (oracle/cache8.py).

* append bit for bit: codes and scale bytes of every tile, and every byte that is not the call's own as it was;
* attention: each output within what its roundings can be off (below); no token, no page, NaN behind the last token and
  in tokens that a query does not see; the split key range; caches beyond 2^31 bytes; streams and graphs.
"""
import numpy as np
import pytest

from helpers import say, to_dev
from oracle import cache8, fp8

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


def _bf16(torch, a):
    return torch.from_numpy(np.asarray(a, np.float32)).bfloat16()


def _oracle_pool(rng, pages, heads, hd, table, empty=0x7F):
    z = lambda *s: np.full(s, empty, np.uint8)  # noqa: E731
    return cache8.Cache(z(pages, heads, 64, hd), z(pages, heads, hd, 64), z(pages, heads), z(pages, heads), table)


def _device_pool(torch, f3c, c):
    return f3c.Cache8(to_dev(c.k), to_dev(c.v), to_dev(c.ks), to_dev(c.vs), to_dev(c.table.astype(np.int32)))


def _same(pool, c):
    for got, want in zip(pool, (c.k, c.v, c.ks, c.vs)):
        assert np.array_equal(got.cpu().numpy(), want)


def _table(rng, lens, spare=2):
    """Pages without order for this many tokens of each sample; entries behind them name no page."""
    need = [-(-n // 64) for n in lens]
    order = rng.permutation(sum(need) + spare)
    t = np.full((len(lens), max(max(need), 1)), -1, np.int64)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n]
        at += n
    return t, sum(need) + spare


# -------------------------------------------------------------------------------------------------------- append

def _check_append(torch, f3c, dtype, heads, hd, steps, pad=0, seed=0, scale=2.0):
    """steps: new tokens of each sample, call by call."""
    rng = np.random.default_rng(seed + hd)
    B = len(steps[0])
    table, pages = _table(rng, np.sum(steps, axis=0))
    c = _oracle_pool(rng, pages, heads, hd, table)
    pool = _device_pool(torch, f3c, c)
    lens = [0] * B
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    for new in steps:
        off = np.concatenate([[1], 1 + np.cumsum(new)])                # a row in front that no sample has
        R, w = int(off[-1]) + 1, heads * hd
        x = [(rng.standard_normal((R, w)) * np.exp(rng.uniform(-scale, scale, (R, 1)))).astype(np.float32) for _ in "kv"]
        d = []
        for a in x:
            buf = torch.full((R, w + pad), 1e30, device="cuda").to(t)
            buf[:, :w] = to_dev(a)
            d.append(buf[:, :w])
        say("append", dtype, heads, hd, new, lens)
        f3c.op_cache8_append(f3c.F3C_F32 if dtype == "f32" else f3c.F3C_BF16, pool, lens, [int(o) for o in off], *d)
        torch.cuda.synchronize()
        k, v = (a.float().cpu().numpy() for a in d)
        for b in range(B):
            c.append(b, lens[b], k[off[b]:off[b + 1]], v[off[b]:off[b + 1]])
            lens[b] += int(new[b])
        _same(pool, c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,hd", [(1, 32), (3, 64), (2, 128)])
@pytest.mark.parametrize("steps", [[[1]], [[64]], [[200]], [[1, 0, 63, 64, 65]], [[5, 60], [1, 1], [1, 4], [130, 0], [0, 1]],
                                   [[1]] * 5])
def test_append_bit_exact(torch, f3c, dtype, heads, hd, steps):
    _check_append(torch, f3c, dtype, heads, hd, steps, seed=len(steps))


def test_append_strides_and_many_samples(torch, f3c):
    rng = np.random.default_rng(0)
    _check_append(torch, f3c, "bf16", 2, 64, [list(rng.integers(0, 90, 64)), [1] * 64, list(rng.integers(0, 9, 64))], pad=24)


def test_append_scale_growth_over_all_exponents(torch, f3c):
    """Tokens that grow: what a page holds is rounded anew, down to e4m3's subnormals and to zero."""
    _check_append(torch, f3c, "f32", 1, 32, [[1]] * 20, seed=3, scale=12.0)


def test_append_extremes(torch, f3c):
    rng = np.random.default_rng(9)
    table = np.array([[1, 0]])
    c = _oracle_pool(rng, 3, 1, 32, table)
    pool = _device_pool(torch, f3c, c)
    x = rng.standard_normal((70, 32)).astype(np.float32)
    x[0, 0], x[1, 1], x[2, 2], x[3], x[5] = np.nan, np.inf, -np.inf, 0.0, 2.0 ** -149
    x[66] = 3.4e38
    y = x * np.float32(2.0 ** -60)
    y[:64] = 0.0
    say("append extremes")
    at = 0
    for n in (1, 3, 62, 4):
        f3c.op_cache8_append(f3c.F3C_F32, pool, [at], [0, n], to_dev(x[at:at + n]), to_dev(y[at:at + n]))
        c.append(0, at, x[at:at + n], y[at:at + n])
        at += n
    for got, want in zip(pool[:2], (c.k, c.v)):                        # (NaN has two codes)
        g, w = (np.where((a & 0x7F) == 0x7F, 0x7F, a) for a in (got.cpu().numpy(), want))
        assert np.array_equal(g, w)
    assert np.array_equal(pool[2].cpu().numpy(), c.ks) and np.array_equal(pool[3].cpu().numpy(), c.vs)


def test_append_passes_over_pages_that_are_none(torch, f3c):
    rng = np.random.default_rng(4)
    for bad in (-1, 5, 2 ** 31 - 1, -2 ** 31):
        c = _oracle_pool(rng, 5, 2, 64, [[3, bad, 0], [bad, 2, 1]])
        pool = _device_pool(torch, f3c, c)
        k, v = (rng.standard_normal((340, 128)).astype(np.float32) for _ in "kv")
        say("append bad page", bad)
        f3c.op_cache8_append(f3c.F3C_F32, pool, [0, 10], [0, 170, 340], to_dev(k), to_dev(v))
        c.append(0, 0, k[:170], v[:170])
        c.append(1, 10, k[170:], v[170:])
        _same(pool, c)


# ----------------------------------------------------------------------------------------------------- attention

def _filled(torch, f3c, rng, lens, heads, hd, table=None, pages=None, spread=1.0):
    """Caches of random tokens, whole pages in front of NaN bytes behind each sample's last token."""
    if table is None:
        table, pages = _table(rng, lens)
    c = _oracle_pool(rng, pages, heads, hd, table)
    for b, n in enumerate(lens):
        k, v = (rng.standard_normal((n, heads * hd)) * np.exp(rng.uniform(-spread, spread, (n, 1))) for _ in "kv")
        c.append(b, 0, k, v)
    return c, _device_pool(torch, f3c, c)


def _bounds(out, mag, top, hd):
    """How far an output may be off. A score is a float32 sum of hd products, at most hd + 2 roundings of 2^-24 of the
    largest sum of |q k| (and twice that where its maximum is subtracted), so that a probability is off by the factor
    e^ds; it is rounded to bf16 (2^-8) for the product with V but not for the sum; the exponential and float32 sums of
    positive terms add less than 2^-12; the result is rounded to bf16."""
    ds = np.repeat(3 * (hd + 2) * 2.0 ** -24 * top, hd, axis=1)
    tol = (2.0 ** -8 + 2.0 ** -12 + 2 * ds) * mag
    return tol + 2.0 ** -8 * (np.abs(out) + tol)


def _queries(torch, rng, rows, w, scale=1.5):
    q = _bf16(torch, rng.standard_normal((rows, w)) * scale)
    return q.cuda(), q.float().numpy()


def _check_attention(torch, f3c, c, pool, heads, lens, nq, causal, rng, pad=0, workspace=None, prescaled=False, scale=1.5):
    hd = c.k.shape[3]
    off = [0]
    for n in nq:
        off.append(off[-1] + n)
    off = [o + 2 for o in off]                                         # rows in front and behind that no sample has
    R, w = off[-1] + 1, heads * hd
    d, q = _queries(torch, rng, R, w, scale)
    if prescaled:
        d = (d.float() * f3c.attention_q_scale(hd)).bfloat16()
        q = d.float().cpu().numpy() / f3c.attention_q_scale(hd)
    wide = torch.full((R, w + pad), 9.0, device="cuda").bfloat16()
    wide[:, :w] = d
    o = torch.full((R, w + pad), 5.0, device="cuda").bfloat16()
    say("attention", heads, c.heads, hd, lens[:8], nq[:8], causal)
    f3c.op_cache8_attention(pool, heads, off, lens, wide[:, :w], o[:, :w], causal=causal, workspace=workspace,
                            q_prescaled=prescaled)
    torch.cuda.synchronize()
    got = o.float().cpu().numpy()
    assert np.all(got[:, w:] == 5) and np.all(got[:2] == 5) and np.all(got[off[-1]:] == 5)
    for b, n in enumerate(lens):
        rows = slice(off[b], off[b + 1])
        want, mag, top = c.attention(b, n, q[rows], causal)
        err, tol = np.abs(got[rows, :w] - want), _bounds(want, mag, top, hd)
        assert np.array_equal(np.isnan(got[rows, :w]), np.isnan(want)), b
        ok = ~np.isnan(want)
        assert np.all(err[ok] <= tol[ok] + 1e-37), (b, n, nq[b], float(np.max((err / (tol + 1e-37))[ok])))
    return o


CASES = [([1], [1]), ([64], [1]), ([65], [3]), ([300], [17]), ([1374], [1]), ([1374], [130]), ([0, 5, 63, 64, 129], [2, 1, 5, 0, 9]),
         ([700, 1, 130], [100, 33, 65])]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("heads,kv,hd", [(2, 2, 32), (2, 2, 64), (4, 2, 128), (7, 1, 64), (6, 2, 32)])
@pytest.mark.parametrize("lens,nq", CASES)
def test_attention_against_float64(torch, f3c, heads, kv, hd, lens, nq, causal):
    rng = np.random.default_rng(sum(lens) + hd + heads)
    c, pool = _filled(torch, f3c, rng, lens, kv, hd)
    _check_attention(torch, f3c, c, pool, heads, lens, nq, causal, rng)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_many_rows(torch, f3c, hd, causal):
    """Rows enough for every form of the kernel, ragged against its tiles."""
    rng = np.random.default_rng(hd)
    lens, nq = [333, 200], [301, 270]
    c, pool = _filled(torch, f3c, rng, lens, 1, hd)
    _check_attention(torch, f3c, c, pool, 1, lens, nq, causal, rng)
    _check_attention(torch, f3c, c, pool, 3, lens, nq, causal, rng, pad=16, prescaled=True)


def test_attention_large_scores(torch, f3c):
    """One key far above the rest, maxima that move from page to page."""
    rng = np.random.default_rng(3)
    lens = [400]
    for hd in (32, 64, 128):
        c, pool = _filled(torch, f3c, rng, lens, 1, hd, spread=3.0)
        _check_attention(torch, f3c, c, pool, 2, lens, [40], False, rng, scale=6.0)


def test_attention_samples_at_most(torch, f3c):
    rng = np.random.default_rng(1)
    lens = [int(n) for n in rng.integers(0, 200, 64)]
    c, pool = _filled(torch, f3c, rng, lens, 1, 32)
    _check_attention(torch, f3c, c, pool, 2, lens, [int(n) for n in rng.integers(0, 4, 64)], True, rng)


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_attention_split_key_range(torch, f3c, hd):
    """Few queries, long keys: split over workgroups as far as the workspace goes, the same within roundings without."""
    rng = np.random.default_rng(hd)
    lens, nq = [9000, 3, 4097], [1, 2, 3]
    c, pool = _filled(torch, f3c, rng, lens, 1, hd)
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(3 * 4096 * 8, device="cuda")):
        for causal in (False, True):
            a = _check_attention(torch, f3c, c, pool, 2, lens, nq, causal, np.random.default_rng(5), workspace=ws)
            b = _check_attention(torch, f3c, c, pool, 2, lens, nq, causal, np.random.default_rng(5), workspace=ws)
            assert torch.equal(a, b)


@pytest.mark.parametrize("nq", [1, 40, 200])
def test_attention_pages_that_are_none_or_shared(torch, f3c, nq):
    rng = np.random.default_rng(6)
    lens = [200, 200, 128, 200]
    table = np.array([[1, 2, 3, 4], [1, 2, 3, 0], [5, 6, -1, 7], [7, 5, 6, 1]])
    c, pool = _filled(torch, f3c, rng, [200, 0, 128, 0], 2, 64, table, 8)
    c.append(1, 192, rng.standard_normal((8, 128)), rng.standard_normal((8, 128)))
    c.append(3, 0, rng.standard_normal((64, 128)), rng.standard_normal((64, 128)))
    c.k[1, :, :8], c.ks[1] = c.k[2, :, :8], c.ks[2]
    for bad in (-1, 8, 2 ** 31 - 1, -2 ** 31):
        c.table = table.copy()
        c.table[2, 0] = c.table[3, 1] = c.table[3, 3] = bad
        _check_attention(torch, f3c, c, _device_pool(torch, f3c, c), 4, lens, [nq] * 4, False, rng)
        _check_attention(torch, f3c, c, _device_pool(torch, f3c, c), 4, lens, [nq] * 4, True, rng)
    c.table[:] = -1
    o = _check_attention(torch, f3c, c, _device_pool(torch, f3c, c), 4, lens, [nq] * 4, False, rng)
    assert bool((o[2:2 + 4 * nq] == 0).all())


@pytest.mark.parametrize("nq", [20, 150])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_attention_nan_reaches_the_queries_that_see_it(torch, f3c, nq, hd):
    rng = np.random.default_rng(8)
    lens = [200]
    c, _ = _filled(torch, f3c, rng, lens, 2, hd)

    def plant(token, head, is_v, col):
        page = c.page(0, token)
        codes = c.tile(is_v, page, head)
        codes[token % 64, col] = 0xFF
        c.put(is_v, page, head, codes)

    plant(190, 0, True, 3)             # seen by the last ten queries of a causal call, in one column
    plant(195, 1, False, 5)            # and by the last five, in all columns
    plant(199, 0, True, 17)
    _check_attention(torch, f3c, c, _device_pool(torch, f3c, c), 4, lens, [nq], True, rng)
    _check_attention(torch, f3c, c, _device_pool(torch, f3c, c), 4, lens, [nq], False, rng)


def test_attention_bad_queries_stay_alone(torch, f3c):
    rng = np.random.default_rng(2)
    c, pool = _filled(torch, f3c, rng, [150], 1, 64)
    for n in (5, 200):
        d, _ = _queries(torch, rng, n, 128)
        o, p = torch.empty_like(d), torch.empty_like(d)
        say("attention NaN query", n)
        f3c.op_cache8_attention(pool, 2, [0, n], [150], d, o)
        d[3, 7], d[n - 1, 100] = float("nan"), float("inf")
        f3c.op_cache8_attention(pool, 2, [0, n], [150], d, p)
        bad = torch.zeros_like(o, dtype=torch.bool)
        bad[3, :64] = bad[n - 1, 64:] = True
        assert bool(p[3, :64].isnan().all()) and torch.equal(o[~bad], p[~bad])


def test_attention_far_pages(torch, f3c):
    """Pages beyond 2^31 bytes of the pool."""
    rng = np.random.default_rng(0)
    heads, hd, pages = 4, 64, 140000
    c, _ = _filled(torch, f3c, rng, [300], heads, hd)
    e = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
    far = f3c.Cache8(e(pages, heads, 64, hd), e(pages, heads, hd, 64), e(pages, heads), e(pages, heads),
                     to_dev((c.table + pages - c.k.shape[0]).astype(np.int32)))
    for t, a in zip(far, (c.k, c.v, c.ks, c.vs)):
        t[pages - a.shape[0]:] = to_dev(a)
    _check_attention(torch, f3c, c, far, 4, [300], [3], True, rng)
    _check_attention(torch, f3c, c, far, 8, [300], [140], True, rng)
    k, v = (rng.standard_normal((20, heads * hd)).astype(np.float32) for _ in "kv")
    f3c.op_cache8_append(f3c.F3C_F32, far, [300], [0, 20], to_dev(k), to_dev(v))
    c.append(0, 300, k, v)
    for t, a in zip(far, (c.k, c.v, c.ks, c.vs)):
        assert np.array_equal(t[pages - a.shape[0]:].cpu().numpy(), a)


# ----------------------------------------------------------------------------------- attention of many rows, on the GPU

def _random_pool(torch, f3c, gen, lens, heads, hd):
    """Random codes with scales of 1/2 to 4, NaN behind each sample's last token, pages without order, and the slots."""
    table, pages = _table(np.random.default_rng(len(lens)), lens)
    slots = torch.from_numpy(cache8.SLOTS).cuda()
    code = lambda: torch.randn(pages, heads, 64, hd, generator=gen, device="cuda").to(torch.float8_e4m3fn).view(torch.uint8)  # noqa: E731
    scale = lambda: torch.randint(126, 130, (pages, heads), generator=gen, device="cuda").to(torch.uint8)  # noqa: E731
    k, v = code(), code()
    for b, n in enumerate(lens):
        if n % 64:
            k[table[b, n // 64], :, n % 64:] = v[table[b, n // 64], :, n % 64:] = 0x7F
    vt = torch.empty(pages, heads, hd, 64, dtype=torch.uint8, device="cuda")
    vt[..., slots] = v.transpose(2, 3)
    return f3c.Cache8(k, vt, scale(), scale(), to_dev(table.astype(np.int32)))


def _tokens(torch, pool, b, held, head):
    """(K, V float64 [held][hd] of a sample's tokens, whether each is there)."""
    pages, slots = pool.k.shape[0], torch.from_numpy(cache8.SLOTS).cuda()
    t = pool.table[b, :-(-held // 64)].long()
    there = (t >= 0) & (t < pages)
    t = torch.where(there, t, 0)

    def values(codes, scale):
        x = codes.contiguous().view(torch.float8_e4m3fn).double() * torch.exp2(scale.double() - 127)[:, None, None]
        return x.reshape(-1, x.shape[-1])[:held]

    return (values(pool.k[t, head], pool.k_scale[t, head]),
            values(pool.v[t, head][..., slots].transpose(1, 2), pool.v_scale[t, head]), there.repeat_interleave(64)[:held])


def _check_rows(torch, f3c, pool, heads, lens, nq, causal, gen, scale=1.5):
    """As _check_attention, with the float64 softmax in torch on the GPU. Scores here are hundreds apart: exponentials below
    2^-126 are zero, and they are taken relative to a reference within 2^24 of the largest, so that a token whose share is
    below 2^-102 of the largest may count as none; held tokens of at most max |v| lose held 2^-102 max |v| in all."""
    kv, hd = pool.k.shape[1], pool.k.shape[3]
    off = [2]
    for n in nq:
        off.append(off[-1] + n)
    q = (torch.randn(off[-1] + 1, heads * hd, generator=gen, device="cuda") * scale).bfloat16()
    o = torch.full_like(q, 5.0)
    say("attention rows", heads, kv, hd, lens, nq, causal)
    f3c.op_cache8_attention(pool, heads, off, lens, q, o, causal=causal)
    torch.cuda.synchronize()
    assert bool((o[:2] == 5).all()) and bool((o[off[-1]:] == 5).all())
    for b, held in enumerate(lens):
        for h in range(heads if held else 0):
            if h % (heads // kv) == 0:
                k, v, there = _tokens(torch, pool, b, held, h // (heads // kv))
                bad_k, bad_v = k.isnan().any(1), v.isnan()
                k, v = k.nan_to_num(nan=0.0), v.nan_to_num(nan=0.0)
            for at in range(0, nq[b], 1024):
                n = min(1024, nq[b] - at)
                rows, cols = slice(off[b] + at, off[b] + at + n), slice(h * hd, (h + 1) * hd)
                see = there[None].expand(n, held)
                if causal:
                    last = held - nq[b] + at + torch.arange(n, device="cuda")
                    see = see & (torch.arange(held, device="cuda")[None] <= last[:, None])
                x = q[rows, cols].double()
                s = (x @ k.t() / hd ** 0.5).masked_fill(~see, float("-inf"))
                p = torch.softmax(s, 1).nan_to_num(nan=0.0)
                want, mag = p @ v, p @ v.abs()
                top = ((x.abs() @ k.abs().t()) / hd ** 0.5).masked_fill(~see, 0.0).amax(1, keepdim=True)
                ds = 3 * (hd + 2) * 2.0 ** -24 * top                   # (as in _bounds)
                tol = (2.0 ** -8 + 2.0 ** -12 + 2 * ds) * mag
                tol = tol + 2.0 ** -8 * (want.abs() + tol) + held * 2.0 ** -102 * v.abs().max()
                nan = (see & bad_k).any(1, keepdim=True) | (see.double() @ bad_v.double() > 0)
                got = o[rows, cols].double()
                assert torch.equal(got.isnan(), nan), (b, h, at)
                assert bool(((got - want).abs() <= tol)[~nan].all()), (b, h, at, float(((got - want).abs() / tol)[~nan].max()))
        if not held:
            assert bool((o[off[b]:off[b + 1]] == 0).all())


# head width, K/V heads, heads, queries, tokens, causal: calls that take 128 and 256 rows a workgroup, their pages in
# one piece and split, one sample and ragged ones
ROWS = [(32, 2, 14, [2050], [333], False), (32, 2, 14, [1500, 500, 1, 0, 750], [333, 166, 111, 333, 33], False),
        (32, 2, 14, [460], [6000], False), (32, 4, 16, [333], [9000], True), (32, 8, 16, [460], [9000], True),
        (32, 8, 16, [1500, 500, 1, 0, 750], [3000, 1500, 1000, 3000, 2700], True), (32, 4, 16, [4500, 900], [4500, 4600], True),
        (64, 2, 14, [2050], [333], False), (64, 2, 14, [4500, 1500, 1, 0, 2250], [333, 166, 111, 333, 33], False),
        (64, 2, 4, [970, 323, 1, 0, 485], [6000, 3000, 2000, 6000, 5700], False), (64, 8, 16, [2050], [6000], False),
        (64, 2, 14, [333], [9000], True), (64, 8, 16, [460], [9000], True), (64, 8, 16, [3000, 5], [4000, 0], True),
        (128, 8, 16, [970], [333], False), (128, 2, 4, [3000, 1000, 1, 0, 1500], [333, 166, 111, 333, 33], False),
        (128, 4, 4, [200, 66, 1, 0, 100], [9000, 4500, 3000, 9000, 8700], False), (128, 2, 14, [1500], [2000], True),
        (128, 4, 4, [200, 66, 1, 0, 100], [9000, 4500, 3000, 9000, 8700], True), (128, 8, 16, [970, 323], [900, 500], True),
        # and calls whose pages two groups of waves share, or do not
        (32, 8, 16, [2050], [333], False), (32, 2, 14, [1500], [2000], False), (32, 8, 16, [700], [6000], True),
        (32, 8, 16, [700, 233, 1, 0, 350], [3000, 1500, 1000, 3000, 2700], True), (32, 2, 4, [4500], [3000], False),
        (32, 2, 4, [970, 323, 1, 0, 485], [9000, 4500, 3000, 9000, 8700], True), (32, 2, 14, [4500], [1000], False),
        (32, 8, 16, [970], [4000], False), (32, 8, 16, [460, 153, 1, 0, 230], [9000, 4500, 3000, 9000, 8700], True),
        (32, 8, 16, [2050], [3000], False),
        (64, 16, 16, [700, 233, 1, 0, 350], [4000, 2000, 1333, 4000, 3700], False), (64, 2, 4, [2050], [6000], True),
        (64, 2, 14, [2050, 683, 1, 0, 1025], [3000, 1500, 1000, 3000, 2700], True),
        (64, 16, 16, [4500, 1500, 1, 0, 2250], [500, 250, 166, 500, 200], False), (64, 8, 16, [2050], [6000], True),
        (64, 2, 14, [1500], [500], False), (64, 2, 14, [2050], [3000], True), (64, 2, 14, [460], [4000], True),
        (64, 2, 4, [970, 323, 1, 0, 485], [4000, 2000, 1333, 4000, 3700], True), (64, 8, 16, [2050], [700], False),
        (64, 2, 14, [4500], [6000], True), (64, 8, 16, [333], [9000], True),
        (64, 2, 4, [4500, 1500, 1, 0, 2250], [1374, 687, 458, 1374, 1074], False),
        (128, 1, 1, [4500], [2000], False), (128, 2, 14, [200, 66, 1, 0, 100], [2000, 1000, 666, 2000, 1700], True),
        (128, 8, 16, [2050, 683, 1, 0, 1025], [3000, 1500, 1000, 3000, 2700], True), (128, 2, 14, [970], [700], False),
        (128, 1, 1, [2050], [6000], False), (128, 2, 4, [333, 111, 1, 0, 166], [6000, 3000, 2000, 6000, 5700], True),
        (128, 8, 16, [700, 233, 1, 0, 350], [1000, 500, 333, 1000, 700], True), (128, 2, 14, [333], [3000], True)]


@pytest.mark.parametrize("hd,kv,heads,nq,lens,causal", ROWS)
def test_attention_rows_against_float64(torch, f3c, hd, kv, heads, nq, lens, causal):
    gen = torch.Generator(device="cuda").manual_seed(hd + sum(lens))
    pool = _random_pool(torch, f3c, gen, lens, kv, hd)
    _check_rows(torch, f3c, pool, heads, lens, nq, causal, gen)
    # scores far apart, their maxima moving from page to page
    pool.k_scale[:] = torch.randint(124, 133, pool.k_scale.shape, generator=gen, device="cuda").to(torch.uint8)
    _check_rows(torch, f3c, pool, heads, lens, nq, causal, gen, scale=4.0)
    # pages that are none at the front, in the middle, two together, the last; all of a sample's
    table = pool.table.clone()
    whole = -(-lens[0] // 64)
    for at, bad in ((0, -1), (whole // 2, pool.k.shape[0]), (whole // 2 + 1, 2 ** 31 - 1), (whole - 1, -2 ** 31)):
        pool.table[0, at] = bad
    if len(lens) > 1:
        pool.table[1] = -1
    _check_rows(torch, f3c, pool, heads, lens, nq, causal, gen)
    pool.table[:] = table
    # NaN: of K in the last token, which a causal call's last query sees, of V in a column of another head's, 200 before
    # it, and of V in a token that all queries see
    def page(b, t):
        return int(table[b, t // 64]), t % 64

    n = lens[0]
    (x, t), (y, u), (z, w) = page(0, n - 1), page(0, n - 201), page(0, 1)
    pool.k[x, 0, t, 5] = 0xFF
    pool.v[y, kv - 1, 7, cache8.slot(u)] = 0x7F
    pool.v[z, 0, 9, cache8.slot(w)] = 0x7F
    _check_rows(torch, f3c, pool, heads, lens, nq, causal, gen)


# ----------------------------------------------------------------------------------------------------- together

def test_block_on_8_bits(torch, f3c):
    """An attention sublayer as a program runs it: rows quantised, q, k, v by integer products, keys and values appended,
    attention, the output quantised and projected into the residual; a first chunk and single tokens, two samples."""
    rng = np.random.default_rng(7)
    D, H, KV, hd = 256, 4, 2, 64
    dev = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    w = {n: to_dev((rng.standard_normal(s) * 0.08).astype(np.float32)) for n, s in
         dict(q=(D, D), k=(KV * hd, D), v=(KV * hd, D), o=(D, D)).items()}
    wq, ws = {n: dev(*t.shape, t=torch.int8) for n, t in w.items()}, {n: dev(t.shape[0], t=torch.float32) for n, t in w.items()}
    for n in w:
        f3c.op_quant_i8(f3c.F3C_F32, w[n], wq[n], ws[n])
    table, pages = _table(rng, [150, 90])
    pool = f3c.Cache8.empty(pages, KV, hd, to_dev(table.astype(np.int32)))
    c = _oracle_pool(rng, pages, KV, hd, table)
    lens = [0, 0]
    for new in ([130, 64], [1, 1], [1, 1], [3, 0]):
        R = sum(new)
        off = [0, new[0], R]
        x, h = to_dev(rng.standard_normal((R, D)).astype(np.float32)), torch.zeros(R, D, device="cuda")
        xq, xs = dev(R, D, t=torch.int8), dev(R, t=torch.float32)
        q, k, v, o = dev(R, D), dev(R, KV * hd), dev(R, KV * hd), dev(R, D)
        say("block", new)
        f3c.op_quant_i8(f3c.F3C_F32, x, xq, xs)
        for n, t in (("q", q), ("k", k), ("v", v)):
            f3c.op_gemm_i8(0, xq, xs, wq[n], ws[n], out=t)
        f3c.op_cache8_append(f3c.F3C_BF16, pool, lens, off, k, v)
        after = [a + n for a, n in zip(lens, new)]
        f3c.op_cache8_attention(pool, H, off, after, q, o, causal=True)
        oq, os = dev(R, D, t=torch.int8), dev(R, t=torch.float32)
        f3c.op_quant_i8(f3c.F3C_BF16, o, oq, os)
        f3c.op_gemm_i8(2, oq, os, wq["o"], ws["o"], resid=h)
        torch.cuda.synchronize()
        kn, vn, qn = (t.float().cpu().numpy() for t in (k, v, q))
        for b in range(2):
            rows = slice(off[b], off[b + 1])
            c.append(b, lens[b], kn[rows], vn[rows])
            want, mag, top = c.attention(b, after[b], qn[rows], True)
            assert np.all(np.abs(o.float().cpu().numpy()[rows] - want) <= _bounds(want, mag, top, hd))
        deq = oq.double() * os.double()[:, None]
        want = deq @ (wq["o"].double() * ws["o"].double()[:, None]).t()
        assert bool(((h - want).abs() <= 2.0 ** -21 * (want.abs() + 1e-3)).all())
        lens = after


def test_streams_and_graphs(torch, f3c):
    """On another stream, and captured with its own workspace beside another graph's; replays between eager calls."""
    rng = np.random.default_rng(1)
    lens = [5000, 700]
    c, pool = _filled(torch, f3c, rng, lens, 2, 64)
    d, _ = _queries(torch, rng, 2, 256)
    o, first = torch.empty_like(d), torch.empty_like(d)
    k, v = (to_dev(rng.standard_normal((2, 128)).astype(np.float32)) for _ in "kv")

    def step(out, ws=None, stream=None):
        f3c.op_cache8_append(f3c.F3C_F32, pool, [4999, 699], [0, 1, 2], k, v, stream=stream)
        f3c.op_cache8_attention(pool, 4, [0, 1, 2], lens, d, out, causal=True, workspace=ws, stream=stream)

    say("cache8 streams")
    step(first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step(o, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(o, first)
    with torch.cuda.stream(side):
        step(o.zero_())
    side.synchronize()
    assert torch.equal(o, first)
    graphs, outs = [], [torch.empty_like(d) for _ in range(2)]
    for out in outs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(out)
    for i in range(3):
        d.copy_(torch.randn(d.shape, device="cuda"))
        k.copy_(torch.randn(k.shape, device="cuda"))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        step(o)
        assert torch.equal(o, outs[0]) and torch.equal(o, outs[1]), i


@pytest.mark.parametrize("hd,kv,heads,nq,lens", [(64, 8, 16, [333], [9000]), (128, 4, 4, [200, 66, 1, 0, 100], [9000, 4500, 3000, 9000, 8700]),
                                                 (32, 2, 4, [970, 323], [9000, 4500])])
def test_rows_at_once_and_replayed(torch, f3c, hd, kv, heads, nq, lens):
    """Calls of many rows whose pages are split: two streams at once, each with memory of its own, and a graph replayed
    between them, bit for bit the same."""
    gen = torch.Generator(device="cuda").manual_seed(hd)
    pool = _random_pool(torch, f3c, gen, lens, kv, hd)
    off = [0] + [int(x) for x in np.cumsum(nq)]
    q = torch.randn(off[-1], heads * hd, generator=gen, device="cuda").bfloat16()
    outs = [torch.empty_like(q) for _ in range(4)]
    say("rows at once", hd, heads, nq, lens)

    def call(o):
        f3c.op_cache8_attention(pool, heads, off, lens, q, o, causal=True)

    call(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[1])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for o in outs[1:]:
            o.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        for s, o in zip(streams, outs[2:]):
            with torch.cuda.stream(s):
                call(o)
        torch.cuda.synchronize()
        assert all(torch.equal(o, outs[0]) for o in outs[1:])
