"""Which form of the 8-bit cache's attention a call takes (no GPU): the cost model again in Python, from the table as it stands
in the source and held against the library's own sizes of workspace; the tests of the forms reach the ones they name.
"""
import ctypes
import math
import os
import random
import re

import pytest

from paper_2511_22533_amd import build, f3c
from test_gpu_cache8 import ROWS
from test_gpu_cache8_far import DEEP, FORMS
from test_gpu_cache8_long import LONG

with open(os.path.join(build.CSRC, "k_cache8.hip")) as _f:
    _text = _f.read()
_body = _text[_text.index("kForms[] = {"):]
TABLE = [[float(x) for x in r.split(",")] for r in re.findall(r"\{([-\d., ]+)\}", _body[:_body.index("};")])]
CONST = {n: float(re.search(rf"\b{n} = ([\d.e]+)[,;]", _text).group(1)) for n in
         ("kLaunchUs", "kJoinUs", "kJoinSplitUs", "kPartialBytesPerUs", "kReadBytesPerUs", "kSplitRounds", "kLeastSplit")}


def form(hd, kv, heads, nq, lens, causal, ws=math.inf):
    """(rows of a tile, groups of waves, pages split, items with their heads, bytes of partial results)."""
    group, B = heads // kv, len(nq)
    pages = [-(-n // 64) for n in lens]
    order = sorted(range(B), key=lambda b: -pages[b])
    most_rows = max(n * group for n in nq)
    ragged = causal or any(n != lens[0] for n in lens)
    longest = max([1] + [max(pages[b], 1) for b in range(B) if nq[b]])
    best = None
    for rows, width, groups, first, page, own in TABLE:
        if width != hd or (rows > 16 and most_rows <= 16):
            continue
        tiles = {b: -(-nq[b] * group // int(rows)) for b in order}
        work = read = whole = 0.0
        for b in order:
            unseen = 0.0
            if causal and nq[b]:
                unseen = nq[b] / 128.0 if nq[b] <= lens[b] else pages[b] - pages[b] * lens[b] / (2.0 * nq[b])
            work += tiles[b] * max(pages[b] - unseen, 0.5) * kv
            whole += tiles[b] * kv
            read += 2.0 * pages[b] * 64 * hd * kv if tiles[b] else 0.0
        k = 1
        while k <= 128:
            p = -(-longest // k)
            if k > 1 and p < CONST["kLeastSplit"]:
                break
            items = kv * sum(tiles[b] * max(1, -(-pages[b] // p)) for b in order)
            need = 0.0 if k < 2 else items * rows * (hd + 2) * 4.0
            if k > 1 and (need > ws or items >= 1 << 23 or items * rows * (hd // 4) >= 1 << 31):
                break
            per_cu, load = items / 256.0, work / 256.0
            if rows == 16:
                t = max(load * page + per_cu * own, p * first / (8.0 if items <= 256 else 4.0), read / CONST["kReadBytesPerUs"])
            elif per_cu <= 1.0:
                t = p * first + own
            else:
                if ragged:
                    mean = load / per_cu
                    least = max(2.0 * mean - p, 0.0)
                    after = p - (p - least) / per_cu
                    cu = max(2.0 * after if groups > 1 else p + after, load + (0.33 if groups > 1 else 0.38) * mean)
                else:
                    cu = load * (1.0 + (math.ceil(per_cu) / per_cu - 1.0) * (0.89 if groups > 1 else 0.97))
                t = max(p * first, cu * page) + per_cu * own
            t += CONST["kLaunchUs"]
            if k > 1:
                t += CONST["kJoinUs"] + CONST["kJoinSplitUs"] * k + 2.0 * need / CONST["kPartialBytesPerUs"]
                if rows > 16 and whole > 256.0:
                    t *= CONST["kSplitRounds"]
            if best is None or t < best[0]:
                split = any(tiles[b] and pages[b] > p for b in order)
                # (a sample without queries has no items)
                best = (t, (int(rows), int(groups), split, items, int(items * rows * (hd + 2) * 4) if split else 0))
            k = k + 1 if k < 4 else 2 * k
    return best[1]


def _bytes(hd, kv, heads, nq, lens, causal):
    ints = lambda v: (ctypes.c_int32 * len(v))(*v)  # noqa: E731
    off = [0]
    for n in nq:
        off.append(off[-1] + n)
    size = ctypes.c_size_t(0)
    args = f3c.Cache8Args(kv, hd, 1, 1 << 20, None, None, None, None, None)
    f3c.check(f3c.lib().f3c_op_cache8_attention_bytes(args, heads, len(nq), ints(off), ints(lens), int(causal), size))
    return size.value


def test_the_model_here_is_the_librarys():
    rng, seen = random.Random(3), set()
    for _ in range(3000):
        hd, kv = rng.choice([32, 64, 128]), rng.choice([1, 2, 4, 5, 8, 16])
        heads, B = kv * rng.choice([1, 2, 4, 7]), rng.choice([1, 1, 2, 5, 64])
        lens = [int(2 ** rng.uniform(0, 16)) for _ in range(B)]
        nq = [int(2 ** rng.uniform(0, 13)) - rng.randint(0, 1) for _ in range(B)]
        call = (hd, kv, heads, nq, lens, rng.random() < 0.5)
        want = form(*call)
        assert _bytes(*call) == want[4], call
        seen.add((hd,) + want[:3])
    assert len(seen) > 20


# (256 rows of 32 columns in one group take no call in one piece: their samples that are not split have others beside them)
REACHED = {(hd, rows, groups, split) for hd in (32, 64, 128) for rows, groups in ((16, 1), (128, 1), (128, 2), (256, 1), (256, 2))
           for split in (False, True) if not (hd == 128 and rows == 256)
           and (hd, rows, groups, split) != (32, 256, 1, False) and not (rows == 16 and groups == 2)}


def test_calls_far_out_reach_every_form():
    assert {(c[0],) + form(*c)[:3] for c in FORMS} == REACHED


def test_deep_calls_look_pages_up_twice():
    forms = [form(*c, ws=0) for c in DEEP]
    assert all(-(-c[4][0] // 64) > 64 * f[1] for c, f in zip(DEEP, forms))
    assert {(c[0],) + f[:2] for c, f in zip(DEEP, forms)} == {r[:3] for r in REACHED if r[1] > 16} - {(32, 256, 1)}


def test_calls_of_many_rows_reach_every_form_of_theirs():
    assert {(c[0],) + form(c[0], c[1], c[2], *c[3:])[:3] for c in ROWS} >= {r for r in REACHED if r[1] > 16}


@pytest.mark.parametrize("hd,kv,heads,nq,lens,waves", LONG)
def test_long_calls_take_more_than_64_pages_a_wave(hd, kv, heads, nq, lens, waves):
    rows, groups, split, items, size = form(hd, kv, heads, nq, lens, True, ws=0)
    assert (rows, groups, split, size) == (16, 1, False, 0) and (8 if items <= 256 else 4) == waves
    assert max(lens) > 64 * 64 * waves
