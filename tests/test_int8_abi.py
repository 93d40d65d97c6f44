"""Refusals of the integer products and of the 8-bit cache: every bad argument is an error before any device work (no
GPU needed: the pointers here are host addresses that nothing reads)."""
import ctypes

import numpy as np
import pytest

from paper_2511_22533_amd import f3c

P = 1 << 20              # an aligned address


def _quant(**kw):
    a = dict(dtype=1, rows=4, K=256, x=P, ldx=256, q=P, ldq=256, scale=P)
    a.update(kw)
    return f3c.lib().f3c_op_quant_i8(*a.values(), None)


def _gemm(**kw):
    a = dict(epi=0, M=4, N=256, K=256, A=P, lda=256, sa=P, W=P, ldw=256, sw=P, bias=P, gate=None, out=P, ldo=256,
             resid=None, ldr=0)
    a.update(kw)
    return f3c.lib().f3c_op_gemm_i8(*a.values(), None)


def _ints(v):
    return None if v is None else (ctypes.c_int32 * len(v))(*v)


def _cache(kw):
    c = dict(kv_heads=4, head_dim=64, n_pages=9, max_pages=4, k=P, v=P, k_scale=P, v_scale=P, table=P)
    c.update({n: kw.pop(n) for n in list(kw) if n in c})
    return None if kw.pop("null", False) else ctypes.byref(f3c.Cache8Args(*c.values()))


def _append(**kw):
    c = _cache(kw)
    a = dict(dtype=1, batch=2, lens=(5, 200), off=(0, 1, 3), x=P, ldx=256, y=P, ldy=256)
    a.update(kw)
    a["lens"], a["off"] = _ints(a["lens"]), _ints(a["off"])
    return f3c.lib().f3c_op_cache8_append(c, *a.values(), None)


def _attn(**kw):
    c = _cache(kw)
    a = dict(heads=8, batch=2, off=(0, 1, 3), lens=(5, 256), q=P, ldq=512, o=P, ldo=512, causal=0, pre=0, ws=None, size=0)
    a.update(kw)
    a["lens"], a["off"] = _ints(a["lens"]), _ints(a["off"])
    return f3c.lib().f3c_op_cache8_attention(c, *a.values(), None)


def _bytes(**kw):
    c = _cache(kw)
    out = ctypes.c_size_t(77)
    a = dict(heads=8, batch=2, off=(0, 1, 3), lens=(5, 256), causal=0)
    a.update(kw)
    a["lens"], a["off"] = _ints(a["lens"]), _ints(a["off"])
    return f3c.lib().f3c_op_cache8_attention_bytes(c, *a.values(), ctypes.byref(out)), out.value


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 24), dict(K=0),
                                dict(K=100), dict(K=1 << 30, ldx=1 << 30, ldq=1 << 30), dict(x=None), dict(q=None),
                                dict(scale=None), dict(ldx=248), dict(ldx=257), dict(ldq=250), dict(ldq=260),
                                dict(x=P + 8), dict(q=P + 4), dict(scale=P + 2)])
def test_quant_refuses(kw):
    assert _quant(**kw) == f3c.F3C_EINVAL
    assert f3c.lib().f3c_last_error()


@pytest.mark.parametrize("kw", [dict(epi=-1), dict(epi=3), dict(M=-1), dict(M=1 << 30), dict(N=0), dict(K=0), dict(N=250),
                                dict(K=264), dict(K=133136, lda=133136, ldw=133136), dict(A=None), dict(W=None),
                                dict(sa=None), dict(sw=None), dict(sa=P + 2), dict(sw=P + 1), dict(lda=240),
                                dict(ldw=240), dict(lda=264), dict(ldw=264), dict(lda=1 << 22), dict(ldw=1 << 22),
                                dict(A=P + 8), dict(W=P + 4), dict(bias=P + 4), dict(gate=P), dict(out=None),
                                dict(ldo=248), dict(ldo=260), dict(out=P + 8), dict(epi=2), dict(epi=2, resid=P, ldr=250),
                                dict(epi=2, resid=P, ldr=258), dict(epi=2, resid=P + 8, ldr=256),
                                dict(epi=2, resid=P, ldr=256, gate=P + 8), dict(M=(1 << 30) - 1, N=16, K=16),
                                dict(M=1 << 25, N=1 << 10, K=128, ldo=1 << 10)])
def test_gemm_refuses(kw):
    assert _gemm(**kw) == f3c.F3C_EINVAL
    assert f3c.lib().f3c_last_error()


CACHE = [dict(null=True), dict(kv_heads=0), dict(kv_heads=1025), dict(head_dim=0), dict(head_dim=48), dict(head_dim=256),
         dict(n_pages=-1), dict(max_pages=-1), dict(max_pages=(1 << 24) + 1), dict(off=None), dict(lens=None),
         dict(batch=0), dict(batch=65), dict(off=(1, 0, 3)), dict(off=(-1, 0, 3)), dict(lens=(-1, 5)),
         dict(lens=(5, 257)), dict(max_pages=0)]
MEMORY = [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(table=None), dict(k=P + 8),
          dict(v=P + 4), dict(table=P + 2)]


@pytest.mark.parametrize("kw", CACHE + MEMORY + [
    dict(dtype=2), dict(x=None), dict(y=None), dict(ldx=248), dict(ldy=248), dict(ldx=260), dict(ldy=260), dict(x=P + 8),
    dict(y=P + 2), dict(lens=(5, 255)),                        # 255 + 2 tokens in four pages
    dict(lens=(0, 0), off=(0, 0, 2147483647), max_pages=1 << 24, n_pages=1 << 24)])
def test_append_refuses(kw):
    assert _append(**kw) == f3c.F3C_EINVAL
    assert f3c.lib().f3c_last_error()


@pytest.mark.parametrize("kw", CACHE + [dict(heads=0), dict(heads=6), dict(heads=65536), dict(causal=2),
                                        dict(off=(0, 0, 1 << 27), heads=4)])
def test_attention_refuses(kw):
    assert _attn(**kw) == f3c.F3C_EINVAL and f3c.lib().f3c_last_error()
    assert _bytes(**kw)[0] == f3c.F3C_EINVAL


@pytest.mark.parametrize("kw", MEMORY + [dict(pre=2), dict(q=None), dict(o=None), dict(ldq=504), dict(ldo=508),
                                         dict(ldq=516), dict(ldo=514), dict(q=P + 8), dict(o=P + 4), dict(ws=P + 8)])
def test_attention_refuses_memory(kw):
    assert _attn(**kw) == f3c.F3C_EINVAL
    assert f3c.lib().f3c_last_error()


def test_no_rows_is_no_work():
    assert _quant(rows=0, x=None, q=None, scale=None) == f3c.F3C_OK
    assert _gemm(M=0, A=None, sa=None, out=None) == f3c.F3C_OK
    assert _append(off=(3, 3, 3), x=None, y=None) == f3c.F3C_OK
    assert _append(off=(0, 0, 0), lens=(0, 0), max_pages=0, table=None, n_pages=0, k=None, v=None, k_scale=None,
                   v_scale=None) == f3c.F3C_OK
    assert _attn(off=(3, 3, 3), q=None, o=None) == f3c.F3C_OK


def test_workspace_bytes_ask_for_no_memory():
    no = dict(k=None, v=None, k_scale=None, v_scale=None, table=None)
    assert _bytes(**no) == (f3c.F3C_OK, 0)                     # a few pages: one workgroup takes them
    rc, size = _bytes(off=(0, 0, 1), lens=(0, 64 * 2000), max_pages=2000, **no)
    assert rc == f3c.F3C_OK and size > 0 and size % 4 == 0
    assert f3c.lib().f3c_op_cache8_attention_bytes(_cache({}), 8, 2, _ints((0, 1, 3)), _ints((5, 256)), 0,
                                                   None) == f3c.F3C_EINVAL


def test_bindings_refuse_what_does_not_fit():
    import torch
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t)  # noqa: E731
    u8, i8, bf, i32 = torch.uint8, torch.int8, torch.bfloat16, torch.int32
    cache = f3c.Cache8(e(3, 2, 64, 32, t=u8), e(3, 2, 32, 64, t=u8), e(3, 2, t=u8), e(3, 2, t=u8), e(1, 3, t=i32))
    bad = [
        lambda: f3c.op_quant_i8(f3c.F3C_FP8, e(4, 256), e(4, 256, t=i8), e(4)),
        lambda: f3c.op_quant_i8(f3c.F3C_F32, e(4, 256), e(4, 256, t=i8), e(4)),                  # not on the GPU
        lambda: f3c.op_gemm_i8(3, e(4, 256, t=i8), e(4), e(256, 256, t=i8), e(256)),
        lambda: f3c.op_gemm_i8(0, e(4, 256, t=i8), e(4), e(256, 256, t=i8), e(256)),
        lambda: f3c.op_gemm_i8(2, e(4, 256, t=i8), e(4), e(256, 256, t=i8), e(256), out=e(4, 256, t=bf)),
        lambda: f3c.op_gemm_i8(0, e(4, 256, t=i8), None, e(256, 256, t=i8), e(256), out=e(4, 256, t=bf)),
        lambda: f3c.op_cache8_append(f3c.F3C_FP8, cache, [0], [0, 2], e(2, 64, t=bf), e(2, 64, t=bf)),
        lambda: f3c.op_cache8_append(f3c.F3C_BF16, cache, [0], [0, 2], e(2, 64, t=bf), e(2, 64, t=bf)),
        lambda: f3c.op_cache8_attention(cache, 2, [0, 1], [4], e(1, 64, t=bf), e(1, 64, t=bf)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()


def test_bindings_look_at_the_cache(monkeypatch):
    """A cache whose tensors do not belong together is refused (checks that need no GPU)."""
    import torch
    monkeypatch.setattr(f3c, "_device", lambda t, torch: t.get_device())
    monkeypatch.setattr(f3c, "_stream_on", lambda *a: 0)
    e = lambda *s, t=torch.uint8: torch.empty(*s, dtype=t)  # noqa: E731
    good = dict(k=e(3, 2, 64, 32), v=e(3, 2, 32, 64), k_scale=e(3, 2), v_scale=e(3, 2), table=e(1, 3, t=torch.int32))
    q = e(1, 64, t=torch.bfloat16)
    for name, t in [("k", e(3, 2, 32, 32)), ("k", e(3, 64, 32)), ("k", e(3, 2, 64, 32, t=torch.int8)),
                    ("v", e(3, 2, 64, 32)), ("v", e(2, 2, 32, 64)), ("k_scale", e(3, 1)), ("v_scale", e(2, 3)),
                    ("k_scale", e(3, 2, t=torch.float32)), ("table", e(0, 3, t=torch.int32)),
                    ("table", e(1, 3, t=torch.int64)), ("table", e(3, t=torch.int32)),
                    ("k", e(3, 64, 2, 32).transpose(1, 2)), ("table", e(3, 1, t=torch.int32).t()[:, ::2])]:
        with pytest.raises(ValueError, match="cache"):
            f3c.op_cache8_attention(f3c.Cache8(**dict(good, **{name: t})), 2, [0, 1], [4], q, q)
    for off, lens in (([0, 2], [4]), ([-1, 1], [4]), ([0, 1], [4, 4]), ([0], [])):
        with pytest.raises(ValueError, match="off"):
            f3c.op_cache8_attention(f3c.Cache8(**good), 2, off, lens, q, q)


def test_host_lists_of_any_integers(monkeypatch):
    """Lengths and offsets as lists, tuples, NumPy arrays, elements of tensors: the values at the call; none that 32 bits
    do not hold."""
    import torch
    got = []

    class Library:
        def f3c_op_cache8_append(self, args, dtype, batch, held, off, *rest):
            got.append([list((ctypes.c_int32 * n).from_address(a)) for a, n in ((held, batch), (off, batch + 1))])
            return f3c.F3C_OK

    monkeypatch.setattr(f3c, "_lib", Library())
    monkeypatch.setattr(f3c, "_device", lambda t, torch: t.get_device())
    monkeypatch.setattr(f3c, "_stream_on", lambda *a: 0)
    e = lambda *s, t=torch.uint8: torch.empty(*s, dtype=t)  # noqa: E731
    cache = f3c.Cache8(e(3, 2, 64, 32), e(3, 2, 32, 64), e(3, 2), e(3, 2), e(2, 3, t=torch.int32))
    k = e(4, 64, t=torch.bfloat16)
    for lens, off in (([5, 0], [0, 1, 4]), ((5, 0), (0, 1, 4)), (np.array([5, 0]), np.array([0, 1, 4], np.int64)),
                      ([np.int32(5), torch.tensor(0)], torch.tensor([0, 1, 4]))):
        f3c.op_cache8_append(f3c.F3C_BF16, cache, lens, off, k, k)
    assert got == [[[5, 0], [0, 1, 4]]] * 4
    for lens, off in (([2 ** 32 + 5, 0], [0, 1, 4]), ([5, 0], [0, 1, 2 ** 32 + 4]), ([5, -2 ** 31 - 1], [0, 1, 4])):
        with pytest.raises(ValueError, match="32-bit"):
            f3c.op_cache8_append(f3c.F3C_BF16, cache, lens, off, k, k)
    assert len(got) == 4
