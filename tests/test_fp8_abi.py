"""Refusals of the 8-bit operators: every bad argument is an error before any device work (no GPU needed: the pointers
here are host addresses that nothing reads)."""
import ctypes

import numpy as np
import pytest

from paper_2511_22533_amd import f3c

P = 1 << 20              # an aligned address


def _quant(**kw):
    a = dict(dtype=1, block_rows=1, rows=4, K=256, x=P, ldx=256, q=P, ldq=256, scale=P, lds=4)
    a.update(kw)
    return f3c.lib().f3c_op_quant_fp8(*a.values(), None)


def _gemm(**kw):
    a = dict(epi=0, M=4, N=256, K=256, A=P, lda=256, sa=P, ldsa=4, W=P, ldw=256, sw=P, ldsw=4, bias=P, gate=None, out=P,
             ldo=256, so=None, ldso=0, resid=None, ldr=0)
    a.update(kw)
    return f3c.lib().f3c_op_gemm_fp8(*a.values(), None)


def _norm(cfg=None, off=(0, 4), null_cfg=False, **kw):
    c = dict(dtype=1, out_dtype=2, post=1, pre=2, eps=1e-6, rs=1.0)
    c.update(cfg or {})
    a = dict(d=256, batch=len(off) - 1, off=(ctypes.c_int32 * len(off))(*off), y=P, ldy=256, post_w=P, gate=P, h=P,
             ldh=256, pre_w=P, shift=P, scale=P, ldm=0, out=P, ldo=256, so=P, lds=4)
    a.update(kw)
    s = f3c.ResidNormCfg(*c.values())
    return f3c.lib().f3c_op_resid_norm(None if null_cfg else ctypes.byref(s), *a.values(), None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dtype=-1), dict(block_rows=2), dict(block_rows=0), dict(rows=-1),
                                dict(K=0), dict(K=100), dict(x=None), dict(q=None), dict(scale=None), dict(ldx=248),
                                dict(ldx=257), dict(ldq=250), dict(ldq=260), dict(x=P + 8), dict(q=P + 4),
                                dict(scale=P + 1), dict(lds=1), dict(lds=6), dict(K=520, ldx=520, ldq=520, lds=4),
                                dict(rows=1 << 28, K=128),
                                dict(rows=(1 << 31) - 1, K=264, ldx=264, ldq=264, block_rows=128)])
def test_quant_refuses(kw):
    assert _quant(**kw) == f3c.F3C_EINVAL
    assert f3c.lib().f3c_last_error()


@pytest.mark.parametrize("kw", [dict(epi=-1), dict(epi=4), dict(M=-1), dict(M=1 << 30), dict(N=0), dict(K=0), dict(N=250),
                                dict(K=264),
                                dict(A=None), dict(W=None), dict(sa=None), dict(sw=None), dict(lda=240), dict(ldw=240),
                                dict(lda=264), dict(ldw=264), dict(lda=1 << 22), dict(ldw=1 << 22), dict(A=P + 8),
                                dict(W=P + 4), dict(sa=P + 2), dict(sw=P + 2), dict(ldsa=1), dict(ldsw=5),
                                dict(bias=P + 4), dict(gate=P), dict(out=None), dict(ldo=248), dict(ldo=260),
                                dict(out=P + 8), dict(epi=2), dict(epi=2, resid=P, ldr=250),
                                dict(epi=2, resid=P, ldr=258), dict(epi=2, resid=P, ldr=256, gate=P + 8),
                                dict(epi=3), dict(epi=3, so=P, ldso=1), dict(epi=3, so=P + 1, ldso=4),
                                dict(epi=3, so=P, ldso=4, ldo=264)])
def test_gemm_refuses(kw):
    assert _gemm(**kw) == f3c.F3C_EINVAL
    assert f3c.lib().f3c_last_error()


@pytest.mark.parametrize("cfg,kw", [
    (dict(dtype=2), {}), (dict(out_dtype=3), {}), (dict(out_dtype=-1), {}), (dict(post=3), {}), (dict(pre=-1), {}),
    (dict(eps=0.0), {}), (dict(eps=-1.0), {}), (dict(eps=float("nan")), {}), (dict(eps=float("inf")), {}),
    (dict(rs=float("nan")), {}), ({}, dict(d=0)), ({}, dict(d=12)), ({}, dict(d=8200)), ({}, dict(batch=0)),
    ({}, dict(batch=65)), ({}, dict(off=(3, 2))), ({}, dict(off=(-1, 2))), ({}, dict(off=None, batch=1)),
    ({}, dict(h=None)), ({}, dict(ldh=252)), ({}, dict(ldh=258)), ({}, dict(h=P + 4)), ({}, dict(ldy=248)),
    ({}, dict(ldy=260)), ({}, dict(y=P + 8)), ({}, dict(ldo=252)), ({}, dict(out=P + 4)), ({}, dict(so=None)),
    ({}, dict(lds=1)), ({}, dict(so=P + 2)), ({}, dict(shift=None)), ({}, dict(scale=None)), ({}, dict(ldm=128)),
    ({}, dict(ldm=258)), ({}, dict(gate=P + 4)), ({}, dict(post_w=P + 8)), ({}, dict(pre_w=P + 8)),
    (dict(out_dtype=0), dict(ldo=258)), (dict(out_dtype=1), dict(ldo=260))])
def test_resid_norm_refuses(cfg, kw):
    if "off" in kw and kw["off"] is None:
        kw = dict(kw, off=(0, 4))
        s = f3c.ResidNormCfg(1, 2, 1, 2, 1e-6, 1.0)
        assert f3c.lib().f3c_op_resid_norm(ctypes.byref(s), 256, 1, None, P, 256, P, P, P, 256, P, P, P, 0, P, 256, P,
                                           4, None) == f3c.F3C_EINVAL
        return
    assert _norm(cfg, **kw) == f3c.F3C_EINVAL
    assert f3c.lib().f3c_last_error()
    assert _norm(null_cfg=True) == f3c.F3C_EINVAL


@pytest.mark.parametrize("call,kw", [
    # 2^32 threads, or a block count past 32 bits
    (_quant, dict(rows=(1 << 28) - 15, K=128, ldx=128, ldq=128)),
    (_quant, dict(rows=(1 << 26) - 3, K=512, ldx=512, ldq=512)),
    (_quant, dict(rows=1, K=(1 << 31) - 8, ldx=(1 << 31) - 8, ldq=(1 << 31) - 8, lds=1 << 24)),
    (_quant, dict(rows=1, K=1 << 30, ldx=1 << 30, ldq=1 << 30, lds=1 << 23, block_rows=128)),
    (_quant, dict(rows=(1 << 31) - 1, K=128, ldx=128, ldq=128, lds=4, block_rows=128)),
    (_gemm, dict(M=(1 << 30) - 1, N=16, K=16)),
    (_gemm, dict(M=(1 << 29) + 1, N=64, K=16)),
    (_gemm, dict(M=1, N=(1 << 30) - 16, ldo=(1 << 30) - 16)),
    (_gemm, dict(M=1 << 25, N=1 << 10, K=128, ldo=1 << 10))])
def test_more_than_a_launch_holds_is_refused(call, kw):
    assert call(**kw) == f3c.F3C_EINVAL
    assert f3c.lib().f3c_last_error()


def test_no_rows_is_no_work():
    assert _quant(rows=0, x=None, q=None, scale=None) == f3c.F3C_OK
    assert _gemm(M=0, A=None, sa=None, out=None) == f3c.F3C_OK
    assert _norm(off=(5, 5, 5), h=None, y=None, out=None, so=None) == f3c.F3C_OK


def test_bindings_refuse_what_does_not_fit():
    import torch
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t)  # noqa: E731
    u8, f8, bf = torch.uint8, torch.float8_e4m3fn, torch.bfloat16
    bad = [
        lambda: f3c.op_quant_fp8(f3c.F3C_BF16, e(4, 256), e(4, 256, t=u8), e(4, 4, t=u8)),
        lambda: f3c.op_quant_fp8(f3c.F3C_FP8, e(4, 256, t=u8), e(4, 256, t=u8), e(4, 4, t=u8)),
        lambda: f3c.op_quant_fp8(f3c.F3C_F32, e(256, 4).t(), e(4, 256, t=u8), e(4, 4, t=u8)),
        lambda: f3c.op_quant_fp8(f3c.F3C_F32, e(4, 256), e(4, 256, t=u8), e(4, 4, t=u8)),      # not on the GPU
        lambda: f3c.op_quant_fp8(f3c.F3C_F32, e(4, 256), e(4, 256, t=u8), e(4, 4, t=u8), block_rows=64),
        lambda: f3c.op_gemm_fp8(5, e(4, 256, t=f8), e(4, 4, t=u8), e(256, 256, t=f8), e(2, 4, t=u8)),
        lambda: f3c.op_gemm_fp8(0, e(4, 256, t=bf), e(4, 4, t=u8), e(256, 256, t=f8), e(2, 4, t=u8)),
        lambda: f3c.op_resid_norm(f3c.F3C_FP8, f3c.F3C_F32, e(4, 256)),
        lambda: f3c.op_resid_norm(f3c.F3C_F32, 7, e(4, 256)),
        lambda: f3c.op_resid_norm(f3c.F3C_F32, f3c.F3C_F32, e(4, 256, t=bf)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()


def test_scale_stride():
    assert [f3c.fp8_scale_stride(n) for n in (1, 128, 129, 512, 513, 1024)] == [4, 4, 4, 4, 8, 8]


def test_resid_norm_takes_scalars_as_they_are_at_the_call(monkeypatch):
    """Scalars held in a tensor or an array that changes between calls, and zeros of either sign, reach the library with
    the values that they have at each call."""
    import torch
    got = []

    class Library:
        def f3c_op_resid_norm(self, cfg, *rest):
            got.append((cfg._obj.eps, cfg._obj.resid_scale))
            return f3c.F3C_OK

    monkeypatch.setattr(f3c, "_lib", Library())
    monkeypatch.setattr(f3c, "_device", lambda t, torch: t.get_device())
    monkeypatch.setattr(f3c, "_stream_on", lambda *a: 0)
    h = torch.zeros(2, 8)
    call = lambda **kw: f3c.op_resid_norm(f3c.F3C_F32, f3c.F3C_F32, h, y=h, **kw)  # noqa: E731
    for scale, eps in ((torch.tensor(0.5), torch.tensor(0.25)), (np.array(0.5), np.array(0.25))):
        got.clear()
        call(resid_scale=scale, eps=eps)
        scale[...], eps[...] = 2.0, 0.125
        call(resid_scale=scale, eps=eps)
        assert got == [(0.25, 0.5), (0.125, 2.0)]
    got.clear()
    call(resid_scale=0.0)
    call(resid_scale=-0.0)
    assert [np.signbit(s) for _, s in got] == [False, True]
