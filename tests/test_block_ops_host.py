"""Refusals of the gated linears, the block norms and the rotary positions, all before any launch."""
import pytest
import torch

from paper_2605_26632_amd import binding as rtl

FAKE = 0x10000      # non-null, aligned, never dereferenced
NULL, SHAPE, ALIGN, WORKSPACE, ARG = 1, 2, 3, 4, 5
BIG = 1 << 30
NAN = float("nan")


def caller(name, defaults):
    def f(**kw):
        assert set(kw) <= set(defaults)
        return getattr(rtl.lib(), name)(*dict(defaults, **kw).values())
    return f


def passes(status):
    """Through the argument checks: what is left is the device, which has no GPU here (or runs: then the call was not made)."""
    return status in (6, 7)


no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses pass the checks")


def gated():
    return caller("rtl_gated_linear", dict(X=FAKE, W=FAKE, bias=None, H=FAKE, P=None, act=0, M=16, F=24, K=64, ldx=64, ldw=64, ldh=24, ldp=48, stream=None))


def test_gated_refusals():
    f = gated()
    assert f(act=3) == ARG and f(act=-1) == ARG
    assert f(M=-1) == SHAPE and f(F=-1) == SHAPE and f(K=0) == SHAPE and f(K=96) == SHAPE and f(F=(1 << 29) + 1, ldh=BIG) == SHAPE and f(M=BIG + 1) == SHAPE
    assert f(ldx=56) == SHAPE and f(ldw=56) == SHAPE and f(ldh=23) == SHAPE and f(P=FAKE, ldp=47) == SHAPE
    assert f(ldx=(1 << 22) + 8) == SHAPE and f(ldw=(1 << 22) + 8) == SHAPE
    assert f(M=BIG, F=1 << 20, ldh=1 << 20) == SHAPE                  # 2^23 tiles and more
    for p in ("X", "W", "H"):
        assert f(**{p: None}) == NULL and f(**{p: FAKE + 1}) == ALIGN
    assert f(ldx=68) == ALIGN and f(ldw=68) == ALIGN and f(bias=FAKE + 1) == ALIGN and f(P=FAKE + 1) == ALIGN
    assert f(M=0) == 0 and f(F=0, ldh=0) == 0


@no_gpu
def test_gated_accepts():
    f = gated()
    assert passes(f()) and passes(f(ldh=25, H=FAKE + 2)) and passes(f(P=FAKE + 2, ldp=49, act=2)) and passes(f(F=1, ldh=1)) and passes(f(ldp=0))


def gated_backward():
    return caller("rtl_gated_linear_backward", dict(dH=FAKE, X=FAKE, W=FAKE, P=FAKE, dX=FAKE, dW=FAKE, db=FAKE, H=FAKE, act=0, type=0, M=16, F=24, K=64, lddh=24,
                                                    ldx=64, ldw=64, ldp=48, lddx=64, lddw=64, ldh=24, ws=FAKE, wsb=1 << 20, stream=None))


def test_gated_backward_refusals():
    f = gated_backward()
    assert f(act=3) == ARG and f(type=2) == ARG
    assert f(M=-1) == SHAPE and f(F=22) == SHAPE and f(K=60) == SHAPE and f(K=0) == SHAPE and f(F=(1 << 21) + 4) == SHAPE
    assert f(F=0) == SHAPE and f(F=0, dX=None) == 0
    assert f(lddh=20) == SHAPE and f(ldp=47) == SHAPE and f(ldh=20) == SHAPE and f(ldx=56) == SHAPE and f(ldw=56) == SHAPE and f(lddx=56) == SHAPE
    assert f(lddw=56) == SHAPE and f(lddw=(1 << 22) + 8) == SHAPE
    assert f(dH=None) == NULL and f(P=None) == NULL and f(X=None) == NULL and f(W=None) == NULL and f(dW=None) == NULL
    for p in ("X", "W", "dX", "dW"):
        assert f(**{p: FAKE + 8}) == ALIGN
    assert f(dH=FAKE + 1) == ALIGN and f(db=FAKE + 1) == ALIGN and f(db=FAKE + 2, type=1) == ALIGN and f(ldx=68) == ALIGN and f(lddw=68) == ALIGN
    need = 4 * 16 * 24
    assert f(ws=None) == WORKSPACE and f(wsb=need - 1) == WORKSPACE and f(ws=FAKE + 64) == ALIGN
    assert f(M=0, dW=None, db=None) == 0
    assert rtl.gated_linear_backward_workspace(16, 24, 64) >= need and rtl.gated_linear_backward_workspace(-1, 24, 64) == 0


@no_gpu
def test_gated_backward_accepts():
    f = gated_backward()
    assert passes(f()) and passes(f(wsb=4 * 16 * 24)) and passes(f(X=None, dW=None, db=None, ldx=0, lddw=0)) and passes(f(W=None, dX=None, ldw=0, lddx=0))
    assert passes(f(H=None, ldh=0)) and passes(f(X=None, W=None, dX=None, dW=None, db=None, K=0)) and passes(f(M=0)) and passes(f(dH=FAKE + 2, lddh=25, P=FAKE + 2, ldp=49))


def norm():
    return caller("rtl_residual_norm", dict(x=FAKE, y=FAKE, gate=FAKE, w_post=FAKE, w_pre=FAKE, scale=FAKE, shift=FAKE, off=FAKE, xo=FAKE, h=FAKE, type=0, post=1,
                                            pre=2, alpha=1.0, eps=1e-6, clear=0, T=16, S=3, D=64, ldx=64, ldy=64, ldg=64, ldm=64, ldxo=64, ldh=64, stream=None))


def check_norm(f):
    assert f(type=2) == ARG and f(post=3) == ARG and f(pre=-1) == ARG and f(alpha=NAN) == ARG and f(alpha=float("inf")) == ARG and f(eps=-1.0) == ARG and f(eps=NAN) == ARG
    assert f(T=-1) == SHAPE and f(T=1 << 24) == SHAPE and f(S=-1) == SHAPE and f(S=65536) == SHAPE and f(D=60) == SHAPE and f(D=-8) == SHAPE and f(D=8200) == SHAPE
    assert f(off=None) == SHAPE                                    # one sequence only without offsets
    assert f(off=FAKE + 2) == ALIGN
    assert f(ldy=56) == SHAPE and f(ldg=56) == SHAPE and f(ldm=56) == SHAPE and f(ldxo=56) == SHAPE and f(ldg=0) == SHAPE
    for p in ("y", "gate", "w_post", "w_pre", "scale"):
        assert f(**{p: FAKE + 8}) == ALIGN
    assert f(ldy=68) == ALIGN and f(ldg=68) == ALIGN and f(ldm=68) == ALIGN and f(ldxo=68) == ALIGN and f(D=0) == 0


def test_norm_refusals():
    f = norm()
    check_norm(f)
    assert f(x=None) == NULL and f(xo=None, h=None) == NULL
    assert f(ldx=56) == SHAPE and f(ldh=56) == SHAPE and f(x=FAKE + 8) == ALIGN and f(xo=FAKE + 8) == ALIGN and f(h=FAKE + 8) == ALIGN and f(shift=FAKE + 8) == ALIGN
    assert f(ldx=66, type=1) == ALIGN and f(T=0) == 0


@no_gpu
def test_norm_accepts():
    f = norm()
    assert passes(f()) and passes(f(type=1, ldx=68)) and passes(f(xo=None, ldxo=0)) and passes(f(h=None, ldh=0)) and passes(f(y=None, ldy=0))
    assert passes(f(off=None, S=1)) and passes(f(S=0)) and passes(f(gate=None, ldg=0, scale=None, shift=None, ldm=0, w_post=None, w_pre=None))


def norm_backward():
    return caller("rtl_residual_norm_backward", dict(dxo=FAKE, dh=FAKE, xo=FAKE, y=FAKE, gate=FAKE, w_post=FAKE, w_pre=FAKE, scale=FAKE, off=FAKE, dx=FAKE, dy=FAKE,
                                                     dgate=FAKE, dscale=FAKE, dshift=FAKE, dw_post=FAKE, dw_pre=FAKE, type=0, post=1, pre=2, alpha=1.0, eps=1e-6,
                                                     clear=0, T=16, S=3, D=64, lddxo=64, lddh=64, ldxo=64, ldy=64, ldg=64, ldm=64, lddx=64, lddy=64, ws=FAKE,
                                                     wsb=1 << 30, stream=None))


def test_norm_backward_refusals():
    f = norm_backward()
    check_norm(f)
    assert f(dxo=None, dh=None) == NULL and f(xo=None) == NULL and f(y=None) == NULL
    assert f(lddx=56) == SHAPE and f(lddy=56) == SHAPE and f(lddh=56) == SHAPE and f(lddxo=56) == SHAPE
    for p in ("dgate", "dscale", "dshift", "dw_post", "dw_pre"):
        assert f(**{p: FAKE + 2}) == ALIGN
    assert f(dx=FAKE + 8) == ALIGN and f(dy=FAKE + 8) == ALIGN
    need = rtl.residual_norm_backward_workspace(16, 3, 64)
    assert f(ws=None) == WORKSPACE and f(wsb=need - 1) == WORKSPACE and f(ws=FAKE + 64) == ALIGN
    none = dict(dgate=None, dscale=None, dshift=None, dw_post=None, dw_pre=None)
    assert f(T=0, **none) == 0
    assert rtl.residual_norm_backward_workspace(0, 0, 64) == 0


@no_gpu
def test_norm_backward_accepts():
    f = norm_backward()
    none = dict(dgate=None, dscale=None, dshift=None, dw_post=None, dw_pre=None)
    assert passes(f(wsb=rtl.residual_norm_backward_workspace(16, 3, 64))) and passes(f(ws=None, wsb=0, **none)) and passes(f(dh=None, xo=None))
    assert passes(f(dxo=None)) and passes(f(y=None, dy=None, dgate=None, dw_post=None)) and passes(f(T=0)) and passes(f(off=None, S=1))


ROTARY = dict(q=FAKE, k=FAKE, pos=FAKE, freq=FAKE, axis=FAKE, wq=FAKE, wk=FAKE, qo=FAKE, ko=FAKE, norm=1, eps=1e-6, inter=1, T=16, Hq=4, Hk=2, D=64, pairs=32,
              axes=3, ldq=256, sq=64, ldk=128, sk=64, ldqo=256, sqo=64, ldko=128, sko=64, stream=None)
ROTARY_BACK = dict(dqo=FAKE, dko=FAKE, q=FAKE, k=FAKE, pos=FAKE, freq=FAKE, axis=FAKE, wq=FAKE, wk=FAKE, dq=FAKE, dk=FAKE, dwq=FAKE, dwk=FAKE, norm=1, eps=1e-6,
                   inter=1, T=16, Hq=4, Hk=2, D=64, pairs=32, axes=3, lddqo=256, sdqo=64, lddko=128, sdko=64, ldq=256, sq=64, ldk=128, sk=64, lddq=256, sdq=64,
                   lddk=128, sdk=64, ws=FAKE, wsb=1 << 30, stream=None)


def check_rotary(f, out_q, out_k, ld, s):
    assert f(norm=2) == ARG and f(norm=-1) == ARG and f(eps=-1.0) == ARG
    assert f(T=-1) == SHAPE and f(T=1 << 24) == SHAPE and f(Hq=-1) == SHAPE and f(Hk=65533) == SHAPE and f(D=60) == SHAPE and f(D=0) == SHAPE and f(D=520) == SHAPE
    assert f(pairs=36) == SHAPE and f(pairs=30) == SHAPE and f(pairs=28, inter=0) == SHAPE and f(pairs=-4) == SHAPE and f(axes=0) == SHAPE and f(axes=17) == SHAPE
    assert f(ldq=56) == SHAPE and f(sk=56) == SHAPE and f(**{ld: 56}) == SHAPE and f(**{s: 56}) == SHAPE
    for p in ("q", "k", "pos", "freq", "axis", out_q, out_k):
        assert f(**{p: None}) == NULL
        assert f(**{p: FAKE + 2}) == ALIGN
    assert f(ldq=260) == ALIGN and f(sk=68) == ALIGN and f(**{ld: 260}) == ALIGN and f(wq=FAKE + 8) == ALIGN


def test_rotary_refusals():
    f = caller("rtl_norm_rotary", ROTARY)
    check_rotary(f, "qo", "ko", "ldqo", "sqo")
    assert f(norm=0) == ARG                                        # weights without a norm
    assert f(T=0) == 0 and f(Hq=0, Hk=0) == 0


def test_rotary_backward_refusals():
    f = caller("rtl_norm_rotary_backward", ROTARY_BACK)
    check_rotary(f, "dq", "dk", "lddq", "sdq")
    assert f(dqo=None) == NULL and f(norm=0, wq=None, wk=None) == ARG
    assert f(ws=None) == WORKSPACE and f(wsb=rtl.norm_rotary_backward_workspace(64) - 1) == WORKSPACE and f(ws=FAKE + 64) == ALIGN and f(dwq=FAKE + 2) == ALIGN
    assert f(T=0, dwq=None, dwk=None) == 0
    assert rtl.norm_rotary_backward_workspace(0) == 0


@no_gpu
def test_rotary_accepts():
    f = caller("rtl_norm_rotary", ROTARY)
    assert passes(f()) and passes(f(norm=0, wq=None, wk=None)) and passes(f(q=None, qo=None, Hq=0, ldq=0, sq=0, ldqo=0, sqo=0)) and passes(f(T=1, ldq=0, ldko=0))
    assert passes(f(pairs=0, pos=None, freq=None, axis=None)) and passes(f(pairs=28)) and passes(f(ldq=64, sq=64 * 16, inter=0))
    f = caller("rtl_norm_rotary_backward", ROTARY_BACK)
    assert passes(f()) and passes(f(dwq=None, dwk=None, ws=None, wsb=0)) and passes(f(norm=0, wq=None, wk=None, dwq=None, dwk=None, q=None, k=None, ws=None, wsb=0))


def test_binding_refuses_host_tensors_and_wrong_shapes():
    bf = torch.bfloat16
    x = torch.zeros(4, 64, dtype=bf)
    for call in (lambda: rtl.gated_linear(x, torch.zeros(8, 64, dtype=bf)), lambda: rtl.residual_norm(x), lambda: rtl.norm_rotary(x.view(4, 1, 64), None, None, None, None),
                 lambda: rtl.gated_linear_backward(x, x, x, x), lambda: rtl.residual_norm_backward(x, x, x),
                 lambda: rtl.norm_rotary_backward(x.view(4, 1, 64), None, None, None, None, None, None)):
        with pytest.raises(ValueError):
            call()


def test_binding_names_what_it_takes():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for call, where in ((lambda: rtl.residual_norm(None), "x expected"), (lambda: rtl.norm_rotary(None, None, None, None, None), "q or k"),
                        (lambda: rtl.residual_norm(None, post="l2"), "post: one of none, rms, layer"), (lambda: rtl.residual_norm(None, pre=1), "pre: one of none, rms, layer"),
                        (lambda: rtl.gated_linear(None, None, act="relu"), "X and W|act: one of silu, gelu, gelu_tanh"),
                        (lambda: rtl.norm_rotary(None, None, None, None, None, norm="rms "), "norm: one of none, rms, layer"),
                        (lambda: rtl.residual_norm(x), "current device only"), (lambda: rtl.residual_norm([1.0]), "tensor or None"),
                        (lambda: rtl.residual_norm(None, out=(None,)), "out: 2 tensors")):
        with pytest.raises(ValueError, match=where):
            call()
