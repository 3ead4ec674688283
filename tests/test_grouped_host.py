"""Refusals of the entry points of linears grouped by expert, all before any launch."""
import pytest
import torch

from paper_2605_26632_amd import binding as rtl

FAKE = 0x10000      # non-null, aligned, never dereferenced
NULL, SHAPE, ALIGN, WORKSPACE, ARG = 1, 2, 3, 4, 5
BIG = 1 << 30


def caller(name, defaults):
    def f(**kw):
        assert set(kw) <= set(defaults)
        return getattr(rtl.lib(), name)(*dict(defaults, **kw).values())
    return f


def check_common(f, pointers):
    assert f(T=-1) == SHAPE and f(E=-1) == SHAPE and f(N=-8) == SHAPE and f(K=-64) == SHAPE
    assert f(T=BIG + 1) == SHAPE and f(E=65537) == SHAPE
    for p in pointers:
        assert f(**{p: None}) == NULL
        assert f(**{p: FAKE + 1}) == ALIGN


def test_forward_refusals():
    f = caller("rtl_grouped_linear", dict(X=FAKE, off=FAKE, W=FAKE, bias=None, Y=FAKE, T=16, E=2, N=24, K=64, ldx=64, ldw=64, sw=24 * 64, ldy=24,
                                          stream=None))
    check_common(f, ("X", "off", "W", "Y"))
    assert f(K=32) == SHAPE and f(K=0) == SHAPE and f(ldx=56) == SHAPE and f(ldw=56) == SHAPE and f(ldy=23) == SHAPE and f(sw=-8) == SHAPE
    assert f(ldx=(1 << 22) + 8) == SHAPE and f(ldw=(1 << 22) + 8) == SHAPE
    assert f(T=BIG, N=BIG, ldy=BIG) == SHAPE                       # 2^24 workgroups and more
    assert f(ldx=68) == ALIGN and f(ldw=68) == ALIGN and f(sw=24 * 64 + 4) == ALIGN and f(bias=FAKE + 1) == ALIGN
    assert f(T=0) == 0 and f(E=0) == 0 and f(N=0) == 0


def test_mxfp4_forward_refusals():
    f = caller("rtl_grouped_mxfp4_linear", dict(X=FAKE, off=FAKE, Wq=FAKE, Ws=FAKE, bias=None, Y=FAKE, T=16, E=2, N=24, K=64, ldx=64, ldw=32,
                                                sw=24 * 32, ldy=24, ws=FAKE, wsb=1 << 20, stream=None))
    check_common(f, ("X", "off", "Wq", "Ws", "Y"))
    assert f(K=48) == SHAPE and f(ldw=16) == SHAPE and f(ldx=56) == SHAPE
    assert f(ldw=40) == ALIGN and f(sw=24 * 32 + 8) == ALIGN and f(ws=FAKE + 64) == ALIGN
    assert f(ws=None) == WORKSPACE and f(wsb=511) == WORKSPACE and f(wsb=rtl.grouped_mxfp4_linear_workspace(16, 2, 24, 64) - 1) == WORKSPACE
    assert f(T=0) == 0 and f(E=0) == 0 and f(N=0) == 0


def test_input_gradient_refusals():
    f = caller("rtl_grouped_linear_dgrad", dict(dY=FAKE, off=FAKE, W=FAKE, dX=FAKE, T=16, E=2, N=24, K=64, lddy=24, ldw=64, sw=24 * 64, lddx=64,
                                                stream=None))
    check_common(f, ("dY", "off", "W", "dX"))
    assert f(N=20) == SHAPE and f(K=60) == SHAPE and f(lddy=16) == SHAPE and f(ldw=56) == SHAPE and f(lddx=56) == SHAPE and f(N=0) == SHAPE
    assert f(lddy=28) == ALIGN and f(lddx=68) == ALIGN and f(dX=FAKE + 8) == ALIGN
    assert f(T=0) == 0 and f(E=0) == 0 and f(K=0) == 0


def test_weight_gradient_refusals():
    f = caller("rtl_grouped_linear_wgrad", dict(dY=FAKE, X=FAKE, off=FAKE, dW=FAKE, db=None, type=0, T=16, E=2, N=24, K=64, lddy=24, ldx=64, lddw=64,
                                                sdw=24 * 64, ws=None, wsb=0, stream=None))
    check_common(f, ("dY", "X", "off", "dW"))
    assert f(type=2) == ARG and f(type=-1) == ARG
    assert f(N=20) == SHAPE and f(K=60) == SHAPE and f(lddw=56) == SHAPE
    assert f(sdw=23 * 64 + 56) == SHAPE and f(sdw=0) == SHAPE          # the experts' gradients would overlap
    assert f(lddw=68, sdw=24 * 72) == ALIGN and f(dW=FAKE + 8) == ALIGN and f(db=FAKE + 1) == ALIGN and f(db=FAKE + 2, type=1) == ALIGN
    assert f(E=0) == 0 and f(N=0) == 0 and f(K=0) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    w = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    off = torch.zeros(3, dtype=torch.int32)
    for f in (lambda: rtl.grouped_linear(x, off, w), lambda: rtl.grouped_linear_dgrad(x, off, w), lambda: rtl.grouped_linear_wgrad(x, x, off),
              lambda: rtl.grouped_mxfp4_linear(x, off, w, w)):
        with pytest.raises(ValueError):
            f()


def test_clear_refusals():
    f = caller("rtl_grouped_clear", dict(off=FAKE, Y=FAKE, T=16, E=2, cols=24, ld=24, stream=None))
    assert f(T=-1) == SHAPE and f(E=-1) == SHAPE and f(cols=-1) == SHAPE and f(ld=23) == SHAPE and f(T=BIG + 1) == SHAPE and f(E=65537) == SHAPE
    assert f(off=None) == NULL and f(Y=None) == NULL and f(off=FAKE + 2) == ALIGN and f(Y=FAKE + 1) == ALIGN
    assert f(T=0) == 0 and f(cols=0) == 0
    with pytest.raises(ValueError):
        rtl.grouped_clear(torch.zeros(3, dtype=torch.int32), torch.zeros(4, 8, dtype=torch.bfloat16))


def test_weight_gradient_refuses_a_bias_gradient_without_columns():
    """K == 0 leaves no weight gradient to write, and nothing would write dbias, which is not empty."""
    f = caller("rtl_grouped_linear_wgrad", dict(dY=FAKE, X=FAKE, off=FAKE, dW=FAKE, db=FAKE, type=0, T=16, E=2, N=24, K=0, lddy=24, ldx=0, lddw=0,
                                                sdw=0, ws=None, wsb=0, stream=None))
    assert f() == SHAPE and f(T=0) == SHAPE and f(type=1) == SHAPE
    assert f(db=None) == 0 and f(E=0) == 0 and f(N=0) == 0


@pytest.mark.parametrize("E,N,K", [(256, 4096, 7168), (384, 4096, 7168), (128, 16384, 5120), (32768, 128, 128), (65536, 1024, 1024), (2048, 8192, 8192)])
@pytest.mark.parametrize("T", [0, 1, 8192, 65536])
def test_weight_gradient_takes_large_stacks(T, E, N, K):
    """What is refused is the launch that the call would make (2^32 threads and more), not one of more parts or smaller tiles: forward and input
    gradient take these stacks too. (Every size check comes before the pointers are looked at.)"""
    rows = max(T, 1)
    f = caller("rtl_grouped_linear_wgrad", dict(dY=FAKE, X=FAKE, off=FAKE, dW=None, db=None, type=0, T=T, E=E, N=N, K=K, lddy=N, ldx=K, lddw=K, sdw=N * K,
                                                ws=None, wsb=0, stream=None))
    assert f() == NULL and f(type=1) == NULL and f(ws=FAKE, wsb=1 << 40) == NULL
    fwd = caller("rtl_grouped_linear", dict(X=FAKE, off=FAKE, W=None, bias=None, Y=FAKE, T=rows, E=E, N=N, K=K, ldx=K, ldw=K, sw=N * K, ldy=N, stream=None))
    grad = caller("rtl_grouped_linear_dgrad", dict(dY=FAKE, off=FAKE, W=None, dX=FAKE, T=rows, E=E, N=N, K=K, lddy=N, ldw=K, sw=N * K, lddx=K, stream=None))
    assert fwd() == NULL and grad() == NULL


@pytest.mark.parametrize("T", [0, 1, 65536])
def test_weight_gradient_refuses_more_workgroups_than_a_launch_takes(T):
    """Tiles of 256 x 256 have 512 threads, tiles of 128 x 128 have 256: fewer than 2^23 or 2^24 of them, an expert's rounded up to eights."""
    f = caller("rtl_grouped_linear_wgrad", dict(dY=FAKE, X=FAKE, off=FAKE, dW=None, db=None, type=0, T=T, E=65536, N=4096, K=4096, lddy=4096, ldx=4096,
                                                lddw=4096, sdw=4096 * 4096, ws=None, wsb=0, stream=None))
    assert f() == SHAPE and f(N=2048) == SHAPE and f(N=1024, K=1024) == NULL
