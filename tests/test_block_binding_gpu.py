"""What the Python entry points of the block operators refuse, before anything is launched, and what they hand back."""
import pytest
import torch

from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32


def ones(*shape, dtype=bf, device=DEV):
    return torch.ones(*shape, dtype=dtype, device=device)


def wrong(t):
    """The same tensor in ways that do not do: on the host, of another type, of another shape, columns apart."""
    apart = torch.ones(*t.shape, 2, dtype=t.dtype, device=DEV)[..., 0]
    return [t.cpu(), t.to(torch.float16 if t.dtype is not torch.float16 else bf), torch.ones(*t.shape, 1, dtype=t.dtype, device=DEV),
            torch.ones(*[n + 8 for n in t.shape], dtype=t.dtype, device=DEV), apart, 3.0]


def check(f, kw, optional=()):
    """f takes kw as it is, and none of it in a wrong way."""
    f(**kw)
    for name, value in kw.items():
        if not isinstance(value, torch.Tensor):
            continue
        for bad in wrong(value) + ([] if name in optional else [None]):
            with pytest.raises((ValueError, rtl.RtlError)):
                f(**dict(kw, **{name: bad}))
    torch.cuda.synchronize()


def test_gated_linear():
    check(rtl.gated_linear, dict(X=ones(16, 64), W=ones(48, 64), bias=ones(48), out=ones(16, 24), pre=ones(16, 48)), ("bias", "out", "pre"))
    for bad in ("relu", None, 0):
        with pytest.raises(ValueError):
            rtl.gated_linear(ones(16, 64), ones(48, 64), act=bad)
    with pytest.raises(ValueError):
        rtl.gated_linear(ones(16, 64), ones(47, 64))
    with pytest.raises(rtl.RtlError):
        rtl.gated_linear(ones(16, 40), ones(48, 40))
    out, pre = ones(16, 24), ones(16, 48)
    got = rtl.gated_linear(ones(16, 64), ones(48, 64), out=out, pre=pre)
    assert got[0] is out and got[1] is pre


def test_gated_linear_backward():
    kw = dict(dH=ones(16, 24), X=ones(16, 64), W=ones(48, 64), P=ones(16, 48))
    check(rtl.gated_linear_backward, kw, ("X", "W"))
    out = (ones(16, 64), ones(48, 64, dtype=f32), ones(48, dtype=f32), ones(16, 24))
    assert all(a is b for a, b in zip(rtl.gated_linear_backward(out=out, **kw), out))
    for i, t in enumerate(out):
        for bad in wrong(t):
            if isinstance(bad, torch.Tensor) and i == 1 and bad.dtype is bf:
                continue
            with pytest.raises((ValueError, rtl.RtlError)):
                rtl.gated_linear_backward(out=out[:i] + (bad,) + out[i + 1:], **kw)
    for bad in (out[:3], out + out, 5, out[:1] + (None,) + out[2:]):
        with pytest.raises(ValueError):
            rtl.gated_linear_backward(out=bad, **kw)
    for name, i in (("X", 1), ("W", 0)):
        with pytest.raises(ValueError):
            rtl.gated_linear_backward(out=out, **dict(kw, **{name: None}))
    with pytest.raises(ValueError):
        rtl.gated_linear_backward(dtype=torch.float16, **kw)
    with pytest.raises(rtl.RtlError):
        rtl.gated_linear_backward(ws=torch.empty(256, dtype=torch.uint8, device=DEV), **kw)


def norms(**kw):
    return dict(y=ones(16, 64), gate=ones(3, 64), w_post=ones(64), w_pre=ones(64), scale=ones(3, 64),
                offsets=torch.tensor([0, 3, 9, 16], dtype=i32, device=DEV), post="rms", pre="rms", **kw)


def test_residual_norm():
    check(rtl.residual_norm, norms(x=ones(16, 64, dtype=f32), shift=ones(3, 64)), ("y", "gate", "w_post", "w_pre", "scale", "shift"))
    x = ones(16, 64)
    for bad in (dict(post="batch"), dict(pre=None), dict(alpha="a"), dict(out=(x,)), dict(out=x), dict(out=(ones(16, 64, dtype=f32), x)),
                dict(shift=ones(3, 128)[:, :64])):
        with pytest.raises((ValueError, TypeError)):
            rtl.residual_norm(**dict(norms(x=x, shift=ones(3, 64)), **bad))
    with pytest.raises(rtl.RtlError):
        rtl.residual_norm(x, with_x=False, with_h=False)
    a, b = ones(16, 64), ones(16, 64)
    got = rtl.residual_norm(**norms(x=x, out=(a, b)))
    assert got[0] is a and got[1] is b


def test_residual_norm_backward():
    kw = norms(dx_out=ones(16, 64, dtype=f32), dh=ones(16, 64), x_out=ones(16, 64, dtype=f32))
    check(rtl.residual_norm_backward, kw, ("dx_out", "dh", "y", "gate", "w_post", "w_pre", "scale"))
    got = rtl.residual_norm_backward(**kw)
    assert [None if t is None else (tuple(t.shape), t.dtype) for t in got] == [((16, 64), f32), ((16, 64), bf)] + [((3, 64), f32)] * 3 + [((64,), f32)] * 2
    assert rtl.residual_norm_backward(**dict(kw, with_shift=False))[4] is None and rtl.residual_norm_backward(**dict(kw, scale=None, with_shift=True))[4] is not None
    for i, t in enumerate(got):
        for bad in wrong(t):
            with pytest.raises((ValueError, rtl.RtlError)):
                rtl.residual_norm_backward(out=got[:i] + (bad,) + got[i + 1:], **kw)
    with pytest.raises(ValueError):
        rtl.residual_norm_backward(None, ones(16, 64), None)
    with pytest.raises(rtl.RtlError):
        rtl.residual_norm_backward(ws=torch.empty(256, dtype=torch.uint8, device=DEV), **kw)


def heads(**kw):
    return dict(q=ones(16, 4, 64), k=ones(16, 2, 64), pos=ones(16, 2, dtype=f32), freq=ones(32, dtype=f32), axis=torch.zeros(32, dtype=i32, device=DEV), wq=ones(64),
                wk=ones(64), **kw)


def test_norm_rotary():
    check(rtl.norm_rotary, heads(), ("q", "k", "freq", "wq", "wk"))
    for bad in (dict(norm="layer"), dict(norm="x"), dict(norm="none"), dict(out=(ones(16, 4, 64), None)), dict(out=ones(16, 4, 64)), dict(q=None, k=None)):
        with pytest.raises((ValueError, rtl.RtlError)):
            rtl.norm_rotary(**dict(heads(), **bad))
    out = ones(16, 4, 64), ones(16, 2, 64)
    got = rtl.norm_rotary(out=out, **heads())
    assert got[0] is out[0] and got[1] is out[1]


def test_norm_rotary_backward():
    kw = heads(dq_out=ones(16, 4, 64), dk_out=ones(16, 2, 64))
    check(rtl.norm_rotary_backward, kw, ("freq", "wq", "wk"))
    got = rtl.norm_rotary_backward(**kw)
    assert [tuple(t.shape) for t in got] == [(16, 4, 64), (16, 2, 64), (64,), (64,)]
    for i, t in enumerate(got):
        for bad in wrong(t):
            with pytest.raises((ValueError, rtl.RtlError)):
                rtl.norm_rotary_backward(out=got[:i] + (bad,) + got[i + 1:], **kw)
    only = rtl.norm_rotary_backward(ones(16, 4, 64), None, None, None, None, None, None, norm="none")
    assert only[1:] == (None, None, None) and torch.equal(only[0], ones(16, 4, 64))


def test_references_are_given_back():
    """Calls, refused ones too, keep no tensor alive and let none go."""
    import sys
    x, w = ones(16, 64), ones(64)
    before = sys.getrefcount(x), sys.getrefcount(w), sys.getrefcount(None)
    for _ in range(200):
        rtl.residual_norm(x, w_pre=w, out=(x, None))
        rtl.residual_norm_backward(x, x, x, w_pre=w)
        with pytest.raises(ValueError):
            rtl.residual_norm(x, w_pre=x)
    assert (sys.getrefcount(x), sys.getrefcount(w)) == before[:2] and abs(sys.getrefcount(None) - before[2]) < 100
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    for _ in range(20):
        rtl.residual_norm_backward(x, x, x, w_pre=w)
    assert torch.cuda.memory_allocated() == held
