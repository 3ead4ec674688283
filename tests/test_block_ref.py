"""The block operators' reference (block_ref): its forward values and gradients against torch's functions and autograd in 64 bits, and that `close` sees mistakes."""
import itertools
import math

import pytest
import torch
import torch.nn.functional as fn

import block_ref as ref

EPS = 1e-6
ACTS = {"silu": fn.silu, "gelu": fn.gelu, "gelu_tanh": lambda g: fn.gelu(g, approximate="tanh")}


def values(seed, *shapes):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=gen).to(torch.bfloat16) for s in shapes]


def leaf(t):
    return t.double().requires_grad_()


def near(a, b):
    assert torch.allclose(a.double(), b.detach(), rtol=1e-11, atol=1e-11)


@pytest.mark.parametrize("kind", ACTS)
def test_gated(kind):
    X, W, b, dH = values(1, (13, 24), (20, 24), (20,), (13, 10))
    x, w, c = leaf(X), leaf(W), leaf(b)
    p = fn.linear(x, w, c)
    p.retain_grad()
    g, u = p.chunk(2, dim=1)
    h = ACTS[kind](g) * u
    h.backward(dH.double())
    H, _, P, _ = ref.gated(X, W, b, kind)
    near(H, h)
    near(P, p)
    got = ref.gated_backward(dH, X, W, p.detach(), kind)
    for name, want in (("dX", x.grad), ("dW", w.grad), ("db", c.grad), ("H", h)):
        near(got[name][0], want)


def normed(v, kind):
    if kind == "layer":
        return fn.layer_norm(v, v.shape[-1:], eps=EPS)
    return v / torch.sqrt(v.square().mean(-1, keepdim=True) + EPS) if kind == "rms" else v


@pytest.mark.parametrize("post,pre", itertools.product(("none", "rms", "layer"), repeat=2))
def test_residual_norm(post, pre):
    T, D, S, alpha = 12, 16, 3, 0.75
    X, Y, GX, GH, gate, scale, shift, wy, wx = values(2, (T, D), (T, D), (T, D), (T, D), (S, D), (S, D), (S, D), (D,), (D,))
    offsets = torch.tensor([1, 5, 5, 11], dtype=torch.int32)
    seq = torch.tensor([-1] + [0] * 4 + [2] * 6 + [-1])
    mine, at = seq >= 0, seq.clamp(min=0)
    x, y, g, s, b, p, q = (leaf(t) for t in (X, Y, gate, scale, shift, wy, wx))
    x1 = alpha * x + g[at] * p * normed(y, post)
    x1.retain_grad()
    h = q * normed(x1, pre) * (1 + s[at]) + b[at]
    (x1[mine] * GX.double()[mine]).sum().add((h[mine] * GH.double()[mine]).sum()).backward()
    (gx, _), (gh, _) = ref.residual_norm(X, Y, gate, wy, wx, scale, shift, offsets, post, pre, alpha, EPS)
    near(gx, x1 * mine[:, None])
    near(gh, h * mine[:, None])
    got = ref.residual_norm_backward(GX, GH, x1.detach(), Y, gate, wy, wx, scale, offsets, post, pre, alpha, EPS)
    for name, want in (("dx", x), ("dy", y), ("dgate", g), ("dscale", s), ("dshift", b), ("dw_post", p), ("dw_pre", q)):
        near(got[name][0][mine] if name in ("dx", "dy") else got[name][0], want.grad[mine] if name in ("dx", "dy") else want.grad)


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("norm", ["rms", "none"])
def test_norm_rotary(interleaved, norm):
    T, H, D, P = 5, 3, 32, 8
    V, DV, W = values(3, (T, H, D), (T, H, D), (D,))
    gen = torch.Generator().manual_seed(4)
    pos, freq, axis = torch.randn(T, 2, generator=gen) * 50, torch.rand(P, generator=gen), torch.arange(P, dtype=torch.int32) % 2
    w = W if norm == "rms" else None
    v, u = leaf(V), leaf(W)
    n = u * normed(v, "rms") if norm == "rms" else v
    turn = torch.polar(torch.ones(T, P, dtype=torch.float64), pos.double()[:, axis.long()] * freq.double())[:, None]
    part = n[..., :2 * P]
    if interleaved:
        out = torch.view_as_real(torch.view_as_complex(part.reshape(T, H, P, 2)) * turn).flatten(-2)
    else:
        z = torch.complex(part[..., :P], part[..., P:]) * turn
        out = torch.cat([z.real, z.imag], -1)
    out = torch.cat([out, n[..., 2 * P:]], -1)
    out.backward(DV.double())
    near(ref.norm_rotary(V, pos, freq, axis, w, norm, EPS, interleaved)[0], out)
    (dv, _), dw = ref.norm_rotary_backward(DV, V, pos, freq, axis, w, norm, EPS, interleaved)
    near(dv, v.grad)
    if norm == "rms":
        near(dw[0], u.grad)
    else:
        assert dw is None


def test_slopes_against_differences():
    g = torch.linspace(-9, 9, 181, dtype=torch.float64)
    for kind in ACTS:
        step = 1e-5
        ahead, behind = (ref.act(g + t, kind)[0] for t in (step, -step))
        # third derivatives are below 3, and the differences of values up to 9 carry 64-bit roundings
        assert bool(((ahead - behind) / (2 * step) - ref.act(g, kind)[1]).abs().max() < 3 * step * step / 6 + 9 * 2.0 ** -52 / step)


def plain_norm(X, Y, gate, S, pre):
    """The operator in fp32."""
    x1 = X.float() + gate.float()[0] * Y.float()
    return x1, normed(x1, pre) * (1 + S.float()[0])


MISTAKES = {
    "biased variance": lambda x, h: h * math.sqrt(511 / 512),
    "scale without one": lambda x, h: h - 1e-2 * x,
    "rounded statistics": lambda x, h: h * (1 + 2.0 ** -7),
    "a column too far": lambda x, h: h.roll(1, 1),
    "one value": lambda x, h: torch.where(torch.arange(h.numel()).view(h.shape) == 700, h * 1.02, h),
    "a row left out": lambda x, h: torch.where(torch.arange(h.shape[0])[:, None] == 3, torch.zeros_like(h), h),
}


@pytest.mark.parametrize("mistake", [None] + list(MISTAKES))
def test_mistakes_are_seen(mistake):
    X, Y, gate, scale = values(5, (7, 512), (7, 512), (1, 512), (1, 512))
    _, (h, err) = ref.residual_norm(X, Y, gate, None, None, scale, None, None, "none", "layer", 1.0, EPS)
    got = plain_norm(X, Y, gate, scale, "layer")[1].to(torch.bfloat16)
    if mistake is None:
        ref.close(got, h, err)
        return
    with pytest.raises(AssertionError):
        ref.close(got, MISTAKES[mistake](X.double(), h), err)


def test_other_mistakes_are_seen():
    X, W = values(6, (9, 64), (16, 64))
    want = ref.gated(X, W, None, "silu")
    p = X.float() @ W.float().t()
    h = (fn.silu(p[:, :8]) * p[:, 8:]).to(torch.bfloat16)
    ref.close(h, want[0], want[1])
    for other in (ref.gated(X, W, None, "gelu"), ref.gated(X, W.roll(8, 0), None, "silu"), ref.gated(X[:, :-1], W[:, :-1], None, "silu")):
        with pytest.raises(AssertionError):
            ref.close(h, other[0], want[1])
    V, = values(7, (5, 2, 32))
    pos, freq, axis = torch.arange(5.0)[:, None], torch.linspace(0.1, 1, 16), torch.zeros(16, dtype=torch.int32)
    right = ref.norm_rotary(V, pos, freq, axis, None, "none", EPS, True)
    ref.close(right[0].to(torch.bfloat16), *right)
    for other in (ref.norm_rotary(V, pos, freq, axis, None, "none", EPS, False), ref.norm_rotary(V, -pos, freq, axis, None, "none", EPS, True),
                  ref.norm_rotary(V, pos, freq, axis, None, "rms", EPS, True), ref.norm_rotary(V, pos + 0.1, freq, axis, None, "none", EPS, True)):
        with pytest.raises(AssertionError):
            ref.close(right[0].to(torch.bfloat16), other[0], right[1])
