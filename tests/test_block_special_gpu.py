"""The block operators on the GPU where care is called for: vectors that should not matter and are not finite, gates far below zero, launches of the largest size."""
import math

import pytest
import torch

import block_plan as plan
import block_ref as ref
from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
BAD = [float("inf"), float("-inf"), float("nan")]
NAMES = ("dx", "dy", "dgate", "dscale", "dshift", "dw_post", "dw_pre")


def normal(seed, *shape, dtype=torch.bfloat16, std=1.0, mean=0.0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(dtype)


def spoilt(seed, *shape, bad):
    """A vector with one value that is not finite in each of its rows."""
    t = normal(seed, *shape)
    t[..., 5] = bad
    return t


# two sequences with rows and one without, as in a batch of fixed size that is not full; D of one wave, and of several
OFFSETS = [0, 7, 7, 20]


@pytest.mark.parametrize("D", [64, 1032])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("wide", [False, True])
def test_no_branch_no_gate(D, bad, wide):
    """Without y x' is alpha x whatever gate and w_post hold, the sign of a zero too."""
    x = normal(1, 20, D, dtype=torch.float32 if wide else torch.bfloat16)
    x[3] = -0.0
    offsets = torch.tensor(OFFSETS, dtype=torch.int32, device=DEV)
    how = dict(offsets=offsets, post="rms", pre="rms", alpha=0.5, eps=EPS)
    want = rtl.residual_norm(x, **how)
    got = rtl.residual_norm(x, gate=spoilt(2, 3, D, bad=bad), w_post=spoilt(3, D, bad=bad), **how)
    assert torch.equal(got[0], x * 0.5) and bool(torch.signbit(got[0][3]).all())
    assert torch.equal(got[1], want[1]) and bool(torch.isfinite(got[1]).all())


@pytest.mark.parametrize("D", [64, 1032])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("post,pre", [("none", "layer"), ("rms", "rms")])
def test_no_gradient_no_modulation(D, bad, post, pre):
    """With dh None nothing passes through the second norm, whatever w_pre and scale hold: their gradients are zeros, the others those of ordinary ones."""
    dx, x, y = (normal(i, 20, D) for i in (4, 5, 6))
    offsets = torch.tensor(OFFSETS, dtype=torch.int32, device=DEV)
    how = dict(gate=normal(7, 3, D), w_post=normal(8, D), offsets=offsets, post=post, pre=pre, alpha=0.5, eps=EPS)
    want = rtl.residual_norm_backward(dx, None, x, y, w_pre=normal(9, D), scale=normal(10, 3, D), **how)
    got = rtl.residual_norm_backward(dx, None, x, y, w_pre=spoilt(9, D, bad=bad), scale=spoilt(10, 3, D, bad=bad), **how)
    for name, g, w in zip(NAMES, got, want):
        assert torch.equal(g, w) and bool(torch.isfinite(g).all()), name
    for i in (3, 4, 6):
        assert bool((got[i] == 0).all())
    one = dict(how, gate=how["gate"][:1], offsets=None)             # (a single sequence has its sums from another kernel)
    got = dict(zip(NAMES, rtl.residual_norm_backward(dx, None, x, y, w_pre=spoilt(9, D, bad=bad), scale=spoilt(10, 1, D, bad=bad), **one)))
    for name in ("dscale", "dshift", "dw_pre"):
        assert bool((got[name] == 0).all()), name


@pytest.mark.parametrize("D", [64, 1032])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("behind", [0, 5])
def test_vectors_of_empty_sequences(D, bad, behind):
    """What gate and scale hold for a sequence without rows reaches no weight's gradient; its own gradients are zeros, whatever the weights hold."""
    dx, dh, x, y = (normal(i, 20, D) for i in (11, 12, 13, 14))
    offsets = torch.tensor([o if i < 3 else 20 - behind for i, o in enumerate(OFFSETS + [20])], dtype=torch.int32, device=DEV)      # the last one empty too
    gate, scale = normal(15, 4, D), normal(16, 4, D)
    how = dict(w_post=normal(17, D), w_pre=normal(18, D), offsets=offsets, post="rms", pre="layer", eps=EPS)
    want = rtl.residual_norm_backward(dx, dh, x, y, gate=gate, scale=scale, **how)
    gate[1], gate[3], scale[1], scale[3] = bad, bad, bad, bad
    got = rtl.residual_norm_backward(dx, dh, x, y, gate=gate, scale=scale, **how)
    for name, g, w in zip(NAMES, got, want):
        assert torch.equal(g, w) and bool(torch.isfinite(g).all()), name
    got = dict(zip(NAMES, rtl.residual_norm_backward(dx, dh, x, y, gate=gate, scale=scale, **dict(how, w_post=spoilt(17, D, bad=bad), w_pre=spoilt(18, D, bad=bad)))))
    for name in ("dgate", "dscale", "dshift"):
        assert bool((got[name][1] == 0).all()) and bool((got[name][3] == 0).all()), name
    # a single sequence without rows, and no rows at all
    none = torch.tensor([4, 4], dtype=torch.int32, device=DEV)
    for rows, off in ((20, none), (0, None)):
        got = rtl.residual_norm_backward(dx[:rows], dh[:rows], x[:rows], y[:rows], gate=gate[1:2], scale=scale[1:2],
                                         **dict(how, offsets=off, w_post=spoilt(17, D, bad=bad), w_pre=spoilt(18, D, bad=bad)))
        for name, g in zip(NAMES, got):
            assert bool((g == 0).all()), name


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("D,pairs", [(64, 8), (72, 24), (128, 48), (96, 0), (264, 8), (24, 8)])
def test_values_behind_the_pairs_pass(interleaved, bad, D, pairs):
    """Each by itself: one that is not finite leaves the others as they are, and a negative zero keeps its sign."""
    T, H = 9, 3
    pos, freq = normal(21, T, 2, dtype=torch.float32), normal(22, pairs, dtype=torch.float32)
    axis = torch.arange(pairs, dtype=torch.int32, device=DEV) % 2
    v = normal(23, T, H, D)
    v[:, 1, 2 * pairs:] = -0.0
    for at in range(2 * pairs, D):
        v[at % T, 2, at] = bad                                     # in each place once, several in a head where there are more places than tokens
    how = dict(norm="none", interleaved=interleaved)
    turned = rtl.norm_rotary(v, None, pos, freq, axis, **how)[0]
    back = rtl.norm_rotary_backward(v, None, None, None, pos, freq, axis, **how)[0]
    plain = v.clone()
    plain[..., 2 * pairs:] = 0
    want = rtl.norm_rotary(plain, None, pos, freq, axis, **how)[0], rtl.norm_rotary_backward(plain, None, None, None, pos, freq, axis, **how)[0]
    for got, w in zip((turned, back), want):
        assert torch.equal(got[..., :2 * pairs], w[..., :2 * pairs])
        a, b = got[..., 2 * pairs:], v[..., 2 * pairs:]
        assert bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all()) and bool(torch.signbit(a[:, 1]).all())


def far_gates():
    return torch.linspace(-12.5, -0.5, 400).to(torch.bfloat16).to(DEV)


def gelu_below_zero(g):
    """Value and slope of g < 0 in 64 bits and how far they may be off. U = 2^-24; Phi(g) = .5 P(t) e, e = exp(-x), x = g^2 / 2. P is off by 2e-7 of itself as a formula;
    t by 4 U, which P magnifies at most 3.4 times; its evaluation has eight steps of two roundings, each of at most twice P: 14 + 32 U. e: 4 x U from its
    argument's roundings and 4 U. Two products: 2 U. In all (4 x + 52) U + 2e-7 of Phi itself, so that nothing is forgiven where Phi is small."""
    g = g.double()
    x, phi = g * g / 2, 0.5 * torch.special.erfc(-g / math.sqrt(2))
    rel = (4 * x + 52) * ref.U + 2e-7
    bell = g * torch.exp(-x) / math.sqrt(2 * math.pi)
    return g * phi, (g * phi).abs() * (rel + ref.U), phi + bell, phi * rel + bell.abs() * (4 * x + 10) * ref.U + ref.U * (phi + bell).abs()


# rows and contractions that reach each form of the launch at 400 columns
GELU_SIZES = [(1, 64), (20, 256), (400, 512), (800, 1024), (2100, 2048), (4000, 64), (3000, 128), (20, 64), (6000, 64), (12000, 64)]


def test_gelu_sizes_reach_their_forms():
    assert [plan.gated_form(M, 400, K) for M, K in GELU_SIZES] == ["few", 0, 1, 2, 3, 4, 5, 6, "tails", "192"]


@pytest.mark.parametrize("M,K", GELU_SIZES)
def test_gelu_far_below_zero(M, K):
    """H at gates whose Phi is down to 4e-36: right to a rounding."""
    g = far_gates()
    F = g.numel()
    X, W = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV), torch.zeros(2 * F, K, dtype=torch.bfloat16, device=DEV)
    X[:, 0], W[:F, 0], W[F:, 0] = 1.0, g, 1.0
    value, err, _, _ = gelu_below_zero(g)
    ref.close(rtl.gated_linear(X, W, act="gelu"), value.expand(M, F), err.expand(M, F), "H")


def test_gelu_gradients_far_below_zero():
    g = far_gates()
    M, F = 3, g.numel()
    P = torch.cat([g, torch.ones_like(g)]).expand(M, 2 * F).contiguous()
    eye, dH = torch.eye(2 * F, dtype=torch.bfloat16, device=DEV), torch.ones(M, F, dtype=torch.bfloat16, device=DEV)
    dP, _, _, H = rtl.gated_linear_backward(dH, None, eye, P, act="gelu", with_hidden=True)        # (weights of the identity: dX is [dG dU])
    value, err, slope, err_slope = gelu_below_zero(g)
    ref.close(H, value.expand(M, F), err.expand(M, F), "H")
    ref.close(dP[:, F:], value.expand(M, F), err.expand(M, F), "dU")
    ref.close(dP[:, :F], slope.expand(M, F), err_slope.expand(M, F), "dG")


def test_zz_most_rows_of_wide_norms():
    """So many rows of more than 4096 columns that one launch would have 2^32 threads and more: each row is taken once."""
    T, D, step = (1 << 23) + 3, 4104, 1 << 20
    x = torch.empty(T, D, dtype=torch.bfloat16, device=DEV)
    mark = (torch.arange(T, device=DEV) % 255 + 1).to(torch.bfloat16)[:, None]
    for i in range(0, T, step):
        x[i:i + step] = mark[i:i + step]
    rtl.residual_norm(x, alpha=0.5, out=(x, None))
    for i in range(0, T, step):
        assert bool((x[i:i + step] == mark[i:i + step] * 0.5).all())
    del x
    torch.cuda.empty_cache()
