"""What a transformer block does between its linears, in 64 bits, and how far fp32 arithmetic and the roundings may be off it.

HALF[t] is half a step of type t relative to the value, U = 2^-24 that of fp32. A sum of n fp32 terms in any order is off by at most n U times the sum of
their magnitudes. Each function returns the value and a bound on what is left of |error| before the one rounding at the store; `close` adds that rounding."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2, torch.float32: U}
TINY = 2.0 ** -126           # below it values may be flushed to zero


def d(t):
    return None if t is None else t.detach().double()


def close(got, want, err, what=""):
    """got is want off by at most err and one rounding."""
    want, err = want.to(got.device), err.to(got.device)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert bool(torch.isfinite(want).all()) and bool(torch.isfinite(got).all()), what
    far = (got.double() - want).abs()
    room = err + HALF[got.dtype] * (want.abs() + err) + TINY
    bad = far > room
    if bool(bad.any()):
        at = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d off, first at %s: %r for %r, room %.3g" % (
            what, int(bad.sum()), bad.numel(), at, got[at].item(), want[at].item(), room[at].item()))


# ---- gated linear ---------------------------------------------------------------------------------

def act(g, kind):
    """(value, slope, second derivative's bound) in 64 bits."""
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu":
        phi = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    x = 2 * c * (g + 0.044715 * g ** 3)
    s = torch.sigmoid(x)
    return g * s, s + g * s * (1 - s) * 2 * c * (1 + 3 * 0.044715 * g * g)


def act_errors(g, kind):
    """How far value and slope of a given g may be off in fp32: the argument x of e^x is off by 4 U |x| (its polynomial and the factor log2 e) and e^x by that
    of itself, e^x and 1 / y by 2 units each, another 4 U for the sum and the products: (4 |x| + 10) U of the logistic function, cut where it is
    zero anyway; for gelu the approximation's 1.5e-7 and the same. The slope's terms are each at most (1 + |x'| |value|) of it."""
    if kind == "gelu":
        x, xp = 0.5 * g * g, g.abs()
        rel = (4 * x.clamp(max=90) + 16) * U
        e = torch.exp(-x) * rel + 1.5e-7
        return g.abs() * (e + 4 * U), e + xp * torch.exp(-x) * rel + 8 * U * (1 + xp * torch.exp(-x))
    c2 = 2 * math.sqrt(2 / math.pi)
    x, xp = (g.abs(), torch.ones_like(g)) if kind == "silu" else (c2 * (g + 0.044715 * g ** 3).abs(), c2 * (1 + 3 * 0.044715 * g * g))
    s = torch.sigmoid(g if kind == "silu" else c2 * (g + 0.044715 * g ** 3))
    rel = (4 * x.clamp(max=90) + 10) * U
    value = g.abs() * s
    return value * rel, s * rel + value * xp * (1 - s) * rel + value * xp * s * rel + 8 * U * (s + value * xp * (1 - s))


def gated(X, W, b, kind):
    """H, P and their errors. fp32 sums of K products and the bias: (K + 2) U of their magnitudes; |act'| <= 1.2."""
    x, w = d(X), d(W)
    F, K = w.shape[0] // 2, w.shape[1]
    p, mag = x @ w.t(), x.abs() @ w.abs().t()
    if b is not None:
        p, mag = p + d(b), mag + d(b).abs()
    ep = (K + 2) * U * mag
    g, u, eg, eu = p[:, :F], p[:, F:], ep[:, :F], ep[:, F:]
    value, _ = act(g, kind)
    ev = act_errors(g, kind)[0] * 2 + 1.2 * eg
    return value * u, ev * (u.abs() + eu) + value.abs() * eu + 2 * U * (value * u).abs(), p, ep


def gated_backward(dH, X, W, P, kind):
    """dict of (value, error): dX, dW, db, H. [dG dU] is rounded to bf16, so that it is off by HALF of itself too."""
    F = P.shape[1] // 2
    g, u, dh = d(P)[:, :F], d(P)[:, F:], d(dH)
    value, slope = act(g, kind)
    ev, es = act_errors(g, kind)
    dp = torch.cat([dh * u * slope, dh * value], dim=1)
    edp = torch.cat([(dh * u).abs() * es, dh.abs() * ev], dim=1) + 3 * U * dp.abs()
    edp = edp + HALF[torch.bfloat16] * (dp.abs() + edp) + TINY
    out = dict(H=(value * u, ev * u.abs() + 2 * U * (value * u).abs()))
    size = dp.abs() + edp
    if W is not None:
        w = d(W)
        out["dX"] = (dp @ w, edp @ w.abs() + 2 * F * U * (size @ w.abs()))
    if X is not None:
        x = d(X)
        out["dW"] = (dp.t() @ x, edp.t() @ x.abs() + x.shape[0] * U * (size.t() @ x.abs()))
        out["db"] = (dp.sum(0), edp.sum(0) + x.shape[0] * U * size.sum(0))
    return out


# ---- norms with gate, residual and modulation --------------------------------------------------------

def normed(v, kind, eps):
    """(norm(v), factor, error). Sums along a row: 8 values of a thread (16 where a row has at most 8 waves), the lanes of a wave, at most 16 waves: chains of at
    most 16 + 6 + 16 additions, so that mean, mean square and with them the factor are off by 64 U of their magnitudes; a difference to the mean by that of the
    mean and its own."""
    if kind == "none":
        return v, torch.ones_like(v[:, :1]), torch.zeros_like(v)
    m = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    c = v - m
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    ec = 64 * U * v.abs().mean(1, keepdim=True) * (kind == "layer") + 2 * U * (v.abs() + m.abs()) * (kind == "layer")
    er = r * (64 * U + r * r * (c.abs() * ec + ec * ec).mean(1, keepdim=True))
    return c * r, r, ec * r + c.abs() * er + 4 * U * (c * r).abs()


def rows_of(offsets, T):
    o = [0, T] if offsets is None else offsets.tolist()
    seq = torch.full((T,), -1, dtype=torch.long)
    for s in range(len(o) - 1):
        seq[o[s]:o[s + 1]] = s
    return seq


def one(t, T, D, like, default):
    return torch.full((T, D), default, dtype=torch.float64, device=like.device) if t is None else d(t)


def residual_norm(x, y, gate, w_post, w_pre, scale, shift, offsets, post, pre, alpha, eps):
    """((x', error), (h, error)), rows of nobody zero."""
    T, D = x.shape
    seq = rows_of(offsets, T).to(x.device)
    use, at = (seq >= 0)[:, None], seq.clamp(min=0)
    S = 1 if offsets is None else offsets.numel() - 1
    pick = lambda t, v: one(t, S, D, x, v)[at] if S else torch.zeros(T, D, dtype=torch.float64, device=x.device)  # noqa: E731
    g, sc, sh = pick(gate, 1.0), pick(scale, 0.0), pick(shift, 0.0)
    wy, wx = one(w_post, 1, D, x, 1.0).reshape(1, D), one(w_pre, 1, D, x, 1.0).reshape(1, D)
    x = torch.where(use, d(x), 0.0)
    new, err = alpha * x, 2 * U * (alpha * x).abs()
    if y is not None:
        n, _, en = normed(torch.where(use, d(y), 0.0), post, eps)
        z = g * wy * n
        new, err = new + z, err + (g * wy).abs() * en + 4 * U * (z.abs() + new.abs())
    n, r, en = normed(new, pre, eps)
    if pre == "none":
        en = en + err
    else:                              # an error e of x' moves its norm by at most r (e + mean e + |n| rms e)
        en = en + 2 * r * (err + err.mean(1, keepdim=True) + n.abs() * err.square().mean(1, keepdim=True).sqrt())
    h = wx * n * (1 + sc) + sh
    eh = (wx * (1 + sc)).abs() * en + 6 * U * ((wx * n).abs() * (1 + sc.abs()) + sh.abs())
    return (torch.where(use, new, 0.0), torch.where(use, err, 0.0)), (torch.where(use, h, 0.0), torch.where(use, eh, 0.0))


def through(dn, edn, n, en, r, kind):
    """The norm's part of a gradient and its error: differences of terms that are off by U and by what dn and n are."""
    if kind == "none":
        return dn, edn
    mean = lambda t: t.mean(1, keepdim=True)  # noqa: E731
    mn, m = mean(dn * n), mean(dn) * (kind == "layer")
    emn = mean(edn * n.abs() + dn.abs() * en) + 64 * U * mean((dn * n).abs())
    em = (mean(edn) + 64 * U * mean(dn.abs())) * (kind == "layer")
    out = r * (dn - m - n * mn)
    return out, r * (edn + em + n.abs() * emn + en * mn.abs()) + 80 * U * r * (dn.abs() + m.abs() + (n * mn).abs())


def residual_norm_backward(dx_out, dh, x_out, y, gate, w_post, w_pre, scale, offsets, post, pre, alpha, eps):
    """dict of (value, error)."""
    like = x_out if x_out is not None else dx_out
    T, D = like.shape
    S = 1 if offsets is None else offsets.numel() - 1
    seq = rows_of(offsets, T).to(like.device)
    use, at = (seq >= 0)[:, None], seq.clamp(min=0)
    zero = torch.zeros(T, D, dtype=torch.float64, device=like.device)
    clean = lambda t: zero if t is None else torch.where(use, d(t), 0.0)  # noqa: E731
    g, sc = one(gate, S, D, like, 1.0), one(scale, S, D, like, 0.0)
    wy, wx = one(w_post, 1, D, like, 1.0).reshape(1, D), one(w_pre, 1, D, like, 1.0).reshape(1, D)
    dh, dt, edt = clean(dh), clean(dx_out), zero
    n, r, en = normed(clean(x_out), pre, eps)
    f = wx * (1 + sc[at])
    dn = dh * f
    back, eb = through(dn, 4 * U * dn.abs(), n, en, r, pre)
    dt, edt = dt + back, eb + 2 * U * (dt.abs() + back.abs())
    out = dict(dx=(alpha * dt, abs(alpha) * edt + U * (alpha * dt).abs()))
    mine = (seq[None] == torch.arange(S, device=like.device)[:, None]).double()
    total = lambda v, e: (mine @ v, mine @ e + (mine.sum(1, keepdim=True) + 64) * U * (mine @ (v.abs() + e)))  # noqa: E731
    weigh = lambda w, t: (w * t[0], w.abs() * t[1] + 2 * U * (w * t[0]).abs())  # noqa: E731
    over = lambda w, t: ((w * t[0]).sum(0), (w.abs() * t[1]).sum(0) + (S + 4) * U * (w.abs() * (t[0].abs() + t[1])).sum(0))  # noqa: E731
    a = total(dh * n, dh.abs() * en + U * (dh * n).abs())
    out["dscale"], out["dshift"], out["dw_pre"] = weigh(wx, a), total(dh, zero), over(1 + sc, a)
    if y is not None:
        ny, ry, eny = normed(clean(y), post, eps)
        c = total(dt * ny, dt.abs() * eny + edt * ny.abs() + U * (dt * ny).abs())
        out["dgate"], out["dw_post"] = weigh(wy, c), over(g, c)
        fy = g[at] * wy
        dz = dt * fy
        out["dy"] = through(dz, edt * fy.abs() + 4 * U * dz.abs(), ny, eny, ry, post)
    return out


# ---- head norm and rotary positions ----------------------------------------------------------------------

def _turn(v, e, angle, interleaved, back=False):
    P = angle.shape[1]
    i, j = (torch.arange(P) * 2, torch.arange(P) * 2 + 1) if interleaved else (torch.arange(P), torch.arange(P) + P)
    c, s = torch.cos(angle)[:, None], (-1.0 if back else 1.0) * torch.sin(angle)[:, None]
    a, b = v[..., i], v[..., j]
    out, err = v.clone(), e.clone()
    out[..., i], out[..., j] = a * c - b * s, a * s + b * c
    # sine and cosine: 2e-9 of the series, 8 U of its fp32 evaluation; two products and a sum
    both = (a.abs() + b.abs()) * (12 * U + 2e-9)
    err[..., i] = e[..., i] * c.abs() + e[..., j] * s.abs() + both
    err[..., j] = e[..., i] * s.abs() + e[..., j] * c.abs() + both
    return out, err


def _angles(pos, freq, axis, T, like):
    if freq is None:
        return torch.zeros(T, 0, dtype=torch.float64, device=like.device)
    return d(pos)[:, axis.long()] * d(freq)


def _head_norm(v, eps):
    """Chains of 16 + 5 additions."""
    r = 1 / torch.sqrt(v.square().mean(-1, keepdim=True) + eps)
    return v * r, r, 32 * U * (v * r).abs()


def norm_rotary(v, pos, freq, axis, w, norm, eps, interleaved):
    t = d(v)
    e = torch.zeros_like(t)
    if norm == "rms":
        t, _, e = _head_norm(t, eps)
        if w is not None:
            t, e = t * d(w), e * d(w).abs() + 2 * U * (t * d(w)).abs()
    return _turn(t, e, _angles(pos, freq, axis, v.shape[0], v), interleaved)


def norm_rotary_backward(dv, v, pos, freq, axis, w, norm, eps, interleaved):
    """((dv, error), (dw, error) or None)."""
    g, e = _turn(d(dv), torch.zeros_like(d(dv)), _angles(pos, freq, axis, dv.shape[0], dv), interleaved, back=True)
    if norm != "rms":
        return (g, e), None
    n, r, en = _head_norm(d(v), eps)
    rows = v.shape[0] * v.shape[1]
    dn = (g * n).reshape(rows, -1)
    edn = (e * n.abs() + g.abs() * en + U * (g * n).abs()).reshape(rows, -1)
    dw = dn.sum(0), edn.sum(0) + (rows + 64) * U * (dn.abs() + edn).sum(0)
    if w is not None:
        g, e = g * d(w), e * d(w).abs() + U * (g * d(w)).abs()
    m = (g * n).mean(-1, keepdim=True)
    em = (e * n.abs() + g.abs() * en).mean(-1, keepdim=True) + 32 * U * (g * n).abs().mean(-1, keepdim=True)
    return (r * (g - n * m), r * (e + n.abs() * em + en * m.abs()) + 40 * U * r * (g.abs() + (n * m).abs())), dw
