"""What a transformer block does between its linears, and its gated feed-forward linear: the work whose speed is measured, and its
plain form.

`op` of a case names the work:
  "gated"           gated_linear: G = X W[:F]^T + b[:F], U = X W[F:]^T + b[F:], H = act(G) U; with `pre` P = [G U] comes too
  "gated_backward"  gated_linear_backward: from dH, X, W and P the gradients dX, dW, db, and H again for the linear behind it
  "norm"            residual_norm: x' = alpha x + gate_s (w_post norm(y)), h = w_pre norm(x') (1 + scale_s) + shift_s, for rows of
                    sequence s; rows of no sequence are zeros
  "norm_backward"   residual_norm_backward: from dx', dh, x' and y the gradients of x, y, gate, scale, shift and both weights
  "rotary"          norm_rotary: the heads of q and k normed (w q / rms(q)), then their pairs turned by pos[t, axis[j]] freq[j]
  "rotary_backward" norm_rotary_backward: the gradients of q, k and both weights

Norms: "rms" v / sqrt(mean v^2 + eps), "layer" (v - mean v) / sqrt(mean (v - mean v)^2 + eps), "none". Everything is bf16 but the
residual stream x, x' with `wide` (float32), positions and frequencies, and the gradients of what all rows share (float32;
bf16 for dW and db). `own` false computes all of it from elementary torch operations.
"""
import math
import random

import torch

own = False
DEV = "cuda"
EPS = 1e-6
ALPHA = 0.75


def _gated(name, M, F, K, act="silu", bias=False, pre=False):
    return dict(name=name, op="gated", M=M, F=F, K=K, act=act, bias=bias, pre=pre)


def _gated_backward(name, M, F, K, act="silu", bias=False):
    return dict(name=name, op="gated_backward", M=M, F=F, K=K, act=act, bias=bias)


def _norm(name, op, T, D, S, post="none", pre="layer", wide=False, spare=0, sizes=1):
    return dict(name=name, op=op, T=T, D=D, S=S, post=post, pre=pre, wide=wide, spare=spare, sizes=sizes)


def _rotary(name, op, T, Hq, Hk, D, pairs, axes, norm=True, interleaved=True):
    return dict(name=name, op=op, T=T, Hq=Hq, Hk=Hk, D=D, pairs=pairs, axes=axes, norm=norm, interleaved=interleaved)


def listed():
    return [
        # one conditioning vector or one token through a feed-forward layer of the Z-Image size: the bytes of the weight
        _gated("gated_one_token", 1, 10240, 3840, bias=True),
        # a text prompt: odd rows and width
        _gated("gated_prompt_odd", 333, 2739, 4032, act="gelu_tanh", bias=True),
        # the image tokens of a training step through the Z-Image feed-forward layer, pre-activations kept for the backward pass
        _gated("gated_image", 4096, 10240, 3840, pre=True),
        # training of a small layer, ragged rows
        _gated_backward("gated_backward_small", 701, 704, 512, act="gelu", bias=True),
        # ordinary training batch
        _gated_backward("gated_backward", 4096, 8192, 2048),
        # one token of four requests between two blocks: latency
        _norm("norm_four_tokens", "norm", 4, 3840, 4, post="rms", pre="rms"),
        # a batch of four images at high resolution between two blocks
        _norm("norm_images", "norm", 16896, 3840, 4),
        # training on packed samples of uneven length, float32 residual stream, sandwich norms, room behind the last sample
        _norm("norm_backward_packed", "norm_backward", 2111, 2048, 5, post="rms", pre="rms", wide=True, spare=77),
        # training on two large images
        _norm("norm_backward_images", "norm_backward", 8192, 3840, 2),
        # a decoding step: one token, shared key heads, half-split pairs, part of the head turned
        _rotary("rotary_one_token", "rotary", 1, 32, 8, 128, 48, 1, interleaved=False),
        # the tokens of a large image: time, height and width
        _rotary("rotary_image", "rotary", 16896, 30, 30, 128, 64, 3),
        # training on a small video clip, odd token count
        _rotary("rotary_backward_video", "rotary_backward", 4433, 30, 30, 128, 64, 3),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    cap_flops = max(work(c)["flops"] for c in listed())
    cap_bytes = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["gated", "gated_backward", "norm", "norm_backward", "rotary", "rotary_backward"])
        act = rng.choice(["silu", "gelu", "gelu_tanh"])
        if op == "gated":
            case = _gated("", _log_uniform(rng, 1, 16896), _log_uniform(rng, 64, 10240), _log_uniform(rng, 1, 160) * 64, act,
                          bias=rng.random() < 0.5, pre=rng.random() < 0.5)
        elif op == "gated_backward":
            case = _gated_backward("", _log_uniform(rng, 1, 16896), _log_uniform(rng, 16, 2560) * 4, _log_uniform(rng, 1, 160) * 64, act,
                                   bias=rng.random() < 0.5)
        elif op in ("norm", "norm_backward"):
            rows = _log_uniform(rng, 1, 16896)
            case = _norm("", op, rows, _log_uniform(rng, 8, 1024) * 8, _log_uniform(rng, 1, min(32, rows)),
                         post=rng.choice(["none", "rms", "layer"]), pre=rng.choice(["rms", "layer"]), wide=rng.random() < 0.5,
                         spare=rng.choice([0, 0, rng.randrange(1, 200)]), sizes=rng.randrange(1 << 30))
        else:
            heads, D = _log_uniform(rng, 1, 48), rng.choice([64, 72, 80, 96, 128, 192, 256])
            interleaved = rng.random() < 0.5
            pairs = D // 2 if D % 16 == 0 and rng.random() < 0.6 else rng.randrange(1, D // 16 + 1) * 8
            case = _rotary("", op, _log_uniform(rng, 1, 16896), heads, rng.choice([h for h in range(1, heads + 1) if heads % h == 0]), D, pairs,
                           rng.randrange(1, 4), norm=rng.random() < 0.7, interleaved=interleaved)
        del case["name"]
        w = work(case)
        if w["flops"] <= cap_flops and w["bytes"] <= cap_bytes:
            return case


def _offsets(case):
    """First rows of the sequences and the end of the last one; behind it lie `spare` rows that belong to nobody."""
    rng = random.Random(case["sizes"])
    if case["T"] == case["S"]:
        return list(range(case["T"] + 1))
    return [0] + sorted(rng.randrange(case["T"] + 1) for _ in range(case["S"] - 1)) + [case["T"]]


def work(case):
    op = case["op"]
    if op in ("gated", "gated_backward"):
        M, F, K = case["M"], case["F"], case["K"]
        b = 4 * F if case["bias"] else 0
        if op == "gated":
            return dict(bytes=2 * M * K + 4 * F * K + b + 2 * M * F * (3 if case["pre"] else 1), flops=4 * M * F * K)
        return dict(bytes=2 * (4 * M * F + 2 * M * K) + 8 * F * K + b, flops=8 * M * F * K)
    if op in ("norm", "norm_backward"):
        T, D, S, x = case["T"], case["D"], case["S"], 4 if case["wide"] else 2
        weights = 2 * D * ((case["post"] == "rms") + (case["pre"] == "rms"))
        if op == "norm":
            return dict(bytes=T * D * (2 * x + 4) + 6 * S * D + weights, flops=14 * T * D)
        return dict(bytes=T * D * (3 * x + 6) + 16 * S * D + 3 * weights, flops=30 * T * D)
    heads, D, T = case["Hq"] + case["Hk"], case["D"], case["T"]
    if op == "rotary":
        return dict(bytes=4 * T * heads * D + 4 * T * case["axes"], flops=7 * T * heads * D)
    return dict(bytes=(6 if case["norm"] else 4) * T * heads * D + 4 * T * case["axes"], flops=12 * T * heads * D)


# ---- inputs ---------------------------------------------------------------------------------------

def _normal(gen, *shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(dtype)


def _activation(gen, rows, cols, dtype=torch.bfloat16):
    """Heavy tails along a row and a few channels much larger than the rest, as the residual stream and the inputs of linears have them."""
    x = torch.randn(rows, cols, generator=gen, device=DEV)
    x *= torch.randn(rows, cols, generator=gen, device=DEV).abs()
    x *= 1.0 + 9.0 * (torch.rand(cols, generator=gen, device=DEV) < 0.01)
    return x.to(dtype)


def _positions(case):
    """Places on a grid around its middle, the last axis running fastest; of a video clip the frames come at 1 / 24 s."""
    T, axes = case["T"], case["axes"]
    t = torch.arange(T, dtype=torch.float32, device=DEV)
    if axes == 1:
        return (t + 8191.0).reshape(T, 1)
    w = max(1, int(math.isqrt(T)))
    cols = [t % w - w // 2, torch.div(t, w, rounding_mode="floor") - w // 2]
    if axes == 3:
        cols.insert(0, torch.div(t, 256, rounding_mode="floor") / 24.0)
    return torch.stack(cols, dim=1).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000003 * seed + 29)
    st, op, bf = dict(case=case), case["op"], torch.bfloat16
    if op in ("gated", "gated_backward"):
        M, F, K = case["M"], case["F"], case["K"]
        st["x"] = _normal(gen, M, K)
        st["w"] = _normal(gen, 2 * F, K, std=K ** -0.5)
        st["b"] = _normal(gen, 2 * F, std=0.2) if case["bias"] else None
        if op == "gated_backward":
            st["p"] = _normal(gen, M, 2 * F)
            st["dh"] = _normal(gen, M, F)
        if own and op == "gated":
            st["out"] = torch.empty(M, F, dtype=bf, device=DEV)
            st["pre"] = torch.empty(M, 2 * F, dtype=bf, device=DEV) if case["pre"] else None
        if own and op == "gated_backward":
            from paper_2605_26632_amd import binding as rtl
            st["room"] = torch.empty(rtl.gated_linear_backward_workspace(M, F, K), dtype=torch.uint8, device=DEV)
        return st
    if op in ("norm", "norm_backward"):
        T, D, S = case["T"] + case["spare"], case["D"], case["S"]
        kind = torch.float32 if case["wide"] else bf
        st["off"] = _offsets(case)
        st["offsets"] = torch.tensor(st["off"], dtype=torch.int32, device=DEV)
        st["x"] = _activation(gen, T, D, kind)        # x' where gradients are asked for
        st["y"] = _normal(gen, T, D)
        mod = _normal(gen, S, 6 * D, std=0.3)         # what the conditioning's linear gives: three vectors for each half of a block
        st["shift"], st["scale"], st["gate"] = mod[:, :D], mod[:, D:2 * D], mod[:, 5 * D:]
        st["w_post"] = _normal(gen, D, std=0.1, mean=1.0) if case["post"] == "rms" else None
        st["w_pre"] = _normal(gen, D, std=0.1, mean=1.0) if case["pre"] == "rms" else None
        if op == "norm_backward":
            st["dx"] = _normal(gen, T, D, dtype=kind)
            st["dh"] = _normal(gen, T, D)
        elif own:
            # a program keeps its results; where rows belong to nobody it takes new ones, in which the call writes those rows as zeros
            st["out"] = None if case["spare"] else (torch.empty(T, D, dtype=kind, device=DEV), torch.empty(T, D, dtype=bf, device=DEV))
        if own and op == "norm_backward":
            from paper_2605_26632_amd import binding as rtl
            st["room"] = torch.empty(rtl.residual_norm_backward_workspace(T, S, D), dtype=torch.uint8, device=DEV)
        return st
    T, Hq, Hk, D, P, A = (case[k] for k in ("T", "Hq", "Hk", "D", "pairs", "axes"))
    qkv = _normal(gen, T, (Hq + 2 * Hk) * D)          # one product gives q, k and v
    st["q"], st["k"] = qkv[:, :Hq * D].view(T, Hq, D), qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
    st["pos"] = _positions(case)
    # pairs dealt to the axes in runs, the first axis the shortest, frequencies falling over each run
    cut = [0] + [P * (a + 1) // (A + 1) for a in range(A - 1)] + [P]
    j = torch.arange(P, device=DEV)
    st["axis"] = torch.bucketize(j, torch.tensor(cut[1:], device=DEV), right=True).to(torch.int32)
    first, length = torch.tensor(cut, device=DEV)[st["axis"].long()], torch.tensor([max(1, cut[a + 1] - cut[a]) for a in range(A)], device=DEV)[st["axis"].long()]
    st["freq"] = torch.pow(10000.0, -((j - first).double() / length.double())).float()
    st["wq"] = _normal(gen, D, std=0.1, mean=1.0) if case["norm"] else None
    st["wk"] = _normal(gen, D, std=0.1, mean=1.0) if case["norm"] else None
    if op == "rotary_backward":
        st["dq"], st["dk"] = _normal(gen, T, Hq, D), _normal(gen, T, Hk, D)
    elif own:
        st["out"] = (torch.empty(T, Hq, D, dtype=bf, device=DEV), torch.empty(T, Hk, D, dtype=bf, device=DEV))
    return st


# ---- the plain form ---------------------------------------------------------------------------------

def _act(g, kind):
    """Value and derivative of the activation."""
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if kind == "gelu":
        phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    c = math.sqrt(2.0 / math.pi)
    th = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * c * (1.0 + 3 * 0.044715 * g * g)


def _plain_gated(st):
    case, bf, F = st["case"], torch.bfloat16, st["case"]["F"]
    x, w = st["x"].float(), st["w"].float()
    if case["op"] == "gated":
        p = x @ w.t()
        if case["bias"]:
            p = p + st["b"].float()
        h = _act(p[:, :F], case["act"])[0] * p[:, F:]
        return dict(h=h.to(bf), p=p.to(bf)) if case["pre"] else dict(h=h.to(bf))
    dh, g, u = st["dh"].float(), st["p"][:, :F].float(), st["p"][:, F:].float()
    a, da = _act(g, case["act"])
    dp = torch.cat([dh * u * da, dh * a], dim=1)
    out = dict(dx=(dp @ w).to(bf), dw=(dp.t() @ x).to(bf), h=(a * u).to(bf))
    if case["bias"]:
        out["db"] = dp.sum(dim=0).to(bf)
    return out


def _normed(v, kind):
    """norm(v) and what multiplies its differences."""
    if kind == "none":
        return v, None
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    r = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    return v * r, r


def _norm_back(dn, n, r, kind):
    if kind == "none":
        return dn
    d = dn - n * (dn * n).mean(dim=1, keepdim=True)
    if kind == "layer":
        d = d - dn.mean(dim=1, keepdim=True)
    return d * r


def _times(v, w):
    return v if w is None else v * w.float()


def _plain_norm(st):
    case, bf = st["case"], torch.bfloat16
    T, S = st["x"].shape[0], case["S"]
    kind = st["x"].dtype
    row = torch.arange(T, device=DEV)
    seq = torch.bucketize(row, st["offsets"][1:], right=True).clamp(max=S - 1)
    used = (row < st["offsets"][S])[:, None]
    gate, scale = st["gate"].float()[seq], 1.0 + st["scale"].float()[seq]
    ny, ry = _normed(st["y"].float(), case["post"])
    if case["op"] == "norm":
        x = ALPHA * st["x"].float() + gate * _times(ny, st["w_post"])
        h = _times(_normed(x, case["pre"])[0], st["w_pre"]) * scale + st["shift"].float()[seq]
        return dict(x=(x * used).to(kind), h=(h * used).to(bf))
    dh = st["dh"].float() * used
    nx, rx = _normed(st["x"].float(), case["pre"])
    dt = (st["dx"].float() + _norm_back(_times(dh * scale, st["w_pre"]), nx, rx, case["pre"])) * used
    dz = gate * dt
    dy = _norm_back(_times(dz, st["w_post"]), ny, ry, case["post"])
    mine = (seq == torch.arange(S, device=DEV)[:, None]).float()          # sums over the rows of each sequence
    of_gate, of_scale = mine @ (dt * ny), mine @ (dh * nx)
    out = dict(dx=(ALPHA * dt).to(kind), dy=dy.to(bf), dgate=_times(of_gate, st["w_post"]), dscale=_times(of_scale, st["w_pre"]), dshift=mine @ dh)
    if st["w_post"] is not None:
        out["dw_post"] = (st["gate"].float() * of_gate).sum(dim=0)
    if st["w_pre"] is not None:
        out["dw_pre"] = ((1.0 + st["scale"].float()) * of_scale).sum(dim=0)
    return out


def _turned(v, cos, sin, case):
    P = case["pairs"]
    if case["interleaved"]:
        a, b = v[..., 0:2 * P:2], v[..., 1:2 * P:2]
    else:
        a, b = v[..., :P], v[..., P:2 * P]
    a, b = a * cos - b * sin, a * sin + b * cos
    both = torch.stack([a, b], dim=-1).flatten(-2) if case["interleaved"] else torch.cat([a, b], dim=-1)
    return torch.cat([both, v[..., 2 * P:]], dim=-1)


def _plain_rotary(st):
    case, bf = st["case"], torch.bfloat16
    angle = st["pos"].double()[:, st["axis"].long()] * st["freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def there(v, w):
        v = v.float()
        if case["norm"]:
            v = v * torch.rsqrt((v * v).mean(dim=-1, keepdim=True) + EPS) * w.float()
        return _turned(v, cos, sin, case).to(bf)

    def back(d, v, w):
        d = _turned(d.float(), cos, -sin, case)
        if not case["norm"]:
            return d.to(bf), None
        v = v.float()
        r = torch.rsqrt((v * v).mean(dim=-1, keepdim=True) + EPS)
        n = v * r
        dw = (d * n).sum(dim=0).sum(dim=0)
        d = d * w.float()
        return (r * (d - n * (d * n).mean(dim=-1, keepdim=True))).to(bf), dw

    if case["op"] == "rotary":
        return dict(q=there(st["q"], st["wq"]), k=there(st["k"], st["wk"]))
    dq, dwq = back(st["dq"], st["q"], st["wq"])
    dk, dwk = back(st["dk"], st["k"], st["wk"])
    return dict(dq=dq, dk=dk, dwq=dwq, dwk=dwk) if case["norm"] else dict(dq=dq, dk=dk)


def _own(st):
    from paper_2605_26632_amd import binding as rtl
    case, op = st["case"], st["case"]["op"]
    if op == "gated":
        got = rtl.gated_linear(st["x"], st["w"], st["b"], act=case["act"], out=st["out"], pre=st["pre"])
        return dict(h=got[0], p=got[1]) if case["pre"] else dict(h=got)
    if op == "gated_backward":
        dx, dw, db, h = rtl.gated_linear_backward(st["dh"], st["x"], st["w"], st["p"], act=case["act"], with_bias=case["bias"], with_hidden=True,
                                                  ws=st["room"])
        return dict(dx=dx, dw=dw, h=h, db=db) if case["bias"] else dict(dx=dx, dw=dw, h=h)
    if op in ("norm", "norm_backward"):
        how = dict(gate=st["gate"], w_post=st["w_post"], w_pre=st["w_pre"], scale=st["scale"], offsets=st["offsets"], post=case["post"],
                   pre=case["pre"], alpha=ALPHA, eps=EPS)
        if op == "norm":
            x, h = rtl.residual_norm(st["x"], st["y"], shift=st["shift"], out=st["out"], **how)
            return dict(x=x, h=h)
        got = rtl.residual_norm_backward(st["dx"], st["dh"], st["x"], st["y"], ws=st["room"], **how)
        names = ("dx", "dy", "dgate", "dscale", "dshift", "dw_post", "dw_pre")
        return {n: v for n, v in zip(names, got) if v is not None}
    how = dict(wq=st["wq"], wk=st["wk"], norm="rms" if case["norm"] else "none", eps=EPS, interleaved=case["interleaved"])
    if op == "rotary":
        q, k = rtl.norm_rotary(st["q"], st["k"], st["pos"], st["freq"], st["axis"], out=st["out"], **how)
        return dict(q=q, k=k)
    got = rtl.norm_rotary_backward(st["dq"], st["dk"], st["q"], st["k"], st["pos"], st["freq"], st["axis"], **how)
    return {n: v for n, v in zip(("dq", "dk", "dwq", "dwk"), got) if v is not None}


def run(st):
    if own:
        return _own(st)
    op = st["case"]["op"]
    return _plain_gated(st) if op.startswith("gated") else _plain_norm(st) if op.startswith("norm") else _plain_rotary(st)


# ---- the definition in 64 bits: the forward formulas alone, their gradients by differentiation -----------------------

def _exact_leaf(t):
    return None if t is None else t.detach().double().requires_grad_(True)


def _exact_act(g, kind):
    f = torch.nn.functional
    return f.silu(g) if kind == "silu" else f.gelu(g, approximate="none" if kind == "gelu" else "tanh")


def _exact_norm_rows(v, kind):
    if kind == "none":
        return v
    if kind == "layer":
        return (v - v.mean(-1, keepdim=True)) / torch.sqrt(v.var(-1, unbiased=False, keepdim=True) + EPS)
    return v / torch.sqrt(v.square().mean(-1, keepdim=True) + EPS)


def _exact_rotary(v, w, angle, case):
    """One head after the other as complex numbers."""
    P = case["pairs"]
    if case["norm"]:
        v = _exact_norm_rows(v, "rms") * w
    at = torch.arange(P, device=v.device)
    i, j = (2 * at, 2 * at + 1) if case["interleaved"] else (at, at + P)
    z = torch.complex(v[..., i], v[..., j]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return v.index_copy(-1, i, z.real).index_copy(-1, j, z.imag)


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op in ("gated", "gated_backward"):
        F = case["F"]
        x, w = st["x"].double(), st["w"].double()
        if op == "gated":
            p = torch.matmul(x, w.t().contiguous())
            if st["b"] is not None:
                p += st["b"].double()
            h = _exact_act(p[:, :F], case["act"]) * p[:, F:]
            return dict(h=h, p=p) if case["pre"] else dict(h=h)
        p = _exact_leaf(st["p"])
        h = _exact_act(p[:, :F], case["act"]) * p[:, F:]
        dp, = torch.autograd.grad(h, p, st["dh"].double())
        out = dict(dx=torch.matmul(dp, w), dw=torch.matmul(dp.t().contiguous(), x), h=h.detach())
        if case["bias"]:
            out["db"] = torch.matmul(torch.ones(1, dp.shape[0], dtype=torch.float64, device=DEV), dp)[0]
        return out
    if op in ("norm", "norm_backward"):
        off, S = st["off"], case["S"]
        y, gate, scale, shift, w_post, w_pre = (_exact_leaf(st[k]) for k in ("y", "gate", "scale", "shift", "w_post", "w_pre"))
        x = _exact_leaf(st["x"])
        xs, hs, zs = [], [], []
        for s in range(S):
            rows = slice(off[s], off[s + 1])
            z = _exact_norm_rows(y[rows], case["post"])
            z = gate[s] * (z if w_post is None else z * w_post)
            # in the backward pass x is x' itself: what the gradient reaches x' with goes on to z
            new = ALPHA * x[rows] + z if op == "norm" else x[rows]
            n = _exact_norm_rows(new, case["pre"])
            h = (n if w_pre is None else n * w_pre) * (1.0 + scale[s]) + shift[s]
            xs.append(new)
            hs.append(h)
            zs.append(z)
        if op == "norm":
            full = [torch.zeros_like(x, requires_grad=False) for _ in range(2)]
            full[0][:off[S]], full[1][:off[S]] = torch.cat(xs).detach(), torch.cat(hs).detach()
            return dict(x=full[0], h=full[1])
        h, z = torch.cat(hs), torch.cat(zs)
        leaves = [t for t in (x, scale, shift, w_pre) if t is not None]
        got = list(torch.autograd.grad(h, leaves, st["dh"][:off[S]].double(), retain_graph=False))
        dt = torch.zeros_like(x, requires_grad=False)
        dt[:off[S]] = got[0][:off[S]] + st["dx"][:off[S]].double()
        leaves = [t for t in (y, gate, w_post) if t is not None]
        more = list(torch.autograd.grad(z, leaves, dt[:off[S]]))
        out = dict(dx=ALPHA * dt, dy=more[0], dgate=more[1], dscale=got[1], dshift=got[2])
        if w_post is not None:
            out["dw_post"] = more[2]
        if w_pre is not None:
            out["dw_pre"] = got[3]
        return out
    q, k, wq, wk = (_exact_leaf(st[n]) for n in ("q", "k", "wq", "wk"))
    angle = torch.stack([st["pos"][:, a].double() * f.double() for a, f in zip(st["axis"].tolist(), st["freq"])], dim=1)
    tq, tk = _exact_rotary(q, wq, angle, case), _exact_rotary(k, wk, angle, case)
    if op == "rotary":
        return dict(q=tq.detach(), k=tk.detach())
    leaves = [q, k] + ([wq, wk] if case["norm"] else [])
    got = torch.autograd.grad([tq, tk], leaves, [st["dq"].double(), st["dk"].double()])
    return dict(zip(("dq", "dk", "dwq", "dwk"), got))
