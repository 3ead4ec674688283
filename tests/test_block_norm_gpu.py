"""Norms of a block with gate, residual and modulation, and their gradients, on the GPU against the formulas in 64 bits."""
import itertools

import pytest
import torch

import block_ref as ref
from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
NAMES = ("dx", "dy", "dgate", "dscale", "dshift", "dw_post", "dw_pre")


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def normal(gen, *shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(dtype)


def strided(t, pad=8, fill=float("nan")):
    wide = torch.full((t.shape[0], t.shape[1] + 2 * pad), fill, dtype=t.dtype, device=DEV)
    wide[:, pad:-pad] = t
    return wide[:, pad:-pad]


def offsets_of(ends):
    return torch.tensor(ends, dtype=torch.int32, device=DEV)


class Case:
    """Inputs of T rows; those of no sequence hold NaN."""

    def __init__(self, T, D, offsets, seed, wide=False, with_y=True, with_mod=True, weights=True, mean=0.0):
        gen = generator(seed)
        kind = torch.float32 if wide else torch.bfloat16
        self.S = 1 if offsets is None else len(offsets) - 1
        self.offsets = None if offsets is None else offsets_of(offsets)
        self.x, self.y = strided(normal(gen, T, D, dtype=kind, mean=mean, std=2.0)), strided(normal(gen, T, D, mean=mean)) if with_y else None
        self.dx, self.dh = strided(normal(gen, T, D, dtype=kind)), strided(normal(gen, T, D))
        if offsets is not None:
            nobody = ref.rows_of(self.offsets, T) < 0
            for t in (self.x, self.y, self.dx, self.dh):
                if t is not None:
                    t[nobody.to(DEV)] = float("nan")
        mod = normal(gen, self.S, 6 * D, std=0.4)
        self.shift, self.scale, self.gate = (mod[:, :D], mod[:, D:2 * D], mod[:, 5 * D:]) if with_mod else (None,) * 3
        self.w_post, self.w_pre = (normal(gen, D, std=0.2, mean=1.0), normal(gen, D, std=0.2, mean=1.0)) if weights else (None, None)

    def forward(self, post, pre, alpha, **kw):
        return rtl.residual_norm(self.x, self.y, self.gate, self.w_post, self.w_pre, self.scale, self.shift, self.offsets, post=post, pre=pre, alpha=alpha,
                                 eps=EPS, **kw)

    def want(self, post, pre, alpha):
        return ref.residual_norm(self.x, self.y, self.gate, self.w_post, self.w_pre, self.scale, self.shift, self.offsets, post, pre, alpha, EPS)

    def backward(self, post, pre, alpha, dx="dx", dh="dh", **kw):
        return rtl.residual_norm_backward(getattr(self, dx, None), getattr(self, dh, None), self.x, self.y, self.gate, self.w_post, self.w_pre, self.scale,
                                          self.offsets, post=post, pre=pre, alpha=alpha, eps=EPS, **kw)

    def want_back(self, post, pre, alpha, dx="dx", dh="dh"):
        return ref.residual_norm_backward(getattr(self, dx, None), getattr(self, dh, None), self.x, self.y, self.gate, self.w_post, self.w_pre, self.scale,
                                          self.offsets, post, pre, alpha, EPS)


# T, D, ends of the sequences (None: one sequence): one row, widths of every team and just behind it, empty sequences, rows of nobody in front and behind,
# a sequence for each row, more sequences than a wave has lanes
SIZES = [(1, 8, None), (1, 3840, None), (3, 64, [0, 1, 2, 3]), (7, 512, [2, 2, 5]), (70, 520, [0, 70]), (130, 1024, [3, 3, 40, 41, 41, 128]), (65, 1032, list(range(66))),
         (200, 264, [0] + list(range(0, 200, 2)) + [200]), (33, 2048, [1, 20, 30]), (50, 2056, None), (37, 4096, [0, 16, 32, 37]), (20, 4104, [0, 5, 20]),
         (9, 8192, [0, 9]), (17, 8184, [2, 4, 17]), (600, 136, [10, 300, 300, 599]), (5000, 24, [0, 5000])]


@pytest.mark.parametrize("T,D,ends", SIZES)
@pytest.mark.parametrize("post,pre,wide", [("none", "layer", False), ("rms", "rms", True), ("layer", "rms", False)])
def test_forward(T, D, ends, post, pre, wide):
    c = Case(T, D, ends, T + D, wide)
    (x, ex), (h, eh) = c.want(post, pre, 0.75)
    xo, ho = c.forward(post, pre, 0.75)
    assert xo.dtype is c.x.dtype and ho.dtype is torch.bfloat16
    ref.close(xo, x, ex, "x")
    ref.close(ho, h, eh, "h")
    # rows of nobody, and what lies between the rows, stay as they were
    xp, hp = (torch.full((T, D + 16), 3.0, dtype=t, device=DEV) for t in (c.x.dtype, torch.bfloat16))
    c.forward(post, pre, 0.75, out=(xp[:, 8:-8], hp[:, 8:-8]))
    mine = (ref.rows_of(c.offsets, T) >= 0).to(DEV)
    for place, new in ((xp, xo), (hp, ho)):
        assert torch.equal(place[mine, 8:-8], new[mine]) and bool((place[~mine] == 3.0).all())
        assert bool((place[:, :8] == 3.0).all()) and bool((place[:, -8:] == 3.0).all())


@pytest.mark.parametrize("T,D,ends", SIZES)
@pytest.mark.parametrize("post,pre,wide", [("none", "layer", False), ("rms", "rms", True), ("layer", "rms", False)])
def test_backward(T, D, ends, post, pre, wide):
    c = Case(T, D, ends, T * 3 + D, wide)
    want, got = c.want_back(post, pre, 0.75), dict(zip(NAMES, c.backward(post, pre, 0.75)))
    assert got["dx"].dtype is c.x.dtype and got["dy"].dtype is torch.bfloat16
    nobody = (ref.rows_of(c.offsets, T) < 0).to(DEV)
    for name in NAMES:
        ref.close(got[name], *want[name], name)
    assert bool((got["dx"][nobody] == 0).all()) and bool((got["dy"][nobody] == 0).all())
    again = c.backward(post, pre, 0.75)                            # the same bits every time
    assert all(torch.equal(a, got[n]) for n, a in zip(NAMES, again))


@pytest.mark.parametrize("post,pre", itertools.product(("none", "rms", "layer"), repeat=2))
@pytest.mark.parametrize("with_y,with_mod,weights", [(True, False, True), (True, True, False), (False, True, True), (False, False, False)])
def test_absent_vectors(post, pre, with_y, with_mod, weights):
    c = Case(90, 328, [1, 30, 88], 5, False, with_y, with_mod, weights)
    (x, ex), (h, eh) = c.want(post, pre, 1.0)
    xo, ho = c.forward(post, pre, 1.0)
    ref.close(xo, x, ex, "x")
    ref.close(ho, h, eh, "h")
    xo, none = c.forward(post, pre, 1.0, with_h=False)
    assert none is None
    ref.close(xo, x, ex, "x")
    none, again = c.forward(post, pre, 1.0, with_x=False)
    assert none is None and torch.equal(again, ho)
    want, got = c.want_back(post, pre, 1.0), dict(zip(NAMES, c.backward(post, pre, 1.0)))
    for name, missing in (("dy", not with_y), ("dgate", not (with_y and with_mod)), ("dscale", not with_mod), ("dshift", not with_mod),
                          ("dw_post", not (with_y and weights)), ("dw_pre", not weights)):
        assert (got[name] is None) == missing, name
    for name in NAMES:
        if got[name] is not None:
            ref.close(got[name], *want[name], name)
    # gradients of absent vectors, and one gradient alone
    out = [torch.empty_like(got["dx"])] + [None] * 6
    for i, n in ((3, c.S), (4, c.S), (6, 1)):
        out[i] = torch.empty((n, 328) if n > 1 else (328,), dtype=torch.float32, device=DEV)
    if with_y:
        out[2] = torch.empty((c.S, 328), dtype=torch.float32, device=DEV)
    out[0].fill_(7.0)
    c.backward(post, pre, 1.0, out=out)
    for name, t in zip(NAMES[1:], out[1:]):
        if t is not None:
            ref.close(t, *want[name], name)
    ref.close(out[0][1:88], want["dx"][0][1:88], want["dx"][1][1:88], "dx")
    assert bool((out[0][0] == 7.0).all()) and bool((out[0][88:] == 7.0).all())
    lone = torch.empty(c.S, 328, dtype=torch.float32, device=DEV)
    assert c.backward(post, pre, 1.0, out=[None] * 4 + [lone, None, None])[4] is lone
    ref.close(lone, *want["dshift"], "dshift")


@pytest.mark.parametrize("absent", ["dx", "dh"])
@pytest.mark.parametrize("post,pre", [("none", "layer"), ("rms", "rms")])
def test_one_gradient_only(absent, post, pre):
    c = Case(60, 520, [0, 7, 60], 6, True)
    kw = {absent: "nothing"}
    want, got = c.want_back(post, pre, 0.5, **kw), dict(zip(NAMES, c.backward(post, pre, 0.5, **kw)))
    for name in NAMES:
        ref.close(got[name], *want[name], name)


@pytest.mark.parametrize("post,pre", [("rms", "layer"), ("layer", "rms")])
def test_large_mean_and_empty_rows(post, pre):
    """A mean far above the spread, rows of zeros, rows of one value."""
    c = Case(40, 1024, [0, 40], 7, True, mean=100.0)
    c.x[3], c.y[3], c.y[4] = 0.0, 0.0, 5.0
    (x, ex), (h, eh) = c.want(post, pre, 0.5)
    xo, ho = c.forward(post, pre, 0.5)
    ref.close(xo, x, ex, "x")
    ref.close(ho, h, eh, "h")


@pytest.mark.parametrize("D", [512, 520, 1024, 1032, 2048, 2056, 3840, 4096, 4104, 8192])
@pytest.mark.parametrize("wide", [False, True])
def test_many_rows(D, wide):
    """Either side of the number of rows from which fewer waves take a row, and the same rows on both."""
    c = Case(2049, D, [1, 1000, 2047], D, wide)
    (x, ex), (h, eh) = c.want("rms", "layer", 0.75)
    xo, ho = c.forward("rms", "layer", 0.75)
    mine = slice(1, 2047)
    ref.close(xo[mine], x[mine], ex[mine], "x")
    ref.close(ho[mine], h[mine], eh[mine], "h")
    for t in (xo, ho):
        assert bool((t[:1] == 0).all()) and bool((t[2047:] == 0).all())
    c.x, c.y = c.x[:2048], c.y[:2048]
    xo, ho = c.forward("rms", "layer", 0.75)
    ref.close(xo[mine], x[mine], ex[mine], "x")
    ref.close(ho[mine], h[mine], eh[mine], "h")
    assert bool((xo[2047:] == 0).all())


def test_rows_do_not_meet():
    c = Case(50, 264, [0, 25, 50], 8)
    (x, ex), (h, eh) = c.want("rms", "layer", 1.0)
    c.x[10], c.y[11] = float("inf"), float("nan")
    xo, ho = c.forward("rms", "layer", 1.0)
    keep = torch.ones(50, dtype=torch.bool, device=DEV)
    keep[10:12] = False
    ref.close(xo[keep], x[keep], ex[keep])
    ref.close(ho[keep], h[keep], eh[keep])
    assert bool(torch.isnan(ho[10:12]).all())


def test_any_offsets_stay_inside():
    """Offsets that do not ascend, or lead outside of the rows: what they ask for is unspecified, but nothing around the results is written."""
    for ends in ([0, 1000, 50], [40, 20, 10, 70], [-5, 3, 90], [-9, -3], [100, 200, 300], [5, 5, 5], [0], [2147483647, -2147483648, 7]):
        c = Case(50, 264, None, 9)
        c.offsets, c.S = offsets_of(ends), len(ends) - 1
        c.gate = c.scale = c.shift = None
        xp, hp = (torch.full((54, 264), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        c.forward("rms", "layer", 1.0, out=(xp[2:-2], hp[2:-2]))
        sums = torch.full((c.S + 2, 264), 3.0, device=DEV)
        c.backward("rms", "layer", 1.0, out=[xp[2:-2], hp[2:-2], sums[1:-1], None, None, None, None])
        torch.cuda.synchronize()
        for t in (xp[:2], xp[-2:], hp[:2], hp[-2:], sums[:1], sums[-1:]):
            assert bool((t == 3.0).all())


def test_no_rows_and_empty_sequences():
    c = Case(0, 64, [0, 0, 0], 10)
    got = dict(zip(NAMES, c.backward("rms", "rms", 1.0)))
    for name in NAMES[2:]:
        assert bool((got[name] == 0).all())
    assert got["dx"].shape == (0, 64)
    xo, ho = c.forward("rms", "rms", 1.0)
    assert xo.shape == ho.shape == (0, 64)


def test_most_sequences():
    """A sequence for every row but the last ones, as many as are taken."""
    S, D = 65535, 8
    c = Case(S + 4, D, list(range(S + 1)), 15)
    (x, ex), (h, eh) = c.want("none", "rms", 1.0)
    xo, ho = c.forward("none", "rms", 1.0)
    ref.close(xo, x, ex, "x")
    ref.close(ho, h, eh, "h")
    got = dict(zip(NAMES, c.backward("none", "rms", 1.0)))
    seq = slice(0, S)
    n, _, _ = ref.normed(c.x[seq].double(), "rms", EPS)
    dh = c.dh[seq].double()
    ref.close(got["dshift"], dh, torch.zeros_like(dh))
    want = dh * n * c.w_pre.double()
    ref.close(got["dscale"], want, 128 * ref.U * (want.abs() + (dh * c.w_pre.double()).abs() * n.abs()))
    total = (1 + c.scale.double()) * dh * n
    ref.close(got["dw_pre"], total.sum(0), (S + 200) * ref.U * total.abs().sum(0))


def test_in_place():
    c = Case(100, 520, [3, 60, 98], 11)
    xo, ho = c.forward("rms", "layer", 0.5)
    back = c.backward("rms", "layer", 0.5)
    x, y = c.x, c.y
    c.forward("rms", "layer", 0.5, out=(x, y))
    assert torch.equal(x[3:98], xo[3:98]) and torch.equal(y[3:98], ho[3:98]) and bool(torch.isnan(x[:3]).all())
    c = Case(100, 520, [3, 60, 98], 11)
    dx, dh = c.dx, c.dh
    sums = [torch.empty_like(t) for t in back[2:]]
    c.backward("rms", "layer", 0.5, out=[dx, dh] + sums)
    assert torch.equal(dx[3:98], back[0][3:98]) and torch.equal(dh[3:98], back[1][3:98])
    assert all(torch.equal(a, b) for a, b in zip(sums, back[2:]))


def test_shared_vectors_of_stride_zero():
    """One vector for all sequences, as an expanded tensor has it: a row stride of 0 is refused, a copy is not."""
    c = Case(20, 64, [0, 10, 20], 12)
    c.gate = c.gate[:1].expand(2, 64)
    with pytest.raises(rtl.RtlError):
        c.forward("rms", "rms", 1.0)
    c.gate = c.gate.contiguous()
    (x, ex), _ = c.want("rms", "rms", 1.0)
    ref.close(c.forward("rms", "rms", 1.0)[0], x, ex)


def test_against_differences():
    """The gradients are those of the forward formula: central differences in 64 bits."""
    c = Case(6, 24, [0, 2, 6], 13, True)
    post, pre, alpha, e = "layer", "rms", 0.5, 1e-6
    back = dict(zip(NAMES, c.backward(post, pre, alpha)))

    def loss(x_new, y, gate, scale, shift, w_post, w_pre):
        seq = ref.rows_of(c.offsets, 6).to(DEV)
        z = gate[seq] * w_post * ref.normed(y, post, EPS)[0]
        h = w_pre * ref.normed(x_new, pre, EPS)[0] * (1 + scale[seq]) + shift[seq]
        return z, h

    at = dict(x=c.x, y=c.y, gate=c.gate, scale=c.scale, shift=c.shift, w_post=c.w_post, w_pre=c.w_pre)
    at = {k: v.double() for k, v in at.items()}
    base_z = loss(at["x"], at["y"], at["gate"], at["scale"], at["shift"], at["w_post"], at["w_pre"])[0].clone()

    def total(**kw):
        v = dict(at, **kw)
        z = loss(v["x"], v["y"], v["gate"], v["scale"], v["shift"], v["w_post"], v["w_pre"])[0]
        new = v["x"] + (z - base_z)                                # x' moves with z
        h = loss(new, v["y"], v["gate"], v["scale"], v["shift"], v["w_post"], v["w_pre"])[1]
        return ((c.dx.double() * new).sum() + (c.dh.double() * h).sum()).item()

    for name, grad, factor in (("x", "dx", alpha), ("y", "dy", 1.0), ("gate", "dgate", 1.0), ("scale", "dscale", 1.0), ("shift", "dshift", 1.0),
                               ("w_post", "dw_post", 1.0), ("w_pre", "dw_pre", 1.0)):
        want, err = c.want_back(post, pre, alpha)[grad]
        for place in ((0,), (5,), (23,)) if at[name].dim() == 1 else ((0, 0), (-1, 7), (1, 23)):
            up, down = at[name].clone(), at[name].clone()
            up[place] += e
            down[place] -= e
            slope = factor * (total(**{name: up}) - total(**{name: down})) / (2 * e)
            # differences: 1e-16 / e of the loss (below 1e3) and e^2 of the third derivative, both far below 1e-6
            assert abs(back[grad][place].item() - slope) <= err[place].item() + ref.HALF[back[grad].dtype] * abs(slope) + 1e-6 * (1 + abs(slope)), (name, place)


def test_captured_and_replayed():
    c = Case(300, 520, [0, 100, 290], 14)
    c.x, c.y, c.dx, c.dh = (torch.nan_to_num(t).contiguous() for t in (c.x, c.y, c.dx, c.dh))
    first = c.backward("rms", "layer", 1.0)
    out = [torch.zeros_like(t) for t in first]
    fwd = (torch.zeros_like(c.x), torch.zeros_like(c.y))
    ws = torch.empty(rtl.residual_norm_backward_workspace(300, c.S, 520), dtype=torch.uint8, device=DEV)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        c.forward("rms", "layer", 1.0, out=fwd)
        c.backward("rms", "layer", 1.0, out=out, ws=ws)
    for ends in ([0, 100, 290], [0, 10, 300], [5, 5, 200]):
        c.offsets.copy_(offsets_of(ends))
        for t in fwd + tuple(out):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(fwd + tuple(out), c.forward("rms", "layer", 1.0) + c.backward("rms", "layer", 1.0)):
            assert torch.equal(a, b)
