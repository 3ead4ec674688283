"""The block operators together, as a transformer block uses them, on the GPU: every step against its formula on what the step before it left."""
import pytest
import torch

import block_ref as ref
from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


class Block:
    """Two sequences, rows of nobody behind them, the feed-forward half of a block and the heads of its attention, forward and backward."""
    T, D, F, H, head, pairs = 333, 384, 520, 3, 128, 48

    def __init__(self, seed):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        bf = lambda *s, std=1.0, mean=0.0: (torch.randn(*s, generator=gen, device=DEV) * std + mean).to(torch.bfloat16)  # noqa: E731
        self.x = torch.randn(self.T, self.D, generator=gen, device=DEV) * 2
        self.offsets = torch.tensor([0, 130, 320], dtype=torch.int32, device=DEV)
        self.mod = bf(2, 6 * self.D, std=0.3)
        self.w_in, self.w_pre, self.w_post = bf(self.D, mean=1.0, std=0.1), bf(self.D, mean=1.0, std=0.1), bf(self.D, mean=1.0, std=0.1)
        self.w_qkv, self.w_up, self.w_down = bf(3 * self.H * self.head, self.D, std=0.05), bf(2 * self.F, self.D, std=0.05), bf(self.D, 576, std=0.05)
        self.wq, self.wk = bf(self.head, mean=1.0, std=0.1), bf(self.head, mean=1.0, std=0.1)
        self.pos = torch.arange(self.T, device=DEV).float()[:, None] * torch.tensor([0.25, 1.0], device=DEV)
        self.freq = torch.rand(self.pairs, generator=gen, device=DEV)
        self.axis = (torch.arange(self.pairs, device=DEV) % 2).to(torch.int32)
        self.grad_x, self.grad_h = torch.randn(self.T, self.D, generator=gen, device=DEV), bf(self.T, self.D)
        self.hidden = torch.zeros(self.T, 576, dtype=torch.bfloat16, device=DEV)      # 520 columns and zeros up to what the down product takes

    def part(self, i):
        return self.mod[:, i * self.D:(i + 1) * self.D]

    def run(self):
        """All steps, none waits for the host. Returns them by name."""
        r = {}
        first = dict(w_pre=self.w_in, scale=self.part(1), offsets=self.offsets, pre="layer", eps=EPS)
        last = dict(gate=self.part(2), w_post=self.w_post, w_pre=self.w_pre, scale=self.part(4), offsets=self.offsets, post="rms", pre="rms", eps=EPS)
        r["h"] = rtl.residual_norm(self.x, shift=self.part(0), with_x=False, **first)[1]
        qkv = rtl.dense_linear(r["h"], self.w_qkv)
        n = self.H * self.head
        r["q0"], r["k0"] = (qkv[:, i * n:(i + 1) * n].view(self.T, self.H, self.head) for i in range(2))
        r["q"], r["k"] = rtl.norm_rotary(r["q0"], r["k0"], self.pos, self.freq, self.axis, self.wq, self.wk, eps=EPS)
        _, r["p"] = rtl.gated_linear(r["h"], self.w_up, out=self.hidden[:, :self.F], with_pre=True)
        r["a"] = self.hidden[:, :self.F]
        r["y"] = rtl.dense_linear(self.hidden, self.w_down)
        r["x1"], r["h1"] = rtl.residual_norm(self.x, r["y"], shift=self.part(3), **last)
        back = rtl.residual_norm_backward(self.grad_x, self.grad_h, r["x1"], r["y"], **last)
        r.update(zip(("dx", "dy", "dgate", "dscale", "dshift", "dw_post", "dw_pre"), back))
        one = torch.tensor([0, self.T], dtype=torch.int32, device=DEV) if not hasattr(self, "one") else self.one
        self.one = one
        r["da"] = rtl.grouped_linear_dgrad(r["dy"], one, self.w_down[None])[:, :self.F]
        r["dh"], r["dw_up"], _, r["a2"] = rtl.gated_linear_backward(r["da"], r["h"], self.w_up, r["p"], with_hidden=True)
        r["dq"], r["dk"], r["dwq"], r["dwk"] = rtl.norm_rotary_backward(r["q"], r["k"], r["q0"], r["k0"], self.pos, self.freq, self.axis, self.wq, self.wk, eps=EPS)
        r["dx0"] = rtl.residual_norm_backward(r["dx"], r["dh"], self.x, **first)[0]
        return r


def test_steps():
    b = Block(1)
    r = b.run()
    S, off = 2, b.offsets
    _, h = ref.residual_norm(b.x, None, None, None, b.w_in, b.part(1), b.part(0), off, "none", "layer", 1.0, EPS)
    ref.close(r["h"], *h, "h")
    for name, w in (("q", b.wq), ("k", b.wk)):
        ref.close(r[name], *ref.norm_rotary(r[name + "0"], b.pos, b.freq, b.axis, w, "rms", EPS, True), name)
        want, dw = ref.norm_rotary_backward(r[name], r[name + "0"], b.pos, b.freq, b.axis, w, "rms", EPS, True)
        ref.close(r["d" + name], *want, "d" + name)
        ref.close(r["dw" + name], *dw, "dw" + name)
    a, ea, p, ep = ref.gated(r["h"], b.w_up, None, "silu")
    ref.close(r["a"], a, ea, "a")
    ref.close(r["p"], p, ep, "p")
    x1, h1 = ref.residual_norm(b.x, r["y"], b.part(2), b.w_post, b.w_pre, b.part(4), b.part(3), off, "rms", "rms", 1.0, EPS)
    ref.close(r["x1"], *x1, "x1")
    ref.close(r["h1"], *h1, "h1")
    want = ref.residual_norm_backward(b.grad_x, b.grad_h, r["x1"], r["y"], b.part(2), b.w_post, b.w_pre, b.part(4), off, "rms", "rms", 1.0, EPS)
    for name, (value, err) in want.items():
        assert value.shape[0] in (S, b.T, b.D)
        ref.close(r[name], value, err, name)
    want = ref.gated_backward(r["da"], r["h"], b.w_up, r["p"], "silu")
    ref.close(r["dh"], *want["dX"], "dh")
    ref.close(r["dw_up"], *want["dW"], "dw_up")
    ref.close(r["a2"], *want["H"], "a2")
    want = ref.residual_norm_backward(r["dx"], r["dh"], b.x, None, None, None, b.w_in, b.part(1), off, "none", "layer", 1.0, EPS)
    ref.close(r["dx0"], *want["dx"], "dx0")


def test_captured_together():
    """The whole run as one graph, replayed on other inputs, with eager runs and synchronisations between the replays."""
    b = Block(2)
    b.run()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        got = b.run()
    for seed in (3, 4, 5):
        other = Block(seed)
        for name in ("x", "mod", "w_up", "w_qkv", "grad_x", "grad_h", "pos"):
            getattr(b, name).copy_(getattr(other, name))
        for name in ("w_in", "w_pre", "w_post", "w_down", "wq", "wk", "freq"):
            getattr(b, name).copy_(getattr(other, name))
        graph.replay()
        torch.cuda.synchronize()
        kept = {k: v.clone() for k, v in got.items()}
        eager = other.run()
        torch.cuda.synchronize()
        for name, value in eager.items():
            assert torch.equal(kept[name], value), name


def test_two_streams_at_once():
    """Two blocks side by side on streams of their own, each call with a workspace of its own."""
    blocks, want = [Block(6), Block(7)], []
    for b in blocks:
        want.append({k: v.clone() for k, v in b.run().items()})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    got = [None, None]
    for _ in range(3):
        for i, (b, s) in enumerate(zip(blocks, streams)):
            with torch.cuda.stream(s):
                got[i] = b.run()
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for name in w:
            assert torch.equal(g[name], w[name]), name


@pytest.fixture
def large():
    """Gives the memory of large tensors back."""
    yield
    torch.cuda.empty_cache()


def far(t, ld=(1 << 23) + 8):
    """The same values in rows so far apart that the last ones lie more than 2^32 bytes behind the first."""
    assert (t.shape[0] - 1) * ld * t.element_size() > 1 << 32
    wide = torch.empty(t.shape[0] * ld, dtype=t.dtype, device=DEV).as_strided(t.shape, (ld,) + tuple(t.stride()[1:]))
    wide.copy_(t)
    return wide


def same(got, want):
    assert all((g is None and w is None) or torch.equal(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("M,F", [(300, 100), (1030, 4), (2080, 516)])
def test_gated_rows_far_apart(M, F, large):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(M)
    X, W, dH = (torch.randn(*s, generator=gen, device=DEV).to(torch.bfloat16) for s in ((M, 64), (2 * F, 64), (M, F)))
    H, P = rtl.gated_linear(X, W, with_pre=True)
    ld = (1 << 33) // M // 8 * 8                                  # (X and dX up to 2^22)
    ldx = min(ld, 1 << 22)
    big = [far(torch.zeros_like(H), ld), far(torch.zeros_like(P), ld)]
    wide_x = far(X, ldx) if (M - 1) * ldx * 2 > 1 << 32 else X
    rtl.gated_linear(wide_x, W, out=big[0], pre=big[1])
    same(big, (H, P))
    want = rtl.gated_linear_backward(dH, X, W, P, with_hidden=True)
    big[0].zero_()
    wide_dx = torch.zeros_like(X) if wide_x is X else far(torch.zeros_like(X), ldx)
    got = rtl.gated_linear_backward(far(dH, ld), wide_x, W, big[1], out=[wide_dx, torch.zeros_like(W), None, big[0]])
    same(got, want)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_norm_rows_far_apart(kind, large):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    T, D = 300, 264
    x, dx = (torch.randn(T, D, generator=gen, device=DEV).to(kind) for _ in range(2))
    y, dh = (torch.randn(T, D, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    gate, scale, shift = (torch.randn(2, D, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(3))
    offsets = torch.tensor([1, 100, 298], dtype=torch.int32, device=DEV)
    how = dict(offsets=offsets, post="rms", pre="layer")
    want = rtl.residual_norm(x, y, gate=gate, scale=scale, shift=shift, **how)
    fx, fy = far(x), far(y)
    big = [far(torch.zeros_like(w)) for w in want]
    same(rtl.residual_norm(fx, fy, gate=gate, scale=scale, shift=shift, out=big, **how), want)
    want = rtl.residual_norm_backward(dx, dh, x, y, gate=gate, scale=scale, **how)
    for t in big:
        t.zero_()
    same(rtl.residual_norm_backward(far(dx), far(dh), fx, fy, gate=gate, scale=scale, out=big + [None if w is None else torch.empty_like(w) for w in want[2:]], **how),
         want)


@pytest.mark.parametrize("interleaved", [True, False])
def test_tokens_and_heads_far_apart(interleaved, large):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(4)
    T, H, D = 9, 300, 32
    q, k = (torch.randn(T, H, D, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    w = torch.randn(D, generator=gen, device=DEV).to(torch.bfloat16)
    pos, freq = torch.randn(T, 2, generator=gen, device=DEV), torch.rand(16, generator=gen, device=DEV)
    axis = torch.arange(16, dtype=torch.int32, device=DEV) % 2
    fq, fk = far(q, (1 << 28) + 8), far(k.transpose(0, 1)).transpose(0, 1)             # tokens, and heads
    want = rtl.norm_rotary(q, k, pos, freq, axis, w, w, interleaved=interleaved)
    out = [far(torch.zeros_like(q), (1 << 28) + 8), far(torch.zeros_like(k).transpose(0, 1)).transpose(0, 1)]
    same(rtl.norm_rotary(fq, fk, pos, freq, axis, w, w, interleaved=interleaved, out=out), want)
    want = rtl.norm_rotary_backward(k, q, q, k, pos, freq, axis, w, w, interleaved=interleaved)
    gq, gk = far(k, (1 << 28) + 8), far(q.transpose(0, 1)).transpose(0, 1)
    same(rtl.norm_rotary_backward(gq, gk, fq, fk, pos, freq, axis, w, w, interleaved=interleaved, out=out + [torch.empty(D, device=DEV), torch.empty(D, device=DEV)]),
         want)
