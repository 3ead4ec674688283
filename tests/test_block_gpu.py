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
