"""Head norm and rotary positions, and their gradients, on the GPU against the formulas in 64 bits."""
import pytest
import torch

import block_ref as ref
from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def normal(gen, *shape, std=1.0, mean=0.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(torch.bfloat16)


def rotation(gen, T, pairs, axes, far=100.0):
    pos = (torch.randn(T, axes, generator=gen, device=DEV) * far).round()
    if axes > 1:
        pos[:, 0] /= 24.0                                          # no whole numbers
    axis = torch.randint(0, axes, (pairs,), generator=gen, device=DEV).to(torch.int32)
    freq = torch.rand(pairs, generator=gen, device=DEV).pow(4)
    return pos, freq, axis


# T, Hq, Hk, D, pairs: one token, head widths of every lane count and odd ones, parts of the head, shared key heads, without q or k
SIZES = [(1, 32, 8, 128, 64), (1, 1, 1, 8, 0), (3, 5, 5, 16, 8), (7, 2, 1, 24, 8), (33, 4, 4, 64, 32), (10, 30, 30, 128, 64), (65, 3, 3, 72, 24), (19, 16, 2, 80, 40),
         (40, 7, 0, 96, 48), (12, 0, 9, 136, 8), (100, 9, 3, 256, 128), (9, 3, 1, 264, 64), (5, 2, 2, 512, 256), (700, 12, 4, 64, 16), (5000, 2, 1, 128, 48)]


@pytest.mark.parametrize("T,Hq,Hk,D,pairs", SIZES)
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("norm,axes", [("rms", 3), ("none", 1)])
def test_forward_and_backward(T, Hq, Hk, D, pairs, interleaved, norm, axes):
    gen = generator(T + Hq + D)
    qkv = normal(gen, T, (Hq + 2 * Hk) * D + 8, std=2.0)             # one product that gives q, k and v
    q, k = qkv[:, :Hq * D].view(T, Hq, D), qkv[:, Hq * D:(Hq + Hk) * D].view(T, Hk, D)
    wq, wk = (normal(gen, D, std=0.3, mean=1.0), normal(gen, D, std=0.3, mean=1.0)) if norm == "rms" else (None, None)
    pos, freq, axis = rotation(gen, T, pairs, axes)
    q, k = q if Hq else None, k if Hk else None
    how = dict(norm=norm, eps=EPS, interleaved=interleaved)
    got = rtl.norm_rotary(q, k, pos, freq, axis, wq, wk, **how)
    for t, v, w in ((got[0], q, wq), (got[1], k, wk)):
        assert (t is None) == (v is None)
        if v is not None:
            ref.close(t, *ref.norm_rotary(v, pos, freq, axis, w, norm, EPS, interleaved), "forward")
    # results with heads in front of tokens, into a larger tensor
    dq, dk = (normal(gen, T, H, D) if H else None for H in (Hq, Hk))
    back = rtl.norm_rotary_backward(dq, dk, q if norm == "rms" else None, k if norm == "rms" else None, pos, freq, axis, wq, wk, **how)
    for i, (dv, v, w) in enumerate(((dq, q, wq), (dk, k, wk))):
        if v is None:
            assert back[i] is None
            if w is not None:
                assert bool((back[i + 2] == 0).all())
            continue
        want, dw = ref.norm_rotary_backward(dv, v, pos, freq, axis, w, norm, EPS, interleaved)
        ref.close(back[i], *want, "backward")
        if dw is None:
            assert back[i + 2] is None
        else:
            ref.close(back[i + 2], *dw, "dw")
    again = rtl.norm_rotary_backward(dq, dk, q, k, pos, freq, axis, wq, wk, **how)
    assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(back, again))


@pytest.mark.parametrize("interleaved", [True, False])
def test_layouts(interleaved):
    """Heads in front of tokens, results inside larger tensors, in place."""
    gen = generator(1)
    T, Hq, Hk, D, pairs = 50, 6, 3, 80, 32
    q, k = normal(gen, T, Hq, D), normal(gen, T, Hk, D)
    wq, wk = normal(gen, D, mean=1.0, std=0.2), normal(gen, D, mean=1.0, std=0.2)
    pos, freq, axis = rotation(gen, T, pairs, 2)
    how = dict(interleaved=interleaved)
    want = rtl.norm_rotary(q, k, pos, freq, axis, wq, wk, **how)
    qh, kh = q.transpose(0, 1).contiguous().transpose(0, 1), k.transpose(0, 1).contiguous().transpose(0, 1)
    full = torch.full((Hq + Hk + 1, T + 1, D + 8), 3.0, dtype=torch.bfloat16, device=DEV)
    out = full[:Hq, :T, :D].transpose(0, 1), full[Hq:Hq + Hk, :T, :D].transpose(0, 1)
    got = rtl.norm_rotary(qh, kh, pos, freq, axis, wq, wk, out=out, **how)
    assert got[0] is out[0] and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert bool((full[..., D:] == 3.0).all()) and bool((full[:, T:] == 3.0).all()) and bool((full[Hq + Hk:] == 3.0).all())
    dq, dk = normal(gen, T, Hq, D), normal(gen, T, Hk, D)
    back = rtl.norm_rotary_backward(dq, dk, qh, kh, pos, freq, axis, wq, wk, **how)
    rtl.norm_rotary_backward(dq, dk, q, k, pos, freq, axis, wq, wk, out=(dq, k.clone(), None, None), **how)
    assert torch.equal(dq, back[0])
    rtl.norm_rotary(q, k, pos, freq, axis, wq, wk, out=(q, k), **how)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_far_positions():
    """Angles of 10^8 and more: in 32 bits they would be off by whole radians."""
    gen = generator(2)
    T, H, D, pairs = 64, 2, 64, 32
    q = normal(gen, T, H, D)
    pos = (torch.rand(T, 1, generator=gen, device=DEV) * 2 ** 24).round() * torch.where(torch.arange(T, device=DEV) % 2 == 0, 1.0, -1.0)[:, None]
    freq = torch.cat([torch.tensor([1.0, 0.1, 31.0, 63.9], device=DEV), torch.rand(28, generator=gen, device=DEV)])
    axis = torch.zeros(pairs, dtype=torch.int32, device=DEV)
    got, _ = rtl.norm_rotary(q, None, pos, freq, axis, norm="none")
    ref.close(got, *ref.norm_rotary(q, pos, freq, axis, None, "none", EPS, True))


def test_quarter_turns():
    """Every quarter of the turn, its borders and both signs."""
    pairs = 256
    q = torch.zeros(1, 1, 512, dtype=torch.bfloat16, device=DEV)
    q[..., 0::2] = 1.0
    freq = torch.linspace(-14.0, 14.0, pairs, device=DEV)
    axis = torch.zeros(pairs, dtype=torch.int32, device=DEV)
    got, _ = rtl.norm_rotary(q, None, torch.ones(1, 1, device=DEV), freq, axis, norm="none")
    ref.close(got, *ref.norm_rotary(q, torch.ones(1, 1, device=DEV), freq, axis, None, "none", EPS, True))


def test_axis_outside_and_special_values():
    gen = generator(3)
    q = normal(gen, 4, 2, 16)
    pos, freq = normal(gen, 4, 2).float(), torch.rand(8, device=DEV)
    axis = torch.tensor([0, 1, 2, 7, -1, -9, 1, 0], dtype=torch.int32, device=DEV)        # cut to 0 and 1
    got, _ = rtl.norm_rotary(q, None, pos, freq, axis, norm="none")
    ref.close(got, *ref.norm_rotary(q, pos, freq, axis.clamp(0, 1), None, "none", EPS, True))
    q[1, 0, 3], q[2, 1, 5] = float("nan"), float("inf")
    pos[3, 0] = float("nan")
    bad, _ = rtl.norm_rotary(q, None, pos, freq, axis, norm="rms", eps=EPS)
    assert bool(torch.isnan(bad[1, 0]).all()) and bool(torch.isfinite(bad[1, 1]).all()) and bool(torch.isfinite(bad[2, 0]).all())
    assert bool(torch.isnan(bad[3, :, 0]).all()) and bool(torch.isfinite(bad[3, :, 2:8]).all()) and bool(torch.isfinite(bad[0]).all())


def test_zero_heads_and_no_tokens():
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=DEV)
    assert bool((rtl.norm_rotary(q, None, None, None, None)[0] == 0).all())
    e = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    w = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    assert rtl.norm_rotary(e, e, None, None, None, w, w)[0].shape == (0, 2, 64)
    back = rtl.norm_rotary_backward(e, e, e, e, None, None, None, w, w)
    assert bool((back[2] == 0).all()) and bool((back[3] == 0).all())


def test_norm_alone():
    gen = generator(4)
    q, k = normal(gen, 30, 4, 96), normal(gen, 30, 2, 96)
    got = rtl.norm_rotary(q, k, None, None, None, eps=EPS)
    for t, v in zip(got, (q, k)):
        ref.close(t, *ref.norm_rotary(v, None, None, None, None, "rms", EPS, True))


def test_turning_back():
    """Without a norm the backward pass is the turn by the negative angle: forward and back gives the values again."""
    gen = generator(5)
    q = normal(gen, 40, 3, 128)
    pos, freq, axis = rotation(gen, 40, 64, 3)
    there, _ = rtl.norm_rotary(q, None, pos, freq, axis, norm="none")
    back = rtl.norm_rotary_backward(there, None, None, None, pos, freq, axis, norm="none")[0]
    # the values of `there` are off by half a step each, and the result by its own
    length = torch.sqrt(q.double()[..., 0::2] ** 2 + q.double()[..., 1::2] ** 2).repeat_interleave(2, -1)
    ref.close(back, q.double(), (2 ** 0.5 * ref.HALF[torch.bfloat16] + 64 * ref.U + 1e-8) * length)


def test_more_tokens_than_waves_are_launched_for():
    """So many that a wave goes over a token's heads twice; rows across the tensor against the formula, all of them against a call on the last ones."""
    gen = generator(8)
    T, H, D = (1 << 22) + 5, 17, 8
    q = normal(gen, T, H, D)
    w = normal(gen, D, std=0.1, mean=1.0)
    pos, freq, axis = rotation(gen, T, 4, 2)
    out = rtl.norm_rotary(q, None, pos, freq, axis, w)[0]
    some = torch.cat([torch.arange(0, T, 40009, device=DEV), torch.arange(T - 9, T, device=DEV)])
    ref.close(out[some], *ref.norm_rotary(q[some], pos[some], freq, axis, w, "rms", EPS, True), "forward")
    half = T // 2
    assert torch.equal(out[:half], rtl.norm_rotary(q[:half], None, pos[:half], freq, axis, w)[0])
    assert torch.equal(out[half:], rtl.norm_rotary(q[half:], None, pos[half:], freq, axis, w)[0])
    del q, out, pos
    torch.cuda.empty_cache()


def test_captured_and_replayed():
    gen = generator(6)
    q, k = normal(gen, 200, 6, 64), normal(gen, 200, 2, 64)
    wq, wk = normal(gen, 64, mean=1.0, std=0.1), normal(gen, 64, mean=1.0, std=0.1)
    pos, freq, axis = rotation(gen, 200, 32, 2)
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    out, back = (torch.empty_like(q), torch.empty_like(k)), (dq, dk, torch.empty(64, device=DEV), torch.empty(64, device=DEV))
    ws = torch.empty(rtl.norm_rotary_backward_workspace(64), dtype=torch.uint8, device=DEV)
    rtl.init()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        rtl.norm_rotary(q, k, pos, freq, axis, wq, wk, out=out)
        rtl.norm_rotary_backward(out[0], out[1], q, k, pos, freq, axis, wq, wk, out=back, ws=ws)
    for _ in range(3):
        pos.copy_((pos + 7.0))
        graph.replay()
        torch.cuda.synchronize()
        a = rtl.norm_rotary(q, k, pos, freq, axis, wq, wk)
        b = rtl.norm_rotary_backward(a[0], a[1], q, k, pos, freq, axis, wq, wk)
        assert all(torch.equal(x, y) for x, y in zip(out + back, a + b))
