"""Linears grouped by expert and their gradients on the GPU against plain products in 64 bits."""
import numpy as np
import pytest
import torch

import grouped_plan as plan
import mx_ref as ref
from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bf16(gen, *shape, std=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * std).to(torch.bfloat16)


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def offsets_of(counts, front=0):
    return torch.tensor([front + sum(counts[:e]) for e in range(len(counts) + 1)], dtype=torch.int32, device=DEV)


def split(rng, T, E, empty):
    """T rows over E experts, some of them without."""
    w = rng.random(E) ** 2 * (rng.random(E) >= empty)
    w[rng.integers(E)] += 0.1
    return rng.multinomial(T, w / w.sum()).tolist()


def strided(t, pad=8, fill=float("nan")):
    """The same matrix or stack of matrices with rows further apart, NaN between them."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + 2 * pad), fill, dtype=t.dtype, device=DEV)
    wide[..., pad:-pad] = t
    return wide[..., pad:-pad]


# T, E, N, K, share of empty experts: from one row to several tiles an expert, every tile shape, more experts than one wave has lanes, few rows
# on average and more than sixteen of them with one expert
SIZES = [(1, 1, 40, 64, 0.0), (1, 5, 24, 128, 0.0), (7, 3, 264, 192, 0.3), (70, 70, 64, 64, 0.5), (90, 2, 136, 320, 0.0), (300, 130, 72, 128, 0.3),
         (130, 3, 256, 576, 0.0), (500, 4, 200, 256, 0.2), (600, 2, 520, 192, 0.0), (1030, 3, 312, 448, 0.3), (777, 1, 264, 320, 0.0), (60, 8, 96, 704, 0.6),
         (8, 2, 1304, 64, 0.0), (40, 5, 4752, 64, 0.2), (160, 20, 2504, 64, 0.3), (9, 8, 1400, 704, 0.3)]


@pytest.mark.parametrize("T,E,N,K,empty", SIZES)
@pytest.mark.parametrize("bias", [False, True])
def test_forward(T, E, N, K, empty, bias):
    """Any split of the rows; strided operands with NaN between their rows; rows of nobody hold NaN, are not used and stay as they were."""
    gen, rng = generator(T + E + N + K), np.random.default_rng(T * E)
    counts, front, behind = split(rng, T, E, empty), 3, 5
    off = offsets_of(counts, front)
    X = torch.full((front + T + behind, K), float("nan"), dtype=torch.bfloat16, device=DEV)
    X[front:front + T] = bf16(gen, T, K)
    n = N - 3                                                   # no multiple of anything
    W, b = strided(bf16(gen, E, n, K)), bf16(gen, E, n) if bias else None
    for pitch in (n + 4, (n + 23) // 8 * 8):                      # element and 16-byte stores
        full = torch.full((front + T + behind, pitch), 3.0, dtype=torch.bfloat16, device=DEV)
        Y = rtl.grouped_linear(strided(X), off, W, bias=b, out=full[:, :n])
        assert (full[:, n:] == 3.0).all() and (full[:front] == 3.0).all() and (full[front + T:] == 3.0).all()
        o = off.tolist()
        for e in range(E):
            if counts[e]:
                ref.check_product(Y[o[e]:o[e + 1]], ref.values(X[o[e]:o[e + 1]]), ref.values(W[e]), None if b is None else ref.values(b[e]))


DGRAD_SIZES = SIZES + [(1230, 20, 40, 1720, 0.0), (22, 20, 40, 4264, 0.3)]


@pytest.mark.parametrize("T,E,N,K,empty", DGRAD_SIZES)
def test_input_gradient(T, E, N, K, empty):
    gen, rng = generator(T + E + N + K + 1), np.random.default_rng(T * E + 1)
    counts, front, behind = split(rng, T, E, empty), 2, 4
    off = offsets_of(counts, front)
    dY = torch.full((front + T + behind, N), float("nan"), dtype=torch.bfloat16, device=DEV)
    dY[front:front + T] = bf16(gen, T, N)
    k = K - 24                                                    # no multiple of a tile or a 64-wide stage
    W = strided(bf16(gen, E, N, k))
    full = torch.full((front + T + behind, k + 16), 3.0, dtype=torch.bfloat16, device=DEV)
    dX = rtl.grouped_linear_dgrad(strided(dY), off, W, out=full[:, :k])
    assert (full[:, k:] == 3.0).all() and (full[:front] == 3.0).all() and (full[front + T:] == 3.0).all()
    o = off.tolist()
    for e in range(E):
        if counts[e]:
            ref.check_product(dX[o[e]:o[e + 1]], ref.values(dY[o[e]:o[e + 1]]), ref.values(W[e]).T)


WGRAD_SIZES = SIZES + [(700, 2, 1040, 3080, 0.0), (200, 40, 520, 640, 0.5), (5000, 1, 136, 200, 0.0), (7001, 3, 264, 64, 0.3)]


@pytest.mark.parametrize("T,E,N,K,empty", WGRAD_SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weight_and_bias_gradient(T, E, N, K, empty, dtype):
    """Every element is written; NaN in the rows of nobody and between the rows stays out; an expert's NaN reaches its own gradient only."""
    gen, rng = generator(T + E + N + K + 2), np.random.default_rng(T * E + 2)
    counts, front, behind = split(rng, T, E, empty), 70, 90
    off = offsets_of(counts, front)
    dY = torch.full((front + T + behind, N), float("nan"), dtype=torch.bfloat16, device=DEV)
    X = torch.full((front + T + behind, K), float("nan"), dtype=torch.bfloat16, device=DEV)
    dY[front:front + T], X[front:front + T] = bf16(gen, T, N), bf16(gen, T, K)
    sick = None
    if E > 2 and sum(c > 0 for c in counts) > 1:
        sick = next(e for e in range(E) if counts[e])
        X[off[sick], 0] = float("nan")
        dY[off[sick], 1] = float("inf")
    full = torch.full((E + 1, N, K + 8), 3.0, dtype=dtype, device=DEV)
    db = torch.full((E, N), 3.0, dtype=dtype, device=DEV)
    dW, _ = rtl.grouped_linear_wgrad(strided(dY), strided(X), off, out=(full[:E, :, :K], db))
    assert (full[E:] == 3.0).all() and (full[..., K:] == 3.0).all()
    o = off.tolist()
    for e in range(E):
        if e == sick:
            assert torch.isnan(dW[e, :, 0]).all() and not torch.isfinite(db[e, 1])
            continue
        g, x = ref.values(dY[o[e]:o[e + 1]]), ref.values(X[o[e]:o[e + 1]])
        if counts[e] == 0:
            assert (dW[e] == 0).all() and (db[e] == 0).all()
            continue
        ref.check_product(dW[e], g.T, x.T, dtype=dtype)
        ref.check_product(db[e:e + 1], np.ones((1, counts[e])), g.T, dtype=dtype)
    again = rtl.grouped_linear_wgrad(dY, X, off, with_bias=True, dtype=dtype)
    keep = [e for e in range(E) if e != sick]
    assert torch.equal(again[0][keep], dW[keep]) and torch.equal(again[1][keep], db[keep])      # the same bits every time


# rows of the experts, columns of Y in tiles of 256, and the heights that they are cut into
HEIGHTS = [([47, 85, 20], 68, {128}), ([197, 139, 337], 41, {256, 128}), ([0, 768, 5, 0, 900, 1], 40, {256, 128}), ([1024, 512], 41, {256}),
           ([600, 300], 45, {256, 128})]


@pytest.mark.parametrize("counts,tiles_n,want", HEIGHTS)
def test_panels_of_either_height(counts, tiles_n, want):
    """Forward (bf16 and 4-bit) and input gradient on panels of 256 and 128 rows."""
    p = plan.heights(counts, tiles_n, 2)
    left = sum(n // 256 for n in counts) > p or any(n % 256 for n in counts)
    assert want == ({256} if p else set()) | ({128} if left else set())
    gen, rng = generator(11), np.random.default_rng(11)
    T, E, wide = sum(counts), len(counts), tiles_n * 256 - 40
    off = offsets_of(counts)
    o = off.tolist()
    assert plan.forward_form(T, E, wide, 128) == 3 and plan.forward_form(T, E, wide, 512, True) == 3 and plan.dgrad_form(T, E, 128, wide) == 2
    X, W, b = bf16(gen, T, 128), bf16(gen, E, wide, 128), bf16(gen, E, wide)
    Y = rtl.grouped_linear(X, off, W, bias=b)
    X4 = bf16(gen, T, 512)
    wc, wb = ref.random_codes(rng, E * wide, 512)
    wq, ws = ref.on_device(wc, wb)
    Y4 = rtl.grouped_mxfp4_linear(X4, off, wq.reshape(E, wide, 256), ws, bias=b)
    G, V = bf16(gen, T, 128), bf16(gen, E, 128, wide)
    dX = rtl.grouped_linear_dgrad(G, off, V)
    x4 = ref.decode(*ref.quantize(ref.values(X4)))
    w4 = ref.decode(wc, wb).reshape(E, wide, 512)
    for e in range(E):
        if counts[e]:
            r = slice(o[e], o[e + 1])
            ref.check_product(Y[r], ref.values(X[r]), ref.values(W[e]), ref.values(b[e]))
            ref.check_product(Y4[r], x4[r], w4[e], ref.values(b[e]))
            ref.check_product(dX[r], ref.values(G[r]), ref.values(V[e]).T)


def test_sizes_reach_every_form():
    assert {plan.forward_form(T + 8, E, N - 3, K) for T, E, N, K, _ in SIZES} == {0, 1, 2, 3, 4}
    assert {plan.forward_form(T + 3, E, N - 3, K, True) for T, E, N, K, _ in MX_SIZES} == {0, 1, 2, 3, 4}
    assert {plan.dgrad_form(T + 6, E, N, K - 24) for T, E, N, K, _ in DGRAD_SIZES} == {0, 1, 2}
    assert {(s, p > 1) for s, p in (plan.wgrad_form(T + 160, E, N, K) for T, E, N, K, _ in WGRAD_SIZES)} == {(0, False), (1, False), (2, False), (0, True)}


def test_gradients_against_differences():
    """Small integers, so that everything is exact: moving X, W or b by a step changes sum(Y * G) by the step times the gradient."""
    rng = np.random.default_rng(7)
    T, E, N, K = 40, 3, 32, 64
    counts = [11, 0, 29]
    off = offsets_of(counts)
    ints = lambda *s: torch.from_numpy(rng.integers(-1, 2, s)).to(DEV).to(torch.bfloat16)
    X, W, b, G = ints(T, K), ints(E, N, K), ints(E, N), ints(T, N)
    loss = lambda x, w, c: (rtl.grouped_linear(x, off, w, bias=c).double() * G.double()).sum().item()
    dX = rtl.grouped_linear_dgrad(G, off, W)
    dW, db = rtl.grouped_linear_wgrad(G, X, off, with_bias=True, dtype=torch.float32)
    for _ in range(8):
        sx, sw, sb = ints(T, K), ints(E, N, K), ints(E, N)
        assert loss(X + sx, W, b) - loss(X, W, b) == (dX.double() * sx.double()).sum().item()
        assert loss(X, W + sw, b) - loss(X, W, b) == (dW.double() * sw.double()).sum().item()
        assert loss(X, W, b + sb) - loss(X, W, b) == (db.double() * sb.double()).sum().item()


# (the last three: few rows on average of stacks with many columns, quantised by the workgroups and before them; few rows not quantised by them)
MX_SIZES = SIZES + [(64, 32, 300, 992, 0.3), (2000, 3, 700, 544, 0.0), (40, 33, 2051, 288, 0.2), (200, 33, 2051, 2080, 0.2), (60, 8, 96, 1600, 0.6)]


@pytest.mark.parametrize("T,E,N,K,empty", MX_SIZES)
@pytest.mark.parametrize("bias", [False, True])
def test_mxfp4_forward(T, E, N, K, empty, bias):
    gen, rng = generator(T + E + N + K + 3), np.random.default_rng(T * E + 3)
    counts, front, behind = split(rng, T, E, empty), 1, 2
    off = offsets_of(counts, front)
    X = bf16(gen, front + T + behind, K)
    X[front + T:] = float("nan")
    n = N - 3
    wc, wb = ref.random_codes(rng, E * n, K)
    wq, ws = ref.on_device(wc, wb)
    stack = torch.full((E, n, K // 2 + 16), 0x77, dtype=torch.uint8, device=DEV)
    stack[..., :K // 2] = wq.reshape(E, n, K // 2)
    b = bf16(gen, E, n) if bias else None
    full = torch.full((front + T + behind, n + 5), 3.0, dtype=torch.bfloat16, device=DEV)
    Y = rtl.grouped_mxfp4_linear(X, off, stack[..., :K // 2], ws, bias=b, out=full[:, :n])
    assert (full[:, n:] == 3.0).all() and (full[:front] == 3.0).all() and (full[front + T:] == 3.0).all()
    w = ref.decode(wc, wb).reshape(E, n, K)
    o = off.tolist()
    for e in range(E):
        if counts[e]:
            ref.check_product(Y[o[e]:o[e + 1]], ref.decode(*ref.quantize(ref.values(X[o[e]:o[e + 1]]))), w[e], None if b is None else ref.values(b[e]))


def test_one_weight_for_all_experts():
    """A broadcast weight: forward and input gradient use it; its weight gradient has to be a stack of its own."""
    gen = generator(4)
    off = offsets_of([9, 30, 1])
    X, W, G = bf16(gen, 40, 128), bf16(gen, 1, 72, 128), bf16(gen, 40, 72)
    wide = W.expand(3, 72, 128)
    ref.check_product(rtl.grouped_linear(X, off, wide), ref.values(X), ref.values(W[0]))
    ref.check_product(rtl.grouped_linear_dgrad(G, off, wide), ref.values(G), ref.values(W[0]).T)
    with pytest.raises(rtl.RtlError):
        rtl.grouped_linear_wgrad(G, X, off, out=(wide, None))


@pytest.mark.parametrize("bad", [[0, 50, 20, 40], [-7, 10, 20, 90], [60, 40, 20, 0], [0, 2 ** 31 - 1, -2 ** 31, 40], [40, 40, 40, 40]])
def test_offsets_that_are_no_offsets_touch_nothing_else(bad):
    gen = generator(5)
    T, E, N, K = 40, 3, 72, 64
    off = torch.tensor(bad, dtype=torch.int64).to(torch.int32).to(DEV)
    X, W, G = bf16(gen, T, K), bf16(gen, E, N, K), bf16(gen, T, N)
    wq, ws = rtl.quantize_mxfp4(W.reshape(E * N, K))
    for f, width in ((lambda o: rtl.grouped_linear(X, off, W, out=o), N), (lambda o: rtl.grouped_linear_dgrad(G, off, W, out=o), K),
                     (lambda o: rtl.grouped_mxfp4_linear(X, off, wq.reshape(E, N, K // 2), ws, out=o), N)):
        full = torch.full((T + 64, width + 64), 3.0, dtype=torch.bfloat16, device=DEV)
        f(full[32:32 + T, 32:32 + width])
        full[32:32 + T, 32:32 + width] = 3.0
        assert (full == 3.0).all()
    dW, db = rtl.grouped_linear_wgrad(G, X, off, with_bias=True)
    assert torch.isfinite(dW).all() and torch.isfinite(db).all()


def test_no_rows():
    W = torch.randn(3, 16, 64, device=DEV).to(torch.bfloat16)
    off = offsets_of([0, 0, 0])
    X, G = (torch.empty(0, n, dtype=torch.bfloat16, device=DEV) for n in (64, 16))
    assert rtl.grouped_linear(X, off, W).shape == (0, 16) and rtl.grouped_linear_dgrad(G, off, W).shape == (0, 64)
    dW = torch.full_like(W, 5.0)
    rtl.grouped_linear_wgrad(G, X, off, out=(dW, None))
    assert (dW == 0).all()


def test_training_step_captured_and_replayed():
    """Forward and both gradients in one graph on another stream, the rows divided anew between the replays without a word to the host."""
    rtl.init()
    gen = generator(6)
    T, E, N, K = 300, 5, 136, 192
    X, W, G = bf16(gen, T, K), bf16(gen, E, N, K), bf16(gen, T, N)
    b = bf16(gen, E, N)
    off = offsets_of([60] * 5)
    Y, dX = torch.zeros(T, N, dtype=torch.bfloat16, device=DEV), torch.zeros(T, K, dtype=torch.bfloat16, device=DEV)
    dW, db = torch.zeros(E, N, K, device=DEV), torch.zeros(E, N, device=DEV)
    wq, ws = rtl.quantize_mxfp4(W.reshape(E * N, K))
    Yq = torch.zeros_like(Y)
    room = torch.empty(rtl.grouped_mxfp4_linear_workspace(T, E, N, K), dtype=torch.uint8, device=DEV)
    room_w = torch.empty(max(rtl.grouped_linear_wgrad_workspace(T, E, N, K), 256), dtype=torch.uint8, device=DEV)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        rtl.grouped_linear(X, off, W, bias=b, out=Y)
        rtl.grouped_mxfp4_linear(X, off, wq.reshape(E, N, K // 2), ws, bias=b, out=Yq, ws=room)
        rtl.grouped_linear_dgrad(G, off, W, out=dX)
        rtl.grouped_linear_wgrad(G, X, off, out=(dW, db), ws=room_w)
    for counts in ([300, 0, 0, 0, 0], [1, 99, 0, 150, 50], [0, 0, 0, 0, 300], [60] * 5):
        off.copy_(offsets_of(counts))
        X.copy_(bf16(gen, T, K))
        graph.replay()
        want = (rtl.grouped_linear(X, off, W, bias=b), rtl.grouped_mxfp4_linear(X, off, wq.reshape(E, N, K // 2), ws, bias=b),
                rtl.grouped_linear_dgrad(G, off, W), *rtl.grouped_linear_wgrad(G, X, off, with_bias=True, dtype=torch.float32))
        torch.cuda.synchronize()
        for got, w in zip((Y, Yq, dX, dW, db), want):
            assert torch.equal(got, w)


def test_offsets_past_32_bits():
    """More than 2^31 elements in front of the rows that count: the last ones of every operand against the definition."""
    T, E, N, K = 36000, 2, 40, 65536                       # X and dX: 4.7 GB
    off = torch.tensor([0, T - 70, T], dtype=torch.int32, device=DEV)
    gen = generator(8)
    X = torch.zeros(T, K, dtype=torch.bfloat16, device=DEV)
    X[T - 70:] = bf16(gen, 70, K)
    W = bf16(gen, E, N, K)
    G = torch.zeros(T, N, dtype=torch.bfloat16, device=DEV)
    G[T - 70:] = bf16(gen, 70, N)
    x, w, g = X[T - 70:].double(), W[1].double(), G[T - 70:].double()
    half = 2.0 ** -8

    def near(y, a, b):
        want, mag = a @ b.contiguous(), a.abs() @ b.abs().contiguous()
        assert ((y.double() - want).abs() <= (a.shape[1] + 2) * 2.0 ** -24 * mag * (1 + half) + half * want.abs()).all()

    Y = rtl.grouped_linear(X, off, W)
    near(Y[T - 70:], x, w.t())
    assert (Y[:T - 70] == 0).all()
    dX = rtl.grouped_linear_dgrad(G, off, W)
    near(dX[T - 70:], g, w)
    del dX
    dW, _ = rtl.grouped_linear_wgrad(G, X, off)
    near(dW[1], g.t().contiguous(), x)
    assert (dW[0] == 0).all()
    q, s = rtl.quantize_mxfp4(X)
    tail = rtl.quantize_mxfp4(X[T - 70:])
    assert torch.equal(q[T - 70:], tail[0]) and torch.equal(s[:, T - 70:], tail[1])
    values = rtl.dequantize_mxfp4(q, s)
    assert torch.equal(values[T - 70:], rtl.dequantize_mxfp4(*tail))
    del values
    wq, ws = rtl.quantize_mxfp4(W.view(E * N, K))
    Yq = rtl.grouped_mxfp4_linear(X, off, wq.view(E, N, K // 2), ws)
    near(Yq[T - 70:], rtl.dequantize_mxfp4(*tail).double(), rtl.dequantize_mxfp4(wq, ws)[N:].double().t())


@pytest.mark.parametrize("T,offsets", [(1, [0, 1]), (1, [1, 1]), (9, [0, 4, 9]), (9, [3, 3, 5]), (9, [9]), (700, [1, 2, 699]), (700, [690, 700]), (40, [-5, 7, 90]),
                                       (40, [2 ** 31 - 1, -2 ** 31]), (40, [30, 10, 20])])
@pytest.mark.parametrize("cols,front", [(1, 0), (7, 1), (64, 0), (1027, 3), (1024, 8)])
def test_clear_rows_of_no_expert(T, offsets, cols, front):
    """Zeros in the rows before the first expert's and behind the last one's, at any alignment; the others, and what lies between rows, stay."""
    full = torch.full((T, cols + front + 5), float("nan"), dtype=torch.bfloat16, device=DEV)
    rtl.grouped_clear(torch.tensor(offsets, dtype=torch.int32, device=DEV), full[:, front:front + cols])
    first = min(max(offsets[0], 0), T)
    last = max(first, min(max(offsets[-1], 0), T))
    want = torch.full_like(full, float("nan"))
    want[:first, front:front + cols] = 0
    want[last:, front:front + cols] = 0
    assert torch.equal(full.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("offsets", [[4, 10, 10, 25], [0, 0, 0, 0], [31, 31, 31, 31], [0, 5, 20, 31]])
def test_new_results_hold_zeros_in_rows_of_no_expert(offsets):
    """Results the calls allocate, in memory that held NaN before; three experts, and none at all."""
    gen, T, N, K, first, last = generator(3), 31, 72, 64, offsets[0], offsets[-1]
    X, G, W = bf16(gen, T, K), bf16(gen, T, N), bf16(gen, 3, N, K)
    off, (Wq, Ws) = torch.tensor(offsets, dtype=torch.int32, device=DEV), rtl.quantize_mxfp4(W.view(3 * N, K))
    calls = [lambda out=None: rtl.grouped_linear(X, off, W, out=out), lambda out=None: rtl.grouped_linear_dgrad(G, off, W, out=out),
             lambda out=None: rtl.grouped_mxfp4_linear(X, off, Wq.view(3, N, K // 2), Ws, out=out)]
    for call, cols in zip(calls, (N, K, N)):
        for _ in range(3):
            dirty = torch.full((T, cols), float("nan"), dtype=torch.bfloat16, device=DEV)
            given = call(torch.zeros_like(dirty))
            del dirty
            new = call()
            assert torch.equal(new.view(torch.int16), given.view(torch.int16))
            assert (new[:first] == 0).all() and (new[last:] == 0).all()
    empty = rtl.grouped_linear(X, off[:1].contiguous(), W[:0])
    assert empty.shape == (T, N) and (empty == 0).all()


def test_weight_gradient_of_more_experts_than_rows():
    """40000 experts of one small tile each: every expert's gradient, in small integers and so exact."""
    gen = generator(21)
    T, E, N, K = 30000, 40000, 8, 16
    where = torch.sort(torch.randint(0, E, (T,), generator=gen, device=DEV)).values
    counts = torch.bincount(where, minlength=E)
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), counts.cumsum(0)]).to(torch.int32)
    X, G = (torch.randint(-3, 4, (T, n), generator=gen, device=DEV).to(torch.bfloat16) for n in (K, N))
    dW = torch.full((E, N, K), 7.0, device=DEV)
    db = torch.full((E, N), 7.0, device=DEV)
    rtl.grouped_linear_wgrad(G, X, off, out=(dW, db))
    want = torch.zeros(E, N, K, device=DEV).index_add_(0, where, G.float()[:, :, None] * X.float()[:, None, :])
    assert torch.equal(dW, want) and torch.equal(db, torch.zeros(E, N, device=DEV).index_add_(0, where, G.float()))


def test_weight_gradient_of_a_large_stack():
    """More than 2^18 tiles of 128 x 128: 52 experts of [16384, 5120], rows with three of them."""
    gen = generator(22)
    E, N, K = 52, 16384, 5120
    counts = [0] * E
    counts[0], counts[30], counts[51] = 3, 70, 1
    off = offsets_of(counts)
    X, G = bf16(gen, sum(counts), K), bf16(gen, sum(counts), N)
    dW = torch.full((E, N, K), 7.0, dtype=torch.bfloat16, device=DEV)
    db = torch.full((E, N), 7.0, dtype=torch.bfloat16, device=DEV)
    rtl.grouped_linear_wgrad(G, X, off, out=(dW, db))
    o, pick = off.tolist(), torch.randint(0, N, (64,), generator=gen, device=DEV)
    pick[0], pick[1] = 0, N - 1
    for e in range(E):
        if counts[e] == 0:
            assert (dW[e] == 0).all() and (db[e] == 0).all()
            continue
        r = slice(o[e], o[e + 1])
        ref.check_product(dW[e][pick], ref.values(G[r][:, pick]).T, ref.values(X[r]).T)
        ref.check_product(db[e:e + 1], np.ones((1, counts[e])), ref.values(G[r]).T)


def test_products_of_a_large_stack():
    """Weights of more than 2^31 elements: the last expert's rows of forward, input gradient and 4-bit product."""
    gen = generator(23)
    E, N, K = 52, 16384, 5120
    counts = [0] * E
    counts[0], counts[50], counts[51] = 2, 40, 9
    off, T = offsets_of(counts), sum(counts)
    W = torch.zeros(E, N, K, dtype=torch.bfloat16, device=DEV)
    for e in (0, 50, 51):
        W[e] = bf16(gen, N, K, std=0.05)
    X, G, pick = bf16(gen, T, K), bf16(gen, T, N), torch.cat([torch.arange(40, device=DEV), torch.arange(N - 40, N, device=DEV)])
    Y, dX = rtl.grouped_linear(X, off, W), rtl.grouped_linear_dgrad(G, off, W)
    wq, ws = rtl.quantize_mxfp4(W.view(E * N, K))
    Y4 = rtl.grouped_mxfp4_linear(X, off, wq.view(E, N, K // 2), ws)
    x4, o = ref.decode(*ref.quantize(ref.values(X))), off.tolist()
    for e in (0, 50, 51):
        r = slice(o[e], o[e + 1])
        ref.check_product(Y[r][:, pick], ref.values(X[r]), ref.values(W[e][pick]))
        ref.check_product(dX[r][:, :80], ref.values(G[r]), ref.values(W[e][:, :80]).T)
        ref.check_product(Y4[r][:, pick], x4[r], ref.decode(*ref.quantize(ref.values(W[e][pick]))))


@pytest.mark.parametrize("counts", [[130, 0, 126], [3, 7, 1]])
def test_row_strides_at_the_limit(counts):
    """Row strides of 2^22 elements, the largest that is taken: matrices that are the first columns of much wider ones."""
    gen, ld, T, E, N, K = generator(24), 1 << 22, sum(counts), len(counts), 256, 192
    off = offsets_of(counts)

    def wide(t):
        full = torch.empty(t.shape[0], ld, dtype=t.dtype, device=DEV)
        view = full[:, 8:8 + t.shape[1]]
        view.copy_(t)
        return view

    X, G, W = wide(bf16(gen, T, K)), wide(bf16(gen, T, N)), wide(bf16(gen, E * N, K)).unflatten(0, (E, N))
    Y, dX = wide(torch.zeros(T, N, dtype=torch.bfloat16, device=DEV)), wide(torch.zeros(T, K, dtype=torch.bfloat16, device=DEV))
    dW = wide(torch.zeros(E * N, K, dtype=torch.bfloat16, device=DEV)).unflatten(0, (E, N))
    rtl.grouped_linear(X, off, W, out=Y)
    rtl.grouped_linear_dgrad(G, off, W, out=dX)
    rtl.grouped_linear_wgrad(G, X, off, out=(dW, None))
    o = off.tolist()
    for e in range(E):
        r = slice(o[e], o[e + 1])
        if counts[e]:
            ref.check_product(Y[r], ref.values(X[r]), ref.values(W[e]))
            ref.check_product(dX[r], ref.values(G[r]), ref.values(W[e]).T)
            ref.check_product(dW[e], ref.values(G[r]).T, ref.values(X[r]).T)
        else:
            assert (dW[e] == 0).all()


@pytest.mark.parametrize("T", [300, 70000])
def test_as_many_experts_as_are_taken(T):
    """65536 experts; small integers, so that every sum is exact, in 4 bits too."""
    gen, E, N, K = generator(25), 65536, 24, 64
    where = torch.sort(torch.randint(0, E, (T,), generator=gen, device=DEV)).values
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), torch.bincount(where, minlength=E).cumsum(0)]).to(torch.int32)
    ints = lambda *s: torch.randint(-3, 4, s, generator=gen, device=DEV).to(torch.bfloat16)
    X, G, W, b = ints(T, K), ints(T, N), ints(E, N, K), ints(E, N)
    Y = (W[where].float() @ X.float()[:, :, None])[:, :, 0]
    bf = lambda t: t.to(torch.bfloat16)
    assert torch.equal(rtl.grouped_linear(X, off, W, bias=b), bf(Y + b[where].float()))
    wq, ws = rtl.quantize_mxfp4(W.view(E * N, K))
    assert torch.equal(rtl.grouped_mxfp4_linear(X, off, wq.view(E, N, K // 2), ws, bias=b), bf(Y + b[where].float()))
    assert torch.equal(rtl.grouped_linear_dgrad(G, off, W), bf((G.float()[:, None, :] @ W[where].float())[:, 0]))
    dW, db = rtl.grouped_linear_wgrad(G, X, off, with_bias=True, dtype=torch.float32)
    assert torch.equal(dW, torch.zeros(E, N, K, device=DEV).index_add_(0, where, G.float()[:, :, None] * X.float()[:, None, :]))
    assert torch.equal(db, torch.zeros(E, N, device=DEV).index_add_(0, where, G.float()))
