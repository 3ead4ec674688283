"""Contractions long enough for every tile form of the 4-bit and grouped products to go round its ring of LDS buffers more than twice, so that buffers
are requested again while others are read; each with and without a last block that is not full. Sampled rows and columns against products in 64 bits."""
import numpy as np
import pytest
import torch

import grouped_plan as plan
import mx_ref as ref
from paper_2605_26632_amd import binding as rtl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def bf16(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV).to(torch.bfloat16)


def codes(gen, rows, cols):
    """Random codes and scales on the device; the scale bytes behind the last block are random too (they count as nothing)."""
    mid = 127 - int(np.log2(cols) / 2)
    return (torch.randint(0, 256, (rows, cols // 2), generator=gen, device=DEV, dtype=torch.uint8),
            torch.randint(mid - 4, mid + 5, rtl.mxfp4_scales_shape(rows, cols), generator=gen, device=DEV, dtype=torch.uint8))


def decoded(q, s, rows):
    """Values of some rows of codes and scales."""
    p = q[rows].cpu().numpy()
    byte = s[:, rows].transpose(0, 1).reshape(len(p), -1)[:, :p.shape[1] // 16].cpu().numpy()
    return ref.decode(np.stack([p & 15, p >> 4], axis=2).reshape(len(p), -1), byte)


def sample(rng, n, most):
    """Sorted numbers below n: the first and last ones, both sides of each multiple of 128 (some of them) and others."""
    if n <= most:
        return torch.arange(n, device=DEV)
    edges = [i + d for i in rng.choice(range(0, n, 128), 6) for d in (-1, 0)]
    pick = np.unique(np.clip(np.concatenate([[0, 1, n - 2, n - 1], edges, rng.integers(0, n, most - 16)]), 0, n - 1))
    return torch.from_numpy(pick).to(DEV)


def uneven(rng, T, E):
    """T rows over E experts, one of them without."""
    w = rng.random(E) + 0.25
    counts = rng.multinomial(max(T - E, 0), w / w.sum()) + 1 if T > E else rng.multinomial(T, w / w.sum())
    if E > 3:
        counts[0], counts[1] = counts[0] + counts[1], 0
    return counts.tolist()


def offsets_of(counts, front=0):
    return torch.tensor(np.concatenate([[front], front + np.cumsum(counts)]), dtype=torch.int32, device=DEV)


def surrounded(t, front, behind):
    out = torch.full((front + t.shape[0] + behind, t.shape[1]), float("nan"), dtype=t.dtype, device=DEV)
    out[front:front + t.shape[0]] = t
    return out


def check_rows(rng, y, x_of, w_of, bias, counts, front, width):
    """y against x w^T + bias: x_of(rows) and w_of(expert, columns) give values."""
    at = front
    for e, n in enumerate(counts):
        if n:
            r, c = at + sample(rng, n, 48), sample(rng, width, 160 if len(counts) < 64 else 48)
            ref.check_product(y[r][:, c], x_of(r), w_of(e, c), None if bias is None else ref.values(bias[e][c]))
        at += n


# (form of grouped_plan, its groups of the contraction, its ring): (T, E, N, K)
FORWARD = {(0, 4, 4): [(28, 2, 106, 2496), (100, 4, 90, 3008)], (1, 2, 4): [(60, 5, 2805, 1216), (60, 5, 2805, 1280)], (2, 1, 3): [(333, 9, 2897, 512), (700, 4, 2300, 704)],
           (3, 1, 3): [(1764, 9, 2840, 1088)], (4, 4, 4): [(48, 8, 768, 3008), (20, 5, 1600, 2560)]}
MX_FORWARD = {(0, 4, 4): [(26, 2, 131, 10496), (28, 2, 104, 9280)], (1, 2, 4): [(78, 6, 2847, 5120), (60, 5, 2728, 4928)], (2, 1, 3): [(441, 7, 2771, 2048), (342, 9, 2893, 1920)],
              (4, 4, 2): [(3, 6, 300, 4640), (20, 5, 2458, 4640), (30, 33, 2051, 4064)]}
cases = lambda forms: [(f, *size) for f, sizes in forms.items() for size in sizes]


@pytest.mark.parametrize("form,T,E,N,K", cases(FORWARD))
def test_forward(form, T, E, N, K):
    f, groups, ring = form
    assert plan.forward_form(T + 8, E, N, K) == f and K // 64 // groups > 2 * ring
    gen, rng = generator(T + N + K), np.random.default_rng(T)
    counts = uneven(rng, T, E)
    X, W, b = surrounded(bf16(gen, T, K), 3, 5), bf16(gen, E, N, K), bf16(gen, E, N)
    Y = rtl.grouped_linear(X, offsets_of(counts, 3), W, bias=b)
    assert (Y[:3] == 0).all() and (Y[3 + T:] == 0).all()
    check_rows(rng, Y, lambda r: ref.values(X[r]), lambda e, c: ref.values(W[e][c]), b, counts, 3, N)


@pytest.mark.parametrize("form,T,E,N,K", cases(MX_FORWARD))
def test_mxfp4_forward(form, T, E, N, K):
    f, groups, ring = form
    assert plan.forward_form(T + 3, E, N, K, True) == f and (K + 255) // 256 // groups >= (ring if f == 4 else 2 * ring + 1)
    gen, rng = generator(T + N + K + 1), np.random.default_rng(T + 1)
    counts = uneven(rng, T, E)
    X, b = surrounded(bf16(gen, T, K), 1, 2), bf16(gen, E, N)
    wq, ws = codes(gen, E * N, K)
    Y = rtl.grouped_mxfp4_linear(X, offsets_of(counts, 1), wq.view(E, N, K // 2), ws, bias=b)
    check_rows(rng, Y, lambda r: ref.decode(*ref.quantize(ref.values(X[r]))), lambda e, c: decoded(wq, ws, e * N + c), b, counts, 1, N)


# rows of the experts, column tiles of 256; stages of the contraction
PANELS = [([197, 139, 337], 52, 9), ([0, 768, 5, 0, 900, 1], 40, 8), ([1024, 512], 45, 9), ([2000, 300, 700], 26, 10)]


@pytest.mark.parametrize("counts,tiles_n,stages", PANELS)
@pytest.mark.parametrize("short", [0, 1])
def test_panels(counts, tiles_n, stages, short):
    """Panels of 256 rows (ring of two) and 128 (ring of three), more tiles than workgroups; `short`: the last block is not full (4-bit, input gradient)."""
    tall = plan.heights(counts, tiles_n, stages)
    assert tall > 0 and stages > 2 * 3 and (sum(-(-n // 128) for n in counts) - tall) * tiles_n > 256
    T, E, N = sum(counts), len(counts), tiles_n * 256 - 40
    K, K4, D = stages * 64, stages * 256 - 96 * short, stages * 64 - 40 * short
    assert plan.forward_form(T, E, N, K) == 3 and plan.forward_form(T, E, N, K4, True) == 3 and plan.dgrad_form(T, E, D, N) == 2
    gen, rng = generator(stages), np.random.default_rng(stages)
    off, b = offsets_of(counts), bf16(gen, E, N)
    if not short:
        X, W = bf16(gen, T, K), bf16(gen, E, N, K)
        check_rows(rng, rtl.grouped_linear(X, off, W, bias=b), lambda r: ref.values(X[r]), lambda e, c: ref.values(W[e][c]), b, counts, 0, N)
        del X, W
    X4 = bf16(gen, T, K4)
    wq, ws = codes(gen, E * N, K4)
    Y4 = rtl.grouped_mxfp4_linear(X4, off, wq.view(E, N, K4 // 2), ws, bias=b)
    check_rows(rng, Y4, lambda r: ref.decode(*ref.quantize(ref.values(X4[r]))), lambda e, c: decoded(wq, ws, e * N + c), b, counts, 0, N)
    G, V = bf16(gen, T, D), bf16(gen, E, D, N)
    dX = rtl.grouped_linear_dgrad(G, off, V)
    check_rows(rng, dX, lambda r: ref.values(G[r]), lambda e, c: ref.values(V[e][:, c]).T, None, counts, 0, N)


# form: (T, E, N, K); all with a ring of four
DGRAD = {0: [(24, 2, 704, 80), (60, 3, 648, 200)], 1: [(640, 8, 640, 4064), (684, 9, 608, 3376)]}


@pytest.mark.parametrize("form,T,E,N,K", cases(DGRAD))
def test_input_gradient(form, T, E, N, K):
    assert plan.dgrad_form(T + 6, E, N, K) == form and N > 64 * 2 * 4
    gen, rng = generator(T + N + K + 2), np.random.default_rng(T + 2)
    counts = uneven(rng, T, E)
    dY, W = surrounded(bf16(gen, T, N), 2, 4), bf16(gen, E, N, K)
    dX = rtl.grouped_linear_dgrad(dY, offsets_of(counts, 2), W)
    check_rows(rng, dX, lambda r: ref.values(dY[r]), lambda e, c: ref.values(W[e][:, c]).T, None, counts, 2, K)


# (form, ring): (T, E, N, K), the rows uneven
WGRAD = {(0, 4): [(6000, 4, 1504, 1104), (4000, 4, 1304, 1096)], (1, 2): [(11087, 17, 144, 2856), (9000, 12, 400, 2080)], (2, 2): [(6185, 9, 3104, 136), (3000, 3, 1304, 1800)]}


@pytest.mark.parametrize("form,T,E,N,K", cases(WGRAD) + [(("parts", 4), 10374, 2, 840, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weight_and_bias_gradient(form, T, E, N, K, dtype):
    f, ring = form
    shape, parts = plan.wgrad_form(T + 160, E, N, K)
    gen, rng = generator(T + N + K + 3), np.random.default_rng(T + 3)
    counts = uneven(rng, T, E)
    assert (shape, parts) == (f, 1) if f != "parts" else parts > 1
    assert max(counts) > 64 * parts * (2 * ring + 1)
    dY, X = surrounded(bf16(gen, T, N), 70, 90), surrounded(bf16(gen, T, K), 70, 90)
    dW, db = rtl.grouped_linear_wgrad(dY, X, offsets_of(counts, 70), with_bias=True, dtype=dtype)
    at = 70
    for e, n in enumerate(counts):
        g, x = dY[at:at + n], X[at:at + n]
        c, k = sample(rng, N, 96), sample(rng, K, 160)
        if n:
            ref.check_product(dW[e][c][:, k], ref.values(g[:, c]).T, ref.values(x[:, k]).T, dtype=dtype)
            ref.check_product(db[e:e + 1], np.ones((1, n)), ref.values(g).T, dtype=dtype)
        else:
            assert (dW[e] == 0).all() and (db[e] == 0).all()
        at += n


# (form of mx_ref.choice or the body width of the 256-row plan, groups, ring): (M, N, K), each with a full last block and without
DENSE4 = {(0, 4, 4): [(18, 44, 10496), (18, 70, 9504)], (1, 4, 3): [(33, 4130, 9472), (35, 4130, 8000)], (2, 2, 4): [(66, 5039, 4864), (68, 4460, 4704)],
          (3, 2, 3): [(131, 5587, 3840), (129, 5626, 3936)], (4, 1, 3): [(389, 4371, 2304), (257, 5510, 2080)], (5, 1, 3): [(556, 6922, 2048), (4647, 811, 1856)],
          ("tails", 1, 3): [(2322, 2020, 2304), (2322, 2020, 2080)], ("192", 1, 2): [(2053, 3643, 2304), (2053, 3643, 2080)],
          ("192 and tails", 1, 3): [(4691, 3347, 2080), (4691, 3347, 2304)], ("256", 1, 2): [(4890, 2314, 2304), (4890, 2314, 2080), (4608, 3000, 3360)]}


@pytest.mark.parametrize("form,M,N,K", cases(DENSE4))
def test_mxfp4_product(form, M, N, K):
    f, groups, ring = form
    shape, splits, _ = ref.choice(M, N, K)
    assert splits == 1 and (K + 255) // 256 // groups > 2 * ring
    if isinstance(f, str):
        p = rtl.diag_tile_plan(M, N, True)
        assert shape == -1 and ("tails" in f) == (p["tail_tiles"] > 0) and (f == "tails") == (p["body_tiles"] == 0) and (p["body_width"] == int(f[:3]) if f != "tails" else True)
    else:
        assert shape == f
    gen, rng = generator(M + N + K), np.random.default_rng(M)
    xq, xs = codes(gen, M, K)
    wq, ws = codes(gen, N, K)
    b = bf16(gen, 1, N)
    y = rtl.mxfp4_packed_linear(xq, xs, wq, ws, bias=b[0])
    check_rows(rng, y, lambda r: decoded(xq, xs, r), lambda e, c: decoded(wq, ws, c), b, [M], 0, N)


@pytest.mark.parametrize("M,N", [(20, 70), (300, 70), (2552, 1558)])
@pytest.mark.parametrize("negative", [False, True])
def test_what_lds_held_does_not_reach_a_result(M, N, negative):
    """The chunks behind K of a last block that is not full are not loaded: whatever codes an earlier launch left there, sums of an instruction that lie
    right between two fp32 values round as they do alone. (1 + 3/2 of a step: to the even neighbour, 1 + 2 steps; 1 + 1/2 step: to 1; 0 stays +0.)"""
    big, K = 4096, 96
    a = torch.full((4608, big // 2), 0x77, dtype=torch.uint8, device=DEV)
    w = torch.full((4608, big // 2), 0xFF if negative else 0x77, dtype=torch.uint8, device=DEV)
    s = torch.full(rtl.mxfp4_scales_shape(4608, big), 100, dtype=torch.uint8, device=DEV)
    byte = np.full((M, 3), 127, np.uint8)
    byte[:, 2] = 127 - 24
    b = torch.full((N,), -1.0, dtype=torch.bfloat16, device=DEV)
    for x_code, w_code, want in ((3, 4, 2.0 ** -22), (2, 2, 0.0), (0, 0, -1.0)):
        x, v = np.zeros((M, K), np.uint8), np.zeros((N, K), np.uint8)
        x[:, 0], v[:, 0] = (2 if x_code else 0), 10 if not x_code else 2
        x[:, 64], v[:, 64] = x_code, w_code
        args = (*ref.on_device(x, byte), *ref.on_device(v, np.full((N, 3), 127, np.uint8)))
        rtl.mxfp4_packed_linear(a, s, w, s)
        y = rtl.mxfp4_packed_linear(*args, bias=b)
        assert (y.double() == want).all()
        if not x_code:
            rtl.mxfp4_packed_linear(a, s, w, s)
            assert (rtl.mxfp4_packed_linear(*args).view(torch.int16) == 0).all()


@pytest.mark.parametrize("E,T,tiles_n,stages", [(130, 9000, 8, 4), (200, 20000, 6, 9), (70, 12000, 9, 5), (300, 4000, 9, 5)])
def test_panels_of_more_experts_than_a_wave_has_lanes(E, T, tiles_n, stages):
    """Tall panels on both sides of the 64th expert, experts without rows between them, several rounds of tiles."""
    rng, N = np.random.default_rng(E), tiles_n * 256 - 40
    w = rng.random(E) ** 3
    w[::7] = 0
    counts = rng.multinomial(T, w / w.sum()).tolist()
    K, K4, D = stages * 64, stages * 256 - 96, stages * 64 - 24
    assert plan.forward_form(T + 3, E, N, K) == 3 and plan.forward_form(T + 3, E, N, K4, True) == 3
    assert E == 300 or 0 < sum(n // 256 for n in counts[:64]) < plan.heights(counts, tiles_n, stages)
    gen, off = generator(E), offsets_of(counts, 1)
    X, W, b = surrounded(bf16(gen, T, K), 1, 2), bf16(gen, E, N, K), bf16(gen, E, N)
    check_rows(rng, rtl.grouped_linear(X, off, W, bias=b), lambda r: ref.values(X[r]), lambda e, c: ref.values(W[e][c]), b, counts, 1, N)
    X4 = surrounded(bf16(gen, T, K4), 1, 2)
    wq, ws = codes(gen, E * N, K4)
    Y4 = rtl.grouped_mxfp4_linear(X4, off, wq.view(E, N, K4 // 2), ws, bias=b)
    check_rows(rng, Y4, lambda r: ref.decode(*ref.quantize(ref.values(X4[r]))), lambda e, c: decoded(wq, ws, e * N + c), b, counts, 1, N)
    G, V = surrounded(bf16(gen, T, D), 1, 2), bf16(gen, E, D, N)
    check_rows(rng, rtl.grouped_linear_dgrad(G, off, V), lambda r: ref.values(G[r]), lambda e, c: ref.values(V[e][:, c]).T, None, counts, 1, N)
    dW, db = rtl.grouped_linear_wgrad(G, X, off, with_bias=True)
    at = 1
    for e, n in enumerate(counts):
        g, x = G[at:at + n], X[at:at + n]
        if n and (e % 8 == 1 or e > E - 3):
            ref.check_product(dW[e], ref.values(g).T, ref.values(x).T)
            ref.check_product(db[e:e + 1], np.ones((1, n)), ref.values(g).T)
        elif n == 0:
            assert (dW[e] == 0).all() and (db[e] == 0).all()
        at += n
