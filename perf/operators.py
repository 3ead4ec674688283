"""Linears on microscaled 4-bit floating point and linears grouped by expert: the work whose speed is measured, and its plain form.

`op` of a case names the work:
  "quant"     quantize_mxfp4 and dequantize_mxfp4: blocks of 32 values along a row ("cols"), down a column ("rows") or both in one
              pass; the outputs are the values that the codes stand for
  "mx"        mxfp4_linear: Y = q(X) Wq^T + b with X quantised in the call, or ("packed") mxfp4_packed_linear on codes
  "grouped"   grouped_linear: Y[rows of expert e] = X[rows of expert e] W[e]^T + b[e]
  "backward"  its gradients: grouped_linear_dgrad and grouped_linear_wgrad
  "grouped_mx" grouped_mxfp4_linear: grouped_linear with 4-bit weights, X quantised in the call

Blocks of 32 share a power of two 2^(floor(log2(max|x|)) - 2), kept as a biased exponent byte; a value is rounded to the nearest of
0, .5, 1, 1.5, 2, 3, 4, 6 times it, ties to the even code, at most 6. Two codes share a byte, the lower index in the low half. The byte of
block b of row r lies at [b // 8, r, b % 8]. `own` false computes all of it from elementary torch operations.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quant(name, rows, cols, along):
    return dict(name=name, op="quant", rows=rows, cols=cols, along=along)


def _mx(name, M, N, K, bias=False, packed=False):
    return dict(name=name, op="mx", M=M, N=N, K=K, bias=bias, packed=packed)


def _grouped(name, op, T, E, N, K, bias=False, skew=0.5, spare=0, wide=False, sizes=1):
    return dict(name=name, op=op, T=T, E=E, N=N, K=K, bias=bias, skew=skew, spare=spare, wide=wide, sizes=sizes)


def listed():
    return [
        # the input of an MLP-down layer at 1024 x 1024 pixels and text
        _quant("quant_mlp_down_input", 4608, 12288, "cols"),
        # the gradient of a small layer's output in a 4-bit training step, which is contracted along both of its axes; ragged rows
        _quant("quant_gradient_both", 2111, 2048, "both"),
        # one conditioning vector through a 4-bit layer: latency and the weight's bytes
        _mx("mx_one_token", 1, 12288, 3072, bias=True),
        # a text prompt, odd row count, a width that is no multiple of a tile and a last block group that is not full
        _mx("mx_prompt_odd", 333, 2739, 4000, bias=True),
        # MLP-down layer at full token count: the largest product
        _mx("mx_mlp_down", 4608, 3072, 12288),
        # weight gradient of a 4-bit training step: both operands are there as codes
        _mx("mx_packed_weight_gradient", 2048, 2048, 8192, packed=True),
        # a decoding step: few tokens, most of the experts' weights are read for one or two rows
        _grouped("grouped_decode", "grouped", 24, 32, 1408, 1024, bias=True, skew=1.0),
        # ordinary training or prefill batch, uneven experts, room for more rows behind the last one
        _grouped("grouped_prefill", "grouped", 8192, 8, 4096, 2048, spare=77),
        # gradients of a small layer, float32 weight gradients, some experts without a row
        _grouped("grouped_backward_small", "backward", 701, 16, 704, 512, bias=True, skew=2.0, wide=True),
        # gradients of the batch above
        _grouped("grouped_backward", "backward", 8192, 8, 4096, 2048, bias=True),
        # decoding with 4-bit experts
        _grouped("grouped_mx_decode", "grouped_mx", 24, 32, 2816, 2048, skew=1.0),
        # prefill with 4-bit experts
        _grouped("grouped_mx_prefill", "grouped_mx", 8192, 8, 4096, 2048, bias=True, spare=77),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    cap_flops = max(work(c)["flops"] for c in listed())
    cap_bytes = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["quant", "mx", "mx", "grouped", "grouped", "backward", "backward", "grouped_mx", "grouped_mx"])
        if op == "quant":
            case = _quant("", _log_uniform(rng, 1, 16896), _log_uniform(rng, 1, 480) * 32, rng.choice(["cols", "rows", "both"]))
        elif op == "mx":
            case = _mx("", _log_uniform(rng, 1, 16896), _log_uniform(rng, 128, 15360), _log_uniform(rng, 4, 480) * 32,
                       bias=rng.random() < 0.5, packed=rng.random() < 0.3)
        else:
            granule = 8 if op == "backward" else 1
            case = _grouped("", op, _log_uniform(rng, 1, 16896), _log_uniform(rng, 1, 128),
                            _log_uniform(rng, 64, 8192) // granule * granule, _log_uniform(rng, 1, 128) * 64,
                            bias=rng.random() < 0.5, skew=rng.uniform(0.0, 2.0), spare=rng.choice([0, 0, rng.randrange(1, 200)]),
                            wide=op == "backward" and rng.random() < 0.5, sizes=rng.randrange(1 << 30))
        del case["name"]
        w = work(case)
        if w["flops"] <= cap_flops and w["bytes"] <= cap_bytes:
            return case


def _offsets(case):
    """First rows of the experts and the end of the last one; behind it lie `spare` rows that belong to nobody."""
    rng = random.Random(case["sizes"])
    weight = [math.exp(case["skew"] * rng.gauss(0.0, 1.0)) for _ in range(case["E"])]
    counts = [0] * case["E"]
    for e in rng.choices(range(case["E"]), weights=weight, k=case["T"]):
        counts[e] += 1
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _blocks8(cols):
    return (cols + 255) // 256


def work(case):
    if case["op"] == "quant":
        rows, cols, n = case["rows"], case["cols"], 0
        if case["along"] != "rows":
            n += rows * cols
        if case["along"] != "cols":
            n += cols * ((rows + 31) // 32 * 32)
        return dict(bytes=2 * rows * cols + 2 * n, flops=3 * n)
    N, K = case["N"], case["K"]
    if case["op"] == "mx":
        M = case["M"]
        x = M * K // 2 + M * K // 32 if case["packed"] else 2 * M * K
        return dict(bytes=x + N * K // 2 + N * K // 32 + 2 * M * N + (2 * N if case["bias"] else 0), flops=2 * M * N * K)
    T, E, off = case["T"], case["E"], _offsets(case)
    hit = sum(off[e + 1] > off[e] for e in range(E))
    flops = 2 * T * N * K
    if case["op"] == "backward":
        grad = 4 if case["wide"] else 2
        return dict(bytes=2 * (T * N + T * K) + 2 * hit * N * K + 2 * T * K + grad * E * N * (K + (1 if case["bias"] else 0)),
                    flops=2 * flops + (T * N if case["bias"] else 0))
    weight = 2 * N * K if case["op"] == "grouped" else N * K // 2 + N * K // 32
    return dict(bytes=2 * T * K + hit * weight + 2 * T * N + (2 * hit * N if case["bias"] else 0), flops=flops)


# ---- inputs ---------------------------------------------------------------------------------------

def _normal(gen, *shape, std=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * std).to(torch.bfloat16)


def _activation(gen, rows, cols):
    """Heavy tails along a row and a few channels much larger than the rest, as the inputs of linears have them."""
    x = torch.randn(rows, cols, generator=gen, device=DEV)
    x *= torch.randn(rows, cols, generator=gen, device=DEV).abs()
    x *= 1.0 + 9.0 * (torch.rand(cols, generator=gen, device=DEV) < 0.01)
    return x.to(torch.bfloat16)


def _codes(x):
    """The 4-bit form of the rows of x: (codes [rows, cols / 2], scale bytes [cols / 256 rounded up, rows, 8])."""
    rows, cols = x.shape
    v, e = _rounded(x)
    mag = torch.bucketize(v.abs(), torch.tensor(GRID, device=x.device))
    code = (mag + 8 * (v < 0)).to(torch.uint8).reshape(rows, cols // 2, 2)
    s = torch.zeros(rows, _blocks8(cols) * 8, dtype=torch.uint8, device=x.device)
    s[:, :cols // 32] = (e + 127).to(torch.uint8)
    return code[..., 0] + 16 * code[..., 1], s.reshape(rows, -1, 8).transpose(0, 1).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000003 * seed + 17)
    if own:
        from paper_2605_26632_amd import binding as rtl
    st = dict(case=case)
    if case["op"] == "quant":
        st["x"] = _activation(gen, case["rows"], case["cols"])
        return st
    N, K = case["N"], case["K"]
    if case["op"] == "mx":
        M = case["M"]
        x = _activation(gen, M, K)
        st["wq"], st["ws"] = _codes(_normal(gen, N, K, std=K ** -0.5))
        st["b"] = _normal(gen, N) if case["bias"] else None
        if case["packed"]:
            st["xq"], st["xs"] = _codes(x)
        else:
            st["x"] = x
        if own:
            st["y"] = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
            size = rtl.mxfp4_packed_linear_workspace if case["packed"] else rtl.mxfp4_linear_workspace
            st["room"] = torch.empty(max(size(M, N, K), 256), dtype=torch.uint8, device=DEV)
        return st
    T, E, rows = case["T"], case["E"], case["T"] + case["spare"]
    st["off"] = _offsets(case)
    st["offsets"] = torch.tensor(st["off"], dtype=torch.int32, device=DEV)
    st["x"] = _activation(gen, rows, K)
    if case["op"] == "grouped_mx":
        wq, st["ws"] = _codes(_normal(gen, E * N, K, std=K ** -0.5))
        st["wq"] = wq.reshape(E, N, K // 2)
    else:
        st["w"] = _normal(gen, E, N, K, std=K ** -0.5)
    if case["op"] == "backward":
        st["dy"] = _normal(gen, rows, N)
    else:
        st["b"] = _normal(gen, E, N) if case["bias"] else None
    if own:
        # rows behind the last expert's are never written: they stay as the program has them, zeros here
        st["y"] = torch.zeros(rows, K if case["op"] == "backward" else N, dtype=torch.bfloat16, device=DEV)
        if case["op"] == "grouped_mx":
            st["room"] = torch.empty(max(rtl.grouped_mxfp4_linear_workspace(rows, E, N, K), 256), dtype=torch.uint8, device=DEV)
        if case["op"] == "backward":
            dtype = torch.float32 if case["wide"] else torch.bfloat16
            st["dw"] = torch.empty(E, N, K, dtype=dtype, device=DEV)
            st["db"] = torch.empty(E, N, dtype=dtype, device=DEV) if case["bias"] else None
            st["room"] = torch.empty(max(rtl.grouped_linear_wgrad_workspace(rows, E, N, K), 256), dtype=torch.uint8, device=DEV)
    return st


# ---- the plain form ---------------------------------------------------------------------------------

def _rounded(x):
    """Rows of x to the nearest 4-bit values: (values in units of their block's scale, exponents of the scales)."""
    rows, cols = x.shape
    b = x.float().reshape(rows, cols // 32, 32)
    top = b.abs().amax(dim=2)
    e = torch.where(top > 0, torch.floor(torch.log2(top.double())).float() - 2, -127.0).clamp(min=-127)
    v = torch.ldexp(b, -e[..., None])
    step = torch.where(v.abs() >= 4, 2.0, torch.where(v.abs() >= 2, 1.0, 0.5))
    v = (torch.round(v / step) * step).clamp(-6, 6)
    return v.reshape(rows, cols), e


def _quantised(x):
    v, e = _rounded(x)
    return torch.ldexp(v.reshape(*e.shape, 32), e[..., None]).reshape(x.shape)


def _decoded(q, s):
    """The values of codes and scale bytes."""
    rows, cols = q.shape[0], q.shape[1] * 2
    code = torch.stack([q & 15, q >> 4], dim=2).reshape(rows, cols).long()
    v = torch.tensor(GRID + tuple(-g for g in GRID), device=q.device)[code]
    e = s.transpose(0, 1).reshape(rows, -1)[:, :cols // 32].float() - 127
    return torch.ldexp(v.reshape(rows, cols // 32, 32), e[..., None]).reshape(rows, cols)


def _padded_t(x):
    """x transposed, its rows filled up to whole blocks of 32 with zeros."""
    return torch.nn.functional.pad(x, (0, 0, 0, -x.shape[0] % 32)).t()


def _plain(st):
    case = st["case"]
    op = case["op"]
    bf = torch.bfloat16
    if op == "quant":
        out = []
        if case["along"] != "rows":
            out.append(_quantised(st["x"]).to(bf))
        if case["along"] != "cols":
            out.append(_quantised(_padded_t(st["x"]).contiguous()).to(bf))
        return out
    if op == "mx":
        x = _decoded(st["xq"], st["xs"]) if case["packed"] else _quantised(st["x"])
        y = x @ _decoded(st["wq"], st["ws"]).t()
        return (y + st["b"].float() if case["bias"] else y).to(bf)
    E, N, off = case["E"], case["N"], st["off"]
    if op == "backward":
        wide = torch.float32 if case["wide"] else bf
        dx = torch.zeros(st["x"].shape, dtype=bf, device=DEV)
        dw = torch.empty(st["w"].shape, dtype=wide, device=DEV)
        db = torch.empty(E, N, dtype=wide, device=DEV)
        for e in range(E):
            dy, x = st["dy"][off[e]:off[e + 1]].float(), st["x"][off[e]:off[e + 1]].float()
            dx[off[e]:off[e + 1]] = (dy @ st["w"][e].float()).to(bf)
            dw[e] = (dy.t() @ x).to(wide)
            db[e] = dy.sum(dim=0).to(wide)
        return [dx, dw, db] if case["bias"] else [dx, dw]
    x = _quantised(st["x"]) if op == "grouped_mx" else st["x"].float()
    y = torch.zeros(x.shape[0], N, dtype=bf, device=DEV)
    for e in range(E):
        if off[e + 1] > off[e]:
            if op == "grouped_mx":
                w = _decoded(st["wq"][e], st["ws"][:, e * N:(e + 1) * N])
            else:
                w = st["w"][e].float()
            r = x[off[e]:off[e + 1]] @ w.t()
            y[off[e]:off[e + 1]] = (r + st["b"][e].float() if case["bias"] else r).to(bf)
    return y


def run(st):
    if not own:
        return _plain(st)
    from paper_2605_26632_amd import binding as rtl
    case = st["case"]
    op = case["op"]
    if op == "quant":
        codes = rtl.quantize_mxfp4(st["x"], along=case["along"])
        return [rtl.dequantize_mxfp4(codes[i], codes[i + 1]) for i in range(0, len(codes), 2)]
    if op == "mx":
        if case["packed"]:
            return rtl.mxfp4_packed_linear(st["xq"], st["xs"], st["wq"], st["ws"], bias=st["b"], out=st["y"], ws=st["room"])
        return rtl.mxfp4_linear(st["x"], st["wq"], st["ws"], bias=st["b"], out=st["y"], ws=st["room"])
    if op == "grouped":
        return rtl.grouped_linear(st["x"], st["offsets"], st["w"], bias=st["b"], out=st["y"])
    if op == "grouped_mx":
        return rtl.grouped_mxfp4_linear(st["x"], st["offsets"], st["wq"], st["ws"], bias=st["b"], out=st["y"], ws=st["room"])
    dx = rtl.grouped_linear_dgrad(st["dy"], st["offsets"], st["w"], out=st["y"])
    dw, db = rtl.grouped_linear_wgrad(st["dy"], st["x"], st["offsets"], out=(st["dw"], st["db"]), ws=st["room"])
    return [dx, dw, db] if case["bias"] else [dx, dw]


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _exact_values(x):
    """4-bit values of the rows of x, from the distances to the two neighbours on the grid."""
    x = x.double()
    rows, cols = x.shape
    b = x.reshape(rows, cols // 32, 32)
    _, ex = torch.frexp(b.abs().amax(dim=2))
    unit = torch.pow(2.0, (ex - 3).clamp(min=-127).double())[..., None]      # frexp's mantissa lies in [.5, 1)
    mag = (b.abs() / unit).clamp(max=6.0)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    hi = torch.bucketize(mag, grid).clamp(1, 7)
    low, high = mag - grid[hi - 1], grid[hi] - mag
    up = (high < low) | ((high == low) & (hi % 2 == 0))
    mag = torch.where(up, grid[hi], grid[hi - 1])
    return (torch.sign(b) * mag * unit).reshape(rows, cols)


def _exact_decode(q, s):
    rows, half = q.shape
    sign_mag = np.array([g * sgn for sgn in (1, -1) for g in GRID])
    qn, sn = q.cpu().numpy(), s.cpu().numpy()
    v = np.empty((rows, 2 * half))
    v[:, 0::2] = sign_mag[qn % 16]
    v[:, 1::2] = sign_mag[qn // 16]
    e = np.concatenate(list(sn), axis=1)[:, :half // 16].astype(np.float64) - 127.0
    return torch.from_numpy(v * np.repeat(np.exp2(e), 32, axis=1)).to(q.device)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "quant":
        out, x = [], st["x"]
        if case["along"] in ("cols", "both"):
            out.append(_exact_values(x))
        if case["along"] in ("rows", "both"):
            full = torch.zeros((x.shape[0] + 31) // 32 * 32, x.shape[1], dtype=torch.float64, device=DEV)
            full[:x.shape[0]] = x
            out.append(_exact_values(full.t().contiguous()))
        return out
    if op == "mx":
        x = _exact_decode(st["xq"], st["xs"]) if case["packed"] else _exact_values(st["x"])
        y = torch.matmul(x, _exact_decode(st["wq"], st["ws"]).t().contiguous())
        return y if st["b"] is None else y + st["b"].double()
    E, N, K = case["E"], case["N"], case["K"]
    off = np.array(st["off"])
    if op == "backward":
        dx = torch.zeros(st["x"].shape, dtype=torch.float64, device=DEV)
        dw = torch.zeros(E, N, K, dtype=torch.float64, device=DEV)
        db = torch.zeros(E, N, dtype=torch.float64, device=DEV)
        for e in np.nonzero(np.diff(off))[0].tolist():
            rows = slice(int(off[e]), int(off[e + 1]))
            dy = st["dy"][rows].double()
            dx[rows] = torch.matmul(dy, st["w"][e].double())
            dw[e] = torch.matmul(dy.t().contiguous(), st["x"][rows].double())
            db[e] = torch.matmul(torch.ones(1, dy.shape[0], dtype=torch.float64, device=DEV), dy)[0]
        return [dx, dw, db] if case["bias"] else [dx, dw]
    y = torch.zeros(st["x"].shape[0], N, dtype=torch.float64, device=DEV)
    for e in np.nonzero(np.diff(off))[0].tolist():
        rows = slice(int(off[e]), int(off[e + 1]))
        if op == "grouped_mx":
            x, w = _exact_values(st["x"][rows]), _exact_decode(st["wq"][e], st["ws"][:, e * N:(e + 1) * N])
        else:
            x, w = st["x"][rows].double(), st["w"][e].double()
        y[rows] = torch.matmul(x, w.t().contiguous())
        if case["bias"]:
            y[rows] += st["b"][e].double()
    return y
