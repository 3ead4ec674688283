"""Plain 64-bit forms of the microscaled 4-bit operators, from their definition."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def values(x):
    """bf16 tensor -> float64 array."""
    return x.detach().cpu().to(torch.float64).numpy()


def quantize(x):
    """float64 [rows, cols] -> (codes [rows, cols] 0 .. 15, scale bytes [rows, cols / 32])."""
    rows, cols = x.shape
    b = x.reshape(rows, cols // 32, 32)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(axis=2, initial=0.0)
    with np.errstate(divide="ignore"):
        e = np.where(top > 0, np.frexp(top)[1] - 3, -127).clip(min=-127)
    mag = np.abs(b) / np.exp2(e.astype(np.float64))[..., None]
    code = np.zeros(b.shape, dtype=np.int64)
    for c in range(1, 8):
        mid = (GRID[c - 1] + GRID[c]) / 2
        code = np.where((mag > mid) | ((mag == mid) & (c % 2 == 0)), c, code)
    code += 8 * np.signbit(b)
    code[bad] = 0
    return code.reshape(rows, cols).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def pack(code):
    return code[:, 0::2] | (code[:, 1::2] << 4)


def scale_array(byte):
    """[rows, blocks] -> the layout of the library, zeros behind the last block."""
    rows, blocks = byte.shape
    out = np.zeros((rows, (blocks + 7) // 8 * 8), dtype=np.uint8)
    out[:, :blocks] = byte
    return np.ascontiguousarray(out.reshape(rows, -1, 8).transpose(1, 0, 2))


def padded_t(x):
    return np.pad(x, ((0, -x.shape[0] % 32), (0, 0))).T


def decode(code, byte):
    """Values of codes [rows, cols] and scale bytes [rows, cols / 32]."""
    v = np.where(code & 8, -1.0, 1.0) * GRID[code & 7]
    s = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=1)


def random_codes(rng, rows, cols, spread=6):
    """Codes and scale bytes around 1 / sqrt(cols)."""
    code = rng.integers(0, 16, (rows, cols), dtype=np.uint8)
    mid = 127 - int(np.log2(max(cols, 1)) / 2)
    byte = rng.integers(mid - spread, mid + spread + 1, (rows, cols // 32)).astype(np.uint8)
    return code, byte


def on_device(code, byte, dev="cuda:0"):
    return torch.from_numpy(pack(code)).to(dev), torch.from_numpy(scale_array(byte)).to(dev)


def check_product(y, x, w, bias=None, dtype=torch.bfloat16):
    """y against x w^T + bias in float64. The products are exact. An fp32 sum of k terms in any grouping is off by less than k 2^-24
    of the sum of magnitudes; the matrix instruction rounds once for 128 terms, so that is a wide bound. Storing y costs half a step."""
    ref = x @ w.T
    mag = np.abs(x) @ np.abs(w).T
    if bias is not None:
        ref = ref + bias
        mag = mag + np.abs(bias)
    half = torch.finfo(dtype).eps / 2
    tol = (x.shape[1] + 2) * 2.0 ** -24 * mag * (1 + half) + half * np.abs(ref) + 1e-38
    err = np.abs(values(y) - ref)
    assert y.shape == ref.shape and np.isfinite(values(y)).all()
    worst = np.unravel_index((err - tol).argmax(), err.shape) if err.size else None
    assert (err <= tol).all(), (worst, values(y)[worst], ref[worst], tol[worst])


def choice(M, N, K, room=64 << 20):
    """(index of the small tile shape or -1, parts of the contraction, rows of the part tile) of a 4-bit product: an internal host
    function of the library, not part of its ABI."""
    import ctypes as C
    from paper_2605_26632_amd import binding as rtl
    f = rtl.lib()._ZN3rtl9mx_choiceElllmPi
    f.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_size_t, C.POINTER(C.c_int)]
    f.restype = None
    out = (C.c_int * 3)()
    f(M, N, K, room, out)
    return tuple(out)
