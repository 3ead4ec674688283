"""Which form a grouped launch takes: the library's host functions (internal, not part of its ABI), and the heights that its kernels choose
on the device (groups.h), computed again."""
import ctypes as C
import math

from paper_2605_26632_amd import binding as rtl


def _call(name, *args):
    f = getattr(rtl.lib(), name)
    f.argtypes = [C.c_int64] * 4 + ([C.c_bool] if len(args) == 5 else [])
    f.restype = C.c_int
    return f(*args)


def forward_form(T, E, N, K, fp4=False):
    return _call("_ZN3rtl12grouped_formEllllb", T, E, N, K, fp4)


def dgrad_form(T, E, N, K):
    return _call("_ZN3rtl11dgrad_shapeEllll", T, E, N, K)


def wgrad_form(T, E, N, K, room=64 << 20):
    f = rtl.lib()._ZN3rtl12wgrad_choiceEllllmPi
    f.argtypes = [C.c_int64] * 4 + [C.c_size_t, C.POINTER(C.c_int)]
    f.restype = None
    out = (C.c_int * 2)()
    f(T, E, N, K, room, out)
    return tuple(out)


def _time(tall, half, c):
    x, least = tall % 256, max((half * c + tall % 256) / 256, 1.0 if tall % 256 else 0.0)
    held = lambda t: (256 - x) * int(t / c + 0.01) + x * int(max(t - 1, 0) / c + 0.01)
    ends = [max((math.ceil(least / c - 0.01) + k) * c, least) for k in range(3)]
    if x:
        ends += [1 + (math.ceil(max(least - 1, 0) / c - 0.01) + k) * c for k in range(3)]
    return tall // 256 + min(t for t in ends if held(t) >= half)


def heights(counts, tiles_n, stages):
    """How many panels of 256 rows experts of these row counts get; the rest of the rows is cut into panels of 128."""
    full, rest = sum(n // 256 for n in counts), sum(-(-(n % 256) // 128) for n in counts)
    cost = 8 + 1.5 * stages
    best = None
    for lane in range(64):
        p = max(full - lane * max(1, 16 // tiles_n), 0)
        us = int(_time(p * tiles_n, ((full - p) * 2 + rest) * tiles_n, (8 + 0.78 * stages) / cost) * cost * 16)
        if best is None or us < best[0]:
            best = (us, p)
    return best[1]
