"""Which form a launch takes: the library's host functions (internal, not part of its ABI)."""
import ctypes as C

from paper_2605_26632_amd import binding as rtl


class _Form(C.Structure):
    _fields_ = [("shape", C.c_int), ("use_192", C.c_bool), ("m_split", C.c_int64), ("body_tiles", C.c_int), ("tail_tiles", C.c_int)]


def gated_form(M, F, K):
    """A small tile by its index, or "256" / "192" for the 256-row plan with that body, "tails" added where there are tails, or tails alone."""
    f = rtl.lib()._ZN3rtl10gated_formElll
    f.argtypes, f.restype = [C.c_int64] * 3, _Form
    r = f(M, F, K)
    if M <= 16:
        return "few"
    if r.shape >= 0:
        return r.shape
    return " ".join(([] if not r.body_tiles else ["192" if r.use_192 else "256"]) + (["tails"] if r.tail_tiles else []))


def pair_form(M, F, K, dx=True, dw=True, room=64 << 20):
    """(form, parts of dX's contraction, parts of dW's) of gated_linear_backward's products."""
    f = rtl.lib()._ZN3rtl11pair_choiceElllbbmPi
    f.argtypes, f.restype = [C.c_int64] * 3 + [C.c_bool] * 2 + [C.c_size_t, C.POINTER(C.c_int)], None
    out = (C.c_int * 3)()
    f(M, 2 * F, K, dx, dw, room, out)
    return tuple(out)
