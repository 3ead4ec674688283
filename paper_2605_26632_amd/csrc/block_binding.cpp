// Argument marshalling of the block operators (gated linears, norms of a block, rotary positions), compiled: their smallest calls keep the GPU busy for 3 to 10 us,
// and looking a dozen tensors over in Python, allocating the results and calling through ctypes took 6 to 20. Nothing is computed here; the functions of
// binding.py wrap these, which are called with all arguments in place and return their results in a tuple, or the number of an error.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>
#include <ATen/ops/empty.h>
#include "rtlynx.h"

namespace {

using at::Tensor;
constexpr auto kBf16 = at::kBFloat16;
constexpr auto kF32 = at::kFloat;

const char* name_of(at::ScalarType t) { return t == kBf16 ? "torch.bfloat16" : t == kF32 ? "torch.float32" : t == at::kInt ? "torch.int32" : "torch.uint8"; }

// A result: the caller's tensor, held while the call runs without the interpreter's lock, a new one, or none.
struct Result {
    THPObjectPtr given;
    Tensor fresh;
    const Tensor* t = nullptr;
};

PyObject *current_device = nullptr, *current_stream = nullptr;        // torch's functions: the number of the current device, and the stream of one

constexpr const char* kActs[] = {"silu", "gelu", "gelu_tanh"};          // rtl_act
constexpr const char* kNorms[] = {"none", "rms", "layer"};              // rtl_norm

struct Call {
    PyObject* const* args;
    Py_ssize_t next = 0;
    int64_t dev = -1;
    void* stream = nullptr;

    Call(PyObject* const* a, Py_ssize_t n, Py_ssize_t expected) : args(a) { TORCH_CHECK(n == expected, "block binding: ", expected, " arguments expected"); }
    // the current device and its stream; asked for by the first tensor of a device, since there is none to ask about before
    void place() {
        THPObjectPtr d(PyObject_CallNoArgs(current_device));
        if (!d) throw python_error();
        THPObjectPtr s(PyObject_CallOneArg(current_stream, d.get()));
        if (!s) throw python_error();
        dev = PyLong_AsLongLong(d.get());
        stream = reinterpret_cast<void*>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLong(s.get())));
        if (PyErr_Occurred()) throw python_error();
    }
    template <int N>
    int choice(const char* const (&names)[N], const char* what) {
        PyObject* o = args[next++];
        for (int i = 0; PyUnicode_Check(o) && i < N; ++i)
            if (PyUnicode_CompareWithASCIIString(o, names[i]) == 0) return i;
        std::string all;
        for (const char* n : names) all += (all.empty() ? "" : ", ") + std::string(n);
        TORCH_CHECK_VALUE(false, what, ": one of ", all);
    }
    rtl_act act() { return static_cast<rtl_act>(choice(kActs, "act")); }
    rtl_norm norm(const char* what) { return static_cast<rtl_norm>(choice(kNorms, what)); }
    int64_t integer() {
        const long long v = PyLong_AsLongLong(args[next++]);
        if (v == -1 && PyErr_Occurred()) throw python_error();
        return v;
    }
    float real() {
        const double v = PyFloat_AsDouble(args[next++]);
        if (v == -1.0 && PyErr_Occurred()) throw python_error();
        return static_cast<float>(v);
    }
    bool truth() {
        const int v = PyObject_IsTrue(args[next++]);
        if (v < 0) throw python_error();
        return v != 0;
    }
    // the next tensor, which has to lie on the current device; NULL for None
    const Tensor* tensor(PyObject* o) {
        if (o == Py_None) return nullptr;
        TORCH_CHECK_VALUE(THPVariable_Check(o), "tensor or None expected, not ", Py_TYPE(o)->tp_name);
        const Tensor& t = THPVariable_Unpack(o);
        TORCH_CHECK_VALUE(t.is_cuda(), "librtlynx takes tensors of the current device only, not of ", t.device());
        if (dev < 0) place();
        TORCH_CHECK_VALUE(t.get_device() == dev, "librtlynx takes tensors of the current device (", dev, ") only, not of ", t.device());
        return &t;
    }
    const Tensor* tensor() { return tensor(args[next++]); }
    // N results: those of a sequence, or none yet
    template <int N>
    bool results(Result (&r)[N]) {
        PyObject* o = args[next++];
        if (o == Py_None) return false;
        TORCH_CHECK_VALUE((PyTuple_Check(o) || PyList_Check(o)) && PySequence_Fast_GET_SIZE(o) == N, "out: ", N, " tensors or None expected");
        for (int i = 0; i < N; ++i) {
            PyObject* item = PySequence_Fast_GET_ITEM(o, i);
            r[i].t = tensor(item);
            if (!r[i].t) continue;
            Py_INCREF(item);
            r[i].given = item;
        }
        return true;
    }
    void make(Result& r, at::IntArrayRef shape, at::ScalarType type) const {
        r.fresh = at::empty(shape, at::TensorOptions().dtype(type).device(c10::Device(c10::DeviceType::CUDA, static_cast<c10::DeviceIndex>(dev))));
        r.t = &r.fresh;
    }
};

void* at_of(const Tensor* t) { return t ? t->data_ptr() : nullptr; }
float* floats_of(const Result& r) { return static_cast<float*>(at_of(r.t)); }

struct Matrix {
    int64_t rows, cols, ld;
};
// torch leaves any stride there for a single row
Matrix matrix(const Tensor& t, at::ScalarType type, const char* name) {
    TORCH_CHECK_VALUE(t.dim() == 2 && t.scalar_type() == type, name, ": ", name_of(type), " matrix expected");
    const int64_t rows = t.size(0), cols = t.size(1);
    TORCH_CHECK_VALUE(t.stride(1) == 1 || cols <= 1, name, ": contiguous rows expected");
    return Matrix{rows, cols, rows > 1 ? t.stride(0) : cols};
}
// Row stride of a matrix of this shape; 0 for none.
int64_t rows_of(const Tensor* t, int64_t rows, int64_t cols, at::ScalarType type, const char* name) {
    if (!t) return 0;
    const Matrix m = matrix(*t, type, name);
    TORCH_CHECK_VALUE(m.rows == rows && m.cols == cols, name, ": shape (", rows, ", ", cols, ") expected");
    return m.ld;
}
// A contiguous tensor of just this shape, or none.
void whole(const Tensor* t, at::IntArrayRef shape, at::ScalarType type, const char* name) {
    TORCH_CHECK_VALUE(!t || (t->sizes() == shape && t->scalar_type() == type && t->is_contiguous()), name, ": contiguous ", name_of(type), " tensor of shape ",
                      shape, " expected");
}
at::ScalarType residual_type(const Tensor& t, const char* name) {
    TORCH_CHECK_VALUE(t.scalar_type() == kBf16 || t.scalar_type() == kF32, name, ": bf16 or float32 expected");
    return t.scalar_type();
}
// Workspace: the caller's, whole, or a new one.
struct Workspace {
    Tensor fresh;
    void* at = nullptr;
    size_t bytes = 0;
    void take(const Call& c, const Tensor* given, size_t need) {
        if (!given && need) {
            fresh = at::empty({static_cast<int64_t>(need)}, at::TensorOptions().dtype(at::kByte).device(c10::Device(c10::DeviceType::CUDA, static_cast<c10::DeviceIndex>(c.dev))));
            given = &fresh;
        }
        if (!given) return;
        at = given->data_ptr();
        bytes = given->is_contiguous() ? given->nbytes() : 0;
    }
};

template <int N>
PyObject* answer(rtl_status status, Result (&r)[N]) {
    PyObject* out = status == RTL_OK ? PyTuple_New(N) : PyLong_FromLong(status);
    if (!out) throw python_error();
    if (status != RTL_OK) return out;
    for (int i = 0; i < N; ++i) {
        PyObject* o = r[i].given ? r[i].given.release() : r[i].t ? THPVariable_Wrap(std::move(r[i].fresh)) : Py_None;
        if (o == Py_None) Py_INCREF(o);
        PyTuple_SET_ITEM(out, i, o);
    }
    return out;
}
#define WITHOUT_GIL(call)    \
    rtl_status status;       \
    {                        \
        pybind11::gil_scoped_release without; \
        status = (call);     \
    }

// X, W, bias, act, with_pre, (H, P) or None
PyObject* gated_linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c(args, n, 6);
    const Tensor *X = c.tensor(), *W = c.tensor(), *bias = c.tensor();
    TORCH_CHECK_VALUE(X && W, "X and W expected");
    const rtl_act act = c.act();
    const bool with_pre = c.truth();
    Result r[2];
    c.results(r);
    const Matrix x = matrix(*X, kBf16, "X"), w = matrix(*W, kBf16, "W");
    TORCH_CHECK_VALUE(w.cols == x.cols && w.rows % 2 == 0, "W: shape (2F, ", x.cols, ") expected");
    whole(bias, {w.rows}, kBf16, "bias");
    if (!r[0].t) c.make(r[0], {x.rows, w.rows / 2}, kBf16);
    if (!r[1].t && with_pre) c.make(r[1], {x.rows, w.rows}, kBf16);
    const int64_t ldh = rows_of(r[0].t, x.rows, w.rows / 2, kBf16, "out"), ldp = rows_of(r[1].t, x.rows, w.rows, kBf16, "pre");
    WITHOUT_GIL(rtl_gated_linear(at_of(X), at_of(W), at_of(bias), at_of(r[0].t), at_of(r[1].t), act, x.rows, w.rows / 2, x.cols, x.ld, w.ld, ldh, ldp, c.stream))
    return answer(status, r);
    END_HANDLE_TH_ERRORS
}

// dH, X, W, P, act, with_bias, with_hidden, float32, (dX, dW, db, H) or None, workspace
PyObject* gated_linear_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c(args, n, 10);
    const Tensor *dH = c.tensor(), *X = c.tensor(), *W = c.tensor(), *P = c.tensor();
    TORCH_CHECK_VALUE(dH && P, "dH and P expected");
    const rtl_act act = c.act();
    const bool with_bias = c.truth(), with_hidden = c.truth();
    at::ScalarType type = c.truth() ? kF32 : kBf16;
    Result r[4];
    const bool given = c.results(r);
    const Tensor* ws = c.tensor();
    const Matrix h = matrix(*dH, kBf16, "dH");
    const int64_t M = h.rows, F = h.cols, ldp = rows_of(P, M, 2 * F, kBf16, "P");
    int64_t K = 0, ldx = 0, ldw = 0;
    if (X) {
        const Matrix x = matrix(*X, kBf16, "X");
        TORCH_CHECK_VALUE(x.rows == M, "dH and X differ in rows");
        K = x.cols;
        ldx = x.ld;
    }
    if (W) {
        const Matrix w = matrix(*W, kBf16, "W");
        TORCH_CHECK_VALUE(w.rows == 2 * F && (!X || w.cols == K), "W: shape (", 2 * F, ", K) expected, K as in X");
        K = w.cols;
        ldw = w.ld;
    }
    if (!given) {
        if (W) c.make(r[0], {M, K}, kBf16);
        if (X) c.make(r[1], {2 * F, K}, type);
        if (X && with_bias) c.make(r[2], {2 * F}, type);
        if (with_hidden) c.make(r[3], {M, F}, kBf16);
    }
    TORCH_CHECK_VALUE(W || !r[0].t, "dX needs W");
    TORCH_CHECK_VALUE(X || !r[1].t, "dW needs X");
    TORCH_CHECK_VALUE(r[1].t || !r[2].t, "db comes with dW");
    if (r[1].t) type = residual_type(*r[1].t, "dW");
    const int64_t lddx = rows_of(r[0].t, M, K, kBf16, "dX"), lddw = rows_of(r[1].t, 2 * F, K, type, "dW"), ldh = rows_of(r[3].t, M, F, kBf16, "H");
    whole(r[2].t, {2 * F}, type, "db");
    Workspace work;
    work.take(c, ws, ws ? 0 : std::max<size_t>(rtl_gated_linear_backward_workspace(M, F, K > 0 ? K : 1), 256));
    WITHOUT_GIL(rtl_gated_linear_backward(at_of(dH), at_of(X), at_of(W), at_of(P), at_of(r[0].t), at_of(r[1].t), at_of(r[2].t), at_of(r[3].t), act,
                                          type == kF32 ? RTL_F32 : RTL_BF16, M, F, K, h.ld, ldx, ldw, ldp, lddx, lddw, ldh, work.at, work.bytes, c.stream))
    return answer(status, r);
    END_HANDLE_TH_ERRORS
}

int64_t sequences(const Tensor* offsets) {
    if (!offsets) return 1;
    TORCH_CHECK_VALUE(offsets->numel() >= 1, "offsets: at least one number expected");
    whole(offsets, {offsets->numel()}, at::kInt, "offsets");
    return offsets->numel() - 1;
}

// x, y, gate, w_post, w_pre, scale, shift, offsets, post, pre, alpha, eps, with_x, with_h, (x', h) or None
PyObject* residual_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c(args, n, 15);
    const Tensor *x = c.tensor(), *y = c.tensor(), *gate = c.tensor(), *w_post = c.tensor(), *w_pre = c.tensor(), *scale = c.tensor(), *shift = c.tensor(),
                 *offsets = c.tensor();
    const rtl_norm post = c.norm("post"), pre = c.norm("pre");
    const float alpha = c.real(), eps = c.real();
    const bool with_x = c.truth(), with_h = c.truth();
    Result r[2];
    const bool given = c.results(r);
    TORCH_CHECK_VALUE(x, "x expected");
    const auto type = residual_type(*x, "x");
    const int64_t S = sequences(offsets);
    const Matrix m = matrix(*x, type, "x");
    const int64_t T = m.rows, D = m.cols, ldy = rows_of(y, T, D, kBf16, "y"), ld_gate = rows_of(gate, S, D, kBf16, "gate");
    const int64_t ld_scale = rows_of(scale, S, D, kBf16, "scale"), ld_shift = rows_of(shift, S, D, kBf16, "shift");
    TORCH_CHECK_VALUE(!scale || !shift || ld_scale == ld_shift, "scale and shift differ in their row stride");
    whole(w_post, {D}, kBf16, "w_post");
    whole(w_pre, {D}, kBf16, "w_pre");
    if (!given) {
        if (with_x) c.make(r[0], {T, D}, type);
        if (with_h) c.make(r[1], {T, D}, kBf16);
    }
    const int64_t ldxo = rows_of(r[0].t, T, D, type, "x'"), ldh = rows_of(r[1].t, T, D, kBf16, "h");
    WITHOUT_GIL(rtl_residual_norm(at_of(x), at_of(y), at_of(gate), at_of(w_post), at_of(w_pre), at_of(scale), at_of(shift),
                                  static_cast<const int32_t*>(at_of(offsets)), at_of(r[0].t), at_of(r[1].t), type == kF32 ? RTL_F32 : RTL_BF16, post, pre, alpha, eps,
                                  !given, T, S, D, m.ld, ldy, ld_gate, scale ? ld_scale : ld_shift, ldxo, ldh, c.stream))
    return answer(status, r);
    END_HANDLE_TH_ERRORS
}

// dx_out, dh, x_out, y, gate, w_post, w_pre, scale, offsets, post, pre, alpha, eps, with_shift (-1: with scale), seven results or None, workspace
PyObject* residual_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c(args, n, 16);
    const Tensor *dx_out = c.tensor(), *dh = c.tensor(), *x_out = c.tensor(), *y = c.tensor(), *gate = c.tensor(), *w_post = c.tensor(), *w_pre = c.tensor(),
                 *scale = c.tensor(), *offsets = c.tensor();
    const rtl_norm post = c.norm("post"), pre = c.norm("pre");
    const float alpha = c.real(), eps = c.real();
    const int64_t with_shift = c.integer();
    Result r[7];
    const bool given = c.results(r);
    const Tensor* ws = c.tensor();
    const Tensor* like = x_out ? x_out : dx_out;
    TORCH_CHECK_VALUE(like, "x' or its gradient expected");
    const auto type = residual_type(*like, "x'");
    const int64_t S = sequences(offsets);
    const Matrix m = matrix(*like, type, "x'");
    const int64_t T = m.rows, D = m.cols;
    const int64_t lddxo = rows_of(dx_out, T, D, type, "dx_out"), lddh = rows_of(dh, T, D, kBf16, "dh"), ldxo = rows_of(x_out, T, D, type, "x'"),
                  ldy = rows_of(y, T, D, kBf16, "y"), ld_gate = rows_of(gate, S, D, kBf16, "gate"), ld_mod = rows_of(scale, S, D, kBf16, "scale");
    whole(w_post, {D}, kBf16, "w_post");
    whole(w_pre, {D}, kBf16, "w_pre");
    if (!given) {
        c.make(r[0], {T, D}, type);
        if (y) c.make(r[1], {T, D}, kBf16);
        if (y && gate) c.make(r[2], {S, D}, kF32);
        if (scale) c.make(r[3], {S, D}, kF32);
        if (with_shift < 0 ? scale != nullptr : with_shift != 0) c.make(r[4], {S, D}, kF32);
        if (y && w_post) c.make(r[5], {D}, kF32);
        if (w_pre) c.make(r[6], {D}, kF32);
    } else {
        const char* names[] = {"dgate", "dscale", "dshift"};
        for (int i = 0; i < 3; ++i) whole(r[2 + i].t, {S, D}, kF32, names[i]);
        whole(r[5].t, {D}, kF32, "dw_post");
        whole(r[6].t, {D}, kF32, "dw_pre");
    }
    const int64_t lddx = rows_of(r[0].t, T, D, type, "dx"), lddy = rows_of(r[1].t, T, D, kBf16, "dy");
    const bool sums = r[2].t || r[3].t || r[4].t || r[5].t || r[6].t;
    Workspace work;
    work.take(c, ws, ws || !sums ? 0 : rtl_residual_norm_backward_workspace(T, S, D));
    WITHOUT_GIL(rtl_residual_norm_backward(at_of(dx_out), at_of(dh), at_of(x_out), at_of(y), at_of(gate), at_of(w_post), at_of(w_pre), at_of(scale),
                                           static_cast<const int32_t*>(at_of(offsets)), at_of(r[0].t), at_of(r[1].t), floats_of(r[2]), floats_of(r[3]),
                                           floats_of(r[4]), floats_of(r[5]), floats_of(r[6]), type == kF32 ? RTL_F32 : RTL_BF16, post, pre, alpha, eps, !given, T, S, D,
                                           lddxo, lddh, ldxo, ldy, ld_gate, ld_mod, lddx, lddy, work.at, work.bytes, c.stream))
    return answer(status, r);
    END_HANDLE_TH_ERRORS
}

struct Heads {
    int64_t count = 0, ld = 0, stride = 0;
};
Heads heads(const Tensor* t, int64_t T, int64_t D, const char* name, int64_t expected = -1) {
    if (!t) return Heads{};
    TORCH_CHECK_VALUE(t->dim() == 3 && t->scalar_type() == kBf16, name, ": bf16 tensor of shape [T, heads, D] expected");
    TORCH_CHECK_VALUE(t->size(0) == T && t->size(2) == D && (expected < 0 || t->size(1) == expected), name, ": shape (", T, ", heads, ", D, ") expected");
    TORCH_CHECK_VALUE(t->stride(2) == 1, name, ": contiguous heads expected");
    return Heads{t->size(1), t->stride(0), t->stride(1)};
}
struct Rotation {
    const float *pos = nullptr, *freq = nullptr;
    const int32_t* axis = nullptr;
    int64_t pairs = 0, axes = 1;
    Rotation(const Tensor* p, const Tensor* f, const Tensor* a, int64_t T) {
        if (!f) return;
        TORCH_CHECK_VALUE(p && a && p->dim() == 2, "pos of shape (T, axes) and axis expected with freq");
        pairs = f->numel();
        axes = p->size(1);
        whole(p, {T, axes}, kF32, "pos");
        whole(f, {pairs}, kF32, "freq");
        whole(a, {pairs}, at::kInt, "axis");
        pos = static_cast<const float*>(p->data_ptr());
        freq = static_cast<const float*>(f->data_ptr());
        axis = static_cast<const int32_t*>(a->data_ptr());
    }
};

// q, k, pos, freq, axis, wq, wk, norm, eps, interleaved, (q', k') or None
PyObject* norm_rotary(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c(args, n, 11);
    const Tensor *q = c.tensor(), *k = c.tensor(), *pos = c.tensor(), *freq = c.tensor(), *axis = c.tensor(), *wq = c.tensor(), *wk = c.tensor();
    const rtl_norm norm = c.norm("norm");
    const float eps = c.real();
    const bool interleaved = c.truth();
    Result r[2];
    const bool given = c.results(r);
    const Tensor* like = q ? q : k;
    TORCH_CHECK_VALUE(like && like->dim() == 3, "q or k of shape [T, heads, D] expected");
    const int64_t T = like->size(0), D = like->size(2);
    const Heads hq = heads(q, T, D, "q"), hk = heads(k, T, D, "k");
    const Rotation turn(pos, freq, axis, T);
    whole(wq, {D}, kBf16, "wq");
    whole(wk, {D}, kBf16, "wk");
    if (!given) {
        if (q) c.make(r[0], {T, hq.count, D}, kBf16);
        if (k) c.make(r[1], {T, hk.count, D}, kBf16);
    }
    TORCH_CHECK_VALUE(!q == !r[0].t && !k == !r[1].t, "out: tensors for what is passed expected");
    const Heads oq = heads(r[0].t, T, D, "q'", hq.count), ok = heads(r[1].t, T, D, "k'", hk.count);
    WITHOUT_GIL(rtl_norm_rotary(at_of(q), at_of(k), turn.pos, turn.freq, turn.axis, at_of(wq), at_of(wk), at_of(r[0].t), at_of(r[1].t), norm, eps, interleaved, T,
                                hq.count, hk.count, D, turn.pairs, turn.axes, hq.ld, hq.stride, hk.ld, hk.stride, oq.ld, oq.stride, ok.ld, ok.stride, c.stream))
    return answer(status, r);
    END_HANDLE_TH_ERRORS
}

// dq_out, dk_out, q, k, pos, freq, axis, wq, wk, norm, eps, interleaved, (dq, dk, dwq, dwk) or None, workspace
PyObject* norm_rotary_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Call c(args, n, 14);
    const Tensor *dq_out = c.tensor(), *dk_out = c.tensor(), *q = c.tensor(), *k = c.tensor(), *pos = c.tensor(), *freq = c.tensor(), *axis = c.tensor(),
                 *wq = c.tensor(), *wk = c.tensor();
    const rtl_norm norm = c.norm("norm");
    const float eps = c.real();
    const bool interleaved = c.truth();
    Result r[4];
    const bool given = c.results(r);
    const Tensor* ws = c.tensor();
    const Tensor* like = dq_out ? dq_out : dk_out;
    TORCH_CHECK_VALUE(like && like->dim() == 3, "a gradient of shape [T, heads, D] expected");
    const int64_t T = like->size(0), D = like->size(2);
    const Heads gq = heads(dq_out, T, D, "dq_out"), gk = heads(dk_out, T, D, "dk_out");
    const Heads hq = heads(q, T, D, "q", gq.count), hk = heads(k, T, D, "k", gk.count);
    const Rotation turn(pos, freq, axis, T);
    whole(wq, {D}, kBf16, "wq");
    whole(wk, {D}, kBf16, "wk");
    if (!given) {
        if (dq_out) c.make(r[0], {T, gq.count, D}, kBf16);
        if (dk_out) c.make(r[1], {T, gk.count, D}, kBf16);
        if (wq) c.make(r[2], {D}, kF32);
        if (wk) c.make(r[3], {D}, kF32);
    }
    whole(r[2].t, {D}, kF32, "dwq");
    whole(r[3].t, {D}, kF32, "dwk");
    const Heads oq = heads(r[0].t, T, D, "dq", gq.count), ok = heads(r[1].t, T, D, "dk", gk.count);
    Workspace work;
    work.take(c, ws, ws || !(r[2].t || r[3].t) ? 0 : rtl_norm_rotary_backward_workspace(D));
    WITHOUT_GIL(rtl_norm_rotary_backward(at_of(dq_out), at_of(dk_out), at_of(q), at_of(k), turn.pos, turn.freq, turn.axis, at_of(wq), at_of(wk), at_of(r[0].t),
                                         at_of(r[1].t), floats_of(r[2]), floats_of(r[3]), norm, eps, interleaved, T, gq.count, gk.count, D, turn.pairs, turn.axes,
                                         gq.ld, gq.stride, gk.ld, gk.stride, hq.ld, hq.stride, hk.ld, hk.stride, oq.ld, oq.stride, ok.ld, ok.stride, work.at,
                                         work.bytes, c.stream))
    return answer(status, r);
    END_HANDLE_TH_ERRORS
}

#define METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(gated_linear),          METHOD(gated_linear_backward), METHOD(residual_norm), METHOD(residual_norm_backward),
                         METHOD(norm_rotary), METHOD(norm_rotary_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_block", "Argument marshalling of the block operators.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__block() {
    PyObject* torch = PyImport_ImportModule("torch._C");
    if (!torch) return nullptr;
    current_device = PyObject_GetAttrString(torch, "_cuda_getDevice");
    current_stream = current_device ? PyObject_GetAttrString(torch, "_cuda_getCurrentRawStream") : nullptr;
    Py_DECREF(torch);
    return current_stream ? PyModule_Create(&module) : nullptr;
}
