// calls.cpp -- the Python calls of the losses over the vocabulary, of the embedding,
// of the norm, of 8-bit operands and of the decode under penalties (the Python extension
// _loss_calls.so): checks torch tensors, makes the outputs that are not given, and calls
// the C ABI.  Of a small call's time the
// host's is the larger part, and most of that is Python's: a distill_loss took
// 13.4 us to issue from Python (6.7 of them two allocations), of which the
// library's call is 3.4.
//
// Every function returns its outputs, or the library's status where that is not
// 0; what a tensor does not fit raises ValueError or TypeError.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <optional>

#include "domino.h"

namespace {

// The library's entry points, as bind() was given them: the build that the
// process has loaded (the debug build, for one).
decltype(&domino_token_loss) g_token_loss;
decltype(&domino_token_loss_grad) g_token_loss_grad;
decltype(&domino_distill_loss) g_distill_loss;
decltype(&domino_distill_grad) g_distill_grad;
decltype(&domino_embed) g_embed;
decltype(&domino_embed_grad) g_embed_grad;
decltype(&domino_norm) g_norm;
decltype(&domino_norm8) g_norm8;
decltype(&domino_norm_grad) g_norm_grad;
decltype(&domino_quantize8) g_quantize8;
decltype(&domino_logits8) g_logits8;
decltype(&domino_mask_logits_penalized) g_mask_logits_penalized;
decltype(&domino_mask_sample_penalized) g_mask_sample_penalized;

// What a call raises: kept until its arguments have all been read.
struct Refused {
    PyObject* type;
    const char* what;
    const char* why;
};

int64_t integer(PyObject* o, const char* what) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, what, "an integer expected"};
    }
    return v;
}
int32_t integer32(PyObject* o, const char* what) {
    const int64_t v = integer(o, what);
    if (v != (int32_t)v) throw Refused{PyExc_ValueError, what, "too large"};
    return (int32_t)v;
}
float number(PyObject* o, const char* what) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{PyExc_TypeError, what, "a number expected"};
    }
    return (float)v;
}

// While it lives, torch's current stream of the device is the call's: outputs come from that stream's memory, not from
// blocks that the current one has given back and may still be using.  They stay in use (made()) until what the current
// stream does with them has ended.
class OnStream {
  public:
    OnStream(void* stream, int device) {
        if (device < 0) return;
        const c10::cuda::CUDAStream now = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device);
        if ((void*)now.stream() == stream) return;
        current_ = now;
        // cudaStreamLegacy is the default stream's other name
        cudaStream_t to = (cudaStream_t)stream == cudaStreamLegacy ? nullptr : (cudaStream_t)stream;
        c10::cuda::setCurrentCUDAStream(c10::cuda::getStreamFromExternal(to, (c10::DeviceIndex)device));
    }
    OnStream(const OnStream&) = delete;
    ~OnStream() {
        if (current_) c10::cuda::setCurrentCUDAStream(*current_);
    }
    at::Tensor made(at::Tensor t) const {
        if (current_) t.record_stream(current_->unwrap());
        return t;
    }

  private:
    std::optional<c10::cuda::CUDAStream> current_;
};

struct Call {
    domino_t h;
    int device;
    void* stream;
    OnStream on;
    Call(PyObject* const* args, PyObject* st)
        : h((domino_t)(uintptr_t)(args[0] == Py_None ? 0 : integer(args[0], "handle"))),
          device(integer32(args[1], "device")),
          stream(st == Py_None ? (device < 0 ? nullptr : (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream())
                               : (void*)(uintptr_t)integer(st, "stream")),
          on(stream, device) {}
};

struct Matrix {
    at::Tensor t;
    int64_t rows, cols, step;   // elements from a row to the next; of at most one row, its length
    int32_t dtype;
    void* p() const { return t.data_ptr(); }
};

const at::Tensor& tensor(PyObject* o, int device, const char* what) {
    if (!THPVariable_Check(o)) throw Refused{PyExc_TypeError, what, "a tensor expected"};
    const at::Tensor& t = THPVariable_Unpack(o);
    // autograd does not see these calls: what they return would be a constant to it
    if (t.requires_grad() && at::GradMode::is_enabled())
        throw Refused{PyExc_RuntimeError, what,
                      "requires a gradient, which these calls do not record; pass detach(), or call under torch.no_grad()"};
    if (!t.is_cuda() || t.get_device() != device) throw Refused{PyExc_ValueError, what, "not on the handle's device"};
    return t;
}

Matrix matrix(PyObject* o, int device, const char* what) {
    const at::Tensor& t = tensor(o, device, what);
    if (t.dim() != 2) throw Refused{PyExc_ValueError, what, "a matrix expected"};
    Matrix m{t, t.size(0), t.size(1), t.stride(0), 0};
    if (m.cols > 1 && t.stride(1) != 1) throw Refused{PyExc_ValueError, what, "rows must be contiguous"};
    if (m.rows <= 1) m.step = m.cols;
    if (m.rows > INT32_MAX || m.cols > INT32_MAX) throw Refused{PyExc_ValueError, what, "too large"};
    if (t.scalar_type() == at::kBFloat16) m.dtype = DOMINO_DTYPE_BF16;
    else if (t.scalar_type() == at::kFloat) m.dtype = DOMINO_DTYPE_F32;
    else throw Refused{PyExc_TypeError, what, "must be float32 or bfloat16"};
    return m;
}

// The matrix given, or a new one.
Matrix output(PyObject* o, const Call& c, const char* what, int64_t rows, int64_t cols, const Matrix& like) {
    if (o == Py_None) return Matrix{c.on.made(at::empty({rows, cols}, like.t.options())), rows, cols, cols, like.dtype};
    Matrix m = matrix(o, c.device, what);
    if (m.rows != rows || m.cols != cols) throw Refused{PyExc_ValueError, what, "another shape expected"};
    if (m.dtype != like.dtype) throw Refused{PyExc_TypeError, what, "must be of the inputs' type"};
    return m;
}

// n contiguous values of a 4-byte type.
const at::Tensor& words(PyObject* o, int device, at::ScalarType type, int64_t n, const char* what) {
    const at::Tensor& t = tensor(o, device, what);
    if (t.scalar_type() != type)
        throw Refused{PyExc_TypeError, what, type == at::kInt ? "must be int32" : "must be float32"};
    if (t.numel() != n || !t.is_contiguous()) throw Refused{PyExc_ValueError, what, "another number of contiguous values expected"};
    return t;
}
at::Tensor floats(PyObject* o, const Call& c, int64_t n, const char* what, const Matrix& like) {
    return o == Py_None ? c.on.made(at::empty({n}, like.t.options().dtype(at::kFloat))) : words(o, c.device, at::kFloat, n, what);
}

const uint32_t* mask_words(PyObject* o, int device, int64_t rows, int64_t n_tokens) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, device, "mask");
    if (t.scalar_type() != at::kInt && t.scalar_type() != at::kUInt32)
        throw Refused{PyExc_TypeError, "mask", "must be int32 or uint32"};
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != (n_tokens + 31) / 32 || !t.is_contiguous())
        throw Refused{PyExc_ValueError, "mask", "one contiguous row of ceil(n_tokens / 32) 32-bit words per row expected"};
    return (const uint32_t*)t.data_ptr();
}

PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
    PyObject* r = PyTuple_New(2);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(a));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(b));
    return r;
}

// torch.OutOfMemoryError, which every torch allocation raises.
PyObject* out_of_memory() {
    static PyObject* const type = [] {
        PyObject* torch = PyImport_ImportModule("torch");
        PyObject* t = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        Py_XDECREF(torch);
        if (!t) PyErr_Clear();
        return t ? t : PyExc_RuntimeError;
    }();
    return type;
}

// Runs f, whose exceptions become Python's.
template <int N, typename F>
PyObject* guarded(Py_ssize_t n, F f) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, not %zd", N, n);
        return nullptr;
    }
    try {
        return f();
    } catch (const Refused& r) {
        PyErr_Format(r.type, "%s: %s", r.what, r.why);
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(out_of_memory(), e.what_without_backtrace());
    } catch (const std::exception& e) {   // torch's
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

struct LossInputs {
    Matrix hidden, weight;
    const int32_t* targets;
    const uint32_t* mask;
    LossInputs(PyObject* h, PyObject* w, PyObject* y, PyObject* m, int device)
        : hidden(matrix(h, device, "hidden")), weight(matrix(w, device, "weight")) {
        if (weight.cols != hidden.cols) throw Refused{PyExc_ValueError, "weight", "hidden's number of columns expected"};
        if (weight.dtype != hidden.dtype) throw Refused{PyExc_TypeError, "weight", "must be of hidden's type"};
        targets = (const int32_t*)words(y, device, at::kInt, hidden.rows, "targets").data_ptr();
        mask = mask_words(m, device, hidden.rows, weight.rows);
    }
};

// (handle, device, hidden, weight, targets, mask, loss, lse, stream)
PyObject* token_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<9>(n, [&]() -> PyObject* {
        const Call c(a, a[8]);
        const LossInputs in(a[2], a[3], a[4], a[5], c.device);
        const at::Tensor loss = floats(a[6], c, in.hidden.rows, "loss", in.hidden);
        const at::Tensor lse = floats(a[7], c, in.hidden.rows, "lse", in.hidden);
        const int s = g_token_loss(c.h, in.hidden.p(), in.hidden.step, in.weight.p(), in.weight.step, in.hidden.dtype,
                                   (int32_t)in.hidden.rows, (int32_t)in.hidden.cols, (int32_t)in.weight.rows, in.mask, in.targets,
                                   (float*)loss.data_ptr(), (float*)lse.data_ptr(), c.stream);
        return s ? PyLong_FromLong(s) : pair(loss, lse);
    });
}

// (handle, device, hidden, weight, targets, lse, grad_loss, mask, dhidden, dweight, stream)
PyObject* token_loss_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<11>(n, [&]() -> PyObject* {
        const Call c(a, a[10]);
        const LossInputs in(a[2], a[3], a[4], a[7], c.device);
        const at::Tensor &lse = words(a[5], c.device, at::kFloat, in.hidden.rows, "lse"),
                         &g = words(a[6], c.device, at::kFloat, in.hidden.rows, "grad_loss");
        const Matrix dh = output(a[8], c, "dhidden", in.hidden.rows, in.hidden.cols, in.hidden);
        const Matrix dw = output(a[9], c, "dweight", in.weight.rows, in.weight.cols, in.hidden);
        const int s = g_token_loss_grad(c.h, in.hidden.p(), in.hidden.step, in.weight.p(), in.weight.step, in.hidden.dtype,
                                        (int32_t)in.hidden.rows, (int32_t)in.hidden.cols, (int32_t)in.weight.rows, in.mask,
                                        in.targets, (const float*)lse.data_ptr(), (const float*)g.data_ptr(), dh.p(), dh.step,
                                        dw.p(), dw.step, c.stream);
        return s ? PyLong_FromLong(s) : pair(dh.t, dw.t);
    });
}

struct DistillInputs {
    Matrix logits, teacher;
    const int32_t* ids;
    const uint32_t* mask;
    float temperature;
    DistillInputs(PyObject* x, PyObject* t, PyObject* i, PyObject* tau, PyObject* m, int device)
        : logits(matrix(x, device, "logits")), teacher(matrix(t, device, "teacher")) {
        if (teacher.rows != logits.rows || teacher.step != teacher.cols)
            throw Refused{PyExc_ValueError, "teacher", "the logits' number of contiguous rows expected"};
        const at::Tensor& id = words(i, device, at::kInt, teacher.rows * teacher.cols, "ids");
        if (id.sizes() != teacher.t.sizes()) throw Refused{PyExc_ValueError, "ids", "the teacher's shape expected"};
        ids = (const int32_t*)id.data_ptr();
        mask = mask_words(m, device, logits.rows, logits.cols);
        temperature = number(tau, "temperature");
    }
};

// (handle, device, logits, teacher, ids, temperature, mask, loss, lse, stream)
PyObject* distill_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<10>(n, [&]() -> PyObject* {
        const Call c(a, a[9]);
        const DistillInputs in(a[2], a[3], a[4], a[5], a[6], c.device);
        const at::Tensor loss = floats(a[7], c, in.logits.rows, "loss", in.logits);
        const at::Tensor lse = floats(a[8], c, in.logits.rows, "lse", in.logits);
        const int s = g_distill_loss(c.h, in.logits.p(), in.logits.dtype, (int32_t)in.logits.rows, in.logits.step,
                                     (int32_t)in.logits.cols, in.mask, in.teacher.p(), in.teacher.dtype, in.ids,
                                     (int32_t)in.teacher.cols, in.temperature, (float*)loss.data_ptr(), (float*)lse.data_ptr(),
                                     c.stream);
        return s ? PyLong_FromLong(s) : pair(loss, lse);
    });
}

// (handle, device, logits, teacher, ids, temperature, lse, grad_loss, mask, out, stream)
PyObject* distill_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<11>(n, [&]() -> PyObject* {
        const Call c(a, a[10]);
        const DistillInputs in(a[2], a[3], a[4], a[5], a[8], c.device);
        const at::Tensor &lse = words(a[6], c.device, at::kFloat, in.logits.rows, "lse"),
                         &g = words(a[7], c.device, at::kFloat, in.logits.rows, "grad_loss");
        const Matrix out = output(a[9], c, "out", in.logits.rows, in.logits.cols, in.logits);
        const int s = g_distill_grad(c.h, in.logits.p(), in.logits.dtype, (int32_t)in.logits.rows, in.logits.step,
                                     (int32_t)in.logits.cols, in.mask, in.teacher.p(), in.teacher.dtype, in.ids,
                                     (int32_t)in.teacher.cols, in.temperature, (const float*)lse.data_ptr(),
                                     (const float*)g.data_ptr(), out.p(), out.step, c.stream);
        return s ? PyLong_FromLong(s) : THPVariable_Wrap(out.t);
    });
}

// (handle, device, tokens, weight, scale, out, stream)
PyObject* embed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<7>(n, [&]() -> PyObject* {
        const Call c(a, a[6]);
        const at::Tensor& t = tensor(a[2], c.device, "tokens");
        const Matrix w = matrix(a[3], c.device, "weight");
        words(a[2], c.device, at::kInt, t.numel(), "tokens");
        if (t.numel() > INT32_MAX) throw Refused{PyExc_ValueError, "tokens", "too large"};
        const Matrix out = output(a[5], c, "out", t.numel(), w.cols, w);
        const int s = g_embed(c.h, (const int32_t*)t.data_ptr(), (int32_t)t.numel(), w.p(), w.step, w.dtype, (int32_t)w.rows,
                              (int32_t)w.cols, number(a[4], "scale"), out.p(), out.step, c.stream);
        return s ? PyLong_FromLong(s) : THPVariable_Wrap(out.t);
    });
}

// (handle, device, tokens, grad, n_tokens, scale, into or out, whether it is added to, stream)
PyObject* embed_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<9>(n, [&]() -> PyObject* {
        const Call c(a, a[8]);
        const Matrix g = matrix(a[3], c.device, "grad");
        const at::Tensor& t = words(a[2], c.device, at::kInt, g.rows, "tokens");
        const int32_t V = integer32(a[4], "n_tokens");
        if (V < 1) throw Refused{PyExc_ValueError, "n_tokens", "at least 1 expected"};
        const Matrix dw = output(a[6], c, "into", V, g.cols, g);
        const int s = g_embed_grad(c.h, (const int32_t*)t.data_ptr(), (int32_t)g.rows, g.p(), g.step, g.dtype, V,
                                   (int32_t)g.cols, number(a[5], "scale"), a[7] == Py_True ? 1 : 0, dw.p(), dw.step, c.stream);
        return s ? PyLong_FromLong(s) : THPVariable_Wrap(dw.t);
    });
}

// Codes: rows on 16-byte boundaries.
struct Codes {
    at::Tensor t;
    int64_t rows, cols, step;
    uint8_t* p() const { return (uint8_t*)t.data_ptr(); }
};
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

Codes codes(PyObject* o, int device, const char* what) {
    const at::Tensor& t = tensor(o, device, what);
    if (t.dim() != 2) throw Refused{PyExc_ValueError, what, "a matrix expected"};
    if (t.scalar_type() != at::kFloat8_e4m3fn) throw Refused{PyExc_TypeError, what, "must be float8_e4m3fn"};
    Codes c{t, t.size(0), t.size(1), t.stride(0)};
    if (c.cols > 1 && t.stride(1) != 1) throw Refused{PyExc_ValueError, what, "rows must be contiguous"};
    if (c.rows <= 1) c.step = up16(c.cols);
    if (c.rows > INT32_MAX || c.cols > INT32_MAX) throw Refused{PyExc_ValueError, what, "too large"};
    if (c.step % 16 || (uintptr_t)t.data_ptr() % 16)
        throw Refused{PyExc_ValueError, what, "rows must begin on 16-byte boundaries (as quantize8 and norm8 return them)"};
    return c;
}
Codes codes_out(PyObject* o, const Call& c, const char* what, int64_t rows, int64_t cols, const at::Tensor& like) {
    if (o == Py_None) {
        const int64_t step = up16(cols);
        return {c.on.made(at::empty_strided({rows, cols}, {step, 1}, like.options().dtype(at::kFloat8_e4m3fn))), rows, cols, step};
    }
    Codes m = codes(o, c.device, what);
    if (m.rows != rows || m.cols != cols) throw Refused{PyExc_ValueError, what, "another shape expected"};
    return m;
}
// A contiguous fp32 matrix.
at::Tensor scales(PyObject* o, const Call& c, const char* what, int64_t rows, int64_t cols, const at::Tensor* like) {
    if (like && o == Py_None) return c.on.made(at::empty({rows, cols}, like->options().dtype(at::kFloat)));
    const at::Tensor& t = words(o, c.device, at::kFloat, rows * cols, what);
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) throw Refused{PyExc_ValueError, what, "another shape expected"};
    return t;
}
int64_t blocks(int64_t n) { return (n + 127) / 128; }

PyObject* three(const at::Tensor& a, const at::Tensor& b, const at::Tensor& d) {
    PyObject* r = PyTuple_New(3);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(a));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(b));
    PyTuple_SET_ITEM(r, 2, THPVariable_Wrap(d));
    return r;
}

// A vector of a matrix's type and width.
const at::Tensor& vector(PyObject* o, int device, const Matrix& like, const char* what) {
    const at::Tensor& t = tensor(o, device, what);
    if (t.scalar_type() != like.t.scalar_type()) throw Refused{PyExc_TypeError, what, "must be of the stream's type"};
    if (t.dim() != 1 || t.size(0) != like.cols || !t.is_contiguous()) throw Refused{PyExc_ValueError, what, "a value for each column expected"};
    return t;
}
// A matrix of another's shape and type, or none.
std::optional<Matrix> beside(PyObject* o, int device, const Matrix& like, const char* what) {
    if (o == Py_None) return std::nullopt;
    Matrix m = matrix(o, device, what);
    if (m.rows != like.rows || m.cols != like.cols) throw Refused{PyExc_ValueError, what, "another shape expected"};
    if (m.dtype != like.dtype) throw Refused{PyExc_TypeError, what, "must be of the stream's type"};
    return m;
}

struct NormInputs {
    Matrix x;
    const at::Tensor& weight;
    std::optional<Matrix> residual;
    float eps;
    Matrix sum;                    // x without a residual
    NormInputs(PyObject* x_, PyObject* w, PyObject* r, PyObject* e, PyObject* s, const Call& c)
        : x(matrix(x_, c.device, "x")), weight(vector(w, c.device, x, "weight")), residual(beside(r, c.device, x, "residual")),
          eps(number(e, "eps")), sum(x) {
        if (residual) sum = output(s, c, "sum", x.rows, x.cols, x);
        else if (s != Py_None) throw Refused{PyExc_ValueError, "sum", "is x where there is no residual"};
    }
    const void* residual_p() const { return residual ? residual->p() : nullptr; }
    int64_t residual_step() const { return residual ? residual->step : 0; }
    void* sum_p() const { return residual ? sum.p() : nullptr; }
};

// (handle, device, x, weight, residual, eps, y, sum, rstd, stream)
PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<10>(n, [&]() -> PyObject* {
        const Call c(a, a[9]);
        const NormInputs in(a[2], a[3], a[4], a[5], a[7], c);
        const Matrix y = output(a[6], c, "y", in.x.rows, in.x.cols, in.x);
        const at::Tensor rstd = floats(a[8], c, in.x.rows, "rstd", in.x);
        const int s = g_norm(c.h, in.x.p(), in.x.step, in.residual_p(), in.residual_step(), in.weight.data_ptr(), in.x.dtype,
                             (int32_t)in.x.rows, (int32_t)in.x.cols, in.eps, y.p(), y.step, in.sum_p(), in.sum.step,
                             (float*)rstd.data_ptr(), c.stream);
        return s ? PyLong_FromLong(s) : three(y.t, in.sum.t, rstd);
    });
}

// (handle, device, x, weight, residual, eps, codes, scales, sum, stream)
PyObject* norm8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<10>(n, [&]() -> PyObject* {
        const Call c(a, a[9]);
        const NormInputs in(a[2], a[3], a[4], a[5], a[8], c);
        const Codes q = codes_out(a[6], c, "codes", in.x.rows, in.x.cols, in.x.t);
        const at::Tensor sc = scales(a[7], c, "scales", in.x.rows, blocks(in.x.cols), &in.x.t);
        const int s = g_norm8(c.h, in.x.p(), in.x.step, in.residual_p(), in.residual_step(), in.weight.data_ptr(), in.x.dtype,
                              (int32_t)in.x.rows, (int32_t)in.x.cols, in.eps, q.p(), q.step, (float*)sc.data_ptr(), in.sum_p(),
                              in.sum.step, c.stream);
        return s ? PyLong_FromLong(s) : three(q.t, sc, in.sum.t);
    });
}

// (handle, device, sum, weight, rstd, dy, dsum, dx, dweight, stream)
PyObject* norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<10>(n, [&]() -> PyObject* {
        const Call c(a, a[9]);
        const Matrix h = matrix(a[2], c.device, "sum");
        const at::Tensor& w = vector(a[3], c.device, h, "weight");
        const at::Tensor& rstd = words(a[4], c.device, at::kFloat, h.rows, "rstd");
        const std::optional<Matrix> dy = beside(a[5], c.device, h, "dy"), ds = beside(a[6], c.device, h, "dsum");
        if (!dy) throw Refused{PyExc_TypeError, "dy", "a tensor expected"};
        const Matrix dx = output(a[7], c, "dx", h.rows, h.cols, h);
        const at::Tensor dw = a[8] == Py_None ? c.on.made(at::empty({h.cols}, h.t.options())) : vector(a[8], c.device, h, "dweight");
        const int s = g_norm_grad(c.h, h.p(), h.step, w.data_ptr(), (const float*)rstd.data_ptr(), dy->p(), dy->step,
                                  ds ? ds->p() : nullptr, ds ? ds->step : 0, h.dtype, (int32_t)h.rows, (int32_t)h.cols, dx.p(),
                                  dx.step, dw.data_ptr(), c.stream);
        return s ? PyLong_FromLong(s) : pair(dx.t, dw);
    });
}

// (handle, device, x, block, codes, scales, stream)
PyObject* quantize8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<7>(n, [&]() -> PyObject* {
        const Call c(a, a[6]);
        const Matrix x = matrix(a[2], c.device, "x");
        const int32_t block = integer32(a[3], "block");
        if (block != 1 && block != 128) throw Refused{PyExc_ValueError, "block", "1 or 128 expected"};
        const Codes q = codes_out(a[4], c, "codes", x.rows, x.cols, x.t);
        const at::Tensor sc = scales(a[5], c, "scales", block == 1 ? x.rows : blocks(x.rows), blocks(x.cols), &x.t);
        const int s = g_quantize8(c.h, x.p(), x.step, x.dtype, (int32_t)x.rows, (int32_t)x.cols, block, q.p(), q.step,
                                  (float*)sc.data_ptr(), c.stream);
        return s ? PyLong_FromLong(s) : pair(q.t, sc);
    });
}

// The type of logits: that of `out` where none is given, fp32 where there is none either.
int32_t logits_type(PyObject* dtype, PyObject* out) {
    at::ScalarType t = at::kFloat;
    if (dtype != Py_None) {
        if (!THPDtype_Check(dtype)) throw Refused{PyExc_TypeError, "dtype", "a torch.dtype expected"};
        t = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
    } else if (THPVariable_Check(out)) {
        t = THPVariable_Unpack(out).scalar_type();
    }
    if (t != at::kFloat && t != at::kBFloat16) throw Refused{PyExc_TypeError, "dtype", "must be float32 or bfloat16"};
    return t == at::kBFloat16 ? DOMINO_DTYPE_BF16 : DOMINO_DTYPE_F32;
}

// (handle, device, codes, scales, weight codes, weight scales, dtype, out, stream)
PyObject* logits8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<9>(n, [&]() -> PyObject* {
        const int32_t dtype = logits_type(a[6], a[7]);
        const Call c(a, a[8]);
        const Codes h = codes(a[2], c.device, "codes"), w = codes(a[4], c.device, "weight codes");
        if (w.cols != h.cols) throw Refused{PyExc_ValueError, "weight codes", "the hidden codes' number of columns expected"};
        const at::Tensor hs = scales(a[3], c, "scales", h.rows, blocks(h.cols), nullptr);
        const at::Tensor ws = scales(a[5], c, "weight scales", blocks(w.rows), blocks(w.cols), nullptr);
        Matrix out;
        if (a[7] == Py_None) {   // rows on 16-byte boundaries
            const int64_t per = dtype == DOMINO_DTYPE_BF16 ? 8 : 4, step = (w.rows + per - 1) / per * per;
            out = Matrix{c.on.made(at::empty_strided({h.rows, w.rows}, {step, 1},
                                                     h.t.options().dtype(dtype == DOMINO_DTYPE_BF16 ? at::kBFloat16 : at::kFloat))),
                         h.rows, w.rows, step, dtype};
        } else {
            out = matrix(a[7], c.device, "out");
            if (out.rows != h.rows || out.cols != w.rows) throw Refused{PyExc_ValueError, "out", "another shape expected"};
            if (out.dtype != dtype) throw Refused{PyExc_TypeError, "out", "must be of dtype"};
        }
        const int s = g_logits8(c.h, h.p(), h.step, (const float*)hs.data_ptr(), w.p(), w.step, (const float*)ws.data_ptr(),
                                (int32_t)h.rows, (int32_t)h.cols, (int32_t)w.rows, dtype, out.p(), out.step, c.stream);
        return s ? PyLong_FromLong(s) : THPVariable_Wrap(out.t);
    });
}

// logits, history, lengths, prompt_lengths, repetition, presence, frequency, bias_ids, bias_values, mask
struct Penalized {
    Matrix logits;
    domino_penalties p{};
    const uint32_t* mask;
    Penalized(PyObject* const* a, int device) : logits(matrix(a[0], device, "logits")) {
        const int64_t rows = logits.rows;
        const auto each = [&](PyObject* o, at::ScalarType type, const char* what) -> const void* {
            return o == Py_None ? nullptr : words(o, device, type, rows, what).data_ptr();
        };
        const auto table = [&](PyObject* o, at::ScalarType type, const char* what, int32_t& columns) -> const void* {
            if (o == Py_None) return nullptr;
            const at::Tensor& t = tensor(o, device, what);
            if (t.dim() != 2 || t.size(0) != rows) throw Refused{PyExc_ValueError, what, "a matrix with a row for each of the logits' expected"};
            if (t.size(1) > INT32_MAX) throw Refused{PyExc_ValueError, what, "too large"};
            columns = (int32_t)t.size(1);
            return words(o, device, type, rows * t.size(1), what).data_ptr();
        };
        p.history_dev = (const int32_t*)table(a[1], at::kInt, "history", p.history_len);
        p.lengths_dev = (const int32_t*)each(a[2], at::kInt, "lengths");
        p.prompt_lengths_dev = (const int32_t*)each(a[3], at::kInt, "prompt_lengths");
        p.repetition_dev = (const float*)each(a[4], at::kFloat, "repetition");
        p.presence_dev = (const float*)each(a[5], at::kFloat, "presence");
        p.frequency_dev = (const float*)each(a[6], at::kFloat, "frequency");
        int32_t values = 0;
        p.bias_ids_dev = (const int32_t*)table(a[7], at::kInt, "bias_ids", p.n_bias);
        p.bias_values_dev = (const float*)table(a[8], at::kFloat, "bias_values", values);
        if (values != p.n_bias || (a[7] == Py_None) != (a[8] == Py_None))
            throw Refused{PyExc_ValueError, "bias_values", "a value for each of bias_ids expected"};
        mask = mask_words(a[9], device, rows, logits.cols);
    }
};

// (handle, device, the ten of Penalized, argmax, lse or whether it is wanted, logprobs or whether they are, stream)
PyObject* mask_logits_penalized(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<16>(n, [&]() -> PyObject* {
        const Call c(a, a[15]);
        const Penalized in(a + 2, c.device);
        const int64_t rows = in.logits.rows, V = in.logits.cols;
        const at::Tensor argmax = a[12] == Py_None ? c.on.made(at::empty({rows}, in.logits.t.options().dtype(at::kInt)))
                                                   : words(a[12], c.device, at::kInt, rows, "argmax");
        // None: not wanted; True: a new one
        std::optional<at::Tensor> lse, lp;
        if (a[13] != Py_None) lse = floats(a[13] == Py_True ? Py_None : a[13], c, rows, "lse", in.logits);
        if (a[14] != Py_None) lp = scales(a[14] == Py_True ? Py_None : a[14], c, "logprobs", rows, V, &in.logits.t);
        const int s = g_mask_logits_penalized(c.h, in.logits.p(), in.logits.dtype, (int32_t)rows, in.logits.step, (int32_t)V, &in.p,
                                              in.mask, (int32_t*)argmax.data_ptr(), lse ? (float*)lse->data_ptr() : nullptr,
                                              lp ? (float*)lp->data_ptr() : nullptr, c.stream);
        if (s) return PyLong_FromLong(s);
        PyObject* r = PyTuple_New(3);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(argmax));
        PyTuple_SET_ITEM(r, 1, lse ? THPVariable_Wrap(*lse) : Py_NewRef(Py_None));
        PyTuple_SET_ITEM(r, 2, lp ? THPVariable_Wrap(*lp) : Py_NewRef(Py_None));
        return r;
    });
}

// (handle, device, the ten of Penalized, temperature, seed, offset, tokens, stream)
PyObject* mask_sample_penalized(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<17>(n, [&]() -> PyObject* {
        const Call c(a, a[16]);
        const Penalized in(a + 2, c.device);
        const float temperature = number(a[12], "temperature");
        const auto bits = [](PyObject* o, const char* what) {
            const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
            if (PyErr_Occurred()) {
                PyErr_Clear();
                throw Refused{PyExc_TypeError, what, "an integer expected"};
            }
            return (uint64_t)v;
        };
        const uint64_t seed = bits(a[13], "seed"), offset = bits(a[14], "offset");
        const at::Tensor tokens = a[15] == Py_None ? c.on.made(at::empty({in.logits.rows}, in.logits.t.options().dtype(at::kInt)))
                                                   : words(a[15], c.device, at::kInt, in.logits.rows, "tokens");
        const int s = g_mask_sample_penalized(c.h, in.logits.p(), in.logits.dtype, (int32_t)in.logits.rows, in.logits.step,
                                              (int32_t)in.logits.cols, &in.p, in.mask, temperature, seed, offset,
                                              (int32_t*)tokens.data_ptr(), c.stream);
        return s ? PyLong_FromLong(s) : THPVariable_Wrap(tokens);
    });
}

// The entry points' addresses.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<13>(n, [&]() -> PyObject* {
        g_token_loss = (decltype(g_token_loss))integer(a[0], "address");
        g_token_loss_grad = (decltype(g_token_loss_grad))integer(a[1], "address");
        g_distill_loss = (decltype(g_distill_loss))integer(a[2], "address");
        g_distill_grad = (decltype(g_distill_grad))integer(a[3], "address");
        g_embed = (decltype(g_embed))integer(a[4], "address");
        g_embed_grad = (decltype(g_embed_grad))integer(a[5], "address");
        g_norm = (decltype(g_norm))integer(a[6], "address");
        g_norm8 = (decltype(g_norm8))integer(a[7], "address");
        g_norm_grad = (decltype(g_norm_grad))integer(a[8], "address");
        g_quantize8 = (decltype(g_quantize8))integer(a[9], "address");
        g_logits8 = (decltype(g_logits8))integer(a[10], "address");
        g_mask_logits_penalized = (decltype(g_mask_logits_penalized))integer(a[11], "address");
        g_mask_sample_penalized = (decltype(g_mask_sample_penalized))integer(a[12], "address");
        Py_RETURN_NONE;
    });
}

#define DOMINO_CALL(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {DOMINO_CALL(bind),         DOMINO_CALL(token_loss), DOMINO_CALL(token_loss_grad),
                           DOMINO_CALL(distill_loss), DOMINO_CALL(distill_grad), DOMINO_CALL(embed),
                           DOMINO_CALL(embed_grad),   DOMINO_CALL(norm),       DOMINO_CALL(norm8),
                           DOMINO_CALL(norm_grad),    DOMINO_CALL(quantize8),  DOMINO_CALL(logits8),
                           DOMINO_CALL(mask_logits_penalized), DOMINO_CALL(mask_sample_penalized),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_loss_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__loss_calls() { return PyModule_Create(&g_module); }
