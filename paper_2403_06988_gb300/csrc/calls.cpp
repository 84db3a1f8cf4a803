// calls.cpp -- the Python calls of the losses over the vocabulary and of the
// embedding (the Python extension _loss_calls.so): checks torch tensors, makes the
// outputs that are not given, and calls the C ABI.  Of a small call's time the
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

// The six entry points' addresses.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded<6>(n, [&]() -> PyObject* {
        g_token_loss = (decltype(g_token_loss))integer(a[0], "address");
        g_token_loss_grad = (decltype(g_token_loss_grad))integer(a[1], "address");
        g_distill_loss = (decltype(g_distill_loss))integer(a[2], "address");
        g_distill_grad = (decltype(g_distill_grad))integer(a[3], "address");
        g_embed = (decltype(g_embed))integer(a[4], "address");
        g_embed_grad = (decltype(g_embed_grad))integer(a[5], "address");
        Py_RETURN_NONE;
    });
}

#define DOMINO_CALL(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {DOMINO_CALL(bind),         DOMINO_CALL(token_loss), DOMINO_CALL(token_loss_grad),
                           DOMINO_CALL(distill_loss), DOMINO_CALL(distill_grad), DOMINO_CALL(embed),
                           DOMINO_CALL(embed_grad),   {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_loss_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__loss_calls() { return PyModule_Create(&g_module); }
