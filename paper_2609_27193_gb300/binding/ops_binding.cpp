// ops_binding.cpp -- the operators of a training step over torch tensors: checks
// of what a raw pointer cannot carry, outputs from torch's allocator, and one call
// of the C ABI each.  Python's ops.py has the interface and its documentation.
//
// In C++ and not through ctypes: with a few tokens the kernels take 2 to 10 us, and
// a call that allocates three outputs took 17 to 22 us on the host that way.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAStream.h>
#include <cuda_runtime_api.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <map>
#include <stdexcept>
#include <string>
#include <utility>

#include "layercheck.h"

namespace {

PyObject* g_error = nullptr;   // the package's LCError
PyObject* g_memory = nullptr;  // torch's OutOfMemoryError

struct TypeError : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct ValueError : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct StatusError {
    lc_status status;
};
struct Raised {};              // a Python error is set already

void check(lc_status st) {
    if (st != LC_OK) throw StatusError{st};
}

// --- arguments ----------------------------------------------------------------

struct Args {
    PyObject* const* a;
    Py_ssize_t n, at = 0;
    Args(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t want) : a(args), n(nargs) {
        if (nargs != want) throw TypeError("wrong number of arguments");
    }
    // A tensor, or an undefined one for None.
    at::Tensor tensor() {
        PyObject* o = a[at++];
        if (o == Py_None) return at::Tensor();
        if (!THPVariable_Check(o)) throw TypeError("a tensor is needed");
        return THPVariable_Unpack(o);
    }
    int64_t integer() {
        const long long v = PyLong_AsLongLong(a[at++]);
        if (v == -1 && PyErr_Occurred()) throw Raised{};
        return v;
    }
    double number() {
        const double v = PyFloat_AsDouble(a[at++]);
        if (v == -1.0 && PyErr_Occurred()) throw Raised{};
        return v;
    }
    bool truth() {
        const int v = PyObject_IsTrue(a[at++]);
        if (v < 0) throw Raised{};
        return v != 0;
    }
};

int code_of(const at::Tensor& t, const char* name) {
    if (t.scalar_type() == at::kBFloat16) return LC_BF16;
    if (t.scalar_type() == at::kFloat) return LC_F32;
    throw TypeError(std::string(name) + " must be bfloat16 or float32");
}
at::ScalarType type_of(int64_t code) { return code == LC_BF16 ? at::kBFloat16 : at::kFloat; }

int cuda_index(const at::Tensor& t) {
    if (!t.defined()) throw TypeError("a tensor is needed");
    if (!t.is_cuda()) throw ValueError("the operators need CUDA tensors");
    return t.get_device();
}
void same_device(int index, const at::Tensor& t) {
    if (t.defined() && (!t.is_cuda() || t.get_device() != index))
        throw ValueError("every tensor must be on one CUDA device");
}

lc_rows rows_of(const at::Tensor& t, const char* name) {
    lc_rows r{};
    r.dtype = code_of(t, name);
    if (t.dim() != 2 || (t.stride(1) != 1 && t.size(1) > 1))
        throw ValueError(std::string(name) + " must be 2-D with contiguous rows");
    r.data = t.data_ptr();
    r.stride = t.stride(0);
    return r;
}
void shaped(const at::Tensor& t, int64_t rows, int64_t dim, const char* name) {
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != dim)
        throw ValueError(std::string(name) + " must have shape [" + std::to_string(rows) + ", " + std::to_string(dim) + "]");
}
void* param_of(const at::Tensor& t, int64_t dim, const char* name) {
    code_of(t, name);
    if (t.dim() != 1 || t.size(0) != dim || !t.is_contiguous())
        throw ValueError(std::string(name) + " must be contiguous with " + std::to_string(dim) + " elements");
    return t.data_ptr();
}
float* stat_of(const at::Tensor& t, int64_t n) {
    if (!t.defined()) return nullptr;
    if (t.scalar_type() != at::kFloat || t.dim() != 1 || t.size(0) != n || !t.is_contiguous())
        throw ValueError("mean and rstd must be contiguous float32 with " + std::to_string(n) + " elements");
    return t.data_ptr<float>();
}
int ids_of(const at::Tensor& t) {
    if (!t.defined()) throw TypeError("a tensor is needed");
    const int code = t.scalar_type() == at::kInt ? LC_I32 : t.scalar_type() == at::kLong ? LC_I64 : -1;
    if (code < 0) throw TypeError("ids must be int32 or int64");
    if (t.dim() != 1 || !t.is_contiguous()) throw ValueError("ids must be 1-D and contiguous");
    return code;
}
// A checkpoint of n rows of dim values.  What was checked when it was made is checked
// for every call: its tensors and its width can be other ones by now.
lc_act act_of(const at::Tensor& q, const at::Tensor& e, int64_t n, int64_t dim) {
    const int64_t blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    if (!q.defined() || !e.defined() || dim < 1 || q.scalar_type() != at::kChar || e.scalar_type() != at::kChar || q.dim() != 2 ||
        e.dim() != 2 || q.size(0) != n || e.size(0) != n || q.size(1) < blocks * LC_ACT_BLOCK || e.size(1) < blocks ||
        q.stride(1) != 1 || (e.stride(1) != 1 && e.size(1) > 1))
        throw ValueError("a checkpoint of " + std::to_string(n) + " rows of " + std::to_string(dim) + " has int8 rows of " +
                         std::to_string(blocks * LC_ACT_BLOCK) + " values and " + std::to_string(blocks) + " exponents");
    // (the stride of a single row may be anything)
    return lc_act{static_cast<int8_t*>(q.data_ptr()), n > 1 ? q.stride(0) : blocks * LC_ACT_BLOCK, static_cast<int8_t*>(e.data_ptr()),
                  n > 1 ? e.stride(0) : blocks};
}

// The forward calls leave no trace for autograd: with it on, what a parameter went into
// would come out detached, and training would go on without that parameter's gradient.
void unrecorded(const char* call, std::initializer_list<const at::Tensor*> inputs) {
    if (!at::GradMode::is_enabled()) return;
    for (const at::Tensor* t : inputs)
        if (t->defined() && t->requires_grad())
            throw std::runtime_error(std::string(call) + " is not recorded by autograd, and an input requires a gradient: call it under "
                                     "torch.no_grad() or in the forward of a torch.autograd.Function");
}
// A tensor that was passed in has other contents now; torch's check of what a backward
// saved goes by this count (which inference tensors do not have).
void written(const at::Tensor& t) {
    if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// A new tensor on the device of another one (past torch's dispatcher: 1 us less a tensor).
at::Tensor make(at::IntArrayRef size, at::ScalarType type, const at::Tensor& like) {
    return at::detail::empty_cuda(size, type, like.device(), std::nullopt);
}

void* stream_of(int index) { return c10::cuda::getCurrentCUDAStream(c10::DeviceIndex(index)).stream(); }

// Scratch of one call.  Of a device and stream there is one tensor, which grows to the
// largest call; the stream's order keeps its users apart.  A call that is captured has a
// tensor of its own: a graph holds its address for as long as it can be replayed, on any
// stream, and memory allocated during a capture belongs to the graph.  So has a call that
// needs more than kHeldMost, which the program gets back: such calls write and read tens of
// megabytes, which takes longer than the allocation's microsecond.
constexpr uint64_t kHeldMost = 32u << 20;
struct Scratch {
    at::Tensor own;
    void* p = nullptr;
    Scratch(const at::Tensor& like, int index, void* stream, uint64_t bytes) {
        static auto* held = new std::map<std::pair<int, void*>, at::Tensor>;   // never freed: the driver may be gone by then
        if (!bytes) return;
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(static_cast<cudaStream_t>(stream), &capture) != cudaSuccess)
            throw std::runtime_error("cannot tell whether the stream is being captured");
        at::Tensor& w = capture == cudaStreamCaptureStatusNone && bytes <= kHeldMost ? (*held)[{index, stream}] : own;
        if (!w.defined() || uint64_t(w.numel()) < bytes) w = make({int64_t(bytes)}, at::kByte, like);
        p = w.data_ptr();
    }
};

PyObject* wrapped(const at::Tensor& t) {
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
template <typename... T>
PyObject* tuple(const T&... t) {
    PyObject* r = PyTuple_New(sizeof...(t));
    if (!r) throw Raised{};
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(r, i++, wrapped(t)), ...);
    return r;
}

// --- the operators --------------------------------------------------------------

PyObject* embed(PyObject* const* args, Py_ssize_t nargs) {
    Args a(args, nargs, 4);
    const at::Tensor table = a.tensor(), ids = a.tensor();
    const double scale = a.number();
    at::Tensor out = a.tensor();
    const int index = cuda_index(table), type = ids_of(ids);
    same_device(index, ids);
    same_device(index, out);
    unrecorded("embed", {&table, &out});
    const lc_rows rt = rows_of(table, "table");
    const int64_t n = ids.numel(), dim = table.size(1);
    if (out.defined()) shaped(out, n, dim, "out");
    else out = make({n, dim}, table.scalar_type(), table);
    const lc_rows ro = rows_of(out, "out");
    check(lc_embed(index, stream_of(index), &rt, table.size(0), dim, ids.data_ptr(), type, n, float(scale), &ro));
    written(out);
    return wrapped(out);
}

PyObject* embed_grad(PyObject* const* args, Py_ssize_t nargs) {
    Args a(args, nargs, 8);
    const at::Tensor dy = a.tensor(), ids = a.tensor();
    int64_t vocab = a.integer();
    const double scale = a.number();
    at::Tensor grad = a.tensor();
    const int64_t dtype = a.integer(), skip = a.integer();
    const bool accumulate = a.truth();
    const int index = cuda_index(dy), type = ids_of(ids);
    same_device(index, ids);
    same_device(index, grad);
    const lc_rows rd = rows_of(dy, "dy");
    const int64_t n = dy.size(0), dim = dy.size(1);
    if (ids.numel() != n) throw ValueError("dy and ids must have the same number of tokens");
    if (grad.defined()) {
        if (vocab >= 0 && (!grad.dim() || grad.size(0) != vocab)) throw ValueError("grad must have vocab rows");
        vocab = grad.dim() ? grad.size(0) : 0;
        shaped(grad, vocab, dim, "grad");
    } else {
        if (accumulate) throw ValueError("accumulate needs grad");
        if (vocab < 0) throw ValueError("vocab or grad is needed");
        grad = make({vocab, dim}, dtype < 0 ? dy.scalar_type() : type_of(dtype), dy);
    }
    const lc_rows rg = rows_of(grad, "grad");
    void* stream = stream_of(index);
    const uint64_t need = lc_embed_grad_workspace(n, vocab, dim);
    const Scratch scratch(dy, index, stream, need);
    check(lc_embed_grad(index, stream, &rd, ids.data_ptr(), type, n, float(scale), skip, &rg, vocab, dim, accumulate,
                        scratch.p, need));
    written(grad);
    return wrapped(grad);
}

PyObject* act_save(PyObject* const* args, Py_ssize_t nargs) {
    Args a(args, nargs, 3);
    const at::Tensor x = a.tensor(), q = a.tensor(), e = a.tensor();
    const int index = cuda_index(x);
    same_device(index, q);
    same_device(index, e);
    const lc_rows rx = rows_of(x, "x");
    const lc_act act = act_of(q, e, x.size(0), x.size(1));
    check(lc_act_save(index, stream_of(index), &rx, x.size(0), x.size(1), &act));
    written(q);
    written(e);
    Py_RETURN_NONE;
}

PyObject* act_load(PyObject* const* args, Py_ssize_t nargs) {
    Args a(args, nargs, 5);
    const at::Tensor q = a.tensor(), e = a.tensor();
    const int64_t dim = a.integer();
    at::Tensor out = a.tensor();
    const int64_t dtype = a.integer();
    const int index = cuda_index(q);
    same_device(index, e);
    same_device(index, out);
    if (!q.dim()) throw ValueError("a checkpoint has rows");
    const int64_t n = q.size(0);
    const lc_act act = act_of(q, e, n, dim);
    if (out.defined()) shaped(out, n, dim, "out");
    else out = make({n, dim}, type_of(dtype), q);
    const lc_rows ro = rows_of(out, "out");
    check(lc_act_load(index, stream_of(index), &act, n, dim, &ro));
    written(out);
    return wrapped(out);
}

PyObject* new_act(PyObject* const* args, Py_ssize_t nargs) {
    Args a(args, nargs, 1);
    const at::Tensor x = a.tensor();
    cuda_index(x);
    if (x.dim() != 2 || x.size(1) < 1) throw ValueError("x must be 2-D with contiguous rows");
    const int64_t blocks = (x.size(1) + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    return tuple(make({x.size(0), blocks * LC_ACT_BLOCK}, at::kChar, x), make({x.size(0), blocks}, at::kChar, x));
}

PyObject* norm(PyObject* const* args, Py_ssize_t nargs) {
    Args a(args, nargs, 8);
    const at::Tensor x = a.tensor(), weight = a.tensor(), bias = a.tensor();
    const double eps = a.number();
    const int kind = int(a.integer());
    at::Tensor out = a.tensor();
    const at::Tensor q = a.tensor(), e = a.tensor();
    const int index = cuda_index(x);
    cuda_index(weight);
    for (const at::Tensor* t : {&weight, &bias, static_cast<const at::Tensor*>(&out), &q, &e}) same_device(index, *t);
    unrecorded("norm", {&x, &weight, &bias, &out});
    const lc_rows rx = rows_of(x, "x");
    const int64_t n = x.size(0), dim = x.size(1);
    const void* w = param_of(weight, dim, "weight");
    const void* b = bias.defined() ? param_of(bias, dim, "bias") : nullptr;
    if (b && bias.scalar_type() != weight.scalar_type()) throw ValueError("weight and bias must have one type");
    if (out.defined()) shaped(out, n, dim, "out");
    else out = make({n, dim}, x.scalar_type(), x);
    const lc_rows ro = rows_of(out, "out");
    const at::Tensor rstd = make({n}, at::kFloat, x), mean = kind == LC_NORM_LAYER ? make({n}, at::kFloat, x) : at::Tensor();
    lc_act keep{};
    if (q.defined()) keep = act_of(q, e, n, dim);
    check(lc_norm(index, stream_of(index), kind, &rx, n, dim, w, b, code_of(weight, "weight"), eps, &ro, stat_of(mean, n),
                  stat_of(rstd, n), q.defined() ? &keep : nullptr));
    for (const at::Tensor* t : {static_cast<const at::Tensor*>(&out), &q, &e}) written(*t);
    return tuple(out, mean, rstd);
}

PyObject* norm_grad(PyObject* const* args, Py_ssize_t nargs) {
    Args a(args, nargs, 14);
    const at::Tensor dy = a.tensor(), x = a.tensor(), q = a.tensor(), e = a.tensor();
    const int64_t kept_dim = a.integer();
    const at::Tensor weight = a.tensor(), mean = a.tensor(), rstd = a.tensor();
    const bool bias = a.truth();
    at::Tensor dx = a.tensor(), dweight = a.tensor(), dbias = a.tensor();
    const int64_t dtype = a.integer();
    const bool accumulate = a.truth();
    const int index = cuda_index(dy);
    cuda_index(weight);
    cuda_index(rstd);
    for (const at::Tensor* t : {&x, &q, &e, &weight, &mean, &rstd, static_cast<const at::Tensor*>(&dx),
                                static_cast<const at::Tensor*>(&dweight), static_cast<const at::Tensor*>(&dbias)})
        same_device(index, *t);
    const lc_rows rd = rows_of(dy, "dy");
    const int64_t n = dy.size(0), dim = dy.size(1);
    const void* w = param_of(weight, dim, "weight");
    lc_rows rx{};
    lc_act kept{};
    if (q.defined()) {
        if (kept_dim != dim) throw ValueError("x must have dy's shape");
        kept = act_of(q, e, n, dim);
    } else {
        cuda_index(x);
        rx = rows_of(x, "x");
        if (x.size(0) != n || x.size(1) != dim) throw ValueError("x must have dy's shape");
    }
    const float *m = stat_of(mean, n), *r = stat_of(rstd, n);
    if (accumulate && (!dweight.defined() || (bias && !dbias.defined())))
        throw ValueError("accumulate needs the gradients to add to");
    if (dx.defined()) shaped(dx, n, dim, "dx");
    else dx = make({n, dim}, dy.scalar_type(), dy);
    if (!dweight.defined()) dweight = make({dim}, dbias.defined() ? dbias.scalar_type() : type_of(dtype), dy);
    if (!dbias.defined() && bias) dbias = make({dim}, dweight.scalar_type(), dy);
    const lc_rows rdx = rows_of(dx, "dx");
    void* pw = param_of(dweight, dim, "dweight");
    void* pb = dbias.defined() ? param_of(dbias, dim, "dbias") : nullptr;
    if (pb && dbias.scalar_type() != dweight.scalar_type()) throw ValueError("dweight and dbias must have one type");
    void* stream = stream_of(index);
    const uint64_t need = lc_norm_grad_workspace(n, dim);
    const Scratch scratch(dy, index, stream, need);
    check(lc_norm_grad(index, stream, mean.defined() ? LC_NORM_LAYER : LC_NORM_RMS, &rd, q.defined() ? nullptr : &rx,
                       q.defined() ? &kept : nullptr, n, dim, w, code_of(weight, "weight"), m, r, &rdx, pw, pb,
                       code_of(dweight, "dweight"), accumulate, scratch.p, need));
    for (const at::Tensor* t : {&dx, &dweight, &dbias}) written(*t);
    return tuple(dx, dweight, dbias);
}

PyObject* weight_grad(PyObject* const* args, Py_ssize_t nargs) {
    Args a(args, nargs, 7);
    const at::Tensor dy = a.tensor(), q = a.tensor(), e = a.tensor();
    const int64_t dim = a.integer();
    at::Tensor grad = a.tensor();
    const int64_t dtype = a.integer();
    const bool accumulate = a.truth();
    const int index = cuda_index(dy);
    for (const at::Tensor* t : {&q, &e, static_cast<const at::Tensor*>(&grad)}) same_device(index, *t);
    const lc_rows rd = rows_of(dy, "dy");
    const int64_t n = dy.size(0), rows = dy.size(1);
    const lc_act act = act_of(q, e, n, dim);
    if (grad.defined()) {
        shaped(grad, rows, dim, "grad");
    } else {
        if (accumulate) throw ValueError("accumulate needs grad");
        grad = make({rows, dim}, type_of(dtype), dy);
    }
    const lc_rows rg = rows_of(grad, "grad");
    void* stream = stream_of(index);
    const uint64_t need = lc_weight_grad_workspace_of(&rd, n, rows, dim);
    const Scratch scratch(dy, index, stream, need);
    check(lc_weight_grad(index, stream, &rd, &act, n, rows, dim, &rg, accumulate, scratch.p, need));
    written(grad);
    return wrapped(grad);
}

PyObject* set_errors(PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 2) throw TypeError("wrong number of arguments");
    Py_INCREF(args[0]);
    Py_XSETREF(g_error, args[0]);
    Py_INCREF(args[1]);
    Py_XSETREF(g_memory, args[1]);
    Py_RETURN_NONE;
}

// No C++ exception leaves a call.
template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    try {
        return F(args, nargs);
    } catch (const StatusError& e) {
        PyObject* err = g_error ? PyObject_CallFunction(g_error, "is", int(e.status), lc_last_error()) : nullptr;
        if (err) {
            PyErr_SetObject(g_error, err);
            Py_DECREF(err);
        } else if (!PyErr_Occurred()) {
            PyErr_SetString(PyExc_RuntimeError, lc_last_error());
        }
    } catch (const TypeError& e) {
        PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const ValueError& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Raised&) {
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(g_memory ? g_memory : PyExc_MemoryError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

#define LC_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {LC_METHOD(embed),    LC_METHOD(embed_grad), LC_METHOD(act_save),    LC_METHOD(act_load), LC_METHOD(new_act),
                         LC_METHOD(norm),     LC_METHOD(norm_grad),  LC_METHOD(weight_grad), LC_METHOD(set_errors),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops() { return PyModule_Create(&module); }
