// The classes Recurrence, Block and Dropout from Python to the C ABI: checks of the tensors, outputs from the caching allocator, the
// current stream, one call of the library.  As Python this takes longer than the kernels of small calls (a token for 32 sequences of
// 768 channels 11.4 us a call, the kernel 3; here 5.3); nothing is computed here.  The library's functions come as addresses, so that
// one module serves the product library and the checked build.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/hyenand.h"

namespace {

using at::ScalarType;
using at::Tensor;
using Shape = std::vector<int64_t>;

struct PythonError : std::exception {};                      // the interpreter's error is set

struct Arguments {
    int device = -1;
    // None: a null pointer where that is allowed
    const Tensor *operator()(PyObject *o, const char *name, ScalarType type, c10::IntArrayRef shape, bool optional = false)
    {
        if (o == Py_None && optional) return nullptr;
        if (!THPVariable_Check(o)) {
            PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
            throw PythonError();
        }
        const Tensor &t = THPVariable_Unpack(o);
        bool good = t.is_cuda() && t.scalar_type() == type && t.sizes() == shape && t.is_contiguous();
        if (good) {
            if (device < 0) device = c10::cuda::current_device();
            good = t.get_device() == device;
        }
        if (!good) {
            std::string s;
            for (int64_t d : shape) s += (s.empty() ? "" : ", ") + std::to_string(d);
            const char *kind = type == at::kBFloat16 ? "torch.bfloat16" : type == at::kFloat ? "torch.float32" : type == at::kInt ? "torch.int32" : "torch.int64";
            PyErr_Format(PyExc_ValueError, "%s must be a contiguous %s tensor of shape (%s) on the current CUDA device", name, kind, s.c_str());
            throw PythonError();
        }
        return &t;
    }
    Tensor empty(c10::IntArrayRef shape, ScalarType type) const
    {
        return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, (c10::DeviceIndex)device), std::nullopt);
    }
    void *stream() const { return (void *)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
};

bool truth(PyObject *o)
{
    const int t = PyObject_IsTrue(o);
    if (t < 0) throw PythonError();
    return t == 1;
}
void *data(const Tensor *t) { return t ? t->data_ptr() : nullptr; }
PyObject *wrap(const Tensor &t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }
PyObject *tuple(std::initializer_list<Tensor> ts)
{
    PyObject *r = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const Tensor &t : ts) PyTuple_SET_ITEM(r, i++, wrap(t));
    return r;
}

// `raise_error` is the Python function that turns a code into the library's exception
void check(int code, PyObject *raise_error)
{
    if (code == HYENAND_OK) return;
    Py_XDECREF(PyObject_CallFunction(raise_error, "i", code));
    if (!PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "hyenand error %d", code);
    throw PythonError();
}

template <typename F> PyObject *guarded(F f)
{
    try {
        return f();
    } catch (const PythonError &) {
        return nullptr;
    } catch (...) {                                          // (as torch's own calls raise it: an allocation that fails is OutOfMemoryError)
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    }
}

bool count(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, n);
    return false;
}

ScalarType type_of(int dtype) { return dtype == HYENAND_F32 ? at::kFloat : at::kBFloat16; }

// ---- recurrence -----------------------------------------------------------------------------------------------------

struct Recurrence {
    int B, C, L, decay, dtype;
    int64_t workspace;
    ScalarType type;
    Shape shape, states, marks, batch;
    decltype(&hyenand_recurrence_forward) forward;
    decltype(&hyenand_recurrence_backward) backward;
    decltype(&hyenand_recurrence_step) step;
    PyObject *raise_error;
};
template <typename S> S *handle(PyObject *o)
{
    S *s = (S *)PyCapsule_GetPointer(o, nullptr);
    if (!s) throw PythonError();
    return s;
}
template <typename S> void release(PyObject *o)
{
    S *s = (S *)PyCapsule_GetPointer(o, nullptr);
    if (s) { Py_DECREF(s->raise_error); delete s; }
}

PyObject *make_recurrence(PyObject *, PyObject *args)
{
    int B, C, L, marks, decay, dtype;
    long long workspace;
    unsigned long long f, b, st;
    PyObject *raise_error;
    if (!PyArg_ParseTuple(args, "iiiiiiLKKKO", &B, &C, &L, &marks, &decay, &dtype, &workspace, &f, &b, &st, &raise_error)) return nullptr;
    auto *r = new Recurrence{B, C, L, decay, dtype, workspace, type_of(dtype), {B, C, L}, {B, C}, {B, C, marks}, {B}, (decltype(&hyenand_recurrence_forward))f,
                             (decltype(&hyenand_recurrence_backward))b, (decltype(&hyenand_recurrence_step))st, Py_NewRef(raise_error)};
    return PyCapsule_New(r, nullptr, release<Recurrence>);
}

// handle, q, k, v, g, s0, lengths, marks, y
PyObject *recurrence_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 9)) return nullptr;
    return guarded([&] {
        const Recurrence *r = handle<Recurrence>(a[0]);
        Arguments want;
        const Tensor *q = want(a[1], "q", r->type, r->shape), *k = want(a[2], "k", r->type, r->shape), *v = want(a[3], "v", r->type, r->shape),
                     *g = want(a[4], "g", r->type, r->shape), *s0 = want(a[5], "s0", at::kFloat, r->states, true),
                     *len = want(a[6], "lengths", at::kInt, r->batch, true), *given = want(a[8], "y", r->type, r->shape, true);
        const Tensor y = given ? *given : want.empty(r->shape, r->type), end = want.empty(r->states, at::kFloat);
        const bool keep = truth(a[7]);
        const Tensor marks = keep ? want.empty(r->marks, at::kFloat) : Tensor(), work = r->workspace ? want.empty({r->workspace}, at::kByte) : Tensor();
        check(r->forward(r->B, r->C, r->L, r->decay, r->dtype, data(q), data(k), data(v), data(g), (const float *)data(s0), (const int *)data(len),
                         y.data_ptr(), (float *)end.data_ptr(), keep ? (float *)marks.data_ptr() : nullptr, r->workspace ? work.data_ptr() : nullptr, want.stream()), r->raise_error);
        return keep ? tuple({y, end, marks}) : tuple({y, end});
    });
}

// handle, q, k, v, g, marks, dy, ds_end, lengths
PyObject *recurrence_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 9)) return nullptr;
    return guarded([&] {
        const Recurrence *r = handle<Recurrence>(a[0]);
        Arguments want;
        const Tensor *q = want(a[1], "q", r->type, r->shape), *k = want(a[2], "k", r->type, r->shape), *v = want(a[3], "v", r->type, r->shape),
                     *g = want(a[4], "g", r->type, r->shape), *marks = want(a[5], "marks", at::kFloat, r->marks), *dy = want(a[6], "dy", r->type, r->shape),
                     *ds = want(a[7], "ds_end", at::kFloat, r->states, true), *len = want(a[8], "lengths", at::kInt, r->batch, true);
        Tensor o[4];
        for (Tensor &t : o) t = want.empty(r->shape, r->type);
        const Tensor ds0 = want.empty(r->states, at::kFloat), work = r->workspace ? want.empty({r->workspace}, at::kByte) : Tensor();
        check(r->backward(r->B, r->C, r->L, r->decay, r->dtype, data(q), data(k), data(v), data(g), (const int *)data(len), (const float *)data(marks),
                          data(dy), (const float *)data(ds), o[0].data_ptr(), o[1].data_ptr(), o[2].data_ptr(), o[3].data_ptr(),
                          (float *)ds0.data_ptr(), r->workspace ? work.data_ptr() : nullptr, want.stream()), r->raise_error);
        return tuple({o[0], o[1], o[2], o[3], ds0});
    });
}

// handle, q, k, v, g, state, new_state, active, y
PyObject *recurrence_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 9)) return nullptr;
    return guarded([&] {
        const Recurrence *r = handle<Recurrence>(a[0]);
        Arguments want;
        const Tensor *q = want(a[1], "q", r->type, r->states), *k = want(a[2], "k", r->type, r->states), *v = want(a[3], "v", r->type, r->states),
                     *g = want(a[4], "g", r->type, r->states), *state = want(a[5], "state", at::kFloat, r->states),
                     *next = want(a[6], "new_state", at::kFloat, r->states, true), *active = want(a[7], "active", at::kInt, r->batch, true),
                     *given = want(a[8], "y", r->type, r->states, true);
        const Tensor y = given ? *given : want.empty(r->states, r->type);
        check(r->step(r->B, r->C, r->decay, r->dtype, data(q), data(k), data(v), data(g), (const float *)data(state), (const int *)data(active),
                      y.data_ptr(), (float *)data(next ? next : state), want.stream()), r->raise_error);
        return wrap(y);
    });
}

// ---- block ----------------------------------------------------------------------------------------------------------

struct Block {
    int B, C, T, dtype, gate, site;
    float eps, p;
    int64_t workspace;
    ScalarType type;
    Shape shape, stats, channels;
    decltype(&hyenand_block_forward) forward;
    decltype(&hyenand_block_backward) backward;
    PyObject *raise_error;
};
const Shape kTwo = {2};

PyObject *make_block(PyObject *, PyObject *args)
{
    int B, C, T, dtype, gate, site;
    float eps, p;
    long long workspace;
    unsigned long long f, b;
    PyObject *dims, *raise_error;
    if (!PyArg_ParseTuple(args, "O!iiiiiffiLKKO", &PyTuple_Type, &dims, &B, &C, &T, &dtype, &gate, &eps, &p, &site, &workspace, &f, &b, &raise_error)) return nullptr;
    Shape shape = {B, C};
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(dims); ++i) shape.push_back(PyLong_AsLongLong(PyTuple_GET_ITEM(dims, i)));
    if (PyErr_Occurred()) return nullptr;
    auto *r = new Block{B, C, T, dtype, gate, site, eps, p, workspace, type_of(dtype), shape, {2, B, T}, {C}, (decltype(&hyenand_block_forward))f,
                        (decltype(&hyenand_block_backward))b, Py_NewRef(raise_error)};
    return PyCapsule_New(r, nullptr, release<Block>);
}

// handle, x, m, z, g_post, scale, g_pre, rng, stats
PyObject *block_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 9)) return nullptr;
    return guarded([&] {
        const Block *b = handle<Block>(a[0]);
        Arguments want;
        const Tensor *x = want(a[1], "x", b->type, b->shape), *m = want(a[2], "m", b->type, b->shape), *z = want(a[3], "z", b->type, b->shape, true),
                     *gp = want(a[4], "g_post", at::kFloat, b->channels, true), *sc = want(a[5], "scale", at::kFloat, b->channels, true),
                     *gn = want(a[6], "g_pre", at::kFloat, b->channels, true), *rng = want(a[7], "rng", at::kLong, kTwo, true);
        const bool keep = truth(a[8]);
        const Tensor r = want.empty(b->shape, b->type), nn = gn ? want.empty(b->shape, b->type) : Tensor(),
                     st = keep ? want.empty(b->stats, at::kFloat) : Tensor();
        check(b->forward(b->B, b->C, b->T, b->dtype, data(x), data(m), data(z), (const float *)data(gp), (const float *)data(sc), (const float *)data(gn),
                         b->eps, b->gate, b->p, (const long long *)data(rng), b->site, r.data_ptr(), gn ? nn.data_ptr() : nullptr,
                         keep ? (float *)st.data_ptr() : nullptr, want.stream()), b->raise_error);
        return keep ? tuple({r, nn, st}) : tuple({r, nn});
    });
}

// handle, x, m, stats, z, g_post, scale, g_pre, rng, dr, dn
PyObject *block_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 11)) return nullptr;
    return guarded([&] {
        const Block *b = handle<Block>(a[0]);
        Arguments want;
        const Tensor *x = want(a[1], "x", b->type, b->shape), *m = want(a[2], "m", b->type, b->shape), *st = want(a[3], "stats", at::kFloat, b->stats, true),
                     *z = want(a[4], "z", b->type, b->shape, true), *gp = want(a[5], "g_post", at::kFloat, b->channels, true),
                     *sc = want(a[6], "scale", at::kFloat, b->channels, true), *gn = want(a[7], "g_pre", at::kFloat, b->channels, true),
                     *rng = want(a[8], "rng", at::kLong, kTwo, true), *dr = want(a[9], "dr", b->type, b->shape, true),
                     *dn = want(a[10], "dn", b->type, b->shape, true);
        const Tensor dx = want.empty(b->shape, b->type), dm = want.empty(b->shape, b->type), dz = z ? want.empty(b->shape, b->type) : Tensor(),
                     dgp = gp ? want.empty(b->channels, at::kFloat) : Tensor(), dsc = sc ? want.empty(b->channels, at::kFloat) : Tensor(),
                     dgn = gn ? want.empty(b->channels, at::kFloat) : Tensor(), work = want.empty({b->workspace}, at::kByte);
        check(b->backward(b->B, b->C, b->T, b->dtype, data(x), data(m), data(z), (const float *)data(gp), (const float *)data(sc), (const float *)data(gn),
                          b->eps, b->gate, b->p, (const long long *)data(rng), b->site, (const float *)data(st), data(dr), data(dn), dx.data_ptr(),
                          dm.data_ptr(), z ? dz.data_ptr() : nullptr, gp ? (float *)dgp.data_ptr() : nullptr, sc ? (float *)dsc.data_ptr() : nullptr,
                          gn ? (float *)dgn.data_ptr() : nullptr, work.data_ptr(), want.stream()), b->raise_error);
        return tuple({dx, dm, dz, dgp, dsc, dgn});
    });
}

// ---- dropout --------------------------------------------------------------------------------------------------------

// address of hyenand_dropout, function that raises, p, site, x, rng, y
PyObject *dropout(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 7)) return nullptr;
    return guarded([&] {
        if (!THPVariable_Check(a[4])) { PyErr_SetString(PyExc_TypeError, "x must be a tensor"); throw PythonError(); }
        const ScalarType type = THPVariable_Unpack(a[4]).scalar_type();
        if (type != at::kFloat && type != at::kBFloat16) { PyErr_SetString(PyExc_ValueError, "x must be a float32 or bfloat16 tensor"); throw PythonError(); }
        Arguments want;
        const c10::IntArrayRef shape = THPVariable_Unpack(a[4]).sizes();
        const Tensor *x = want(a[4], "x", type, shape), *rng = want(a[5], "rng", at::kLong, kTwo), *given = want(a[6], "y", type, shape, true);
        const auto f = (decltype(&hyenand_dropout))PyLong_AsUnsignedLongLong(a[0]);
        const float p = (float)PyFloat_AsDouble(a[2]);
        const int site = (int)PyLong_AsLong(a[3]);
        if (PyErr_Occurred()) throw PythonError();
        const Tensor y = given ? *given : want.empty(shape, type);
        if (x->numel())
            check(f(x->numel(), type == at::kFloat ? HYENAND_F32 : HYENAND_BF16, x->data_ptr(), p, (const long long *)rng->data_ptr(), site, y.data_ptr(),
                    want.stream()), a[1]);
        return given ? Py_NewRef(a[6]) : wrap(y);
    });
}

PyMethodDef methods[] = {
    {"make_recurrence", make_recurrence, METH_VARARGS, nullptr},
    {"recurrence_forward", (PyCFunction)(void (*)(void))recurrence_forward, METH_FASTCALL, nullptr},
    {"recurrence_backward", (PyCFunction)(void (*)(void))recurrence_backward, METH_FASTCALL, nullptr},
    {"recurrence_step", (PyCFunction)(void (*)(void))recurrence_step, METH_FASTCALL, nullptr},
    {"make_block", make_block, METH_VARARGS, nullptr},
    {"block_forward", (PyCFunction)(void (*)(void))block_forward, METH_FASTCALL, nullptr},
    {"block_backward", (PyCFunction)(void (*)(void))block_backward, METH_FASTCALL, nullptr},
    {"dropout", (PyCFunction)(void (*)(void))dropout, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Recurrence, Block and Dropout: from tensors to the C ABI", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
