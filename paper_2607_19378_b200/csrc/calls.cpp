// The classes Recurrence, DeltaRule, Heads, Block and Dropout from Python to the C ABI: checks of the tensors, outputs from the caching allocator, the
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

// ---- delta rule -----------------------------------------------------------------------------------------------------

struct Delta {
    int B, H, Hk, L, Dk, Dv, decay, dtype;
    int64_t work_forward, work_backward;
    ScalarType type;
    Shape keys, values, gates, states, marks, key, value, gate, batch;      // (of a sequence, of a token)
    decltype(&hyenand_delta_forward) forward;
    decltype(&hyenand_delta_backward) backward;
    decltype(&hyenand_delta_step) step;
    PyObject *raise_error;
};

PyObject *make_delta(PyObject *, PyObject *args)
{
    int B, H, Hk, L, Dk, Dv, decay, dtype;
    long long marks, wf, wb;
    unsigned long long f, b, st;
    PyObject *raise_error;
    if (!PyArg_ParseTuple(args, "iiiiiiLiiLLKKKO", &B, &H, &Hk, &L, &Dk, &Dv, &marks, &decay, &dtype, &wf, &wb, &f, &b, &st, &raise_error)) return nullptr;
    const int64_t kc = (int64_t)Hk * Dk, vc = (int64_t)H * Dv;
    auto *d = new Delta{B, H, Hk, L, Dk, Dv, decay, dtype, wf, wb, type_of(dtype), {B, kc, L}, {B, vc, L}, {B, H, L}, {B, H, Dv, Dk}, {B, H, marks},
                        {B, kc}, {B, vc}, {B, H}, {B}, (decltype(&hyenand_delta_forward))f, (decltype(&hyenand_delta_backward))b,
                        (decltype(&hyenand_delta_step))st, Py_NewRef(raise_error)};
    return PyCapsule_New(d, nullptr, release<Delta>);
}
// g: a tensor where there is a decay, None where there is none
const Tensor *gate_of(Arguments &want, PyObject *o, const Delta *d, const Shape &shape)
{
    if (d->decay != HYENAND_DECAY_NONE) return want(o, "g", at::kFloat, shape);
    if (o != Py_None) { PyErr_SetString(PyExc_ValueError, "g must be None where there is no decay"); throw PythonError(); }
    return nullptr;
}

// handle, q, k, v, g, beta, s0, lengths, marks, y
PyObject *delta_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 10)) return nullptr;
    return guarded([&] {
        const Delta *d = handle<Delta>(a[0]);
        Arguments want;
        const Tensor *q = want(a[1], "q", d->type, d->keys), *k = want(a[2], "k", d->type, d->keys), *v = want(a[3], "v", d->type, d->values),
                     *g = gate_of(want, a[4], d, d->gates), *beta = want(a[5], "beta", at::kFloat, d->gates), *s0 = want(a[6], "s0", at::kFloat, d->states, true),
                     *len = want(a[7], "lengths", at::kInt, d->batch, true), *given = want(a[9], "y", d->type, d->values, true);
        const bool keep = truth(a[8]);
        const Tensor y = given ? *given : want.empty(d->values, d->type), end = want.empty(d->states, at::kFloat),
                     marks = keep ? want.empty(d->marks, at::kFloat) : Tensor(), work = want.empty({d->work_forward}, at::kByte);
        check(d->forward(d->B, d->H, d->Hk, d->L, d->Dk, d->Dv, d->decay, d->dtype, data(q), data(k), data(v), (const float *)data(g), (const float *)data(beta),
                         (const float *)data(s0), (const int *)data(len), y.data_ptr(), (float *)end.data_ptr(), keep ? (float *)marks.data_ptr() : nullptr,
                         work.data_ptr(), want.stream()), d->raise_error);
        return keep ? tuple({y, end, marks}) : tuple({y, end});
    });
}

// handle, q, k, v, g, beta, marks, dy, ds_end, lengths
PyObject *delta_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 10)) return nullptr;
    return guarded([&] {
        const Delta *d = handle<Delta>(a[0]);
        Arguments want;
        const Tensor *q = want(a[1], "q", d->type, d->keys), *k = want(a[2], "k", d->type, d->keys), *v = want(a[3], "v", d->type, d->values),
                     *g = gate_of(want, a[4], d, d->gates), *beta = want(a[5], "beta", at::kFloat, d->gates), *marks = want(a[6], "marks", at::kFloat, d->marks),
                     *dy = want(a[7], "dy", d->type, d->values), *ds = want(a[8], "ds_end", at::kFloat, d->states, true),
                     *len = want(a[9], "lengths", at::kInt, d->batch, true);
        const Tensor dq = want.empty(d->keys, d->type), dk = want.empty(d->keys, d->type), dv = want.empty(d->values, d->type),
                     dg = g ? want.empty(d->gates, at::kFloat) : Tensor(), dbeta = want.empty(d->gates, at::kFloat), ds0 = want.empty(d->states, at::kFloat),
                     work = want.empty({d->work_backward}, at::kByte);
        check(d->backward(d->B, d->H, d->Hk, d->L, d->Dk, d->Dv, d->decay, d->dtype, data(q), data(k), data(v), (const float *)data(g), (const float *)data(beta),
                          (const int *)data(len), (const float *)data(marks), data(dy), (const float *)data(ds), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                          g ? (float *)dg.data_ptr() : nullptr, (float *)dbeta.data_ptr(), (float *)ds0.data_ptr(), work.data_ptr(), want.stream()), d->raise_error);
        return tuple({dq, dk, dv, dg, dbeta, ds0});
    });
}

// handle, q, k, v, g, beta, state, new_state, active, y
PyObject *delta_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 10)) return nullptr;
    return guarded([&] {
        const Delta *d = handle<Delta>(a[0]);
        Arguments want;
        const Tensor *q = want(a[1], "q", d->type, d->key), *k = want(a[2], "k", d->type, d->key), *v = want(a[3], "v", d->type, d->value),
                     *g = gate_of(want, a[4], d, d->gate), *beta = want(a[5], "beta", at::kFloat, d->gate), *state = want(a[6], "state", at::kFloat, d->states),
                     *next = want(a[7], "new_state", at::kFloat, d->states, true), *active = want(a[8], "active", at::kInt, d->batch, true),
                     *given = want(a[9], "y", d->type, d->value, true);
        const Tensor y = given ? *given : want.empty(d->value, d->type);
        check(d->step(d->B, d->H, d->Hk, d->Dk, d->Dv, d->decay, d->dtype, data(q), data(k), data(v), (const float *)data(g), (const float *)data(beta),
                      (const float *)data(state), (const int *)data(active), y.data_ptr(), (float *)data(next ? next : state), want.stream()), d->raise_error);
        return wrap(y);
    });
}

// ---- heads ----------------------------------------------------------------------------------------------------------

struct Heads {
    int ndim, dims[3], axes[3], B, Hq, Hk, D, dtype, norm;
    double base;
    float eps;
    int64_t workspace;
    ScalarType type;
    Shape queries, keys, weights, places;
    decltype(&hyenand_heads_forward) forward;
    decltype(&hyenand_heads_backward) backward;
    PyObject *raise_error;
};

PyObject *make_heads(PyObject *, PyObject *args)
{
    PyObject *dims, *axes, *raise_error;
    int B, Hq, Hk, D, dtype, norm;
    double base;
    float eps;
    long long workspace;
    unsigned long long f, b;
    if (!PyArg_ParseTuple(args, "O!O!iiiiiidfLKKO", &PyTuple_Type, &dims, &PyTuple_Type, &axes, &B, &Hq, &Hk, &D, &dtype, &norm, &base, &eps, &workspace, &f, &b, &raise_error))
        return nullptr;
    auto *h = new Heads{(int)PyTuple_GET_SIZE(dims), {0}, {0}, B, Hq, Hk, D, dtype, norm, base, eps, workspace, type_of(dtype), {B, (int64_t)Hq * D}, {B, (int64_t)Hk * D}, {D},
                        {B, (int64_t)PyTuple_GET_SIZE(dims)}, (decltype(&hyenand_heads_forward))f, (decltype(&hyenand_heads_backward))b, Py_NewRef(raise_error)};
    for (int i = 0; i < h->ndim && i < 3; ++i) {
        h->dims[i] = (int)PyLong_AsLong(PyTuple_GET_ITEM(dims, i));
        h->axes[i] = (int)PyLong_AsLong(PyTuple_GET_ITEM(axes, i));
        h->queries.push_back(h->dims[i]);
        h->keys.push_back(h->dims[i]);
        h->places.push_back(h->dims[i]);
    }
    PyObject *c = PyCapsule_New(h, nullptr, release<Heads>);
    if (PyErr_Occurred()) { Py_XDECREF(c); return nullptr; }
    return c;
}

// handle, q, k, g_q, g_k, positions, q_out, k_out
PyObject *heads_forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 8)) return nullptr;
    return guarded([&] {
        const Heads *h = handle<Heads>(a[0]);
        Arguments want;
        const Tensor *q = want(a[1], "q", h->type, h->queries), *k = want(a[2], "k", h->type, h->keys), *gq = want(a[3], "g_q", at::kFloat, h->weights, true),
                     *gk = want(a[4], "g_k", at::kFloat, h->weights, true), *pos = want(a[5], "positions", at::kInt, h->places, true),
                     *oq = want(a[6], "q_out", h->type, h->queries, true), *ok = want(a[7], "k_out", h->type, h->keys, true);
        const Tensor yq = oq ? *oq : want.empty(h->queries, h->type), yk = ok ? *ok : want.empty(h->keys, h->type);
        check(h->forward(h->ndim, h->dims, h->B, h->Hq, h->Hk, h->D, h->dtype, h->norm, h->axes, h->base, h->eps, data(q), data(k), (const float *)data(gq),
                         (const float *)data(gk), (const int *)data(pos), yq.data_ptr(), yk.data_ptr(), want.stream()), h->raise_error);
        return tuple({yq, yk});
    });
}

// handle, q, k, dq_out, dk_out, g_q, g_k, positions
PyObject *heads_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!count(n, 8)) return nullptr;
    return guarded([&] {
        const Heads *h = handle<Heads>(a[0]);
        Arguments want;
        const Tensor *q = want(a[1], "q", h->type, h->queries), *k = want(a[2], "k", h->type, h->keys), *yq = want(a[3], "dq_out", h->type, h->queries),
                     *yk = want(a[4], "dk_out", h->type, h->keys), *gq = want(a[5], "g_q", at::kFloat, h->weights, true),
                     *gk = want(a[6], "g_k", at::kFloat, h->weights, true), *pos = want(a[7], "positions", at::kInt, h->places, true);
        const Tensor dq = want.empty(h->queries, h->type), dk = want.empty(h->keys, h->type), dgq = gq ? want.empty(h->weights, at::kFloat) : Tensor(),
                     dgk = gk ? want.empty(h->weights, at::kFloat) : Tensor(), work = gq || gk ? want.empty({h->workspace}, at::kByte) : Tensor();
        check(h->backward(h->ndim, h->dims, h->B, h->Hq, h->Hk, h->D, h->dtype, h->norm, h->axes, h->base, h->eps, data(q), data(k), (const float *)data(gq),
                          (const float *)data(gk), (const int *)data(pos), data(yq), data(yk), dq.data_ptr(), dk.data_ptr(), gq ? (float *)dgq.data_ptr() : nullptr,
                          gk ? (float *)dgk.data_ptr() : nullptr, gq || gk ? work.data_ptr() : nullptr, want.stream()), h->raise_error);
        return tuple({dq, dk, dgq, dgk});
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
    {"make_delta", make_delta, METH_VARARGS, nullptr},
    {"delta_forward", (PyCFunction)(void (*)(void))delta_forward, METH_FASTCALL, nullptr},
    {"delta_backward", (PyCFunction)(void (*)(void))delta_backward, METH_FASTCALL, nullptr},
    {"delta_step", (PyCFunction)(void (*)(void))delta_step, METH_FASTCALL, nullptr},
    {"make_heads", make_heads, METH_VARARGS, nullptr},
    {"heads_forward", (PyCFunction)(void (*)(void))heads_forward, METH_FASTCALL, nullptr},
    {"heads_backward", (PyCFunction)(void (*)(void))heads_backward, METH_FASTCALL, nullptr},
    {"dropout", (PyCFunction)(void (*)(void))dropout, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Recurrence, DeltaRule, Heads, Block and Dropout: from tensors to the C ABI", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
