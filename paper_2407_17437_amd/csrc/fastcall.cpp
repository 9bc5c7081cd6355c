// The calls that a training or inference loop makes, from Python objects to the C ABI in one step.
// Through ctypes a call spends as much on its arguments as the library does on a launch -- data_ptr() and three properties of
// every tensor, each a Python call, then the conversions: 1.8 us for sparse_linear_forward, 3.3 for
// sparse_linear_backward (with an empty function in the place of either), 0.14 and 0.15 here.  The entry points come as addresses from the library that the
// package has loaded (bind), so that there is one copy of it in the process.  Every call releases the interpreter lock and returns the
// status code.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <vector>

namespace {

using Forward = int (*)(const void *, const float *, int32_t, float *, int32_t, int32_t, void *);
using Backward = int (*)(void *, const float *, int32_t, const float *, int32_t, const float *, int32_t, float *, int32_t, float *, float *,
                         int32_t, void *);
using Update = int (*)(float *, float *, const float *, int64_t, float, float, void *);
using TrainStep = int (*)(void *, const float *, int32_t, const int32_t *, int32_t, float, float, void *, size_t, float *, void *);
using MlpForward = int (*)(void *, const float *, int32_t, int32_t, void *, size_t, void *);

Forward g_forward;
Backward g_backward;
Update g_update, g_update_nesterov;
TrainStep g_train_step;
MlpForward g_mlp_forward;

// Reads the arguments of one call in order; the first that cannot be read leaves a Python exception and `ok` false.
struct Args {
    PyObject *const *v;
    bool ok = true;

    int64_t integer()
    {
        PyObject *o = *v++;
        if (!ok) return 0;
        const long long x = PyLong_AsLongLong(o);
        if (x == -1 && PyErr_Occurred()) ok = false;
        return x;
    }
    float real()
    {
        PyObject *o = *v++;
        if (!ok) return 0.f;
        const double x = PyFloat_AsDouble(o);
        if (x == -1.0 && PyErr_Occurred()) ok = false;
        return static_cast<float>(x);
    }
    // a handle or address as an int, or None
    void *address()
    {
        PyObject *o = *v++;
        if (!ok || o == Py_None) return nullptr;
        void *p = PyLong_AsVoidPtr(o);
        if (!p && PyErr_Occurred()) ok = false;
        return p;
    }
    const at::Tensor *tensor(PyObject *o)
    {
        if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
        PyErr_SetString(PyExc_TypeError, "expected a tensor");
        ok = false;
        return nullptr;
    }
    // a tensor's memory, or None
    void *memory()
    {
        PyObject *o = *v++;
        if (!ok || o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o);
        return t ? t->data_ptr() : nullptr;
    }
    // the same, or an address as an int
    void *memory_or_address()
    {
        if (PyLong_Check(*v)) return address();
        return memory();
    }
    void *buffer(size_t &bytes)
    {
        PyObject *o = *v++;
        bytes = 0;
        const at::Tensor *t = ok ? tensor(o) : nullptr;
        if (!t) return nullptr;
        bytes = t->nbytes();
        return t->data_ptr();
    }
    // a float32 matrix with unit column stride and its leading dimension, or None
    float *matrix(int32_t &ld)
    {
        PyObject *o = *v++;
        ld = 0;
        if (!ok || o == Py_None) return nullptr;
        const at::Tensor *t = tensor(o);
        if (!t) return nullptr;
        if (t->dim() != 2 || t->stride(1) != 1 || t->scalar_type() != at::kFloat) {
            PyErr_SetString(PyExc_AssertionError, "expected a float32 matrix with contiguous rows");
            ok = false;
            return nullptr;
        }
        ld = static_cast<int32_t>(t->stride(0));
        return static_cast<float *>(t->data_ptr());
    }
    // a matrix, or an address, followed by its leading dimension: None takes the matrix's own
    float *matrix_with_ld(int32_t &ld)
    {
        if (v[1] == Py_None) {
            float *p = matrix(ld);
            ++v;
            return p;
        }
        float *p = static_cast<float *>(memory_or_address());
        ld = static_cast<int32_t>(integer());
        return p;
    }
    // None: torch's current stream; a torch stream; or a handle
    void *stream()
    {
        PyObject *o = *v++;
        if (!ok) return nullptr;
        if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
        if (PyLong_Check(o)) return PyLong_AsVoidPtr(o);
        PyObject *h = PyObject_GetAttrString(o, "cuda_stream");
        if (!h) {
            ok = false;
            return nullptr;
        }
        void *s = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
        if (!s && PyErr_Occurred()) ok = false;
        return s;
    }
};

// Runs `call`, which reads its arguments and returns a closure for the library call.
template <typename F>
PyObject *run(PyObject *const *args, Py_ssize_t n, Py_ssize_t expected, F &&read)
{
    if (n != expected) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, expected);
        return nullptr;
    }
    try {
        Args a{args};
        auto call = read(a);
        if (!a.ok) return nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = call();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (layer, X, Y, batch, stream)
PyObject *forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run(args, n, 5, [](Args &a) {
        int32_t ldx, ldy;
        const void *layer = a.address();
        const float *X = a.matrix(ldx);
        float *Y = a.matrix(ldy);
        const int32_t batch = static_cast<int32_t>(a.integer());
        void *s = a.stream();
        return [=] { return g_forward(layer, X, ldx, Y, ldy, batch, s); };
    });
}

// (layer, X, Y, dY, dX, dvalues, dbias, batch, stream)
PyObject *backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run(args, n, 9, [](Args &a) {
        int32_t ldx, ldy, lddy, lddx;
        void *layer = a.address();
        const float *X = a.matrix(ldx), *Y = a.matrix(ldy), *dY = a.matrix(lddy);
        float *dX = a.matrix(lddx), *dv = static_cast<float *>(a.memory()), *db = static_cast<float *>(a.memory());
        const int32_t batch = static_cast<int32_t>(a.integer());
        void *s = a.stream();
        return [=] { return g_backward(layer, X, ldx, Y, ldy, dY, lddy, dX, lddx, dv, db, batch, s); };
    });
}

// (values, velocity, grad, n, lr, momentum, nesterov, stream)
PyObject *update(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run(args, n, 8, [](Args &a) {
        float *w = static_cast<float *>(a.memory()), *v = static_cast<float *>(a.memory());
        const float *g = static_cast<const float *>(a.memory());
        const int64_t count = a.integer();
        const float lr = a.real(), mu = a.real();
        const Update f = a.integer() ? g_update_nesterov : g_update;
        void *s = a.stream();
        return [=] { return f(w, v, g, count, lr, mu, s); };
    });
}

// (mlp, X, ldx, labels, batch, lr, momentum, workspace, loss, stream)
PyObject *train_step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run(args, n, 10, [](Args &a) {
        void *mlp = a.address();
        int32_t ldx;
        const float *X = a.matrix_with_ld(ldx);
        const int32_t *labels = static_cast<const int32_t *>(a.memory_or_address());
        const int32_t batch = static_cast<int32_t>(a.integer());
        const float lr = a.real(), mu = a.real();
        size_t bytes;
        void *ws = a.buffer(bytes);
        float *loss = static_cast<float *>(a.memory());
        void *s = a.stream();
        return [=] { return g_train_step(mlp, X, ldx, labels, batch, lr, mu, ws, bytes, loss, s); };
    });
}

// (mlp, X, ldx, batch, workspace, stream)
PyObject *mlp_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run(args, n, 6, [](Args &a) {
        void *mlp = a.address();
        int32_t ldx;
        const float *X = a.matrix_with_ld(ldx);
        const int32_t batch = static_cast<int32_t>(a.integer());
        size_t bytes;
        void *ws = a.buffer(bytes);
        void *s = a.stream();
        return [=] { return g_mlp_forward(mlp, X, ldx, batch, ws, bytes, s); };
    });
}

// (workspace, rows, batch, ld, offset in floats): the (rows, batch) matrix there
PyObject *view(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, 5 expected", n);
        return nullptr;
    }
    try {
        Args a{args + 1};
        const at::Tensor *ws = a.tensor(args[0]);
        const int64_t rows = a.integer(), batch = a.integer(), ld = a.integer(), offset = a.integer();
        if (!a.ok) return nullptr;
        return THPVariable_Wrap(ws->as_strided({rows, batch}, {ld, 1}, ws->storage_offset() + offset));
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// addresses of sparse_linear_forward, sparse_linear_backward, sgd_update_values, sgd_update_values_nesterov, mlp_train_step, mlp_forward
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "six addresses expected");
        return nullptr;
    }
    Args a{args};
    g_forward = reinterpret_cast<Forward>(a.address());
    g_backward = reinterpret_cast<Backward>(a.address());
    g_update = reinterpret_cast<Update>(a.address());
    g_update_nesterov = reinterpret_cast<Update>(a.address());
    g_train_step = reinterpret_cast<TrainStep>(a.address());
    g_mlp_forward = reinterpret_cast<MlpForward>(a.address());
    if (!a.ok) return nullptr;
    Py_RETURN_NONE;
}

// ---- mixtures and clipped gradients ------------------------------------------------------------
// These calls look at what they are given besides: types, shapes against the sizes of the call, and that every tensor lies on the current
// device, where the kernels run.

using Route = int (*)(const float *, int32_t, const float *, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, float, int32_t *, float *, int32_t, void *);
using RouteBackward = int (*)(const float *, int32_t, const int32_t *, const float *, int32_t, int32_t, int32_t, int32_t, int32_t, float, float *, int32_t, void *);
using Place = int (*)(const int32_t *, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t *, int32_t *, void *, size_t, void *);
using Dispatch = int (*)(const float *, int32_t, const void *, size_t, int32_t, int32_t, int32_t, int32_t, int32_t, float *, int32_t, void *);
using Combine = int (*)(const float *, int32_t, const void *, size_t, const float *, int32_t, int32_t, int32_t, int32_t, int32_t, int32_t, float *, int32_t, void *);
using CombineBackward = int (*)(const float *, int32_t, const float *, int32_t, const void *, size_t, const float *, int32_t, int32_t, int32_t, int32_t, int32_t,
                                int32_t, float *, float *, void *, size_t, void *);
using Norm = int (*)(int32_t, const float *const *, const int64_t *, void *, size_t, float *, void *);
using Clip = int (*)(int32_t, const float *const *, float *const *, const int64_t *, float, void *, size_t, float *, void *);
using UpdateClipped = int (*)(int32_t, float *const *, float *const *, const float *const *, const int64_t *, float, float, float, int32_t, void *, size_t, float *,
                              void *);

using NormForward = int (*)(const float *, int32_t, const float *, const float *, int32_t, int32_t, int32_t, float, int32_t, float, int32_t, const int64_t *, float *,
                            int32_t, float *, float *, int32_t, void *, size_t, void *);
using NormBackward = int (*)(const float *, int32_t, const float *, const float *, const float *, const float *, int32_t, const float *, int32_t, int32_t, int32_t,
                             int32_t, int32_t, float, int32_t, const int64_t *, float *, int32_t, float *, float *, void *, size_t, void *);
using Dropout = int (*)(const float *, int32_t, int32_t, int32_t, float, int32_t, const int64_t *, float *, int32_t, void *);
using LogProbs = int (*)(const float *, int32_t, const int32_t *, int32_t, int32_t, const int32_t *, int32_t, float *, float *, void *, size_t, void *);
using Policy = int (*)(const float *, int32_t, const int32_t *, const float *, const float *, const float *, const float *, int32_t, int32_t, float, float, float,
                       float *, int32_t, float *, float *, void *, size_t, void *);
using Preference = int (*)(const float *, int32_t, const int32_t *, const int32_t *, const float *, int32_t, int32_t, int32_t, float, float, float *, int32_t, float *,
                           float *, float *, void *, size_t, void *);

Route g_route;
RouteBackward g_route_backward;
Place g_place;
Dispatch g_dispatch;
Combine g_combine;
CombineBackward g_combine_backward;
Norm g_norm;
Clip g_clip;
UpdateClipped g_update_clipped;
NormForward g_norm_forward;
NormBackward g_norm_backward;
Dropout g_dropout;
LogProbs g_log_probs;
Policy g_policy;
Preference g_preference;

// Arguments by position; the first that does not fit leaves a Python exception and `ok` false.
struct Given {
    PyObject *const *v;
    int device = -1;   // the current one, once a tensor has asked for it
    bool ok = true;

    void refuse(const char *name, const char *what)
    {
        if (ok) PyErr_Format(PyExc_AssertionError, "%s: %s expected", name, what);
        ok = false;
    }
    int32_t integer(int i)
    {
        if (!ok) return 0;
        const long long x = PyLong_AsLongLong(v[i]);
        if (x == -1 && PyErr_Occurred()) ok = false;
        else if (x < INT32_MIN || x > INT32_MAX) {
            PyErr_Format(PyExc_OverflowError, "%lld does not fit 32 bits", x);
            ok = false;
        }
        return static_cast<int32_t>(x);
    }
    float real(int i)
    {
        if (!ok) return 0.f;
        const double x = PyFloat_AsDouble(v[i]);
        if (x == -1.0 && PyErr_Occurred()) ok = false;
        return static_cast<float>(x);
    }
    bool none(int i) const { return v[i] == Py_None; }
    // a tensor of this type on the current device
    const at::Tensor *tensor(PyObject *o, const char *name, at::ScalarType type)
    {
        if (!ok) return nullptr;
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_TypeError, "expected a tensor");
            ok = false;
            return nullptr;
        }
        const at::Tensor *t = &THPVariable_Unpack(o);
        if (t->scalar_type() != type) return refuse(name, type == at::kFloat ? "float32" : type == at::kInt ? "int32" : "int64"), nullptr;
        if (!t->is_cuda()) return refuse(name, "a tensor on the GPU"), nullptr;
        if (device < 0) device = c10::hip::current_device();
        if (t->get_device() != device) return refuse(name, "a tensor on the current device"), nullptr;
        return t;
    }
    // (rows, columns) at least, columns next to each other
    template <typename T>
    T *matrix(int i, const char *name, int64_t rows, int64_t columns, int32_t &ld, bool optional = false)
    {
        ld = 0;
        if (optional && none(i)) return nullptr;
        const at::Tensor *t = tensor(v[i], name, sizeof(T) == 4 && std::is_same_v<std::remove_const_t<T>, float> ? at::kFloat : at::kInt);
        if (!t) return nullptr;
        if (t->dim() != 2 || t->stride(1) != 1 || t->size(0) < rows || t->size(1) < columns) return refuse(name, "a matrix of the call's sizes with contiguous rows"), nullptr;
        const int64_t step = t->size(0) > 1 ? t->stride(0) : t->size(1);
        if (step < 0 || step > INT32_MAX) return refuse(name, "rows less than 2^31 entries apart"), nullptr;
        ld = static_cast<int32_t>(step);
        return static_cast<T *>(t->data_ptr());
    }
    // (experts, features, capacity): blocks of rows `ld` apart, one right behind the other
    float *blocks(int i, const char *name, int64_t experts, int64_t features, int64_t capacity, int32_t &ld, bool optional = false)
    {
        ld = 0;
        if (optional && none(i)) return nullptr;
        const at::Tensor *t = tensor(v[i], name, at::kFloat);
        if (!t) return nullptr;
        if (t->dim() != 3 || t->stride(2) != 1 || t->size(0) < experts || t->size(1) != features || t->size(2) < capacity)
            return refuse(name, "blocks (experts, features, capacity) with contiguous rows"), nullptr;
        const int64_t step = features > 1 ? t->stride(1) : t->size(0) > 1 ? t->stride(0) : t->size(2);
        if (step < 0 || step > INT32_MAX || (t->size(0) > 1 && t->stride(0) != features * step)) return refuse(name, "blocks right behind each other"), nullptr;
        ld = static_cast<int32_t>(step);
        return static_cast<float *>(t->data_ptr());
    }
    template <typename T>
    T *vector(int i, const char *name, int64_t n, bool optional = false)
    {
        if (optional && none(i)) return nullptr;
        const at::Tensor *t = tensor(v[i], name, std::is_same_v<T, float> ? at::kFloat : std::is_same_v<T, int64_t> ? at::kLong : at::kInt);
        if (!t) return nullptr;
        if (t->numel() < n || !t->is_contiguous()) return refuse(name, "a contiguous array of the call's size"), nullptr;
        return static_cast<T *>(t->data_ptr());
    }
    // scratch memory of any type
    void *scratch(int i, const char *name, size_t &bytes)
    {
        bytes = 0;
        if (!ok || none(i)) return nullptr;
        const at::Tensor *t = THPVariable_Check(v[i]) ? &THPVariable_Unpack(v[i]) : nullptr;
        t = tensor(v[i], name, t ? t->scalar_type() : at::kFloat);
        if (!t) return nullptr;
        if (!t->is_contiguous()) return refuse(name, "contiguous memory"), nullptr;
        bytes = t->nbytes();
        return t->data_ptr();
    }
    // a list or tuple of contiguous float32 arrays; counts: filled by the first list, compared by the others
    bool arrays(int i, const char *name, std::vector<float *> &p, std::vector<int64_t> &counts, bool first)
    {
        if (!ok) return false;
        if (!PyList_Check(v[i]) && !PyTuple_Check(v[i])) return refuse(name, "a list of tensors"), false;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(v[i]);
        if (!first && static_cast<size_t>(n) != counts.size()) return refuse(name, "as many tensors as gradients"), false;
        PyObject **items = PySequence_Fast_ITEMS(v[i]);
        p.resize(n);
        if (first) counts.resize(n);
        for (Py_ssize_t k = 0; k < n; ++k) {
            const at::Tensor *t = tensor(items[k], name, at::kFloat);
            if (!t) return false;
            if (!t->is_contiguous()) return refuse(name, "contiguous arrays"), false;
            if (first) counts[k] = t->numel();
            else if (counts[k] != t->numel()) return refuse(name, "arrays as long as the gradients"), false;
            p[k] = static_cast<float *>(t->data_ptr());
        }
        return true;
    }
    void *stream(int i)
    {
        if (!ok) return nullptr;
        Args a{v + i};
        void *s = a.stream();
        ok = a.ok;
        return s;
    }
};

template <typename F>
PyObject *run_given(PyObject *const *args, Py_ssize_t n, Py_ssize_t expected, F &&read)
{
    if (n != expected) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, expected);
        return nullptr;
    }
    try {
        Given a{args};
        auto call = read(a);
        if (!a.ok) return nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = call();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (Z, bias, experts, batch, k, groups, top_groups, flags, scale, chosen, weights, stream)
PyObject *route(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 12, [](Given &a) {
        const int32_t experts = a.integer(2), batch = a.integer(3), k = a.integer(4), groups = a.integer(5), top = a.integer(6), flags = a.integer(7);
        const float scale = a.real(8);
        int32_t ldz, ldk, ldw;
        const float *Z = a.matrix<float>(0, "Z", experts, batch, ldz), *bias = a.vector<float>(1, "bias", experts, true);
        int32_t *chosen = a.matrix<int32_t>(9, "chosen", k, batch, ldk);
        float *weights = a.matrix<float>(10, "weights", k, batch, ldw);
        if (a.ok && k > 1 && ldk != ldw) a.refuse("weights", "the row stride of chosen");
        void *s = a.stream(11);
        return [=] { return g_route(Z, ldz, bias, experts, batch, k, groups, top, flags, scale, chosen, weights, ldk, s); };
    });
}

// (Z, chosen, dweights, experts, batch, k, flags, scale, dZ, stream)
PyObject *route_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 10, [](Given &a) {
        const int32_t experts = a.integer(3), batch = a.integer(4), k = a.integer(5), flags = a.integer(6);
        const float scale = a.real(7);
        int32_t ldz, ldk, ldw, lddz;
        const float *Z = a.matrix<float>(0, "Z", experts, batch, ldz);
        const int32_t *chosen = a.matrix<int32_t>(1, "chosen", k, batch, ldk);
        const float *dw = a.matrix<float>(2, "dweights", k, batch, ldw);
        float *dZ = a.matrix<float>(8, "dZ", experts, batch, lddz);
        if (a.ok && k > 1 && ldk != ldw) a.refuse("dweights", "the row stride of chosen");
        void *s = a.stream(9);
        return [=] { return g_route_backward(Z, ldz, chosen, dw, ldk, experts, batch, k, flags, scale, dZ, lddz, s); };
    });
}

// (chosen, experts, batch, k, capacity, slots, counts, placement, stream)
PyObject *place(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 9, [](Given &a) {
        const int32_t experts = a.integer(1), batch = a.integer(2), k = a.integer(3), capacity = a.integer(4);
        int32_t ldk, lds;
        const int32_t *chosen = a.matrix<int32_t>(0, "chosen", k, batch, ldk);
        int32_t *slots = a.matrix<int32_t>(5, "slots", k, batch, lds, true), *counts = a.vector<int32_t>(6, "counts", experts, true);
        if (a.ok && slots && k > 1 && ldk != lds) a.refuse("slots", "the row stride of chosen");
        size_t bytes;
        void *placement = a.scratch(7, "placement", bytes);
        void *s = a.stream(8);
        return [=] { return g_place(chosen, ldk, experts, batch, k, capacity, slots, counts, placement, bytes, s); };
    });
}

// (X, placement, features, experts, batch, k, capacity, Xe, stream)
PyObject *dispatch(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 9, [](Given &a) {
        const int32_t features = a.integer(2), experts = a.integer(3), batch = a.integer(4), k = a.integer(5), capacity = a.integer(6);
        int32_t ldx, lde;
        const float *X = a.matrix<float>(0, "X", features, batch, ldx);
        size_t bytes;
        const void *placement = a.scratch(1, "placement", bytes);
        float *Xe = a.blocks(7, "Xe", experts, features, capacity, lde);
        void *s = a.stream(8);
        return [=] { return g_dispatch(X, ldx, placement, bytes, features, experts, batch, k, capacity, Xe, lde, s); };
    });
}

// (Ye, placement, weights, features, experts, batch, k, capacity, Y, stream)
PyObject *combine(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 10, [](Given &a) {
        const int32_t features = a.integer(3), experts = a.integer(4), batch = a.integer(5), k = a.integer(6), capacity = a.integer(7);
        int32_t lde, ldk, ldy;
        const float *Ye = a.blocks(0, "Ye", experts, features, capacity, lde);
        size_t bytes;
        const void *placement = a.scratch(1, "placement", bytes);
        const float *weights = a.matrix<float>(2, "weights", k, batch, ldk, true);
        float *Y = a.matrix<float>(8, "Y", features, batch, ldy);
        void *s = a.stream(9);
        return [=] { return g_combine(Ye, lde, placement, bytes, weights, ldk, features, experts, batch, k, capacity, Y, ldy, s); };
    });
}

// (Ye, dY, placement, weights, features, experts, batch, k, capacity, dYe, dweights, workspace, stream)
PyObject *combine_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 13, [](Given &a) {
        const int32_t features = a.integer(4), experts = a.integer(5), batch = a.integer(6), k = a.integer(7), capacity = a.integer(8);
        int32_t lde, ldd, lddy, ldk, lddw;
        const float *Ye = a.blocks(0, "Ye", experts, features, capacity, lde, true), *dY = a.matrix<float>(1, "dY", features, batch, lddy);
        size_t bytes, room;
        const void *placement = a.scratch(2, "placement", bytes);
        const float *weights = a.matrix<float>(3, "weights", k, batch, ldk, true);
        float *dYe = a.blocks(9, "dYe", experts, features, capacity, ldd, true), *dw = a.matrix<float>(10, "dweights", k, batch, lddw, true);
        if (a.ok && Ye && dYe && lde != ldd) a.refuse("dYe", "the row stride of Ye");
        if (a.ok && weights && dw && k > 1 && ldk != lddw) a.refuse("dweights", "the row stride of weights");
        void *workspace = a.scratch(11, "workspace", room);
        void *s = a.stream(12);
        return [=, lde = Ye ? lde : ldd, ldk = weights ? ldk : lddw] {
            return g_combine_backward(Ye, lde, dY, lddy, placement, bytes, weights, ldk, features, experts, batch, k, capacity, dYe, dw, workspace, room, s);
        };
    });
}

// (grads, workspace, norm, stream)
PyObject *norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 4, [](Given &a) {
        std::vector<float *> g;
        std::vector<int64_t> counts;
        a.arrays(0, "grads", g, counts, true);
        size_t room;
        void *workspace = a.scratch(1, "workspace", room);
        float *out = a.vector<float>(2, "norm", 1, true);
        void *s = a.stream(3);
        return [=, g = std::move(g), counts = std::move(counts)] { return g_norm(static_cast<int32_t>(g.size()), g.data(), counts.data(), workspace, room, out, s); };
    });
}

// (grads, clipped, max_norm, workspace, norm, stream)
PyObject *clip(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 6, [](Given &a) {
        std::vector<float *> g, out;
        std::vector<int64_t> counts;
        a.arrays(0, "grads", g, counts, true);
        a.arrays(1, "clipped", out, counts, false);
        const float max_norm = a.real(2);
        size_t room;
        void *workspace = a.scratch(3, "workspace", room);
        float *norm = a.vector<float>(4, "norm", 1, true);
        void *s = a.stream(5);
        return [=, g = std::move(g), out = std::move(out), counts = std::move(counts)] {
            return g_clip(static_cast<int32_t>(g.size()), g.data(), out.data(), counts.data(), max_norm, workspace, room, norm, s);
        };
    });
}

// (values, velocities, grads, lr, momentum, max_norm, nesterov, workspace, norm, stream)
PyObject *update_clipped(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 10, [](Given &a) {
        std::vector<float *> w, v, g;
        std::vector<int64_t> counts;
        a.arrays(2, "grads", g, counts, true);
        a.arrays(0, "values", w, counts, false);
        a.arrays(1, "velocities", v, counts, false);
        const float lr = a.real(3), mu = a.real(4), max_norm = a.real(5);
        const int32_t nesterov = a.integer(6);
        size_t room;
        void *workspace = a.scratch(7, "workspace", room);
        float *norm = a.vector<float>(8, "norm", 1, true);
        void *s = a.stream(9);
        return [=, w = std::move(w), v = std::move(v), g = std::move(g), counts = std::move(counts)] {
            return g_update_clipped(static_cast<int32_t>(g.size()), w.data(), v.data(), g.data(), counts.data(), lr, mu, max_norm, nesterov, workspace, room, norm, s);
        };
    });
}

// addresses of the entry points above, in the order of the functions above
PyObject *bind_mixtures(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 9) {
        PyErr_SetString(PyExc_TypeError, "nine addresses expected");
        return nullptr;
    }
    Args a{args};
    g_route = reinterpret_cast<Route>(a.address());
    g_route_backward = reinterpret_cast<RouteBackward>(a.address());
    g_place = reinterpret_cast<Place>(a.address());
    g_dispatch = reinterpret_cast<Dispatch>(a.address());
    g_combine = reinterpret_cast<Combine>(a.address());
    g_combine_backward = reinterpret_cast<CombineBackward>(a.address());
    g_norm = reinterpret_cast<Norm>(a.address());
    g_clip = reinterpret_cast<Clip>(a.address());
    g_update_clipped = reinterpret_cast<UpdateClipped>(a.address());
    if (!a.ok) return nullptr;
    Py_RETURN_NONE;
}

// (X, gamma, beta, features, groups, batch, eps, act, drop, layer, state, Y, mean, rstd, workspace, stream)
PyObject *norm_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 16, [](Given &a) {
        const int32_t features = a.integer(3), groups = a.integer(4), batch = a.integer(5), act = a.integer(7), layer = a.integer(9);
        const float eps = a.real(6), drop = a.real(8);
        int32_t ldx, ldy, lds, ldr;
        const float *X = a.matrix<float>(0, "X", features, batch, ldx), *gamma = a.vector<float>(1, "gamma", features, true), *beta = a.vector<float>(2, "beta", features, true);
        const int64_t *state = a.vector<int64_t>(10, "state", 2, true);
        float *Y = a.matrix<float>(11, "Y", features, batch, ldy), *mean = a.matrix<float>(12, "mean", groups, batch, lds, true),
              *rstd = a.matrix<float>(13, "rstd", groups, batch, ldr, true);
        if (a.ok && mean && rstd && groups > 1 && lds != ldr) a.refuse("rstd", "the row stride of mean");
        size_t room;
        void *workspace = a.scratch(14, "workspace", room);
        void *s = a.stream(15);
        return [=] { return g_norm_forward(X, ldx, gamma, beta, features, groups, batch, eps, act, drop, layer, state, Y, ldy, mean, rstd, lds, workspace, room, s); };
    });
}

// (X, gamma, beta, mean, rstd, dY, features, groups, batch, act, drop, layer, state, dX, dgamma, dbeta, workspace, stream)
PyObject *norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 18, [](Given &a) {
        const int32_t features = a.integer(6), groups = a.integer(7), batch = a.integer(8), act = a.integer(9), layer = a.integer(11);
        const float drop = a.real(10);
        int32_t ldx, lds, ldr, lddy, lddx;
        const float *X = a.matrix<float>(0, "X", features, batch, ldx), *gamma = a.vector<float>(1, "gamma", features, true), *beta = a.vector<float>(2, "beta", features, true);
        const float *mean = a.matrix<float>(3, "mean", groups, batch, lds), *rstd = a.matrix<float>(4, "rstd", groups, batch, ldr);
        if (a.ok && groups > 1 && lds != ldr) a.refuse("rstd", "the row stride of mean");
        const float *dY = a.matrix<float>(5, "dY", features, batch, lddy);
        const int64_t *state = a.vector<int64_t>(12, "state", 2, true);
        float *dX = a.matrix<float>(13, "dX", features, batch, lddx), *dgamma = a.vector<float>(14, "dgamma", features, true), *dbeta = a.vector<float>(15, "dbeta", features, true);
        size_t room;
        void *workspace = a.scratch(16, "workspace", room);
        void *s = a.stream(17);
        return [=] {
            return g_norm_backward(X, ldx, gamma, beta, mean, rstd, lds, dY, lddy, features, groups, batch, act, drop, layer, state, dX, lddx, dgamma, dbeta, workspace,
                                   room, s);
        };
    });
}

// (X, features, batch, drop, layer, state, Y, stream)
PyObject *dropout(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 8, [](Given &a) {
        const int32_t features = a.integer(1), batch = a.integer(2), layer = a.integer(4);
        const float drop = a.real(3);
        int32_t ldx, ldy;
        const float *X = a.matrix<float>(0, "X", features, batch, ldx);
        const int64_t *state = a.vector<int64_t>(5, "state", 2, true);
        float *Y = a.matrix<float>(6, "Y", features, batch, ldy);
        void *s = a.stream(7);
        return [=] { return g_dropout(X, ldx, features, batch, drop, layer, state, Y, ldy, s); };
    });
}

// (Z, labels, classes, batch, starts, sequences, logp, sums, workspace, stream)
PyObject *log_probs(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 10, [](Given &a) {
        const int32_t classes = a.integer(2), batch = a.integer(3), sequences = a.integer(5);
        int32_t ldz;
        const float *Z = a.matrix<float>(0, "Z", classes, batch, ldz);
        const int32_t *labels = a.vector<int32_t>(1, "labels", batch), *starts = a.vector<int32_t>(4, "starts", static_cast<int64_t>(sequences) + 1, true);
        float *logp = a.vector<float>(6, "logp", batch, true), *sums = a.vector<float>(7, "sums", sequences, true);
        size_t room;
        void *workspace = a.scratch(8, "workspace", room);
        void *s = a.stream(9);
        return [=] { return g_log_probs(Z, ldz, labels, classes, batch, starts, sequences, logp, sums, workspace, room, s); };
    });
}

// (Z, labels, old_logp, ref_logp, advantages, weights, classes, batch, clip_low, clip_high, beta, dZ, logp, stats, workspace, stream)
PyObject *policy(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 16, [](Given &a) {
        const int32_t classes = a.integer(6), batch = a.integer(7);
        const float low = a.real(8), high = a.real(9), beta = a.real(10);
        int32_t ldz, lddz;
        const float *Z = a.matrix<float>(0, "Z", classes, batch, ldz);
        const int32_t *labels = a.vector<int32_t>(1, "labels", batch);
        const float *old = a.vector<float>(2, "old_logp", batch), *ref = a.vector<float>(3, "ref_logp", batch, true), *advantages = a.vector<float>(4, "advantages", batch),
                    *weights = a.vector<float>(5, "weights", batch, true);
        float *dZ = a.matrix<float>(11, "dZ", classes, batch, lddz), *logp = a.vector<float>(12, "logp", batch, true), *stats = a.vector<float>(13, "stats", 4);
        size_t room;
        void *workspace = a.scratch(14, "workspace", room);
        void *s = a.stream(15);
        return [=] { return g_policy(Z, ldz, labels, old, ref, advantages, weights, classes, batch, low, high, beta, dZ, lddz, logp, stats, workspace, room, s); };
    });
}

// (Z, labels, starts, ref_sums, classes, batch, pairs, beta, smoothing, dZ, sums, margins, loss, workspace, stream)
PyObject *preference(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return run_given(args, n, 15, [](Given &a) {
        const int32_t classes = a.integer(4), batch = a.integer(5), pairs = a.integer(6);
        const float beta = a.real(7), smoothing = a.real(8);
        const int64_t sequences = 2 * static_cast<int64_t>(pairs);
        int32_t ldz, lddz;
        const float *Z = a.matrix<float>(0, "Z", classes, batch, ldz);
        const int32_t *labels = a.vector<int32_t>(1, "labels", batch), *starts = a.vector<int32_t>(2, "starts", sequences + 1);
        const float *ref = a.vector<float>(3, "ref_sums", sequences, true);
        float *dZ = a.matrix<float>(9, "dZ", classes, batch, lddz), *sums = a.vector<float>(10, "sums", sequences, true), *margins = a.vector<float>(11, "margins", pairs, true),
              *loss = a.vector<float>(12, "loss", 1, true);
        size_t room;
        void *workspace = a.scratch(13, "workspace", room);
        void *s = a.stream(14);
        return [=] { return g_preference(Z, ldz, labels, starts, ref, classes, batch, pairs, beta, smoothing, dZ, lddz, sums, margins, loss, workspace, room, s); };
    });
}

// addresses of the six entry points above, in their order
PyObject *bind_losses(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "six addresses expected");
        return nullptr;
    }
    Args a{args};
    g_norm_forward = reinterpret_cast<NormForward>(a.address());
    g_norm_backward = reinterpret_cast<NormBackward>(a.address());
    g_dropout = reinterpret_cast<Dropout>(a.address());
    g_log_probs = reinterpret_cast<LogProbs>(a.address());
    g_policy = reinterpret_cast<Policy>(a.address());
    g_preference = reinterpret_cast<Preference>(a.address());
    if (!a.ok) return nullptr;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind)), METH_FASTCALL, nullptr},
    {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(forward)), METH_FASTCALL, nullptr},
    {"backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(backward)), METH_FASTCALL, nullptr},
    {"update", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(update)), METH_FASTCALL, nullptr},
    {"train_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(train_step)), METH_FASTCALL, nullptr},
    {"mlp_forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(mlp_forward)), METH_FASTCALL, nullptr},
    {"view", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(view)), METH_FASTCALL, nullptr},
    {"bind_mixtures", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind_mixtures)), METH_FASTCALL, nullptr},
    {"route", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(route)), METH_FASTCALL, nullptr},
    {"route_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(route_backward)), METH_FASTCALL, nullptr},
    {"place", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(place)), METH_FASTCALL, nullptr},
    {"dispatch", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(dispatch)), METH_FASTCALL, nullptr},
    {"combine", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(combine)), METH_FASTCALL, nullptr},
    {"combine_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(combine_backward)), METH_FASTCALL, nullptr},
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(norm)), METH_FASTCALL, nullptr},
    {"clip", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(clip)), METH_FASTCALL, nullptr},
    {"update_clipped", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(update_clipped)), METH_FASTCALL, nullptr},
    {"bind_losses", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind_losses)), METH_FASTCALL, nullptr},
    {"norm_forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(norm_forward)), METH_FASTCALL, nullptr},
    {"norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(norm_backward)), METH_FASTCALL, nullptr},
    {"dropout", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(dropout)), METH_FASTCALL, nullptr},
    {"log_probs", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(log_probs)), METH_FASTCALL, nullptr},
    {"policy", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(policy)), METH_FASTCALL, nullptr},
    {"preference", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(preference)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&module); }
