// The step calls of the Python binding without interpreter work per tensor.
//
// A step of a small model is host time: with every tensor's device, type, shape and strides asked for
// through Python attributes and the messages marshalled through ctypes a call took about 10 us, of which the
// library's own work and launch are 3 to 4.  Here a call looks at the same properties in the tensors
// themselves.  It goes ahead only where everything is plainly as the library assumes it; anything else (another
// type or layout, a tensor subclass, an active function mode, a wrapper without memory) is answered with -1 and
// left to the checks in Python, which name what is wrong or take what is unusual.  Nothing is remembered from
// one call to the next.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/ds.h"

namespace {

using WorkerFn = ds_status_t (*)(ds_ctx_t *, uint64_t, const void *, int64_t, float *, int64_t, const ds_payload_t *, void *);
using ServerFn = ds_status_t (*)(ds_ctx_t *, uint64_t, const ds_payload_t *, float *, const ds_payload_t *, void *);
using UpdateFn = ds_status_t (*)(ds_ctx_t *, const ds_payload_t *, float *, float *, float, float, void *);
using DecodeFn = ds_status_t (*)(ds_ctx_t *, const ds_payload_t *, int32_t, int32_t, float *, void *);
using ServerUpdateFn = ds_status_t (*)(ds_ctx_t *, uint64_t, const ds_payload_t *, float *, const ds_payload_t *, float *, float *, float,
                                       float, void *);
using OrthoFn = ds_status_t (*)(ds_ctx_t *, ds_ortho_t *, const ds_payload_t *, float *, float *, float, float, float, void *);
using AdamWFn = ds_status_t (*)(ds_ctx_t *, const ds_ortho_t *, const ds_payload_t *, uint64_t, float *, float *, float *, double, double,
                                double, double, double, void *);

struct Calls {
    PyObject_HEAD
    ds_ctx_t *ctx;               // null once closed
    int64_t n, d, k;
    int comp;
    bool bf16, nofb, sid;
    PyObject *payload_type, *get_device, *get_stream;
    WorkerFn worker;
    ServerFn server;
    UpdateFn update;
    DecodeFn decode;
    ServerUpdateFn server_update;
    OrthoFn ortho;
    AdamWFn adamw;
    int device;
};

constexpr int kIdentity = 0;
PyObject *s_comp, *s_rows, *s_d, *s_k, *s_cuda_stream, *s_buffers[5];

PyObject *python_decides() { return PyLong_FromLong(-1); }

// A plain tensor with memory on the device.
const at::Tensor *device_tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != c10::kStrided || !t.has_storage() || t.is_conj() || t.is_neg()) return nullptr;
    return &t;
}

// rows == 0: a vector of d elements, else [rows, d] with dense rows.  The pointer, or null.
void *matrix(PyObject *o, c10::ScalarType type, int64_t rows, int64_t d, int64_t *stride)
{
    const at::Tensor *t = device_tensor(o);
    if (!t || t->scalar_type() != type || t->dim() != (rows ? 2 : 1)) return nullptr;
    if (rows == 0) {
        if (t->size(0) != d || t->stride(0) != 1) return nullptr;
    } else {
        if (t->size(0) != rows || t->size(1) != d || t->stride(1) != 1) return nullptr;
        const int64_t s = t->stride(0);
        if (rows > 1 && s < d) return nullptr;
        *stride = (rows > 1 || s > d) ? s : d;       // a single row has no meaningful row stride
    }
    return t->data_ptr();
}

// An attribute that is a plain int.
bool int_attr(PyObject *o, PyObject *name, int64_t *out)
{
    PyObject *v = PyObject_GetAttr(o, name);
    if (!v) { PyErr_Clear(); return false; }
    const bool ok = PyLong_CheckExact(v);
    if (ok) *out = PyLong_AsLongLong(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return ok;
}

// rows < 0: as many as the payload says.  device >= 0: the buffers have to be there.
bool payload(const Calls *c, PyObject *o, int64_t rows, bool server, ds_payload_t *out, int64_t *rows_out = nullptr, int device = -1)
{
    if (reinterpret_cast<PyObject *>(Py_TYPE(o)) != c->payload_type) return false;
    int64_t comp, has_rows, d, k;
    if (!int_attr(o, s_comp, &comp) || !int_attr(o, s_rows, &has_rows) || !int_attr(o, s_d, &d) || !int_attr(o, s_k, &k)) return false;
    if (rows < 0 && c->sid && comp == kIdentity) server = true;
    const int64_t want = (server && c->sid) ? kIdentity : c->comp;
    if (comp != want || d != c->d || (comp != kIdentity && k != c->k) || (rows >= 0 && has_rows != rows)) return false;
    if (rows_out) *rows_out = has_rows;
    void *p[5];
    for (int i = 0; i < 5; ++i) {
        PyObject *v = PyObject_GetAttr(o, s_buffers[i]);
        if (!v) { PyErr_Clear(); return false; }
        p[i] = nullptr;
        bool ok = true;
        if (v != Py_None) {
            const at::Tensor *t = device_tensor(v);
            ok = t && t->is_contiguous() && (device < 0 || t->get_device() == device);
            if (ok) p[i] = t->data_ptr();
        }
        Py_DECREF(v);                                // the payload holds it
        if (!ok) return false;
    }
    *out = ds_payload_t{static_cast<uint64_t *>(p[0]), static_cast<float *>(p[1]), static_cast<uint8_t *>(p[2]),
                        static_cast<ds_pair_t *>(p[3]), static_cast<float *>(p[4])};
    return true;
}

// The stream to launch on: the one given, or the current one of the current device, which is to be `device` if that is >= 0.
bool stream(const Calls *c, PyObject *o, void **out, int device = -1)
{
    PyObject *v;
    if (o == Py_None) {
        PyObject *dev = PyObject_CallNoArgs(c->get_device);
        if (!dev) { PyErr_Clear(); return false; }
        if (device >= 0 && !(PyLong_CheckExact(dev) && PyLong_AsLong(dev) == device)) {
            Py_DECREF(dev);
            PyErr_Clear();
            return false;
        }
        v = PyObject_CallOneArg(c->get_stream, dev);
        Py_DECREF(dev);
    } else {
        v = PyObject_GetAttr(o, s_cuda_stream);
    }
    if (!v) { PyErr_Clear(); return false; }
    const bool ok = PyLong_CheckExact(v);
    if (ok) *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return ok;
}

bool step_of(PyObject *o, uint64_t *out)
{
    if (!PyLong_CheckExact(o)) return false;
    *out = PyLong_AsUnsignedLongLongMask(o);
    return true;
}

bool number(PyObject *o, float *out)
{
    if (PyFloat_CheckExact(o)) *out = static_cast<float>(PyFloat_AS_DOUBLE(o));
    else if (PyLong_CheckExact(o)) *out = static_cast<float>(PyLong_AsDouble(o));
    else return false;
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

bool number(PyObject *o, double *out)
{
    if (PyFloat_CheckExact(o)) *out = PyFloat_AS_DOUBLE(o);
    else if (PyLong_CheckExact(o)) *out = PyLong_AsDouble(o);
    else return false;
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

// A vector of d floats on the context's device.
bool own_vector(const Calls *c, PyObject *o, float **out)
{
    *out = static_cast<float *>(matrix(o, at::kFloat, 0, c->d, nullptr));
    return *out != nullptr && THPVariable_Unpack(o).get_device() == c->device;
}

// A plan's address; the caller has seen that the plan is open and fits.
template <class T>
bool address(PyObject *o, T **out)
{
    if (!PyLong_CheckExact(o)) return false;
    *out = static_cast<T *>(PyLong_AsVoidPtr(o));
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

// A vector of d floats that may be missing (then *out is null).
bool optional_vector(const Calls *c, PyObject *o, float **out)
{
    *out = nullptr;
    if (o == Py_None) return true;
    *out = static_cast<float *>(matrix(o, at::kFloat, 0, c->d, nullptr));
    return *out != nullptr;
}

// Runs `body(c)`, which returns false where Python shall decide and else leaves the status; C++ exceptions of torch
// (a tensor that refuses its pointer) count as "Python decides".
template <class F>
PyObject *call(PyObject *self, Py_ssize_t nargs, Py_ssize_t want, F body)
{
    const Calls *c = reinterpret_cast<Calls *>(self);
    if (!c->ctx || nargs != want || at::impl::PythonTorchFunctionTLS::stack_len() > 0) return python_decides();
    ds_status_t rc = DS_OK;
    try {
        if (!body(c, rc)) return python_decides();
    } catch (const std::exception &) {
        return python_decides();
    }
    return PyLong_FromLong(static_cast<long>(rc));
}

// step, g, delta, out, stream
PyObject *worker(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    return call(self, nargs, 5, [a](const Calls *c, ds_status_t &rc) {
        uint64_t t;
        void *st;
        ds_payload_t out;
        int64_t gs = c->d, ds = c->d;
        if (!step_of(a[0], &t)) return false;
        void *g = matrix(a[1], c->bf16 ? at::kBFloat16 : at::kFloat, c->n, c->d, &gs);
        if (!g) return false;
        void *delta = nullptr;
        if (a[2] != Py_None || !c->nofb) {
            delta = matrix(a[2], at::kFloat, c->n, c->d, &ds);
            if (!delta) return false;
        }
        if (!payload(c, a[3], c->n, false, &out) || !stream(c, a[4], &st)) return false;
        Py_BEGIN_ALLOW_THREADS
        rc = c->worker(c->ctx, t, g, gs, static_cast<float *>(delta), ds, &out, st);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// step, in, delta_s, out, stream
PyObject *server(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    return call(self, nargs, 5, [a](const Calls *c, ds_status_t &rc) {
        uint64_t t;
        void *st;
        float *delta_s;
        ds_payload_t in, out;
        if (!step_of(a[0], &t) || !optional_vector(c, a[2], &delta_s) || (!delta_s && !c->nofb && !c->sid)) return false;
        if (!payload(c, a[1], c->n, false, &in) || !payload(c, a[3], 1, true, &out) || !stream(c, a[4], &st)) return false;
        Py_BEGIN_ALLOW_THREADS
        rc = c->server(c->ctx, t, &in, delta_s, &out, st);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// step, in, delta_s, out, x, m, gamma, beta, stream
PyObject *server_update(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    return call(self, nargs, 9, [a](const Calls *c, ds_status_t &rc) {
        uint64_t t;
        void *st;
        float *delta_s, *x, *m, gamma, beta;
        ds_payload_t in, out{};
        if (!step_of(a[0], &t) || !optional_vector(c, a[2], &delta_s) || (!delta_s && !c->nofb && !c->sid)) return false;
        if (!optional_vector(c, a[4], &x) || !x || !optional_vector(c, a[5], &m)) return false;
        if (!number(a[6], &gamma) || !number(a[7], &beta)) return false;
        if (!payload(c, a[1], c->n, false, &in)) return false;
        if (!(a[3] == Py_None && c->sid) && !payload(c, a[3], 1, true, &out)) return false;
        if (!stream(c, a[8], &st)) return false;
        Py_BEGIN_ALLOW_THREADS
        rc = c->server_update(c->ctx, t, &in, delta_s, &out, x, m, gamma, beta, st);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// srv, x, m, gamma, beta, stream
PyObject *update(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    return call(self, nargs, 6, [a](const Calls *c, ds_status_t &rc) {
        void *st;
        float *x, *m, gamma, beta;
        ds_payload_t srv;
        if (!optional_vector(c, a[1], &x) || !x || !optional_vector(c, a[2], &m)) return false;
        if (!number(a[3], &gamma) || !number(a[4], &beta)) return false;
        if (!payload(c, a[0], 1, true, &srv) || !stream(c, a[5], &st)) return false;
        Py_BEGIN_ALLOW_THREADS
        rc = c->update(c->ctx, &srv, x, m, gamma, beta, st);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// plan, srv, x, m, gamma, beta, decay, stream
PyObject *ortho(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    return call(self, nargs, 8, [a](const Calls *c, ds_status_t &rc) {
        void *st;
        ds_ortho_t *plan;
        float *x, *m = nullptr, gamma, beta, decay;
        ds_payload_t srv;
        if (!address(a[0], &plan) || !own_vector(c, a[2], &x) || (a[3] != Py_None && !own_vector(c, a[3], &m))) return false;
        if (!number(a[4], &gamma) || !number(a[5], &beta) || !number(a[6], &decay)) return false;
        if (!payload(c, a[1], 1, true, &srv, nullptr, c->device) || !stream(c, a[7], &st, c->device)) return false;
        Py_BEGIN_ALLOW_THREADS
        rc = c->ortho(c->ctx, plan, &srv, x, m, gamma, beta, decay, st);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// plan or 0, srv, step, x, m, v, gamma, beta1, beta2, eps, decay, stream
PyObject *adamw(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    return call(self, nargs, 12, [a](const Calls *c, ds_status_t &rc) {
        void *st;
        ds_ortho_t *plan;
        float *x, *m, *v;
        double gamma, beta1, beta2, eps, decay;
        ds_payload_t srv;
        if (!address(a[0], &plan) || !PyLong_CheckExact(a[2])) return false;
        const unsigned long long t = PyLong_AsUnsignedLongLong(a[2]);
        if (PyErr_Occurred()) { PyErr_Clear(); return false; }
        if (!own_vector(c, a[3], &x) || !own_vector(c, a[4], &m) || !own_vector(c, a[5], &v)) return false;
        if (!number(a[6], &gamma) || !number(a[7], &beta1) || !number(a[8], &beta2) || !number(a[9], &eps) || !number(a[10], &decay)) return false;
        if (!payload(c, a[1], 1, true, &srv, nullptr, c->device) || !stream(c, a[11], &st, c->device)) return false;
        Py_BEGIN_ALLOW_THREADS
        rc = c->adamw(c->ctx, plan, &srv, t, x, m, v, gamma, beta1, beta2, eps, decay, st);
        Py_END_ALLOW_THREADS
        return true;
    });
}

// p, row, out, stream
PyObject *decode(PyObject *self, PyObject *const *a, Py_ssize_t nargs)
{
    return call(self, nargs, 4, [a](const Calls *c, ds_status_t &rc) {
        void *st;
        float *out;
        ds_payload_t p;
        int64_t rows;
        if (!PyLong_CheckExact(a[1]) || !optional_vector(c, a[2], &out) || !out) return false;
        const long long row = PyLong_AsLongLong(a[1]);
        if (PyErr_Occurred()) { PyErr_Clear(); return false; }
        if (!payload(c, a[0], -1, false, &p, &rows) || !stream(c, a[3], &st)) return false;
        if (row < 0 || row >= rows || rows > 0x7FFFFFFF) return false;
        Py_BEGIN_ALLOW_THREADS
        rc = c->decode(c->ctx, &p, static_cast<int32_t>(rows), static_cast<int32_t>(row), out, st);
        Py_END_ALLOW_THREADS
        return true;
    });
}

PyObject *close_calls(PyObject *self, PyObject *)
{
    reinterpret_cast<Calls *>(self)->ctx = nullptr;
    Py_RETURN_NONE;
}

// Calls(context, n, d, k, comp, bf16, nofb, sid, device, payload_type, get_device, get_stream, addresses of the seven functions)
int init_calls(PyObject *self, PyObject *args, PyObject *)
{
    Calls *c = reinterpret_cast<Calls *>(self);
    unsigned long long ctx, f[7];
    long long n, d, k;
    int bf16, nofb, sid;
    PyObject *type, *dev, *str;
    if (!PyArg_ParseTuple(args, "KLLLipppiOOOKKKKKKK", &ctx, &n, &d, &k, &c->comp, &bf16, &nofb, &sid, &c->device, &type, &dev, &str, &f[0],
                          &f[1], &f[2], &f[3], &f[4], &f[5], &f[6]))
        return -1;
    c->ctx = reinterpret_cast<ds_ctx_t *>(ctx);
    c->n = n; c->d = d; c->k = k;
    c->bf16 = bf16 != 0; c->nofb = nofb != 0; c->sid = sid != 0;
    Py_INCREF(type); Py_INCREF(dev); Py_INCREF(str);
    Py_XSETREF(c->payload_type, type);
    Py_XSETREF(c->get_device, dev);
    Py_XSETREF(c->get_stream, str);
    c->worker = reinterpret_cast<WorkerFn>(f[0]);
    c->server = reinterpret_cast<ServerFn>(f[1]);
    c->update = reinterpret_cast<UpdateFn>(f[2]);
    c->decode = reinterpret_cast<DecodeFn>(f[3]);
    c->server_update = reinterpret_cast<ServerUpdateFn>(f[4]);
    c->ortho = reinterpret_cast<OrthoFn>(f[5]);
    c->adamw = reinterpret_cast<AdamWFn>(f[6]);
    return 0;
}

void free_calls(PyObject *self)
{
    Calls *c = reinterpret_cast<Calls *>(self);
    Py_XDECREF(c->payload_type);
    Py_XDECREF(c->get_device);
    Py_XDECREF(c->get_stream);
    Py_TYPE(self)->tp_free(self);
}

template <class F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"worker", fast(worker), METH_FASTCALL, nullptr},
    {"server", fast(server), METH_FASTCALL, nullptr},
    {"server_update", fast(server_update), METH_FASTCALL, nullptr},
    {"update", fast(update), METH_FASTCALL, nullptr},
    {"decode", fast(decode), METH_FASTCALL, nullptr},
    {"ortho", fast(ortho), METH_FASTCALL, nullptr},
    {"adamw", fast(adamw), METH_FASTCALL, nullptr},
    {"close", close_calls, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyTypeObject type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall()
{
    type.tp_name = "paper_1905_05957_amd._fastcall.Calls";
    type.tp_basicsize = sizeof(Calls);
    type.tp_flags = Py_TPFLAGS_DEFAULT;
    type.tp_new = PyType_GenericNew;
    type.tp_init = init_calls;
    type.tp_dealloc = free_calls;
    type.tp_methods = methods;
    if (PyType_Ready(&type) < 0) return nullptr;
    const char *buffers[5] = {"sign_words", "scales", "levels", "pairs", "dense"};
    for (int i = 0; i < 5; ++i)
        if (!(s_buffers[i] = PyUnicode_InternFromString(buffers[i]))) return nullptr;
    if (!(s_comp = PyUnicode_InternFromString("comp")) || !(s_rows = PyUnicode_InternFromString("rows")) ||
        !(s_d = PyUnicode_InternFromString("d")) || !(s_k = PyUnicode_InternFromString("k")) ||
        !(s_cuda_stream = PyUnicode_InternFromString("cuda_stream")))
        return nullptr;
    PyObject *m = PyModule_Create(&module);
    if (!m) return nullptr;
    Py_INCREF(&type);
    if (PyModule_AddObject(m, "Calls", reinterpret_cast<PyObject *>(&type)) < 0) { Py_DECREF(&type); Py_DECREF(m); return nullptr; }
    return m;
}
