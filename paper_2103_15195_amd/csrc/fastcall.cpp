// The hot calls of the bindings without ctypes: a small call's launch takes the host 2.6 us, and what ctypes and the Python
// around it took to bring its arguments there nearly as long again.
// Each function takes the arguments in the forms that a hot loop passes -- Python ints, a float, ctypes arrays of addresses, tensors, no
// stream -- and returns the library's status; for anything else it returns None and has done nothing, and the caller takes the ctypes route, which
// converts or refuses as it always did.
// (A pass of four calls on 135 000 elements each, 22.3 us with ctypes, 19.6 so; of two calls over eight groups, 22.1 and 19.0; 161 single calls
// 1610 and 1536.)
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

namespace {

typedef int (*compress_fn)(void *, int32_t, uint32_t, uint64_t, const void *, void *, void *, void *);
typedef int (*decompress_fn)(void *, int32_t, const void *, int32_t, float, const void *, void *);
typedef int (*compress_all_fn)(void *, uint32_t, uint64_t, const void *, const void *, const void *, void *);
typedef int (*decompress_all_fn)(void *, const void *, int32_t, float, const void *, void *);

PyObject *g_data_ptr;                 // the name

// The entry points of one loaded library.
struct Calls {
    PyObject_HEAD
    PyTypeObject *array;              // ctypes.Array
    compress_fn compress, compress_static;
    decompress_fn decompress;
    compress_all_fn compress_all;
    decompress_all_fn decompress_all;
};
// torch's current stream on the current device, as a callable without arguments
struct RawStream {
    PyObject_HEAD
    PyObject *get, *device;
};
extern PyTypeObject RawStreamType;

// An argument that is not in the form expected ends in `other`: None, with no error left behind.
PyObject *other()
{
    PyErr_Clear();
    Py_RETURN_NONE;
}
bool whole(PyObject *o, uint64_t *v)          // as ctypes takes integers: any value, its low bits
{
    if (!PyLong_Check(o)) return false;
    *v = PyLong_AsUnsignedLongLongMask(o);
    return !(*v == (uint64_t)-1 && PyErr_Occurred());
}
bool address(PyObject *o, void **p)
{
    if (!PyLong_Check(o)) return false;
    *p = reinterpret_cast<void *>((uintptr_t)PyLong_AsUnsignedLongLongMask(o));
    return !PyErr_Occurred();
}
// where a ctypes array's elements lie, and how many there are
bool array(const Calls *c, PyObject *o, void **p, Py_ssize_t *n)
{
    if (!PyObject_TypeCheck(o, c->array)) return false;
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) < 0) return false;
    *p = b.buf;
    PyBuffer_Release(&b);                     // (the array lives as long as the caller's argument)
    if (n && (*n = PyObject_Size(o)) < 0) return false;
    return true;
}
bool tensor(PyObject *o, void **p)
{
    PyObject *a = PyObject_CallMethodNoArgs(o, g_data_ptr);
    if (!a) return false;
    const bool ok = address(a, p);
    Py_DECREF(a);
    return ok;
}
PyObject *raw_stream_call(PyObject *self, PyObject *, PyObject *)
{
    RawStream *r = reinterpret_cast<RawStream *>(self);
    PyObject *d = PyObject_CallNoArgs(r->device);
    if (!d) return nullptr;
    PyObject *s = PyObject_CallOneArg(r->get, d);
    Py_DECREF(d);
    return s;
}
// what the callable says, if there is one
bool stream_of(PyObject *callable, void **p)
{
    if (callable == Py_None) return false;
    PyObject *s = Py_TYPE(callable) == &RawStreamType ? raw_stream_call(callable, nullptr, nullptr) : PyObject_CallNoArgs(callable);
    if (!s) return false;
    const bool ok = address(s, p);
    Py_DECREF(s);
    return ok;
}

// (context, group, worker, iteration, gradients, state or None, payload, the stream's callable)
PyObject *compress_by(const Calls *c, compress_fn fn, PyObject *const *a, Py_ssize_t n)
{
    void *ctx, *grads, *state = nullptr, *payload, *stream;
    uint64_t group, worker, iter;
    if (n != 8 || !address(a[0], &ctx) || !whole(a[1], &group) || !whole(a[2], &worker) || !whole(a[3], &iter) || !array(c, a[4], &grads, nullptr) ||
        (a[5] != Py_None && !tensor(a[5], &state)) || !tensor(a[6], &payload) || !stream_of(a[7], &stream)) return other();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(ctx, (int32_t)group, (uint32_t)worker, iter, grads, state, payload, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
const Calls *of(PyObject *self) { return reinterpret_cast<const Calls *>(self); }
PyObject *compress(PyObject *self, PyObject *const *a, Py_ssize_t n) { return compress_by(of(self), of(self)->compress, a, n); }
PyObject *compress_static(PyObject *self, PyObject *const *a, Py_ssize_t n) { return compress_by(of(self), of(self)->compress_static, a, n); }

// (context, group, payloads, alpha, outputs, the stream's callable)
PyObject *decompress(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const Calls *c = of(self);
    void *ctx, *payloads, *outs, *stream;
    uint64_t group;
    Py_ssize_t W;
    if (n != 6 || !address(a[0], &ctx) || !whole(a[1], &group) || !array(c, a[2], &payloads, &W) || !PyFloat_CheckExact(a[3]) ||
        !array(c, a[4], &outs, nullptr) || !stream_of(a[5], &stream)) return other();
    const float alpha = (float)PyFloat_AS_DOUBLE(a[3]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->decompress(ctx, (int32_t)group, payloads, (int32_t)W, alpha, outs, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (context, worker, iteration, gradients, states or None, payloads, the stream's callable)
PyObject *compress_groups(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const Calls *c = of(self);
    void *ctx, *grads, *states = nullptr, *payloads, *stream;
    uint64_t worker, iter;
    if (n != 7 || !address(a[0], &ctx) || !whole(a[1], &worker) || !whole(a[2], &iter) || !array(c, a[3], &grads, nullptr) ||
        (a[4] != Py_None && !array(c, a[4], &states, nullptr)) || !array(c, a[5], &payloads, nullptr) || !stream_of(a[6], &stream)) return other();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->compress_all(ctx, (uint32_t)worker, iter, grads, states, payloads, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// (context, payloads, workers, alpha, outputs, the stream's callable)
PyObject *decompress_groups(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const Calls *c = of(self);
    void *ctx, *payloads, *outs, *stream;
    uint64_t W;
    if (n != 6 || !address(a[0], &ctx) || !array(c, a[1], &payloads, nullptr) || !whole(a[2], &W) || !PyFloat_CheckExact(a[3]) ||
        !array(c, a[4], &outs, nullptr) || !stream_of(a[5], &stream)) return other();
    const float alpha = (float)PyFloat_AS_DOUBLE(a[3]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->decompress_all(ctx, payloads, (int32_t)W, alpha, outs, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// Calls(ctypes.Array, addresses of mc_compress, mc_compress_static, mc_decompress_sum, mc_compress_groups, mc_decompress_sum_groups)
PyObject *calls_new(PyTypeObject *type, PyObject *args, PyObject *)
{
    PyObject *array = nullptr;
    unsigned long long at[5] = {};
    if (!PyArg_ParseTuple(args, "O!KKKKK", &PyType_Type, &array, &at[0], &at[1], &at[2], &at[3], &at[4])) return nullptr;
    Calls *c = reinterpret_cast<Calls *>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    Py_INCREF(array);
    c->array = reinterpret_cast<PyTypeObject *>(array);
    c->compress = (compress_fn)(uintptr_t)at[0];
    c->compress_static = (compress_fn)(uintptr_t)at[1];
    c->decompress = (decompress_fn)(uintptr_t)at[2];
    c->compress_all = (compress_all_fn)(uintptr_t)at[3];
    c->decompress_all = (decompress_all_fn)(uintptr_t)at[4];
    return reinterpret_cast<PyObject *>(c);
}
void calls_gone(PyObject *self)
{
    Py_XDECREF(reinterpret_cast<PyObject *>(reinterpret_cast<Calls *>(self)->array));
    Py_TYPE(self)->tp_free(self);
}
// RawStream(stream of a device, current device): both callable
PyObject *raw_stream_new(PyTypeObject *type, PyObject *args, PyObject *)
{
    PyObject *get, *device;
    if (!PyArg_ParseTuple(args, "OO", &get, &device)) return nullptr;
    RawStream *r = reinterpret_cast<RawStream *>(type->tp_alloc(type, 0));
    if (!r) return nullptr;
    Py_INCREF(get);
    Py_INCREF(device);
    r->get = get;
    r->device = device;
    return reinterpret_cast<PyObject *>(r);
}
void raw_stream_gone(PyObject *self)
{
    RawStream *r = reinterpret_cast<RawStream *>(self);
    Py_XDECREF(r->get);
    Py_XDECREF(r->device);
    Py_TYPE(self)->tp_free(self);
}

// ---- lists of tensors and rows of logits (step.py) -----------------------------------------------------------------------------------------
// The structures of mergecomp_step.h.
struct Logits {
    const void *logits, *labels;
    int64_t rows, vocab, stride;
    int32_t dtype;
    float temperature;
};
struct Policy {
    const void *old_logp, *advantages, *weights, *ref_logp;
    float clip_low, clip_high, kl_coef, grad_scale;
    void *sums, *logp, *dlogits;
    int64_t dlogits_stride;
};
struct Adamw {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;
};
typedef int (*grad_norm_fn)(void *, float, float, void *, void *);
typedef int (*adamw_fn)(void *, const Adamw *, const void *, void *);
typedef int (*token_logp_fn)(void *, const Logits *, void *, void *);
typedef int (*policy_loss_fn)(void *, const Logits *, const Policy *, void *);

PyObject *g_dtype, *g_is_cuda, *g_get_device, *g_shape, *g_stride;      // names

// The entry points, torch's types (of values by their numbers there, and of labels), and the device that all tensors and the current stream
// have to be on, by its index; -1: tensors on any.
struct StepCalls {
    PyObject_HEAD
    PyObject *kinds[3], *int64;
    long device;
    token_logp_fn token_logp;
    policy_loss_fn policy_loss;
    grad_norm_fn grad_norm, grad_clip;
    adamw_fn adamw;
};
bool is_true(PyObject *o, PyObject *name)
{
    PyObject *x = PyObject_GetAttr(o, name);
    Py_XDECREF(x);                    // (a bool: the interpreter's own)
    return x == Py_True;
}
bool is_here(const StepCalls *c, PyObject *o)
{
    if (c->device < 0) return is_true(o, g_is_cuda);
    PyObject *d = PyObject_CallMethodNoArgs(o, g_get_device);
    const long at = d ? PyLong_AsLong(d) : -1;        // (host memory: -1)
    Py_XDECREF(d);
    return at == c->device;
}
// the current stream, if the device that it is on is the one
bool stream_here(const StepCalls *c, PyObject *callable, void **p)
{
    if (c->device < 0 || Py_TYPE(callable) != &RawStreamType) return stream_of(callable, p);
    const RawStream *r = reinterpret_cast<const RawStream *>(callable);
    PyObject *d = PyObject_CallNoArgs(r->device);
    if (!d) return false;
    PyObject *s = PyLong_AsLong(d) == c->device ? PyObject_CallOneArg(r->get, d) : nullptr;
    Py_DECREF(d);
    if (!s) return false;
    const bool ok = address(s, p);
    Py_DECREF(s);
    return ok;
}
// whether the tensor's type is `kind`
bool of_kind(PyObject *o, PyObject *kind)
{
    PyObject *x = PyObject_GetAttr(o, g_dtype);
    Py_XDECREF(x);                    // (torch's types live as long as torch)
    return x && x == kind;
}
// sizes and strides of a tensor of n dimensions
bool layout(PyObject *o, int n, int64_t *size, int64_t *step)
{
    PyObject *shape = PyObject_GetAttr(o, g_shape), *stride = shape ? PyObject_CallMethodNoArgs(o, g_stride) : nullptr;
    bool ok = shape && stride && PyTuple_Check(shape) && PyTuple_Check(stride) && PyTuple_GET_SIZE(shape) == n && PyTuple_GET_SIZE(stride) == n;
    for (int i = 0; ok && i < n; ++i) {
        size[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
        step[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i));
        ok = !PyErr_Occurred();
    }
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    return ok;
}
// a device tensor of one dimension, `count` contiguous elements of a type; None only where allowed
bool vector(const StepCalls *c, PyObject *o, int64_t count, PyObject *kind, const void **p, bool optional = false)
{
    *p = nullptr;
    if (o == Py_None) return optional;
    int64_t size, step;
    void *at;
    if (!of_kind(o, kind) || !is_here(c, o) || !layout(o, 1, &size, &step) || size != count || (step != 1 && size > 1) || !tensor(o, &at)) return false;
    *p = at;
    return true;
}
// rows of contiguous elements: their type's number, or -1
int matrix(const StepCalls *c, PyObject *o, int64_t *size, int64_t *stride, void **p)
{
    int64_t step[2];
    PyObject *kind = PyObject_GetAttr(o, g_dtype);
    int k = 0;
    while (k < 3 && c->kinds[k] != kind) ++k;
    Py_XDECREF(kind);
    if (!kind || k == 3 || !is_here(c, o) || !layout(o, 2, size, step) || (step[1] != 1 && size[1] > 1) || !tensor(o, p)) return -1;
    *stride = size[0] > 1 || step[0] > size[1] ? step[0] : size[1];
    return k;
}
bool number(PyObject *o, float *f)
{
    if (!PyFloat_CheckExact(o)) return false;
    *f = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
bool logits_of(const StepCalls *c, PyObject *logits, PyObject *labels, PyObject *temperature, Logits *x)
{
    int64_t size[2];
    void *at;
    x->dtype = matrix(c, logits, size, &x->stride, &at);
    if (x->dtype < 0) return false;
    x->logits = at;
    x->rows = size[0];
    x->vocab = size[1];
    return vector(c, labels, size[0], c->int64, &x->labels) && number(temperature, &x->temperature);
}
// (handle, logits, labels, log-probabilities, temperature, the stream's callable)
PyObject *token_logp(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const StepCalls *c = reinterpret_cast<const StepCalls *>(self);
    void *handle, *stream;
    const void *logp;
    Logits x;
    if (n != 6 || !address(a[0], &handle) || !logits_of(c, a[1], a[2], a[4], &x) || !vector(c, a[3], x.rows, c->kinds[0], &logp) || !stream_here(c, a[5], &stream)) return other();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->token_logp(handle, &x, const_cast<void *>(logp), stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
// (handle, logits, labels, old_logp, advantages, weights, ref_logp, clip_low, clip_high, kl_coef, temperature, grad_scale, sums, logp, dlogits, the
// stream's callable)
PyObject *policy_loss(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const StepCalls *c = reinterpret_cast<const StepCalls *>(self);
    void *handle, *stream;
    const void *sums, *logp;
    Logits x;
    Policy p;
    PyObject *f32 = c->kinds[0];
    if (n != 16 || !address(a[0], &handle) || !logits_of(c, a[1], a[2], a[10], &x) || !vector(c, a[3], x.rows, f32, &p.old_logp) ||
        !vector(c, a[4], x.rows, f32, &p.advantages) || !vector(c, a[5], x.rows, f32, &p.weights, true) || !vector(c, a[6], x.rows, f32, &p.ref_logp, true) ||
        !number(a[7], &p.clip_low) || !number(a[8], &p.clip_high) || !number(a[9], &p.kl_coef) || !number(a[11], &p.grad_scale) ||
        !vector(c, a[12], 8, f32, &sums) || !vector(c, a[13], x.rows, f32, &logp, true)) return other();
    p.sums = const_cast<void *>(sums);
    p.logp = const_cast<void *>(logp);
    p.dlogits = nullptr;
    p.dlogits_stride = 0;
    if (a[14] != Py_None) {
        int64_t size[2];
        if (matrix(c, a[14], size, &p.dlogits_stride, &p.dlogits) != x.dtype || size[0] != x.rows || size[1] != x.vocab) return other();
    }
    if (!stream_here(c, a[15], &stream)) return other();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->policy_loss(handle, &x, &p, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
// (handle, scale, max_norm, the record, the stream's callable)
PyObject *norm_by(PyObject *self, PyObject *const *a, Py_ssize_t n, bool clip)
{
    const StepCalls *c = reinterpret_cast<const StepCalls *>(self);
    void *handle, *stream;
    const void *out;
    float scale, most;
    if (n != 5 || !address(a[0], &handle) || !number(a[1], &scale) || !number(a[2], &most) || !vector(c, a[3], 2, c->kinds[0], &out) || !stream_here(c, a[4], &stream)) return other();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = (clip ? c->grad_clip : c->grad_norm)(handle, scale, most, const_cast<void *>(out), stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
PyObject *grad_norm(PyObject *self, PyObject *const *a, Py_ssize_t n) { return norm_by(self, a, n, false); }
PyObject *grad_clip(PyObject *self, PyObject *const *a, Py_ssize_t n) { return norm_by(self, a, n, true); }
// (handle, step, lr, beta1, beta2, eps, weight_decay, coefficient or None, the stream's callable)
PyObject *adamw_by(const StepCalls *c, adamw_fn fn, PyObject *const *a, Py_ssize_t n)
{
    void *handle, *stream;
    const void *coef;
    Adamw w;
    double *const at[] = {&w.lr, &w.beta1, &w.beta2, &w.eps, &w.weight_decay};
    if (n != 9 || !address(a[0], &handle) || !PyLong_Check(a[1])) return other();
    w.step = PyLong_AsLongLong(a[1]);
    if (w.step == -1 && PyErr_Occurred()) return other();
    for (int k = 0; k < 5; ++k) {
        if (!PyFloat_CheckExact(a[2 + k])) return other();
        *at[k] = PyFloat_AS_DOUBLE(a[2 + k]);
    }
    if (!vector(c, a[7], 1, c->kinds[0], &coef, true) || !stream_here(c, a[8], &stream)) return other();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(handle, &w, coef, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
PyObject *adamw(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const StepCalls *c = reinterpret_cast<const StepCalls *>(self);
    return adamw_by(c, c->adamw, a, n);
}
// StepCalls(float32, bfloat16, float16, int64, addresses of mc_token_logp, mc_policy_loss, mc_grad_norm, mc_grad_clip, mc_adamw)
PyObject *step_calls_new(PyTypeObject *type, PyObject *args, PyObject *)
{
    PyObject *kinds[4] = {};
    unsigned long long at[5] = {};
    if (!PyArg_ParseTuple(args, "OOOOKKKKK", &kinds[0], &kinds[1], &kinds[2], &kinds[3], &at[0], &at[1], &at[2], &at[3], &at[4])) return nullptr;
    StepCalls *c = reinterpret_cast<StepCalls *>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    for (PyObject *k : kinds) Py_INCREF(k);
    for (int k = 0; k < 3; ++k) c->kinds[k] = kinds[k];
    c->int64 = kinds[3];
    c->device = -1;
    c->token_logp = (token_logp_fn)(uintptr_t)at[0];
    c->policy_loss = (policy_loss_fn)(uintptr_t)at[1];
    c->grad_norm = (grad_norm_fn)(uintptr_t)at[2];
    c->grad_clip = (grad_norm_fn)(uintptr_t)at[3];
    c->adamw = (adamw_fn)(uintptr_t)at[4];
    return reinterpret_cast<PyObject *>(c);
}
// the same for the device of this index
PyObject *on(PyObject *self, PyObject *index)
{
    const long device = PyLong_AsLong(index);
    if (device == -1 && PyErr_Occurred()) return nullptr;
    PyObject *copy = Py_TYPE(self)->tp_alloc(Py_TYPE(self), 0);
    if (!copy) return nullptr;
    StepCalls *c = reinterpret_cast<StepCalls *>(copy);
    const StepCalls *from = reinterpret_cast<const StepCalls *>(self);
    for (int k = 0; k < 3; ++k) Py_INCREF(c->kinds[k] = from->kinds[k]);
    Py_INCREF(c->int64 = from->int64);
    c->device = device;
    c->token_logp = from->token_logp;
    c->policy_loss = from->policy_loss;
    c->grad_norm = from->grad_norm;
    c->grad_clip = from->grad_clip;
    c->adamw = from->adamw;
    return copy;
}
void step_calls_gone(PyObject *self)
{
    StepCalls *c = reinterpret_cast<StepCalls *>(self);
    for (PyObject *k : c->kinds) Py_XDECREF(k);
    Py_XDECREF(c->int64);
    Py_TYPE(self)->tp_free(self);
}

// ---- a step in few bits (mx.py) --------------------------------------------------------------------------------------------------------------
// The structures of mergecomp_mx.h.
struct Matrix {
    void *codes, *scales;
    int64_t rows, cols;
};
struct Source {
    const void *data;
    int64_t rows, cols, stride;
    int32_t dtype;
};
struct Result {
    void *out;
    int64_t stride;
    int32_t dtype, accumulate;
    const void *bias;
};
typedef int (*quantize_fn)(void *, const Source *, const Matrix *, const Matrix *, void *, int64_t, void *);
typedef int (*matmul_fn)(void *, const Matrix *, const Matrix *, const Result *, void *);

PyObject *g_at, *g_index;             // names

// The entry points, and the type of quantised matrices, whose structure lies at the attribute `_at` and whose device has the index `_index`.
struct MxCalls {
    StepCalls base;                   // types and device
    PyTypeObject *matrix;
    quantize_fn quantize;
    matmul_fn matmul;
    adamw_fn adamw8;
};
bool quantised(const MxCalls *c, PyObject *o, const Matrix **m)
{
    if (Py_TYPE(o) != c->matrix) return false;
    PyObject *i = PyObject_GetAttr(o, g_index), *a = i ? PyObject_GetAttr(o, g_at) : nullptr;
    void *p = nullptr;
    const bool ok = a && PyLong_Check(i) && PyLong_AsLong(i) == c->base.device && address(a, &p) && p;
    Py_XDECREF(i);
    Py_XDECREF(a);
    *m = static_cast<const Matrix *>(p);
    return ok;
}
// (handle, x, by_rows or None, by_cols or None, values or None, the stream's callable)
PyObject *quantize(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const MxCalls *c = reinterpret_cast<const MxCalls *>(self);
    void *handle, *stream, *at, *values = nullptr;
    const Matrix *rows = nullptr, *cols = nullptr;
    int64_t size[2], vsize[2], vstride = 0;
    Source x;
    if (n != 6 || !address(a[0], &handle)) return other();
    x.dtype = matrix(&c->base, a[1], size, &x.stride, &at);
    if (x.dtype < 0) return other();
    x.data = at;
    x.rows = size[0];
    x.cols = size[1];
    if (a[2] != Py_None && (!quantised(c, a[2], &rows) || rows->rows != x.rows || rows->cols != x.cols)) return other();
    if (a[3] != Py_None && (!quantised(c, a[3], &cols) || cols->rows != x.cols || cols->cols != x.rows)) return other();
    if (a[4] != Py_None && (matrix(&c->base, a[4], vsize, &vstride, &values) != x.dtype || vsize[0] != x.rows || vsize[1] != x.cols)) return other();
    if (!stream_here(&c->base, a[5], &stream)) return other();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->quantize(handle, &x, rows, cols, values, vstride, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
// (handle, a, b, out, bias or None, accumulate, the stream's callable)
PyObject *matmul(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const MxCalls *c = reinterpret_cast<const MxCalls *>(self);
    void *handle, *stream, *out;
    const Matrix *x, *w;
    int64_t size[2];
    Result y;
    if (n != 7 || !address(a[0], &handle) || !quantised(c, a[1], &x) || !quantised(c, a[2], &w) || (a[5] != Py_False && a[5] != Py_True)) return other();
    y.dtype = matrix(&c->base, a[3], size, &y.stride, &out);
    if (y.dtype < 0 || size[0] != x->rows || size[1] != w->rows || x->cols != w->cols) return other();
    y.out = out;
    y.accumulate = a[5] == Py_True;
    if (!vector(&c->base, a[4], size[1], c->base.kinds[0], &y.bias, true) || !stream_here(&c->base, a[6], &stream)) return other();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = c->matmul(handle, x, w, &y, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
PyObject *adamw8(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const MxCalls *c = reinterpret_cast<const MxCalls *>(self);
    return adamw_by(&c->base, c->adamw8, a, n);
}
// MxCalls(float32, bfloat16, float16, the matrices' type, device index, addresses of mc_mx_quantize, mc_mx_matmul, mc_adamw8)
PyObject *mx_calls_new(PyTypeObject *type, PyObject *args, PyObject *)
{
    PyObject *kinds[3] = {}, *matrix = nullptr;
    long device = 0;
    unsigned long long at[3] = {};
    if (!PyArg_ParseTuple(args, "OOOO!lKKK", &kinds[0], &kinds[1], &kinds[2], &PyType_Type, &matrix, &device, &at[0], &at[1], &at[2])) return nullptr;
    MxCalls *c = reinterpret_cast<MxCalls *>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    for (int k = 0; k < 3; ++k) Py_INCREF(c->base.kinds[k] = kinds[k]);
    Py_INCREF(matrix);
    c->matrix = reinterpret_cast<PyTypeObject *>(matrix);
    c->base.device = device;
    c->quantize = (quantize_fn)(uintptr_t)at[0];
    c->matmul = (matmul_fn)(uintptr_t)at[1];
    c->adamw8 = (adamw_fn)(uintptr_t)at[2];
    return reinterpret_cast<PyObject *>(c);
}
void mx_calls_gone(PyObject *self)
{
    MxCalls *c = reinterpret_cast<MxCalls *>(self);
    for (PyObject *k : c->base.kinds) Py_XDECREF(k);
    Py_XDECREF(reinterpret_cast<PyObject *>(c->matrix));
    Py_TYPE(self)->tp_free(self);
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef calls_methods[] = {FAST(compress), FAST(compress_static), FAST(decompress), FAST(compress_groups), FAST(decompress_groups), {nullptr, nullptr, 0, nullptr}};
PyMethodDef step_calls_methods[] = {FAST(token_logp), FAST(policy_loss), FAST(grad_norm), FAST(grad_clip), FAST(adamw), {"on", on, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyMethodDef mx_calls_methods[] = {FAST(quantize), FAST(matmul), FAST(adamw8), {nullptr, nullptr, 0, nullptr}};
PyTypeObject MxCallsType = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyTypeObject CallsType = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyTypeObject StepCallsType = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyTypeObject RawStreamType = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", "The hot calls of the binding without ctypes.", -1, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void)
{
    const struct { PyObject **at; const char *name; } names[] = {{&g_data_ptr, "data_ptr"}, {&g_dtype, "dtype"}, {&g_is_cuda, "is_cuda"}, {&g_get_device, "get_device"}, {&g_shape, "shape"}, {&g_stride, "stride"}, {&g_at, "_at"}, {&g_index, "_index"}};
    for (const auto &n : names) if (!*n.at && !(*n.at = PyUnicode_InternFromString(n.name))) return nullptr;
    CallsType.tp_name = "_fastcall.Calls";
    CallsType.tp_basicsize = sizeof(Calls);
    CallsType.tp_flags = Py_TPFLAGS_DEFAULT;
    CallsType.tp_new = calls_new;
    CallsType.tp_dealloc = calls_gone;
    CallsType.tp_methods = calls_methods;
    RawStreamType.tp_name = "_fastcall.RawStream";
    RawStreamType.tp_basicsize = sizeof(RawStream);
    RawStreamType.tp_flags = Py_TPFLAGS_DEFAULT;
    RawStreamType.tp_new = raw_stream_new;
    RawStreamType.tp_dealloc = raw_stream_gone;
    RawStreamType.tp_call = raw_stream_call;
    StepCallsType.tp_name = "_fastcall.StepCalls";
    StepCallsType.tp_basicsize = sizeof(StepCalls);
    StepCallsType.tp_flags = Py_TPFLAGS_DEFAULT;
    StepCallsType.tp_new = step_calls_new;
    StepCallsType.tp_dealloc = step_calls_gone;
    StepCallsType.tp_methods = step_calls_methods;
    MxCallsType.tp_name = "_fastcall.MxCalls";
    MxCallsType.tp_basicsize = sizeof(MxCalls);
    MxCallsType.tp_flags = Py_TPFLAGS_DEFAULT;
    MxCallsType.tp_new = mx_calls_new;
    MxCallsType.tp_dealloc = mx_calls_gone;
    MxCallsType.tp_methods = mx_calls_methods;
    if (PyType_Ready(&MxCallsType) < 0 || PyType_Ready(&CallsType) < 0 || PyType_Ready(&RawStreamType) < 0 || PyType_Ready(&StepCallsType) < 0) return nullptr;
    PyObject *m = PyModule_Create(&module);
    if (!m) return nullptr;
    if (PyModule_AddObjectRef(m, "Calls", reinterpret_cast<PyObject *>(&CallsType)) < 0 ||
        PyModule_AddObjectRef(m, "MxCalls", reinterpret_cast<PyObject *>(&MxCallsType)) < 0 ||
        PyModule_AddObjectRef(m, "StepCalls", reinterpret_cast<PyObject *>(&StepCallsType)) < 0 ||
        PyModule_AddObjectRef(m, "RawStream", reinterpret_cast<PyObject *>(&RawStreamType)) < 0) { Py_DECREF(m); return nullptr; }
    return m;
}
