// Argument marshalling of the entry points beside the layer (binding.py): checks torch tensors, makes missing outputs and calls the C
// ABI.  A decode step makes these calls once a layer each, on kernels of a few microseconds; the same checks by attribute from Python take
// longer than the kernels (plan_cache, rotate, rotate_append and attend through ctypes 9.4, 10.3, 12.9 and 9.5 us a call with its launch,
// here 4.6, 4.6, 5.4 and 4.7 on the host).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

namespace {

using at::Tensor;

// the C ABI (include/lookupffn.h), as addresses that binding.py has from the loaded library
using PlanFn = int (*)(const void *, const void *, const void *, void *, void *, void *, void *, void *, void *, int, int64_t, int, int64_t,
                       int64_t, int, void *);
using RotateFn = int (*)(const void *, const void *, const void *, const void *, const void *, const void *, void *, void *, int64_t, int, int,
                         int, int, int64_t, const int64_t *, float, int, int, void *);
using AppendFn = int (*)(const void *, const void *, const void *, const void *, const void *, const void *, const void *, const void *, void *,
                         void *, void *, void *, void *, int64_t, int, int, int, int, int64_t, int64_t, int, const int64_t *, float, int, int,
                         void *);
using AttendFn = int (*)(const void *, const void *, const void *, const void *, const void *, const void *, const void *, const void *, void *,
                         int64_t, int, int, int, int, int64_t, int, int, int64_t, const int64_t *, int64_t, int64_t, int, int, int, void *,
                         int64_t, void *);
PlanFn g_plan = nullptr;
RotateFn g_rotate = nullptr;
AppendFn g_append = nullptr;
AttendFn g_attend = nullptr;
PyObject *g_stream_of = nullptr;   // device index -> raw stream
PyObject *g_check = nullptr;       // status -> None, or raises

struct PythonError {};   // a Python error is set

[[noreturn]] void fail(PyObject *type, const char *format, ...)
{
    va_list args;
    va_start(args, format);
    PyErr_FormatV(type, format, args);
    va_end(args);
    throw PythonError();
}

const Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s must be a tensor", name);
    return THPVariable_Unpack(o);
}
Tensor maybe(PyObject *o, const char *name) { return o == Py_None ? Tensor() : tensor(o, name); }

void of_type(const Tensor &t, const char *name, at::ScalarType type)
{
    if (t.scalar_type() != type) fail(PyExc_TypeError, "%s must be %s, got %s", name, c10::toString(type), c10::toString(t.scalar_type()));
}
// `home`: the call's device, where its first tensor is
void *on_gpu(const Tensor &t, const char *name, at::Device home)
{
    if (!t.is_cuda()) fail(PyExc_ValueError, "%s must live on the GPU", name);
    if (t.device() != home) fail(PyExc_ValueError, "%s lives on %s, the call's device is %s", name, t.device().str().c_str(), home.str().c_str());
    return t.data_ptr();
}
void *dense(const Tensor &t, const char *name, at::Device home)
{
    if (!t.is_contiguous()) fail(PyExc_ValueError, "%s must be contiguous", name);
    return on_gpu(t, name, home);
}
void shaped(const Tensor &t, const char *name, at::IntArrayRef shape)
{
    if (t.sizes() == shape) return;
    std::string got, want;
    for (int64_t v : t.sizes()) got += (got.empty() ? "" : ", ") + std::to_string(v);
    for (int64_t v : shape) want += (want.empty() ? "" : ", ") + std::to_string(v);
    fail(PyExc_ValueError, "%s has shape (%s), expected (%s)", name, got.c_str(), want.c_str());
}
void *ints(const Tensor &t, const char *name, at::IntArrayRef shape, at::Device home)
{
    of_type(t, name, at::kInt);
    shaped(t, name, shape);
    return dense(t, name, home);
}
// rows [tokens][heads][dim] of any strides, columns dense
void *rows(const Tensor &t, const char *name, at::IntArrayRef shape, at::ScalarType type, at::Device home)
{
    of_type(t, name, type);
    shaped(t, name, shape);
    void *p = on_gpu(t, name, home);
    if (t.stride(2) != 1) fail(PyExc_ValueError, "the columns of %s must be dense", name);
    return p;
}
int dtype_code(const Tensor &t)
{
    switch (t.scalar_type()) {
        case at::kFloat: return 0;
        case at::kBFloat16: return 1;
        case at::kHalf: return 2;
        default: fail(PyExc_TypeError, "expected float32, bfloat16 or float16, got %s", c10::toString(t.scalar_type()));
    }
}
void *row_weight(const Tensor &w, const char *name, int64_t dim, at::Device home)
{
    if (!w.defined()) return nullptr;
    of_type(w, name, at::kFloat);
    shaped(w, name, {dim});
    return dense(w, name, home);
}
void three(const Tensor &t, const char *name)
{
    if (t.dim() != 3) fail(PyExc_ValueError, "%s must be [tokens][heads][dim]", name);
}

int64_t whole(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    return v;
}
int small(PyObject *o)
{
    const int64_t v = whole(o);
    if (v < INT32_MIN || v > INT32_MAX) fail(PyExc_OverflowError, "%lld does not fit an int", (long long)v);
    return (int)v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v != 0;
}

void *stream_of(const Tensor &t)
{
    PyObject *index = PyLong_FromLong(t.get_device());
    PyObject *s = index ? PyObject_CallOneArg(g_stream_of, index) : nullptr;
    Py_XDECREF(index);
    if (!s) throw PythonError();
    void *p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!p && PyErr_Occurred()) throw PythonError();
    return p;
}
void checked(int status)
{
    if (status == 0) return;
    PyObject *r = PyObject_CallFunction(g_check, "i", status);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "lookupffn status %d", status);
    throw PythonError();
}

struct Rotation {
    const void *angles = nullptr, *positions = nullptr;
    int rot = 0;
    int64_t n_positions = 0;
    Rotation(PyObject *a, PyObject *p, int64_t n, at::Device home)
    {
        if (a == Py_None) return;
        const Tensor &t = tensor(a, "angles");
        if (t.scalar_type() != at::kFloat || t.dim() != 2) fail(PyExc_TypeError, "angles must be float32 [positions][rot]");
        if (p == Py_None) fail(PyExc_ValueError, "angles need positions");
        angles = dense(t, "angles", home);
        positions = ints(tensor(p, "positions"), "positions", {n}, home);
        rot = (int)t.size(1);
        n_positions = t.size(0);
    }
};

struct Cache {
    int64_t n_blocks;
    int block;
    void *k, *v, *ks, *vs;
    Cache(const Tensor &kc, const Tensor &vc, const Tensor &k_scale, const Tensor &v_scale, int64_t kv_heads, int64_t dim,
          at::Device home)
    {
        of_type(kc, "k_cache", at::kFloat8_e4m3fn);
        of_type(vc, "v_cache", at::kFloat8_e4m3fn);
        if (kc.dim() != 4) fail(PyExc_ValueError, "k_cache must be [blocks][kv heads][block][dim]");
        n_blocks = kc.size(0);
        const int64_t b = kc.size(2);
        shaped(kc, "k_cache", {n_blocks, kv_heads, b, dim});
        shaped(vc, "v_cache", {n_blocks, kv_heads, dim, b});
        of_type(k_scale, "k_scale", at::kFloat);
        of_type(v_scale, "v_scale", at::kFloat);
        shaped(k_scale, "k_scale", {n_blocks, kv_heads});
        shaped(v_scale, "v_scale", {n_blocks, kv_heads});
        block = (int)b;
        k = dense(kc, "k_cache", home);
        v = dense(vc, "v_cache", home);
        ks = dense(k_scale, "k_scale", home);
        vs = dense(v_scale, "v_scale", home);
    }
};

PyObject *tuple_of(std::initializer_list<Tensor> ts)
{
    PyObject *out = PyTuple_New((Py_ssize_t)ts.size());
    if (!out) throw PythonError();
    Py_ssize_t i = 0;
    for (const Tensor &t : ts) PyTuple_SET_ITEM(out, i++, THPVariable_Wrap(t));
    return out;
}

// plan_cache(past, fresh, free, table, n_tokens, block, starts, lengths, slots, positions, counts)
PyObject *plan_cache(PyObject *const *a)
{
    const Tensor &past = tensor(a[0], "past"), &fresh = tensor(a[1], "fresh"), &free = tensor(a[2], "free"), &table = tensor(a[3], "table");
    if (past.dim() != 1) fail(PyExc_ValueError, "past must be a list of counts");
    const int64_t requests = past.size(0), n_tokens = whole(a[4]);
    if (table.scalar_type() != at::kInt || table.dim() != 2 || table.size(0) != requests)
        fail(PyExc_TypeError, "table must be int32 [%lld][blocks of a request]", (long long)requests);
    if (free.dim() != 1) fail(PyExc_ValueError, "free must be a list of blocks");
    if (n_tokens < 0) fail(PyExc_ValueError, "n_tokens must not be negative");
    const at::Device home = past.device();
    void *p_past = ints(past, "past", {requests}, home), *p_fresh = ints(fresh, "fresh", {requests}, home);
    void *p_free = ints(free, "free", {free.size(0)}, home), *p_table = ints(table, "table", {requests, table.size(1)}, home);
    const char *names[5] = {"starts", "lengths", "slots", "positions", "counts"};
    const int64_t sizes[5] = {requests + 1, requests, n_tokens, n_tokens, 2};
    Tensor out[5];
    void *p[5];
    for (int i = 0; i < 5; ++i) {
        out[i] = a[6 + i] == Py_None ? at::empty({sizes[i]}, past.options()) : tensor(a[6 + i], names[i]);
        p[i] = ints(out[i], names[i], {sizes[i]}, home);
    }
    const c10::DeviceGuard guard(home);
    checked(g_plan(p_past, p_fresh, p_free, p_table, p[0], p[1], p[2], p[3], p[4], (int)requests, free.size(0), (int)table.size(1),
                   table.size(1), n_tokens, small(a[5]), stream_of(past)));
    return tuple_of({out[0], out[1], out[2], out[3], out[4]});
}

// rotate(q, k, q_weight, k_weight, angles, positions, q_out, k_out, eps, interleaved)
PyObject *rotate(PyObject *const *a)
{
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k");
    three(q, "q");
    three(k, "k");
    const int64_t n = q.size(0), heads = q.size(1), dim = q.size(2), kv = k.size(1);
    const at::ScalarType type = q.scalar_type();
    const int code = dtype_code(q);
    const at::Device home = q.device();
    void *pq = rows(q, "q", {n, heads, dim}, type, home), *pk = rows(k, "k", {n, kv, dim}, type, home);
    void *qw = row_weight(maybe(a[2], "q_weight"), "q_weight", dim, home), *kw = row_weight(maybe(a[3], "k_weight"), "k_weight", dim, home);
    const Rotation r(a[4], a[5], n, home);
    const Tensor qo = a[6] == Py_None ? at::empty({n, heads, dim}, q.options()) : tensor(a[6], "q_out");
    const Tensor ko = a[7] == Py_None ? at::empty({n, kv, dim}, q.options()) : tensor(a[7], "k_out");
    void *pqo = rows(qo, "q_out", {n, heads, dim}, type, home), *pko = rows(ko, "k_out", {n, kv, dim}, type, home);
    if (n) {
        const int64_t strides[8] = {q.stride(0), q.stride(1), k.stride(0), k.stride(1), qo.stride(0), qo.stride(1), ko.stride(0), ko.stride(1)};
        const double eps = PyFloat_AsDouble(a[8]);
        if (eps == -1.0 && PyErr_Occurred()) throw PythonError();
        const c10::DeviceGuard guard(home);
        checked(g_rotate(pq, pk, qw, kw, r.angles, r.positions, pqo, pko, n, (int)heads, (int)kv, (int)dim, r.rot, r.n_positions, strides,
                         (float)eps, truth(a[9]), code, stream_of(q)));
    }
    return tuple_of({qo, ko});
}

// rotate_append(q, k, v, q_weight, k_weight, angles, positions, slots, k_cache, v_cache, k_scale, v_scale, q_out, eps, interleaved)
PyObject *rotate_append(PyObject *const *a)
{
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    three(q, "q");
    three(k, "k");
    const int64_t n = q.size(0), heads = q.size(1), dim = q.size(2), kv = k.size(1);
    const at::ScalarType type = q.scalar_type();
    const int code = dtype_code(q);
    const at::Device home = q.device();
    void *pq = rows(q, "q", {n, heads, dim}, type, home), *pk = rows(k, "k", {n, kv, dim}, type, home), *pv = rows(v, "v", {n, kv, dim}, type, home);
    void *qw = row_weight(maybe(a[3], "q_weight"), "q_weight", dim, home), *kw = row_weight(maybe(a[4], "k_weight"), "k_weight", dim, home);
    const Rotation r(a[5], a[6], n, home);
    void *slots = ints(tensor(a[7], "slots"), "slots", {n}, home);
    const Cache c(tensor(a[8], "k_cache"), tensor(a[9], "v_cache"), tensor(a[10], "k_scale"), tensor(a[11], "v_scale"), kv, dim, home);
    const Tensor qo = a[12] == Py_None ? at::empty({n, heads, dim}, q.options()) : tensor(a[12], "q_out");
    void *pqo = rows(qo, "q_out", {n, heads, dim}, type, home);
    if (n) {
        const int64_t strides[8] = {q.stride(0), q.stride(1), k.stride(0), k.stride(1), v.stride(0), v.stride(1), qo.stride(0), qo.stride(1)};
        const double eps = PyFloat_AsDouble(a[13]);
        if (eps == -1.0 && PyErr_Occurred()) throw PythonError();
        const c10::DeviceGuard guard(home);
        checked(g_append(pq, pk, pv, qw, kw, r.angles, r.positions, slots, pqo, c.k, c.v, c.ks, c.vs, n, (int)heads, (int)kv, (int)dim, r.rot,
                         r.n_positions, c.n_blocks, c.block, strides, (float)eps, truth(a[14]), code, stream_of(q)));
    }
    return THPVariable_Wrap(qo);
}

// attend(q, k_cache, v_cache, k_scale, v_scale, table, starts, lengths, y, causal, window, max_queries, max_keys, workspace)
PyObject *attend(PyObject *const *a)
{
    const Tensor &q = tensor(a[0], "q"), &kc = tensor(a[1], "k_cache"), &table = tensor(a[5], "table"), &lengths = tensor(a[7], "lengths");
    three(q, "q");
    if (kc.dim() != 4) fail(PyExc_ValueError, "k_cache must be [blocks][kv heads][block][dim]");
    if (lengths.dim() != 1) fail(PyExc_ValueError, "lengths must be a list of counts");
    const int64_t n = q.size(0), heads = q.size(1), dim = q.size(2), kv = kc.size(1), requests = lengths.size(0);
    if (table.dim() != 2 || table.size(0) != requests)
        fail(PyExc_ValueError, "table must be [%lld][blocks of a request]", (long long)requests);
    const at::ScalarType type = q.scalar_type();
    const int code = dtype_code(q);
    const at::Device home = q.device();
    void *pq = rows(q, "q", {n, heads, dim}, type, home);
    const Tensor y = a[8] == Py_None ? at::empty({n, heads, dim}, q.options()) : tensor(a[8], "y");
    void *py = rows(y, "y", {n, heads, dim}, type, home);
    const Cache c(kc, tensor(a[2], "v_cache"), tensor(a[3], "k_scale"), tensor(a[4], "v_scale"), kv, dim, home);
    void *pt = ints(table, "table", {requests, table.size(1)}, home);
    void *ps = ints(tensor(a[6], "starts"), "starts", {requests + 1}, home), *pl = ints(lengths, "lengths", {requests}, home);
    if (n) {
        const int64_t max_queries = a[11] == Py_None ? n : whole(a[11]);
        const int64_t max_keys = a[12] == Py_None ? table.size(1) * c.block : whole(a[12]);
        const Tensor ws = maybe(a[13], "workspace");
        void *pw = ws.defined() ? dense(ws, "workspace", home) : nullptr;
        const int64_t strides[4] = {q.stride(0), q.stride(1), y.stride(0), y.stride(1)};
        const c10::DeviceGuard guard(home);
        checked(g_attend(pq, c.k, c.v, c.ks, c.vs, pt, ps, pl, py, n, (int)requests, (int)heads, (int)kv, (int)dim, c.n_blocks, c.block,
                         (int)table.size(1), table.size(1), strides, max_queries, max_keys, truth(a[9]), small(a[10]), code, pw,
                         ws.defined() ? (int64_t)ws.nbytes() : 0, stream_of(q)));
    }
    return THPVariable_Wrap(y);
}

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != N) return PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
    try {
        return F(args);
    } catch (const PythonError &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// bind(plan_cache, rotate, rotate_append, attend, stream_of, check): the C ABI's addresses, and the two calls back into Python
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) return PyErr_Format(PyExc_TypeError, "expected 6 arguments, got %zd", n);
    void *p[4];
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is 0");
            return nullptr;
        }
    }
    g_plan = reinterpret_cast<PlanFn>(p[0]);
    g_rotate = reinterpret_cast<RotateFn>(p[1]);
    g_append = reinterpret_cast<AppendFn>(p[2]);
    g_attend = reinterpret_cast<AttendFn>(p[3]);
    Py_INCREF(args[4]);
    Py_INCREF(args[5]);
    Py_XSETREF(g_stream_of, args[4]);
    Py_XSETREF(g_check, args[5]);
    Py_RETURN_NONE;
}

template <class F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"bind", fast(&bind), METH_FASTCALL, nullptr},
                         {"plan_cache", fast(&entry<plan_cache, 11>), METH_FASTCALL, nullptr},
                         {"rotate", fast(&entry<rotate, 10>), METH_FASTCALL, nullptr},
                         {"rotate_append", fast(&entry<rotate_append, 15>), METH_FASTCALL, nullptr},
                         {"attend", fast(&entry<attend, 14>), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
