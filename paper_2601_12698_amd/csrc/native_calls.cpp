// The hot entry points as one native call from Python (module _native): the checks of binding.py on torch's own tensors, the
// current stream, and the C entry point, whose address binding.py hands over.
//
// A decode step is a launch of 2.7 us, and the same in Python and ctypes took 4.9 us: fifteen attribute and method calls on
// tensors, one on the stream, the conversion of nine arguments.  Here they are some dozens of loads (3.0 us with the launch).
//
// Each function returns the status of the entry point, or None for what it does not take: a stream that was named, objects
// that are not exactly what is usual (a tensor subclass, a numpy integer), and everything that is to be refused.  binding.py
// then goes its general way, which knows all cases and has the words.
//
// torch's objects are read where the headers of the build say, so the module names the torch it was built for, and binding.py
// does without it where that is another one.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "prefixattn.h"
#include "rotary.h"

namespace {

using RunFn = int (*)(void*, void*, const void*, float, int64_t, int64_t, int, const void*, void*);
using SiluFn = int (*)(const void*, void*, int64_t, int64_t, int, const void*, void*);
using MergeFn = int (*)(const void*, const float*, const void*, const float*, void*, float*, int64_t, int64_t, int, const void*, void*);
using GateFn = int (*)(const void*, const void*, const void*, const void*, int64_t, int, uint32_t, void*, void*);

RunFn g_run;
SiluFn g_silu;
MergeFn g_merge;
GateFn g_gate;
PyObject* g_formats;                                         // dict: name of a storage format -> its number
PyTypeObject* g_cfg;                                         // binding.Cfg

constexpr at::ScalarType kX[] = {at::kBFloat16, at::kHalf, at::kHalf, at::kFloat};
constexpr at::ScalarType kR[] = {at::kBFloat16, at::kHalf, at::kFloat, at::kFloat};

bool whole(PyObject* o, int64_t* out)
{
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    *out = PyLong_AsLongLongAndOverflow(o, &over);
    return over == 0;
}
bool format(PyObject* o, int* out)
{
    int64_t v = -1;
    if (PyUnicode_CheckExact(o)) o = PyDict_GetItem(g_formats, o);               // borrowed; no error is raised
    if (!o || !whole(o, &v) || v < 0 || v > 3) return false;
    *out = static_cast<int>(v);
    return true;
}
// A configuration's eight integers, from where ctypes keeps them; NULL for None.
bool configuration(PyObject* o, const void** out)
{
    *out = nullptr;
    if (o == Py_None) return true;
    if (Py_TYPE(o) != g_cfg) return false;
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) { PyErr_Clear(); return false; }
    *out = b.buf;                                            // lives as long as the object, which the caller holds
    PyBuffer_Release(&b);
    return true;
}
// The tensor's data, if it has `numel` contiguous elements of `type` on the device.
bool data(PyObject* o, at::ScalarType type, int64_t numel, void** out)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.numel() != numel || !t.is_contiguous()) return false;
    *out = t.data_ptr();
    return true;
}
void* stream_of(PyObject* tensor)
{
    return c10::hip::getCurrentHIPStream(THPVariable_Unpack(tensor).get_device()).stream();
}
PyObject* general() { Py_RETURN_NONE; }

// Runs `call` without the interpreter's lock: a launch waits where the stream's queue is full.
template <class Call>
PyObject* status(Call call)
{
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}
// What torch throws (a tensor without storage, a symbolic size) goes the general way, too.
template <class Body>
PyObject* guarded(Body body)
{
    try {
        return body();
    } catch (...) {
        PyErr_Clear();
        return general();
    }
}

// (x, residual, weight, eps, M, N, dtype, cfg)
PyObject* addrms_run(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int dt;
        int64_t M, N, all;
        void *x, *r, *w;
        const void* cfg;
        if (n != 8 || !g_run || !PyFloat_CheckExact(a[3]) || !whole(a[4], &M) || !whole(a[5], &N) || !format(a[6], &dt) ||
            !configuration(a[7], &cfg) || __builtin_mul_overflow(M, N, &all) || !data(a[0], kX[dt], all, &x) ||
            !data(a[1], kR[dt], all, &r) || !data(a[2], kX[dt], N, &w))
            return general();
        const float eps = static_cast<float>(PyFloat_AS_DOUBLE(a[3]));
        void* s = stream_of(a[0]);
        return status([=] { return g_run(x, r, w, eps, M, N, dt, cfg, s); });
    });
}
// (x, out, M, d, dtype, cfg)
PyObject* silumul_run(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int dt;
        int64_t M, d, all, twice;
        void *x, *out;
        const void* cfg;
        if (n != 6 || !g_silu || !whole(a[2], &M) || !whole(a[3], &d) || !format(a[4], &dt) || !configuration(a[5], &cfg) ||
            __builtin_mul_overflow(M, d, &all) || __builtin_add_overflow(all, all, &twice) || !data(a[0], kX[dt], twice, &x) ||
            !data(a[1], kX[dt], all, &out))
            return general();
        void* s = stream_of(a[0]);
        return status([=] { return g_silu(x, out, M, d, dt, cfg, s); });
    });
}
// (v_a, s_a, v_b, s_b, v_out, s_out, rows, d, dtype, cfg)
PyObject* mergestates_run(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int dt;
        int64_t rows, d, all;
        void* p[6];
        const void* cfg;
        if (n != 10 || !g_merge || !whole(a[6], &rows) || !whole(a[7], &d) || !format(a[8], &dt) || !configuration(a[9], &cfg) ||
            __builtin_mul_overflow(rows, d, &all))
            return general();
        for (int i = 0; i < 6; ++i)
            if (!(i % 2 ? data(a[i], at::kFloat, rows, &p[i]) : data(a[i], kX[dt], all, &p[i]))) return general();
        void* s = stream_of(a[0]);
        return status([=] {
            return g_merge(p[0], static_cast<float*>(p[1]), p[2], static_cast<float*>(p[3]), p[4], static_cast<float*>(p[5]), rows, d,
                           dt, cfg, s);
        });
    });
}
// (y, y_ref, residual, residual_ref, dtype, tol, counts_out)
PyObject* gate_probe_noalloc(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int dt;
        int64_t tol;
        void* p[4];
        if (n != 7 || !g_gate || !format(a[4], &dt) || !whole(a[5], &tol) || tol < 0 || tol > UINT32_MAX || !THPVariable_CheckExact(a[0]) ||
            !THPVariable_CheckExact(a[6]))
            return general();
        const int64_t all = THPVariable_Unpack(a[0]).numel();
        for (int i = 0; i < 4; ++i)
            if (!data(a[i], i < 2 ? kX[dt] : kR[dt], all, &p[i])) return general();
        const at::Tensor& counts = THPVariable_Unpack(a[6]);
        if (!counts.is_cuda() || counts.numel() * static_cast<int64_t>(counts.element_size()) < 16) return general();
        void *out = counts.data_ptr(), *s = stream_of(a[0]);
        return status([=] { return g_gate(p[0], p[1], p[2], p[3], all, dt, static_cast<uint32_t>(tol), out, s); });
    });
}

// ---- the operators around a decode step's attention (serving.py) --------------------------------------------------------------

decltype(&::rotary_run) g_rotary;
decltype(&::kvcache_write) g_write;
decltype(&::kvcache_read) g_read;
decltype(&::prefixattn_run) g_attend;

// A plain device tensor of this type and number of axes, on the device of `as` where one is given.
const at::Tensor* device_tensor(PyObject* o, at::ScalarType type, int64_t axes, const at::Tensor* as = nullptr)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.dim() != axes || (as && t.get_device() != as->get_device())) return nullptr;
    return &t;
}
// Its data, if it is contiguous and has these sizes.
template <class... N>
bool whole_data(PyObject* o, at::ScalarType type, const at::Tensor& as, void** out, N... sizes)
{
    const at::Tensor* t = device_tensor(o, type, sizeof...(N), &as);
    const int64_t want[] = {static_cast<int64_t>(sizes)...};
    if (!t || !t->is_contiguous()) return false;
    for (size_t i = 0; i < sizeof...(N); ++i)
        if (t->size(static_cast<int64_t>(i)) != want[i]) return false;
    *out = t->data_ptr();
    return true;
}
// Data and strides of a [tokens, heads, d] tensor.
struct Heads {
    void* data = nullptr;
    int64_t strides[2] = {0, 0};
};
bool heads_of(PyObject* o, at::ScalarType type, const at::Tensor* as, int64_t tokens, int64_t heads, int64_t d, Heads* out)
{
    const at::Tensor* t = device_tensor(o, type, 3, as);
    if (!t || t->size(0) != tokens || t->size(1) != heads || t->size(2) != d || (t->stride(2) != 1 && d > 1)) return false;
    out->data = t->data_ptr();
    out->strides[0] = t->stride(0);
    out->strides[1] = t->stride(1);
    return true;
}
bool truth(PyObject* o, bool* out)
{
    *out = o == Py_True;
    return o == Py_True || o == Py_False;
}
// A cache: pages and scales as serving.py's _cache takes them.
struct Cache {
    void *k = nullptr, *v = nullptr, *ks = nullptr, *vs = nullptr;
    int64_t pages = 0, heads = 0, page = 0, d = 0;
    int format = KVCACHE_SAME;
};
bool scale_of(PyObject* o, const at::Tensor& as, const Cache& c, void** out)
{
    return whole_data(o, at::kByte, as, out, c.pages, c.heads, c.page) || whole_data(o, at::kFloat8_e8m0fnu, as, out, c.pages, c.heads, c.page);
}
bool cache_of(PyObject* const* a, int dt, const at::Tensor& as, Cache* c)
{
    if (!THPVariable_CheckExact(a[0])) return false;
    const at::Tensor& k = THPVariable_Unpack(a[0]);
    const at::ScalarType type = k.scalar_type();
    const bool codes = type == at::kFloat8_e4m3fn || type == at::kByte;
    if (k.dim() != 4 || (!codes && type != kX[dt])) return false;
    c->pages = k.size(0), c->heads = k.size(1), c->page = k.size(2), c->d = k.size(3);
    if (c->heads > INT32_MAX || c->page < 1 || c->page > INT32_MAX || c->d > INT32_MAX) return false;
    if (!whole_data(a[0], type, as, &c->k, c->pages, c->heads, c->page, c->d) || !whole_data(a[1], type, as, &c->v, c->pages, c->heads, c->page, c->d))
        return false;
    if (!codes) return a[2] == Py_None && a[3] == Py_None;
    c->format = KVCACHE_E4M3;
    return scale_of(a[2], as, *c, &c->ks) && scale_of(a[3], as, *c, &c->vs);
}
bool small(int64_t n) { return n <= INT32_MAX; }

// (q, k, q_out, k_out, positions, inv_freq, pair_axis, dtype, interleaved, inverse)
PyObject* rotary_run(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int dt;
        bool inter, inverse;
        if (n != 10 || !g_rotary || !format(a[7], &dt) || dt == 2 || !truth(a[8], &inter) || !truth(a[9], &inverse)) return general();
        const at::Tensor* q = device_tensor(a[0], kX[dt], 3);
        if (!q) return general();
        const int64_t tokens = q->size(0), hq = q->size(1), d = q->size(2);
        int64_t hk = 0;
        Heads hq_in, hk_in, hq_out, hk_out;
        if (!heads_of(a[0], kX[dt], nullptr, tokens, hq, d, &hq_in) || !heads_of(a[2], kX[dt], q, tokens, hq, d, &hq_out)) return general();
        if (a[1] != Py_None) {
            const at::Tensor* k = device_tensor(a[1], kX[dt], 3, q);
            if (!k) return general();
            hk = k->size(1);
            if (!heads_of(a[1], kX[dt], q, tokens, hk, d, &hk_in) || !heads_of(a[3], kX[dt], q, tokens, hk, d, &hk_out)) return general();
        } else if (a[3] != Py_None) {
            return general();
        }
        const at::Tensor *pos = device_tensor(a[4], at::kLong, 2, q), *freq = device_tensor(a[5], at::kDouble, 1, q);
        if (!pos || !freq) return general();
        const int64_t axes = pos->size(0), pairs = freq->size(0);
        void *p, *f, *ax;
        if (!whole_data(a[4], at::kLong, *q, &p, axes, tokens) || !whole_data(a[5], at::kDouble, *q, &f, pairs) ||
            !whole_data(a[6], at::kByte, *q, &ax, pairs) || !small(hq) || !small(hk) || !small(d) || !small(2 * pairs) || !small(axes))
            return general();
        void* s = stream_of(a[0]);
        return status([=, &hq_in, &hk_in, &hq_out, &hk_out] {
            return g_rotary(hq_in.data, hq_in.strides, hk_in.data, hk_in.strides, hq_out.data, hq_out.strides, hk_out.data, hk_out.strides,
                            static_cast<const int64_t*>(p), static_cast<const double*>(f), static_cast<const uint8_t*>(ax), tokens, static_cast<int32_t>(hq),
                            static_cast<int32_t>(hk), static_cast<int32_t>(d), static_cast<int32_t>(2 * pairs), static_cast<int32_t>(axes), dt,
                            (inter ? ROTARY_INTERLEAVED : 0) | (inverse ? ROTARY_INVERSE : 0), s);
        });
    });
}
// (k, v, slots, k_pages, v_pages, k_scale, v_scale, dtype)
PyObject* kvcache_write(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int dt;
        if (n != 8 || !g_write || !format(a[7], &dt) || dt > 1) return general();
        const at::Tensor* k = device_tensor(a[0], kX[dt], 3);
        Cache c;
        Heads kh, vh;
        void* slots;
        if (!k || !cache_of(a + 3, dt, *k, &c)) return general();
        const int64_t tokens = k->size(0);
        if (!heads_of(a[0], kX[dt], nullptr, tokens, c.heads, c.d, &kh) || !heads_of(a[1], kX[dt], k, tokens, c.heads, c.d, &vh) ||
            !whole_data(a[2], at::kLong, *k, &slots, tokens))
            return general();
        void* s = stream_of(a[0]);
        return status([=, &kh, &vh] {
            return g_write(kh.data, kh.strides, vh.data, vh.strides, static_cast<const int64_t*>(slots), c.k, c.v, static_cast<uint8_t*>(c.ks),
                           static_cast<uint8_t*>(c.vs), tokens, static_cast<int32_t>(c.heads), static_cast<int32_t>(c.d), c.pages,
                           static_cast<int32_t>(c.page), dt, c.format, s);
        });
    });
}
// (k_pages, v_pages, k_scale, v_scale, slots, k_out, v_out, dtype)
PyObject* kvcache_read(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int dt;
        if (n != 8 || !g_read || !format(a[7], &dt) || dt > 1) return general();
        const at::Tensor* slots = device_tensor(a[4], at::kLong, 1);
        Cache c;
        void *at, *k, *v;
        if (!slots || !cache_of(a, dt, *slots, &c)) return general();
        const int64_t tokens = slots->size(0);
        if (!whole_data(a[4], at::kLong, *slots, &at, tokens) || !whole_data(a[5], kX[dt], *slots, &k, tokens, c.heads, c.d) ||
            !whole_data(a[6], kX[dt], *slots, &v, tokens, c.heads, c.d))
            return general();
        void* s = stream_of(a[4]);
        return status([=] {
            return g_read(c.k, c.v, static_cast<const uint8_t*>(c.ks), static_cast<const uint8_t*>(c.vs), static_cast<const int64_t*>(at), k, v, tokens,
                          static_cast<int32_t>(c.heads), static_cast<int32_t>(c.d), c.pages, static_cast<int32_t>(c.page), dt, c.format, s);
        });
    });
}
// (q, k_pages, v_pages, k_scale, v_scale, prefix_pages, prefix_len, suffix_pages, suffix_lens, out, lse, scale, dtype, q_len, workspace)
PyObject* prefixattn_run(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        int dt;
        int64_t prefix, q_len;
        if (n != 15 || !g_attend || !format(a[12], &dt) || dt > 1 || !whole(a[6], &prefix) || !whole(a[13], &q_len) || !PyFloat_CheckExact(a[11]))
            return general();
        const at::Tensor* q = device_tensor(a[0], kX[dt], 3);
        Cache c;
        Heads qh;
        if (!q || !cache_of(a + 1, dt, *q, &c)) return general();
        const int64_t rows = q->size(0), hq = q->size(1);
        if (q_len < 1 || !small(q_len) || rows % q_len || !small(rows) || !small(hq) || prefix < 0 || !small(prefix) || !heads_of(a[0], kX[dt], nullptr, rows, hq, c.d, &qh))
            return general();
        void *first = nullptr, *own = nullptr, *lens = nullptr, *out, *lse = nullptr;
        if (prefix) {
            const at::Tensor* t = device_tensor(a[5], at::kInt, 1, q);
            if (!t || !t->is_contiguous() || t->size(0) < (prefix + c.page - 1) / c.page) return general();
            first = t->data_ptr();
        }
        int64_t width = 0;
        if (a[7] != Py_None) {
            const at::Tensor* t = device_tensor(a[7], at::kInt, 2, q);
            if (!t || t->size(1) == 0) return general();
            width = t->size(1);
            if (!whole_data(a[7], at::kInt, *q, &own, rows / q_len, width) || !whole_data(a[8], at::kInt, *q, &lens, rows / q_len)) return general();
        }
        if (!whole_data(a[9], kX[dt], *q, &out, rows, hq, c.d) || (a[10] != Py_None && !whole_data(a[10], at::kFloat, *q, &lse, rows, hq)) ||
            !THPVariable_CheckExact(a[14]))
            return general();
        const at::Tensor& room = THPVariable_Unpack(a[14]);
        if (!room.is_cuda() || room.get_device() != q->get_device() || !room.is_contiguous()) return general();
        void* work = room.data_ptr();
        const int64_t bytes = room.numel() * static_cast<int64_t>(room.element_size());
        prefixattn_shape shape;
        shape.batch = static_cast<int32_t>(rows / q_len), shape.q_len = static_cast<int32_t>(q_len), shape.q_heads = static_cast<int32_t>(hq);
        shape.kv_heads = static_cast<int32_t>(c.heads), shape.d = static_cast<int32_t>(c.d), shape.page_size = static_cast<int32_t>(c.page);
        shape.pages = c.pages, shape.prefix_len = prefix, shape.suffix_width = width, shape.dtype = dt, shape.format = c.format;
        const float scale = static_cast<float>(PyFloat_AS_DOUBLE(a[11]));
        void* s = stream_of(a[0]);
        return status([=, &qh, &shape] {
            return g_attend(qh.data, qh.strides, c.k, c.v, static_cast<const uint8_t*>(c.ks), static_cast<const uint8_t*>(c.vs),
                            static_cast<const int32_t*>(first), static_cast<const int32_t*>(own), static_cast<const int32_t*>(lens), out,
                            static_cast<float*>(lse), scale, &shape, work, bytes, s);
        });
    });
}
// (formats, addresses of rotary_run, kvcache_write, kvcache_read and prefixattn_run)
PyObject* bind_serving(PyObject*, PyObject* args)
{
    PyObject* formats;
    unsigned long long rotary, write, read, attend;
    if (!PyArg_ParseTuple(args, "O!KKKK", &PyDict_Type, &formats, &rotary, &write, &read, &attend)) return nullptr;
    Py_INCREF(formats);
    Py_XSETREF(g_formats, formats);
    g_rotary = reinterpret_cast<decltype(g_rotary)>(static_cast<uintptr_t>(rotary));
    g_write = reinterpret_cast<decltype(g_write)>(static_cast<uintptr_t>(write));
    g_read = reinterpret_cast<decltype(g_read)>(static_cast<uintptr_t>(read));
    g_attend = reinterpret_cast<decltype(g_attend)>(static_cast<uintptr_t>(attend));
    Py_RETURN_NONE;
}

// (formats, Cfg, addresses of addrms_run, silumul_run, mergestates_run and addrms_gate_probe_noalloc)
PyObject* bind(PyObject*, PyObject* args)
{
    PyObject *formats, *cfg;
    unsigned long long run, silu, merge, gate;
    if (!PyArg_ParseTuple(args, "O!O!KKKK", &PyDict_Type, &formats, &PyType_Type, &cfg, &run, &silu, &merge, &gate)) return nullptr;
    Py_INCREF(formats);
    Py_XSETREF(g_formats, formats);
    Py_INCREF(cfg);
    PyTypeObject* old = g_cfg;
    g_cfg = reinterpret_cast<PyTypeObject*>(cfg);
    Py_XDECREF(old);
    g_run = reinterpret_cast<RunFn>(static_cast<uintptr_t>(run));
    g_silu = reinterpret_cast<SiluFn>(static_cast<uintptr_t>(silu));
    g_merge = reinterpret_cast<MergeFn>(static_cast<uintptr_t>(merge));
    g_gate = reinterpret_cast<GateFn>(static_cast<uintptr_t>(gate));
    Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef g_methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                           {"addrms_run", FAST(addrms_run), nullptr},
                           {"silumul_run", FAST(silumul_run), nullptr},
                           {"mergestates_run", FAST(mergestates_run), nullptr},
                           {"addrms_gate_probe_noalloc", FAST(gate_probe_noalloc), nullptr},
                           {"bind_serving", bind_serving, METH_VARARGS, nullptr},
                           {"rotary_run", FAST(rotary_run), nullptr},
                           {"kvcache_write", FAST(kvcache_write), nullptr},
                           {"kvcache_read", FAST(kvcache_read), nullptr},
                           {"prefixattn_run", FAST(prefixattn_run), nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native()
{
    PyObject* m = PyModule_Create(&g_module);
    if (m && PyModule_AddStringConstant(m, "TORCH", TORCH_IDENTITY) != 0) Py_CLEAR(m);
    return m;
}
