// Python side of the C ABI: argument checks, output and workspace allocation, the current stream and the call, without a
// Python frame or a ctypes conversion in between.  The kernels of a small call run a few microseconds, so what the
// host does per call is what such a call costs: st_packed_axpby 8.4 us through ctypes, of which the launch itself is 2.2.
// The module holds no kernel and no reference to a particular library: bind() receives the addresses of the entry points.
#include <Python.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <exception>
#include <initializer_list>
#include <map>
#include <string>
#include <tuple>
#include <utility>
#include "structtensor.h"

namespace {

struct Api {
    decltype(&st_packed_elems) packed_elems;
    decltype(&st_dense_elems) dense_elems;
    decltype(&st_workspace_bytes) workspace_bytes;
    decltype(&st_pack) pack;
    decltype(&st_unpack) unpack;
    decltype(&st_thp) thp;
    decltype(&st_packed_axpby) packed_axpby;
    decltype(&st_packed_mul) packed_mul;
    decltype(&st_sym_moment2) sym_moment2;
    decltype(&st_sym_moment3) sym_moment3;
    decltype(&st_sym_moment4) sym_moment4;
    decltype(&st_mttkrp_tri) mttkrp_tri;
    decltype(&st_mttkrp_slice) mttkrp_slice;
    decltype(&st_ttm_blockdiag) ttm_blockdiag;
    decltype(&st_ttm_packed) ttm_packed;
    decltype(&st_attn_window) attn_window;
    decltype(&st_attn_window_grad) attn_window_grad;
    decltype(&st_attn_window_step) attn_window_step;
    decltype(&st_attn_decay) attn_decay;
    decltype(&st_attn_decay_grad) attn_decay_grad;
    decltype(&st_attn_decay_step) attn_decay_step;
    decltype(&st_attn_rotate) attn_rotate;
    decltype(&st_attn_rotate_grad) attn_rotate_grad;
    decltype(&st_attn_cache_write) attn_cache_write;
    decltype(&st_attn_cache_read) attn_cache_read;
    decltype(&st_attn_cache_step) attn_cache_step;
    decltype(&st_attn_shared_step) attn_shared_step;
} api;

PyObject *error_class, *allocator;             // StError; callable or null
PyObject *dtype_f32, *dtype_u8, *dtype_bf16;   // torch.float32, torch.uint8, torch.bfloat16
PyObject *s_kind, *s_d, *s_inner, *s_kl, *s_ku, *s_nblocks, *s_bs, *s_dtype, *s_device, *s_view;
PyObject *last_ws;                             // dict: device index -> workspace of the most recent compute call

struct Failed {};                              // a Python error is set

[[noreturn]] void fail(PyObject *type, const char *text)
{
    PyErr_SetString(type, text);
    throw Failed();
}

void check(st_status rc, const char *where)
{
    if (rc == ST_OK) return;
    PyObject *e = PyObject_CallFunction(error_class, "is", (int)rc, where);
    if (e) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    }
    throw Failed();
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw Failed();
    }
    return THPVariable_Unpack(o);
}

void *device_ptr(const at::Tensor &t, const char *name)
{
    if (!t.is_cuda()) {
        PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor", name);
        throw Failed();
    }
    if (!t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
        throw Failed();
    }
    return t.data_ptr();
}

const float *f32_ptr(const at::Tensor &t, const char *name) { return (const float *)device_ptr(t, name); }

// The kernels run on one device and take every pointer as its memory.
void want_device_of(const at::Tensor &x, const at::Tensor &t, const char *name)
{
    if (t.device() != x.device()) {
        PyErr_Format(PyExc_ValueError, "%s must be on the device of the first operand", name);
        throw Failed();
    }
}

// The address that `bytes` bytes of results go to.
void *result_ptr(const at::Tensor &x, PyObject *out, size_t bytes)
{
    const at::Tensor &t = tensor(out, "out");
    void *p = device_ptr(t, "out");
    want_device_of(x, t, "out");
    if (t.nbytes() < bytes) {
        PyErr_Format(PyExc_ValueError, "out has %zu bytes, the result %zu", (size_t)t.nbytes(), bytes);
        throw Failed();
    }
    return p;
}

int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failed();
    return v;
}
// What int() makes of it.
int64_t whole(PyObject *o)
{
    PyObject *v = PyNumber_Long(o);
    if (!v) throw Failed();
    const long long x = PyLong_AsLongLong(v);
    Py_DECREF(v);
    if (x == -1 && PyErr_Occurred()) throw Failed();
    return x;
}
unsigned flag_bits(PyObject *o)
{
    const unsigned long v = PyLong_AsUnsignedLongMask(o);
    if (v == (unsigned long)-1 && PyErr_Occurred()) throw Failed();
    return (unsigned)v;
}
float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Failed();
    return (float)v;
}

// The product, or -1, which no element count equals, where it leaves 64 bits.
int64_t times(std::initializer_list<int64_t> factors)
{
    int64_t n = 1;
    for (const int64_t f : factors)
        if (f < 0 || __builtin_mul_overflow(n, f, &n)) return -1;
    return n;
}

int64_t field(PyObject *layout, PyObject *name)
{
    PyObject *v = PyObject_GetAttr(layout, name);
    if (!v) throw Failed();
    const long long x = PyLong_AsLongLong(v);
    Py_DECREF(v);
    if (x == -1 && PyErr_Occurred()) throw Failed();
    return x;
}
st_layout layout_of(PyObject *o)
{
    st_layout l;
    l.kind = (int32_t)field(o, s_kind);
    l.reserved = 0;
    l.d = field(o, s_d);
    l.inner = field(o, s_inner);
    l.kl = field(o, s_kl);
    l.ku = field(o, s_ku);
    l.nblocks = field(o, s_nblocks);
    l.bs = field(o, s_bs);
    return l;
}

// Element type of st_pack / st_unpack: bit copies, so any type of the same size travels.
st_dtype copy_dtype(const at::Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: case at::kInt: case at::kUInt32: return ST_F32;
    case at::kBFloat16: case at::kHalf: case at::kShort: case at::kUInt16: return ST_BF16;
    case at::kDouble: case at::kLong: return ST_F64;
    default: fail(PyExc_TypeError, "unsupported dtype");
    }
}

// A new tensor as a Python object, from torch or from the allocator of set_allocator().
PyObject *allocate(PyObject *like, const at::Tensor &t, at::IntArrayRef shape, at::ScalarType type, PyObject *py_type)
{
    if (!allocator) return THPVariable_Wrap(at::empty(shape, t.options().dtype(type).requires_grad(false)));
    int64_t n = 1;
    for (const int64_t s : shape) n *= s;
    PyObject *device = PyObject_GetAttr(like, s_device);
    PyObject *r = device ? PyObject_CallFunction(allocator, "LOO", (long long)n, py_type, device) : nullptr;
    Py_XDECREF(device);
    if (r && shape.size() != 1) {
        PyObject *dims = PyTuple_New((Py_ssize_t)shape.size());
        for (size_t i = 0; i < shape.size(); ++i) PyTuple_SET_ITEM(dims, (Py_ssize_t)i, PyLong_FromLongLong(shape[i]));
        PyObject *v = PyObject_CallMethodOneArg(r, s_view, dims);
        Py_DECREF(dims);
        Py_DECREF(r);
        r = v;
    }
    return r;
}

// Owned Python reference.
struct Ref {
    PyObject *o;
    explicit Ref(PyObject *p) : o(p) { if (!p) throw Failed(); }
    Ref(const Ref &) = delete;
    Ref(Ref &&r) noexcept : o(r.o) { r.o = nullptr; }
    ~Ref() { Py_XDECREF(o); }
    PyObject *release() { PyObject *p = o; o = nullptr; return p; }
};

// The caller's tensor or a new one of `shape`.
PyObject *output(PyObject *given, PyObject *like, const at::Tensor &t, at::IntArrayRef shape)
{
    if (given != Py_None) {
        (void)tensor(given, "out");
        Py_INCREF(given);
        return given;
    }
    return allocate(like, t, shape, at::kFloat, dtype_f32);
}

struct Workspace {
    Ref ref;                                   // held until the call has been enqueued (another thread may replace last_ws)
    void *ptr;
    size_t bytes;
};

// Workspace bytes by request; the current device decides too (its SM count).  Bounded: forgotten when it grows past
// what a program with many shapes uses.  Accessed with the GIL held.
size_t workspace_size(int op, int64_t a, int64_t b, int64_t c, int64_t e, unsigned flags)
{
    typedef std::tuple<int, int, int64_t, int64_t, int64_t, int64_t, unsigned> Key;
    static std::map<Key, size_t> known;
    const Key key(c10::cuda::current_device(), op, a, b, c, e, flags);
    const auto it = known.find(key);
    if (it != known.end()) return it->second;
    if (known.size() >= 1024) known.clear();
    const size_t n = api.workspace_bytes((st_op)op, a, b, c, e, flags);
    return known[key] = n < 256 ? 256 : n;
}

// The caller's workspace or a new one of the request's size; remembered as its device's last.
Workspace workspace(PyObject *given, PyObject *like, const at::Tensor &t, int op, int64_t a, int64_t b, int64_t c, int64_t e,
                    unsigned flags)
{
    PyObject *o = given;
    if (given == Py_None) {
        const int64_t n = (int64_t)workspace_size(op, a, b, c, e, flags);
        o = allocate(like, t, {n}, at::kByte, dtype_u8);
    } else {
        Py_INCREF(given);
    }
    Ref hold(o);
    const at::Tensor &ws = tensor(o, "ws");
    void *ptr = device_ptr(ws, "ws");
    want_device_of(t, ws, "ws");
    Ref index(PyLong_FromLong(ws.get_device()));
    if (PyDict_SetItem(last_ws, index.o, o) != 0) throw Failed();
    const size_t bytes = ws.nbytes();
    return Workspace{std::move(hold), ptr, bytes};
}

void *stream() { return (void *)c10::cuda::getCurrentCUDAStream().stream(); }

// The C call with the interpreter lock released, as a launch may have to wait for room in the queue.
template <typename F>
void call(const char *where, F f)
{
    void *s = stream();
    st_status rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(s);
    Py_END_ALLOW_THREADS
    check(rc, where);
}

void want_f32(const at::Tensor &t, const char *what)
{
    if (t.scalar_type() != at::kFloat) {
        PyErr_Format(PyExc_TypeError, "%s must be float32", what);
        throw Failed();
    }
}
void want_2d(const at::Tensor &t, const char *what)
{
    if (t.dim() != 2) {
        PyErr_Format(PyExc_ValueError, "%s must have two dimensions", what);
        throw Failed();
    }
}

PyObject *py_pack(PyObject *const *v)                    // dense, layout, out
{
    const at::Tensor &dense = tensor(v[0], "dense");
    const st_layout l = layout_of(v[1]);
    const int64_t n = api.packed_elems(&l);
    if (n < 0) check(ST_ERR_SHAPE, "st_packed_elems");
    if (dense.numel() != api.dense_elems(&l)) {
        PyErr_Format(PyExc_ValueError, "dense has %lld elements, layout needs %lld", (long long)dense.numel(), (long long)api.dense_elems(&l));
        throw Failed();
    }
    const st_dtype type = copy_dtype(dense);
    void *src = device_ptr(dense, "dense");
    Ref out(Py_None == v[2] ? [&] { Ref ty(PyObject_GetAttr(v[0], s_dtype)); return allocate(v[0], dense, {n}, dense.scalar_type(), ty.o); }()
                            : (Py_INCREF(v[2]), v[2]));
    void *dst = result_ptr(dense, out.o, (size_t)n * dense.element_size());
    call("st_pack", [&](void *s) { return api.pack(&l, type, src, dst, s); });
    return out.release();
}

PyObject *py_unpack(PyObject *const *v)                  // packed, layout, fill, out
{
    const at::Tensor &packed = tensor(v[0], "packed");
    const st_layout l = layout_of(v[1]);
    const int64_t n = api.dense_elems(&l);
    if (n < 0) check(ST_ERR_SHAPE, "st_dense_elems");
    if (packed.numel() != api.packed_elems(&l)) {
        PyErr_Format(PyExc_ValueError, "packed has %lld elements, layout needs %lld", (long long)packed.numel(), (long long)api.packed_elems(&l));
        throw Failed();
    }
    const st_dtype type = copy_dtype(packed);
    const st_fill fill = (st_fill)whole(v[2]);
    void *src = device_ptr(packed, "packed");
    Ref out(Py_None == v[3] ? [&] { Ref ty(PyObject_GetAttr(v[0], s_dtype)); return allocate(v[0], packed, {n}, packed.scalar_type(), ty.o); }()
                            : (Py_INCREF(v[3]), v[3]));
    void *dst = result_ptr(packed, out.o, (size_t)n * packed.element_size());
    call("st_unpack", [&](void *s) { return api.unpack(&l, type, src, dst, fill, s); });
    return out.release();
}

PyObject *py_thp(PyObject *const *v)                     // Bp, C, layout, out
{
    const at::Tensor &B = tensor(v[0], "Bp"), &C = tensor(v[1], "C");
    want_f32(B, "inputs");
    want_f32(C, "inputs");
    const st_layout l = layout_of(v[2]);
    if (B.numel() != api.packed_elems(&l) || C.numel() != api.dense_elems(&l)) fail(PyExc_ValueError, "shape mismatch");
    const float *b = f32_ptr(B, "Bp"), *c = f32_ptr(C, "C");
    want_device_of(B, C, "C");
    Ref out(output(v[3], v[0], B, B.sizes()));
    float *o = (float *)result_ptr(B, out.o, sizeof(float) * (size_t)B.numel());
    call("st_thp", [&](void *s) { return api.thp(&l, b, c, o, s); });
    return out.release();
}

void want_pair(const at::Tensor &a, const at::Tensor &b)
{
    if (a.scalar_type() != at::kFloat || b.scalar_type() != at::kFloat || a.numel() != b.numel())
        fail(PyExc_ValueError, "two float32 arrays of the same size are needed");
}

PyObject *py_axpby(PyObject *const *v)                   // alpha, a, beta, b, out
{
    const float alpha = real(v[0]), beta = real(v[2]);
    const at::Tensor &a = tensor(v[1], "a"), &b = tensor(v[3], "b");
    want_pair(a, b);
    const float *pa = f32_ptr(a, "a"), *pb = f32_ptr(b, "b");
    want_device_of(a, b, "b");
    Ref out(output(v[4], v[1], a, a.sizes()));
    float *o = (float *)result_ptr(a, out.o, sizeof(float) * (size_t)a.numel());
    const int64_t n = a.numel();
    call("st_packed_axpby", [&](void *s) { return api.packed_axpby(n, alpha, pa, beta, pb, o, s); });
    return out.release();
}

PyObject *py_mul(PyObject *const *v)                     // a, b, out
{
    const at::Tensor &a = tensor(v[0], "a"), &b = tensor(v[1], "b");
    want_pair(a, b);
    const float *pa = f32_ptr(a, "a"), *pb = f32_ptr(b, "b");
    want_device_of(a, b, "b");
    Ref out(output(v[2], v[0], a, a.sizes()));
    float *o = (float *)result_ptr(a, out.o, sizeof(float) * (size_t)a.numel());
    const int64_t n = a.numel();
    call("st_packed_mul", [&](void *s) { return api.packed_mul(n, pa, pb, o, s); });
    return out.release();
}

PyObject *py_moment2(PyObject *const *v)                 // X, out, ws, flags
{
    const at::Tensor &X = tensor(v[0], "X");
    want_2d(X, "X");
    const bool bf16 = X.scalar_type() == at::kBFloat16;
    if (!bf16 && X.scalar_type() != at::kFloat) fail(PyExc_TypeError, "X must be float32 or bfloat16");
    const st_dtype type = bf16 ? ST_BF16 : ST_F32;
    const int64_t N = X.size(0), d = X.size(1), ldx = X.stride(0);
    const unsigned flags = flag_bits(v[3]);
    const void *x = device_ptr(X, "X");
    Ref out(output(v[1], v[0], X, {d * (d + 1) / 2}));
    const Workspace w = workspace(v[2], v[0], X, ST_OP_SYM_MOMENT2, N, d, type, 0, flags);
    float *o = (float *)result_ptr(X, out.o, sizeof(float) * (size_t)(d * (d + 1) / 2));
    call("st_sym_moment2", [&](void *s) { return api.sym_moment2(x, type, N, d, ldx, o, w.ptr, w.bytes, flags, s); });
    return out.release();
}

PyObject *moment34(PyObject *const *v, int order)        // X, out, ws, flags
{
    const at::Tensor &X = tensor(v[0], "X");
    want_2d(X, "X");
    want_f32(X, "X");
    const int64_t N = X.size(0), d = X.size(1), ldx = X.stride(0);
    const unsigned flags = flag_bits(v[3]);
    const int64_t tet = d * (d + 1) * (d + 2) / 6;
    const float *x = f32_ptr(X, "X");
    Ref out(output(v[1], v[0], X, {order == 3 ? tet : tet * (d + 3) / 4}));
    const Workspace w = workspace(v[2], v[0], X, order == 3 ? ST_OP_SYM_MOMENT3 : ST_OP_SYM_MOMENT4, N, d, 0, 0, flags);
    float *o = (float *)result_ptr(X, out.o, sizeof(float) * (size_t)(order == 3 ? tet : tet * (d + 3) / 4));
    const auto f = order == 3 ? api.sym_moment3 : api.sym_moment4;
    call(order == 3 ? "st_sym_moment3" : "st_sym_moment4", [&](void *s) { return f(x, N, d, ldx, o, w.ptr, w.bytes, flags, s); });
    return out.release();
}
PyObject *py_moment3(PyObject *const *v) { return moment34(v, 3); }
PyObject *py_moment4(PyObject *const *v) { return moment34(v, 4); }

PyObject *py_mttkrp_tri(PyObject *const *v)              // Bp, C, D, out, ws, flags
{
    const at::Tensor &B = tensor(v[0], "Bp"), &C = tensor(v[1], "C"), &D = tensor(v[2], "D");
    want_2d(C, "C");
    want_2d(D, "D");
    for (const at::Tensor *t : {&B, &C, &D}) want_f32(*t, "inputs");
    const int64_t I = C.size(0), R = C.size(1), K = D.size(0);
    const unsigned flags = flag_bits(v[5]);
    const int64_t want = (flags & ST_FLAG_DENSE_CONTROL) ? times({I, I, K}) : times({I % 2 ? I : I / 2, I % 2 ? (I + 1) / 2 : I + 1, K});
    if (B.numel() != want || D.size(1) != R) fail(PyExc_ValueError, "shape mismatch");
    const float *b = f32_ptr(B, "Bp"), *c = f32_ptr(C, "C"), *d = f32_ptr(D, "D");
    want_device_of(B, C, "C");
    want_device_of(B, D, "D");
    Ref out(output(v[3], v[0], B, {I, R}));
    const Workspace w = workspace(v[4], v[0], B, ST_OP_MTTKRP_TRI, I, K, R, 0, flags);
    float *o = (float *)result_ptr(B, out.o, sizeof(float) * (size_t)(I * R));
    call("st_mttkrp_tri", [&](void *s) { return api.mttkrp_tri(b, I, K, c, d, R, o, w.ptr, w.bytes, flags, s); });
    return out.release();
}

PyObject *py_mttkrp_slice(PyObject *const *v)            // Bp, C, D, I, fixed_i, fixed_j, out, ws, flags
{
    const at::Tensor &B = tensor(v[0], "Bp"), &C = tensor(v[1], "C"), &D = tensor(v[2], "D");
    want_2d(C, "C");
    want_2d(D, "D");
    for (const at::Tensor *t : {&B, &C, &D}) want_f32(*t, "inputs");
    const int64_t J = C.size(0), R = C.size(1), K = D.size(0), I = integer(v[3]), fi = integer(v[4]), fj = integer(v[5]);
    const unsigned flags = flag_bits(v[8]);
    const int64_t rows = fi >= 0 ? (fj >= 0 ? 1 : J) : I;
    if (B.numel() != times({rows, K}) || D.size(1) != R) fail(PyExc_ValueError, "shape mismatch");
    const float *b = f32_ptr(B, "Bp"), *c = f32_ptr(C, "C"), *d = f32_ptr(D, "D");
    want_device_of(B, C, "C");
    want_device_of(B, D, "D");
    Ref out(output(v[6], v[0], B, {I, R}));
    const Workspace w = workspace(v[7], v[0], B, ST_OP_MTTKRP_SLICE, I, J, K, R, flags);
    float *o = (float *)result_ptr(B, out.o, sizeof(float) * (size_t)(I * R));
    call("st_mttkrp_slice", [&](void *s) { return api.mttkrp_slice(b, I, J, K, fi, fj, c, d, R, o, w.ptr, w.bytes, flags, s); });
    return out.release();
}

PyObject *py_ttm_blockdiag(PyObject *const *v)           // Bp, U, nblocks, bs, out, ws, flags
{
    const at::Tensor &B = tensor(v[0], "Bp"), &U = tensor(v[1], "U");
    want_2d(U, "U");
    want_f32(B, "inputs");
    want_f32(U, "inputs");
    const int64_t K = U.size(0), R = U.size(1), nb = integer(v[2]), bs = integer(v[3]), d = times({nb, bs});
    const unsigned flags = flag_bits(v[6]);
    const int64_t rows = (flags & ST_FLAG_DENSE_CONTROL) ? times({d, d}) : times({d, bs});
    if (B.numel() != times({rows, K})) fail(PyExc_ValueError, "shape mismatch");
    const float *b = f32_ptr(B, "Bp"), *u = f32_ptr(U, "U");
    want_device_of(B, U, "U");
    Ref out(output(v[4], v[0], B, {rows, R}));
    const Workspace w = workspace(v[5], v[0], B, ST_OP_TTM_BLOCKDIAG, nb, bs, K, R, flags);
    float *o = (float *)result_ptr(B, out.o, sizeof(float) * (size_t)(rows * R));
    call("st_ttm_blockdiag", [&](void *s) { return api.ttm_blockdiag(b, nb, bs, K, u, R, o, w.ptr, w.bytes, flags, s); });
    return out.release();
}

PyObject *py_ttm_packed(PyObject *const *v)              // Bp, U, layout, out, ws, flags
{
    const at::Tensor &B = tensor(v[0], "Bp"), &U = tensor(v[1], "U");
    want_2d(U, "U");
    want_f32(B, "inputs");
    want_f32(U, "inputs");
    const int64_t K = U.size(0), R = U.size(1);
    const st_layout l = layout_of(v[2]);
    if (l.inner != K || B.numel() != api.packed_elems(&l)) fail(PyExc_ValueError, "shape mismatch");
    const int64_t rows = B.numel() / K;
    const unsigned flags = flag_bits(v[5]);
    const float *b = f32_ptr(B, "Bp"), *u = f32_ptr(U, "U");
    want_device_of(B, U, "U");
    Ref out(output(v[3], v[0], B, {rows, R}));
    const Workspace w = workspace(v[4], v[0], B, ST_OP_TTM_BLOCKDIAG, rows, 1, K, R, flags);
    float *o = (float *)result_ptr(B, out.o, sizeof(float) * (size_t)(rows * R));
    call("st_ttm_packed", [&](void *s) { return api.ttm_packed(&l, b, u, R, o, w.ptr, w.bytes, flags, s); });
    return out.release();
}

// ---- attention ------------------------------------------------------------------------

typedef c10::cuda::CUDAGuard Guard;            // the tensors' device is the current one for the call, its stream the call's

const at::Tensor &cuda_tensor(PyObject *o, const char *name)
{
    const at::Tensor &t = tensor(o, name);
    if (!t.is_cuda()) {
        PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor", name);
        throw Failed();
    }
    return t;
}

void want_bf16(const at::Tensor &t, const char *name)
{
    if (t.scalar_type() != at::kBFloat16) {
        PyErr_Format(PyExc_TypeError, "%s must be bfloat16", name);
        throw Failed();
    }
}

void want_shape(const at::Tensor &t, at::IntArrayRef shape, const char *name)
{
    if (t.sizes() != shape) {
        PyErr_Format(PyExc_ValueError, "%s has the wrong shape", name);
        throw Failed();
    }
}

// A bf16 table of `dims` dimensions whose last one is contiguous; the others may have any strides.
const at::Tensor &table(const at::Tensor &x, PyObject *o, const char *name, int64_t dims)
{
    const at::Tensor &t = cuda_tensor(o, name);
    want_device_of(x, t, name);
    want_bf16(t, name);
    if (t.dim() != dims) {
        PyErr_Format(PyExc_ValueError, "%s must have %lld dimensions", name, (long long)dims);
        throw Failed();
    }
    if (t.size(dims - 1) != 1 && t.stride(dims - 1) != 1) {
        PyErr_Format(PyExc_ValueError, "the last dimension of %s must be contiguous", name);
        throw Failed();
    }
    return t;
}

const at::Tensor &contiguous(const at::Tensor &x, PyObject *o, at::ScalarType type, const char *name)
{
    const at::Tensor &t = cuda_tensor(o, name);
    want_device_of(x, t, name);
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s must be %s", name,
                     type == at::kFloat ? "float32" : type == at::kInt ? "int32" : type == at::kLong ? "int64" : "bfloat16");
        throw Failed();
    }
    (void)device_ptr(t, name);
    return t;
}

// One offset more than there are sequences, or None for one sequence of all rows.
const int32_t *offsets_of(const at::Tensor &x, PyObject *o, const char *name, int64_t *nseq)
{
    if (o == Py_None) {
        *nseq = 1;
        return nullptr;
    }
    const at::Tensor &t = contiguous(x, o, at::kInt, name);
    if (t.dim() != 1 || t.size(0) < 2) {
        PyErr_Format(PyExc_ValueError, "%s must be one-dimensional, with one entry more than there are sequences", name);
        throw Failed();
    }
    *nseq = t.size(0) - 1;
    return (const int32_t *)t.data_ptr();
}

// The caller's result or a new one.
PyObject *result(PyObject *given, PyObject *like, const at::Tensor &x, at::IntArrayRef shape, at::ScalarType type, const char *name)
{
    if (given != Py_None) {
        want_shape(contiguous(x, given, type, name), shape, name);
        Py_INCREF(given);
        return given;
    }
    Ref bf16_type(PyObject_GetAttr(like, s_dtype));
    return allocate(like, x, shape, type, type == at::kFloat ? dtype_f32 : bf16_type.o);
}
void *data(const Ref &r) { return THPVariable_Unpack(r.o).data_ptr(); }

float scale_of(PyObject *o, int64_t d) { return o == Py_None ? (float)(1.0 / std::sqrt((double)d)) : real(o); }

// Window or sinks: as many as the kernels count to, where the caller's number is larger.
int64_t count_of(PyObject *o)
{
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) return overflow > 0 ? INT64_MAX : -1;
    if (v == -1 && PyErr_Occurred()) throw Failed();
    return v;
}

struct Qkv {
    const at::Tensor &q, &k, &v;
    st_tokens t;
};

Qkv qkv(PyObject *pq, PyObject *pk, PyObject *pv)
{
    const at::Tensor &q = cuda_tensor(pq, "q");
    table(q, pq, "q", 3);
    const at::Tensor &k = table(q, pk, "k", 3), &v = table(q, pv, "v", 3);
    if (k.size(0) != v.size(0) || k.size(1) != v.size(1) || k.size(2) != q.size(2)) fail(PyExc_ValueError, "shape mismatch");
    st_tokens t;
    t.dtype = ST_BF16;
    t.reserved = 0;
    t.nseq = 1;
    t.nq = q.size(0);
    t.nk = k.size(0);
    t.heads = q.size(1);
    t.kv_heads = k.size(1);
    t.d = q.size(2);
    t.dv = v.size(2);
    t.q_row = q.stride(0);
    t.q_head = q.stride(1);
    t.k_row = k.stride(0);
    t.k_head = k.stride(1);
    t.v_row = v.stride(0);
    t.v_head = v.stride(1);
    return {q, k, v, t};
}

struct Offsets {
    const int32_t *q, *k;
};
Offsets two_offsets(Qkv &x, PyObject *oq, PyObject *ok)
{
    if (oq == Py_None && ok != Py_None) fail(PyExc_ValueError, "k_offsets without q_offsets");
    Offsets o;
    int64_t keys = 1;
    o.q = offsets_of(x.q, oq, "q_offsets", &x.t.nseq);
    o.k = ok == Py_None ? o.q : offsets_of(x.q, ok, "k_offsets", &keys);
    if (ok != Py_None && keys != x.t.nseq) fail(PyExc_ValueError, "q_offsets and k_offsets must have the same length");
    if (oq != Py_None && ok == Py_None && x.t.nq != x.t.nk) fail(PyExc_ValueError, "k_offsets are needed where k has not the rows of q");
    return o;
}

PyObject *pair(Ref a, Ref b)
{
    PyObject *r = PyTuple_New(2);
    if (!r) throw Failed();
    PyTuple_SET_ITEM(r, 0, a.release());
    PyTuple_SET_ITEM(r, 1, b.release());
    return r;
}

PyObject *py_attn_window(PyObject *const *v)             // q, k, v, window, sinks, q_offsets, k_offsets, scale, out, lse, ws
{
    Qkv x = qkv(v[0], v[1], v[2]);
    const Guard guard(x.q.device());
    const int64_t window = count_of(v[3]), sinks = count_of(v[4]);
    const Offsets o = two_offsets(x, v[5], v[6]);
    const float scale = scale_of(v[7], x.t.d);
    Ref out(result(v[8], v[0], x.q, {x.t.nq, x.t.heads, x.t.d}, at::kBFloat16, "out"));
    Ref lse(result(v[9], v[0], x.q, {x.t.nq, x.t.heads}, at::kFloat, "lse"));
    const Workspace w = workspace(v[10], v[0], x.q, ST_OP_ATTN_WINDOW, 0, 0, 0, 0, 0);
    void *po = data(out);
    float *pl = (float *)data(lse);
    const void *q = x.q.data_ptr(), *k = x.k.data_ptr(), *vv = x.v.data_ptr();
    call("st_attn_window", [&](void *s) { return api.attn_window(&x.t, q, k, vv, o.q, o.k, window, sinks, scale, po, pl, w.ptr, w.bytes, s); });
    return pair(std::move(out), std::move(lse));
}

// q, k, v, out, lse, dout, window, sinks, q_offsets, k_offsets, scale, dq, dk, dv, ws
PyObject *py_attn_window_grad(PyObject *const *v)
{
    Qkv x = qkv(v[0], v[1], v[2]);
    const Guard guard(x.q.device());
    const st_tokens &t = x.t;
    const at::Tensor &out = contiguous(x.q, v[3], at::kBFloat16, "out"), &lse = contiguous(x.q, v[4], at::kFloat, "lse"),
                     &dout = contiguous(x.q, v[5], at::kBFloat16, "dout");
    want_shape(out, {t.nq, t.heads, t.d}, "out");
    want_shape(lse, {t.nq, t.heads}, "lse");
    want_shape(dout, {t.nq, t.heads, t.d}, "dout");
    const int64_t window = count_of(v[6]), sinks = count_of(v[7]);
    const Offsets o = two_offsets(x, v[8], v[9]);
    const float scale = scale_of(v[10], t.d);
    Ref dq(result(v[11], v[0], x.q, {t.nq, t.heads, t.d}, at::kBFloat16, "dq"));
    Ref dk(result(v[12], v[0], x.q, {t.nk, t.kv_heads, t.d}, at::kBFloat16, "dk"));
    Ref dv(result(v[13], v[0], x.q, {t.nk, t.kv_heads, t.d}, at::kBFloat16, "dv"));
    const Workspace w = workspace(v[14], v[0], x.q, ST_OP_ATTN_WINDOW_GRAD, t.nq, t.heads, t.kv_heads, sinks, 0);
    const void *q = x.q.data_ptr(), *k = x.k.data_ptr(), *vv = x.v.data_ptr(), *po = out.data_ptr(), *pd = dout.data_ptr();
    const float *pl = (const float *)lse.data_ptr();
    void *pq = data(dq), *pk = data(dk), *pv = data(dv);
    call("st_attn_window_grad", [&](void *s) {
        return api.attn_window_grad(&t, q, k, vv, po, pl, pd, o.q, o.k, window, sinks, scale, pq, pk, pv, w.ptr, w.bytes, s);
    });
    return PyTuple_Pack(3, dq.o, dk.o, dv.o);
}

// q, k, v, k_pages, v_pages, table, lens, window, sinks, scale, out, ws
PyObject *py_attn_window_step(PyObject *const *v)
{
    const at::Tensor &q = cuda_tensor(v[0], "q");
    const Guard guard(q.device());
    contiguous(q, v[0], at::kBFloat16, "q");
    const at::Tensor &k = contiguous(q, v[1], at::kBFloat16, "k"), &vv = contiguous(q, v[2], at::kBFloat16, "v");
    const at::Tensor &kp = table(q, v[3], "k_pages", 4), &vp = table(q, v[4], "v_pages", 4);
    const at::Tensor &tab = contiguous(q, v[5], at::kInt, "table"), &lens = contiguous(q, v[6], at::kInt, "lens");
    if (q.dim() != 3 || k.dim() != 3) fail(PyExc_ValueError, "q and k must have three dimensions");
    const int64_t n = q.size(0), d = q.size(2), kv_heads = k.size(1);
    want_shape(k, {n, kv_heads, d}, "k");
    want_shape(vv, {n, kv_heads, d}, "v");
    want_shape(kp, {kp.size(0), kp.size(1), kv_heads, d}, "k_pages");
    want_shape(vp, kp.sizes(), "v_pages");
    if (kp.strides() != vp.strides()) fail(PyExc_ValueError, "k_pages and v_pages must have the same strides");
    if (tab.dim() != 2 || tab.size(0) != n) fail(PyExc_ValueError, "table must have one row for every sequence");
    want_shape(lens, {n}, "lens");
    st_cache c;
    c.dtype = ST_BF16;
    c.reserved = 0;
    c.nseq = n;
    c.heads = q.size(1);
    c.kv_heads = kv_heads;
    c.d = d;
    c.pages = kp.size(0);
    c.page = kp.size(1);
    c.table_cols = tab.size(1);
    c.page_stride = kp.stride(0);
    c.token_stride = kp.stride(1);
    c.head_stride = kp.stride(2);
    const int64_t window = count_of(v[7]), sinks = count_of(v[8]);
    const float scale = scale_of(v[9], d);
    Ref out(result(v[10], v[0], q, q.sizes(), at::kBFloat16, "out"));
    const Workspace w = workspace(v[11], v[0], q, ST_OP_ATTN_WINDOW_STEP, 0, 0, 0, 0, 0);
    const void *pq = q.data_ptr(), *pk = k.data_ptr(), *pv = vv.data_ptr();
    void *pkp = kp.data_ptr(), *pvp = vp.data_ptr(), *po = data(out);
    const int32_t *pt = (const int32_t *)tab.data_ptr(), *pl = (const int32_t *)lens.data_ptr();
    call("st_attn_window_step", [&](void *s) { return api.attn_window_step(&c, pq, pk, pv, pkp, pvp, pt, pl, window, sinks, scale, po, w.ptr, w.bytes, s); });
    return out.release();
}

const float *decay_of(const Qkv &x, PyObject *o)
{
    const at::Tensor &a = contiguous(x.q, o, at::kFloat, "log_decay");
    want_shape(a, {x.t.heads}, "log_decay");
    return (const float *)a.data_ptr();
}
const float *state_of(const Qkv &x, PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &s = contiguous(x.q, o, at::kFloat, name);
    want_shape(s, {x.t.nseq, x.t.heads, x.t.d, x.t.dv}, name);
    return (const float *)s.data_ptr();
}

PyObject *py_attn_decay(PyObject *const *v)              // q, k, v, log_decay, offsets, state, scale, out, state_out, ws
{
    Qkv x = qkv(v[0], v[1], v[2]);
    const Guard guard(x.q.device());
    st_tokens &t = x.t;
    const float *a = decay_of(x, v[3]);
    const int32_t *at = offsets_of(x.q, v[4], "offsets", &t.nseq);
    const float *in = state_of(x, v[5], "state"), scale = scale_of(v[6], t.d);
    Ref out(result(v[7], v[0], x.q, {t.nq, t.heads, t.dv}, at::kBFloat16, "out"));
    Ref last(result(v[8], v[0], x.q, {t.nseq, t.heads, t.d, t.dv}, at::kFloat, "state_out"));
    const Workspace w = workspace(v[9], v[0], x.q, ST_OP_ATTN_DECAY, t.nq, t.nseq, t.heads, std::max(t.d, t.dv), 0);
    const void *q = x.q.data_ptr(), *k = x.k.data_ptr(), *vv = x.v.data_ptr();
    void *po = data(out);
    float *pl = (float *)data(last);
    call("st_attn_decay", [&](void *s) { return api.attn_decay(&t, q, k, vv, a, at, in, scale, po, pl, w.ptr, w.bytes, s); });
    return pair(std::move(out), std::move(last));
}

// q, k, v, log_decay, dout, offsets, state, dstate_out, scale, dq, dk, dv, dstate, ws
PyObject *py_attn_decay_grad(PyObject *const *v)
{
    Qkv x = qkv(v[0], v[1], v[2]);
    const Guard guard(x.q.device());
    st_tokens &t = x.t;
    const float *a = decay_of(x, v[3]);
    const at::Tensor &dout = contiguous(x.q, v[4], at::kBFloat16, "dout");
    want_shape(dout, {t.nq, t.heads, t.dv}, "dout");
    const int32_t *at = offsets_of(x.q, v[5], "offsets", &t.nseq);
    const float *in = state_of(x, v[6], "state"), *dlast = state_of(x, v[7], "dstate_out"), scale = scale_of(v[8], t.d);
    Ref dq(result(v[9], v[0], x.q, {t.nq, t.heads, t.d}, at::kBFloat16, "dq"));
    Ref dk(result(v[10], v[0], x.q, {t.nk, t.heads, t.d}, at::kBFloat16, "dk"));
    Ref dv(result(v[11], v[0], x.q, {t.nk, t.heads, t.dv}, at::kBFloat16, "dv"));
    const bool wanted = in || v[12] != Py_None;
    Ref first(wanted ? result(v[12], v[0], x.q, {t.nseq, t.heads, t.d, t.dv}, at::kFloat, "dstate") : (Py_INCREF(Py_None), Py_None));
    const Workspace w = workspace(v[13], v[0], x.q, ST_OP_ATTN_DECAY_GRAD, t.nq, t.nseq, t.heads, std::max(t.d, t.dv), 0);
    const void *q = x.q.data_ptr(), *k = x.k.data_ptr(), *vv = x.v.data_ptr(), *pd = dout.data_ptr();
    void *pq = data(dq), *pk = data(dk), *pv = data(dv);
    float *pf = wanted ? (float *)data(first) : nullptr;
    call("st_attn_decay_grad", [&](void *s) { return api.attn_decay_grad(&t, q, k, vv, a, pd, at, in, dlast, scale, pq, pk, pv, pf, w.ptr, w.bytes, s); });
    return PyTuple_Pack(4, dq.o, dk.o, dv.o, first.o);
}

PyObject *py_attn_decay_step(PyObject *const *v)         // q, k, v, log_decay, state, scale, out
{
    Qkv x = qkv(v[0], v[1], v[2]);
    const Guard guard(x.q.device());
    st_tokens &t = x.t;
    (void)device_ptr(x.q, "q");
    (void)device_ptr(x.k, "k");
    (void)device_ptr(x.v, "v");
    const float *a = decay_of(x, v[3]), scale = scale_of(v[5], t.d);
    t.nseq = t.nq;
    if (v[4] == Py_None) fail(PyExc_TypeError, "state must be a tensor");
    float *state = const_cast<float *>(state_of(x, v[4], "state"));
    Ref out(result(v[6], v[0], x.q, {t.nq, t.heads, t.dv}, at::kBFloat16, "out"));
    const void *q = x.q.data_ptr(), *k = x.k.data_ptr(), *vv = x.v.data_ptr();
    void *po = data(out);
    call("st_attn_decay_step", [&](void *s) { return api.attn_decay_step(&t, q, k, vv, a, state, scale, po, s); });
    return out.release();
}

// ---- rotations ------------------------------------------------------------------------

struct Rotation {
    st_rotation r;
    const at::Tensor &q;
    const at::Tensor *k;                       // or null
    const int32_t *positions;
    const float *freq;
    const void *q_weight, *k_weight;
};

const void *weight_of(const Rotation &x, PyObject *o, const char *name, at::ScalarType *type)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &w = cuda_tensor(o, name);
    if (w.scalar_type() != at::kFloat && w.scalar_type() != at::kBFloat16) {
        PyErr_Format(PyExc_TypeError, "%s must be float32 or bfloat16", name);
        throw Failed();
    }
    if (*type != at::kByte && w.scalar_type() != *type) fail(PyExc_TypeError, "q_weight and k_weight must have the same type");
    *type = w.scalar_type();
    contiguous(x.q, o, *type, name);
    want_shape(w, {x.r.d}, name);
    return w.data_ptr();
}

// q, k, positions, freq, interleaved, q_weight, k_weight, eps, factor
Rotation rotation(PyObject *pq, PyObject *pk, PyObject *const *v)
{
    const at::Tensor &q = cuda_tensor(pq, "q");
    table(q, pq, "q", 3);
    const at::Tensor *k = pk == Py_None ? nullptr : &table(q, pk, "k", 3);
    if (k && (k->size(0) != q.size(0) || k->size(2) != q.size(2))) fail(PyExc_ValueError, "shape mismatch");
    Rotation x = {{}, q, k, nullptr, nullptr, nullptr, nullptr};
    st_rotation &r = x.r;
    r.dtype = ST_BF16;
    r.n = q.size(0);
    r.heads = q.size(1);
    r.d = q.size(2);
    r.q_row = q.stride(0);
    r.q_head = q.stride(1);
    if (k) {
        r.kv_heads = k->size(1);
        r.k_row = k->stride(0);
        r.k_head = k->stride(1);
        if (r.kv_heads == 0) fail(PyExc_ValueError, "k has no heads");
    }
    const at::Tensor &positions = contiguous(q, v[0], at::kInt, "positions");
    want_shape(positions, {r.n}, "positions");
    x.positions = (const int32_t *)positions.data_ptr();
    if (v[1] != Py_None) {
        const at::Tensor &freq = contiguous(q, v[1], at::kFloat, "freq");
        if (freq.dim() != 1) fail(PyExc_ValueError, "freq must have one dimension");
        r.rot = 2 * freq.size(0);
        x.freq = (const float *)freq.data_ptr();
    }
    const int interleaved = PyObject_IsTrue(v[2]);
    if (interleaved < 0) throw Failed();
    r.interleaved = interleaved;
    r.norm = v[5] != Py_None;
    r.eps = r.norm ? real(v[5]) : 0.f;
    r.factor = real(v[6]);
    if (!r.norm && (v[3] != Py_None || v[4] != Py_None)) fail(PyExc_ValueError, "weights belong to norms: eps is missing");
    if (!k && v[4] != Py_None) fail(PyExc_ValueError, "k_weight without k");
    at::ScalarType type = at::kByte;
    x.q_weight = weight_of(x, v[3], "q_weight", &type);
    x.k_weight = weight_of(x, v[4], "k_weight", &type);
    r.weight_dtype = type == at::kFloat ? ST_F32 : ST_BF16;
    return x;
}

Ref none() { return Ref((Py_INCREF(Py_None), Py_None)); }

// q, k, positions, freq, interleaved, q_weight, k_weight, eps, factor, q_out, k_out
PyObject *py_attn_rotate(PyObject *const *v)
{
    const Guard guard(cuda_tensor(v[0], "q").device());
    const Rotation x = rotation(v[0], v[1], v + 2);
    const st_rotation &r = x.r;
    Ref q_out(result(v[9], v[0], x.q, {r.n, r.heads, r.d}, at::kBFloat16, "q_out"));
    Ref k_out = x.k ? Ref(result(v[10], v[0], x.q, {r.n, r.kv_heads, r.d}, at::kBFloat16, "k_out")) : none();
    const void *q = x.q.data_ptr(), *k = x.k ? x.k->data_ptr() : nullptr;
    void *po = data(q_out), *ko = x.k ? data(k_out) : nullptr;
    call("st_attn_rotate", [&](void *s) { return api.attn_rotate(&r, q, k, x.positions, x.freq, x.q_weight, x.k_weight, po, ko, s); });
    return pair(std::move(q_out), std::move(k_out));
}

// q, k, dq_out, dk_out, positions, freq, interleaved, q_weight, k_weight, eps, factor, dq, dk, dq_weight, dk_weight, ws
PyObject *py_attn_rotate_grad(PyObject *const *v)
{
    const Guard guard(cuda_tensor(v[0], "q").device());
    const Rotation x = rotation(v[0], v[1], v + 4);
    const st_rotation &r = x.r;
    const at::Tensor &dqo = contiguous(x.q, v[2], at::kBFloat16, "dq_out");
    want_shape(dqo, {r.n, r.heads, r.d}, "dq_out");
    if (!x.k != (v[3] == Py_None)) fail(PyExc_ValueError, "k and dk_out belong together");
    const void *q = x.q.data_ptr(), *k = x.k ? x.k->data_ptr() : nullptr, *pdq = dqo.data_ptr(), *pdk = nullptr;
    if (x.k) {
        const at::Tensor &dko = contiguous(x.q, v[3], at::kBFloat16, "dk_out");
        want_shape(dko, {r.n, r.kv_heads, r.d}, "dk_out");
        pdk = dko.data_ptr();
    }
    Ref dq(result(v[11], v[0], x.q, {r.n, r.heads, r.d}, at::kBFloat16, "dq"));
    Ref dk = x.k ? Ref(result(v[12], v[0], x.q, {r.n, r.kv_heads, r.d}, at::kBFloat16, "dk")) : none();
    Ref dqw = x.q_weight ? Ref(result(v[13], v[0], x.q, {r.d}, at::kFloat, "dq_weight")) : none();
    Ref dkw = x.k_weight ? Ref(result(v[14], v[0], x.q, {r.d}, at::kFloat, "dk_weight")) : none();
    const Workspace w = workspace(v[15], v[0], x.q, ST_OP_ATTN_ROTATE_GRAD, x.q_weight || x.k_weight ? r.d : 0, 0, 0, 0, 0);
    void *po = data(dq), *ko = x.k ? data(dk) : nullptr;
    float *pqw = x.q_weight ? (float *)data(dqw) : nullptr, *pkw = x.k_weight ? (float *)data(dkw) : nullptr;
    call("st_attn_rotate_grad", [&](void *s) {
        return api.attn_rotate_grad(&r, q, k, pdq, pdk, x.positions, x.freq, x.q_weight, x.k_weight, po, ko, pqw, pkw, w.ptr, w.bytes, s);
    });
    return PyTuple_Pack(4, dq.o, dk.o, dqw.o, dkw.o);
}

// ---- caches in cells ------------------------------------------------------------------

struct CellTensors {
    st_cells c;
    void *k, *v, *k_scales, *v_scales;
    const int32_t *table, *lens;
};

// A tensor of `dims` dimensions, of which the last `whole` ones lie without gaps.
const at::Tensor &dense_tail(const at::Tensor &x, PyObject *o, at::ScalarType type, int64_t dims, int64_t whole, const char *name)
{
    const at::Tensor &t = cuda_tensor(o, name);
    want_device_of(x, t, name);
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s has the wrong type", name);
        throw Failed();
    }
    if (t.dim() != dims) {
        PyErr_Format(PyExc_ValueError, "%s must have %lld dimensions", name, (long long)dims);
        throw Failed();
    }
    int64_t want = 1;
    for (int64_t i = dims - 1; i >= dims - whole; --i) {
        if (t.size(i) != 1 && t.stride(i) != want) {
            PyErr_Format(PyExc_ValueError, "the last dimension of %s must be contiguous", name);
            throw Failed();
        }
        want *= t.size(i);
    }
    return t;
}

// k_pages, v_pages, table, lens, k_scales, v_scales; heads and d of what meets them
CellTensors cell_tensors(const at::Tensor &x, PyObject *pk, PyObject *pv, PyObject *ptable, PyObject *plens, PyObject *pks, PyObject *pvs, int64_t heads, int64_t d)
{
    const at::Tensor &k = cuda_tensor(pk, "k_pages");
    const at::ScalarType type = k.scalar_type();
    if (type != at::kBFloat16 && type != at::kChar && type != at::kByte) fail(PyExc_TypeError, "k_pages must be bfloat16, int8 or uint8 (two cells of 4 bits)");
    dense_tail(x, pk, type, 4, 1, "k_pages");
    const at::Tensor &v = dense_tail(x, pv, type, 4, 1, "v_pages");
    if (v.sizes() != k.sizes()) fail(PyExc_ValueError, "v_pages has the wrong shape");
    if (v.strides() != k.strides()) fail(PyExc_ValueError, "k_pages and v_pages must have the same strides");
    CellTensors r = {};
    st_cells &c = r.c;
    c.dtype = type == at::kBFloat16 ? ST_BF16 : type == at::kChar ? ST_I8 : ST_I4;
    const int64_t cols = c.dtype == ST_I4 ? 2 * k.size(3) : k.size(3), bytes = k.element_size();
    if (d >= 0 && cols != d) fail(PyExc_ValueError, "k_pages has the wrong shape");
    const at::Tensor &table = contiguous(x, ptable, at::kInt, "table"), &lens = contiguous(x, plens, at::kInt, "lens");
    if (lens.dim() != 1 || table.dim() != 2 || table.size(0) != lens.size(0)) fail(PyExc_ValueError, "table must have one row for every sequence");
    c.nseq = lens.size(0);
    c.kv_heads = k.size(2);
    c.heads = heads >= 0 ? heads : c.kv_heads;
    c.d = cols;
    c.pages = k.size(0);
    c.page = k.size(1);
    c.table_cols = table.size(1);
    c.page_stride = k.stride(0) * bytes;
    c.token_stride = k.stride(1) * bytes;
    c.head_stride = k.stride(2) * bytes;
    r.k = k.data_ptr();
    r.v = v.data_ptr();
    r.table = (const int32_t *)table.data_ptr();
    r.lens = (const int32_t *)lens.data_ptr();
    if (c.dtype == ST_BF16) {
        if (pks != Py_None || pvs != Py_None) fail(PyExc_ValueError, "bfloat16 pages have no scales");
        return r;
    }
    // float32 [pages, page, heads], or bfloat16 [pages, page, heads, groups, 2] in units of two
    const bool four = c.dtype == ST_I4;
    const at::ScalarType scale_type = four ? at::kBFloat16 : at::kFloat;
    const at::Tensor &ks = dense_tail(x, pks, scale_type, four ? 5 : 3, four ? 2 : 0, "k_scales"), &vs = dense_tail(x, pvs, scale_type, four ? 5 : 3, four ? 2 : 0, "v_scales");
    if (four) want_shape(ks, {c.pages, c.page, c.kv_heads, (c.d + 31) / 32, 2}, "k_scales");
    else want_shape(ks, {c.pages, c.page, c.kv_heads}, "k_scales");
    want_shape(vs, ks.sizes(), "v_scales");
    if (ks.strides() != vs.strides()) fail(PyExc_ValueError, "k_scales and v_scales must have the same strides");
    int64_t *const to[3] = {&c.scale_page, &c.scale_token, &c.scale_head};
    for (int i = 0; i < 3; ++i) {
        if (four && ks.size(i) != 1 && ks.stride(i) % 2 != 0) fail(PyExc_ValueError, "strides of k_scales and v_scales must be even");
        *to[i] = four ? ks.stride(i) / 2 : ks.stride(i);
    }
    r.k_scales = ks.data_ptr();
    r.v_scales = vs.data_ptr();
    return r;
}

// Offsets of rows, one more than there are sequences, or None: a row for every sequence, or one sequence of all rows.
const int32_t *row_offsets(const at::Tensor &x, PyObject *o, const st_cells &c, int64_t n)
{
    int64_t nseq = 0;
    if (o == Py_None) {
        if (c.nseq != 1 && c.nseq != n) fail(PyExc_ValueError, "offsets are needed where there is not one row for every sequence");
        return nullptr;
    }
    const int32_t *p = offsets_of(x, o, "offsets", &nseq);
    if (nseq != c.nseq) fail(PyExc_ValueError, "offsets must have one entry more than there are sequences");
    return p;
}

// k, v, k_pages, v_pages, table, lens, offsets, k_scales, v_scales, ws
PyObject *py_attn_cache_write(PyObject *const *v)
{
    const at::Tensor &k = cuda_tensor(v[0], "k");
    const Guard guard(k.device());
    table(k, v[0], "k", 3);
    const at::Tensor &vv = table(k, v[1], "v", 3);
    want_shape(vv, k.sizes(), "v");
    const CellTensors x = cell_tensors(k, v[2], v[3], v[4], v[5], v[7], v[8], -1, k.size(2));
    if (x.c.kv_heads != k.size(1)) fail(PyExc_ValueError, "k_pages has the wrong shape");
    st_tokens t = {};
    t.dtype = ST_BF16;
    t.nseq = x.c.nseq;
    t.nk = k.size(0);
    t.kv_heads = k.size(1);
    t.d = t.dv = k.size(2);
    t.k_row = k.stride(0);
    t.k_head = k.stride(1);
    t.v_row = vv.stride(0);
    t.v_head = vv.stride(1);
    const int32_t *at = row_offsets(k, v[6], x.c, t.nk);
    const Workspace w = workspace(v[9], v[0], k, ST_OP_ATTN_CACHE, 0, 0, 0, 0, 0);
    const void *pk = k.data_ptr(), *pv = vv.data_ptr();
    call("st_attn_cache_write", [&](void *s) { return api.attn_cache_write(&x.c, &t, pk, pv, x.table, x.lens, at, x.k, x.v, x.k_scales, x.v_scales, w.ptr, w.bytes, s); });
    Py_RETURN_NONE;
}

// k_pages, v_pages, table, lens, offsets, rows, k_scales, v_scales, k, v, ws
PyObject *py_attn_cache_read(PyObject *const *v)
{
    const at::Tensor &kp = cuda_tensor(v[0], "k_pages");
    const Guard guard(kp.device());
    const CellTensors x = cell_tensors(kp, v[0], v[1], v[2], v[3], v[6], v[7], -1, -1);
    const int64_t n = integer(v[5]);
    if (n <= 0) fail(PyExc_ValueError, "rows must be positive");
    const int32_t *at = row_offsets(kp, v[4], x.c, n);
    // new tensors are bfloat16, whatever the pages are
    auto rows = [&](PyObject *given, const char *name) -> PyObject * {
        if (given != Py_None) return result(given, v[0], kp, {n, x.c.kv_heads, x.c.d}, at::kBFloat16, name);
        return allocate(v[0], kp, {n, x.c.kv_heads, x.c.d}, at::kBFloat16, dtype_bf16);
    };
    Ref k(rows(v[8], "k")), vv(rows(v[9], "v"));
    const Workspace w = workspace(v[10], v[0], kp, ST_OP_ATTN_CACHE, 0, 0, 0, 0, 0);
    void *pk = data(k), *pv = data(vv);
    call("st_attn_cache_read", [&](void *s) { return api.attn_cache_read(&x.c, n, x.k, x.v, x.k_scales, x.v_scales, x.table, x.lens, at, pk, pv, w.ptr, w.bytes, s); });
    return pair(std::move(k), std::move(vv));
}

// q, k_pages, v_pages, table, lens, window, sinks, k_scales, v_scales, scale, out, ws
PyObject *py_attn_cache_step(PyObject *const *v)
{
    const at::Tensor &q = cuda_tensor(v[0], "q");
    const Guard guard(q.device());
    table(q, v[0], "q", 3);
    const CellTensors x = cell_tensors(q, v[1], v[2], v[3], v[4], v[7], v[8], q.size(1), q.size(2));
    if (x.c.nseq != q.size(0)) fail(PyExc_ValueError, "table must have one row for every sequence");
    const int64_t window = count_of(v[5]), sinks = count_of(v[6]);
    const float scale = scale_of(v[9], x.c.d);
    Ref out(result(v[10], v[0], q, q.sizes(), at::kBFloat16, "out"));
    const Workspace w = workspace(v[11], v[0], q, ST_OP_ATTN_CACHE_STEP, x.c.nseq, 0, 0, 0, 0);
    const void *pq = q.data_ptr();
    const int64_t row = q.stride(0), head = q.stride(1);
    void *po = data(out);
    call("st_attn_cache_step", [&](void *s) {
        return api.attn_cache_step(&x.c, pq, row, head, x.k, x.v, x.k_scales, x.v_scales, x.table, x.lens, window, sinks, scale, po, w.ptr, w.bytes, s);
    });
    return out.release();
}

// q, k_pages, v_pages, prefix_table, prefix_lens, table, lens, group_offsets, scale, out, ws
PyObject *py_attn_shared_step(PyObject *const *v)
{
    const at::Tensor &q = cuda_tensor(v[0], "q");
    const Guard guard(q.device());
    table(q, v[0], "q", 3);
    want_bf16(cuda_tensor(v[1], "k_pages"), "k_pages");
    const CellTensors x = cell_tensors(q, v[1], v[2], v[5], v[6], Py_None, Py_None, q.size(1), q.size(2));
    if (x.c.nseq != q.size(0)) fail(PyExc_ValueError, "table must have one row for every sequence");
    const at::Tensor &ptable = contiguous(q, v[3], at::kInt, "prefix_table"), &plens = contiguous(q, v[4], at::kInt, "prefix_lens");
    if (plens.dim() != 1 || ptable.dim() != 2 || ptable.size(0) != plens.size(0)) fail(PyExc_ValueError, "prefix_table must have one row for every group");
    const int64_t groups = plens.size(0), cols = ptable.size(1);
    int64_t told = 1;
    const int32_t *at = offsets_of(q, v[7], "group_offsets", &told);
    if (told != groups) fail(PyExc_ValueError, "group_offsets must have one entry more than there are groups");
    const float scale = scale_of(v[8], x.c.d);
    Ref out(result(v[9], v[0], q, q.sizes(), at::kBFloat16, "out"));
    const Workspace w = workspace(v[10], v[0], q, ST_OP_ATTN_SHARED_STEP, x.c.nseq, x.c.heads, x.c.kv_heads, groups, 0);
    const void *pq = q.data_ptr();
    const int64_t row = q.stride(0), head = q.stride(1);
    const int32_t *pt = (const int32_t *)ptable.data_ptr(), *pl = (const int32_t *)plens.data_ptr();
    void *po = data(out);
    call("st_attn_shared_step", [&](void *s) {
        return api.attn_shared_step(&x.c, pq, row, head, x.k, x.v, pt, cols, pl, groups, at, x.table, x.lens, scale, po, w.ptr, w.bytes, s);
    });
    return out.release();
}

// Argument count, and C++ errors as Python ones.
template <PyObject *(*F)(PyObject *const *), int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    if (!api.pack) {
        PyErr_SetString(PyExc_RuntimeError, "bind() has not been called");
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Failed &) {
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

// bind(addresses: dict name -> int, StError, torch.float32, torch.uint8, torch.bfloat16, last_ws: dict)
PyObject *py_bind(PyObject *, PyObject *args)
{
    PyObject *table, *err, *f32, *u8, *b16, *last;
    if (!PyArg_ParseTuple(args, "O!OOOOO!", &PyDict_Type, &table, &err, &f32, &u8, &b16, &PyDict_Type, &last)) return nullptr;
    Api a;
    const struct { const char *name; void *slot; } want[] = {
        {"st_packed_elems", &a.packed_elems}, {"st_dense_elems", &a.dense_elems}, {"st_workspace_bytes", &a.workspace_bytes},
        {"st_pack", &a.pack}, {"st_unpack", &a.unpack}, {"st_thp", &a.thp}, {"st_packed_axpby", &a.packed_axpby},
        {"st_packed_mul", &a.packed_mul}, {"st_sym_moment2", &a.sym_moment2}, {"st_sym_moment3", &a.sym_moment3},
        {"st_sym_moment4", &a.sym_moment4}, {"st_mttkrp_tri", &a.mttkrp_tri}, {"st_mttkrp_slice", &a.mttkrp_slice},
        {"st_ttm_blockdiag", &a.ttm_blockdiag}, {"st_ttm_packed", &a.ttm_packed}, {"st_attn_window", &a.attn_window},
        {"st_attn_window_grad", &a.attn_window_grad}, {"st_attn_window_step", &a.attn_window_step}, {"st_attn_decay", &a.attn_decay},
        {"st_attn_decay_grad", &a.attn_decay_grad}, {"st_attn_decay_step", &a.attn_decay_step}, {"st_attn_rotate", &a.attn_rotate},
        {"st_attn_rotate_grad", &a.attn_rotate_grad}, {"st_attn_cache_write", &a.attn_cache_write}, {"st_attn_cache_read", &a.attn_cache_read},
        {"st_attn_cache_step", &a.attn_cache_step}, {"st_attn_shared_step", &a.attn_shared_step}};
    for (const auto &w : want) {
        PyObject *v = PyDict_GetItemString(table, w.name);
        void *p = v ? PyLong_AsVoidPtr(v) : nullptr;
        if (!p) {
            if (!PyErr_Occurred()) PyErr_Format(PyExc_KeyError, "%s", w.name);
            return nullptr;
        }
        std::memcpy(w.slot, &p, sizeof(p));
    }
    for (PyObject *o : {err, f32, u8, b16, last}) Py_INCREF(o);
    error_class = err;
    dtype_f32 = f32;
    dtype_u8 = u8;
    dtype_bf16 = b16;
    last_ws = last;
    api = a;
    Py_RETURN_NONE;
}

PyObject *py_set_allocator(PyObject *, PyObject *fn)
{
    PyObject *old = allocator;
    allocator = fn == Py_None ? nullptr : (Py_INCREF(fn), fn);
    Py_XDECREF(old);
    Py_RETURN_NONE;
}

#define ENTRY(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&entry<py_##name, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, nullptr},
    {"set_allocator", py_set_allocator, METH_O, nullptr},
    ENTRY(pack, 3), ENTRY(unpack, 4), ENTRY(thp, 4), ENTRY(axpby, 5), ENTRY(mul, 3), ENTRY(moment2, 4), ENTRY(moment3, 4),
    ENTRY(moment4, 4), ENTRY(mttkrp_tri, 6), ENTRY(mttkrp_slice, 9), ENTRY(ttm_blockdiag, 7), ENTRY(ttm_packed, 6),
    ENTRY(attn_window, 11), ENTRY(attn_window_grad, 15), ENTRY(attn_window_step, 12), ENTRY(attn_decay, 10), ENTRY(attn_decay_grad, 14),
    ENTRY(attn_decay_step, 7), ENTRY(attn_rotate, 11), ENTRY(attn_rotate_grad, 16), ENTRY(attn_cache_write, 10), ENTRY(attn_cache_read, 11),
    ENTRY(attn_cache_step, 12), ENTRY(attn_shared_step, 11),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void)
{
    s_kind = PyUnicode_InternFromString("kind");
    s_d = PyUnicode_InternFromString("d");
    s_inner = PyUnicode_InternFromString("inner");
    s_kl = PyUnicode_InternFromString("kl");
    s_ku = PyUnicode_InternFromString("ku");
    s_nblocks = PyUnicode_InternFromString("nblocks");
    s_bs = PyUnicode_InternFromString("bs");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_device = PyUnicode_InternFromString("device");
    s_view = PyUnicode_InternFromString("view");
    return PyModule_Create(&module);
}
