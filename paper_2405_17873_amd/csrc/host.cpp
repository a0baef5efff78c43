// Native marshalling of the eager calls that one small launch follows: a Python extension module (_mqhost) that checks the
// tensors, allocates what the call returns, reads the current stream and calls the C entry point, whose address the
// binding hands over once.  In Python two dozen argument conversions, the allocations and the stream lookup cost 10 us a
// call, more than the kernels of a small layer run: 4 x 1280 x 1280 weight-only 12.9 -> 7.6 us, 256 x 320 x 320 with run-time
// ranges 20.0 -> 12.1, quantising and packing the eight linears of a 1280-channel block 190 -> 89.  Microscaled: 1 x 320 x 1280 15.9 -> 4.9 (with one launch in
// place of two), 1001 x 1952 quantised and read back 19.4 -> 9.4.
//
// Every function takes the ordinary case only, plain tensors on the GPU with the expected sizes and no mode or transform
// that intercepts operations, and returns None for anything else: the binding then goes its general way, which also
// raises the errors.
#include <ATen/ops/empty.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>

namespace {

typedef int (*w_only_fn)(const void*, int, int, int, const void*, int, int, int, const float*, const int32_t*, const void*, void*,
                         int, int, const void*, int, void*, size_t, void*);
typedef int (*w8a8_fn)(const void*, int, int, int, const void*, int, int, int, const float*, const int32_t*, const int32_t*,
                       const float*, const int32_t*, const void*, void*, int, int32_t*, const void*, int, float*, int32_t*, void*,
                       size_t, void*);
typedef int (*wxa8_fn)(const void*, int, int, int, const void*, int, int, const float*, const int32_t*, const int32_t*, const float*,
                       const int32_t*, const void*, void*, int, int32_t*, const void*, int, float*, int32_t*, void*, size_t, void*);
typedef int (*quantize_fn)(const void*, int, int, int, int, int, uint8_t*, float*, int32_t*, void*);
typedef int (*pack_fn)(const uint8_t*, int, int, int, int, int, void*, int32_t*, void*);
typedef size_t (*split_bytes_fn)(int, int, int);
typedef size_t (*a8_bytes_fn)(int, int);
typedef size_t (*packed_bytes_fn)(int, int, int, int);

typedef size_t (*mx_bytes_fn)(int, int);
typedef size_t (*mx_ws_fn)(int, int, int);
typedef int (*mx_quantize_fn)(const void*, int, int, long, int, void*, void*);
typedef int (*mx_dequantize_fn)(const void*, int, int, int, void*, long, void*);
typedef int (*mx_linear_fn)(const void*, int, int, long, const void*, int, const void*, void*, long, int, const void*, long, void*, size_t, void*);
typedef int (*mx_codes_fn)(const void*, int, int, const void*, int, const void*, void*, long, int, const void*, long, void*);
typedef int (*mx_grad_fn)(const void*, int, int, long, const void*, const uint8_t*, int, void*, long, int, void*, size_t, void*);
typedef int (*norm_fn)(const void*, int, int, long, const void*, const void*, int, float, void*, long, int, float*, float*, void*);
typedef int (*norm_mx_fn)(const void*, int, int, long, const void*, const void*, int, float, void*, int, float*, float*, void*);
typedef int (*norm_grad_fn)(const void*, long, const void*, long, int, int, const void*, int, const float*, const float*, const void*, long, void*, long,
                            int, float*, float*, void*, size_t, void*);

struct Entry {
    w_only_fn w_only;
    w8a8_fn w8a8;
    wxa8_fn w4a8, w2a8;
    quantize_fn quantize;
    pack_fn pack;
    split_bytes_fn split_bytes;
    a8_bytes_fn a8_bytes;
    packed_bytes_fn packed_bytes;
    mx_bytes_fn mx_bytes;
    mx_quantize_fn mx_quantize;
    mx_dequantize_fn mx_dequantize;
    mx_ws_fn mx_linear_ws;
    mx_linear_fn mx_linear;
    mx_codes_fn mx_codes;
    mx_ws_fn mx_grad_ws;
    mx_grad_fn mx_grad;
    norm_fn norm;
    norm_mx_fn norm_mx;
    mx_bytes_fn norm_grad_ws;
    norm_grad_fn norm_grad;
} entry;

// An ordinary tensor on the GPU (torch.Tensor or Parameter itself), or nullptr.
const at::Tensor* gpu_tensor(PyObject* o) {
    if (!THPVariable_CheckTypeExact(Py_TYPE(o))) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.has_storage() ? &t : nullptr;
}

// An optional operand: its address (null for None), or false for what is no ordinary tensor.
bool optional_ptr(PyObject* o, void*& p, const at::Tensor** t = nullptr) {
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* v = gpu_tensor(o);
    if (!v) return false;
    p = v->data_ptr();
    if (t) *t = v;
    return true;
}

bool small_int(PyObject* o, int& v) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long l = PyLong_AsLongAndOverflow(o, &over);
    if (over || l < INT32_MIN || l > INT32_MAX) return false;
    v = (int)l;
    return true;
}

bool fits(int64_t v) { return v >= 0 && v <= INT32_MAX; }

// Nothing between the caller and the operators that would want to see the allocations.
bool plain_calls() { return !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set(); }

// Gives the interpreter lock up for as long as it lives: for allocations, which wait for the device when the pool has to
// grow, and for the launch.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

void* stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }

at::Tensor empty(at::IntArrayRef size, at::ScalarType type, at::Device device) {
    return at::empty(size, at::TensorOptions().dtype(type).device(device));
}

// [M, N] residual of x's type: its address and row stride.
bool residual_of(PyObject* o, int64_t M, int64_t N, at::ScalarType type, void*& p, int& ld) {
    const at::Tensor* r = nullptr;
    ld = 0;
    if (!optional_ptr(o, p, &r)) return false;
    if (!r) return true;
    if (r->dim() != 2 || r->size(0) != M || r->size(1) != N || r->stride(1) != 1 || r->scalar_type() != type || !fits(r->stride(0)))
        return false;
    ld = (int)r->stride(0);
    return true;
}

// [M, K] activations with contiguous rows.
bool activations(const at::Tensor* x, int K) {
    return x && x->dim() == 2 && x->stride(1) == 1 && x->size(1) == K && fits(x->size(0)) && fits(x->stride(0));
}

PyObject* general() { Py_RETURN_NONE; }

// (x, packed, N, K, bits, layout, scale, zp, bias, out, residual, ws) -> tensor, error code or None
PyObject* qlinear_w_only(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        int N, K, bits, layout, ldr;
        void *packed, *scale, *zp, *bias, *res, *ws;
        const at::Tensor *x, *out = nullptr, *wst = nullptr;
        if (n != 12 || !plain_calls() || !(x = gpu_tensor(a[0])) || !small_int(a[2], N) || !small_int(a[3], K) || N < 0 ||
            !small_int(a[4], bits) || !small_int(a[5], layout) || !activations(x, K) || !optional_ptr(a[1], packed) ||
            !optional_ptr(a[6], scale) || !optional_ptr(a[7], zp) || !optional_ptr(a[8], bias))
            return general();
        const at::ScalarType type = x->scalar_type();
        if (type != at::kHalf && type != at::kBFloat16) return general();
        const int64_t M = x->size(0);
        if (!residual_of(a[10], M, N, type, res, ldr)) return general();
        if (a[9] != Py_None && (!(out = gpu_tensor(a[9])) || out->dim() < 1 || !fits(out->stride(0)))) return general();
        if (!optional_ptr(a[11], ws, &wst)) return general();
        size_t ws_bytes = wst ? wst->nbytes() : 0;
        const void* xp = x->data_ptr();
        void* yp = out ? out->data_ptr() : nullptr;
        const int ldx = (int)x->stride(0), ldy = out ? (int)out->stride(0) : N, dt = type == at::kHalf ? 0 : 1;
        const at::Device device = x->device();
        at::Tensor y, own_ws;
        int rc;
        {
            Unlocked unlocked;
            if (!out) {
                y = empty({M, N}, type, device);
                yp = y.data_ptr();
            }
            if (!wst && (ws_bytes = entry.split_bytes((int)M, N, K)) != 0) {
                own_ws = empty({(int64_t)ws_bytes}, at::kByte, device);
                ws = own_ws.data_ptr();
            }
            rc = entry.w_only(xp, (int)M, K, ldx, packed, N, bits, layout, (const float*)scale, (const int32_t*)zp, bias, yp, ldy, dt, res,
                              ldr, ws, ws_bytes, stream());
        }
        if (rc) return PyLong_FromLong(rc);
        if (a[9] != Py_None) return Py_NewRef(a[9]);
        return THPVariable_Wrap(std::move(y));
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// (x, packed, N, K, bits, layout, signed, scale, zp, colsum, act_scale, act_zp, bias, out, residual, ws) -> tensor, code or None
PyObject* qlinear_a8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        int N, K, bits, layout, sgn, ldr;
        void *packed, *scale, *zp, *colsum, *act_s, *act_z, *bias, *res, *ws;
        const at::Tensor *x, *out = nullptr, *wst = nullptr;
        if (n != 16 || !plain_calls() || !(x = gpu_tensor(a[0])) || !small_int(a[2], N) || !small_int(a[3], K) || N < 0 ||
            !small_int(a[4], bits) || !small_int(a[5], layout) || !small_int(a[6], sgn) || !activations(x, K) ||
            x->scalar_type() != at::kHalf || !optional_ptr(a[1], packed) || !optional_ptr(a[7], scale) || !optional_ptr(a[8], zp) ||
            !optional_ptr(a[9], colsum) || !optional_ptr(a[10], act_s) || !optional_ptr(a[11], act_z) || !optional_ptr(a[12], bias))
            return general();
        const int64_t M = x->size(0);
        if (!residual_of(a[14], M, N, at::kHalf, res, ldr)) return general();
        if (a[13] != Py_None && (!(out = gpu_tensor(a[13])) || out->dim() < 1 || !fits(out->stride(0)))) return general();
        if (!optional_ptr(a[15], ws, &wst)) return general();
        size_t ws_bytes = wst ? (size_t)wst->numel() : 0;
        const void* xp = x->data_ptr();
        void* yp = out ? out->data_ptr() : nullptr;
        const int ldx = (int)x->stride(0), ldy = out ? (int)out->stride(0) : N;
        const at::Device device = x->device();
        at::Tensor y, own_ws;
        int rc;
        {
            Unlocked unlocked;
            if (!out) {
                y = empty({M, N}, at::kHalf, device);
                yp = y.data_ptr();
            }
            if (!wst) {
                ws_bytes = entry.a8_bytes((int)M, K) + entry.split_bytes((int)M, N, K);
                own_ws = empty({(int64_t)ws_bytes}, at::kByte, device);
                ws = own_ws.data_ptr();
            }
            void* st = stream();
            if (bits == 8)
                rc = entry.w8a8(xp, (int)M, K, ldx, packed, N, layout, sgn, (const float*)scale, (const int32_t*)zp, (const int32_t*)colsum,
                                (const float*)act_s, (const int32_t*)act_z, bias, yp, ldy, nullptr, res, ldr, nullptr, nullptr, ws,
                                ws_bytes, st);
            else
                rc = (bits == 4 ? entry.w4a8 : entry.w2a8)(xp, (int)M, K, ldx, packed, N, layout, (const float*)scale, (const int32_t*)zp,
                                                           (const int32_t*)colsum, (const float*)act_s, (const int32_t*)act_z, bias, yp,
                                                           ldy, nullptr, res, ldr, nullptr, nullptr, ws, ws_bytes, st);
        }
        if (rc) return PyLong_FromLong(rc);
        if (a[13] != Py_None) return Py_NewRef(a[13]);
        return THPVariable_Wrap(std::move(y));
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// (w, bits, symmetric) -> (codes, scale, zp), code or None
PyObject* quantize_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        int bits, sym;
        const at::Tensor* w;
        if (n != 3 || !plain_calls() || !(w = gpu_tensor(a[0])) || !small_int(a[1], bits) || !small_int(a[2], sym) || w->dim() != 2 ||
            !w->is_contiguous() || !fits(w->size(0)) || !fits(w->size(1)))
            return general();
        const at::ScalarType type = w->scalar_type();
        if (type != at::kHalf && type != at::kBFloat16) return general();
        const int64_t N = w->size(0), K = w->size(1);
        const void* wp = w->data_ptr();
        const at::Device device = w->device();
        at::Tensor codes, scale, zp;
        int rc;
        {
            Unlocked unlocked;
            codes = empty({N, K}, at::kByte, device), scale = empty({N}, at::kFloat, device), zp = empty({N}, at::kInt, device);
            rc = entry.quantize(wp, (int)N, (int)K, bits, sym, type == at::kHalf ? 0 : 1, (uint8_t*)codes.data_ptr(), (float*)scale.data_ptr(),
                                (int32_t*)zp.data_ptr(), stream());
        }
        if (rc) return PyLong_FromLong(rc);
        PyObject *c = THPVariable_Wrap(std::move(codes)), *s = THPVariable_Wrap(std::move(scale)), *z = THPVariable_Wrap(std::move(zp));
        PyObject* t = c && s && z ? PyTuple_Pack(3, c, s, z) : nullptr;
        Py_XDECREF(c);
        Py_XDECREF(s);
        Py_XDECREF(z);
        return t;
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// (codes, bits, layout, signed, want_colsum) -> (packed, colsum or None), code or None
PyObject* pack_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        int bits, layout, sgn, want;
        const at::Tensor* codes;
        if (n != 5 || !plain_calls() || !(codes = gpu_tensor(a[0])) || !small_int(a[1], bits) || !small_int(a[2], layout) ||
            !small_int(a[3], sgn) || !small_int(a[4], want) || bits == 16 || codes->scalar_type() != at::kByte || codes->dim() != 2 ||
            !codes->is_contiguous() || !fits(codes->size(0)) || !fits(codes->size(1)))
            return general();
        const int64_t N = codes->size(0), K = codes->size(1);
        const size_t nbytes = entry.packed_bytes((int)N, (int)K, bits, layout);
        const void* cp = codes->data_ptr();
        const at::Device device = codes->device();
        at::Tensor packed, colsum;
        int rc;
        {
            Unlocked unlocked;
            packed = empty({(int64_t)(nbytes ? nbytes : 1)}, at::kByte, device);
            if (want) colsum = empty({N}, at::kInt, device);
            rc = entry.pack((const uint8_t*)cp, (int)N, (int)K, bits, layout, sgn, packed.data_ptr(),
                            want ? (int32_t*)colsum.data_ptr() : nullptr, stream());
        }
        if (rc) return PyLong_FromLong(rc);
        PyObject *p = THPVariable_Wrap(std::move(packed)), *s = want ? THPVariable_Wrap(std::move(colsum)) : Py_NewRef(Py_None);
        PyObject* t = p && s ? PyTuple_Pack(2, p, s) : nullptr;
        Py_XDECREF(p);
        Py_XDECREF(s);
        return t;
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// ---- microscaled 4-bit floats, layer norm, and their gradients

int dtype_of(at::ScalarType t) { return t == at::kHalf ? 0 : t == at::kBFloat16 ? 1 : -1; }

// A 16-bit matrix on the GPU whose rows are contiguous and do not overlap; its size, row stride and type.
struct Matrix {
    const at::Tensor* t;
    void* p;
    int rows, cols, dtype;
    long ld;
};
bool matrix(PyObject* o, Matrix& m) {
    m.t = gpu_tensor(o);
    if (!m.t || m.t->dim() != 2 || !fits(m.t->size(0)) || !fits(m.t->size(1))) return false;
    m.rows = (int)m.t->size(0), m.cols = (int)m.t->size(1), m.dtype = dtype_of(m.t->scalar_type());
    m.ld = m.rows > 1 ? (long)m.t->stride(0) : m.cols;
    m.p = m.t->data_ptr();
    return m.dtype >= 0 && m.rows > 0 && m.cols > 0 && (m.cols == 1 || m.t->stride(1) == 1) && m.ld >= m.cols;
}
// The same as an optional operand of a given size, type and device: all zero for None.
bool optional_matrix(PyObject* o, int rows, int cols, int dtype, at::Device device, Matrix& m) {
    m = Matrix{};
    return o == Py_None || (matrix(o, m) && m.rows == rows && m.cols == cols && m.dtype == dtype && m.t->device() == device);
}
// An optional contiguous vector of n on x's device (its type in *type).
bool vector(PyObject* o, int64_t n, at::Device device, void*& p, at::ScalarType* type) {
    const at::Tensor* t = nullptr;
    if (!optional_ptr(o, p, &t)) return false;
    if (!t) return true;
    if (t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1) || t->device() != device) return false;
    *type = t->scalar_type();
    return true;
}
// A microscaled buffer of rows x K (on the device of another operand): its address, or false.
bool mx_data(PyObject* o, int rows, int K, void*& p, const at::Tensor* beside = nullptr) {
    const at::Tensor* t = gpu_tensor(o);
    if (!t || rows <= 0 || K <= 0 || t->scalar_type() != at::kByte || !t->is_contiguous() || t->nbytes() < entry.mx_bytes(rows, K)) return false;
    if (beside && t->device() != beside->device()) return false;
    p = t->data_ptr();
    return true;
}
// Whether autograd would have to go through a call with these operands (for the general way to refuse).
bool in_graph(std::initializer_list<PyObject*> operands) {
    if (!c10::GradMode::is_enabled()) return false;
    for (PyObject* o : operands) {
        const at::Tensor* t = o == Py_None ? nullptr : gpu_tensor(o);
        if (t && t->requires_grad()) return true;
    }
    return false;
}
at::Tensor workspace(size_t bytes, at::Device device) { return empty({(int64_t)bytes}, at::kByte, device); }
PyObject* pair_or_more(std::initializer_list<at::Tensor> list) {
    PyObject* t = PyTuple_New((Py_ssize_t)list.size());
    Py_ssize_t i = 0;
    for (const at::Tensor& v : list) {
        PyObject* o = t ? THPVariable_Wrap(v) : nullptr;
        if (!o) {
            Py_XDECREF(t);
            return nullptr;
        }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}

// (x) -> data, code or None
PyObject* mx_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        Matrix x;
        if (n != 1 || !plain_calls() || !matrix(a[0], x) || x.cols % 32 != 0) return general();
        at::Tensor data;
        int rc;
        {
            Unlocked unlocked;
            data = workspace(entry.mx_bytes(x.rows, x.cols), x.t->device());
            rc = entry.mx_quantize(x.p, x.rows, x.cols, x.ld, x.dtype, data.data_ptr(), stream());
        }
        return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(std::move(data));
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// (data, rows, K, dtype) -> matrix, code or None
PyObject* mx_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        int rows, K, dtype;
        void* p;
        if (n != 4 || !plain_calls() || !small_int(a[1], rows) || !small_int(a[2], K) || !small_int(a[3], dtype) || (dtype != 0 && dtype != 1) ||
            !mx_data(a[0], rows, K, p))
            return general();
        const at::Device device = gpu_tensor(a[0])->device();
        at::Tensor y;
        int rc;
        {
            Unlocked unlocked;
            y = empty({rows, K}, dtype ? at::kBFloat16 : at::kHalf, device);
            rc = entry.mx_dequantize(p, rows, K, dtype, y.data_ptr(), K, stream());
        }
        return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(std::move(y));
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// (x, w, N, K, bias, residual) -> y, code or None: the output and the workspace are allocated here
PyObject* mx_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        Matrix x, res;
        int N, K;
        void *w, *bias;
        if (n != 6 || !plain_calls() || !matrix(a[0], x) || !small_int(a[2], N) || !small_int(a[3], K) || x.cols != K ||
            !mx_data(a[1], N, K, w, x.t) || in_graph({a[0], a[4], a[5]}))
            return general();
        const at::Device device = x.t->device();
        at::ScalarType type = x.t->scalar_type();
        if (!vector(a[4], N, device, bias, &type) || type != x.t->scalar_type() || !optional_matrix(a[5], x.rows, N, x.dtype, device, res)) return general();
        at::Tensor y, ws;
        int rc;
        {
            Unlocked unlocked;
            y = empty({x.rows, N}, type, device);
            const size_t need = entry.mx_linear_ws(x.rows, N, K);
            if (need) ws = workspace(need, device);
            rc = entry.mx_linear(x.p, x.rows, K, x.ld, w, N, bias, y.data_ptr(), N, x.dtype, res.p, res.ld, need ? ws.data_ptr() : nullptr, need, stream());
        }
        return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(std::move(y));
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// (data, M, K, w, N, bias, residual, dtype) -> y, code or None
PyObject* mx_linear_codes(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        Matrix res;
        int M, K, N, dtype;
        void *x, *w, *bias;
        if (n != 8 || !plain_calls() || !small_int(a[1], M) || !small_int(a[2], K) || !small_int(a[4], N) || !small_int(a[7], dtype) ||
            (dtype != 0 && dtype != 1) || !mx_data(a[0], M, K, x) || !mx_data(a[3], N, K, w, gpu_tensor(a[0])) || in_graph({a[5], a[6]}))
            return general();
        const at::Device device = gpu_tensor(a[0])->device();
        const at::ScalarType want = dtype ? at::kBFloat16 : at::kHalf;
        at::ScalarType type = want;
        if (!vector(a[5], N, device, bias, &type) || type != want || !optional_matrix(a[6], M, N, dtype, device, res)) return general();
        at::Tensor y;
        int rc;
        {
            Unlocked unlocked;
            y = empty({M, N}, want, device);
            rc = entry.mx_codes(x, M, K, w, N, bias, y.data_ptr(), N, dtype, res.p, res.ld, stream());
        }
        return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(std::move(y));
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// (dy, w, N, K, top) -> dx, code or None
PyObject* mx_linear_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        Matrix dy;
        int N, K;
        void* w;
        const at::Tensor* top;
        if (n != 5 || !plain_calls() || !matrix(a[0], dy) || !small_int(a[2], N) || !small_int(a[3], K) || dy.cols != N || !mx_data(a[1], N, K, w, dy.t) ||
            !(top = gpu_tensor(a[4])) || top->scalar_type() != at::kByte || !top->is_contiguous() || top->numel() != K / 32 || top->device() != dy.t->device() ||
            in_graph({a[0]}))
            return general();
        const void* tp = top->data_ptr();
        const at::Device device = dy.t->device();
        at::Tensor dx, ws;
        int rc;
        {
            Unlocked unlocked;
            dx = empty({dy.rows, K}, dy.t->scalar_type(), device);
            const size_t need = entry.mx_grad_ws(dy.rows, N, K);
            if (need) ws = workspace(need, device);
            rc = entry.mx_grad(dy.p, dy.rows, N, dy.ld, w, (const uint8_t*)tp, K, dx.data_ptr(), K, dy.dtype, need ? ws.data_ptr() : nullptr, need, stream());
        }
        return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(std::move(dx));
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// Weight and bias of a norm over x's columns: addresses and type number.
bool norm_params(PyObject* weight, PyObject* bias, const Matrix& x, void*& w, void*& b, int& type) {
    at::ScalarType tw = at::kFloat, tb = at::kFloat;
    if (!vector(weight, x.cols, x.t->device(), w, &tw) || !vector(bias, x.cols, x.t->device(), b, &tb) || (w && b && tw != tb)) return false;
    const at::ScalarType t = w ? tw : tb;
    type = t == at::kFloat ? 2 : dtype_of(t);
    return type >= 0;
}
bool flag(PyObject* o, bool& v) {
    if (!PyBool_Check(o)) return false;
    v = o == Py_True;
    return true;
}

// (x, weight, bias, eps, want_stats, mx) -> y or data, or (it, mean, rstd); code or None
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        Matrix x;
        void *w, *b;
        int pt;
        bool stats, mx;
        if (n != 6 || !plain_calls() || !matrix(a[0], x) || !norm_params(a[1], a[2], x, w, b, pt) || !PyFloat_CheckExact(a[3]) || !flag(a[4], stats) ||
            !flag(a[5], mx) || (mx && x.cols % 32 != 0) || in_graph({a[0], a[1], a[2]}))
            return general();
        const float eps = (float)PyFloat_AS_DOUBLE(a[3]);
        const at::Device device = x.t->device();
        at::Tensor y, mean, rstd;
        int rc;
        {
            Unlocked unlocked;
            y = mx ? workspace(entry.mx_bytes(x.rows, x.cols), device) : empty({x.rows, x.cols}, x.t->scalar_type(), device);
            if (stats) mean = empty({x.rows}, at::kFloat, device), rstd = empty({x.rows}, at::kFloat, device);
            float *mp = stats ? (float*)mean.data_ptr() : nullptr, *rp = stats ? (float*)rstd.data_ptr() : nullptr;
            rc = mx ? entry.norm_mx(x.p, x.rows, x.cols, x.ld, w, b, pt, eps, y.data_ptr(), x.dtype, mp, rp, stream())
                    : entry.norm(x.p, x.rows, x.cols, x.ld, w, b, pt, eps, y.data_ptr(), x.cols, x.dtype, mp, rp, stream());
        }
        if (rc) return PyLong_FromLong(rc);
        return stats ? pair_or_more({y, mean, rstd}) : THPVariable_Wrap(std::move(y));
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// (dy, x, weight, mean, rstd, residual) -> (dx, dweight, dbias), code or None
PyObject* layer_norm_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        Matrix dy, x, res;
        void *w, *b, *mean, *rstd;
        int pt;
        at::ScalarType tm = at::kFloat, tr = at::kFloat;
        if (n != 6 || !plain_calls() || !matrix(a[1], x) || !matrix(a[0], dy) || dy.rows != x.rows || dy.cols != x.cols || dy.dtype != x.dtype ||
            !norm_params(a[2], Py_None, x, w, b, pt) || !vector(a[3], x.rows, x.t->device(), mean, &tm) ||
            !vector(a[4], x.rows, x.t->device(), rstd, &tr) || !mean || !rstd || tm != at::kFloat || tr != at::kFloat ||
            dy.t->device() != x.t->device() || !optional_matrix(a[5], x.rows, x.cols, x.dtype, x.t->device(), res) || in_graph({a[0]}))
            return general();
        const at::Device device = x.t->device();
        at::Tensor dx, dw, db, ws;
        int rc;
        {
            Unlocked unlocked;
            dx = empty({x.rows, x.cols}, x.t->scalar_type(), device);
            dw = empty({x.cols}, at::kFloat, device), db = empty({x.cols}, at::kFloat, device);
            const size_t need = entry.norm_grad_ws(x.rows, x.cols);
            ws = workspace(need, device);
            rc = entry.norm_grad(dy.p, dy.ld, x.p, x.ld, x.rows, x.cols, w, pt, (const float*)mean, (const float*)rstd, res.p, res.ld, dx.data_ptr(), x.cols,
                                 x.dtype, (float*)dw.data_ptr(), (float*)db.data_ptr(), ws.data_ptr(), need, stream());
        }
        return rc ? PyLong_FromLong(rc) : pair_or_more({dx, dw, db});
    } catch (const std::exception&) {
        PyErr_Clear();
        return general();
    }
}

// Addresses of the C entry points, in the order of Entry.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr int COUNT = sizeof(Entry) / sizeof(void*);
    void* p[COUNT];
    if (n != COUNT) {
        PyErr_SetString(PyExc_TypeError, "bind takes the address of every entry point");
        return nullptr;
    }
    for (int i = 0; i < COUNT; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
            return nullptr;
        }
    }
    entry = Entry{(w_only_fn)p[0], (w8a8_fn)p[1], (wxa8_fn)p[2], (wxa8_fn)p[3], (quantize_fn)p[4], (pack_fn)p[5], (split_bytes_fn)p[6],
                  (a8_bytes_fn)p[7], (packed_bytes_fn)p[8], (mx_bytes_fn)p[9], (mx_quantize_fn)p[10], (mx_dequantize_fn)p[11], (mx_ws_fn)p[12],
                  (mx_linear_fn)p[13], (mx_codes_fn)p[14], (mx_ws_fn)p[15], (mx_grad_fn)p[16], (norm_fn)p[17], (norm_mx_fn)p[18],
                  (mx_bytes_fn)p[19], (norm_grad_fn)p[20]};
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"qlinear_w_only", (PyCFunction)(void (*)(void))qlinear_w_only, METH_FASTCALL, nullptr},
    {"qlinear_a8", (PyCFunction)(void (*)(void))qlinear_a8, METH_FASTCALL, nullptr},
    {"quantize_weights", (PyCFunction)(void (*)(void))quantize_weights, METH_FASTCALL, nullptr},
    {"pack_weights", (PyCFunction)(void (*)(void))pack_weights, METH_FASTCALL, nullptr},
    {"mx_quantize", (PyCFunction)(void (*)(void))mx_quantize, METH_FASTCALL, nullptr},
    {"mx_dequantize", (PyCFunction)(void (*)(void))mx_dequantize, METH_FASTCALL, nullptr},
    {"mx_linear", (PyCFunction)(void (*)(void))mx_linear, METH_FASTCALL, nullptr},
    {"mx_linear_codes", (PyCFunction)(void (*)(void))mx_linear_codes, METH_FASTCALL, nullptr},
    {"mx_linear_grad", (PyCFunction)(void (*)(void))mx_linear_grad, METH_FASTCALL, nullptr},
    {"layer_norm", (PyCFunction)(void (*)(void))layer_norm, METH_FASTCALL, nullptr},
    {"layer_norm_grad", (PyCFunction)(void (*)(void))layer_norm_grad, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mqhost", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mqhost(void) {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "made_for", MQ_MADE_FOR) < 0) Py_CLEAR(m);
    return m;
}
