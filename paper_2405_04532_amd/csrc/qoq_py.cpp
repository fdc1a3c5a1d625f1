// Native argument marshalling of the calls that a serving loop makes per layer: checks the tensors, allocates the results,
// takes the current stream and calls the C ABI.  The same checks and results as their Python counterparts in api.py had;
// through ctypes a call of the activation quantizer took 10.6 us of host time and a GEMM 7.7 us, more than their kernels at
// decode sizes, of which the launch itself is about 2 us (the rest: argument objects, torch.empty, the stream lookup).
// Nothing is kept between calls.  The interpreter lock is released around the library call, as ctypes does.
#include <Python.h>

#include <algorithm>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/qoq_w4a8.h"
#include "qoq_workspace.h"

namespace {

PyObject* g_raise_status = nullptr;             // Python callable that raises the error of a status code

bool counted(Py_ssize_t got, Py_ssize_t want)
{
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return false;
}

// a tensor argument; nullptr with an exception set if it is something else
const at::Tensor* tensor(PyObject* o, const char* name)
{
    if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor", name);
    return nullptr;
}

// a contiguous tensor of this type on the GPU
const at::Tensor* dev_tensor(PyObject* o, at::ScalarType dtype, const char* name)
{
    const at::Tensor* t = tensor(o, name);
    if (!t || (t->is_cuda() && t->scalar_type() == dtype && t->is_contiguous())) return t;
    const char* type = dtype == at::kHalf ? "torch.float16" : dtype == at::kChar ? "torch.int8" : dtype == at::kInt ? "torch.int32" : dtype == at::kByte ? "torch.uint8" : "torch.float32";
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous %s tensor on the GPU", name, type);
    return nullptr;
}

bool has_dims(const at::Tensor& t, int64_t dims, const char* name)
{
    if (t.dim() == dims) return true;
    PyErr_Format(PyExc_ValueError, "%s: expected %lld dimensions, got %lld", name, (long long)dims, (long long)t.dim());
    return false;
}

// address of a tensor or None; false with an exception set for anything else
bool pointer(PyObject* o, const char* name, void** p)
{
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = tensor(o, name);
    if (!t) return false;
    *p = t->data_ptr();
    return true;
}

bool integer(PyObject* o, int64_t* v)
{
    *v = PyLong_AsLongLong(o);
    return !(*v == -1 && PyErr_Occurred());
}

// a truth value, as `if o:` takes it; false with the exception set if it has none
bool flag(PyObject* o, bool* v)
{
    const int t = PyObject_IsTrue(o);
    *v = t == 1;
    return t >= 0;
}

bool number(PyObject* o, double* v)             // as float(o) takes it
{
    PyObject* f = PyNumber_Float(o);
    if (!f) return false;
    *v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return true;
}

void* stream_of(const at::Tensor& t) { return c10::hip::getCurrentHIPStream(t.get_device()).stream(); }

at::Tensor new_like(const at::Tensor& on, at::IntArrayRef shape, at::ScalarType dtype)
{
    return at::empty(shape, at::TensorOptions().dtype(dtype).device(on.device()));
}

template <class F>
bool call(F&& f)                                // true: QOQ_OK; false: the status's exception is set
{
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    if (status == QOQ_OK) return true;
    PyObject* r = PyObject_CallFunction(g_raise_status, "i", status);
    Py_XDECREF(r);
    return false;
}

// the results of a quantizing call, in the order in which api.py returns them
struct Quantized {
    at::Tensor y, qx, sx, rowsum, tx;
    Quantized(const at::Tensor& on, int64_t M, int64_t K, bool want_y, bool want_rowsum, bool want_tx)
    {
        if (want_y) y = new_like(on, {M, K}, at::kHalf);
        qx = new_like(on, {M, K}, at::kChar);
        sx = new_like(on, {M}, at::kHalf);
        if (want_rowsum) rowsum = new_like(on, {M}, at::kInt);
        if (want_tx) tx = new_like(on, {M}, at::kFloat);
    }
    static void* at_or_null(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
    static PyObject* wrap(const at::Tensor& t)
    {
        if (t.defined()) return THPVariable_Wrap(t);
        Py_RETURN_NONE;
    }
    void* y_ptr() const { return at_or_null(y); }
    int8_t* qx_ptr() const { return static_cast<int8_t*>(qx.data_ptr()); }
    void* sx_ptr() const { return sx.data_ptr(); }
    int32_t* rowsum_ptr() const { return static_cast<int32_t*>(at_or_null(rowsum)); }
    float* tx_ptr() const { return static_cast<float*>(at_or_null(tx)); }
    PyObject* result(bool with_y) const
    {
        return with_y ? Py_BuildValue("NNNNN", wrap(y), wrap(qx), wrap(sx), wrap(rowsum), wrap(tx))
                      : Py_BuildValue("NNNN", wrap(qx), wrap(sx), wrap(rowsum), wrap(tx));
    }
};

PyObject* quant_act(PyObject*, PyObject* const* a, Py_ssize_t n)    // x, want_rowsum, want_tx
{
    HANDLE_TH_ERRORS
    if (!counted(n, 3)) return nullptr;
    const at::Tensor* x = dev_tensor(a[0], at::kHalf, "x");
    bool want_rowsum, want_tx;
    if (!x || !has_dims(*x, 2, "x") || !flag(a[1], &want_rowsum) || !flag(a[2], &want_tx)) return nullptr;
    const int64_t M = x->size(0), K = x->size(1);
    const Quantized q(*x, M, K, false, want_rowsum, want_tx);
    void* s = stream_of(*x);
    const void* xp = x->data_ptr();
    if (!call([&] { return qoq_quant_act_per_token(xp, M, K, q.qx_ptr(), q.sx_ptr(), q.rowsum_ptr(), q.tx_ptr(), s); })) return nullptr;
    return q.result(false);
    END_HANDLE_TH_ERRORS
}

PyObject* quant_act_reordered(PyObject*, PyObject* const* a, Py_ssize_t n)    // x, perm, want_rowsum, want_tx
{
    HANDLE_TH_ERRORS
    if (!counted(n, 4)) return nullptr;
    const at::Tensor* x = dev_tensor(a[0], at::kHalf, "x");
    if (!x) return nullptr;
    const at::Tensor* perm = dev_tensor(a[1], at::kInt, "perm");
    bool want_rowsum, want_tx;
    if (!perm || !has_dims(*x, 2, "x") || !flag(a[2], &want_rowsum) || !flag(a[3], &want_tx)) return nullptr;
    const int64_t M = x->size(0), K = x->size(1);
    const Quantized q(*x, M, K, false, want_rowsum, want_tx);
    void* s = stream_of(*x);
    const void* xp = x->data_ptr();
    const int32_t* pp = static_cast<const int32_t*>(perm->data_ptr());
    if (!call([&] { return qoq_quant_act_per_token_reordered(xp, pp, M, K, q.qx_ptr(), q.sx_ptr(), q.rowsum_ptr(), q.tx_ptr(), s); }))
        return nullptr;
    return q.result(false);
    END_HANDLE_TH_ERRORS
}

PyObject* rmsnorm_quant(PyObject*, PyObject* const* a, Py_ssize_t n)    // x, gamma, eps, want_y, want_rowsum, want_tx
{
    HANDLE_TH_ERRORS
    if (!counted(n, 6)) return nullptr;
    const at::Tensor* x = dev_tensor(a[0], at::kHalf, "x");
    if (!x) return nullptr;
    const at::Tensor* gamma = dev_tensor(a[1], at::kHalf, "gamma");
    bool want_y, want_rowsum, want_tx;
    double eps;
    if (!gamma || !has_dims(*x, 2, "x") || !number(a[2], &eps) || !flag(a[3], &want_y) || !flag(a[4], &want_rowsum) || !flag(a[5], &want_tx))
        return nullptr;
    const int64_t M = x->size(0), K = x->size(1);
    const Quantized q(*x, M, K, want_y, want_rowsum, want_tx);
    void* s = stream_of(*x);
    const void *xp = x->data_ptr(), *gp = gamma->data_ptr();
    if (!call([&] { return qoq_rmsnorm_quant(xp, gp, eps, M, K, q.y_ptr(), q.qx_ptr(), q.sx_ptr(), q.rowsum_ptr(), q.tx_ptr(), s); }))
        return nullptr;
    return q.result(true);
    END_HANDLE_TH_ERRORS
}

PyObject* silu_mul_quant(PyObject*, PyObject* const* a, Py_ssize_t n)    // gate_up, want_y, want_rowsum, want_tx
{
    HANDLE_TH_ERRORS
    if (!counted(n, 4)) return nullptr;
    const at::Tensor* x = dev_tensor(a[0], at::kHalf, "gate_up");
    bool want_y, want_rowsum, want_tx;
    if (!x || !has_dims(*x, 2, "gate_up") || !flag(a[1], &want_y) || !flag(a[2], &want_rowsum) || !flag(a[3], &want_tx)) return nullptr;
    const int64_t M = x->size(0), K = x->size(1) / 2;
    const Quantized q(*x, M, K, want_y, want_rowsum, want_tx);
    void* s = stream_of(*x);
    const void* xp = x->data_ptr();
    if (!call([&] { return qoq_silu_mul_quant(xp, M, K, q.y_ptr(), q.qx_ptr(), q.sx_ptr(), q.rowsum_ptr(), q.tx_ptr(), s); })) return nullptr;
    return q.result(true);
    END_HANDLE_TH_ERRORS
}

// the caller's tensor, or a new one of this shape; `owned` keeps the new one alive and becomes the result
PyObject* given_or_new(PyObject* given, const at::Tensor& on, at::IntArrayRef shape, at::ScalarType dtype, const char* name, void** p)
{
    if (given == Py_None) {
        at::Tensor t = new_like(on, shape, dtype);
        *p = t.data_ptr();
        return THPVariable_Wrap(std::move(t));
    }
    if (!pointer(given, name, p)) return nullptr;
    Py_INCREF(given);
    return given;
}

struct Ref {                                    // an owned reference that is dropped unless it is released
    PyObject* o;
    explicit Ref(PyObject* p) : o(p) {}
    ~Ref() { Py_XDECREF(o); }
    PyObject* release() { PyObject* r = o; o = nullptr; return r; }
    explicit operator bool() const { return o != nullptr; }
};

// Workspace of a GEMM call: the caller's, or one of what the call exchanges, its counters zeroed on the stream (zeroing all of it, as
// a workspace that is kept is prepared, took 4 to 11 us more for 12 to 39 MB).
struct Workspace {
    at::Tensor own;
    void* ptr = nullptr;
    size_t bytes = 0;
    bool ready(PyObject* given, const at::Tensor& on, int64_t M, int64_t N, int64_t K, int64_t mode, void* stream)
    {
        if (given != Py_None) {
            const at::Tensor* t = tensor(given, "workspace");
            if (!t) return false;
            ptr = t->data_ptr();
            bytes = (size_t)t->numel() * t->element_size();
            return true;
        }
        bytes = qoq::gemm_fresh_workspace_bytes(M, N, K, (int)mode);
        if (!bytes) return true;
        own = new_like(on, {(int64_t)bytes}, at::kByte);
        ptr = own.data_ptr();
        return call([&] { return qoq_gemm_workspace_prepare(ptr, std::min(bytes, (size_t)QOQ_GEMM_COUNTER_BYTES), stream); });
    }
};

PyObject* w4a8_gemm(PyObject*, PyObject* const* a, Py_ssize_t n)    // qx, sx, packed, N, mode, rowsum, out, workspace
{
    HANDLE_TH_ERRORS
    if (!counted(n, 8)) return nullptr;
    const at::Tensor* qx = dev_tensor(a[0], at::kChar, "qx");
    int64_t N, mode;
    void *sx, *packed, *rowsum, *out;
    if (!qx || !has_dims(*qx, 2, "qx") || !integer(a[3], &N) || !integer(a[4], &mode) || !pointer(a[1], "sx", &sx) ||
        !pointer(a[2], "packed", &packed) || !pointer(a[5], "rowsum", &rowsum))
        return nullptr;
    const int64_t M = qx->size(0), K = qx->size(1);
    void* s = stream_of(*qx);
    Ref res(given_or_new(a[6], *qx, {M, N}, at::kHalf, "out", &out));
    Workspace ws;
    if (!res || !ws.ready(a[7], *qx, M, N, K, mode, s)) return nullptr;
    const int8_t* xp = static_cast<const int8_t*>(qx->data_ptr());
    if (!call([&] { return qoq_w4a8_gemm(xp, sx, static_cast<int32_t*>(rowsum), packed, M, N, K, (int)mode, out, ws.ptr, ws.bytes, s); }))
        return nullptr;
    return res.release();
    END_HANDLE_TH_ERRORS
}

PyObject* w4a8_gemm_noalloc(PyObject*, PyObject* const* a, Py_ssize_t n)    // qx, sx, packed, N, out, mode, rowsum
{
    HANDLE_TH_ERRORS
    if (!counted(n, 7)) return nullptr;
    const at::Tensor* qx = dev_tensor(a[0], at::kChar, "qx");
    if (!qx) return nullptr;
    const at::Tensor* out = dev_tensor(a[4], at::kHalf, "out");
    int64_t N, mode;
    void *sx, *packed, *rowsum;
    if (!out || !has_dims(*qx, 2, "qx") || !integer(a[3], &N) || !integer(a[5], &mode) || !pointer(a[1], "sx", &sx) ||
        !pointer(a[2], "packed", &packed) || !pointer(a[6], "rowsum", &rowsum))
        return nullptr;
    const int64_t M = qx->size(0), K = qx->size(1);
    void *s = stream_of(*qx), *op = out->data_ptr();
    const int8_t* xp = static_cast<const int8_t*>(qx->data_ptr());
    if (!call([&] { return qoq_w4a8_gemm_noalloc(xp, sx, static_cast<int32_t*>(rowsum), packed, M, N, K, (int)mode, op, s); })) return nullptr;
    Py_INCREF(a[4]);
    return a[4];
    END_HANDLE_TH_ERRORS
}

PyObject* w4a8_gemm_token_sum(PyObject*, PyObject* const* a, Py_ssize_t n)    // qx, sx, tx, packed, N, out, workspace
{
    HANDLE_TH_ERRORS
    if (!counted(n, 7)) return nullptr;
    const at::Tensor* qx = dev_tensor(a[0], at::kChar, "qx");
    if (!qx) return nullptr;
    const at::Tensor* tx = dev_tensor(a[2], at::kFloat, "tx");
    int64_t N;
    void *sx, *packed, *out;
    if (!tx || !has_dims(*qx, 2, "qx") || !integer(a[4], &N) || !pointer(a[1], "sx", &sx) || !pointer(a[3], "packed", &packed)) return nullptr;
    const int64_t M = qx->size(0), K = qx->size(1);
    void* s = stream_of(*qx);
    Ref res(given_or_new(a[5], *qx, {M, N}, at::kHalf, "out", &out));
    Workspace ws;
    if (!res || !ws.ready(a[6], *qx, M, N, K, QOQ_PER_CHANNEL, s)) return nullptr;
    const int8_t* xp = static_cast<const int8_t*>(qx->data_ptr());
    const float* tp = static_cast<const float*>(tx->data_ptr());
    if (!call([&] { return qoq_w4a8_gemm_token_sum(xp, sx, tp, packed, M, N, K, out, ws.ptr, ws.bytes, s); })) return nullptr;
    return res.release();
    END_HANDLE_TH_ERRORS
}

PyObject* w4a8_linear(PyObject*, PyObject* const* a, Py_ssize_t n)    // x, packed, N, mode, out, qx, sx, rowsum, workspace
{
    HANDLE_TH_ERRORS
    if (!counted(n, 9)) return nullptr;
    const at::Tensor* x = dev_tensor(a[0], at::kHalf, "x");
    int64_t N, mode;
    void *packed, *out, *qx, *sx, *rowsum;
    if (!x || !has_dims(*x, 2, "x") || !integer(a[2], &N) || !integer(a[3], &mode) || !pointer(a[1], "packed", &packed)) return nullptr;
    const int64_t M = x->size(0), K = x->size(1);
    void* s = stream_of(*x);
    Ref r_out(given_or_new(a[4], *x, {M, N}, at::kHalf, "out", &out));
    Ref r_qx(r_out ? given_or_new(a[5], *x, {M, K}, at::kChar, "qx", &qx) : nullptr);
    Ref r_sx(r_qx ? given_or_new(a[6], *x, {M}, at::kHalf, "sx", &sx) : nullptr);
    Ref r_rs(r_sx ? given_or_new(a[7], *x, {M}, at::kInt, "rowsum", &rowsum) : nullptr);
    Workspace ws;
    if (!r_rs || !ws.ready(a[8], *x, M, N, K, mode, s)) return nullptr;
    const void* xp = x->data_ptr();
    if (!call([&] {
            return qoq_w4a8_linear(xp, packed, M, N, K, (int)mode, out, static_cast<int8_t*>(qx), sx, static_cast<int32_t*>(rowsum), ws.ptr,
                                   ws.bytes, s);
        }))
        return nullptr;
    return Py_BuildValue("NNNN", r_out.release(), r_qx.release(), r_sx.release(), r_rs.release());
    END_HANDLE_TH_ERRORS
}

PyObject* kv4_append(PyObject*, PyObject* const* a, Py_ssize_t n)    // cache, k, v, positions, S_max
{
    HANDLE_TH_ERRORS
    if (!counted(n, 5)) return nullptr;
    const at::Tensor* k = dev_tensor(a[1], at::kHalf, "k");
    const at::Tensor* v = k ? dev_tensor(a[2], at::kHalf, "v") : nullptr;
    const at::Tensor* pos = v ? dev_tensor(a[3], at::kInt, "positions") : nullptr;
    int64_t S_max;
    void* cache;
    if (!pos || !has_dims(*k, 4, "k") || !integer(a[4], &S_max) || !pointer(a[0], "cache", &cache)) return nullptr;
    const int64_t B = k->size(0), T = k->size(1), Hkv = k->size(2), D = k->size(3);
    void* s = stream_of(*k);
    const void *kp = k->data_ptr(), *vp = v->data_ptr();
    const int32_t* pp = static_cast<const int32_t*>(pos->data_ptr());
    if (!call([&] { return qoq_kv4_append(kp, vp, pp, B, T, Hkv, D, S_max, cache, s); })) return nullptr;
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

PyObject* kv4_attention_decode(PyObject*, PyObject* const* a, Py_ssize_t n)    // q, cache, seq_lens, Hkv, S_max, out, workspace
{
    HANDLE_TH_ERRORS
    if (!counted(n, 7)) return nullptr;
    const at::Tensor* q = dev_tensor(a[0], at::kHalf, "q");
    const at::Tensor* lens = q ? dev_tensor(a[2], at::kInt, "seq_lens") : nullptr;
    int64_t Hkv, S_max;
    void *cache, *out;
    if (!lens || !has_dims(*q, 3, "q") || !integer(a[3], &Hkv) || !integer(a[4], &S_max) || !pointer(a[1], "cache", &cache)) return nullptr;
    const int64_t B = q->size(0), H = q->size(1), D = q->size(2);
    void* s = stream_of(*q);
    Ref res(given_or_new(a[5], *q, {B, H, D}, at::kHalf, "out", &out));
    if (!res) return nullptr;
    const void* qp = q->data_ptr();
    const int32_t* lp = static_cast<const int32_t*>(lens->data_ptr());
    if (a[6] == Py_None) {
        if (!call([&] { return qoq_kv4_attention_decode(qp, cache, lp, B, H, Hkv, D, S_max, out, s); })) return nullptr;
    } else {
        const at::Tensor* ws = tensor(a[6], "workspace");
        if (!ws) return nullptr;
        void* wp = ws->data_ptr();
        const size_t bytes = (size_t)ws->numel();
        if (!call([&] { return qoq_kv4_attention_decode_split(qp, cache, lp, B, H, Hkv, D, S_max, out, wp, bytes, s); })) return nullptr;
    }
    return res.release();
    END_HANDLE_TH_ERRORS
}

// ---- paged cache and prompt attention: every tensor of a call lies on one GPU, which is the current one while the call launches ----

// heads of tokens: FP16 [rows, heads, 128] on `device`, contiguous but for the stride from token to token
const at::Tensor* heads_tensor(PyObject* o, const char* name, int device)
{
    const at::Tensor* t = tensor(o, name);
    if (!t) return nullptr;
    if (!t->is_cuda() || t->scalar_type() != at::kHalf) {
        PyErr_Format(PyExc_TypeError, "%s: expected a torch.float16 tensor on the GPU", name);
        return nullptr;
    }
    if (!has_dims(*t, 3, name)) return nullptr;
    if (device >= 0 && t->get_device() != device) {
        PyErr_Format(PyExc_ValueError, "%s: expected on the GPU of the other tensors", name);
        return nullptr;
    }
    if (t->size(2) != 128 || (t->stride(2) != 1 && t->numel()) || (t->stride(1) != 128 && t->size(1) > 1 && t->numel())) {
        PyErr_Format(PyExc_ValueError, "%s: expected [rows, heads, 128] with contiguous heads", name);
        return nullptr;
    }
    return t;
}
// elements from token to token; a single token's stride means nothing
int64_t token_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : (t.size(1) * 128 + 7) / 8 * 8; }

bool have_shape(const at::Tensor& t, at::IntArrayRef shape, const char* name)
{
    if (t.sizes() == shape) return true;
    PyErr_Format(PyExc_ValueError, "%s: unexpected shape", name);
    return false;
}

// a contiguous tensor of this type and number of dimensions on `device`
const at::Tensor* dense(PyObject* o, at::ScalarType dtype, int64_t dims, const char* name, int device)
{
    const at::Tensor* t = dev_tensor(o, dtype, name);
    if (!t || !has_dims(*t, dims, name)) return nullptr;
    if (t->get_device() == device) return t;
    PyErr_Format(PyExc_ValueError, "%s: expected on the GPU of the other tensors", name);
    return nullptr;
}

// None, or as above
bool dense_or_none(PyObject* o, at::ScalarType dtype, int64_t dims, const char* name, int device, const at::Tensor** t)
{
    *t = nullptr;
    return o == Py_None || (*t = dense(o, dtype, dims, name, device)) != nullptr;
}

struct Pool {
    const at::Tensor *bytes, *table;
    int64_t pages, width;
    bool ready(PyObject* pool, PyObject* block_table, int64_t B, int64_t Hkv, int device)
    {
        bytes = dense(pool, at::kByte, 1, "pool", device);
        table = bytes ? dense(block_table, at::kInt, 2, "block_table", device) : nullptr;
        if (!table) return false;
        if (table->size(0) != B) {
            PyErr_SetString(PyExc_ValueError, "block_table: expected a row for each sequence");
            return false;
        }
        const size_t page = qoq_kv4_pool_bytes(1, Hkv, 128);
        pages = page ? (int64_t)((size_t)bytes->numel() / page) : 0;      // none: refused by the call
        width = table->size(1);
        return true;
    }
};

struct Scratch {
    void* ptr = nullptr;
    size_t bytes = 0;
    bool ready(PyObject* o, int device)
    {
        if (o == Py_None) return true;
        const at::Tensor* t = tensor(o, "workspace");
        if (!t) return false;
        if (!t->is_cuda() || t->get_device() != device || !t->is_contiguous()) {
            PyErr_SetString(PyExc_TypeError, "workspace: expected a contiguous tensor on the GPU of the other tensors");
            return false;
        }
        ptr = t->data_ptr();
        bytes = (size_t)t->numel() * t->element_size();
        return true;
    }
};

// q, k, v, pool, block_table, cu, starts, angles, q_gamma, k_gamma, eps, interleaved, q_out, k_out, want_k
PyObject* qk_rope_kv4_append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (!counted(n, 15)) return nullptr;
    const at::Tensor* k = heads_tensor(a[1], "k", -1);
    if (!k) return nullptr;
    const int dev = k->get_device();
    const at::Tensor* v = heads_tensor(a[2], "v", dev);
    if (!v) return nullptr;
    const at::Tensor* q = nullptr;
    if (a[0] != Py_None && !(q = heads_tensor(a[0], "q", dev))) return nullptr;
    const at::Tensor* cu = dense(a[5], at::kInt, 1, "cu", dev);
    if (!cu) return nullptr;
    const int64_t M = k->size(0), Hkv = k->size(1), H = q ? q->size(1) : 0, B = cu->numel() - 1;
    if (!have_shape(*v, {M, Hkv, 128}, "v") || (q && !have_shape(*q, {M, H, 128}, "q"))) return nullptr;
    const at::Tensor *starts, *angles, *qg, *kg;
    Pool pool;
    double eps;
    bool interleaved, want_k;
    if (!dense_or_none(a[6], at::kInt, 1, "starts", dev, &starts) || (starts && !have_shape(*starts, {B}, "starts")) ||
        !dense_or_none(a[7], at::kFloat, 2, "angles", dev, &angles) || !dense_or_none(a[8], at::kHalf, 1, "q_gamma", dev, &qg) ||
        (qg && !have_shape(*qg, {128}, "q_gamma")) || !dense_or_none(a[9], at::kHalf, 1, "k_gamma", dev, &kg) ||
        (kg && !have_shape(*kg, {128}, "k_gamma")) || !pool.ready(a[3], a[4], B, Hkv, dev) || !number(a[10], &eps) || !flag(a[11], &interleaved) ||
        !flag(a[14], &want_k))
        return nullptr;
    c10::hip::HIPGuard guard(static_cast<c10::DeviceIndex>(dev));
    at::Tensor q_out, k_out;
    if (a[12] != Py_None) {
        const at::Tensor* t = heads_tensor(a[12], "q_out", dev);
        if (!t || !have_shape(*t, {M, H, 128}, "q_out")) return nullptr;
        q_out = *t;
    } else if (q) {
        q_out = new_like(*q, {M, H, 128}, at::kHalf);
    }
    if (a[13] != Py_None) {
        const at::Tensor* t = heads_tensor(a[13], "k_out", dev);
        if (!t || !have_shape(*t, {M, Hkv, 128}, "k_out")) return nullptr;
        k_out = *t;
    } else if (want_k) {
        k_out = new_like(*k, {M, Hkv, 128}, at::kHalf);
    }
    void* s = stream_of(*k);
    auto at_or_null = [](const at::Tensor* t) { return t ? t->data_ptr() : nullptr; };
    const void *qp = at_or_null(q), *kp = k->data_ptr(), *vp = v->data_ptr(), *qgp = at_or_null(qg), *kgp = at_or_null(kg);
    const float* ap = static_cast<const float*>(at_or_null(angles));
    const int32_t *cp = static_cast<const int32_t*>(cu->data_ptr()), *sp = static_cast<const int32_t*>(at_or_null(starts));
    const int32_t* tp = static_cast<const int32_t*>(pool.table->data_ptr());
    void *pp = pool.bytes->data_ptr(), *qo = q_out.defined() ? q_out.data_ptr() : nullptr, *ko = k_out.defined() ? k_out.data_ptr() : nullptr;
    const int64_t qs = q ? token_stride(*q) : 0, ks = token_stride(*k), vs = token_stride(*v), qos = q_out.defined() ? token_stride(q_out) : 0,
                  kos = k_out.defined() ? token_stride(k_out) : 0, rows = angles ? angles->size(0) : 0, rot = angles ? angles->size(1) : 0;
    if (!call([&] {
            return qoq_qk_rope_kv4_append(qp, qs, kp, ks, vp, vs, qgp, kgp, eps, ap, rows, rot, interleaved, cp, sp, M, B, H, Hkv, 128, pp, pool.pages, tp,
                                          pool.width, qo, qos, ko, kos, s);
        }))
        return nullptr;
    return Py_BuildValue("NN", Quantized::wrap(q_out), Quantized::wrap(k_out));
    END_HANDLE_TH_ERRORS
}

// the caller's tensor of this shape, contiguous, or a new one
bool dense_or_new(PyObject* o, const at::Tensor& on, at::IntArrayRef shape, const char* name, at::Tensor& t)
{
    if (o == Py_None) {
        t = new_like(on, shape, at::kHalf);
        return true;
    }
    const at::Tensor* given = dense(o, at::kHalf, (int64_t)shape.size(), name, on.get_device());
    if (!given || !have_shape(*given, shape, name)) return false;
    t = *given;
    return true;
}

PyObject* kv4_paged_gather(PyObject*, PyObject* const* a, Py_ssize_t n)    // pool, block_table, cu, starts, rows, Hkv, k_out, v_out
{
    HANDLE_TH_ERRORS
    if (!counted(n, 8)) return nullptr;
    const at::Tensor* cu = dev_tensor(a[2], at::kInt, "cu");
    if (!cu || !has_dims(*cu, 1, "cu")) return nullptr;
    const int dev = cu->get_device();
    const int64_t B = cu->numel() - 1;
    const at::Tensor* starts;
    int64_t M, Hkv;
    Pool pool;
    if (!dense_or_none(a[3], at::kInt, 1, "starts", dev, &starts) || (starts && !have_shape(*starts, {B}, "starts")) || !integer(a[4], &M) ||
        !integer(a[5], &Hkv) || !pool.ready(a[0], a[1], B, Hkv, dev))
        return nullptr;
    c10::hip::HIPGuard guard(static_cast<c10::DeviceIndex>(dev));
    at::Tensor k, v;
    if (M < 0 || Hkv < 0) return call([] { return (int)QOQ_ERR_SHAPE; }), nullptr;
    if (!dense_or_new(a[6], *cu, {M, Hkv, 128}, "k_out", k) || !dense_or_new(a[7], *cu, {M, Hkv, 128}, "v_out", v)) return nullptr;
    void *s = stream_of(*cu), *kp = k.data_ptr(), *vp = v.data_ptr();
    const void* pp = pool.bytes->data_ptr();
    const int32_t *tp = static_cast<const int32_t*>(pool.table->data_ptr()), *cp = static_cast<const int32_t*>(cu->data_ptr());
    const int32_t* sp = starts ? static_cast<const int32_t*>(starts->data_ptr()) : nullptr;
    if (!call([&] { return qoq_kv4_paged_gather(pp, pool.pages, tp, pool.width, cp, sp, M, B, Hkv, 128, kp, vp, s); })) return nullptr;
    return Py_BuildValue("NN", THPVariable_Wrap(k), THPVariable_Wrap(v));
    END_HANDLE_TH_ERRORS
}

// q, pool, block_table, seq_lens, Hkv, window, sinks, out, workspace
PyObject* kv4_paged_attention_decode(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (!counted(n, 9)) return nullptr;
    const at::Tensor* q = heads_tensor(a[0], "q", -1);
    if (!q) return nullptr;
    const int dev = q->get_device();
    const int64_t B = q->size(0), H = q->size(1);
    const at::Tensor* lens = dense(a[3], at::kInt, 1, "seq_lens", dev);
    int64_t Hkv, window, sinks;
    Pool pool;
    Scratch ws;
    at::Tensor out;
    if (!lens || !have_shape(*lens, {B}, "seq_lens") || !integer(a[4], &Hkv) || !integer(a[5], &window) || !integer(a[6], &sinks) ||
        !pool.ready(a[1], a[2], B, Hkv, dev) || !ws.ready(a[8], dev))
        return nullptr;
    c10::hip::HIPGuard guard(static_cast<c10::DeviceIndex>(dev));
    if (!dense_or_new(a[7], *q, {B, H, 128}, "out", out)) return nullptr;
    void *s = stream_of(*q), *op = out.data_ptr();
    const void *qp = q->data_ptr(), *pp = pool.bytes->data_ptr();
    const int32_t *tp = static_cast<const int32_t*>(pool.table->data_ptr()), *lp = static_cast<const int32_t*>(lens->data_ptr());
    const int64_t stride = token_stride(*q);
    if (!call([&] {
            return qoq_kv4_paged_attention_decode(qp, stride, pp, pool.pages, tp, pool.width, lp, B, H, Hkv, 128, window, sinks, op, ws.ptr, ws.bytes, s);
        }))
        return nullptr;
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

PyObject* attention_prefill(PyObject*, PyObject* const* a, Py_ssize_t n)    // q, k, v, cu_q, cu_k, window, sinks, out, workspace
{
    HANDLE_TH_ERRORS
    if (!counted(n, 9)) return nullptr;
    const at::Tensor* q = heads_tensor(a[0], "q", -1);
    if (!q) return nullptr;
    const int dev = q->get_device();
    const at::Tensor* k = heads_tensor(a[1], "k", dev);
    const at::Tensor* v = k ? heads_tensor(a[2], "v", dev) : nullptr;
    const at::Tensor* cu_q = v ? dense(a[3], at::kInt, 1, "cu_q", dev) : nullptr;
    const at::Tensor* cu_k = cu_q ? dense(a[4], at::kInt, 1, "cu_k", dev) : nullptr;
    int64_t window, sinks;
    Scratch ws;
    at::Tensor out;
    if (!cu_k || !have_shape(*v, k->sizes(), "v") || !have_shape(*cu_k, cu_q->sizes(), "cu_k") || !integer(a[5], &window) || !integer(a[6], &sinks) ||
        !ws.ready(a[8], dev))
        return nullptr;
    const int64_t M = q->size(0), H = q->size(1), Mk = k->size(0), Hkv = k->size(1), B = cu_q->numel() - 1;
    c10::hip::HIPGuard guard(static_cast<c10::DeviceIndex>(dev));
    if (!dense_or_new(a[7], *q, {M, H, 128}, "out", out)) return nullptr;
    void *s = stream_of(*q), *op = out.data_ptr();
    const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
    const int32_t *cq = static_cast<const int32_t*>(cu_q->data_ptr()), *ck = static_cast<const int32_t*>(cu_k->data_ptr());
    const int64_t qs = token_stride(*q), ks = token_stride(*k), vs = token_stride(*v);
    if (!call([&] { return qoq_attention_prefill(qp, qs, kp, ks, vp, vs, cq, ck, M, Mk, B, H, Hkv, 128, window, sinks, op, ws.ptr, ws.bytes, s); }))
        return nullptr;
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

PyObject* set_raise_status(PyObject*, PyObject* f)
{
    Py_INCREF(f);
    Py_XSETREF(g_raise_status, f);
    Py_RETURN_NONE;
}

// The order of salient channels, and whether it is one: the kernel says so in pinned host memory.  The call returns when the order is complete,
// which callers may then use, and salience reuse, on any stream.  (Returning with the verdict, which is there when the others begin to
// sort, 4096 x 14336 reordered and packed takes 96 us a pass and not 109, but other streams then read an order that is not there yet.  Flags that
// the sorting workgroups set when their parts are in memory, polled in place of the stream, 108; with a system-wide fence each 113.)
PyObject* channel_order(PyObject*, PyObject* const* a, Py_ssize_t n)    // salience
{
    HANDLE_TH_ERRORS
    if (!counted(n, 1)) return nullptr;
    const at::Tensor* sal = dev_tensor(a[0], at::kFloat, "salience");
    if (!sal) return nullptr;
    const hipStream_t s = static_cast<hipStream_t>(stream_of(*sal));
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(s, &capture) != hipSuccess || capture != hipStreamCaptureStatusNone) {
        (void)hipGetLastError();                // (the default stream beside a capture: not the next launch's error)
        PyErr_SetString(PyExc_RuntimeError, "channel_order reads a result on the host: not while the stream is being captured");
        return nullptr;
    }
    const int64_t K = sal->numel();
    at::Tensor perm = new_like(*sal, {K}, at::kInt);
    at::Tensor pinned = at::empty({1}, at::TensorOptions().dtype(at::kInt).pinned_memory(true));
    int32_t* verdict = static_cast<int32_t*>(pinned.data_ptr());
    const float* sp = static_cast<const float*>(sal->data_ptr());
    int32_t* pp = static_cast<int32_t*>(perm.data_ptr());
    __atomic_store_n(verdict, -1, __ATOMIC_RELEASE);
    if (!call([&] {
            const int status = qoq_channel_order(sp, K, pp, verdict, s);
            if (status != QOQ_OK) return status;
            if (hipStreamSynchronize(s) != hipSuccess) return (int)QOQ_ERR_HIP;
            const int v = __atomic_load_n(verdict, __ATOMIC_ACQUIRE);
            return v == 0 ? (int)QOQ_OK : v > 0 ? (int)QOQ_ERR_SHAPE : (int)QOQ_ERR_HIP;
        }))
        return nullptr;
    return THPVariable_Wrap(perm);
    END_HANDLE_TH_ERRORS
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(quant_act), FAST(quant_act_reordered), FAST(rmsnorm_quant), FAST(silu_mul_quant), FAST(w4a8_gemm),
                         FAST(w4a8_gemm_noalloc), FAST(w4a8_gemm_token_sum), FAST(w4a8_linear), FAST(kv4_append), FAST(kv4_attention_decode), FAST(channel_order),
                         FAST(qk_rope_kv4_append), FAST(kv4_paged_gather), FAST(kv4_paged_attention_decode), FAST(attention_prefill),
                         {"set_raise_status", set_raise_status, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
#undef FAST
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qoq_py", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: the torch whose classes this was compiled against; api.py refuses any other.
PyMODINIT_FUNC PyInit__qoq_py(void)
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", QOQ_TORCH_VERSION) != 0) Py_CLEAR(m);
    return m;
}
