// Argument marshalling of the layer's online calls in native code.  A decode step of a small layer runs for
// 5 to 7 us on the GPU; marshalling it in Python (attribute look-ups, two torch.empty, twenty ctypes conversions)
// took the host about 11 us per call, so that a loop of eager calls was bound by it: 1 x 4096 x 4096 13.9 us a
// call with it, 5.9 us with this.  The calls around the layer (norm 6.9 us here on the host, cache write 4.4, read 6.5) bind their
// smallest steps the same way.
//
// Every function takes the address of the C entry point (the library is loaded by Python) and returns
//   a tensor or a tuple of tensors   on success,
//   an int                           the entry point's status when it is not W4A8_OK,
//   NotImplemented                   for operands that are not plain torch tensors of the expected kind, and sizes
//                                    that are not 64-bit ints: the caller's Python form decides what to do with them.
// Nothing is cached between calls.  The GIL is released around the entry points, as ctypes does.
#include <torch/extension.h>

#include "../../include/w4a8.h"

namespace {

constexpr int LAYOUT_TILED = W4A8_LAYOUT_TILED;

// an int that fits 64 bits; anything else (floats, strings, array scalars) is the Python form's to convert or refuse
bool to_i64(PyObject *o, int64_t &v)
{
    if (!PyLong_Check(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}
template <typename F>
bool to_fn(PyObject *o, F &f)
{
    f = reinterpret_cast<F>(PyLong_AsVoidPtr(o));
    return !PyErr_Occurred();
}

// plain tensors only (no subclass may observe or replace these calls)
bool plain(PyObject *o) { return THPVariable_CheckExact(o); }
bool plain_or_none(PyObject *o) { return o == Py_None || THPVariable_CheckExact(o); }
void *ptr(PyObject *o) { return o == Py_None ? nullptr : THPVariable_Unpack(o).data_ptr(); }

// element type of activations / outputs: its id, or -1
int dtype_id(at::ScalarType t)
{
    switch (t) {
        case at::kFloat: return W4A8_F32;
        case at::kHalf: return W4A8_F16;
        case at::kBFloat16: return W4A8_BF16;
        default: return -1;
    }
}
at::ScalarType y_type(int64_t id)
{
    return id == W4A8_F16 ? at::kHalf : id == W4A8_BF16 ? at::kBFloat16 : at::kFloat;
}

struct Rows {   // a 2-D activation tensor with contiguous rows
    int64_t M, K, ld;
    int dtype;
    bool ok;
};
Rows rows_of(const at::Tensor &X)
{
    Rows r{0, 0, 0, -1, false};
    if (X.dim() != 2 || X.stride(1) != 1) return r;
    r.M = X.size(0);
    r.K = X.size(1);
    r.ld = r.M > 1 ? X.stride(0) : std::max(X.stride(0), r.K);
    r.dtype = dtype_id(X.scalar_type());
    r.ok = r.dtype >= 0;
    return r;
}

at::Tensor make(const at::Tensor &like, at::IntArrayRef size, at::ScalarType t)
{
    return at::empty(size, like.options().dtype(t));
}

// Scratch of the size that a call would like, or of the size that it has to have where the allocator does not give so much
// (undefined for none).
at::Tensor scratch(const at::Tensor &like, size_t preferred, size_t least)
{
    if (preferred > least) {
        try {
            return make(like, {(int64_t)preferred}, at::kByte);
        } catch (const c10::OutOfMemoryError &) {
        }
    }
    return least > 0 ? make(like, {(int64_t)least}, at::kByte) : at::Tensor();
}
void *data(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
size_t size(const at::Tensor &t) { return t.defined() ? (size_t)t.numel() : 0; }

PyObject *not_implemented() { Py_RETURN_NOTIMPLEMENTED; }
PyObject *status(int rc) { return PyLong_FromLong(rc); }

// act_quant(entry, X, s, stream) -> (Xq, sx)
PyObject *act_quant(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS   // (torch's own translation: an allocation that fails stays torch.OutOfMemoryError)
    if (n != 4 || !plain(a[1]) || !plain_or_none(a[2])) return not_implemented();
    decltype(&quantize_act_int8) entry;
    int64_t stream;
    if (!to_fn(a[0], entry)) return nullptr;
    if (!to_i64(a[3], stream)) return not_implemented();
    const at::Tensor &X = THPVariable_Unpack(a[1]);
    const Rows r = rows_of(X);
    if (!r.ok) return not_implemented();
    at::Tensor Xq = make(X, {r.M, r.K}, at::kChar), sx = make(X, {r.M}, at::kFloat);
    const void *x = X.data_ptr();
    const float *s = (const float *)ptr(a[2]);
    int8_t *q = (int8_t *)Xq.data_ptr();
    float *sxp = (float *)sx.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(x, r.dtype, r.M, r.K, r.ld, s, q, sxp, (void *)stream);
    Py_END_ALLOW_THREADS
    if (rc != W4A8_OK) return status(rc);
    return PyTuple_Pack(2, py::reinterpret_steal<py::object>(THPVariable_Wrap(Xq)).ptr(),
                        py::reinterpret_steal<py::object>(THPVariable_Wrap(sx)).ptr());
    END_HANDLE_TH_ERRORS
}

// act_quant_asym(entry, X, s, stream) -> (Xq, sx, zx)
PyObject *act_quant_asym(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 4 || !plain(a[1]) || !plain_or_none(a[2])) return not_implemented();
    decltype(&quantize_act_int8_asym) entry;
    int64_t stream;
    if (!to_fn(a[0], entry)) return nullptr;
    if (!to_i64(a[3], stream)) return not_implemented();
    const at::Tensor &X = THPVariable_Unpack(a[1]);
    const Rows r = rows_of(X);
    if (!r.ok) return not_implemented();
    at::Tensor Xq = make(X, {r.M, r.K}, at::kChar), sx = make(X, {r.M}, at::kFloat), zx = make(X, {r.M}, at::kInt);
    const void *x = X.data_ptr();
    const float *s = (const float *)ptr(a[2]);
    int8_t *q = (int8_t *)Xq.data_ptr();
    float *sxp = (float *)sx.data_ptr();
    int32_t *zxp = (int32_t *)zx.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(x, r.dtype, r.M, r.K, r.ld, s, q, sxp, zxp, (void *)stream);
    Py_END_ALLOW_THREADS
    if (rc != W4A8_OK) return status(rc);
    return PyTuple_Pack(3, py::reinterpret_steal<py::object>(THPVariable_Wrap(Xq)).ptr(),
                        py::reinterpret_steal<py::object>(THPVariable_Wrap(sx)).ptr(),
                        py::reinterpret_steal<py::object>(THPVariable_Wrap(zx)).ptr());
    END_HANDLE_TH_ERRORS
}

// gemm(entry, preferred_workspace_entry, workspace_entry, Xq, sx, Wp, step, zero, N, K, group_size, layout, y_dtype, stream) -> Y
PyObject *gemm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 14) return not_implemented();
    for (int i = 3; i < 8; ++i)
        if (!plain(a[i])) return not_implemented();
    decltype(&w4a8_gemm) entry;
    decltype(&w4a8_gemm_workspace_bytes) wish, need;
    int64_t N, K, G, layout, yd, stream;
    if (!to_fn(a[0], entry) || !to_fn(a[1], wish) || !to_fn(a[2], need)) return nullptr;
    if (!to_i64(a[8], N) || !to_i64(a[9], K) || !to_i64(a[10], G) ||
        !to_i64(a[11], layout) || !to_i64(a[12], yd) || !to_i64(a[13], stream))
        return not_implemented();
    const at::Tensor &Xq = THPVariable_Unpack(a[3]);
    if (Xq.dim() < 1 || N < 0) return not_implemented();
    const int64_t M = Xq.size(0);
    at::Tensor Y = make(Xq, {M, N}, y_type(yd));
    const at::Tensor ws = scratch(Xq, wish(M, N, K, G, (int)layout), need(M, N, K, G, (int)layout));
    const size_t bytes = size(ws);
    const int8_t *q = (const int8_t *)ptr(a[3]);
    const float *sx = (const float *)ptr(a[4]), *step = (const float *)ptr(a[6]);
    const uint8_t *Wp = (const uint8_t *)ptr(a[5]), *zero = (const uint8_t *)ptr(a[7]);
    void *y = Y.data_ptr(), *w = data(ws);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(q, sx, M, Wp, (int)layout, step, zero, N, K, G, y, (int)yd, N, nullptr, w, bytes, (void *)stream);
    Py_END_ALLOW_THREADS
    return rc != W4A8_OK ? status(rc) : THPVariable_Wrap(Y);
    END_HANDLE_TH_ERRORS
}

// gemm_asym(entry, workspace_entry, Xq, sx, zx, Wp, step, zero, wsum, tsum, N, K, group_size, layout, y_dtype,
//           stream) -> Y
PyObject *gemm_asym(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 16) return not_implemented();
    for (int i = 2; i < 10; ++i)
        if (!plain(a[i])) return not_implemented();
    decltype(&w4a8_gemm_asym) entry;
    decltype(&w4a8_gemm_workspace_bytes) need;
    int64_t N, K, G, layout, yd, stream;
    if (!to_fn(a[0], entry) || !to_fn(a[1], need)) return nullptr;
    if (!to_i64(a[10], N) || !to_i64(a[11], K) || !to_i64(a[12], G) ||
        !to_i64(a[13], layout) || !to_i64(a[14], yd) || !to_i64(a[15], stream))
        return not_implemented();
    const at::Tensor &Xq = THPVariable_Unpack(a[2]);
    if (Xq.dim() < 1 || N < 0) return not_implemented();
    const int64_t M = Xq.size(0);
    at::Tensor Y = make(Xq, {M, N}, y_type(yd));
    const size_t bytes = need(M, N, K, G, (int)layout);
    at::Tensor ws;
    if (bytes > 0) ws = make(Xq, {(int64_t)bytes}, at::kByte);
    const int8_t *q = (const int8_t *)ptr(a[2]);
    const float *sx = (const float *)ptr(a[3]), *step = (const float *)ptr(a[6]);
    const int32_t *zx = (const int32_t *)ptr(a[4]), *wsum = (const int32_t *)ptr(a[8]), *tsum = (const int32_t *)ptr(a[9]);
    const uint8_t *Wp = (const uint8_t *)ptr(a[5]), *zero = (const uint8_t *)ptr(a[7]);
    void *y = Y.data_ptr(), *w = bytes > 0 ? ws.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(q, sx, zx, M, Wp, (int)layout, step, zero, wsum, tsum, N, K, G, y, (int)yd, N, nullptr, w, bytes,
               (void *)stream);
    Py_END_ALLOW_THREADS
    return rc != W4A8_OK ? status(rc) : THPVariable_Wrap(Y);
    END_HANDLE_TH_ERRORS
}

// linear(entry, preferred_workspace_entry, workspace_entry, act_quant_entry, gemm_entry, gemm_workspace_entry, X, s, Wp, step,
//        zero, N, group_size, layout, y_dtype, stream) -> Y
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 16 || !plain(a[6]) || !plain_or_none(a[7]) || !plain(a[8]) || !plain(a[9]) || !plain(a[10]))
        return not_implemented();
    decltype(&w4a8_linear) entry;
    decltype(&w4a8_linear_workspace_bytes) wish, need;
    decltype(&quantize_act_int8) quantize;
    decltype(&w4a8_gemm) product;
    decltype(&w4a8_gemm_workspace_bytes) product_need;
    int64_t N, G, layout, yd, stream;
    if (!to_fn(a[0], entry) || !to_fn(a[1], wish) || !to_fn(a[2], need) || !to_fn(a[3], quantize) ||
        !to_fn(a[4], product) || !to_fn(a[5], product_need))
        return nullptr;
    if (!to_i64(a[11], N) || !to_i64(a[12], G) ||
        !to_i64(a[13], layout) || !to_i64(a[14], yd) || !to_i64(a[15], stream))
        return not_implemented();
    const at::Tensor &X = THPVariable_Unpack(a[6]);
    const Rows r = rows_of(X);
    if (!r.ok || N < 0) return not_implemented();
    at::Tensor Y = make(X, {r.M, N}, y_type(yd));
    const void *x = X.data_ptr();
    const float *s = (const float *)ptr(a[7]), *step = (const float *)ptr(a[9]);
    const uint8_t *Wp = (const uint8_t *)ptr(a[8]), *zero = (const uint8_t *)ptr(a[10]);
    void *y = Y.data_ptr();
    int rc = W4A8_ERR_WORKSPACE;
    if (r.M > 4 && r.M <= 16 && r.K >= 5120 && r.dtype == W4A8_F16 && layout == LAYOUT_TILED) {
        // the two steps by themselves, faster here than in one launch (the times stand beside w4a8_linear's rule)
        const size_t bytes = product_need(r.M, N, r.K, G, (int)layout);
        const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };   // (one allocation: three cost the host 0.3 us more)
        const int64_t sx_at = up(r.M * r.K), ws_at = sx_at + up(4 * r.M);
        const at::Tensor room = make(X, {ws_at + (int64_t)bytes}, at::kByte);
        uint8_t *p = (uint8_t *)room.data_ptr();
        int8_t *q = (int8_t *)p;
        float *sxp = (float *)(p + sx_at);
        void *w = bytes > 0 ? p + ws_at : nullptr;
        Py_BEGIN_ALLOW_THREADS
        rc = quantize(x, r.dtype, r.M, r.K, r.ld, s, q, sxp, (void *)stream);
        if (rc == W4A8_OK)
            rc = product(q, sxp, r.M, Wp, (int)layout, step, zero, N, r.K, G, y, (int)yd, N, nullptr, w, bytes, (void *)stream);
        Py_END_ALLOW_THREADS
        return rc != W4A8_OK ? status(rc) : THPVariable_Wrap(Y);
    }
    auto call = [&](void *w, size_t bytes) {
        Py_BEGIN_ALLOW_THREADS
        rc = entry(x, r.dtype, r.M, r.K, r.ld, s, Wp, (int)layout, step, zero, N, G, y, (int)yd, N, nullptr, nullptr,
                   nullptr, w, bytes, (void *)stream);
        Py_END_ALLOW_THREADS
    };
    // The one-launch decode step needs no workspace: try without (a call that needs one is turned down
    // before anything is launched).
    if (r.M <= 16 && r.dtype == W4A8_F16 && layout == LAYOUT_TILED) call(nullptr, 0);
    if (rc == W4A8_ERR_WORKSPACE) {
        const at::Tensor ws = scratch(X, wish(r.M, N, r.K, G, (int)layout), need(r.M, N, r.K, G, (int)layout));
        call(data(ws), size(ws));
    }
    return rc != W4A8_OK ? status(rc) : THPVariable_Wrap(Y);
    END_HANDLE_TH_ERRORS
}

// rms_norm(entry, X, w, eps, residual, s, stream) -> (Xq, sx) or (Xq, sx, h)
PyObject *rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 7 || !plain(a[1]) || !plain(a[2]) || !PyFloat_Check(a[3]) || !plain_or_none(a[4]) || !plain_or_none(a[5])) return not_implemented();
    decltype(&rms_norm_act_int8) entry;
    int64_t stream;
    if (!to_fn(a[0], entry)) return nullptr;
    if (!to_i64(a[6], stream)) return not_implemented();
    const at::Tensor &X = THPVariable_Unpack(a[1]), &w = THPVariable_Unpack(a[2]);
    const Rows r = rows_of(X);
    const int wd = dtype_id(w.scalar_type());
    if (!r.ok || wd < 0 || w.dim() != 1 || w.size(0) != r.K || !w.is_contiguous() || w.device() != X.device()) return not_implemented();
    const float *s = nullptr;
    if (a[5] != Py_None) {
        const at::Tensor &st = THPVariable_Unpack(a[5]);
        if (st.scalar_type() != at::kFloat || st.dim() != 1 || st.size(0) != r.K || !st.is_contiguous() || st.device() != X.device()) return not_implemented();
        s = (const float *)st.data_ptr();
    }
    at::Tensor h;
    Rows rr{0, 0, 0, -1, false};
    const void *res = nullptr;
    if (a[4] != Py_None) {
        const at::Tensor &R = THPVariable_Unpack(a[4]);
        rr = rows_of(R);
        if (!rr.ok || rr.M != r.M || rr.K != r.K || rr.dtype != r.dtype || R.device() != X.device()) return not_implemented();
        res = R.data_ptr();
        h = make(X, {r.M, r.K}, X.scalar_type());
    }
    at::Tensor Xq = make(X, {r.M, r.K}, at::kChar), sx = make(X, {r.M}, at::kFloat);
    const void *x = X.data_ptr(), *wp = w.data_ptr();
    void *hp = data(h);
    int8_t *q = (int8_t *)Xq.data_ptr();
    float *sxp = (float *)sx.data_ptr();
    const double eps = PyFloat_AS_DOUBLE(a[3]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(x, r.dtype, r.M, r.K, r.ld, res, rr.ld, wp, wd, eps, s, hp, r.K, q, sxp, (void *)stream);
    Py_END_ALLOW_THREADS
    if (rc != W4A8_OK) return status(rc);
    py::object o0 = py::reinterpret_steal<py::object>(THPVariable_Wrap(Xq)), o1 = py::reinterpret_steal<py::object>(THPVariable_Wrap(sx));
    if (!h.defined()) return PyTuple_Pack(2, o0.ptr(), o1.ptr());
    py::object o2 = py::reinterpret_steal<py::object>(THPVariable_Wrap(h));
    return PyTuple_Pack(3, o0.ptr(), o1.ptr(), o2.ptr());
    END_HANDLE_TH_ERRORS
}

// The cache (four tensors) and the step's start, count, table: false where they are not what the entry points take.
bool kv_operands(PyObject *const *c, PyObject *const *t, w4a8_kv_cache &cache, w4a8_kv_tokens &tok, c10::Device &device)
{
    for (int i = 0; i < 4; ++i)
        if (!plain(c[i])) return false;
    if (!plain(t[0]) || !plain_or_none(t[1]) || !plain(t[2])) return false;
    const at::Tensor &kp = THPVariable_Unpack(c[0]);
    if (kp.dim() != 4) return false;
    device = kp.device();
    cache.pages = kp.size(0);
    cache.heads = kp.size(1);
    cache.page_size = kp.size(2);
    cache.head_dim = 2 * kp.size(3);
    for (int i = 0; i < 4; ++i) {
        const at::Tensor &x = THPVariable_Unpack(c[i]);
        const bool words = i & 1;
        if (x.dim() != (words ? 3 : 4) || x.scalar_type() != (words ? at::kInt : at::kByte) || x.device() != device) return false;
        for (int d = 0; d < x.dim(); ++d)
            if (x.size(d) != kp.size(d)) return false;
        // rows contiguous in a (page, head), and as far apart in all four (a dimension of one has no distance)
        const int64_t row = words ? 1 : kp.size(3), page = x.size(0) > 1 ? x.stride(0) : 0, head = x.size(1) > 1 ? x.stride(1) : 0;
        if (row < 1 || (!words && row > 1 && x.stride(3) != 1) || (x.size(2) > 1 && x.stride(2) != row) || page % row != 0 || head % row != 0) return false;
        if (i == 0) {
            cache.page_ld = page / row;
            cache.head_ld = head / row;
        } else if (cache.page_ld != page / row || cache.head_ld != head / row) {
            return false;
        }
    }
    cache.k_packed = (uint8_t *)kp.data_ptr();
    cache.k_words = (int32_t *)ptr(c[1]);
    cache.v_packed = (uint8_t *)ptr(c[2]);
    cache.v_words = (int32_t *)ptr(c[3]);
    const at::Tensor &start = THPVariable_Unpack(t[0]), &table = THPVariable_Unpack(t[2]);
    tok.batch = start.dim() == 1 ? start.size(0) : -1;
    const auto vec = [&](const at::Tensor &x) { return x.dim() == 1 && x.size(0) == tok.batch && x.scalar_type() == at::kInt && x.is_contiguous() && x.device() == device; };
    if (!vec(start) || (t[1] != Py_None && !vec(THPVariable_Unpack(t[1])))) return false;
    if (table.dim() != 2 || table.size(0) != tok.batch || table.scalar_type() != at::kInt || table.device() != device) return false;
    if (table.stride(1) != 1 && table.size(1) > 1) return false;
    tok.start = (const int32_t *)start.data_ptr();
    tok.count = (const int32_t *)ptr(t[1]);
    tok.table = (const int32_t *)table.data_ptr();
    tok.table_pages = table.size(1);
    tok.table_ld = tok.batch > 1 ? table.stride(0) : std::max(table.stride(0), table.size(1));
    return true;
}

// [batch, tokens, heads, channels] with the channels contiguous
bool kv_rows(const at::Tensor &x, const w4a8_kv_cache &cache, const w4a8_kv_tokens &tok, const c10::Device &device, int64_t (&ld)[3])
{
    if (x.dim() != 4 || x.size(0) != tok.batch || x.size(3) != cache.head_dim || x.stride(3) != 1 || x.device() != device) return false;
    for (int i = 0; i < 3; ++i) ld[i] = x.size(i) > 1 ? x.stride(i) : 0;
    return dtype_id(x.scalar_type()) >= 0;
}

// kv_write(entry, K, V, k_packed, k_words, v_packed, v_words, start, count, table, stream) -> None
PyObject *kv_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    decltype(&kv_cache_write_dint4) entry;
    int64_t stream, k_ld[3], v_ld[3];
    w4a8_kv_cache cache;
    w4a8_kv_tokens tok;
    c10::Device device(c10::kCPU);
    if (n != 11 || !plain(a[1]) || !plain(a[2]) || !kv_operands(a + 3, a + 7, cache, tok, device)) return not_implemented();
    if (!to_fn(a[0], entry)) return nullptr;
    if (!to_i64(a[10], stream)) return not_implemented();
    const at::Tensor &K = THPVariable_Unpack(a[1]), &V = THPVariable_Unpack(a[2]);
    if (!kv_rows(K, cache, tok, device, k_ld) || !kv_rows(V, cache, tok, device, v_ld) || K.sizes() != V.sizes() ||
        K.size(2) != cache.heads || K.scalar_type() != V.scalar_type())
        return not_implemented();
    tok.new_tokens = K.size(1);
    const void *k = K.data_ptr(), *v = V.data_ptr();
    const int dtype = dtype_id(K.scalar_type());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(k, k_ld, v, v_ld, dtype, &cache, &tok, (void *)stream);
    Py_END_ALLOW_THREADS
    if (rc != W4A8_OK) return status(rc);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// kv_read(entry, k_packed, k_words, v_packed, v_words, start, count, table, new_tokens, dtype, stream) -> (K, V)
PyObject *kv_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    decltype(&kv_cache_read_dint4) entry;
    int64_t S, dtype, stream;
    w4a8_kv_cache cache;
    w4a8_kv_tokens tok;
    c10::Device device(c10::kCPU);
    if (n != 11 || !kv_operands(a + 1, a + 5, cache, tok, device)) return not_implemented();
    if (!to_fn(a[0], entry)) return nullptr;
    if (!to_i64(a[8], S) || !to_i64(a[9], dtype) || !to_i64(a[10], stream) || S < 0) return not_implemented();
    tok.new_tokens = S;
    const at::Tensor &like = THPVariable_Unpack(a[1]);
    const int64_t size[4] = {tok.batch, S, cache.heads, cache.head_dim};
    at::Tensor K = make(like, size, y_type(dtype)), V = make(like, size, y_type(dtype));
    void *k = K.data_ptr(), *v = V.data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(&cache, &tok, k, v, (int)dtype, (void *)stream);
    Py_END_ALLOW_THREADS
    if (rc != W4A8_OK) return status(rc);
    return PyTuple_Pack(2, py::reinterpret_steal<py::object>(THPVariable_Wrap(K)).ptr(),
                        py::reinterpret_steal<py::object>(THPVariable_Wrap(V)).ptr());
    END_HANDLE_TH_ERRORS
}

// kv_attention(entry, workspace_entry, Q, k_packed, k_words, v_packed, v_words, start, count, table, scale, max_len, stream) -> out
PyObject *kv_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    decltype(&attention_kv_dint4) entry;
    decltype(&attention_kv_dint4_workspace_bytes) need;
    int64_t max_len, stream, q_ld[3];
    w4a8_kv_cache cache;
    w4a8_kv_tokens tok;
    c10::Device device(c10::kCPU);
    if (n != 13 || !plain(a[2]) || !kv_operands(a + 3, a + 7, cache, tok, device) || !PyFloat_Check(a[10])) return not_implemented();
    if (!to_fn(a[0], entry) || !to_fn(a[1], need)) return nullptr;
    if (!to_i64(a[11], max_len) || !to_i64(a[12], stream)) return not_implemented();
    const at::Tensor &Q = THPVariable_Unpack(a[2]);
    if (!kv_rows(Q, cache, tok, device, q_ld)) return not_implemented();
    tok.new_tokens = Q.size(1);
    const int64_t heads = Q.size(2);
    const int dtype = dtype_id(Q.scalar_type());
    at::Tensor out = make(Q, Q.sizes(), Q.scalar_type()), ws;
    const size_t bytes = need(dtype, heads, &cache, &tok, max_len);
    if (bytes > 0) ws = make(Q, {(int64_t)bytes}, at::kByte);
    const void *q = Q.data_ptr();
    void *o = out.data_ptr(), *w = data(ws);
    const float scale = (float)PyFloat_AS_DOUBLE(a[10]);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(q, q_ld, dtype, heads, &cache, &tok, scale, max_len, o, w, bytes, (void *)stream);
    Py_END_ALLOW_THREADS
    return rc != W4A8_OK ? status(rc) : THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"rms_norm", (PyCFunction)(void (*)(void))rms_norm, METH_FASTCALL, nullptr},
    {"kv_write", (PyCFunction)(void (*)(void))kv_write, METH_FASTCALL, nullptr},
    {"kv_read", (PyCFunction)(void (*)(void))kv_read, METH_FASTCALL, nullptr},
    {"kv_attention", (PyCFunction)(void (*)(void))kv_attention, METH_FASTCALL, nullptr},
    {"act_quant", (PyCFunction)(void (*)(void))act_quant, METH_FASTCALL, nullptr},
    {"act_quant_asym", (PyCFunction)(void (*)(void))act_quant_asym, METH_FASTCALL, nullptr},
    {"gemm", (PyCFunction)(void (*)(void))gemm, METH_FASTCALL, nullptr},
    {"gemm_asym", (PyCFunction)(void (*)(void))gemm_asym, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
