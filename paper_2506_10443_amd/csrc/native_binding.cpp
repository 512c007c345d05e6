// CPython side of the calls a serving loop makes for every token: argument checks, current stream, call into
// libmnnq.so.  The work of such a call on the GPU is 4 - 15 us, and the marshalling used to take as long: through
// ctypes (12 converted arguments, a Python frame per check, a call to size the packed buffer) a decode call cost the
// host about 9 us, four of them - one transformer block - 36 us.  Here it is a parse of the argument vector, reads of
// tensor fields and the launch itself.  Names, arguments, defaults, checks and errors are those of the functions in
// binding.py that this module provides; nothing is computed here and nothing is kept between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <exception>

#include "../../include/mnnq.h"

namespace {

constexpr int kGroup = 64;
constexpr int kMaxArgs = 16;

// Thrown with a Python error already set.
struct PyError {};

[[noreturn]] void fail(PyObject* type, const char* fmt, const char* what, long long a = 0, long long b = 0)
{
    PyErr_Format(type, fmt, what, a, b);
    throw PyError{};
}

// Parameter list of one function: names interned at import, the first `required` without a default.
struct Params {
    const char* function;
    int count, required;
    const char* names[kMaxArgs];
    PyObject* interned[kMaxArgs];
};

// Positional and keyword arguments -> v[0 .. count), nullptr where the default applies.
void parse(const Params& p, PyObject* const* args, Py_ssize_t n_pos, PyObject* kwnames, PyObject** v)
{
    for (int i = 0; i < p.count; ++i) v[i] = nullptr;
    if (n_pos > p.count) fail(PyExc_TypeError, "%s() takes %lld arguments (%lld given)", p.function, p.count, n_pos);
    for (Py_ssize_t i = 0; i < n_pos; ++i) v[i] = args[i];
    const Py_ssize_t n_kw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t k = 0; k < n_kw; ++k) {
        PyObject* name = PyTuple_GET_ITEM(kwnames, k);
        int at = 0;
        while (at < p.count && p.interned[at] != name) ++at;
        if (at == p.count)   // (a name built at run time is not interned)
            for (at = 0; at < p.count && PyUnicode_Compare(p.interned[at], name) != 0;) ++at;
        if (at == p.count) {
            PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", p.function, name);
            throw PyError{};
        }
        if (v[at]) {
            PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%U'", p.function, name);
            throw PyError{};
        }
        v[at] = args[n_pos + k];
    }
    for (int i = 0; i < p.required; ++i)
        if (!v[i]) {
            PyErr_Format(PyExc_TypeError, "%s() missing required argument: '%s'", p.function, p.names[i]);
            throw PyError{};
        }
}

int64_t integer(PyObject* o)
{
    long long v = PyLong_CheckExact(o) ? PyLong_AsLongLong(o) : -1;
    if (!PyLong_CheckExact(o)) {
        PyObject* i = PyNumber_Index(o);
        if (!i) throw PyError{};
        v = PyLong_AsLongLong(i);
        Py_DECREF(i);
    }
    if (v == -1 && PyErr_Occurred()) throw PyError{};
    return v;
}

int mode_of(PyObject* o, int def) { return o ? (int)integer(o) : def; }

bool given(PyObject* o) { return o && o != Py_None; }

const at::Tensor& tensor(PyObject* o, const char* what)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s must be a tensor", what);
    return THPVariable_Unpack(o);
}

const char* dtype_name(at::ScalarType t)
{
    switch (t) {
        case at::kByte: return "torch.uint8";
        case at::kChar: return "torch.int8";
        case at::kHalf: return "torch.float16";
        case at::kInt: return "torch.int32";
        default: return "torch.float32";
    }
}

// A contiguous tensor of the wanted type on the GPU.
const at::Tensor& on_gpu(PyObject* o, at::ScalarType type, const char* what)
{
    const at::Tensor& t = tensor(o, what);
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous()) {
        PyErr_Format(PyExc_TypeError, "%s must be a contiguous %s tensor on the GPU", what, dtype_name(type));
        throw PyError{};
    }
    return t;
}

// The C-ABI trusts the sizes it is told; a buffer smaller than the shape implies is refused here.
void need(const at::Tensor& t, int64_t n, const char* what)
{
    if (t.numel() < n) fail(PyExc_ValueError, "%s holds %lld elements, the shape needs %lld", what, t.numel(), n);
}

const void* optional_ptr(PyObject* o, int64_t n, const char* what)
{
    if (!given(o)) return nullptr;
    const at::Tensor& t = tensor(o, what);
    need(t, n, what);
    return t.data_ptr();
}

const at::Tensor& packed_arg(PyObject* o, int64_t N, int64_t K, int mode)
{
    const at::Tensor& t = on_gpu(o, at::kByte, "packed");
    const size_t size = mnnq_packed_size(N, K, kGroup, mode);
    if (size == 0) {
        PyErr_Format(PyExc_ValueError, "unsupported shape N=%lld K=%lld mode=%d", (long long)N, (long long)K, mode);
        throw PyError{};
    }
    need(t, (int64_t)size, "packed");
    return t;
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

[[noreturn]] void raise_status(int status, const char* what)
{
    PyObject* m = PyImport_ImportModule("paper_2506_10443_amd.binding");
    PyObject* cls = m ? PyObject_GetAttrString(m, "MnnqError") : nullptr;
    PyObject* e = cls ? PyObject_CallFunction(cls, "is", status, what) : nullptr;
    if (e) PyErr_SetObject(cls, e);
    Py_XDECREF(e);
    Py_XDECREF(cls);
    Py_XDECREF(m);
    throw PyError{};
}

// Runs a C-ABI call without the interpreter lock (a launch can wait for room in the stream's queue).
template <typename F>
void call(F&& f, const char* what)
{
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = f();
    Py_END_ALLOW_THREADS;
    if (status != 0) raise_status(status, what);
}

// The output: the caller's tensor (a new reference), or a new one of the given shape.
struct Output {
    PyObject* object = nullptr;
    void* ptr = nullptr;
    ~Output() { Py_XDECREF(object); }
    Output(PyObject* out, at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like, int64_t n, bool check_type)
    {
        if (given(out)) {
            const at::Tensor& t = tensor(out, "out");
            need(t, n, "out");
            if (check_type) on_gpu(out, type, "out");
            ptr = t.data_ptr();
            Py_INCREF(out);
            object = out;
        } else {
            at::Tensor t = at::empty(shape, like.options().dtype(type));
            ptr = t.data_ptr();
            object = THPVariable_Wrap(std::move(t));
            if (!object) throw PyError{};
        }
    }
    PyObject* release()
    {
        PyObject* o = object;
        object = nullptr;
        return o;
    }
};

struct Workspace {
    void* ptr = nullptr;
    size_t bytes = 0;
    at::Tensor own;
    const bool callers;
    explicit Workspace(PyObject* o) : callers(given(o))
    {
        if (!callers) return;
        const at::Tensor& t = on_gpu(o, at::kByte, "workspace");
        ptr = t.data_ptr();
        bytes = (size_t)t.numel();
    }
    void bring(const at::Tensor& like, int64_t M, int64_t N, int64_t K, int mode)
    {
        if (callers) return;     // (too small or empty: the call says so)
        const size_t n = mnnq_workspace_size(M, N, K, kGroup, mode);
        own = at::empty({(int64_t)(n < 16 ? 16 : n)}, like.options());
        ptr = own.data_ptr();
        bytes = (size_t)own.numel();
    }
};

// M of an [M, K] array; dimensions behind the second are not looked at ([M, K, 1] is one).
int64_t rows_of(const at::Tensor& t, int64_t K, const char* message)
{
    if (t.dim() < 2) fail(PyExc_IndexError, "%s", message);
    if (t.size(1) != K) fail(PyExc_ValueError, "%s", message);
    return t.size(0);
}

template <bool OUT16>
constexpr at::ScalarType out_type() { return OUT16 ? at::kHalf : at::kFloat; }

// ---- the calls

template <bool OUT16>
PyObject* decode(const Params& p, PyObject** v)   // packed, N, K, xq, sx, bias, out, mode
{
    const int64_t N = integer(v[1]), K = integer(v[2]);
    const int mode = mode_of(v[7], MNNQ_W4_ZP_INT);
    const at::Tensor& packed = packed_arg(v[0], N, K, mode);
    const at::Tensor& xq = on_gpu(v[3], at::kChar, "xq");
    const at::Tensor& sx = on_gpu(v[4], at::kFloat, "sx");
    if (xq.numel() != K) fail(PyExc_ValueError, "%s", "xq must hold K values");
    Output y(v[6], {N}, out_type<OUT16>(), packed, N, OUT16);
    const void* w = packed.data_ptr();
    const int8_t* q = static_cast<const int8_t*>(xq.data_ptr());
    const float* s = static_cast<const float*>(sx.data_ptr());
    const float* bias = static_cast<const float*>(optional_ptr(v[5], N, "bias"));
    void* st = stream();
    call([&] {
        return OUT16 ? mnnq_linear_decode_o16(w, N, K, kGroup, mode, q, s, bias, static_cast<uint16_t*>(y.ptr), st)
                     : mnnq_linear_decode(w, N, K, kGroup, mode, q, s, bias, static_cast<float*>(y.ptr), nullptr, 0, st);
    }, p.function);
    return y.release();
}

template <bool OUT16>
PyObject* decode_fused(const Params& p, PyObject** v)   // packed, N, K, x, bias, out, workspace, mode
{
    const int64_t N = integer(v[1]), K = integer(v[2]);
    const int mode = mode_of(v[7], MNNQ_W4_ZP_INT);
    const at::Tensor& packed = packed_arg(v[0], N, K, mode);
    const at::Tensor& x = on_gpu(v[3], at::kFloat, "x");
    if (x.numel() != K) fail(PyExc_ValueError, "%s", "x must hold K values");
    Output y(v[5], {N}, out_type<OUT16>(), packed, N, OUT16);
    const Workspace ws(v[6]);
    const void* w = packed.data_ptr();
    const float* xp = static_cast<const float*>(x.data_ptr());
    const float* bias = static_cast<const float*>(optional_ptr(v[4], N, "bias"));
    void* st = stream();
    call([&] {
        return OUT16 ? mnnq_linear_decode_fused_o16(w, N, K, kGroup, mode, xp, bias, static_cast<uint16_t*>(y.ptr), ws.ptr,
                                                    ws.bytes, st)
                     : mnnq_linear_decode_fused(w, N, K, kGroup, mode, xp, bias, static_cast<float*>(y.ptr), ws.ptr,
                                                ws.bytes, st);
    }, p.function);
    return y.release();
}

template <bool OUT16>
PyObject* prefill(const Params& p, PyObject** v)   // packed, N, K, xq, sx, bias, out, mode[, workspace]
{
    const int64_t N = integer(v[1]), K = integer(v[2]);
    const int mode = mode_of(v[7], MNNQ_W4_ZP_INT);
    const at::Tensor& packed = packed_arg(v[0], N, K, mode);
    const at::Tensor& xq = on_gpu(v[3], at::kChar, "xq");
    const at::Tensor& sx = on_gpu(v[4], at::kFloat, "sx");
    const int64_t M = rows_of(xq, K, "xq must be [M,K] and sx [M]");
    if (sx.numel() != M) fail(PyExc_ValueError, "%s", "xq must be [M,K] and sx [M]");
    const Workspace ws(OUT16 ? nullptr : v[8]);
    Output y(v[6], {M, N}, out_type<OUT16>(), packed, M * N, OUT16);
    const void* w = packed.data_ptr();
    const int8_t* q = static_cast<const int8_t*>(xq.data_ptr());
    const float* s = static_cast<const float*>(sx.data_ptr());
    const float* bias = static_cast<const float*>(optional_ptr(v[5], N, "bias"));
    void* st = stream();
    call([&] {
        return OUT16 ? mnnq_linear_prefill_o16(w, M, N, K, kGroup, mode, q, s, bias, static_cast<uint16_t*>(y.ptr), st)
                     : mnnq_linear_prefill(w, M, N, K, kGroup, mode, q, s, bias, static_cast<float*>(y.ptr), ws.ptr,
                                           ws.bytes, st);
    }, p.function);
    return y.release();
}

template <bool OUT16>
PyObject* prefill_fused(const Params& p, PyObject** v)   // packed, N, K, x, bias, out, workspace, mode
{
    const int64_t N = integer(v[1]), K = integer(v[2]);
    const int mode = mode_of(v[7], MNNQ_W4_ZP_INT);
    const at::Tensor& packed = packed_arg(v[0], N, K, mode);
    const at::Tensor& x = on_gpu(v[3], at::kFloat, "x");
    const int64_t M = rows_of(x, K, "x must be [M,K]");
    Workspace ws(v[6]);
    ws.bring(packed, M, N, K, mode);
    Output y(v[5], {M, N}, out_type<OUT16>(), packed, M * N, OUT16);
    const void* w = packed.data_ptr();
    const float* xp = static_cast<const float*>(x.data_ptr());
    const float* bias = static_cast<const float*>(optional_ptr(v[4], N, "bias"));
    void* st = stream();
    call([&] {
        return OUT16 ? mnnq_linear_prefill_fused_o16(w, M, N, K, kGroup, mode, xp, bias, static_cast<uint16_t*>(y.ptr),
                                                     ws.ptr, ws.bytes, st)
                     : mnnq_linear_prefill_fused(w, M, N, K, kGroup, mode, xp, bias, static_cast<float*>(y.ptr), ws.ptr,
                                                 ws.bytes, st);
    }, p.function);
    return y.release();
}

template <bool OUT16>
PyObject* decode_f16(const Params& p, PyObject** v)   // packed, N, K, x16, bias, out, mode
{
    const int64_t N = integer(v[1]), K = integer(v[2]);
    const int mode = mode_of(v[6], MNNQ_W4_ZP_INT);
    const at::Tensor& packed = packed_arg(v[0], N, K, mode);
    const at::Tensor& x = on_gpu(v[3], at::kHalf, "x16");
    if (x.numel() != K) fail(PyExc_ValueError, "%s", "x16 must hold K values");
    Output y(v[5], {N}, out_type<OUT16>(), packed, N, OUT16);
    const void* w = packed.data_ptr();
    const uint16_t* xp = static_cast<const uint16_t*>(x.data_ptr());
    const float* bias = static_cast<const float*>(optional_ptr(v[4], N, "bias"));
    void* st = stream();
    call([&] {
        return OUT16 ? mnnq_linear_decode_f16_o16(w, N, K, kGroup, mode, xp, bias, static_cast<uint16_t*>(y.ptr), st)
                     : mnnq_linear_decode_f16(w, N, K, kGroup, mode, xp, bias, static_cast<float*>(y.ptr), nullptr, 0, st);
    }, p.function);
    return y.release();
}

template <bool OUT16>
PyObject* prefill_f16(const Params& p, PyObject** v)   // packed, N, K, x16, bias, out, row_scale, mode
{
    const int64_t N = integer(v[1]), K = integer(v[2]);
    const int mode = mode_of(v[7], MNNQ_W4_ZP_INT);
    const at::Tensor& packed = packed_arg(v[0], N, K, mode);
    const at::Tensor& x = on_gpu(v[3], at::kHalf, "x16");
    const int64_t M = rows_of(x, K, "x16 must be [M,K]");
    Output y(v[5], {M, N}, out_type<OUT16>(), packed, M * N, OUT16);
    const void* w = packed.data_ptr();
    const uint16_t* xp = static_cast<const uint16_t*>(x.data_ptr());
    const float* bias = static_cast<const float*>(optional_ptr(v[4], N, "bias"));
    const float* rs = static_cast<const float*>(optional_ptr(v[6], 0, "row_scale"));
    void* st = stream();
    call([&] {
        return OUT16 ? mnnq_linear_prefill_f16_o16(w, M, N, K, kGroup, mode, xp, rs, bias, static_cast<uint16_t*>(y.ptr), st)
                     : mnnq_linear_prefill_f16(w, M, N, K, kGroup, mode, xp, rs, bias, static_cast<float*>(y.ptr), nullptr,
                                               0, st);
    }, p.function);
    return y.release();
}

PyObject* pack_weights(const Params& p, PyObject** v)   // W, out, mode
{
    const at::Tensor& W = on_gpu(v[0], at::kFloat, "W");
    if (W.dim() != 2) fail(PyExc_ValueError, "%s", "W must be [N, K]");
    const int64_t N = W.size(0), K = W.size(1);
    const int mode = mode_of(v[2], MNNQ_W4_ZP_INT);
    const float* wp = static_cast<const float*>(W.data_ptr());
    void* st = stream();
    const int64_t size = (int64_t)mnnq_packed_size(N, K, kGroup, mode);
    if (size == 0)   // the call says what is wrong with the shape (its checks run before it touches the buffer)
        call([&] { return mnnq_pack_weights(wp, N, K, kGroup, mode, const_cast<float*>(wp), 0, st); }, p.function);
    PyObject* out = v[1];
    if (given(out)) tensor(out, "out");
    // (the size of a caller's buffer is checked by the call itself: a status, not a ValueError)
    Output packed(out, {size}, at::kByte, W, 0, false);
    const size_t bytes = given(out) ? (size_t)THPVariable_Unpack(out).numel() : (size_t)size;
    call([&] { return mnnq_pack_weights(wp, N, K, kGroup, mode, packed.ptr, bytes, st); }, p.function);
    return packed.release();
}

// ---- attention: q, k, v and out are [tokens, heads, head_dim] views whose last dimension is dense

struct RowsArg {
    void* ptr;
    int64_t tokens, heads, dim, token, head;
};

RowsArg rows_arg(PyObject* o, const char* what, at::ScalarType* type)
{
    const at::Tensor& t = tensor(o, what);
    const at::ScalarType st = t.scalar_type();
    if (!t.is_cuda() || (st != at::kHalf && st != at::kBFloat16))
        fail(PyExc_TypeError, "%s must be a float16 or bfloat16 tensor on the GPU", what);
    if (t.dim() != 3) fail(PyExc_ValueError, "%s must be [tokens, heads, head_dim]", what);
    if (t.size(2) > 1 && t.stride(2) != 1) fail(PyExc_ValueError, "the last dimension of %s must be contiguous", what);
    if (*type == at::kFloat) *type = st;       // (the first array decides)
    if (*type != st) fail(PyExc_TypeError, "%s has another type than the first array", what);
    return {t.data_ptr(), t.size(0), t.size(1), t.size(2), t.stride(0), t.stride(1)};
}

int type_code(at::ScalarType t) { return t == at::kBFloat16 ? MNNQ_BF16 : MNNQ_F16; }

const int32_t* ints(PyObject* o, int64_t n, const char* what)
{
    const at::Tensor& t = on_gpu(o, at::kInt, what);
    need(t, n, what);
    return static_cast<const int32_t*>(t.data_ptr());
}

int form_of(const at::Tensor& t, const char* what)
{
    const at::ScalarType st = t.scalar_type();
    if (!t.is_cuda() || !t.is_contiguous() || (st != at::kChar && st != at::kFloat8_e4m3fn))
        fail(PyExc_TypeError, "%s must be a contiguous int8 or float8_e4m3fn tensor on the GPU", what);
    if (t.dim() != 4) fail(PyExc_ValueError, "%s must be [blocks, kv_heads, block_tokens, head_dim]", what);
    return st == at::kChar ? MNNQ_KV_INT8 : MNNQ_KV_FP8;
}

// k_codes, k_range, v_codes, v_range, block_table, lengths
mnnq_kv_cache cache_arg(PyObject** v)
{
    const at::Tensor& k = tensor(v[0], "k_codes");
    const at::Tensor& vv = tensor(v[2], "v_codes");
    mnnq_kv_cache c;
    c.k_form = form_of(k, "k_codes");
    c.v_form = form_of(vv, "v_codes");
    if (k.sizes() != vv.sizes()) fail(PyExc_ValueError, "%s", "k_codes and v_codes must have the same shape");
    const at::Tensor& kr = on_gpu(v[1], at::kFloat, "k_range");
    const at::Tensor& vr = on_gpu(v[3], at::kFloat, "v_range");
    need(kr, k.size(0) * k.size(1), "k_range");
    need(vr, k.size(0) * k.size(1), "v_range");
    const at::Tensor& table = on_gpu(v[4], at::kInt, "block_table");
    const at::Tensor& lengths = on_gpu(v[5], at::kInt, "lengths");
    if (table.dim() != 2) fail(PyExc_ValueError, "%s", "block_table must be [sequences, blocks]");
    need(lengths, table.size(0), "lengths");
    if (k.size(1) > INT32_MAX || k.size(2) > INT32_MAX || k.size(3) > INT32_MAX)
        fail(PyExc_ValueError, "%s", "k_codes: a dimension is too large");
    c.k_codes = k.data_ptr();
    c.v_codes = vv.data_ptr();
    c.k_range = static_cast<float*>(kr.data_ptr());
    c.v_range = static_cast<float*>(vr.data_ptr());
    c.block_table = static_cast<const int32_t*>(table.data_ptr());
    c.lengths = static_cast<const int32_t*>(lengths.data_ptr());
    c.blocks = k.size(0);
    c.sequences = table.size(0);
    c.table_blocks = table.size(1);
    c.kv_heads = (int32_t)k.size(1);
    c.block_tokens = (int32_t)k.size(2);
    c.head_dim = (int32_t)k.size(3);
    return c;
}

float scale_arg(PyObject* o, int64_t dim)
{
    if (!given(o)) return 1.0f / std::sqrt((float)dim);
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyError{};
    return (float)v;
}

// The output rows of an attention call: the caller's view, or a new dense array.
struct RowsOut {
    PyObject* object = nullptr;
    RowsArg rows;
    ~RowsOut() { Py_XDECREF(object); }
    RowsOut(PyObject* out, const RowsArg& q, at::ScalarType type, const at::Tensor& like)
    {
        if (given(out)) {
            at::ScalarType t = type;
            rows = rows_arg(out, "out", &t);
            if (rows.tokens != q.tokens || rows.heads != q.heads || rows.dim != q.dim)
                fail(PyExc_ValueError, "%s", "out must have the shape of q");
            Py_INCREF(out);
            object = out;
        } else {
            at::Tensor t = at::empty({q.tokens, q.heads, q.dim}, like.options());
            rows = {t.data_ptr(), q.tokens, q.heads, q.dim, q.heads * q.dim, q.dim};
            object = THPVariable_Wrap(std::move(t));
            if (!object) throw PyError{};
        }
    }
    PyObject* release()
    {
        PyObject* o = object;
        object = nullptr;
        return o;
    }
};

PyObject* attn_prefill(const Params& p, PyObject** v)   // q, k, v, q_start, k_start, scale, out
{
    at::ScalarType type = at::kFloat;
    const RowsArg q = rows_arg(v[0], "q", &type), k = rows_arg(v[1], "k", &type), vv = rows_arg(v[2], "v", &type);
    if (k.tokens != vv.tokens || k.heads != vv.heads || k.dim != vv.dim || k.dim != q.dim)
        fail(PyExc_ValueError, "%s", "k and v must have the same shape, and the head_dim of q");
    if (q.heads > INT32_MAX || k.heads > INT32_MAX || q.dim > INT32_MAX) fail(PyExc_ValueError, "%s", "q: a dimension is too large");
    const at::Tensor& starts = on_gpu(v[3], at::kInt, "q_start");
    const int64_t sequences = starts.numel() - 1;
    const int32_t* qs = static_cast<const int32_t*>(starts.data_ptr());
    const int32_t* ks = given(v[4]) ? ints(v[4], sequences + 1, "k_start") : qs;
    const float scale = scale_arg(v[5], q.dim);
    RowsOut out(v[6], q, type, tensor(v[0], "q"));
    const RowsArg& o = out.rows;
    void* st = stream();
    call([&] {
        return mnnq_attn_prefill(type_code(type), sequences, qs, ks, q.tokens, k.tokens, (int)q.heads, (int)k.heads, (int)q.dim,
                                 scale, q.ptr, q.token, q.head, k.ptr, k.token, k.head, vv.ptr, vv.token, vv.head, o.ptr,
                                 o.token, o.head, st);
    }, p.function);
    return out.release();
}

PyObject* kv_append(const Params& p, PyObject** v)   // k, v, k_codes, k_range, v_codes, v_range, block_table, lengths, start
{
    at::ScalarType type = at::kFloat;
    const RowsArg k = rows_arg(v[0], "k", &type), vv = rows_arg(v[1], "v", &type);
    const mnnq_kv_cache c = cache_arg(v + 2);
    if (k.tokens != vv.tokens || k.heads != vv.heads || k.dim != vv.dim || k.heads != c.kv_heads || k.dim != c.head_dim)
        fail(PyExc_ValueError, "%s", "k and v must be [tokens, kv_heads, head_dim] of the cache");
    const int32_t* start = given(v[8]) ? ints(v[8], c.sequences + 1, "start") : nullptr;
    void* st = stream();
    call([&] {
        return mnnq_kv_append(&c, type_code(type), start, k.tokens, k.ptr, k.token, k.head, vv.ptr, vv.token, vv.head, st);
    }, p.function);
    Py_RETURN_NONE;
}

// q, k_codes, k_range, v_codes, v_range, block_table, lengths, max_length, scale, out, weights, workspace
PyObject* attn_decode(const Params& p, PyObject** v)
{
    at::ScalarType type = at::kFloat;
    const RowsArg q = rows_arg(v[0], "q", &type);
    const mnnq_kv_cache c = cache_arg(v + 1);
    if (q.dim != c.head_dim) fail(PyExc_ValueError, "%s", "q must have the head_dim of the cache");
    if (c.sequences == 0 || q.tokens % c.sequences != 0 || q.heads > INT32_MAX)
        fail(PyExc_ValueError, "%s", "q must hold the same number of tokens for every sequence");
    const int64_t tokens = q.tokens / c.sequences, most = given(v[7]) ? integer(v[7]) : 0;
    const float scale = scale_arg(v[8], q.dim);
    const at::Tensor& like = tensor(v[0], "q");
    RowsOut out(v[9], q, type, like);
    float* weights = nullptr;
    int64_t stride = 0;
    if (given(v[10])) {
        const at::Tensor& w = on_gpu(v[10], at::kFloat, "weights");
        if (w.dim() != 3 || w.size(0) != c.sequences || w.size(1) != c.kv_heads)
            fail(PyExc_ValueError, "%s", "weights must be [sequences, kv_heads, tokens]");
        weights = static_cast<float*>(w.data_ptr());
        stride = w.size(2);
    }
    const size_t bytes = mnnq_attn_decode_workspace_size(&c, tokens, (int)q.heads, most, weights != nullptr);
    at::Tensor own;
    void* ws = nullptr;
    size_t ws_bytes = 0;
    if (given(v[11])) {
        const at::Tensor& t = on_gpu(v[11], at::kByte, "workspace");
        ws = t.data_ptr();
        ws_bytes = (size_t)t.numel();
    } else if (bytes > 0) {
        own = at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
        ws = own.data_ptr();
        ws_bytes = bytes;
    }
    const RowsArg& o = out.rows;
    void* st = stream();
    call([&] {
        return mnnq_attn_decode(&c, type_code(type), tokens, (int)q.heads, most, scale, q.ptr, q.token, q.head, o.ptr, o.token,
                                o.head, weights, stride, ws, ws_bytes, st);
    }, p.function);
    return out.release();
}

// k_codes, k_range, v_codes, v_range, block_table, lengths, weights, keep, recent, new_table, new_weights, kept, new_lengths
PyObject* kv_evict(const Params& p, PyObject** v)
{
    const mnnq_kv_cache c = cache_arg(v);
    const at::Tensor& w = on_gpu(v[6], at::kFloat, "weights");
    const at::Tensor& nw = on_gpu(v[10], at::kFloat, "new_weights");
    for (const at::Tensor* t : {&w, &nw})
        if (t->dim() != 3 || t->size(0) != c.sequences || t->size(1) != c.kv_heads)
            fail(PyExc_ValueError, "%s", "weights and new_weights must be [sequences, kv_heads, tokens]");
    const int64_t keep = integer(v[7]), recent = integer(v[8]);
    const at::Tensor& table = on_gpu(v[9], at::kInt, "new_table");
    if (table.dim() != 2 || table.size(0) != c.sequences) fail(PyExc_ValueError, "%s", "new_table must be [sequences, blocks]");
    const int64_t room = keep > 0 ? keep : 0;
    auto array = [&](PyObject* o, at::IntArrayRef shape, int64_t n, const char* what) {
        if (given(o)) {
            need(on_gpu(o, at::kInt, what), n, what);
            return THPVariable_Unpack(o);
        }
        return at::empty(shape, w.options().dtype(at::kInt));
    };
    at::Tensor kept = array(v[11], {c.sequences, c.kv_heads, room}, c.sequences * c.kv_heads * room, "kept");
    at::Tensor lengths = array(v[12], {c.sequences}, c.sequences, "new_lengths");
    int32_t dummy;      // (an empty array has no address; the call refuses keep = 0 before it looks at one)
    int32_t* kp = room > 0 ? static_cast<int32_t*>(kept.data_ptr()) : &dummy;
    void* st = stream();
    call([&] {
        return mnnq_kv_evict(&c, static_cast<const float*>(w.data_ptr()), w.size(2), keep, recent,
                             static_cast<const int32_t*>(table.data_ptr()), table.size(1), kp,
                             static_cast<int32_t*>(lengths.data_ptr()), static_cast<float*>(nw.data_ptr()), nw.size(2), st);
    }, p.function);
    PyObject* a = THPVariable_Wrap(std::move(kept));
    PyObject* b = a ? THPVariable_Wrap(std::move(lengths)) : nullptr;
    PyObject* both = b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    if (!both) throw PyError{};
    return both;
}

typedef PyObject* (*Body)(const Params&, PyObject**);

PyObject* run(Params& p, Body body, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames)
{
    PyObject* v[kMaxArgs];
    try {
        parse(p, args, nargs, kwnames, v);
        return body(p, v);
    } catch (const PyError&) {
    } catch (...) {     // torch's own errors as its Python calls raise them (OutOfMemoryError among them)
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

#define MNNQ_FUNCTION(NAME, BODY, REQUIRED, ...)                                                                        \
    Params params_##NAME{#NAME, (int)(sizeof((const char*[]){__VA_ARGS__}) / sizeof(char*)), REQUIRED, {__VA_ARGS__}, {}}; \
    PyObject* py_##NAME(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames)                          \
    {                                                                                                                   \
        return run(params_##NAME, BODY, args, nargs, kwnames);                                                          \
    }

MNNQ_FUNCTION(mnnq_linear_decode, decode<false>, 5, "packed", "N", "K", "xq", "sx", "bias", "out", "mode")
MNNQ_FUNCTION(mnnq_linear_decode_o16, decode<true>, 5, "packed", "N", "K", "xq", "sx", "bias", "out", "mode")
MNNQ_FUNCTION(mnnq_linear_decode_fused, decode_fused<false>, 4, "packed", "N", "K", "x", "bias", "out", "workspace", "mode")
MNNQ_FUNCTION(mnnq_linear_decode_fused_o16, decode_fused<true>, 4, "packed", "N", "K", "x", "bias", "out", "workspace",
              "mode")
MNNQ_FUNCTION(mnnq_linear_prefill, prefill<false>, 5, "packed", "N", "K", "xq", "sx", "bias", "out", "mode", "workspace")
MNNQ_FUNCTION(mnnq_linear_prefill_o16, prefill<true>, 5, "packed", "N", "K", "xq", "sx", "bias", "out", "mode")
MNNQ_FUNCTION(mnnq_linear_prefill_fused, prefill_fused<false>, 4, "packed", "N", "K", "x", "bias", "out", "workspace",
              "mode")
MNNQ_FUNCTION(mnnq_linear_prefill_fused_o16, prefill_fused<true>, 4, "packed", "N", "K", "x", "bias", "out", "workspace",
              "mode")
MNNQ_FUNCTION(mnnq_linear_decode_f16, decode_f16<false>, 4, "packed", "N", "K", "x16", "bias", "out", "mode")
MNNQ_FUNCTION(mnnq_linear_decode_f16_o16, decode_f16<true>, 4, "packed", "N", "K", "x16", "bias", "out", "mode")
MNNQ_FUNCTION(mnnq_linear_prefill_f16, prefill_f16<false>, 4, "packed", "N", "K", "x16", "bias", "out", "row_scale", "mode")
MNNQ_FUNCTION(mnnq_linear_prefill_f16_o16, prefill_f16<true>, 4, "packed", "N", "K", "x16", "bias", "out", "row_scale",
              "mode")
MNNQ_FUNCTION(mnnq_pack_weights, pack_weights, 1, "W", "out", "mode")
MNNQ_FUNCTION(mnnq_attn_prefill, attn_prefill, 4, "q", "k", "v", "q_start", "k_start", "scale", "out")
MNNQ_FUNCTION(mnnq_kv_append, kv_append, 8, "k", "v", "k_codes", "k_range", "v_codes", "v_range", "block_table", "lengths",
              "start")
MNNQ_FUNCTION(mnnq_attn_decode, attn_decode, 7, "q", "k_codes", "k_range", "v_codes", "v_range", "block_table", "lengths",
              "max_length", "scale", "out", "weights", "workspace")
MNNQ_FUNCTION(mnnq_kv_evict, kv_evict, 11, "k_codes", "k_range", "v_codes", "v_range", "block_table", "lengths", "weights",
              "keep", "recent", "new_table", "new_weights", "kept", "new_lengths")

#define MNNQ_METHOD(NAME, SIGNATURE, DOC)                                                                  \
    {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(py_##NAME)),                    \
     METH_FASTCALL | METH_KEYWORDS, #NAME "(" SIGNATURE ")\n--\n\n" DOC}

PyMethodDef methods[] = {
    MNNQ_METHOD(mnnq_linear_decode, "packed, N, K, xq, sx, bias=None, out=None, mode=0",
                "One token: xq i8 [K] (or [1,K]), sx f32 [1] -> y f32 [N]."),
    MNNQ_METHOD(mnnq_linear_decode_o16, "packed, N, K, xq, sx, bias=None, out=None, mode=0",
                "One token: xq i8 [K], sx f32 [1] -> y fp16 [N]."),
    MNNQ_METHOD(mnnq_linear_decode_fused, "packed, N, K, x, bias=None, out=None, workspace=None, mode=0",
                "One token, activation quantizer fused in: x f32 [K] (or [1,K]) -> y f32 [N].\n"
                "workspace: optional uint8 tensor of mnnq_workspace_size(1, N, K) bytes."),
    MNNQ_METHOD(mnnq_linear_decode_fused_o16, "packed, N, K, x, bias=None, out=None, workspace=None, mode=0",
                "One token, activation quantizer fused in: x f32 [K] -> y fp16 [N]."),
    MNNQ_METHOD(mnnq_linear_prefill, "packed, N, K, xq, sx, bias=None, out=None, mode=0, workspace=None",
                "M tokens: xq i8 [M,K], sx f32 [M] -> y f32 [M,N].  workspace: optional uint8 tensor\n"
                "(mnnq_workspace_size bytes); with the matrix-core plane in `packed` it selects the fp6 GEMM."),
    MNNQ_METHOD(mnnq_linear_prefill_o16, "packed, N, K, xq, sx, bias=None, out=None, mode=0",
                "M tokens: xq i8 [M,K], sx f32 [M] -> y fp16 [M,N]."),
    MNNQ_METHOD(mnnq_linear_prefill_fused, "packed, N, K, x, bias=None, out=None, workspace=None, mode=0",
                "M tokens, activation quantizer inside the call: x f32 [M,K] -> y f32 [M,N].\n"
                "workspace: uint8 tensor of at least mnnq_workspace_size(M, N, K) bytes (required by the library;\n"
                "this wrapper brings one along when none is given)."),
    MNNQ_METHOD(mnnq_linear_prefill_fused_o16, "packed, N, K, x, bias=None, out=None, workspace=None, mode=0",
                "M tokens, activation quantizer inside the call: x f32 [M,K] -> y fp16 [M,N]."),
    MNNQ_METHOD(mnnq_linear_decode_f16, "packed, N, K, x16, bias=None, out=None, mode=0",
                "One token, fp16 activations (W4A16; W8A16 with MODE_W8_MIN_FLOAT): x16 fp16 [K] -> y f32 [N]."),
    MNNQ_METHOD(mnnq_linear_decode_f16_o16, "packed, N, K, x16, bias=None, out=None, mode=0",
                "One token, fp16 activations: x16 fp16 [K] -> y fp16 [N]."),
    MNNQ_METHOD(mnnq_linear_prefill_f16, "packed, N, K, x16, bias=None, out=None, row_scale=None, mode=0",
                "M tokens, fp16 activations (W4A16; W8A16 with MODE_W8_MIN_FLOAT): x16 fp16 [M,K] -> y f32 [M,N];\n"
                "row_scale f32 [M] optional."),
    MNNQ_METHOD(mnnq_linear_prefill_f16_o16, "packed, N, K, x16, bias=None, out=None, row_scale=None, mode=0",
                "M tokens, fp16 activations: x16 fp16 [M,K] -> y fp16 [M,N]; row_scale f32 [M] optional."),
    MNNQ_METHOD(mnnq_pack_weights, "W, out=None, mode=0", "W fp32 [N, K] on the GPU -> packed uint8 buffer."),
    MNNQ_METHOD(mnnq_attn_prefill, "q, k, v, q_start, k_start=None, scale=None, out=None",
                "Causal attention over packed prompts: q [tokens, heads, head_dim], k and v [tokens, kv_heads, head_dim]\n"
                "(fp16 or bf16, views with a dense last dimension), q_start and k_start int32 [sequences + 1] (k_start: as\n"
                "q_start where None), scale 1 / sqrt(head_dim) where None -> [tokens, heads, head_dim]."),
    MNNQ_METHOD(mnnq_kv_append, "k, v, k_codes, k_range, v_codes, v_range, block_table, lengths, start=None",
                "Quantizes rows k and v [tokens, kv_heads, head_dim] into the cache behind its first `lengths` tokens: codes int8\n"
                "or float8_e4m3fn [blocks, kv_heads, block_tokens, head_dim], ranges f32 [blocks, kv_heads], block_table int32\n"
                "[sequences, blocks], lengths int32 [sequences] (not changed); start int32 [sequences + 1], or None: the same\n"
                "number of rows for every sequence."),
    MNNQ_METHOD(mnnq_attn_decode,
                "q, k_codes, k_range, v_codes, v_range, block_table, lengths, max_length=None, scale=None, out=None, "
                "weights=None, workspace=None",
                "Attention of q [sequences * tokens, heads, head_dim], the queries of every sequence's last tokens, over the\n"
                "cache.  max_length: bound of the lengths (the table's room where None); weights f32 [sequences, kv_heads,\n"
                "tokens]: the attention that each cached token was given is added; workspace: uint8 tensor of\n"
                "mnnq_attn_decode_workspace_size bytes (brought along where None)."),
    MNNQ_METHOD(mnnq_kv_evict,
                "k_codes, k_range, v_codes, v_range, block_table, lengths, weights, keep, recent, new_table, new_weights, "
                "kept=None, new_lengths=None",
                "Moves of every sequence and head the last `recent` tokens and those with the greatest weights, `keep` in all,\n"
                "to the blocks of new_table; their weights to new_weights, zeros behind -> (kept int32 [sequences, kv_heads,\n"
                "keep], new_lengths int32 [sequences])."),
    {nullptr, nullptr, 0, nullptr}};

Params* const all_params[] = {
    &params_mnnq_linear_decode, &params_mnnq_linear_decode_o16, &params_mnnq_linear_decode_fused,
    &params_mnnq_linear_decode_fused_o16, &params_mnnq_linear_prefill, &params_mnnq_linear_prefill_o16,
    &params_mnnq_linear_prefill_fused, &params_mnnq_linear_prefill_fused_o16, &params_mnnq_linear_decode_f16,
    &params_mnnq_linear_decode_f16_o16, &params_mnnq_linear_prefill_f16, &params_mnnq_linear_prefill_f16_o16,
    &params_mnnq_pack_weights, &params_mnnq_attn_prefill, &params_mnnq_kv_append, &params_mnnq_attn_decode,
    &params_mnnq_kv_evict};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native",
                      "The per-token calls of libmnnq.so as CPython functions; see binding.py.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void)
{
    for (Params* p : all_params)
        for (int i = 0; i < p->count; ++i)
            if (!(p->interned[i] = PyUnicode_InternFromString(p->names[i]))) return nullptr;
    return PyModule_Create(&module);
}
