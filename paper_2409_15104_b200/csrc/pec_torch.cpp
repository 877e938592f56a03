// Marshalling of the paged serving calls from torch tensors: checks that the C ABI cannot make (type, device, shape, innermost
// stride), output and workspace tensors, the current stream; the library does everything else.  binding.py wraps these functions
// with names, defaults and documentation.
//
// Why compiled: one of these calls is 3 to 15 us of device work in a decode step, and the same marshalling in Python and ctypes
// took 12 (append) to 22 us (attention) of the host.
#include <Python.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>
#include <cstdarg>
#include <string>
#include "pec.h"

namespace {

int (*g_norm_rope)(const pec_norm_rope_args *, void *) = nullptr;
int (*g_append)(const pec_kv_append_args *, void *) = nullptr;
int (*g_attn)(const pec_paged_args *, void *) = nullptr;
size_t (*g_workspace)(const pec_paged_args *) = nullptr;
int (*g_append_q4)(const pec_kv_append_q4_args *, void *) = nullptr;
int (*g_read_q4)(const pec_kv_read_q4_args *, void *) = nullptr;
int (*g_attn_q4)(const pec_paged_q4_args *, void *) = nullptr;
size_t (*g_workspace_q4)(const pec_paged_q4_args *) = nullptr;

using at::Tensor;

// Sets the Python error and leaves through the functions' common exit.
[[noreturn]] void fail(PyObject *type, const char *format, ...)
{
    va_list ap;
    va_start(ap, format);
    PyErr_FormatV(type, format, ap);
    va_end(ap);
    throw python_error();
}
[[noreturn]] void refuse(const char *what, const char *need) { fail(PyExc_ValueError, "%s: need %s", what, need); }

const Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s: need a tensor", what);
    return THPVariable_Unpack(o);
}
int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}
int32_t type_code(at::ScalarType t)
{
    if (t == at::kBFloat16) return PEC_BF16;
    if (t == at::kFloat) return PEC_F32;
    fail(PyExc_TypeError, "unsupported dtype %s", c10::toString(t));
}

// What every tensor of a call has to share.
struct Like { at::ScalarType type; at::Device device; };
Like first(const Tensor &t)
{
    type_code(t.scalar_type());
    if (!t.is_cuda()) refuse("the call's tensors", "a CUDA device");
    return {t.scalar_type(), t.device()};
}
void same(const Tensor &t, const char *what, const Like &l, at::ScalarType type, int dims)
{
    if (t.scalar_type() != type || t.device() != l.device || t.dim() != dims || (t.stride(-1) != 1 && t.size(-1) > 1))
        fail(PyExc_ValueError, "%s: need a %d-dimensional %s tensor on %s with a contiguous innermost dimension", what, dims, c10::toString(type),
                                l.device.str().c_str());
}
// These dimensions go through the C ABI in 32 bits.
int32_t narrow(int64_t size, const char *what)
{
    if (size > INT32_MAX) refuse(what, "dimensions below 2^31");
    return (int32_t)size;
}
// A dimension of one entry has no stride of its own, whatever torch says.
int64_t stride(const Tensor &t, int i) { return t.size(i) > 1 ? t.stride(i) : 128; }

const void *vector(PyObject *o, const char *what, const Like &l, at::ScalarType type, int64_t n)
{
    const Tensor &t = tensor(o, what);
    same(t, what, l, type, 1);
    if (!t.is_contiguous() || (n >= 0 && t.size(0) != n)) fail(PyExc_ValueError, "%s: need a contiguous vector of %lld entries", what, (long long)n);
    return t.data_ptr();
}
const void *weight(PyObject *o, bool norm, const Like &l)
{
    if (o == Py_None) return nullptr;
    if (!norm) refuse("weight", "norm=True");
    return vector(o, "weight", l, l.type, 128);
}
const float *rope_table(PyObject *o, int64_t n_pos, const Like &l)
{
    if (o == Py_None) return nullptr;
    const float *at = static_cast<const float *>(vector(o, "tables", l, at::kFloat, -1));
    if (n_pos < 0 || THPVariable_Unpack(o).size(0) < 8192 + (n_pos + 63) / 64 * 128) refuse("tables", "a table as long as n_pos asks for");
    return at;
}
int32_t *status_word(PyObject *o, const Like &l)
{
    const Tensor &t = tensor(o, "status");
    same(t, "status", l, at::kInt, 1);
    return static_cast<int32_t *>(t.data_ptr());
}

// Batch fields, the same in all argument structures: block_table, cu_q, kv_lens.
template <class A>
void batch(A &a, PyObject *const *o, int64_t T, const Like &l)
{
    const Tensor &table = tensor(o[0], "block_table"), &cu = tensor(o[1], "cu_q"), &lens = tensor(o[2], "kv_lens");
    same(table, "block_table", l, at::kInt, 2);
    same(cu, "cu_q", l, at::kInt, 1);
    same(lens, "kv_lens", l, at::kInt, 1);
    const int64_t B = lens.size(0);
    if (cu.size(0) != B + 1 || table.size(0) != B) fail(PyExc_ValueError, "need cu_q [B + 1], kv_lens [B] and block_table [B, pages]");
    if (!cu.is_contiguous() || !lens.is_contiguous()) fail(PyExc_ValueError, "need contiguous cu_q and kv_lens");
    a.block_table = static_cast<const int32_t *>(table.data_ptr());
    a.max_pages = narrow(table.size(1), "block_table");
    a.table_stride = B > 1 ? table.stride(0) : table.size(1);
    a.cu_q = static_cast<const int32_t *>(cu.data_ptr());
    a.kv_lens = static_cast<const int32_t *>(lens.data_ptr());
    a.B = narrow(B, "kv_lens"); a.T = T;
}

// Cache and batch: k_pages, v_pages, block_table, cu_q, kv_lens.
template <class A>
void paged(A &a, PyObject *const *o, int64_t T, const Like &l)
{
    const Tensor &k = tensor(o[0], "k_pages"), &v = tensor(o[1], "v_pages");
    same(k, "k_pages", l, l.type, 4);
    same(v, "v_pages", l, l.type, 4);
    if (v.sizes() != k.sizes()) refuse("v_pages", "k_pages' shape");
    batch(a, o + 2, T, l);
    a.k_pages = k.data_ptr(); a.v_pages = v.data_ptr();
    a.k_pages_stride_p = stride(k, 0); a.k_pages_stride_t = stride(k, 1); a.k_pages_stride_h = stride(k, 2);
    a.v_pages_stride_p = stride(v, 0); a.v_pages_stride_t = stride(v, 1); a.v_pages_stride_h = stride(v, 2);
    a.num_pages = k.size(0); a.page_size = narrow(k.size(1), "k_pages"); a.Hkv = narrow(k.size(2), "k_pages"); a.D = narrow(k.size(3), "k_pages");
}

// The same of a cache held in 4 bits: k_pages, k_scales, v_pages, v_scales, block_table, cu_q, kv_lens.
void paged_q4(pec_q4_cache &a, PyObject *const *o, int64_t T, const Like &l)
{
    const Tensor &k = tensor(o[0], "k_pages"), &ks = tensor(o[1], "k_scales"), &v = tensor(o[2], "v_pages"), &vs = tensor(o[3], "v_scales");
    for (const Tensor *t : {&k, &v}) {
        if (t->scalar_type() != at::kByte && t->scalar_type() != at::kFloat4_e2m1fn_x2) fail(PyExc_TypeError, "k_pages, v_pages: need bytes, or pairs of 4-bit floats");
        same(*t, t == &k ? "k_pages" : "v_pages", l, t->scalar_type(), 4);
    }
    for (const Tensor *t : {&ks, &vs})
        if (t->scalar_type() != at::kBFloat16 || t->device() != l.device || t->dim() != 3 || t->sizes() != k.sizes().slice(0, 3))
            refuse(t == &ks ? "k_scales" : "v_scales", "a bf16 tensor of the pages' first three dimensions on their device");
    if (v.sizes() != k.sizes()) refuse("v_pages", "k_pages' shape");
    batch(a, o + 4, T, l);
    a.k_pages = k.data_ptr(); a.v_pages = v.data_ptr(); a.k_scales = ks.data_ptr(); a.v_scales = vs.data_ptr();
    a.k_pages_stride_p = stride(k, 0); a.k_pages_stride_t = stride(k, 1); a.k_pages_stride_h = stride(k, 2);
    a.v_pages_stride_p = stride(v, 0); a.v_pages_stride_t = stride(v, 1); a.v_pages_stride_h = stride(v, 2);
    a.k_scales_stride_p = stride(ks, 0); a.k_scales_stride_t = stride(ks, 1); a.k_scales_stride_h = stride(ks, 2);
    a.v_scales_stride_p = stride(vs, 0); a.v_scales_stride_t = stride(vs, 1); a.v_scales_stride_h = stride(vs, 2);
    a.num_pages = k.size(0); a.page_size = narrow(k.size(1), "k_pages"); a.Hkv = narrow(k.size(2), "k_pages");
    a.D = narrow(2 * k.size(3), "k_pages");
}

// (straight from the CUDA allocator, 0.3 us a tensor less than through the dispatcher)
Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Like &l) { return at::detail::empty_cuda(shape, type, l.device, std::nullopt); }
PyObject *keep(PyObject *o) { Py_INCREF(o); return o; }
void arguments(Py_ssize_t got, Py_ssize_t want)
{
    if (got != want) fail(PyExc_TypeError, "need %zd arguments, got %zd", want, got);
}
// The answer (rc, tensors ...); takes over the references.
PyObject *answer(int rc, PyObject *a, PyObject *b)
{
    PyObject *t = a && b ? Py_BuildValue("iNN", rc, a, b) : nullptr;
    if (!t) { Py_XDECREF(a); Py_XDECREF(b); }
    return t;
}

// q, k | None, q_out | None, k_out | None, inplace, norm, q_weight, k_weight, eps, table, n_pos, positions, pos0, status -> (rc, q_out, k_out)
PyObject *norm_rope(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 14);
    const Tensor &q = tensor(o[0], "q");
    const Like l = first(q);
    same(q, "q", l, l.type, 3);
    const c10::cuda::CUDAGuard guard(l.device);
    const bool inplace = truth(o[4]), norm = truth(o[5]), has_k = o[1] != Py_None;
    pec_norm_rope_args a{};
    a.dtype = type_code(l.type);
    a.T = q.size(0); a.Hq = narrow(q.size(1), "q"); a.D = narrow(q.size(2), "q");
    a.q = q.data_ptr(); a.q_stride_t = stride(q, 0); a.q_stride_h = stride(q, 1);
    // The output of one side: the tensor given, the input itself, or a new one.
    auto out = [&](PyObject *given, PyObject *input, const char *what) -> PyObject * {
        const Tensor &in = THPVariable_Unpack(input);
        if (given != Py_None) {
            const Tensor &t = tensor(given, what);
            same(t, what, l, l.type, 3);
            if (t.sizes() != in.sizes()) refuse(what, "the input's shape");
            return keep(given);
        }
        return inplace ? keep(input) : THPVariable_Wrap(empty(in.sizes(), l.type, l));
    };
    if (has_k) {
        const Tensor &k = tensor(o[1], "k");
        same(k, "k", l, l.type, 3);
        if (k.size(0) != a.T || k.size(2) != q.size(2)) refuse("k", "q's tokens and head dimension");
        a.Hkv = narrow(k.size(1), "k");
        a.k = k.data_ptr(); a.k_stride_t = stride(k, 0); a.k_stride_h = stride(k, 1);
    }
    a.norm = norm; a.eps = real(o[8]);
    a.q_weight = weight(o[6], norm, l); a.k_weight = weight(o[7], norm, l);
    a.n_pos = integer(o[10]);
    a.rope_table = rope_table(o[9], a.n_pos, l);
    if (o[11] != Py_None) a.positions = static_cast<const int32_t *>(vector(o[11], "positions", l, at::kInt, a.T));
    a.pos0 = integer(o[12]);
    a.status = status_word(o[13], l);
    THPObjectPtr qo(out(o[2], o[0], "q_out")), ko(has_k ? out(o[3], o[1], "k_out") : keep(Py_None));
    if (!qo || !ko) throw python_error();
    int rc = PEC_OK;
    if (a.T > 0 && a.Hq + a.Hkv > 0) {                          // tensors without elements have no address
        const Tensor &t = THPVariable_Unpack(qo.get());
        a.q_out = t.data_ptr(); a.q_out_stride_t = stride(t, 0); a.q_out_stride_h = stride(t, 1);
        if (has_k) {
            const Tensor &u = THPVariable_Unpack(ko.get());
            a.k_out = u.data_ptr(); a.k_out_stride_t = stride(u, 0); a.k_out_stride_h = stride(u, 1);
        }
        rc = g_norm_rope(&a, c10::cuda::getCurrentCUDAStream(l.device.index()).stream());
    }
    return answer(rc, qo.release(), ko.release());
    END_HANDLE_TH_ERRORS
}

// k, v, k_pages, v_pages, block_table, cu_q, kv_lens, norm, k_weight, eps, table, n_pos, status -> rc
PyObject *kv_append(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 13);
    const Tensor &k = tensor(o[0], "k"), &v = tensor(o[1], "v");
    const Like l = first(k);
    same(k, "k", l, l.type, 3);
    same(v, "v", l, l.type, 3);
    if (v.sizes() != k.sizes()) refuse("v", "k's shape");
    const c10::cuda::CUDAGuard guard(l.device);
    pec_kv_append_args a{};
    paged(a, o + 2, k.size(0), l);
    if (a.Hkv != k.size(1) || a.D != k.size(2)) refuse("k_pages", "k's heads and head dimension");
    a.dtype = type_code(l.type);
    a.k = k.data_ptr(); a.v = v.data_ptr();
    a.k_stride_t = stride(k, 0); a.k_stride_h = stride(k, 1); a.v_stride_t = stride(v, 0); a.v_stride_h = stride(v, 1);
    a.norm = truth(o[7]);
    a.k_weight = weight(o[8], a.norm != 0, l);
    a.eps = real(o[9]);
    a.n_pos = integer(o[11]);
    a.rope_table = rope_table(o[10], a.n_pos, l);
    a.status = status_word(o[12], l);
    return PyLong_FromLong(a.T > 0 ? g_append(&a, c10::cuda::getCurrentCUDAStream(l.device.index()).stream()) : PEC_OK);
    END_HANDLE_TH_ERRORS
}

// The rest of an attention call from `o` on: max_q_len, causal, scale, out_dtype, o, lse, workspace, status -> (rc, o, lse)
template <class A>
PyObject *attend(A &a, const Tensor &q, int64_t D, PyObject *const *o, const Like &l, size_t (*workspace)(const A *), int (*call)(const A *, void *))
{
    if (D != q.size(2)) refuse("k_pages", "q's head dimension");
    a.dtype = type_code(l.type);
    a.q = q.data_ptr(); a.q_stride_t = stride(q, 0); a.q_stride_h = stride(q, 1);
    a.Hq = narrow(q.size(1), "q");
    const int64_t most = integer(o[0]);
    if (most < 0 || most > INT32_MAX) refuse("max_q_len", "0 <= max_q_len < 2^31");
    a.max_q_len = (int32_t)most;
    a.causal = truth(o[1]); a.softmax_scale = real(o[2]);
    at::ScalarType type = l.type;
    if (o[3] != Py_None) {
        if (!THPDtype_Check(o[3])) fail(PyExc_TypeError, "out_dtype: need a dtype");
        type = reinterpret_cast<THPDtype *>(o[3])->scalar_type;
    }
    THPObjectPtr out, lse;
    if (o[4] != Py_None) {
        const Tensor &t = tensor(o[4], "o");
        if (t.device() != l.device || !t.is_contiguous() || t.sizes() != q.sizes() || (o[3] != Py_None && t.scalar_type() != type))
            refuse("o", "a contiguous tensor of q's shape (and of out_dtype) on its device");
        type = t.scalar_type();
        out = THPObjectPtr(keep(o[4]));
    }
    a.o_dtype = type_code(type);
    if (!out) out = THPObjectPtr(THPVariable_Wrap(empty(q.sizes(), type, l)));
    if (o[5] != Py_None) {
        const Tensor &t = tensor(o[5], "lse");
        if (t.device() != l.device || !t.is_contiguous() || t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != q.size(0) || t.size(1) != q.size(1))
            refuse("lse", "a contiguous fp32 tensor [T, Hq] on q's device");
        lse = THPObjectPtr(keep(o[5]));
    } else {
        lse = THPObjectPtr(THPVariable_Wrap(empty({q.size(0), q.size(1)}, at::kFloat, l)));
    }
    if (!out || !lse) throw python_error();
    a.status = status_word(o[7], l);
    int rc = PEC_OK;
    if (q.size(0) > 0 && a.Hq > 0) {                            // tensors without elements have no address
        a.o = THPVariable_Unpack(out.get()).data_ptr();
        a.lse = static_cast<float *>(THPVariable_Unpack(lse.get()).data_ptr());
        Tensor scratch;                                         // its memory goes back to this stream's pool
        if (o[6] != Py_None) {
            const Tensor &t = tensor(o[6], "workspace");
            if (t.device() != l.device || !t.is_contiguous()) refuse("workspace", "a contiguous tensor on q's device");
            a.workspace = t.data_ptr(); a.workspace_bytes = t.nbytes();
        } else if (const size_t bytes = workspace(&a)) {
            scratch = empty({(int64_t)bytes}, at::kByte, l);
            a.workspace = scratch.data_ptr(); a.workspace_bytes = bytes;
        }
        rc = call(&a, c10::cuda::getCurrentCUDAStream(l.device.index()).stream());
    }
    return answer(rc, out.release(), lse.release());
}

// q, k_pages, v_pages, block_table, cu_q, kv_lens, then as above
PyObject *paged_attn(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 14);
    const Tensor &q = tensor(o[0], "q");
    const Like l = first(q);
    same(q, "q", l, l.type, 3);
    const c10::cuda::CUDAGuard guard(l.device);
    pec_paged_args a{};
    paged(a, o + 1, q.size(0), l);
    return attend(a, q, a.D, o + 6, l, g_workspace, g_attn);
    END_HANDLE_TH_ERRORS
}

// q, k_pages, k_scales, v_pages, v_scales, block_table, cu_q, kv_lens, then as above
PyObject *paged_attn_q4(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 16);
    const Tensor &q = tensor(o[0], "q");
    const Like l = first(q);
    same(q, "q", l, l.type, 3);
    const c10::cuda::CUDAGuard guard(l.device);
    pec_paged_q4_args a{};
    paged_q4(a.cache, o + 1, q.size(0), l);
    return attend(a, q, a.cache.D, o + 8, l, g_workspace_q4, g_attn_q4);
    END_HANDLE_TH_ERRORS
}

// k, v, k_pages, k_scales, v_pages, v_scales, block_table, cu_q, kv_lens, norm, k_weight, eps, table, n_pos, status -> rc
PyObject *kv_append_q4(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 15);
    const Tensor &k = tensor(o[0], "k"), &v = tensor(o[1], "v");
    const Like l = first(k);
    same(k, "k", l, l.type, 3);
    same(v, "v", l, l.type, 3);
    if (v.sizes() != k.sizes()) refuse("v", "k's shape");
    const c10::cuda::CUDAGuard guard(l.device);
    pec_kv_append_q4_args a{};
    paged_q4(a.cache, o + 2, k.size(0), l);
    if (a.cache.Hkv != k.size(1) || a.cache.D != k.size(2)) refuse("k_pages", "k's heads and head dimension");
    a.dtype = type_code(l.type);
    a.k = k.data_ptr(); a.v = v.data_ptr();
    a.k_stride_t = stride(k, 0); a.k_stride_h = stride(k, 1); a.v_stride_t = stride(v, 0); a.v_stride_h = stride(v, 1);
    a.norm = truth(o[9]);
    a.k_weight = weight(o[10], a.norm != 0, l);
    a.eps = real(o[11]);
    a.n_pos = integer(o[13]);
    a.rope_table = rope_table(o[12], a.n_pos, l);
    a.status = status_word(o[14], l);
    return PyLong_FromLong(a.cache.T > 0 ? g_append_q4(&a, c10::cuda::getCurrentCUDAStream(l.device.index()).stream()) : PEC_OK);
    END_HANDLE_TH_ERRORS
}

// k_pages, k_scales, v_pages, v_scales, block_table, cu_q, kv_lens, tokens, dtype, k_out | None, v_out | None, status -> (rc, k_out, v_out)
PyObject *kv_read_q4(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 12);
    const Tensor &pages = tensor(o[0], "k_pages");
    if (!THPDtype_Check(o[8])) fail(PyExc_TypeError, "dtype: need a dtype");
    const Like l = {reinterpret_cast<THPDtype *>(o[8])->scalar_type, pages.device()};
    if (!pages.is_cuda()) refuse("the call's tensors", "a CUDA device");
    const c10::cuda::CUDAGuard guard(l.device);
    pec_kv_read_q4_args a{};
    const int64_t T = integer(o[7]);
    if (T < 0) refuse("tokens", "tokens >= 0");
    paged_q4(a.cache, o, T, l);
    a.dtype = type_code(l.type);
    const int64_t shape[3] = {T, a.cache.Hkv, a.cache.D};
    auto out = [&](PyObject *given, const char *what) -> PyObject * {
        if (given == Py_None) return THPVariable_Wrap(empty(shape, l.type, l));
        const Tensor &t = tensor(given, what);
        same(t, what, l, l.type, 3);
        if (t.sizes() != at::IntArrayRef(shape)) refuse(what, "tokens, the cache's heads and its head dimension");
        return keep(given);
    };
    THPObjectPtr k(out(o[9], "k_out")), v(out(o[10], "v_out"));
    if (!k || !v) throw python_error();
    a.status = status_word(o[11], l);
    int rc = PEC_OK;
    if (T > 0 && a.cache.Hkv > 0) {                             // tensors without elements have no address
        const Tensor &x = THPVariable_Unpack(k.get()), &y = THPVariable_Unpack(v.get());
        a.k_out = x.data_ptr(); a.k_out_stride_t = stride(x, 0); a.k_out_stride_h = stride(x, 1);
        a.v_out = y.data_ptr(); a.v_out_stride_t = stride(y, 0); a.v_out_stride_h = stride(y, 1);
        rc = g_read_q4(&a, c10::cuda::getCurrentCUDAStream(l.device.index()).stream());
    }
    return answer(rc, k.release(), v.release());
    END_HANDLE_TH_ERRORS
}

// Addresses of the library's entry points.
PyObject *bind(PyObject *, PyObject *const *o, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 8);
    g_norm_rope = reinterpret_cast<decltype(g_norm_rope)>(integer(o[0]));
    g_append = reinterpret_cast<decltype(g_append)>(integer(o[1]));
    g_attn = reinterpret_cast<decltype(g_attn)>(integer(o[2]));
    g_workspace = reinterpret_cast<decltype(g_workspace)>(integer(o[3]));
    g_append_q4 = reinterpret_cast<decltype(g_append_q4)>(integer(o[4]));
    g_read_q4 = reinterpret_cast<decltype(g_read_q4)>(integer(o[5]));
    g_attn_q4 = reinterpret_cast<decltype(g_attn_q4)>(integer(o[6]));
    g_workspace_q4 = reinterpret_cast<decltype(g_workspace_q4)>(integer(o[7]));
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

PyMethodDef g_methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"norm_rope", (PyCFunction)(void (*)(void))norm_rope, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, nullptr},
    {"paged_attn", (PyCFunction)(void (*)(void))paged_attn, METH_FASTCALL, nullptr},
    {"kv_append_q4", (PyCFunction)(void (*)(void))kv_append_q4, METH_FASTCALL, nullptr},
    {"kv_read_q4", (PyCFunction)(void (*)(void))kv_read_q4, METH_FASTCALL, nullptr},
    {"paged_attn_q4", (PyCFunction)(void (*)(void))paged_attn_q4, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_pec_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pec_torch(void) { return PyModule_Create(&g_module); }
