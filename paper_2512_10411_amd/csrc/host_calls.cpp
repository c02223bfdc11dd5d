// The way from torch tensors to libswaa's C entry points in native code, for calls in plain form: torch's own dense
// GPU tensors, all on the device that is current, results to be allocated, torch's current stream, no mode
// or transform of torch in between.  Whatever else a call is, these functions return None, and the binding's Python takes
// it, with its checks, messages and streams; so this file refuses nothing and reports nothing by itself.
//
// A prompt of 64 tokens took 8.9 us a call and takes 5.7, decode of 682 tokens 14.2 and 8.4: argument checks, two results
// from torch's allocator and the foreign-function call each cost about as much in Python as the launch.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <torch/version.h>

#include <cmath>
#include <cstring>

#include "swaa.h"

namespace {

// libswaa's entry points: addresses from the library that the binding has loaded.
decltype(&swaa_attn_fwd) fwd_entry;
decltype(&swaa_attn_fwd_fa_decode) fwd_fa_decode_entry;
decltype(&swaa_attn_decode) decode_entry;
decltype(&swaa_attn_decode_workspace_bytes) decode_workspace_entry;
decltype(&swaa_attn_decode_ex) decode_ex_entry;
decltype(&swaa_attn_decode_ex_workspace_bytes) decode_ex_workspace_entry;

// Does nothing of torch stand between a call and its tensors (function or dispatch modes, transforms, tracing)?
bool nothing_between() {
    return at::impl::PythonTorchFunctionTLS::stack_len() == 0 && !c10::impl::dispatch_mode_enabled() &&
           (c10::impl::tls_local_dispatch_key_set().included_.raw_repr() & ~c10::default_included_set.raw_repr()) == 0;
}

// torch's current device and the handle of its current stream (Python's torch._C._cuda_getDevice and _cuda_getCurrentRawStream).
PyObject *current_device, *current_stream;

// Is q one of torch's own tensors, on the GPU that is current?  Then that GPU and its current stream.
bool plain_call(PyObject *q, int &device, void *&stream) {
    if (!THPVariable_CheckExact(q) || !THPVariable_Unpack(q).defined() || !THPVariable_Unpack(q).is_cuda() || !nothing_between())
        return false;
    PyObject *dev = PyObject_CallNoArgs(current_device);
    if (!dev) throw python_error();
    device = (int)PyLong_AsLong(dev);
    PyObject *handle = device == THPVariable_Unpack(q).get_device() ? PyObject_CallOneArg(current_stream, dev) : nullptr;
    Py_DECREF(dev);
    if (PyErr_Occurred()) {
        Py_XDECREF(handle);
        throw python_error();
    }
    if (!handle) return false;
    stream = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (PyErr_Occurred()) throw python_error();
    return true;
}

// The tensor behind o if it is one of torch's own, dense and plain, on GPU `device`; else null.
const at::Tensor *plain_tensor(PyObject *o, int device) {
    static const uint64_t plain_keys = c10::DispatchKeySet({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA,
                                                            c10::DispatchKey::AutocastCUDA, c10::DispatchKey::ADInplaceOrView}).raw_repr();
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || (t.key_set().raw_repr() & ~plain_keys) != 0 || !t.has_storage() || t.get_device() != device)
        return nullptr;
    return &t;
}
bool plain_vector(PyObject *o, int device, int64_t n, const at::Tensor *&t) {  // n ints, contiguous
    t = plain_tensor(o, device);
    return t && t->scalar_type() == at::kInt && t->dim() == 1 && t->is_contiguous() && (n < 0 || t->numel() == n);
}
// An int as ctypes passes it (the low 32 bits), if o is one.
bool plain_int(PyObject *o, int &x) {
    if (!PyLong_CheckExact(o)) return false;
    x = (int)PyLong_AsUnsignedLongMask(o);
    return true;
}
bool plain_scale(PyObject *o, int64_t D, float &scale) {
    if (o == Py_None) {
        if (D <= 0) return false;
        scale = (float)(1.0 / std::sqrt((double)D));
        return true;
    }
    if (!PyFloat_CheckExact(o)) return false;
    scale = (float)PyFloat_AS_DOUBLE(o);
    return true;
}
bool contiguous_bf16_4d(const at::Tensor *t) {
    return t && t->scalar_type() == at::kBFloat16 && t->dim() == 4 && t->is_contiguous();
}

// (out, lse), or the entry point's status for the binding to raise.
PyObject *results(long long rc, const at::Tensor &out, const at::Tensor &lse) {
    if (rc != SWAA_OK) return PyLong_FromLongLong(rc);
    PyObject *pair = PyTuple_New(2);
    if (!pair) return nullptr;
    PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(out));
    PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(lse));
    return pair;
}
at::Tensor result_like(const at::Tensor &t) { return at::empty_strided(t.sizes(), t.strides(), t.options()); }
at::Tensor empty_floats(const at::Tensor &on, at::IntArrayRef sizes) { return at::empty(sizes, on.options().dtype(at::kFloat)); }
at::Tensor empty_bytes(const at::Tensor &on, int64_t n) { return at::empty({n}, on.options().dtype(at::kByte)); }

// fwd(q, k, v, window, n_sink, n_prompt or None, scale or None)
PyObject *fwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int window, n_sink, n_prompt = 0, device;
    float scale;
    void *stream;
    if (n != 7 || !plain_call(a[0], device, stream)) Py_RETURN_NONE;
    const at::Tensor *q = plain_tensor(a[0], device), *k = plain_tensor(a[1], device), *v = plain_tensor(a[2], device);
    if (!contiguous_bf16_4d(q) || !contiguous_bf16_4d(k) || !contiguous_bf16_4d(v)) Py_RETURN_NONE;
    const int64_t B = q->size(0), Hq = q->size(1), N = q->size(2), D = q->size(3), Hkv = k->size(1);
    if (k->sizes() != v->sizes() || k->size(0) != B || k->size(2) != N || k->size(3) != D) Py_RETURN_NONE;
    if (!plain_int(a[3], window) || !plain_int(a[4], n_sink) || !plain_scale(a[6], D, scale)) Py_RETURN_NONE;
    if (a[5] != Py_None && !plain_int(a[5], n_prompt)) Py_RETURN_NONE;
    const at::Tensor out = result_like(*q), lse = empty_floats(*q, {B, Hq, N});
    const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
    void *op = out.data_ptr();
    float *lp = static_cast<float *>(lse.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (a[5] == Py_None)
        rc = fwd_entry(qp, kp, vp, op, lp, (int)B, (int)Hq, (int)Hkv, (int)N, (int)D, window, n_sink, scale, stream);
    else
        rc = fwd_fa_decode_entry(qp, kp, vp, op, lp, (int)B, (int)Hq, (int)Hkv, (int)N, (int)D, window, n_sink, n_prompt, scale, stream);
    Py_END_ALLOW_THREADS
    return results(rc, out, lse);
    END_HANDLE_TH_ERRORS
}

// decode(q, k, v, window, n_sink, scale or None, workspace or None)
PyObject *decode(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int window, n_sink, device;
    float scale;
    void *stream;
    if (n != 7 || !plain_call(a[0], device, stream)) Py_RETURN_NONE;
    const at::Tensor *q = plain_tensor(a[0], device), *k = plain_tensor(a[1], device), *v = plain_tensor(a[2], device);
    if (!contiguous_bf16_4d(q) || !contiguous_bf16_4d(k) || !contiguous_bf16_4d(v)) Py_RETURN_NONE;
    const int64_t B = q->size(0), Hq = q->size(1), Nq = q->size(2), D = q->size(3), Hkv = k->size(1), Nk = k->size(2);
    if (k->sizes() != v->sizes() || k->size(0) != B || k->size(3) != D || q->numel() == 0 || k->numel() == 0) Py_RETURN_NONE;
    if (!plain_int(a[3], window) || !plain_int(a[4], n_sink) || !plain_scale(a[5], D, scale)) Py_RETURN_NONE;
    at::Tensor workspace;
    if (a[6] == Py_None) {
        const long long need = decode_workspace_entry((int)B, (int)Hq, (int)Hkv, (int)Nq, (int)Nk, (int)D, window, n_sink);
        if (need < 0) return PyLong_FromLongLong(need);
        workspace = empty_bytes(*q, need);
    } else {
        const at::Tensor *given = plain_tensor(a[6], device);
        if (!given || given->scalar_type() != at::kByte || !given->is_contiguous()) Py_RETURN_NONE;
        workspace = *given;
    }
    const at::Tensor out = result_like(*q), lse = empty_floats(*q, {B, Hq, Nq});
    const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
    void *op = out.data_ptr(), *wp = workspace.data_ptr();
    float *lp = static_cast<float *>(lse.data_ptr());
    const long long bytes = workspace.numel();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = decode_entry(qp, kp, vp, op, lp, (int)B, (int)Hq, (int)Hkv, (int)Nq, (int)Nk, (int)D, window, n_sink, scale, wp, bytes, stream);
    Py_END_ALLOW_THREADS
    return results(rc, out, lse);
    END_HANDLE_TH_ERRORS
}

bool view_4d(const at::Tensor *t, at::ScalarType dtype) { return t && t->scalar_type() == dtype && t->dim() == 4 && t->stride(3) == 1; }

// decode_ex(q, k, v, window, n_sink, scale, seq_lens, block_table, max_seqlen_k, workspace); None for what is not given
PyObject *decode_ex(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int device;
    swaa_decode_args s{};
    if (n != 10 || !plain_call(a[0], device, s.stream)) Py_RETURN_NONE;
    const at::Tensor *q = plain_tensor(a[0], device), *k = plain_tensor(a[1], device), *v = plain_tensor(a[2], device);
    if (!q || (q->scalar_type() != at::kBFloat16 && q->scalar_type() != at::kHalf) || q->dim() != 4 || !q->is_contiguous()) Py_RETURN_NONE;
    if (!view_4d(k, q->scalar_type()) || !view_4d(v, q->scalar_type())) Py_RETURN_NONE;
    const int64_t B = q->size(0), Hq = q->size(1), Nq = q->size(2), D = q->size(3);
    if (!plain_int(a[3], s.window) || !plain_int(a[4], s.n_sink) || !plain_scale(a[5], D, s.scale)) Py_RETURN_NONE;
    s.B = (int)B, s.Hq = (int)Hq, s.Nq = (int)Nq, s.D = (int)D, s.Hkv = (int)k->size(1), s.Nk = (int)k->size(2);
    const at::Tensor *t;
    if (a[6] != Py_None) {
        if (!plain_vector(a[6], device, B, t)) Py_RETURN_NONE;
        s.seq_lens = static_cast<const int *>(t->data_ptr());
    }
    if (a[7] != Py_None) {
        t = plain_tensor(a[7], device);
        if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || t->stride(1) != 1 || t->size(0) != B || a[8] == Py_None) Py_RETURN_NONE;
        s.block_table = static_cast<const int *>(t->data_ptr());
        s.block_table_stride = (int)t->stride(0), s.page_size = (int)k->size(2), s.num_pages = (int)k->size(0);
    }
    if (a[8] != Py_None && !plain_int(a[8], s.Nk)) Py_RETURN_NONE;
    s.dtype = q->scalar_type() == at::kHalf ? SWAA_F16 : SWAA_BF16;
    s.q = q->data_ptr();
    s.k = {k->data_ptr(), k->stride(0), k->stride(1), k->stride(2)};
    s.v = {v->data_ptr(), v->stride(0), v->stride(1), v->stride(2)};
    at::Tensor workspace;
    if (a[9] == Py_None) {
        const long long need = decode_ex_workspace_entry(&s);
        if (need < 0) return PyLong_FromLongLong(need);
        workspace = empty_bytes(*q, need);
    } else {
        const at::Tensor *given = plain_tensor(a[9], device);
        if (!given) Py_RETURN_NONE;
        workspace = *given;
    }
    s.workspace = workspace.data_ptr(), s.workspace_bytes = workspace.numel();
    const at::Tensor out = result_like(*q), lse = empty_floats(*q, {B, Hq, Nq});
    s.out = out.data_ptr(), s.lse = static_cast<float *>(lse.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = decode_ex_entry(&s);
    Py_END_ALLOW_THREADS
    return results(rc, out, lse);
    END_HANDLE_TH_ERRORS
}

// fill_fwd_ex(args, q, k, v, window, n_sink, n_prompt, scale, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k, block_table,
// total_rows_q, n_prompts): fills the argument block `args` (writable bytes) and returns the results it points at.
PyObject *fill_fwd_ex(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int device;
    swaa_fwd_args s{};
    if (n != 15 || !plain_call(a[1], device, s.stream)) Py_RETURN_NONE;
    const bool packed = a[8] != Py_None || a[9] != Py_None, paged = a[12] != Py_None;
    const at::Tensor *q = plain_tensor(a[1], device), *k = plain_tensor(a[2], device), *v = plain_tensor(a[3], device);
    if (!q || (q->scalar_type() != at::kBFloat16 && q->scalar_type() != at::kHalf)) Py_RETURN_NONE;
    const int64_t q_dims = packed ? 3 : 4, kv_dims = paged ? 4 : q_dims;
    if (q->dim() != q_dims || q->stride(-1) != 1) Py_RETURN_NONE;
    for (const at::Tensor *t : {k, v})
        if (!t || t->scalar_type() != q->scalar_type() || t->dim() != kv_dims || t->stride(-1) != 1) Py_RETURN_NONE;
    const int64_t D = q->size(-1);
    s.D = (int)D, s.Hq = (int)q->size(-3), s.Hkv = (int)k->size(-3);
    if (!plain_int(a[4], s.window) || !plain_int(a[5], s.n_sink) || !plain_scale(a[7], D, s.scale)) Py_RETURN_NONE;
    s.n_prompt = 0x7fffffff;
    if (a[6] != Py_None && !plain_int(a[6], s.n_prompt)) Py_RETURN_NONE;
    int64_t B;
    const at::Tensor *t;
    if (packed) {
        const at::Tensor *cu_q, *cu_k;
        if (!plain_vector(a[8], device, -1, cu_q) || !plain_vector(a[9], device, cu_q->numel(), cu_k)) Py_RETURN_NONE;
        B = cu_q->numel() - 1;
        s.cu_seqlens_q = static_cast<const int *>(cu_q->data_ptr()), s.cu_seqlens_k = static_cast<const int *>(cu_k->data_ptr());
        if (!plain_int(a[10], s.Nq) || !plain_int(a[11], s.Nk)) Py_RETURN_NONE;
    } else {
        B = q->size(0), s.Nq = (int)q->size(2), s.Nk = (int)k->size(2);
    }
    s.B = (int)B;
    if (paged) {
        t = plain_tensor(a[12], device);
        if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || t->stride(1) != 1 || t->size(0) != B || !plain_int(a[11], s.Nk))
            Py_RETURN_NONE;
        s.block_table = static_cast<const int *>(t->data_ptr());
        s.block_table_stride = (int)t->stride(0), s.page_size = (int)k->size(2), s.num_pages = (int)k->size(0);
    }
    s.total_rows_q = packed ? q->size(1) : 0;
    if (a[13] != Py_None) {
        if (!PyLong_CheckExact(a[13])) Py_RETURN_NONE;
        s.total_rows_q = (long long)PyLong_AsUnsignedLongLongMask(a[13]);
    }
    if (a[14] != Py_None) {
        if (!plain_vector(a[14], device, B, t)) Py_RETURN_NONE;
        s.n_prompts = static_cast<const int *>(t->data_ptr());
    }
    s.dtype = q->scalar_type() == at::kHalf ? SWAA_F16 : SWAA_BF16;
    auto strided = [](const at::Tensor &t) {
        return t.dim() == 3 ? swaa_tensor{t.data_ptr(), 0, t.stride(0), t.stride(1)}
                            : swaa_tensor{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
    };
    const at::Tensor out = result_like(*q), lse = packed ? empty_floats(*q, {q->size(0), q->size(1)}) : empty_floats(*q, {B, q->size(1), q->size(2)});
    s.q = strided(*q), s.k = strided(*k), s.v = strided(*v), s.out = strided(out);
    s.lse = static_cast<float *>(lse.data_ptr());
    s.lse_stride_b = packed ? 0 : lse.stride(0), s.lse_stride_h = lse.stride(packed ? 0 : 1);
    Py_buffer block;
    if (PyObject_GetBuffer(a[0], &block, PyBUF_WRITABLE) != 0) return nullptr;
    const bool fits = block.len == (Py_ssize_t)sizeof(s);
    if (fits) std::memcpy(block.buf, &s, sizeof(s));
    PyBuffer_Release(&block);
    if (!fits) Py_RETURN_NONE;
    return results(SWAA_OK, out, lse);
    END_HANDLE_TH_ERRORS
}

decltype(&swaa_qk_norm_rope) norm_rope_entry;
decltype(&swaa_qk_norm_rope_bwd) norm_rope_bwd_entry;
decltype(&swaa_qk_norm_rope_bwd_workspace_bytes) norm_rope_bwd_workspace_entry;

// swaa_tensor of a view [blocks, heads, rows, D] or [heads, rows, D] (a dimension of one entry has no stride to speak of).
swaa_tensor rows_of(const at::Tensor &t) {
    const int64_t d = t.dim() - 3, n = t.size(d + 1);
    return {t.data_ptr(), d && t.size(0) > 1 ? t.stride(0) : 0, t.size(d) > 1 ? t.stride(d) : 0, n > 1 ? t.stride(d + 1) : t.size(d + 2)};
}
// Address of a contiguous tensor of numbers of this type and shape, if it is given; false if it is anything else.
template <typename T>
bool plain_numbers(PyObject *o, int device, at::ScalarType dtype, at::IntArrayRef sizes, const T *&data) {
    if (o == Py_None) return true;
    const at::Tensor *t = plain_tensor(o, device);
    if (!t || t->scalar_type() != dtype || t->sizes() != sizes || !t->is_contiguous()) return false;
    data = static_cast<const T *>(t->data_ptr());
    return true;
}

// norm_rope(q, k, inv_freq, positions, q_weight, k_weight, eps, interleaved, v, k_out, v_out, cu_seqlens_q, cu_seqlens_k, max_seqlen_q,
// max_seqlen_k, seq_lens, block_table, total_rows_q): (q_out, k_out), the latter None if it was given
PyObject *norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int device;
    swaa_norm_rope_args s{};
    if (n != 18 || !plain_call(a[0], device, s.stream)) Py_RETURN_NONE;
    const bool packed = a[11] != Py_None, paged = a[16] != Py_None, cache = a[9] != Py_None;
    const int64_t dims = packed ? 3 : 4;
    const at::Tensor *q = plain_tensor(a[0], device), *k = plain_tensor(a[1], device), *t;
    if (!q || (q->scalar_type() != at::kBFloat16 && q->scalar_type() != at::kHalf)) Py_RETURN_NONE;
    auto like_q = [&](const at::Tensor *x, int64_t d) { return x && x->scalar_type() == q->scalar_type() && x->dim() == d && x->stride(-1) == 1 && x->size(-1) == q->size(-1); };
    if (!like_q(q, dims) || !like_q(k, dims) || k->size(-2) != q->size(-2) || (!packed && k->size(0) != q->size(0))) Py_RETURN_NONE;
    const int64_t D = q->size(-1), T = q->size(-2), Hkv = k->size(-3), B = packed ? 0 : q->size(0);
    s.Hq = (int)q->size(-3), s.Hkv = (int)Hkv, s.D = (int)D;
    if (a[2] != Py_None) {
        t = plain_tensor(a[2], device);
        if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous()) Py_RETURN_NONE;
        s.inv_freq = static_cast<const float *>(t->data_ptr()), s.rot_dim = (int)(2 * t->numel());
    }
    if ((a[4] == Py_None) != (a[5] == Py_None) || !plain_numbers(a[4], device, at::kFloat, {D}, s.q_weight) || !plain_numbers(a[5], device, at::kFloat, {D}, s.k_weight))
        Py_RETURN_NONE;
    if (!PyFloat_CheckExact(a[6]) || !PyBool_Check(a[7])) Py_RETURN_NONE;
    s.eps = (float)PyFloat_AS_DOUBLE(a[6]), s.interleaved = a[7] == Py_True;
    const at::Tensor *v = nullptr, *k_out = nullptr, *v_out = nullptr;
    if (cache) {
        k_out = plain_tensor(a[9], device);
        if (!like_q(k_out, paged ? 4 : dims) || k_out->size(-3) != Hkv || (!packed && !paged && k_out->size(0) != B)) Py_RETURN_NONE;
        if (packed && a[12] == Py_None) Py_RETURN_NONE;
    } else if (paged || a[15] != Py_None || a[12] != Py_None) {
        Py_RETURN_NONE;
    }
    if (a[8] != Py_None) {
        v = plain_tensor(a[8], device), v_out = cache ? plain_tensor(a[10], device) : nullptr;
        if (!like_q(v, dims) || v->sizes() != k->sizes() || !like_q(v_out, k_out ? k_out->dim() : 0) || v_out->sizes() != k_out->sizes()) Py_RETURN_NONE;
        s.v = rows_of(*v), s.v_out = rows_of(*v_out);
    } else if (a[10] != Py_None) {
        Py_RETURN_NONE;
    }
    if (packed) {
        const at::Tensor *cu_q, *cu_k;
        if (!plain_vector(a[11], device, -1, cu_q) || !plain_vector(cache ? a[12] : a[11], device, cu_q->numel(), cu_k) || a[15] != Py_None) Py_RETURN_NONE;
        s.B = (int)cu_q->numel() - 1;
        s.cu_seqlens_q = static_cast<const int *>(cu_q->data_ptr()), s.cu_seqlens_k = static_cast<const int *>(cu_k->data_ptr());
        if (!plain_int(a[13], s.Nq) || !plain_int(cache ? a[14] : a[13], s.Nk)) Py_RETURN_NONE;
        s.total_rows_q = T;
        if (a[17] != Py_None) Py_RETURN_NONE;
    } else {
        const int64_t rows = cache ? k_out->size(-2) : T;
        if (a[12] != Py_None || (paged && a[14] == Py_None)) Py_RETURN_NONE;
        s.B = (int)B, s.Nq = (int)T, s.Nk = (int)rows;
        if (a[14] != Py_None && (!plain_int(a[14], s.Nk) || (!paged && s.Nk > rows))) Py_RETURN_NONE;
        if (!plain_numbers(a[15], device, at::kInt, {B}, s.seq_lens)) Py_RETURN_NONE;
    }
    if (paged) {
        t = plain_tensor(a[16], device);
        if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != s.B || t->size(0) < 1 || (t->size(1) > 1 && t->stride(1) != 1)) Py_RETURN_NONE;
        s.block_table = static_cast<const int *>(t->data_ptr());
        s.block_table_stride = (int)(s.B > 1 ? t->stride(0) : t->size(1)), s.page_size = (int)k_out->size(2), s.num_pages = (int)k_out->size(0);
    }
    if (packed ? !plain_numbers(a[3], device, at::kInt, {T}, s.positions) : !plain_numbers(a[3], device, at::kInt, {B, T}, s.positions)) Py_RETURN_NONE;
    s.dtype = q->scalar_type() == at::kHalf ? SWAA_F16 : SWAA_BF16;
    const at::Tensor q_new = at::empty(q->sizes(), q->options()), k_new = cache ? at::Tensor() : at::empty(k->sizes(), k->options());
    s.q = rows_of(*q), s.k = rows_of(*k), s.q_out = rows_of(q_new), s.k_out = rows_of(cache ? *k_out : k_new);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = norm_rope_entry(&s);
    Py_END_ALLOW_THREADS
    if (rc != SWAA_OK) return PyLong_FromLong(rc);
    PyObject *pair = PyTuple_New(2);
    if (!pair) return nullptr;
    PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(q_new));
    PyObject *second = cache ? Py_None : THPVariable_Wrap(k_new);
    if (cache) Py_INCREF(second);
    PyTuple_SET_ITEM(pair, 1, second);
    return pair;
    END_HANDLE_TH_ERRORS
}

// norm_rope_bwd(dq_out, dk_out, q, k, inv_freq, positions, q_weight, k_weight, eps, interleaved): (dq, dk, dq_weight, dk_weight)
PyObject *norm_rope_bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int device;
    swaa_norm_rope_bwd_args s{};
    if (n != 10 || !plain_call(a[2], device, s.stream)) Py_RETURN_NONE;
    const at::Tensor *x[4], *t;  // dq_out, dk_out, q, k
    for (int i = 0; i < 4; ++i) {
        x[i] = plain_tensor(a[i], device);
        if (!x[i] || x[i]->dim() != 4 || x[i]->stride(3) != 1) Py_RETURN_NONE;
    }
    const at::Tensor &q = *x[2], &k = *x[3];
    if (q.scalar_type() != at::kBFloat16 && q.scalar_type() != at::kHalf) Py_RETURN_NONE;
    for (const at::Tensor *y : x)
        if (y->scalar_type() != q.scalar_type()) Py_RETURN_NONE;
    const int64_t B = q.size(0), N = q.size(2), D = q.size(3);
    if (k.size(0) != B || k.size(2) != N || k.size(3) != D || x[0]->sizes() != q.sizes() || x[1]->sizes() != k.sizes()) Py_RETURN_NONE;
    s.B = (int)B, s.Hq = (int)q.size(1), s.Hkv = (int)k.size(1), s.D = (int)D, s.N = (int)N;
    if (a[4] != Py_None) {
        t = plain_tensor(a[4], device);
        if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous()) Py_RETURN_NONE;
        s.inv_freq = static_cast<const float *>(t->data_ptr()), s.rot_dim = (int)(2 * t->numel());
    }
    if (!plain_numbers(a[5], device, at::kInt, {B, N}, s.positions)) Py_RETURN_NONE;
    const bool norm = a[6] != Py_None;
    if (norm != (a[7] != Py_None) || !plain_numbers(a[6], device, at::kFloat, {D}, s.q_weight) || !plain_numbers(a[7], device, at::kFloat, {D}, s.k_weight))
        Py_RETURN_NONE;
    if (!PyFloat_CheckExact(a[8]) || !PyBool_Check(a[9])) Py_RETURN_NONE;
    s.eps = (float)PyFloat_AS_DOUBLE(a[8]), s.interleaved = a[9] == Py_True;
    s.dtype = q.scalar_type() == at::kHalf ? SWAA_F16 : SWAA_BF16;
    const long long need = norm_rope_bwd_workspace_entry(&s);
    if (need < 0) return PyLong_FromLongLong(need);
    const at::Tensor dq = at::empty_like(q), dk = at::empty_like(k);
    at::Tensor workspace, dw[2];
    if (need > 0) workspace = empty_bytes(q, need), s.workspace = workspace.data_ptr(), s.workspace_bytes = need;
    if (norm) {
        for (at::Tensor &w : dw) w = empty_floats(q, {D});
        s.dq_weight = static_cast<float *>(dw[0].data_ptr()), s.dk_weight = static_cast<float *>(dw[1].data_ptr());
    }
    s.dq_out = rows_of(*x[0]), s.dk_out = rows_of(*x[1]), s.q = rows_of(q), s.k = rows_of(k), s.dq = rows_of(dq), s.dk = rows_of(dk);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = norm_rope_bwd_entry(&s);
    Py_END_ALLOW_THREADS
    if (rc != SWAA_OK) return PyLong_FromLong(rc);
    PyObject *all = PyTuple_New(4);
    if (!all) return nullptr;
    PyTuple_SET_ITEM(all, 0, THPVariable_Wrap(dq));
    PyTuple_SET_ITEM(all, 1, THPVariable_Wrap(dk));
    for (int i = 0; i < 2; ++i) {
        if (!norm) Py_INCREF(Py_None);
        PyTuple_SET_ITEM(all, 2 + i, norm ? THPVariable_Wrap(dw[i]) : Py_None);
    }
    return all;
    END_HANDLE_TH_ERRORS
}

decltype(&swaa_attn_key_weights) key_weights_entry;
decltype(&swaa_attn_key_weights_workspace_bytes) key_weights_workspace_entry;
decltype(&swaa_cache_evict) evict_entry;
decltype(&swaa_cache_evict_workspace_bytes) evict_workspace_entry;

// Weights [B, Hkv, >= Nk] with contiguous rows.
bool plain_weights(PyObject *o, int device, int64_t B, int64_t Hkv, int64_t Nk, float *&data, long long &stride_b, long long &stride_h) {
    const at::Tensor *t = plain_tensor(o, device);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 3 || t->size(0) != B || t->size(1) != Hkv || t->size(2) < Nk || (t->size(2) > 1 && t->stride(2) != 1))
        return false;
    data = static_cast<float *>(t->data_ptr());
    stride_b = B > 1 ? t->stride(0) : 0, stride_h = Hkv > 1 ? t->stride(1) : 0;
    return true;
}
// A block table of B sequences and the pages of `cache`, if there is one.
template <typename Args>
bool plain_pages(PyObject *o, int device, int64_t B, const at::Tensor &cache, Args &s) {
    if (o == Py_None) return true;
    const at::Tensor *t = plain_tensor(o, device);
    if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || t->size(0) != B || B < 1 || (t->size(1) > 1 && t->stride(1) != 1)) return false;
    s.block_table = static_cast<const int *>(t->data_ptr());
    s.block_table_stride = (int)(B > 1 ? t->stride(0) : t->size(1)), s.page_size = (int)cache.size(2), s.num_pages = (int)cache.size(0);
    return true;
}

// key_weights(q, k, lse, window, n_sink, n_prompt, scale, weights, decay, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k, seq_lens,
// block_table, n_prompts): True
PyObject *key_weights(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int device;
    swaa_key_weights_args s{};
    if (n != 16 || !plain_call(a[0], device, s.stream)) Py_RETURN_NONE;
    const bool packed = a[9] != Py_None, paged = a[14] != Py_None;
    const int64_t dims = packed ? 3 : 4;
    const at::Tensor *q = plain_tensor(a[0], device), *k = plain_tensor(a[1], device);
    if (!q || (q->scalar_type() != at::kBFloat16 && q->scalar_type() != at::kHalf) || q->dim() != dims || q->stride(-1) != 1) Py_RETURN_NONE;
    if (!k || k->scalar_type() != q->scalar_type() || k->dim() != (paged ? 4 : dims) || k->stride(-1) != 1 || k->size(-1) != q->size(-1)) Py_RETURN_NONE;
    const int64_t D = q->size(-1), T = q->size(-2), Hq = q->size(-3), Hkv = k->size(-3), rows = k->size(-2);
    int64_t B = packed ? 0 : q->size(0);
    if (!packed && !paged && k->size(0) != B) Py_RETURN_NONE;
    if (packed) {
        const at::Tensor *cu_q, *cu_k;
        if (!plain_vector(a[9], device, -1, cu_q) || !plain_vector(a[10], device, cu_q->numel(), cu_k) || a[13] != Py_None) Py_RETURN_NONE;
        B = cu_q->numel() - 1;
        s.cu_seqlens_q = static_cast<const int *>(cu_q->data_ptr()), s.cu_seqlens_k = static_cast<const int *>(cu_k->data_ptr());
        if (!plain_int(a[11], s.Nq) || !plain_int(a[12], s.Nk)) Py_RETURN_NONE;
    } else {
        if (a[10] != Py_None || (paged && a[12] == Py_None)) Py_RETURN_NONE;
        s.Nq = (int)T, s.Nk = (int)rows;
        if (a[12] != Py_None && (!plain_int(a[12], s.Nk) || (!paged && s.Nk > rows))) Py_RETURN_NONE;
        if (!plain_numbers(a[13], device, at::kInt, {B}, s.seq_lens)) Py_RETURN_NONE;
    }
    s.B = (int)B, s.Hq = (int)Hq, s.Hkv = (int)Hkv, s.D = (int)D;
    if (a[2] == Py_None || !(packed ? plain_numbers(a[2], device, at::kFloat, {Hq, T}, s.lse) : plain_numbers(a[2], device, at::kFloat, {B, Hq, T}, s.lse))) Py_RETURN_NONE;
    s.lse_stride_b = packed ? 0 : Hq * T, s.lse_stride_h = T;
    s.n_prompt = 0x7fffffff;
    if (!plain_int(a[3], s.window) || !plain_int(a[4], s.n_sink) || (a[5] != Py_None && !plain_int(a[5], s.n_prompt))) Py_RETURN_NONE;
    if (!plain_scale(a[6], D, s.scale) || !PyFloat_CheckExact(a[8]) || !plain_pages(a[14], device, B, *k, s)) Py_RETURN_NONE;
    s.decay = (float)PyFloat_AS_DOUBLE(a[8]);
    if (!plain_numbers(a[15], device, at::kInt, {B}, s.n_prompts)) Py_RETURN_NONE;
    if (!plain_weights(a[7], device, B, Hkv, s.Nk, s.weights, s.weights_stride_b, s.weights_stride_h)) Py_RETURN_NONE;
    s.dtype = q->scalar_type() == at::kHalf ? SWAA_F16 : SWAA_BF16;
    s.q = rows_of(*q), s.k = rows_of(*k);
    const long long need = key_weights_workspace_entry(&s);
    if (need < 0) return PyLong_FromLongLong(need);
    at::Tensor workspace;
    if (need > 0) workspace = empty_bytes(*q, need), s.workspace = workspace.data_ptr(), s.workspace_bytes = need;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = key_weights_entry(&s);
    Py_END_ALLOW_THREADS
    if (rc != SWAA_OK) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// evict(k, v, weights, n_keep, n_sink, n_recent, seq_lens, block_table, max_seqlen_k): (kept, new_lens)
PyObject *evict(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int device;
    swaa_evict_args s{};
    if (n != 9 || !plain_call(a[0], device, s.stream)) Py_RETURN_NONE;
    const bool paged = a[7] != Py_None;
    const at::Tensor *k = plain_tensor(a[0], device), *v = plain_tensor(a[1], device);
    for (const at::Tensor *t : {k, v})
        if (!t || (t->scalar_type() != at::kBFloat16 && t->scalar_type() != at::kHalf) || t->dim() != 4 || t->stride(3) != 1) Py_RETURN_NONE;
    if (k->scalar_type() != v->scalar_type() || k->sizes() != v->sizes() || (paged && a[8] == Py_None)) Py_RETURN_NONE;
    const at::Tensor *table = paged ? plain_tensor(a[7], device) : nullptr;
    if (paged && (!table || table->dim() != 2)) Py_RETURN_NONE;
    const int64_t B = paged ? table->size(0) : k->size(0), Hkv = k->size(1);
    s.B = (int)B, s.Hkv = (int)Hkv, s.D = (int)k->size(3), s.Nk = (int)k->size(2);
    if (a[8] != Py_None && (!plain_int(a[8], s.Nk) || (!paged && s.Nk > k->size(2)))) Py_RETURN_NONE;
    if (!plain_int(a[3], s.n_keep) || !plain_int(a[4], s.n_sink) || !plain_int(a[5], s.n_recent) || s.n_keep < 1 || B < 1) Py_RETURN_NONE;
    if (!plain_numbers(a[6], device, at::kInt, {B}, s.seq_lens) || !plain_pages(a[7], device, B, *k, s)) Py_RETURN_NONE;
    if (!plain_weights(a[2], device, B, Hkv, s.Nk, s.weights, s.weights_stride_b, s.weights_stride_h)) Py_RETURN_NONE;
    const at::Tensor kept = at::empty({B, Hkv, s.n_keep}, k->options().dtype(at::kInt)), lens = at::empty({B}, k->options().dtype(at::kInt));
    s.kept = static_cast<int *>(kept.data_ptr()), s.new_lens = static_cast<int *>(lens.data_ptr());
    s.k = rows_of(*k), s.v = rows_of(*v);
    const long long need = evict_workspace_entry(&s);
    if (need < 0) return PyLong_FromLongLong(need);
    at::Tensor workspace;
    if (need > 0) workspace = empty_bytes(*k, need), s.workspace = workspace.data_ptr(), s.workspace_bytes = need;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = evict_entry(&s);
    Py_END_ALLOW_THREADS
    return results(rc, kept, lens);
    END_HANDLE_TH_ERRORS
}

// bind_cache(addresses of the seven entry points above, sizes of the binding's four argument blocks), behind bind, which has checked
// the library.
PyObject *bind_cache(PyObject *, PyObject *const *a, Py_ssize_t n) {
    constexpr int kEntries = 7, kBlocks = 4;
    static const size_t blocks[kBlocks] = {sizeof(swaa_norm_rope_args), sizeof(swaa_norm_rope_bwd_args), sizeof(swaa_key_weights_args), sizeof(swaa_evict_args)};
    if (n != kEntries + kBlocks) {
        PyErr_SetString(PyExc_TypeError, "bind_cache takes seven addresses and four numbers");
        return nullptr;
    }
    void *at[kEntries];
    for (int i = 0; i < kEntries; ++i) {
        at[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    for (int i = 0; i < kBlocks; ++i) {
        const long long bytes = PyLong_AsLongLong(a[kEntries + i]);
        if (PyErr_Occurred()) return nullptr;
        if (bytes != (long long)blocks[i]) {
            PyErr_Format(PyExc_ImportError, "compiled for an argument block of %zu bytes, not %lld", blocks[i], bytes);
            return nullptr;
        }
    }
    norm_rope_entry = reinterpret_cast<decltype(norm_rope_entry)>(at[0]);
    norm_rope_bwd_entry = reinterpret_cast<decltype(norm_rope_bwd_entry)>(at[1]);
    norm_rope_bwd_workspace_entry = reinterpret_cast<decltype(norm_rope_bwd_workspace_entry)>(at[2]);
    key_weights_entry = reinterpret_cast<decltype(key_weights_entry)>(at[3]);
    key_weights_workspace_entry = reinterpret_cast<decltype(key_weights_workspace_entry)>(at[4]);
    evict_entry = reinterpret_cast<decltype(evict_entry)>(at[5]);
    evict_workspace_entry = reinterpret_cast<decltype(evict_workspace_entry)>(at[6]);
    Py_RETURN_NONE;
}

// bind(addresses of the first six entry points, in their order, then current_device and current_stream, the library's version, the
// sizes of the binding's two argument blocks, torch's version).  ImportError if this file was compiled for others: a call from here
// hands the library pointers and strides where the header it was compiled with has them.
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    void *at[6];
    if (n != 12) {
        PyErr_SetString(PyExc_TypeError, "bind takes six addresses, two functions, three numbers and a text");
        return nullptr;
    }
    for (int i = 0; i < 6; ++i) {
        at[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    const long long version = PyLong_AsLongLong(a[8]), fwd_bytes = PyLong_AsLongLong(a[9]), decode_bytes = PyLong_AsLongLong(a[10]);
    const char *torch_version = PyErr_Occurred() ? nullptr : PyUnicode_AsUTF8(a[11]);
    if (!torch_version) return nullptr;
    if (version != SWAA_VERSION || fwd_bytes != (long long)sizeof(swaa_fwd_args) || decode_bytes != (long long)sizeof(swaa_decode_args)) {
        PyErr_Format(PyExc_ImportError, "compiled for libswaa %d with argument blocks of %zu and %zu bytes, not %lld with %lld and %lld",
                     SWAA_VERSION, sizeof(swaa_fwd_args), sizeof(swaa_decode_args), version, fwd_bytes, decode_bytes);
        return nullptr;
    }
    if (std::strncmp(torch_version, TORCH_VERSION, std::strlen(TORCH_VERSION)) != 0) {
        PyErr_Format(PyExc_ImportError, "compiled for torch %s, not %s", TORCH_VERSION, torch_version);
        return nullptr;
    }
    fwd_entry = reinterpret_cast<decltype(fwd_entry)>(at[0]);
    fwd_fa_decode_entry = reinterpret_cast<decltype(fwd_fa_decode_entry)>(at[1]);
    decode_entry = reinterpret_cast<decltype(decode_entry)>(at[2]);
    decode_workspace_entry = reinterpret_cast<decltype(decode_workspace_entry)>(at[3]);
    decode_ex_entry = reinterpret_cast<decltype(decode_ex_entry)>(at[4]);
    decode_ex_workspace_entry = reinterpret_cast<decltype(decode_ex_workspace_entry)>(at[5]);
    Py_INCREF(a[6]);
    Py_INCREF(a[7]);
    Py_XSETREF(current_device, a[6]);
    Py_XSETREF(current_stream, a[7]);
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(bind_cache), METHOD(fwd), METHOD(decode), METHOD(decode_ex), METHOD(fill_fwd_ex), METHOD(norm_rope), METHOD(norm_rope_bwd),
                         METHOD(key_weights), METHOD(evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host_calls() { return PyModule_Create(&module); }
