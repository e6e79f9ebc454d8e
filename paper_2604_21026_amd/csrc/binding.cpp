// The calls that a program makes once per layer, from torch tensors without a trip through ctypes:
// nvq.gemv_w4a16 and its like spend 2.8 us in Python on shapes, types and the stream (2048 x 2048 at one
// token: 6.4 us a call, of which the launch takes 3.6 and the kernel 2.7).
//
// Only the ordinary case is served here: tensors (no subclasses, which may say themselves where their
// data is) of the expected types on a device (all but the int4 layers' calls: on the current one), contiguous
// (queries, keys, values and logits: or with tokens apart), with fitting shapes and room for what is written
// and read.  For everything else a function returns None and the caller takes its own way, which names what
// is wrong.  The library's entry points are handed over by address (bind); a call returns their status.
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "nvq.h"

namespace {

decltype(&nvq_gemv_w4a16) g_gemv_w4a16;
decltype(&nvq_gemv_w4a8) g_gemv_w4a8;
decltype(&nvq_quant_act_i8) g_quant_act_i8;
decltype(&nvq_gemm_w4a16) g_gemm_w4a16;
decltype(&nvq_quant_mxfp4) g_quant_mxfp4;
decltype(&nvq_dequant_mxfp4) g_dequant_mxfp4;
decltype(&nvq_gemv_mxfp4) g_gemv_mxfp4;
decltype(&nvq_gemm_mxfp4) g_gemm_mxfp4;
decltype(&nvq_moe_route) g_moe_route;
decltype(&nvq_moe_experts) g_moe_experts;
decltype(&nvq_cache_append) g_cache_append;
decltype(&nvq_cache_read) g_cache_read;
decltype(&nvq_attention) g_attention;
decltype(&nvq_sample) g_sample;
decltype(&nvq_adapters_add) g_adapters_add;

constexpr int kAny = -1, kNone = -2;  // for a device's number: any, one that no tensor is on

// A contiguous tensor of that type on device `device`; dims < 0: any shape.
const at::Tensor *device_tensor(PyObject *o, at::ScalarType type, int64_t dims, int device = kAny) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.scalar_type() != type || !t.is_contiguous()) return nullptr;
    if (dims >= 0 && t.dim() != dims) return nullptr;
    if (device != kAny && t.get_device() != device) return nullptr;
    return &t;
}

// The same with room for n values.
const at::Tensor *device_room(PyObject *o, at::ScalarType type, int64_t n, int device = kAny) {
    const at::Tensor *const t = device_tensor(o, type, -1, device);
    return t && t->numel() >= n ? t : nullptr;
}

// The output of a product (n results), and its type for the library.
const at::Tensor *output_tensor(PyObject *o, int64_t n, int *y_dtype, int device = kAny) {
    if (const at::Tensor *t = device_room(o, at::kFloat, n, device)) {
        *y_dtype = NVQ_F32;
        return t;
    }
    *y_dtype = NVQ_BF16;
    return device_room(o, at::kBFloat16, n, device);
}

// The number of the current device, if that tensor is on it, or kNone.  (Asked for once a call: 60 ns.)
int device_of(PyObject *o) {
    if (!THPVariable_CheckExact(o)) return kNone;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda()) return kNone;
    return t.get_device() == c10::hip::current_device() ? t.get_device() : kNone;
}

struct Weights {
    const uint8_t *q;
    const uint16_t *s;
    int64_t N, K;
};
bool weights(PyObject *qweight, PyObject *scales, Weights *w) {
    const at::Tensor *q = device_tensor(qweight, at::kByte, 2), *s = device_tensor(scales, at::kShort, 2);
    if (!q || !s) return false;
    w->N = q->size(0);
    w->K = q->size(1) * 2;
    if (s->size(0) != w->N || s->size(1) != w->K / 32 || w->N > INT32_MAX || w->K > INT32_MAX) return false;
    w->q = static_cast<const uint8_t *>(q->data_ptr());
    w->s = static_cast<const uint16_t *>(s->data_ptr());
    return true;
}

void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

PyObject *none() { Py_RETURN_NONE; }

template <typename CALL>
PyObject *status_of(CALL call) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// (qweight, scales, x, y)
template <bool GEMM>
PyObject *product_w4a16(PyObject *const *a, Py_ssize_t n) {
    Weights w;
    int y_dtype;
    if (n != 4 || !weights(a[0], a[1], &w)) return none();
    const at::Tensor *const x = device_tensor(a[2], at::kBFloat16, 2);
    if (!x || x->size(1) != w.K || x->size(0) > INT32_MAX) return none();
    const int64_t M = x->size(0);
    const at::Tensor *const y = output_tensor(a[3], M * w.N, &y_dtype);
    if (!y) return none();
    const uint16_t *const xp = static_cast<const uint16_t *>(x->data_ptr());
    void *const yp = y->data_ptr(), *const st = current_stream();
    if (GEMM) return status_of([&] { return g_gemm_w4a16(w.q, w.s, w.N, w.K, xp, M, yp, y_dtype, st); });
    return status_of([&] { return g_gemv_w4a16(w.q, w.s, (int)w.N, (int)w.K, xp, (int)M, yp, y_dtype, st); });
}

PyObject *gemv_w4a16(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    return product_w4a16<false>(a, n);
    END_HANDLE_TH_ERRORS
}

PyObject *gemm_w4a16(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    return product_w4a16<true>(a, n);
    END_HANDLE_TH_ERRORS
}

// An int that fits the library's, or false (another type, too large).
bool small_int(PyObject *o, int *v) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow;
    const long l = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || l < INT32_MIN || l > INT32_MAX) return false;
    *v = (int)l;
    return true;
}

// (qweight, scales, xq, xscale, xgsum, act_group, y)
PyObject *gemv_w4a8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Weights w;
    int y_dtype, group;
    if (n != 7 || !weights(a[0], a[1], &w) || !small_int(a[5], &group)) return none();
    const at::Tensor *const xq = device_tensor(a[2], at::kChar, 2);
    if (!xq || xq->size(1) != w.K || xq->size(0) > INT32_MAX) return none();
    const int M = (int)xq->size(0);
    const int64_t groups = M * (w.K / 32);
    const at::Tensor *const xs = device_room(a[3], at::kFloat, group == 32 ? groups : M),
                     *const gs = device_room(a[4], at::kInt, M <= 3 ? groups : 0),  // (read for up to three tokens)
                     *const y = output_tensor(a[6], M * w.N, &y_dtype);
    if (!xs || !gs || !y) return none();
    const int8_t *const xp = static_cast<const int8_t *>(xq->data_ptr());
    const float *const sp = static_cast<const float *>(xs->data_ptr());
    const int32_t *const gp = static_cast<const int32_t *>(gs->data_ptr());
    void *const yp = y->data_ptr(), *const st = current_stream();
    return status_of([&] {
        return g_gemv_w4a8(w.q, w.s, (int)w.N, (int)w.K, xp, sp, gp, group, M, yp, y_dtype, nullptr, st);
    });
    END_HANDLE_TH_ERRORS
}

// (x, act_group, xq, xscale, xgsum)
PyObject *quant_act_i8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int group;
    if (n != 5 || !small_int(a[1], &group)) return none();
    const at::Tensor *x = device_tensor(a[0], at::kBFloat16, 2);
    if (!x || x->size(0) > INT32_MAX || x->size(1) > INT32_MAX) return none();
    const int64_t M = x->size(0), groups = M * (x->size(1) / 32);
    const at::Tensor *const xq = device_room(a[2], at::kChar, M * x->size(1)),
                     *const xs = device_room(a[3], at::kFloat, group == 32 ? groups : M),
                     *const gs = device_room(a[4], at::kInt, groups);
    if (!xq || !xs || !gs) return none();
    const uint16_t *const xp = static_cast<const uint16_t *>(x->data_ptr());
    int8_t *const q = static_cast<int8_t *>(xq->data_ptr());
    float *const s = static_cast<float *>(xs->data_ptr());
    int32_t *const g = static_cast<int32_t *>(gs->data_ptr());
    void *const st = current_stream();
    return status_of([&] { return g_quant_act_i8(xp, (int)x->size(0), (int)x->size(1), group, q, s, g, st); });
    END_HANDLE_TH_ERRORS
}

// A microscaled matrix: codes [rows][K / 2], scale bytes [rows][K / 32].
struct Scaled {
    const uint8_t *q, *s;
    int64_t rows, K;
};
bool scaled(PyObject *codes, PyObject *scales, int device, Scaled *w) {
    const at::Tensor *q = device_tensor(codes, at::kByte, 2, device), *s = device_tensor(scales, at::kByte, 2, device);
    if (!q || !s) return false;
    w->rows = q->size(0);
    w->K = q->size(1) * 2;
    if (s->size(0) != w->rows || s->size(1) != w->K / 32 || w->rows > INT32_MAX || w->K > INT32_MAX) return false;
    w->q = static_cast<const uint8_t *>(q->data_ptr());
    w->s = static_cast<const uint8_t *>(s->data_ptr());
    return true;
}

// (x, q, scales)
PyObject *quant_mxfp4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 3) return none();
    const int here = device_of(a[0]);
    int dtype = NVQ_BF16;
    const at::Tensor *x = device_tensor(a[0], at::kBFloat16, 2, here);
    if (!x) {
        dtype = NVQ_F32;
        x = device_tensor(a[0], at::kFloat, 2, here);
    }
    if (!x || x->size(0) > INT32_MAX || x->size(1) > INT32_MAX) return none();
    const int64_t M = x->size(0), K = x->size(1);
    const at::Tensor *const q = device_room(a[1], at::kByte, M * (K / 2), here),
                     *const s = device_room(a[2], at::kByte, M * (K / 32), here);
    if (!q || !s) return none();
    const void *const xp = x->data_ptr();
    uint8_t *const qp = static_cast<uint8_t *>(q->data_ptr()), *const sp = static_cast<uint8_t *>(s->data_ptr());
    void *const st = current_stream();
    return status_of([&] { return g_quant_mxfp4(xp, dtype, M, K, qp, sp, st); });
    END_HANDLE_TH_ERRORS
}

// (q, scales, out)
PyObject *dequant_mxfp4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 3) return none();
    const int here = device_of(a[0]);
    Scaled w;
    if (!scaled(a[0], a[1], here, &w)) return none();
    const at::Tensor *const out = device_tensor(a[2], at::kBFloat16, 2, here);
    if (!out || out->size(0) != w.rows || out->size(1) != w.K) return none();
    uint16_t *const p = static_cast<uint16_t *>(out->data_ptr());
    void *const st = current_stream();
    return status_of([&] { return g_dequant_mxfp4(w.q, w.s, w.rows, w.K, p, st); });
    END_HANDLE_TH_ERRORS
}

// (qweight, scales, x, y)
PyObject *gemv_mxfp4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 4) return none();
    const int here = device_of(a[0]);
    Scaled w;
    int y_dtype;
    if (!scaled(a[0], a[1], here, &w)) return none();
    const at::Tensor *const x = device_tensor(a[2], at::kBFloat16, 2, here);
    if (!x || x->size(1) != w.K || x->size(0) > INT32_MAX) return none();
    const int M = (int)x->size(0);
    const at::Tensor *const y = output_tensor(a[3], M * w.rows, &y_dtype, here);
    if (!y) return none();
    const uint16_t *const xp = static_cast<const uint16_t *>(x->data_ptr());
    void *const yp = y->data_ptr(), *const st = current_stream();
    return status_of([&] { return g_gemv_mxfp4(w.q, w.s, (int)w.rows, (int)w.K, xp, M, yp, y_dtype, st); });
    END_HANDLE_TH_ERRORS
}

// (qweight, scales, xq, xscale, y)
PyObject *gemm_mxfp4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 5) return none();
    const int here = device_of(a[0]);
    Scaled w, x;
    int y_dtype;
    if (!scaled(a[0], a[1], here, &w) || !scaled(a[2], a[3], here, &x) || x.K != w.K) return none();
    const at::Tensor *const y = output_tensor(a[4], x.rows * w.rows, &y_dtype, here);
    if (!y) return none();
    void *const yp = y->data_ptr(), *const st = current_stream();
    return status_of([&] { return g_gemm_mxfp4(w.q, w.s, w.rows, w.K, x.q, x.s, x.rows, yp, y_dtype, st); });
    END_HANDLE_TH_ERRORS
}

// (x, router, top_k, renormalise, ids, weights, workspace)
PyObject *moe_route(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int top_k, renormalise;
    if (n != 7 || !small_int(a[2], &top_k) || !small_int(a[3], &renormalise) || top_k < 1) return none();
    const int here = device_of(a[0]);
    const at::Tensor *const x = device_tensor(a[0], at::kBFloat16, 2, here),
                     *const r = device_tensor(a[1], at::kBFloat16, 2, here);
    if (!x || !r || x->size(1) != r->size(1) || x->size(0) > INT32_MAX || r->size(0) > INT32_MAX || x->size(1) > INT32_MAX)
        return none();
    const int M = (int)x->size(0), E = (int)r->size(0), K = (int)x->size(1);
    const at::Tensor *const ids = device_room(a[4], at::kInt, (int64_t)M * top_k, here),
                     *const wt = device_room(a[5], at::kFloat, (int64_t)M * top_k, here),
                     *const ws = device_tensor(a[6], at::kByte, -1, here);
    if (!ids || !wt || !ws) return none();
    const uint16_t *const xp = static_cast<const uint16_t *>(x->data_ptr());
    const uint16_t *const rp = static_cast<const uint16_t *>(r->data_ptr());
    int32_t *const ip = static_cast<int32_t *>(ids->data_ptr());
    float *const wp = static_cast<float *>(wt->data_ptr());
    void *const sp = ws->data_ptr(), *const st = current_stream();
    const size_t bytes = (size_t)ws->numel();
    return status_of([&] { return g_moe_route(xp, rp, M, E, K, top_k, renormalise, ip, wp, sp, bytes, st); });
    END_HANDLE_TH_ERRORS
}

// (address of an nvq_experts, its K, its device, x, ids, weights, y, workspace)
PyObject *moe_experts(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int K, device, y_dtype;
    if (n != 8 || !PyLong_CheckExact(a[0]) || !small_int(a[1], &K) || !small_int(a[2], &device)) return none();
    const nvq_experts *const e = static_cast<const nvq_experts *>(PyLong_AsVoidPtr(a[0]));
    if (!e) {
        PyErr_Clear();
        return none();
    }
    const int here = device_of(a[3]);
    if (here != device) return none();
    const at::Tensor *const x = device_tensor(a[3], at::kBFloat16, 2, here),
                     *const ids = device_tensor(a[4], at::kInt, 2, here),
                     *const wt = device_tensor(a[5], at::kFloat, 2, here),
                     *const ws = device_tensor(a[7], at::kByte, -1, here);
    if (!x || !ids || !wt || !ws || x->size(1) != K || x->size(0) != ids->size(0) || wt->size(0) != ids->size(0) ||
        wt->size(1) != ids->size(1) || ids->size(0) > INT32_MAX || ids->size(1) > INT32_MAX)
        return none();
    const at::Tensor *const y = output_tensor(a[6], x->size(0) * K, &y_dtype, here);
    if (!y) return none();
    const uint16_t *const xp = static_cast<const uint16_t *>(x->data_ptr());
    const int32_t *const ip = static_cast<const int32_t *>(ids->data_ptr());
    const float *const wp = static_cast<const float *>(wt->data_ptr());
    const int M = (int)ids->size(0), top_k = (int)ids->size(1);
    void *const yp = y->data_ptr(), *const sp = ws->data_ptr(), *const st = current_stream();
    const size_t bytes = (size_t)ws->numel();
    return status_of([&] { return g_moe_experts(e, xp, ip, wp, M, top_k, yp, y_dtype, sp, bytes, st); });
    END_HANDLE_TH_ERRORS
}

// The handle of a call: the address of the struct that the library takes and the number of its device.  The device's
// number if that is the current one, else kNone.
template <typename T>
int handle_of(PyObject *address, PyObject *device, const T **h) {
    int d;
    if (!PyLong_CheckExact(address) || !small_int(device, &d)) return kNone;
    *h = static_cast<const T *>(PyLong_AsVoidPtr(address));
    if (!*h) {
        PyErr_Clear();
        return kNone;
    }
    return d == c10::hip::current_device() ? d : kNone;
}

// bf16 [T][heads][D] whose tokens may lie apart, on that device.
struct Rows {
    const uint16_t *p;
    int64_t T, heads, stride;
};
bool rows_of(PyObject *o, int64_t D, int device, Rows *r) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.scalar_type() != at::kBFloat16 || t.get_device() != device || t.dim() != 3) return false;
    r->T = t.size(0);
    r->heads = t.size(1);
    if (t.size(2) != D || t.stride(2) != 1 || (r->heads > 1 && t.stride(1) != D) || r->T > INT32_MAX || r->heads > INT32_MAX)
        return false;
    r->stride = r->T > 1 ? t.stride(0) : r->heads * D;
    r->p = static_cast<const uint16_t *>(t.data_ptr());
    return true;
}

// The address of a tensor as above, or null for None.
template <typename T>
bool room_or_none(PyObject *o, at::ScalarType type, int64_t n, int device, T **p) {
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *const t = device_room(o, type, n, device);
    if (t) *p = static_cast<T *>(t->data_ptr());
    return t != nullptr;
}

// The tokens of cache_append and cache_read.
struct Tokens {
    const int32_t *table, *positions, *sequences;
    int B, width, T;
};
bool tokens_of(PyObject *table, PyObject *positions, PyObject *sequences, int here, Tokens *k) {
    const at::Tensor *const t = device_tensor(table, at::kInt, 2, here), *const p = device_tensor(positions, at::kInt, 1, here);
    if (!t || !p || t->size(0) > INT32_MAX || t->size(1) > INT32_MAX || p->size(0) > INT32_MAX) return false;
    k->sequences = nullptr;
    if (sequences != Py_None) {
        const at::Tensor *const s = device_tensor(sequences, at::kInt, 1, here);
        if (!s || s->size(0) != p->size(0)) return false;
        k->sequences = static_cast<const int32_t *>(s->data_ptr());
    }
    k->table = static_cast<const int32_t *>(t->data_ptr());
    k->positions = static_cast<const int32_t *>(p->data_ptr());
    k->B = (int)t->size(0);
    k->width = (int)t->size(1);
    k->T = (int)p->size(0);
    return true;
}

// (address of an nvq_cache, its device, table, positions, k, v, q, cos_sin, interleaved, sequences, out); q, cos_sin,
// sequences, out: or None
PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const nvq_cache *c;
    if (n != 11) return none();
    const int here = handle_of(a[0], a[1], &c);
    Tokens at;
    Rows k, v, q = {nullptr, 0, 0, 0};
    int interleaved;
    if (here == kNone || !tokens_of(a[2], a[3], a[9], here, &at) || !rows_of(a[4], c->head_dim, here, &k) ||
        !rows_of(a[5], c->head_dim, here, &v) || !small_int(a[8], &interleaved))
        return none();
    if (k.T != at.T || v.T != at.T || k.heads != c->heads || v.heads != c->heads) return none();
    uint16_t *out = nullptr;
    if (a[6] != Py_None) {
        if (!rows_of(a[6], c->head_dim, here, &q) || q.T != at.T) return none();
        const at::Tensor *const o = device_room(a[10], at::kBFloat16, q.T * q.heads * c->head_dim, here);
        if (!o) return none();
        out = static_cast<uint16_t *>(o->data_ptr());
    } else if (a[10] != Py_None) {
        return none();
    }
    const float *cos_sin = nullptr;
    int angles = 0, rot = 0;
    if (a[7] != Py_None) {
        const at::Tensor *const t = device_tensor(a[7], at::kFloat, 2, here);
        if (!t || t->size(0) > INT32_MAX || t->size(1) > INT32_MAX) return none();
        cos_sin = static_cast<const float *>(t->data_ptr());
        angles = (int)t->size(0);
        rot = (int)t->size(1);
    }
    void *const st = current_stream();
    return status_of([&] {
        return g_cache_append(c, at.table, at.B, at.width, at.sequences, at.positions, at.T, q.p, q.stride, (int)q.heads, out, k.p,
                              k.stride, v.p, v.stride, cos_sin, angles, rot, interleaved, st);
    });
    END_HANDLE_TH_ERRORS
}

// (address of an nvq_cache, its device, table, positions, sequences or None, k, v)
PyObject *cache_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const nvq_cache *c;
    if (n != 7) return none();
    const int here = handle_of(a[0], a[1], &c);
    Tokens at;
    if (here == kNone || !tokens_of(a[2], a[3], a[4], here, &at)) return none();
    const int64_t values = (int64_t)at.T * c->heads * c->head_dim;
    const at::Tensor *const k = device_room(a[5], at::kBFloat16, values, here), *const v = device_room(a[6], at::kBFloat16, values, here);
    if (!k || !v) return none();
    uint16_t *const kp = static_cast<uint16_t *>(k->data_ptr()), *const vp = static_cast<uint16_t *>(v->data_ptr());
    void *const st = current_stream();
    return status_of([&] { return g_cache_read(c, at.table, at.B, at.width, at.sequences, at.positions, at.T, kp, vp, st); });
    END_HANDLE_TH_ERRORS
}

// (address of an nvq_cache, its device, q, table, lengths, scale, window, softcap, out, lse or None, workspace)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const nvq_cache *c;
    if (n != 11) return none();
    const int here = handle_of(a[0], a[1], &c);
    Rows q;
    int window, out_dtype;
    if (here == kNone || !rows_of(a[2], c->head_dim, here, &q) || !PyFloat_CheckExact(a[5]) || !small_int(a[6], &window) ||
        !PyFloat_CheckExact(a[7]))
        return none();
    const float scale = (float)PyFloat_AS_DOUBLE(a[5]), softcap = (float)PyFloat_AS_DOUBLE(a[7]);
    const at::Tensor *const table = device_tensor(a[3], at::kInt, 2, here), *const lengths = device_tensor(a[4], at::kInt, 1, here),
                     *const out = output_tensor(a[8], q.T * q.heads * c->head_dim, &out_dtype, here),
                     *const ws = device_tensor(a[10], at::kByte, -1, here);
    float *lse;
    if (!table || !lengths || !out || !ws || table->size(0) != q.T || lengths->size(0) != q.T || table->size(1) > INT32_MAX ||
        !room_or_none(a[9], at::kFloat, q.T * q.heads, here, &lse))
        return none();
    const int32_t *const tp = static_cast<const int32_t *>(table->data_ptr()), *const lp = static_cast<const int32_t *>(lengths->data_ptr());
    const int width = (int)table->size(1);
    void *const yp = out->data_ptr(), *const sp = ws->data_ptr(), *const st = current_stream();
    const size_t bytes = (size_t)ws->numel();
    return status_of([&] {
        return g_attention(c, q.p, q.stride, (int)q.heads, tp, (int)q.T, width, lp, scale, window, softcap, yp, out_dtype, lse, sp,
                           bytes, st);
    });
    END_HANDLE_TH_ERRORS
}

// (logits, u, temperature, top_k, top_p, min_p, out, workspace); the four in the middle: or None
PyObject *sample(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8) return none();
    const int here = device_of(a[0]);
    if (here == kNone) return none();
    const at::Tensor &l = THPVariable_Unpack(a[0]);
    if (l.dim() != 2 || (l.scalar_type() != at::kFloat && l.scalar_type() != at::kBFloat16) || (l.size(1) > 1 && l.stride(1) != 1) ||
        l.size(0) > INT32_MAX || l.size(1) > INT32_MAX)
        return none();
    const int M = (int)l.size(0), V = (int)l.size(1), dtype = l.scalar_type() == at::kFloat ? NVQ_F32 : NVQ_BF16;
    const int64_t ld = M > 1 ? l.stride(0) : V;
    const at::Tensor *const u = device_room(a[1], at::kFloat, M, here), *const ids = device_room(a[6], at::kInt, M, here),
                     *const ws = device_tensor(a[7], at::kByte, -1, here);
    float *temperature, *top_p, *min_p;
    int32_t *top_k;
    if (!u || !ids || !ws || !room_or_none(a[2], at::kFloat, M, here, &temperature) || !room_or_none(a[3], at::kInt, M, here, &top_k) ||
        !room_or_none(a[4], at::kFloat, M, here, &top_p) || !room_or_none(a[5], at::kFloat, M, here, &min_p))
        return none();
    const void *const lp = l.data_ptr();
    const float *const up = static_cast<const float *>(u->data_ptr());
    int32_t *const ip = static_cast<int32_t *>(ids->data_ptr());
    void *const sp = ws->data_ptr(), *const st = current_stream();
    const size_t bytes = (size_t)ws->numel();
    return status_of([&] { return g_sample(lp, dtype, ld, M, V, up, temperature, top_k, top_p, min_p, ip, sp, bytes, st); });
    END_HANDLE_TH_ERRORS
}

// (address of an nvq_adapters, its device, x, ids, y, out, workspace)
PyObject *adapters_add(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const nvq_adapters *g;
    if (n != 7) return none();
    const int here = handle_of(a[0], a[1], &g);
    if (here == kNone) return none();
    const at::Tensor *const x = device_tensor(a[2], at::kBFloat16, 2, here), *const ids = device_tensor(a[3], at::kInt, 1, here),
                     *const ws = device_tensor(a[6], at::kByte, -1, here);
    if (!x || !ids || !ws || x->size(1) != g->K || x->size(0) != ids->size(0) || x->size(0) > INT32_MAX) return none();
    const int M = (int)x->size(0);
    int dtype, out_dtype;
    const at::Tensor *const y = output_tensor(a[4], (int64_t)M * g->N, &dtype, here),
                     *const out = output_tensor(a[5], (int64_t)M * g->N, &out_dtype, here);
    if (!y || !out || dtype != out_dtype || y->dim() != 2 || y->size(0) != M || y->size(1) != g->N) return none();
    const uint16_t *const xp = static_cast<const uint16_t *>(x->data_ptr());
    const int32_t *const ip = static_cast<const int32_t *>(ids->data_ptr());
    const void *const yp = y->data_ptr();
    void *const op = out->data_ptr(), *const sp = ws->data_ptr(), *const st = current_stream();
    const size_t bytes = (size_t)ws->numel();
    return status_of([&] { return g_adapters_add(g, xp, ip, M, yp, op, dtype, sp, bytes, st); });
    END_HANDLE_TH_ERRORS
}

// The addresses of gemv_w4a16, gemv_w4a8, quant_act_i8, gemm_w4a16, quant_mxfp4, dequant_mxfp4, gemv_mxfp4, gemm_mxfp4,
// moe_route, moe_experts, cache_append, cache_read, attention, sample, adapters_add in the library.
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    constexpr int kCalls = 15;
    void *p[kCalls];
    if (n != kCalls) {
        PyErr_SetString(PyExc_TypeError, "fifteen addresses");
        return nullptr;
    }
    for (int i = 0; i < kCalls; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
            return nullptr;
        }
    }
    g_gemv_w4a16 = reinterpret_cast<decltype(g_gemv_w4a16)>(p[0]);
    g_gemv_w4a8 = reinterpret_cast<decltype(g_gemv_w4a8)>(p[1]);
    g_quant_act_i8 = reinterpret_cast<decltype(g_quant_act_i8)>(p[2]);
    g_gemm_w4a16 = reinterpret_cast<decltype(g_gemm_w4a16)>(p[3]);
    g_quant_mxfp4 = reinterpret_cast<decltype(g_quant_mxfp4)>(p[4]);
    g_dequant_mxfp4 = reinterpret_cast<decltype(g_dequant_mxfp4)>(p[5]);
    g_gemv_mxfp4 = reinterpret_cast<decltype(g_gemv_mxfp4)>(p[6]);
    g_gemm_mxfp4 = reinterpret_cast<decltype(g_gemm_mxfp4)>(p[7]);
    g_moe_route = reinterpret_cast<decltype(g_moe_route)>(p[8]);
    g_moe_experts = reinterpret_cast<decltype(g_moe_experts)>(p[9]);
    g_cache_append = reinterpret_cast<decltype(g_cache_append)>(p[10]);
    g_cache_read = reinterpret_cast<decltype(g_cache_read)>(p[11]);
    g_attention = reinterpret_cast<decltype(g_attention)>(p[12]);
    g_sample = reinterpret_cast<decltype(g_sample)>(p[13]);
    g_adapters_add = reinterpret_cast<decltype(g_adapters_add)>(p[14]);
    return none();
    END_HANDLE_TH_ERRORS
}

// The handle that the calls pass (for tests).
PyObject *stream_handle(PyObject *, PyObject *) {
    HANDLE_TH_ERRORS
    return PyLong_FromVoidPtr(current_stream());
    END_HANDLE_TH_ERRORS
}

#define NVQ_FAST(name_) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name_)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"bind", NVQ_FAST(bind)},
                         {"gemv_w4a16", NVQ_FAST(gemv_w4a16)},
                         {"gemv_w4a8", NVQ_FAST(gemv_w4a8)},
                         {"quant_act_i8", NVQ_FAST(quant_act_i8)},
                         {"gemm_w4a16", NVQ_FAST(gemm_w4a16)},
                         {"quant_mxfp4", NVQ_FAST(quant_mxfp4)},
                         {"dequant_mxfp4", NVQ_FAST(dequant_mxfp4)},
                         {"gemv_mxfp4", NVQ_FAST(gemv_mxfp4)},
                         {"gemm_mxfp4", NVQ_FAST(gemm_mxfp4)},
                         {"moe_route", NVQ_FAST(moe_route)},
                         {"moe_experts", NVQ_FAST(moe_experts)},
                         {"cache_append", NVQ_FAST(cache_append)},
                         {"cache_read", NVQ_FAST(cache_read)},
                         {"attention", NVQ_FAST(attention)},
                         {"sample", NVQ_FAST(sample)},
                         {"adapters_add", NVQ_FAST(adapters_add)},
                         {"stream_handle", stream_handle, METH_NOARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    PyObject *const m = PyModule_Create(&module);
    // (the caller leaves a module alone that was built for another torch)
    if (m && PyModule_AddStringConstant(m, "torch_version", NVQ_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
