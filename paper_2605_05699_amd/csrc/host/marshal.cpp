// marshal.cpp -- the calls of binding.py that programs make step after step, marshalled in native code (a CPython extension; host
// only, no HIP call of its own).
//
// What bounds it: a small launch takes 2.0-2.5 us of the host, and ctypes and the checks of the tensors in Python cost as much again
// (1.0 us a call of seven arguments, 0.65 us a tensor).  Host time of a call, us, through ctypes -> here: a batched write of 2 plans
// 4.2 -> 3.0, of 64 4.3 -> 3.4; one plan's write 4.9 -> 3.1, read 4.7 -> 3.0; scores 6.1 -> 3.2; decode attention (two launches)
// 9.4 -> 6.0; srft_cache_append by way of lib() 0.3 less.
//
// A function here makes the call where everything is as binding.py wants it (plain tensors of the right type on the device, no
// stream named) and returns the status; it returns None where anything is not, before the call, and binding.py goes its own way,
// which raises what there is to raise.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>

#include "srft_kv.h"

namespace {

// ---- the C entry points, bound by binding.lib() when it loads the library; their types are the header's
struct {
    decltype(&srft_kv_quantize) quantize;
    decltype(&srft_kv_dequantize) dequantize;
    decltype(&srft_kv_quantize_batched) quantize_batched;
    decltype(&srft_kv_dequantize_batched) dequantize_batched;
    decltype(&srft_kv_scores) scores;
    decltype(&srft_kv_decode_attention) attention;
    decltype(&srft_kv_channel_absmax) absmax;
    decltype(&srft_cache_append) append;
    decltype(&srft_scores_workspace_bytes) scores_bytes;
    decltype(&srft_decode_attention_workspace_bytes) attention_bytes;
    decltype(&srft_plan_d) plan_d;
    decltype(&srft_rotary) rotary;
    decltype(&srft_pool_append) pool_append;
    decltype(&srft_pool_attention) pool_attention;
    decltype(&srft_pool_copy) pool_copy;
    decltype(&srft_pool_append_workspace_bytes) pool_append_bytes;
    decltype(&srft_pool_attention_workspace_bytes) pool_attention_bytes;
    decltype(&srft_norm_rotary) norm_rotary;
    decltype(&srft_norm_rotary_backward) norm_backward;
    decltype(&srft_norm_rotary_backward_workspace_bytes) norm_backward_bytes;
    decltype(&srft_pool_attention_sliding) pool_sliding;
    decltype(&srft_pool_attention_sliding_workspace_bytes) pool_sliding_bytes;
    decltype(&srft_pool_attention_shared) pool_shared;
    decltype(&srft_pool_attention_shared_workspace_bytes) pool_shared_bytes;
    bool bound;
} g;

// ---- arguments
template <class T>
bool handle_of(PyObject* o, T** p) {                         // a plan: the address as an int
    if (!PyLong_CheckExact(o)) return false;
    *p = (T*)PyLong_AsVoidPtr(o);
    if (*p || !PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}
// a plain contiguous tensor of this type on the device
const at::Tensor* tensor_of(PyObject* o, at::ScalarType type) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.scalar_type() == type && t.layout() == at::kStrided && t.unsafeGetTensorImpl()->has_storage() &&
                   t.is_contiguous()
               ? &t
               : nullptr;
}
PyTypeObject *cell_type, *array_type;                        // ctypes.c_void_p and ctypes.Array, with the entry points
bool address_of(PyObject* o, void** p) {                     // of a ctypes array or cell
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return false;
    }
    *p = b.buf;
    PyBuffer_Release(&b);
    return true;
}
uint8_t* codes_of(const at::Tensor* t) { return static_cast<uint8_t*>(t->data_ptr()); }
float* floats_of(const at::Tensor* t) { return static_cast<float*>(t->data_ptr()); }
void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// Runs `body` (true: the call was made, its status in *rc), turning what it throws into "not made".
template <class F>
PyObject* made(F body) {
    int rc = 0;
    bool done = false;
    try {
        done = g.bound && body(&rc);
    } catch (...) {
    }
    if (done) return PyLong_FromLong(rc);
    PyErr_Clear();                                           // (an int past 64 bits)
    Py_RETURN_NONE;
}
template <class F>
int without_gil(F call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}
int64_t bytes_of(const at::Tensor& t) { return t.numel() * (int64_t)t.element_size(); }

// quantize(plan, x, codes, scales)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_plan_t* plan;
        if (n != 4 || !handle_of(a[0], &plan)) return false;
        const at::Tensor *x = tensor_of(a[1], at::kHalf), *c = tensor_of(a[2], at::kByte), *s = tensor_of(a[3], at::kFloat);
        if (!x || !c || !s || x->dim() < 1) return false;
        void *const xp = x->data_ptr(), *const st = current_stream();
        uint8_t* const cp = codes_of(c);
        float* const sp = floats_of(s);
        const int64_t count = x->size(0);
        *rc = without_gil([&] { return g.quantize(plan, xp, count, cp, sp, st); });
        return true;
    });
}
// dequantize(plan, codes, scales, out)
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_plan_t* plan;
        if (n != 4 || !handle_of(a[0], &plan)) return false;
        const at::Tensor *c = tensor_of(a[1], at::kByte), *s = tensor_of(a[2], at::kFloat), *o = tensor_of(a[3], at::kHalf);
        if (!c || !s || !o || c->dim() < 1) return false;
        const uint8_t* const cp = codes_of(c);
        const float* const sp = floats_of(s);
        void *const op = o->data_ptr(), *const st = current_stream();
        const int64_t count = c->size(0);
        *rc = without_gil([&] { return g.dequantize(plan, cp, sp, count, op, st); });
        return true;
    });
}
// the arrays of a BatchTable
PyObject *s_plans, *s_big, *s_codes, *s_scales, *s_n_vec, *s_count;
PyObject* batched(PyObject* table, bool write) {
    PyObject* held[6] = {};                                  // (the arrays stay for the call, whatever happens to the table meanwhile)
    PyObject* const r = made([&](int* rc) {
        PyObject* const names[6] = {s_plans, s_big, s_codes, s_scales, s_n_vec, s_count};
        void* p[5];
        for (int i = 0; i < 6; ++i)
            if (!(held[i] = PyObject_GetAttr(table, names[i])) || (i < 5 && (!PyObject_TypeCheck(held[i], array_type) || !address_of(held[i], &p[i])))) {
                PyErr_Clear();
                return false;
            }
        int overflow;
        const long count = PyLong_CheckExact(held[5]) ? PyLong_AsLongAndOverflow(held[5], &overflow) : -1;
        if (count < 0 || count > INT32_MAX) return false;
        void* const st = current_stream();
        *rc = without_gil([&] {
            const auto plans = (const srft_plan_t* const*)p[0];
            const auto n_vec = (const int64_t*)p[4];
            return write ? g.quantize_batched(plans, (const void* const*)p[1], n_vec, (uint8_t* const*)p[2], (float* const*)p[3], (int)count, st)
                         : g.dequantize_batched(plans, (const uint8_t* const*)p[2], (const float* const*)p[3], n_vec, (void* const*)p[1], (int)count, st);
        });
        return true;
    });
    for (PyObject* o : held) Py_XDECREF(o);
    return r;
}
PyObject* quantize_batched(PyObject*, PyObject* table) { return batched(table, true); }
PyObject* dequantize_batched(PyObject*, PyObject* table) { return batched(table, false); }

// scores(plan, q, codes, scales, scores, workspace)
PyObject* scores(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_plan_t* plan;
        if (n != 6 || !handle_of(a[0], &plan) || !plan || !THPVariable_CheckExact(a[5])) return false;
        const at::Tensor *q = tensor_of(a[1], at::kHalf), *c = tensor_of(a[2], at::kByte), *s = tensor_of(a[3], at::kFloat),
                         *o = tensor_of(a[4], at::kFloat), *w = tensor_of(a[5], THPVariable_Unpack(a[5]).scalar_type());
        if (!q || !c || !s || !o || !w || q->dim() < 1 || c->dim() < 1 || o->dim() != 2 || o->size(0) != q->size(0) || o->size(1) != c->size(0) ||
            bytes_of(*w) < g.scores_bytes(plan))
            return false;
        const int64_t n_q = q->size(0), keys = c->size(0);
        const uint8_t* const cp = codes_of(c);
        const float* const sp = floats_of(s);
        float* const op = floats_of(o);
        void *const qp = q->data_ptr(), *const wp = w->data_ptr(), *const st = current_stream();
        if (n_q > INT32_MAX) return false;
        *rc = without_gil([&] { return g.scores(plan, qp, (int)n_q, cp, sp, keys, op, wp, st); });
        return true;
    });
}
// attention(plan_k, plan_v, q, k_codes, k_scales, v_codes, v_scales, softmax_scale, out, workspace)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_plan_t *pk, *pv;
        if (n != 10 || !handle_of(a[0], &pk) || !handle_of(a[1], &pv) || !pk || !pv || !PyFloat_CheckExact(a[7]) || !THPVariable_CheckExact(a[9])) return false;
        const at::Tensor *q = tensor_of(a[2], at::kHalf), *kc = tensor_of(a[3], at::kByte), *ks = tensor_of(a[4], at::kFloat), *vc = tensor_of(a[5], at::kByte),
                         *vs = tensor_of(a[6], at::kFloat), *o = tensor_of(a[8], at::kFloat), *w = tensor_of(a[9], THPVariable_Unpack(a[9]).scalar_type());
        if (!q || !kc || !ks || !vc || !vs || !o || !w || q->dim() < 1 || kc->dim() < 1 || vc->dim() < 1 || vc->size(0) != kc->size(0)) return false;
        const int64_t n_q = q->size(0), keys = kc->size(0);
        if (n_q > INT32_MAX || bytes_of(*w) < g.attention_bytes(pk, pv, (int)n_q, keys)) return false;
        const float scale = (float)PyFloat_AS_DOUBLE(a[7]);
        const uint8_t *const kcp = codes_of(kc), *const vcp = codes_of(vc);
        const float *const ksp = floats_of(ks), *const vsp = floats_of(vs);
        float* const op = floats_of(o);
        void *const qp = q->data_ptr(), *const wp = w->data_ptr(), *const st = current_stream();
        *rc = without_gil([&] { return g.attention(pk, pv, qp, (int)n_q, kcp, ksp, vcp, vsp, keys, scale, op, wp, st); });
        return true;
    });
}
// absmax(plan, x, amax)
PyObject* absmax(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_plan_t* plan;
        if (n != 3 || !handle_of(a[0], &plan) || !plan) return false;
        const at::Tensor *x = tensor_of(a[1], at::kHalf), *m = tensor_of(a[2], at::kFloat);
        if (!x || !m || x->dim() < 1 || m->numel() != g.plan_d(plan)) return false;
        const int64_t count = x->size(0);
        void *const xp = x->data_ptr(), *const st = current_stream();
        float* const mp = floats_of(m);
        *rc = without_gil([&] { return g.absmax(plan, xp, count, mp, st); });
        return true;
    });
}

// ---- rotary positions and the paged cache
// a plain tensor [tokens, heads, channels] on the device whose channels lie next to each other
const at::Tensor* rows_of(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.unsafeGetTensorImpl()->has_storage() && t.dim() == 3 &&
                   (t.size(2) <= 1 || t.stride(2) == 1 || t.numel() == 0)
               ? &t
               : nullptr;
}
// the stride of its tokens (0) or heads (1); 0 where it leads nowhere
int64_t step_of(const at::Tensor& t, int i) { return t.size(i) > 1 && t.numel() > 0 ? t.stride(i) : 0; }
int type_of(const at::Tensor& t) {                           // srft_dtype, or -1
    return t.scalar_type() == at::kFloat ? SRFT_F32 : t.scalar_type() == at::kHalf ? SRFT_F16 : t.scalar_type() == at::kBFloat16 ? SRFT_BF16 : -1;
}
// a plain contiguous tensor of any type
const at::Tensor* space_of(PyObject* o) { return THPVariable_CheckExact(o) ? tensor_of(o, THPVariable_Unpack(o).scalar_type()) : nullptr; }

// rotary(items, positions, freq, layout, factor, inverse)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        if (n != 6 || !PyList_CheckExact(a[0]) || !PyLong_CheckExact(a[3]) || !PyFloat_CheckExact(a[4]) || !PyBool_Check(a[5])) return false;
        const int items = (int)PyList_GET_SIZE(a[0]);
        if (items < 1 || items > SRFT_ROTARY_MAX) return false;
        const at::Tensor *pos = tensor_of(a[1], at::kInt), *freq = tensor_of(a[2], at::kDouble);
        if (!pos || !freq || pos->dim() != 1 || freq->dim() != 1) return false;
        srft_rotary_rows rows[SRFT_ROTARY_MAX] = {};
        const int64_t tokens = pos->size(0);
        int64_t d = 0;
        for (int i = 0; i < items; ++i) {
            PyObject* const pair = PyList_GET_ITEM(a[0], i);
            if (!PyTuple_CheckExact(pair) || PyTuple_GET_SIZE(pair) != 2) return false;
            const at::Tensor *x = rows_of(PyTuple_GET_ITEM(pair, 0)), *y = rows_of(PyTuple_GET_ITEM(pair, 1));
            if (!x || !y || !x->sizes().equals(y->sizes()) || x->size(0) != tokens || type_of(*x) < 0 || type_of(*y) < 0) return false;
            if (i == 0) d = x->size(2);
            if (x->size(2) != d || d > INT32_MAX || x->size(1) > INT32_MAX) return false;
            rows[i].in_dev = x->data_ptr(), rows[i].in_token = step_of(*x, 0), rows[i].in_head = step_of(*x, 1);
            rows[i].out_dev = y->data_ptr(), rows[i].out_token = step_of(*y, 0), rows[i].out_head = step_of(*y, 1);
            rows[i].n_heads = (int32_t)x->size(1), rows[i].in_type = type_of(*x), rows[i].out_type = type_of(*y);
        }
        const long layout = PyLong_AsLong(a[3]);
        const double factor = PyFloat_AS_DOUBLE(a[4]);
        const bool inverse = a[5] == Py_True;
        const int32_t* const pp = static_cast<const int32_t*>(pos->data_ptr());
        const double* const fp = static_cast<const double*>(freq->data_ptr());
        if (freq->size(0) > INT32_MAX / 2) return false;
        const int rot = 2 * (int)freq->size(0);
        void* const st = current_stream();
        *rc = without_gil([&] { return g.rotary(rows, items, tokens, (int)d, rot, (int)layout, pp, fp, factor, inverse, st); });
        return true;
    });
}
// pool_append(pool, sequences, heads, d, k, v, workspace)
PyObject* pool_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_pool_t* pool;
        const srft_paged_seqs* seqs;
        if (n != 7 || !handle_of(a[0], &pool) || !handle_of(a[1], &seqs) || !pool || !seqs || !PyLong_CheckExact(a[2]) || !PyLong_CheckExact(a[3])) return false;
        const at::Tensor *k = rows_of(a[4]), *v = rows_of(a[5]), *w = space_of(a[6]);
        if (!k || !v || !w || k->scalar_type() != at::kHalf || v->scalar_type() != at::kHalf || !k->sizes().equals(v->sizes()) ||
            k->size(1) != PyLong_AsLong(a[2]) || k->size(2) != PyLong_AsLong(a[3]))
            return false;
        const int64_t tokens = k->size(0), need = g.pool_append_bytes(pool, seqs, tokens);
        if (need < 0 || bytes_of(*w) < need) return false;
        void *const kp = k->data_ptr(), *const vp = v->data_ptr(), *const wp = w->data_ptr(), *const st = current_stream();
        const int64_t kt = step_of(*k, 0), kh = step_of(*k, 1), vt = step_of(*v, 0), vh = step_of(*v, 1);
        *rc = without_gil([&] { return g.pool_append(pool, seqs, kp, vp, tokens, kt, kh, vt, vh, wp, st); });
        return true;
    });
}
// pool_attention(pool, sequences, d, q, softmax_scale, out, workspace)
PyObject* pool_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_pool_t* pool;
        const srft_paged_seqs* seqs;
        if (n != 7 || !handle_of(a[0], &pool) || !handle_of(a[1], &seqs) || !pool || !seqs || !PyLong_CheckExact(a[2]) || !PyFloat_CheckExact(a[4])) return false;
        const at::Tensor *q = rows_of(a[3]), *o = rows_of(a[5]), *w = space_of(a[6]);
        if (!q || !o || !w || type_of(*q) <= SRFT_F32 || o->scalar_type() != q->scalar_type() || !q->sizes().equals(o->sizes()) ||
            q->size(2) != PyLong_AsLong(a[2]) || q->size(1) > INT32_MAX)
            return false;
        const int64_t tokens = q->size(0), need = g.pool_attention_bytes(pool, seqs, tokens, (int)q->size(1));
        if (need < 0 || bytes_of(*w) < need) return false;
        void *const qp = q->data_ptr(), *const op = o->data_ptr(), *const wp = w->data_ptr(), *const st = current_stream();
        const int64_t qt = step_of(*q, 0), qh = step_of(*q, 1), ot = step_of(*o, 0), oh = step_of(*o, 1);
        const int heads = (int)q->size(1), type = type_of(*q);
        const float scale = (float)PyFloat_AS_DOUBLE(a[4]);
        *rc = without_gil([&] { return g.pool_attention(pool, seqs, qp, type, tokens, heads, qt, qh, scale, op, ot, oh, wp, st); });
        return true;
    });
}
// positions [tokens] and freq of a call on rows of tokens
struct angles {
    const int32_t* positions;
    const double* freq;
    int64_t tokens;
    int rot;
    bool of(PyObject* p, PyObject* f) {
        const at::Tensor *pos = tensor_of(p, at::kInt), *fr = tensor_of(f, at::kDouble);
        if (!pos || !fr || pos->dim() != 1 || fr->dim() != 1 || fr->size(0) > INT32_MAX / 2) return false;
        positions = static_cast<const int32_t*>(pos->data_ptr()), freq = static_cast<const double*>(fr->data_ptr());
        tokens = pos->size(0), rot = 2 * (int)fr->size(0);
        return true;
    }
};
// weights [d] of a tensor's channels, or None
bool weight_of(PyObject* o, int64_t d, const void** p, int32_t* type) {
    *p = nullptr, *type = 0;
    if (o == Py_None) return true;
    const at::Tensor* const w = space_of(o);
    if (!w || type_of(*w) < 0 || w->dim() != 1 || w->size(0) != d) return false;
    *p = w->data_ptr(), *type = type_of(*w);
    return true;
}
// norm_rotary(items (x, weight, out), positions, freq, layout, factor, eps)
PyObject* norm_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        angles t;
        if (n != 6 || !PyList_CheckExact(a[0]) || !t.of(a[1], a[2]) || !PyLong_CheckExact(a[3]) || !PyFloat_CheckExact(a[4]) || !PyFloat_CheckExact(a[5])) return false;
        const int items = (int)PyList_GET_SIZE(a[0]);
        if (items < 1 || items > SRFT_ROTARY_MAX) return false;
        srft_norm_rows rows[SRFT_ROTARY_MAX] = {};
        int64_t d = 0;
        for (int i = 0; i < items; ++i) {
            PyObject* const item = PyList_GET_ITEM(a[0], i);
            if (!PyTuple_CheckExact(item) || PyTuple_GET_SIZE(item) != 3) return false;
            const at::Tensor *x = rows_of(PyTuple_GET_ITEM(item, 0)), *y = rows_of(PyTuple_GET_ITEM(item, 2));
            if (!x || !y || !x->sizes().equals(y->sizes()) || x->size(0) != t.tokens || type_of(*x) < 0 || type_of(*y) < 0) return false;
            if (i == 0) d = x->size(2);
            if (x->size(2) != d || d > INT32_MAX || x->size(1) > INT32_MAX || !weight_of(PyTuple_GET_ITEM(item, 1), d, &rows[i].weight_dev, &rows[i].weight_type)) return false;
            srft_rotary_rows& r = rows[i].x;
            r.in_dev = x->data_ptr(), r.in_token = step_of(*x, 0), r.in_head = step_of(*x, 1);
            r.out_dev = y->data_ptr(), r.out_token = step_of(*y, 0), r.out_head = step_of(*y, 1);
            r.n_heads = (int32_t)x->size(1), r.in_type = type_of(*x), r.out_type = type_of(*y);
        }
        const int layout = (int)PyLong_AsLong(a[3]);
        const double factor = PyFloat_AS_DOUBLE(a[4]), eps = PyFloat_AS_DOUBLE(a[5]);
        void* const st = current_stream();
        *rc = without_gil([&] { return g.norm_rotary(rows, items, t.tokens, (int)d, t.rot, layout, t.positions, t.freq, factor, eps, st); });
        return true;
    });
}
// norm_backward(items (dy, x, weight, dx, dweight), positions, freq, layout, factor, eps, workspace)
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        angles t;
        if (n != 7 || !PyList_CheckExact(a[0]) || !t.of(a[1], a[2]) || !PyLong_CheckExact(a[3]) || !PyFloat_CheckExact(a[4]) || !PyFloat_CheckExact(a[5])) return false;
        const int items = (int)PyList_GET_SIZE(a[0]);
        if (items < 1 || items > SRFT_ROTARY_MAX) return false;
        srft_norm_grad_rows rows[SRFT_ROTARY_MAX] = {};
        int64_t d = 0;
        for (int i = 0; i < items; ++i) {
            PyObject* const item = PyList_GET_ITEM(a[0], i);
            if (!PyTuple_CheckExact(item) || PyTuple_GET_SIZE(item) != 5) return false;
            const at::Tensor *dy = rows_of(PyTuple_GET_ITEM(item, 0)), *x = rows_of(PyTuple_GET_ITEM(item, 1)), *dx = rows_of(PyTuple_GET_ITEM(item, 3));
            if (!dy || !x || !dx || !x->sizes().equals(dy->sizes()) || !x->sizes().equals(dx->sizes()) || x->size(0) != t.tokens || type_of(*x) < 0 ||
                type_of(*dy) < 0 || dx->scalar_type() != x->scalar_type())
                return false;
            if (i == 0) d = x->size(2);
            srft_norm_grad_rows& r = rows[i];
            if (x->size(2) != d || d > INT32_MAX || x->size(1) > INT32_MAX || !weight_of(PyTuple_GET_ITEM(item, 2), d, &r.weight_dev, &r.weight_type)) return false;
            if (PyTuple_GET_ITEM(item, 4) != Py_None) {
                const at::Tensor* const w = tensor_of(PyTuple_GET_ITEM(item, 4), at::kFloat);
                if (!w || w->dim() != 1 || w->size(0) != d) return false;
                r.dweight_dev = floats_of(w);
            }
            r.dy_dev = dy->data_ptr(), r.dy_token = step_of(*dy, 0), r.dy_head = step_of(*dy, 1);
            r.x_dev = x->data_ptr(), r.x_token = step_of(*x, 0), r.x_head = step_of(*x, 1);
            r.dx_dev = dx->data_ptr(), r.dx_token = step_of(*dx, 0), r.dx_head = step_of(*dx, 1);
            r.n_heads = (int32_t)x->size(1), r.dy_type = type_of(*dy), r.x_type = type_of(*x);
        }
        void* wp = nullptr;
        if (a[6] != Py_None) {
            const at::Tensor* const w = space_of(a[6]);
            const int64_t need = g.norm_backward_bytes(items, (int)d);
            if (!w || need < 0 || bytes_of(*w) < need) return false;
            wp = w->data_ptr();
        }
        const int layout = (int)PyLong_AsLong(a[3]);
        const double factor = PyFloat_AS_DOUBLE(a[4]), eps = PyFloat_AS_DOUBLE(a[5]);
        void* const st = current_stream();
        *rc = without_gil([&] { return g.norm_backward(rows, items, t.tokens, (int)d, t.rot, layout, t.positions, t.freq, factor, eps, wp, st); });
        return true;
    });
}
// the tensors of a call of attention over pages
struct attended {
    void *q, *out, *space, *stream;
    int64_t tokens, qt, qh, ot, oh, bytes;
    int heads, type;
    bool of(PyObject* d, PyObject* q_, PyObject* out_, PyObject* space_) {
        const at::Tensor *x = rows_of(q_), *o = rows_of(out_), *w = space_of(space_);
        if (!x || !o || !w || !PyLong_CheckExact(d) || type_of(*x) <= SRFT_F32 || o->scalar_type() != x->scalar_type() || !x->sizes().equals(o->sizes()) ||
            x->size(2) != PyLong_AsLong(d) || x->size(1) > INT32_MAX)
            return false;
        q = x->data_ptr(), out = o->data_ptr(), space = w->data_ptr(), stream = current_stream();
        tokens = x->size(0), qt = step_of(*x, 0), qh = step_of(*x, 1), ot = step_of(*o, 0), oh = step_of(*o, 1), bytes = bytes_of(*w);
        heads = (int)x->size(1), type = type_of(*x);
        return true;
    }
};
// pool_sliding(pool, sequences, d, q, softmax_scale, recent, sinks, out, workspace)
PyObject* pool_sliding(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_pool_t* pool;
        const srft_paged_seqs* seqs;
        attended t;
        int overflow = 0, more = 0;
        if (n != 9 || !handle_of(a[0], &pool) || !handle_of(a[1], &seqs) || !pool || !seqs || !PyFloat_CheckExact(a[4]) || !PyLong_CheckExact(a[5]) || !PyLong_CheckExact(a[6]) ||
            !t.of(a[2], a[3], a[7], a[8]))
            return false;
        const int64_t recent = PyLong_AsLongLongAndOverflow(a[5], &overflow), sinks = PyLong_AsLongLongAndOverflow(a[6], &more);
        const int64_t need = g.pool_sliding_bytes(pool, seqs, t.tokens, t.heads);
        if (overflow || more || need < 0 || t.bytes < need) return false;
        const float scale = (float)PyFloat_AS_DOUBLE(a[4]);
        *rc = without_gil([&] { return g.pool_sliding(pool, seqs, t.q, t.type, t.tokens, t.heads, t.qt, t.qh, scale, recent, sinks, t.out, t.ot, t.oh, t.space, t.stream); });
        return true;
    });
}
// pool_shared(pool, sequences, prefixes, d, q, softmax_scale, out, workspace)
PyObject* pool_shared(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_pool_t* pool;
        const srft_paged_seqs* seqs;
        const srft_shared_prefixes* prefixes;
        attended t;
        if (n != 8 || !handle_of(a[0], &pool) || !handle_of(a[1], &seqs) || !handle_of(a[2], &prefixes) || !pool || !seqs || !prefixes || !PyFloat_CheckExact(a[5]) ||
            !t.of(a[3], a[4], a[6], a[7]))
            return false;
        const int64_t need = g.pool_shared_bytes(pool, seqs, prefixes, t.tokens, t.heads);
        if (need < 0 || t.bytes < need) return false;
        const float scale = (float)PyFloat_AS_DOUBLE(a[5]);
        *rc = without_gil([&] { return g.pool_shared(pool, seqs, prefixes, t.q, t.type, t.tokens, t.heads, t.qt, t.qh, scale, t.out, t.ot, t.oh, t.space, t.stream); });
        return true;
    });
}
// pool_copy(handles, count, pages, windows)
PyObject* pool_copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return made([&](int* rc) {
        const srft_pool_t* const* pools;
        if (n != 4 || !handle_of(a[0], &pools) || !PyLong_CheckExact(a[1])) return false;
        const at::Tensor *p = tensor_of(a[2], at::kInt), *w = tensor_of(a[3], at::kInt);
        if (!p || !w || p->dim() != 2 || w->dim() != 2 || p->size(1) != 2 || w->size(1) != 2) return false;
        const int32_t *const pp = static_cast<const int32_t*>(p->data_ptr()), *const wp = static_cast<const int32_t*>(w->data_ptr());
        const int64_t pages = p->size(0), windows = w->size(0);
        const int count = (int)PyLong_AsLong(a[1]);
        void* const st = current_stream();
        *rc = without_gil([&] { return g.pool_copy(pools, count, pp, pages, wp, windows, st); });
        return true;
    });
}

// ---- lib().srft_cache_append, a ctypes function of a type of its own whose calls come here first: those with other arguments than
// None, ints, c_void_p and arrays of them go on to ctypes.  (As the type's slot: by way of a __call__ in Python's sight a call took 0.03 us
// more.)
bool pointer_of(PyObject* o, void** p) {
    if (o == Py_None) {
        *p = nullptr;
        return true;
    }
    if (handle_of(o, p)) return true;
    const bool cell = Py_TYPE(o) == cell_type;
    if (!cell && !PyObject_TypeCheck(o, array_type)) return false;
    void* at;
    if (!address_of(o, &at)) return false;
    if (cell) std::memcpy(p, at, sizeof(*p));
    else *p = at;
    return true;
}
PyObject* append_call(PyObject* self, PyObject* args, PyObject* names) {
    void *cache, *fresh, *st;
    if (PyTuple_GET_SIZE(args) == 4 && !names && g.bound) {
        PyObject* const* a = &PyTuple_GET_ITEM(args, 0);
        if (pointer_of(a[0], &cache) && pointer_of(a[1], &fresh) && PyLong_CheckExact(a[2]) && pointer_of(a[3], &st)) {
            int overflow;
            const long t = PyLong_AsLongAndOverflow(a[2], &overflow);
            if (!overflow && t == (int)t)
                return PyLong_FromLong(without_gil([&] { return g.append((srft_cache_t*)cache, (const void* const*)fresh, (int)t, st); }));
        }
    }
    PyTypeObject* base = Py_TYPE(self);
    while (base->tp_call == append_call) base = base->tp_base;
    return base->tp_call(self, args, names);
}
// append(type, native): calls of the type's objects come here, or go to ctypes (again)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 2 || !PyType_Check(a[0]) || !(((PyTypeObject*)a[0])->tp_flags & Py_TPFLAGS_HEAPTYPE)) {
        PyErr_SetString(PyExc_TypeError, "append(type, native)");
        return nullptr;
    }
    PyTypeObject* const type = (PyTypeObject*)a[0];
    type->tp_call = a[1] == Py_True ? append_call : type->tp_base->tp_call;
    PyType_Modified(type);
    Py_RETURN_NONE;
}

// bind(addresses, c_void_p, Array): of the entry points, in the order of the struct above.  True: they are the ones called here; False: those
// of another library are, which came first.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr int kCount = 24;
    void* p[kCount];
    if (n != kCount + 2 || !PyType_Check(a[kCount]) || !PyType_Check(a[kCount + 1])) {
        PyErr_SetString(PyExc_TypeError, "bind takes the addresses of 24 entry points, c_void_p and Array");
        return nullptr;
    }
    for (int i = 0; i < kCount; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no entry point");
            return nullptr;
        }
    }
    if (g.bound) return PyBool_FromLong(std::memcmp(&g, p, sizeof(p)) == 0);
    cell_type = (PyTypeObject*)Py_NewRef(a[kCount]);
    array_type = (PyTypeObject*)Py_NewRef(a[kCount + 1]);
    std::memcpy(&g, p, sizeof(p));
    g.bound = true;
    Py_RETURN_TRUE;
}
static_assert(offsetof(decltype(g), bound) == 24 * sizeof(void*), "bind fills the pointers in order");

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(quantize), FAST(dequantize), FAST(scores), FAST(attention), FAST(absmax), FAST(append), FAST(bind),
                         FAST(rotary), FAST(pool_append), FAST(pool_attention), FAST(pool_copy), FAST(norm_rotary), FAST(norm_backward), FAST(pool_sliding), FAST(pool_shared),
                         {"quantize_batched", quantize_batched, METH_O, nullptr},
                         {"dequantize_batched", dequantize_batched, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
    struct { PyObject** at; const char* name; } const names[] = {{&s_plans, "plans"}, {&s_big, "big"}, {&s_codes, "codes"}, {&s_scales, "scales"}, {&s_n_vec, "n_vec"}, {&s_count, "count"}};
    for (const auto& e : names)
        if (!(*e.at = PyUnicode_InternFromString(e.name))) return nullptr;
    return PyModule_Create(&module);
}
