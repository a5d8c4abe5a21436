// Native marshalling of the cache's operators from Python: checks of tensor
// metadata, the outputs, the current stream, and the call into libbf1.so.  A call
// that takes 2 to 6 us on the device spends 4 in the launch and, from Python code, 5
// to 11 in these steps; here 0.4 to 3 (the binding has the figures).
//
// Every function takes what its Python entry point takes, positionally, and returns
// its result, a status of the library as an int, or None where something is not
// exactly what the usual call has (another type, shape or device, a subclass, an
// argument out of range).  On None the Python code goes through its own checks, which
// name what is wrong or serve the call.
#include <ATen/ops/empty.h>
#include <ATen/ops/unsafe_split_with_sizes.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "../../include/bf1.h"

namespace {

using at::IntArrayRef;
using at::ScalarType;
using at::Tensor;

constexpr ScalarType BF16 = at::kBFloat16, F32 = at::kFloat, F64 = at::kDouble, I32 = at::kInt, I64 = at::kLong;

// The strided tensor with memory on `device` behind a plain torch.Tensor; null for
// anything else.  device -1: the current one.
const Tensor* tensor(PyObject* o, int dims, int* device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.dim() != dims || t.is_neg())
        return nullptr;
    if (*device < 0) *device = c10::hip::current_device();
    return t.get_device() == *device ? &t : nullptr;
}

// The same, contiguous, of type `type` and sizes `sizes`.
const Tensor* exact(PyObject* o, ScalarType type, IntArrayRef sizes, int* device) {
    const Tensor* t = tensor(o, (int)sizes.size(), device);
    return t != nullptr && t->scalar_type() == type && t->sizes() == sizes && t->is_contiguous() ? t : nullptr;
}

// As exact(), of any length.
const Tensor* row(PyObject* o, ScalarType type, int* device) {
    const Tensor* t = tensor(o, 1, device);
    return t != nullptr && t->scalar_type() == type && t->is_contiguous() ? t : nullptr;
}

bool integer(PyObject* o, int64_t* x) {
    if (!PyLong_CheckExact(o)) return false;
    *x = PyLong_AsLongLong(o);
    if (*x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

Tensor empty(IntArrayRef sizes, ScalarType type, int device) {
    return at::empty(sizes, at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, (c10::DeviceIndex)device)));
}

void* stream_of(int device) { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream(); }

// The result of fn() with the interpreter's lock released: a launch waits while the
// device's queue is full, and other Python threads go on.
template <class F>
int unlocked(F fn) {
    struct Lock {
        PyThreadState* state = PyEval_SaveThread();
        ~Lock() { PyEval_RestoreThread(state); }
    } lock;
    return fn();
}

PyObject* status(int st) { return PyLong_FromLong(st); }

// The tensors as a tuple.
PyObject* tuple(std::initializer_list<Tensor> ts) {
    PyObject* out = PyTuple_New((Py_ssize_t)ts.size());
    if (out == nullptr) return nullptr;
    Py_ssize_t i = 0;
    for (const Tensor& t : ts) {
        PyObject* o = THPVariable_Wrap(t);
        if (o == nullptr) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, i++, o);
    }
    return out;
}

// page_step(seq_lens, new_lens, page_table, free_pages, free_head, max_tokens, B)
PyObject* page_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int64_t rows, B;
    int dev = -1;
    if (n != 7 || !integer(a[5], &rows) || !integer(a[6], &B) || rows < 0 || rows >= (int64_t(1) << 31)) Py_RETURN_NONE;
    const Tensor* table = tensor(a[2], 2, &dev);
    if (table == nullptr || table->scalar_type() != I32 || !table->is_contiguous()) Py_RETURN_NONE;
    const int64_t batch = table->size(0);
    const Tensor *lens = exact(a[0], I32, {batch}, &dev), *more = exact(a[1], I32, {batch}, &dev);
    const Tensor *free = row(a[3], I32, &dev), *head = exact(a[4], I32, {1}, &dev);
    if (!lens || !more || !free || !head || batch >= INT32_MAX || table->size(1) > INT32_MAX || free->numel() > INT32_MAX)
        Py_RETURN_NONE;
    // one allocation, slots (8 bytes) first
    auto out = empty({3 * rows + 3 * batch + 3}, I32, dev)
                   .unsafe_split_with_sizes({2 * rows, batch, batch + 1, batch + 1, rows, 1});
    const int st = unlocked([&] {
        return bf1_page_step(
            (int32_t)batch, lens->const_data_ptr<int32_t>(), more->const_data_ptr<int32_t>(), (int32_t*)table->data_ptr(),
            (int32_t)table->size(1), free->const_data_ptr<int32_t>(), (int32_t)free->numel(),
            head->const_data_ptr<int32_t>(), (int32_t)B, rows, (int32_t*)out[1].data_ptr(), (int32_t*)out[2].data_ptr(),
            (int32_t*)out[3].data_ptr(), (int32_t*)out[4].data_ptr(), (int64_t*)out[0].data_ptr(),
            (int32_t*)out[5].data_ptr(), stream_of(dev));
    });
    if (st != BF1_OK) return status(st);
    return tuple({out[1], out[2], out[3], out[4], out[0].view(I64), out[5]});
    END_HANDLE_TH_ERRORS
}

// What rope and norm + rope have in common.
struct Turning {
    int dims, token;                       // 3: rows [tokens, heads, d]; 4: [batch, heads, n, d]
    int64_t batch, rows, d, heads[2];
    const Tensor *x[2], *pos, *freqs;
    bool own;  // positions of each batch entry
};
bool turning(PyObject* qo, PyObject* ko, PyObject* po, PyObject* fo, int* dev, Turning* t) {
    if (!THPVariable_CheckExact(qo)) return false;
    t->dims = (int)THPVariable_Unpack(qo).dim();
    if (t->dims != 3 && t->dims != 4) return false;
    t->x[0] = tensor(qo, t->dims, dev);
    t->x[1] = tensor(ko, t->dims, dev);
    if (!t->x[0] || !t->x[1]) return false;
    const Tensor &q = *t->x[0], &k = *t->x[1];
    t->token = t->dims == 3 ? 0 : 2;
    t->batch = t->dims == 3 ? 1 : q.size(0);
    t->rows = q.size(t->token);
    t->d = q.size(t->dims - 1);
    if (q.scalar_type() != k.scalar_type() || (q.scalar_type() != BF16 && q.scalar_type() != F32) ||
        k.size(t->token) != t->rows || k.size(t->dims - 1) != t->d || (t->dims == 4 && k.size(0) != t->batch) ||
        q.stride(t->dims - 1) != 1 || k.stride(t->dims - 1) != 1)
        return false;
    t->freqs = row(fo, F64, dev);
    if (!t->freqs || t->freqs->numel() < 1 || t->freqs->numel() > t->d / 2) return false;
    t->pos = exact(po, I32, {t->rows}, dev);
    t->own = t->pos == nullptr && t->dims == 4;
    if (t->own) t->pos = exact(po, I32, {t->batch, t->rows}, dev);
    t->heads[0] = q.size(1);
    t->heads[1] = k.size(1);
    return t->pos && t->batch <= INT32_MAX && t->d <= INT32_MAX && t->heads[0] <= INT32_MAX && t->heads[1] <= INT32_MAX;
}
// Strides over batch, heads and tokens.
void strides_of(const Tensor& x, const Turning& t, int64_t* s) {
    s[0] = t.dims == 4 ? x.stride(0) : 0;
    s[1] = x.stride(1);
    s[2] = x.stride(t.token);
}
// rope(q, k, positions, freqs, interleaved, amplitude, transposed): q and k
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int64_t transposed;
    int dev = -1;
    Turning t;
    if (n != 7 || !PyBool_Check(a[4]) || !PyFloat_CheckExact(a[5]) || !integer(a[6], &transposed) ||
        !turning(a[0], a[1], a[2], a[3], &dev, &t))
        Py_RETURN_NONE;
    const ScalarType type = t.x[0]->scalar_type();
    Tensor out[2];
    int64_t strides[12];
    for (int i = 0; i < 2; ++i) {
        out[i] = empty(t.x[i]->sizes(), type, dev);
        strides_of(*t.x[i], t, strides + 6 * i);
        strides_of(out[i], t, strides + 6 * i + 3);
    }
    const int32_t ty = type == BF16 ? BF1_TYPE_BF16 : BF1_TYPE_F32;
    const int32_t interleaved = a[4] == Py_True;
    const float amplitude = (float)PyFloat_AS_DOUBLE(a[5]);
    const int st = unlocked([&] {
        return bf1_rope(t.x[0]->data_ptr(), t.x[1]->data_ptr(), t.pos->const_data_ptr<int32_t>(), t.own ? t.rows : 0,
                        t.freqs->const_data_ptr<double>(), out[0].data_ptr(), out[1].data_ptr(), (int32_t)t.batch, t.rows,
                        (int32_t)t.heads[0], (int32_t)t.heads[1], (int32_t)t.d, (int32_t)(2 * t.freqs->numel()), ty, ty,
                        interleaved, amplitude, (int32_t)transposed, strides, stream_of(dev));
    });
    return st == BF1_OK ? tuple({out[0], out[1]}) : status(st);
    END_HANDLE_TH_ERRORS
}

// A step's rows k, v: [tokens, Hkv, d] bf16, elements of a head side by side.
bool step_rows(PyObject* ko, PyObject* vo, int64_t Hkv, int64_t d, int* dev, const Tensor** k, const Tensor** v) {
    *k = tensor(ko, 3, dev);
    *v = tensor(vo, 3, dev);
    return *k && *v && (*k)->scalar_type() == BF16 && (*v)->scalar_type() == BF16 && (*k)->size(1) == Hkv &&
           (*k)->size(2) == d && (*v)->sizes() == (*k)->sizes() && (*k)->stride(2) == 1 && (*v)->stride(2) == 1;
}

// kv_append(k, v, slots, k_pages, v_pages)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1;
    if (n != 5) Py_RETURN_NONE;
    const Tensor* kp = tensor(a[3], 4, &dev);
    if (!kp || kp->scalar_type() != BF16 || !kp->is_contiguous()) Py_RETURN_NONE;
    const Tensor* vp = exact(a[4], BF16, kp->sizes(), &dev);
    const Tensor *k, *v;
    if (!vp || !step_rows(a[0], a[1], kp->size(1), kp->size(3), &dev, &k, &v)) Py_RETURN_NONE;
    const Tensor* slots = exact(a[2], I64, {k->size(0)}, &dev);
    if (!slots || kp->size(0) > INT32_MAX || kp->size(1) > INT32_MAX || kp->size(2) > INT32_MAX) Py_RETURN_NONE;
    return status(unlocked([&] {
        return bf1_kv_append(k->data_ptr(), v->data_ptr(), k->stride(0), k->stride(1), v->stride(0), v->stride(1),
                             slots->const_data_ptr<int64_t>(), kp->data_ptr(), vp->data_ptr(), k->size(0),
                             (int32_t)kp->size(0), (int32_t)kp->size(1), (int32_t)kp->size(3), (int32_t)kp->size(2),
                             stream_of(dev));
    }));
    END_HANDLE_TH_ERRORS
}

struct Cache {
    const Tensor *kp, *vp, *ks, *vs, *kt, *vt;
    int64_t pages, Hkv, B, d;
    int32_t format;
};

// The tensors of a CacheQ8 for `batch` sequences.
bool cache_q8(PyObject* o, int64_t batch, int* dev, Cache* c) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 6) return false;
    c->kp = tensor(PyTuple_GET_ITEM(o, 0), 4, dev);
    if (!c->kp || !c->kp->is_contiguous()) return false;
    const ScalarType type = c->kp->scalar_type();
    if (type != at::kFloat8_e4m3fn && type != at::kChar) return false;
    c->format = type == at::kChar ? BF1_Q8_INT8 : BF1_Q8_E4M3;
    c->pages = c->kp->size(0);
    c->Hkv = c->kp->size(1);
    c->B = c->kp->size(2);
    c->d = c->kp->size(3);
    c->vp = exact(PyTuple_GET_ITEM(o, 1), type, {c->pages, c->Hkv, c->d, c->B}, dev);
    c->ks = exact(PyTuple_GET_ITEM(o, 2), F32, {c->pages, c->Hkv}, dev);
    c->vs = exact(PyTuple_GET_ITEM(o, 3), F32, {c->pages, c->Hkv}, dev);
    c->kt = exact(PyTuple_GET_ITEM(o, 4), BF16, {batch, c->Hkv, c->B, c->d}, dev);
    c->vt = exact(PyTuple_GET_ITEM(o, 5), BF16, {batch, c->Hkv, c->B, c->d}, dev);
    return c->vp && c->ks && c->vs && c->kt && c->vt && c->pages <= INT32_MAX && c->Hkv <= INT32_MAX &&
           c->B <= INT32_MAX && c->d <= INT32_MAX;
}

// kv_append_q8(k, v, lens_before, seq_lens, token_start, block_start, page_table, cache)
PyObject* kv_append_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1;
    if (n != 8) Py_RETURN_NONE;
    const Tensor* table = tensor(a[6], 2, &dev);
    if (!table || table->scalar_type() != I32 || !table->is_contiguous()) Py_RETURN_NONE;
    const int64_t batch = table->size(0);
    Cache c;
    const Tensor *k, *v;
    if (batch >= INT32_MAX || table->size(1) > INT32_MAX || !cache_q8(a[7], batch, &dev, &c) ||
        !step_rows(a[0], a[1], c.Hkv, c.d, &dev, &k, &v))
        Py_RETURN_NONE;
    const Tensor *before = exact(a[2], I32, {batch}, &dev), *after = exact(a[3], I32, {batch}, &dev);
    const Tensor *first = exact(a[4], I32, {batch + 1}, &dev), *blocks = exact(a[5], I32, {batch + 1}, &dev);
    if (!before || !after || !first || !blocks) Py_RETURN_NONE;
    return status(unlocked([&] {
        return bf1_kv_append_q8(
            k->data_ptr(), v->data_ptr(), k->stride(0), k->stride(1), v->stride(0), v->stride(1), k->size(0),
            (int32_t)batch, before->const_data_ptr<int32_t>(), after->const_data_ptr<int32_t>(),
            first->const_data_ptr<int32_t>(), blocks->const_data_ptr<int32_t>(), table->const_data_ptr<int32_t>(),
            (int32_t)table->size(1), (int32_t)c.pages, c.kp->data_ptr(), c.vp->data_ptr(), (float*)c.ks->data_ptr(),
            (float*)c.vs->data_ptr(), c.kt->data_ptr(), c.vt->data_ptr(), (int32_t)c.Hkv, (int32_t)c.d, (int32_t)c.B,
            c.format, stream_of(dev));
    }));
    END_HANDLE_TH_ERRORS
}

// attn_decode_q8(q, cache, seq_lens, plan, B)
PyObject* attn_decode_q8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int64_t B;
    int dev = -1;
    if (n != 5 || !integer(a[4], &B)) Py_RETURN_NONE;
    const Tensor* q = tensor(a[0], 3, &dev);
    if (!q || q->scalar_type() != BF16 || !q->is_contiguous()) Py_RETURN_NONE;
    const int64_t batch = q->size(0), Hq = q->size(1);
    Cache c;
    if (batch > INT32_MAX || Hq > INT32_MAX || !cache_q8(a[1], batch, &dev, &c) || c.B != B || c.d != q->size(2))
        Py_RETURN_NONE;
    const Tensor *lens = exact(a[2], I32, {batch}, &dev), *plan = tensor(a[3], 2, &dev);
    if (!lens || !plan || plan->scalar_type() != I32 || !plan->is_contiguous() || plan->size(0) != batch ||
        plan->size(1) > INT32_MAX)
        Py_RETURN_NONE;
    int64_t need = 0;
    int st = bf1_decode_q8_workspace_size((int32_t)batch, (int32_t)Hq, (int32_t)c.Hkv, (int32_t)c.d, (int32_t)B,
                                          (int32_t)plan->size(1), &need);
    if (st != BF1_OK) return status(st);
    Tensor out = empty(q->sizes(), BF16, dev), lse = empty({batch, Hq}, F32, dev), ws;
    if (need > 0) ws = empty({need}, at::kByte, dev);
    st = unlocked([&] {
        return bf1_decode_attn_q8(
            q->data_ptr(), c.kp->data_ptr(), c.vp->data_ptr(), (const float*)c.ks->data_ptr(),
            (const float*)c.vs->data_ptr(), c.kt->data_ptr(), c.vt->data_ptr(), lens->const_data_ptr<int32_t>(),
            (int32_t)c.pages, plan->const_data_ptr<int32_t>(), (int32_t)plan->size(1), out.data_ptr(),
            (float*)lse.data_ptr(), (int32_t)batch, (int32_t)Hq, (int32_t)c.Hkv, (int32_t)c.d, (int32_t)B, c.format,
            need > 0 ? ws.data_ptr() : nullptr, need, stream_of(dev));
    });
    return st == BF1_OK ? tuple({out, lse}) : status(st);
    END_HANDLE_TH_ERRORS
}

// Gains [d], bf16 or fp32, or None.
bool gains_of(PyObject* qo, PyObject* ko, int64_t d, int* dev, const Tensor** q, const Tensor** k, int32_t* type) {
    *q = *k = nullptr;
    ScalarType st = F32;
    for (int i = 0; i < 2; ++i) {
        PyObject* o = i ? ko : qo;
        if (o == Py_None) continue;
        const Tensor* g = tensor(o, 1, dev);
        if (!g || (g->scalar_type() != BF16 && g->scalar_type() != F32) || !g->is_contiguous() || g->numel() != d) return false;
        if (i && *q && g->scalar_type() != st) return false;
        st = g->scalar_type();
        *(i ? k : q) = g;
    }
    *type = st == BF16 ? BF1_TYPE_BF16 : BF1_TYPE_F32;
    return true;
}
void* ptr(const Tensor* t) { return t ? t->data_ptr() : nullptr; }

// qk_norm_rope(q, k, q_gain, k_gain, positions, freqs, eps, interleaved, amplitude): q and k
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1;
    Turning t;
    const Tensor *qg, *kg;
    int32_t gtype;
    if (n != 9 || !PyFloat_CheckExact(a[6]) || !PyBool_Check(a[7]) || !PyFloat_CheckExact(a[8]) ||
        !turning(a[0], a[1], a[4], a[5], &dev, &t) || !gains_of(a[2], a[3], t.d, &dev, &qg, &kg, &gtype))
        Py_RETURN_NONE;
    const ScalarType type = t.x[0]->scalar_type();
    Tensor out[2];
    int64_t strides[12];
    for (int i = 0; i < 2; ++i) {
        out[i] = empty(t.x[i]->sizes(), type, dev);
        strides_of(*t.x[i], t, strides + 6 * i);
        strides_of(out[i], t, strides + 6 * i + 3);
    }
    const int32_t ty = type == BF16 ? BF1_TYPE_BF16 : BF1_TYPE_F32, interleaved = a[7] == Py_True;
    const float eps = (float)PyFloat_AS_DOUBLE(a[6]), amplitude = (float)PyFloat_AS_DOUBLE(a[8]);
    const int st = unlocked([&] {
        return bf1_qk_norm_rope(t.x[0]->data_ptr(), t.x[1]->data_ptr(), ptr(qg), ptr(kg), gtype,
                                t.pos->const_data_ptr<int32_t>(), t.own ? t.rows : 0, t.freqs->const_data_ptr<double>(),
                                out[0].data_ptr(), out[1].data_ptr(), (int32_t)t.batch, t.rows, (int32_t)t.heads[0],
                                (int32_t)t.heads[1], (int32_t)t.d, (int32_t)(2 * t.freqs->numel()), ty, ty, interleaved, eps,
                                amplitude, strides, stream_of(dev));
    });
    return st == BF1_OK ? tuple({out[0], out[1]}) : status(st);
    END_HANDLE_TH_ERRORS
}

// qk_norm_rope_bwd(dq, dk, q, k, q_gain, k_gain, positions, freqs, eps, interleaved, amplitude):
// the gradients of q, k and both gains
PyObject* qk_norm_rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1;
    Turning t;
    const Tensor *qg, *kg;
    int32_t gtype;
    if (n != 11 || !PyFloat_CheckExact(a[8]) || !PyBool_Check(a[9]) || !PyFloat_CheckExact(a[10]) ||
        !turning(a[2], a[3], a[6], a[7], &dev, &t) || !gains_of(a[4], a[5], t.d, &dev, &qg, &kg, &gtype) || !qg || !kg)
        Py_RETURN_NONE;
    const Tensor* dy[2] = {tensor(a[0], t.dims, &dev), tensor(a[1], t.dims, &dev)};
    const ScalarType type = t.x[0]->scalar_type();
    for (int i = 0; i < 2; ++i)
        if (!dy[i] || dy[i]->sizes() != t.x[i]->sizes() || dy[i]->stride(t.dims - 1) != 1 ||
            (dy[i]->scalar_type() != F32 && dy[i]->scalar_type() != type) || dy[i]->scalar_type() != dy[0]->scalar_type())
            Py_RETURN_NONE;
    const int32_t ty = type == BF16 ? BF1_TYPE_BF16 : BF1_TYPE_F32;
    const int32_t rot = (int32_t)(2 * t.freqs->numel());
    int64_t need = 0;
    int st = bf1_qk_norm_rope_bwd_workspace_size((int32_t)t.batch, t.rows, (int32_t)t.heads[0], (int32_t)t.heads[1],
                                                 (int32_t)t.d, rot, ty, &need);
    if (st != BF1_OK) return status(st);
    Tensor out[2], gain[2], ws;
    int64_t strides[18];
    for (int i = 0; i < 2; ++i) {
        out[i] = empty(t.x[i]->sizes(), type, dev);
        gain[i] = empty({t.d}, F32, dev);
        strides_of(*dy[i], t, strides + 9 * i);
        strides_of(*t.x[i], t, strides + 9 * i + 3);
        strides_of(out[i], t, strides + 9 * i + 6);
    }
    if (need > 0) ws = empty({need}, at::kByte, dev);
    const int32_t interleaved = a[9] == Py_True;
    const float eps = (float)PyFloat_AS_DOUBLE(a[8]), amplitude = (float)PyFloat_AS_DOUBLE(a[10]);
    st = unlocked([&] {
        return bf1_qk_norm_rope_bwd(
            dy[0]->data_ptr(), dy[1]->data_ptr(), dy[0]->scalar_type() == BF16 ? BF1_TYPE_BF16 : BF1_TYPE_F32,
            t.x[0]->data_ptr(), t.x[1]->data_ptr(), ptr(qg), ptr(kg), gtype, t.pos->const_data_ptr<int32_t>(),
            t.own ? t.rows : 0, t.freqs->const_data_ptr<double>(), out[0].data_ptr(), out[1].data_ptr(),
            (float*)gain[0].data_ptr(), (float*)gain[1].data_ptr(), (int32_t)t.batch, t.rows, (int32_t)t.heads[0],
            (int32_t)t.heads[1], (int32_t)t.d, rot, ty, ty, interleaved, eps, amplitude, strides,
            need > 0 ? ws.data_ptr() : nullptr, need, stream_of(dev));
    });
    return st == BF1_OK ? tuple({out[0], out[1], gain[0], gain[1]}) : status(st);
    END_HANDLE_TH_ERRORS
}

// tree_step(parents, token_start, lens_before, seq_lens): masks and positions
PyObject* tree_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1;
    if (n != 4) Py_RETURN_NONE;
    const Tensor *parents = row(a[0], I32, &dev), *before = row(a[2], I32, &dev);
    if (!parents || !before) Py_RETURN_NONE;
    const int64_t rows = parents->numel(), batch = before->numel();
    const Tensor *start = exact(a[1], I32, {batch + 1}, &dev), *after = exact(a[3], I32, {batch}, &dev);
    if (!start || !after || batch > INT32_MAX) Py_RETURN_NONE;
    Tensor masks = empty({rows}, I64, dev), pos = empty({rows}, I32, dev);
    const int st = unlocked([&] {
        return bf1_tree_step(parents->const_data_ptr<int32_t>(), start->const_data_ptr<int32_t>(),
                             before->const_data_ptr<int32_t>(), after->const_data_ptr<int32_t>(), (int32_t)batch, rows,
                             (int64_t*)masks.data_ptr(), (int32_t*)pos.data_ptr(), stream_of(dev));
    });
    return st == BF1_OK ? tuple({masks, pos}) : status(st);
    END_HANDLE_TH_ERRORS
}

// The bf16 pages [num_pages, Hkv, B, d] of a cache.
bool bf16_pages(PyObject* ko, PyObject* vo, int* dev, const Tensor** k, const Tensor** v) {
    *k = tensor(ko, 4, dev);
    if (!*k || (*k)->scalar_type() != BF16 || !(*k)->is_contiguous()) return false;
    *v = exact(vo, BF16, (*k)->sizes(), dev);
    for (int i = 0; i < 4; ++i)
        if ((*k)->size(i) > INT32_MAX) return false;
    return *v != nullptr;
}

// attn_tree(q, k_pages, v_pages, masks, positions, lens_before, token_start, page_table, B, L, dense, max_nodes)
PyObject* attn_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int64_t B, L, most;
    int dev = -1;
    if (n != 12 || !integer(a[8], &B) || !integer(a[9], &L) || !PyBool_Check(a[10]) || !integer(a[11], &most) ||
        L > INT32_MAX || L < INT32_MIN || most > INT32_MAX || most < INT32_MIN)
        Py_RETURN_NONE;
    const Tensor *q = tensor(a[0], 3, &dev), *k, *v;
    if (!q || q->scalar_type() != BF16 || !q->is_contiguous() || !bf16_pages(a[1], a[2], &dev, &k, &v)) Py_RETURN_NONE;
    const int64_t rows = q->size(0), Hq = q->size(1), d = q->size(2);
    const Tensor* table = tensor(a[7], 2, &dev);
    if (k->size(2) != B || k->size(3) != d || Hq > INT32_MAX || !table || table->scalar_type() != I32 ||
        !table->is_contiguous() || table->size(0) > INT32_MAX || table->size(1) > INT32_MAX)
        Py_RETURN_NONE;
    const int64_t batch = table->size(0);
    const Tensor *masks = exact(a[3], I64, {rows}, &dev), *pos = exact(a[4], I32, {rows}, &dev);
    const Tensor *before = exact(a[5], I32, {batch}, &dev), *start = exact(a[6], I32, {batch + 1}, &dev);
    if (!masks || !pos || !before || !start) Py_RETURN_NONE;
    const int32_t dense = a[10] == Py_True;
    int64_t need = 0;
    int st = bf1_attn_tree_workspace_size((int32_t)batch, (int32_t)most, (int32_t)Hq, (int32_t)k->size(1), (int32_t)d,
                                          (int32_t)B, (int32_t)table->size(1), (int32_t)L, dense, &need);
    if (st != BF1_OK) return status(st);
    Tensor out = empty(q->sizes(), BF16, dev), lse = empty({rows, Hq}, F32, dev), ws;
    if (need > 0) ws = empty({need}, at::kByte, dev);
    st = unlocked([&] {
        return bf1_attn_tree(q->data_ptr(), k->data_ptr(), v->data_ptr(), masks->const_data_ptr<int64_t>(),
                             pos->const_data_ptr<int32_t>(), before->const_data_ptr<int32_t>(),
                             start->const_data_ptr<int32_t>(), table->const_data_ptr<int32_t>(), (int32_t)table->size(1),
                             (int32_t)k->size(0), out.data_ptr(), (float*)lse.data_ptr(), (int32_t)batch, rows, (int32_t)most,
                             (int32_t)Hq, (int32_t)k->size(1), (int32_t)d, (int32_t)B, (int32_t)L, dense,
                             need > 0 ? ws.data_ptr() : nullptr, need, stream_of(dev));
    });
    return st == BF1_OK ? tuple({out, lse}) : status(st);
    END_HANDLE_TH_ERRORS
}

// kv_compact(k_pages, v_pages, accepted, lens_before, seq_lens, page_table): the new lengths
PyObject* kv_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1;
    const Tensor *k, *v;
    if (n != 6 || !bf16_pages(a[0], a[1], &dev, &k, &v)) Py_RETURN_NONE;
    const Tensor *table = tensor(a[5], 2, &dev), *accepted = tensor(a[2], 2, &dev);
    if (!table || table->scalar_type() != I32 || !table->is_contiguous() || !accepted || accepted->scalar_type() != I32 ||
        !accepted->is_contiguous() || accepted->size(0) != table->size(0) || accepted->size(1) > INT32_MAX ||
        table->size(0) > INT32_MAX || table->size(1) > INT32_MAX)
        Py_RETURN_NONE;
    const int64_t batch = table->size(0);
    const Tensor *before = exact(a[3], I32, {batch}, &dev), *after = exact(a[4], I32, {batch}, &dev);
    if (!before || !after) Py_RETURN_NONE;
    Tensor out = empty({batch}, I32, dev);
    const int st = unlocked([&] {
        return bf1_kv_compact(k->data_ptr(), v->data_ptr(), accepted->const_data_ptr<int32_t>(), (int32_t)accepted->size(1),
                              before->const_data_ptr<int32_t>(), after->const_data_ptr<int32_t>(),
                              table->const_data_ptr<int32_t>(), (int32_t)batch, (int32_t)table->size(1), (int32_t)k->size(0),
                              (int32_t)k->size(1), (int32_t)k->size(3), (int32_t)k->size(2), (int32_t*)out.data_ptr(),
                              stream_of(dev));
    });
    return st == BF1_OK ? THPVariable_Wrap(out) : status(st);
    END_HANDLE_TH_ERRORS
}

// page_fork(seq_lens, sources, keep_lens, page_table, shares, free_pages, free_head, B)
PyObject* page_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int64_t B;
    int dev = -1;
    if (n != 8 || !integer(a[7], &B)) Py_RETURN_NONE;
    const Tensor* table = tensor(a[3], 2, &dev);
    if (!table || table->scalar_type() != I32 || !table->is_contiguous() || table->size(0) > INT32_MAX ||
        table->size(1) > INT32_MAX)
        Py_RETURN_NONE;
    const int64_t batch = table->size(0), width = table->size(1);
    const Tensor *lens = exact(a[0], I32, {batch}, &dev), *src = exact(a[1], I32, {batch}, &dev);
    const Tensor *keep = exact(a[2], I32, {batch}, &dev), *shares = row(a[4], I32, &dev), *free = row(a[5], I32, &dev);
    const Tensor* head = exact(a[6], I32, {1}, &dev);
    if (!lens || !src || !keep || !shares || !free || !head || shares->numel() > INT32_MAX || free->numel() > INT32_MAX)
        Py_RETURN_NONE;
    // one allocation
    auto out = empty({batch * width + 4 * batch + 1}, I32, dev)
                   .unsafe_split_with_sizes({batch * width, batch, batch, batch, batch, 1});
    const int st = unlocked([&] {
        return bf1_page_fork((int32_t)batch, lens->const_data_ptr<int32_t>(), src->const_data_ptr<int32_t>(),
                             keep->const_data_ptr<int32_t>(), table->const_data_ptr<int32_t>(), (int32_t)width,
                             (int32_t*)shares->data_ptr(), (int32_t)shares->numel(), (int32_t*)free->data_ptr(),
                             (int32_t)free->numel(), head->const_data_ptr<int32_t>(), (int32_t)B, (int32_t*)out[0].data_ptr(),
                             (int32_t*)out[1].data_ptr(), (int32_t*)out[5].data_ptr(), (int32_t*)out[2].data_ptr(),
                             (int32_t*)out[3].data_ptr(), (int32_t*)out[4].data_ptr(), stream_of(dev));
    });
    if (st != BF1_OK) return status(st);
    return tuple({out[0].view({batch, width}), out[1], out[5], out[2], out[3], out[4]});
    END_HANDLE_TH_ERRORS
}

// kv_copy(k_pages, v_pages, copy_from, copy_to, copy_rows)
PyObject* kv_copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int dev = -1;
    const Tensor *k, *v;
    if (n != 5 || !bf16_pages(a[0], a[1], &dev, &k, &v)) Py_RETURN_NONE;
    const Tensor* from = row(a[2], I32, &dev);
    if (!from || from->numel() > INT32_MAX) Py_RETURN_NONE;
    const Tensor *to = exact(a[3], I32, {from->numel()}, &dev), *rows = exact(a[4], I32, {from->numel()}, &dev);
    if (!to || !rows) Py_RETURN_NONE;
    return status(unlocked([&] {
        return bf1_kv_copy(k->data_ptr(), v->data_ptr(), from->const_data_ptr<int32_t>(), to->const_data_ptr<int32_t>(),
                           rows->const_data_ptr<int32_t>(), (int32_t)from->numel(), (int32_t)k->size(0), (int32_t)k->size(1),
                           (int32_t)k->size(3), (int32_t)k->size(2), stream_of(dev));
    }));
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"page_step", (PyCFunction)(void (*)())page_step, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void (*)())rope, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)())kv_append, METH_FASTCALL, nullptr},
    {"kv_append_q8", (PyCFunction)(void (*)())kv_append_q8, METH_FASTCALL, nullptr},
    {"attn_decode_q8", (PyCFunction)(void (*)())attn_decode_q8, METH_FASTCALL, nullptr},
    {"qk_norm_rope", (PyCFunction)(void (*)())qk_norm_rope, METH_FASTCALL, nullptr},
    {"qk_norm_rope_bwd", (PyCFunction)(void (*)())qk_norm_rope_bwd, METH_FASTCALL, nullptr},
    {"tree_step", (PyCFunction)(void (*)())tree_step, METH_FASTCALL, nullptr},
    {"attn_tree", (PyCFunction)(void (*)())attn_tree, METH_FASTCALL, nullptr},
    {"kv_compact", (PyCFunction)(void (*)())kv_compact, METH_FASTCALL, nullptr},
    {"page_fork", (PyCFunction)(void (*)())page_fork, METH_FASTCALL, nullptr},
    {"kv_copy", (PyCFunction)(void (*)())kv_copy, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Native marshalling of the cache's operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
