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

// rope(q, k, positions, freqs, interleaved, amplitude, transposed): q and k
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 7 || !THPVariable_CheckExact(a[0]) || !PyBool_Check(a[4]) || !PyFloat_CheckExact(a[5])) Py_RETURN_NONE;
    int64_t transposed;
    if (!integer(a[6], &transposed)) Py_RETURN_NONE;
    int dev = -1;
    const int dims = (int)THPVariable_Unpack(a[0]).dim();
    if (dims != 3 && dims != 4) Py_RETURN_NONE;
    const Tensor *q = tensor(a[0], dims, &dev), *k = tensor(a[1], dims, &dev);
    if (!q || !k || q->scalar_type() != k->scalar_type() || (q->scalar_type() != BF16 && q->scalar_type() != F32))
        Py_RETURN_NONE;
    const int token = dims == 3 ? 0 : 2;  // rows [tokens, heads, d] or [batch, heads, n, d]
    const int64_t batch = dims == 3 ? 1 : q->size(0), rows = q->size(token), d = q->size(dims - 1);
    if (k->size(token) != rows || k->size(dims - 1) != d || (dims == 4 && k->size(0) != batch) || q->stride(dims - 1) != 1 ||
        k->stride(dims - 1) != 1)
        Py_RETURN_NONE;
    const Tensor* freqs = row(a[3], F64, &dev);
    if (!freqs || freqs->numel() < 1 || freqs->numel() > d / 2) Py_RETURN_NONE;
    const Tensor* pos = exact(a[2], I32, {rows}, &dev);
    const bool own = pos == nullptr && dims == 4;  // positions of each batch entry
    if (own) pos = exact(a[2], I32, {batch, rows}, &dev);
    if (!pos || batch > INT32_MAX || d > INT32_MAX) Py_RETURN_NONE;
    const ScalarType type = q->scalar_type();
    Tensor qo = empty(q->sizes(), type, dev), ko = empty(k->sizes(), type, dev);
    int64_t strides[12];
    int64_t heads[2];
    for (int side = 0; side < 2; ++side) {
        const Tensor& x = side ? *k : *q;
        const int64_t h = heads[side] = x.size(1);
        int64_t* s = strides + 6 * side;
        s[0] = dims == 4 ? x.stride(0) : 0;
        s[1] = x.stride(1);
        s[2] = x.stride(token);
        s[3] = dims == 4 ? h * rows * d : 0;
        s[4] = dims == 4 ? rows * d : d;
        s[5] = dims == 4 ? d : h * d;
    }
    if (heads[0] > INT32_MAX || heads[1] > INT32_MAX) Py_RETURN_NONE;
    const int32_t t = type == BF16 ? BF1_TYPE_BF16 : BF1_TYPE_F32;
    const int32_t interleaved = a[4] == Py_True;
    const float amplitude = (float)PyFloat_AS_DOUBLE(a[5]);
    const int st = unlocked([&] {
        return bf1_rope(q->data_ptr(), k->data_ptr(), pos->const_data_ptr<int32_t>(), own ? rows : 0,
                        freqs->const_data_ptr<double>(), qo.data_ptr(), ko.data_ptr(), (int32_t)batch, rows,
                        (int32_t)heads[0], (int32_t)heads[1], (int32_t)d, (int32_t)(2 * freqs->numel()), t, t, interleaved,
                        amplitude, (int32_t)transposed, strides, stream_of(dev));
    });
    return st == BF1_OK ? tuple({qo, ko}) : status(st);
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

PyMethodDef methods[] = {
    {"page_step", (PyCFunction)(void (*)())page_step, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void (*)())rope, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)())kv_append, METH_FASTCALL, nullptr},
    {"kv_append_q8", (PyCFunction)(void (*)())kv_append_q8, METH_FASTCALL, nullptr},
    {"attn_decode_q8", (PyCFunction)(void (*)())attn_decode_q8, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Native marshalling of the cache's operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
