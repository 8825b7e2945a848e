// Marshalling of the decoder-layer calls: tensors to addresses, shapes and strides, every check, one call of the C ABI.
// Native because a call costs as much as a short kernel: in Python the checks of a dozen tensors take 5 to 12 microseconds.
// Functions return the call's loco_status_t; what a tensor has wrong raises ValueError.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdio>
#include <string>

#include "../../include/loco_layer.h"

namespace {

struct Refused {
    std::string why;
};
[[noreturn]] void refuse(std::string why) { throw Refused{std::move(why)}; }

using at::ScalarType;

const at::Tensor *tensor(PyObject *o, const char *what) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a tensor");
    return &THPVariable_Unpack(o);
}
const at::Tensor &need(PyObject *o, const char *what) {
    const at::Tensor *t = tensor(o, what);
    if (!t) refuse(std::string(what) + " is missing");
    return *t;
}

// The operands' device, which has to be the current one, as for every call of the library.
int device_of(const at::Tensor &t) {
    if (!t.is_cuda()) refuse("expected CUDA tensors");
    const int d = t.get_device();
    if (c10::cuda::current_device() != d) refuse("the operands live on cuda:" + std::to_string(d) + ", which is not the current device");
    return d;
}
void *stream_of(PyObject *stream, int device) {
    if (stream == Py_None) return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
    const unsigned long long raw = PyLong_AsUnsignedLongLong(stream);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        refuse("the stream must be a raw stream's address");
    }
    return reinterpret_cast<void *>(raw);
}

int32_t dtype_of(const at::Tensor &t) {
    if (t.scalar_type() == ScalarType::BFloat16) return LOCO_BF16;
    if (t.scalar_type() == ScalarType::Float) return LOCO_F32;
    refuse("expected bfloat16 or float32");
}

// Heads [batch, row, head, dim] or [row, head, dim] of a shape and type.
loco_heads_t heads(const at::Tensor &t, at::IntArrayRef shape, ScalarType type, int device, const char *what) {
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type) refuse(std::string("all heads must have one type and device: ") + what);
    if (t.sizes() != shape) refuse(std::string("unexpected shape of ") + what);
    const at::IntArrayRef s = t.strides();
    const size_t n = shape.size();
    if (s[n - 1] != 1 && shape[n - 1] != 1) refuse(std::string("the dimensions of a head must be contiguous: ") + what);
    return loco_heads_t{t.data_ptr(), n == 4 ? s[0] : 0, s[n - 3], s[n - 2]};
}

// A contiguous tensor of a shape and type, or none.
void *flat(PyObject *o, at::IntArrayRef shape, ScalarType type, int device, const char *what) {
    const at::Tensor *t = tensor(o, what);
    if (!t) return nullptr;
    if (!t->is_cuda() || t->get_device() != device || t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous())
        refuse(std::string(what) + " must be a contiguous tensor of the documented shape and type on the operands' device");
    return t->data_ptr();
}

// The tokens that take part: a byte each, of truth values or of numbers.
uint8_t *mask_of(PyObject *o, int64_t tokens, int device) {
    const at::Tensor *t = tensor(o, "mask");
    return static_cast<uint8_t *>(flat(o, {tokens}, t && t->scalar_type() == ScalarType::Bool ? ScalarType::Bool : ScalarType::Byte, device, "mask"));
}

int32_t small(int64_t x, const char *what) {
    if (x < 0 || x > 0x7fffffff) refuse(std::string("too large: ") + what);
    return static_cast<int32_t>(x);
}
int64_t integer(PyObject *o, const char *what) {
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(what) + " must be an integer");
    }
    return x;
}
bool truth(PyObject *o, const char *what) {
    const int x = PyObject_IsTrue(o);
    if (x < 0) {
        PyErr_Clear();
        refuse(std::string(what) + " must be true or false");
    }
    return x != 0;
}
float number(PyObject *o, const char *what) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(what) + " must be a number");
    }
    return static_cast<float>(x);
}

// table, q, k, q_out, k_out, positions, layout, inverse, stream
int rotary_apply(PyObject *const *a) {
    const at::Tensor &table = need(a[0], "table"), &q = need(a[1], "q"), &q_out = need(a[3], "q_out");
    const at::Tensor *k = tensor(a[2], "k"), *positions = tensor(a[5], "positions");
    const int device = device_of(q);
    const at::IntArrayRef shape = q.sizes();
    if (shape.size() != 4) refuse("expected heads [batch, seq, heads, dim]");
    if (!table.is_cuda() || table.get_device() != device || table.dim() != 2 || table.scalar_type() != ScalarType::Float || !table.is_contiguous())
        refuse("the table must be a contiguous fp32 tensor [positions, rotary_dim] on the heads' device");
    const ScalarType type = q.scalar_type();
    loco_heads_t x[2] = {heads(q, shape, type, device, "q"), {}}, y[2] = {heads(q_out, shape, type, device, "q_out"), {}};
    int32_t count[2] = {small(shape[2], "heads"), 0};
    if (k) {
        const at::IntArrayRef ks = k->sizes();
        if (ks.size() != 4 || ks[0] != shape[0] || ks[1] != shape[1] || ks[3] != shape[3]) refuse("k must have q's batch, rows and head size");
        x[1] = heads(*k, ks, type, device, "k");
        y[1] = heads(need(a[4], "k_out"), ks, type, device, "k_out");
        count[1] = small(ks[2], "heads");
    }
    int32_t wide = 0;
    if (positions) {
        if (positions->scalar_type() != ScalarType::Int && positions->scalar_type() != ScalarType::Long) refuse("positions must be int32 or int64");
        wide = positions->scalar_type() == ScalarType::Int ? 4 : 8;
    }
    const void *at = positions ? flat(a[5], shape.slice(0, 2), positions->scalar_type(), device, "positions") : nullptr;
    const loco_rotary_t cfg{dtype_of(q), static_cast<int32_t>(integer(a[6], "layout")), small(shape[3], "dim"), small(table.size(1), "rotary_dim"),
                            small(shape[0], "batch"), small(shape[1], "seq"), small(table.size(0), "positions"), wide, truth(a[7], "inverse")};
    return loco_rotary_apply(&cfg, table.const_data_ptr<float>(), at, x, y, count, k ? 2 : 1, stream_of(a[8], device));
}

struct Attention {
    loco_attention_t cfg;
    int device;
    at::IntArrayRef qs, ks;
    int64_t stats[3];
    size_t stat_dims;
    at::IntArrayRef stat_shape() const { return at::IntArrayRef(stats, stat_dims); }
};

// causal, scale, len_q, len_k, cu_q, cu_k, max_q, max_k
Attention attention(const at::Tensor &q, const at::Tensor &k, PyObject *const *a) {
    Attention c{};
    c.device = device_of(q);
    if (q.scalar_type() != ScalarType::BFloat16) refuse("attention takes bfloat16 tensors");
    const bool packed = a[4] != Py_None || a[5] != Py_None;
    c.qs = q.sizes();
    c.ks = k.sizes();
    const size_t n = packed ? 3 : 4;
    if (c.qs.size() != n || c.ks.size() != n || c.ks[n - 1] != c.qs[n - 1])
        refuse("expected heads [batch, row, head, dim], or [row, head, dim] with cu_q and cu_k");
    loco_attention_t &t = c.cfg;
    if (packed) {
        if (a[4] == Py_None || a[5] == Py_None || a[6] == Py_None || a[7] == Py_None || a[2] != Py_None || a[3] != Py_None)
            refuse("packed samples need cu_q, cu_k, max_q and max_k and take no lengths");
        const int64_t offsets = need(a[4], "cu_q").numel();
        t.batch = small(offsets - 1, "batch");
        t.d_len_q = static_cast<const int32_t *>(flat(a[4], {offsets}, ScalarType::Int, c.device, "cu_q"));
        t.d_len_k = static_cast<const int32_t *>(flat(a[5], {offsets}, ScalarType::Int, c.device, "cu_k"));
        t.max_q = small(integer(a[6], "max_q"), "max_q");
        t.max_k = small(integer(a[7], "max_k"), "max_k");
        c.stats[0] = c.qs[1];
        c.stats[1] = c.qs[0];
        c.stat_dims = 2;
    } else {
        if (c.ks[0] != c.qs[0]) refuse("queries and keys must have the same batch");
        t.batch = small(c.qs[0], "batch");
        t.d_len_q = static_cast<const int32_t *>(flat(a[2], {c.qs[0]}, ScalarType::Int, c.device, "len_q"));
        t.d_len_k = static_cast<const int32_t *>(flat(a[3], {c.qs[0]}, ScalarType::Int, c.device, "len_k"));
        c.stats[0] = c.qs[0];
        c.stats[1] = c.qs[2];
        c.stats[2] = c.qs[1];
        c.stat_dims = 3;
    }
    t.heads_q = small(c.qs[n - 2], "heads");
    t.heads_kv = small(c.ks[n - 2], "heads");
    t.head_dim = small(c.qs[n - 1], "dim");
    t.packed = packed;
    t.seq_q = small(c.qs[n - 3], "rows");
    t.seq_k = small(c.ks[n - 3], "rows");
    t.causal = truth(a[0], "causal");
    t.scale = a[1] == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(t.head_dim))) : number(a[1], "scale");
    return c;
}

// q, k, v, o, lse, then causal ... max_k, stream
int attention_forward(PyObject *const *a) {
    const at::Tensor &q = need(a[0], "q"), &k = need(a[1], "k");
    const Attention c = attention(q, k, a + 5);
    const ScalarType type = ScalarType::BFloat16;
    const loco_heads_t hq = heads(q, c.qs, type, c.device, "q"), hk = heads(k, c.ks, type, c.device, "k"),
                       hv = heads(need(a[2], "v"), c.ks, type, c.device, "v"), ho = heads(need(a[3], "o"), c.qs, type, c.device, "o");
    return loco_attention_forward(&c.cfg, &hq, &hk, &hv, &ho, static_cast<float *>(flat(a[4], c.stat_shape(), ScalarType::Float, c.device, "lse")),
                                  stream_of(a[13], c.device));
}

// q, k, v, o, lse, do, dq, dk, dv, work, then causal ... max_k, stream
int attention_backward(PyObject *const *a) {
    const at::Tensor &q = need(a[0], "q"), &k = need(a[1], "k"), &work = need(a[9], "work");
    const Attention c = attention(q, k, a + 10);
    const ScalarType type = ScalarType::BFloat16;
    const loco_heads_t hq = heads(q, c.qs, type, c.device, "q"), hk = heads(k, c.ks, type, c.device, "k"),
                       hv = heads(need(a[2], "v"), c.ks, type, c.device, "v"), ho = heads(need(a[3], "o"), c.qs, type, c.device, "o"),
                       hd = heads(need(a[5], "do"), c.qs, type, c.device, "do"), gq = heads(need(a[6], "dq"), c.qs, type, c.device, "dq"),
                       gk = heads(need(a[7], "dk"), c.ks, type, c.device, "dk"), gv = heads(need(a[8], "dv"), c.ks, type, c.device, "dv");
    if (!work.is_cuda() || work.get_device() != c.device || !work.is_contiguous()) refuse("the workspace must be a contiguous tensor on the operands' device");
    return loco_attention_backward(&c.cfg, &hq, &hk, &hv, &ho, static_cast<float *>(flat(a[4], c.stat_shape(), ScalarType::Float, c.device, "lse")), &hd,
                                   &gq, &gk, &gv, work.data_ptr(), work.nbytes(), stream_of(a[18], c.device));
}

struct Rows {
    loco_router_t cfg;
    int device;
    int64_t tokens, stride;
    void *at;
};
// experts, top_k, normalize, balance_coef, z_coef
Rows rows(const at::Tensor &t, PyObject *const *a, const char *what) {
    Rows r{};
    r.device = device_of(t);
    r.cfg = loco_router_t{dtype_of(t), small(integer(a[0], "experts"), "experts"), small(integer(a[1], "top_k"), "top_k"), truth(a[2], "normalize"),
                          number(a[3], "balance_coef"), number(a[4], "z_coef")};
    if (t.dim() != 2 || t.size(1) != r.cfg.experts || (t.stride(1) != 1 && t.size(1) > 1)) refuse(std::string(what) + " must be [tokens, experts] with contiguous rows");
    r.tokens = t.size(0);
    r.stride = r.tokens > 1 ? t.stride(0) : 0;
    r.at = t.data_ptr();
    return r;
}

// the five of the configuration, logits, index, weight, counts, mean, losses, work, mask, stream
int router_forward(PyObject *const *a) {
    const Rows r = rows(need(a[5], "logits"), a, "logits");
    const at::Tensor &work = need(a[11], "work");
    if (!work.is_cuda() || work.get_device() != r.device || !work.is_contiguous()) refuse("the workspace must be a contiguous tensor on the operands' device");
    const int64_t n = r.tokens, k = r.cfg.top_k, e = r.cfg.experts;
    return loco_router_forward(&r.cfg, n, r.at, r.stride, mask_of(a[12], n, r.device),
                               static_cast<int32_t *>(flat(a[6], {n, k}, ScalarType::Int, r.device, "index")),
                               static_cast<float *>(flat(a[7], {n, k}, ScalarType::Float, r.device, "weight")),
                               static_cast<int32_t *>(flat(a[8], {e + 1}, ScalarType::Int, r.device, "counts")),
                               static_cast<float *>(flat(a[9], {e}, ScalarType::Float, r.device, "mean")),
                               static_cast<float *>(flat(a[10], {2}, ScalarType::Float, r.device, "losses")), work.data_ptr(), work.nbytes(),
                               stream_of(a[13], r.device));
}

// the five of the configuration, logits, index, counts, dlogits, mask, dlosses, dweights, stream
int router_backward(PyObject *const *a) {
    const at::Tensor &logits = need(a[5], "logits"), &dlogits = need(a[8], "dlogits");
    const Rows r = rows(logits, a, "logits"), d = rows(dlogits, a, "dlogits");
    if (d.tokens != r.tokens || dlogits.scalar_type() != logits.scalar_type()) refuse("dlogits must have the logits' shape and type");
    const int64_t n = r.tokens, k = r.cfg.top_k, e = r.cfg.experts;
    return loco_router_backward(&r.cfg, n, r.at, r.stride, mask_of(a[9], n, r.device),
                                static_cast<int32_t *>(flat(a[6], {n, k}, ScalarType::Int, r.device, "index")),
                                static_cast<int32_t *>(flat(a[7], {e + 1}, ScalarType::Int, r.device, "counts")),
                                static_cast<float *>(flat(a[10], {2}, ScalarType::Float, r.device, "dlosses")),
                                static_cast<float *>(flat(a[11], {n, k}, ScalarType::Float, r.device, "dweights")), d.at, d.stride,
                                stream_of(a[12], r.device));
}

template <int (*kCall)(PyObject *const *), int kArgs> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != kArgs) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", kArgs, n);
        return nullptr;
    }
    try {
        return PyLong_FromLong(kCall(args));
    } catch (const Refused &r) {
        PyErr_SetString(PyExc_ValueError, r.why.c_str());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

#define LOCO_ENTRY(name, args) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(entry<name, args>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {LOCO_ENTRY(rotary_apply, 9), LOCO_ENTRY(attention_forward, 14), LOCO_ENTRY(attention_backward, 19),
                         LOCO_ENTRY(router_forward, 14), LOCO_ENTRY(router_backward, 13), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layer_binding", LOCO_BUILT_FOR, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layer_binding() { return PyModule_Create(&module); }
