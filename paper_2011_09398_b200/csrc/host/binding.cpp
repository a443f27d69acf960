// The call path of the Python binding in native code: argument checks, output allocation, the current
// stream and the C-ABI call, for the entry points a model runs per layer.
//
// What bounds these calls is host time: a small layer runs 2-4 us on the GPU, and the same marshalling in
// Python (attribute reads of up to six tensors, a stream lookup, a ctypes call with eight arguments and
// torch.empty) took 11 us per call, 15 us with the output allocated, so a network of small layers was paced
// by its caller.  Here a tensor argument is unwrapped to its at::Tensor once and every check is a field read.
//
// The checks, their order and their messages are the binding's (binding.py holds the Python signatures and
// documents the calls).  The GIL is released around every library call, as ctypes does.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "../row_overlap.cuh"
#include "lce.h"

namespace {

PyObject *g_lce_error = nullptr;  // binding.LceError, set by setup()

// A Python exception is set; unwinds to the entry point.
struct Raised {};

[[noreturn]] void value_error(const std::string &text)
{
    PyErr_SetString(PyExc_ValueError, text.c_str());
    throw Raised{};
}

void check(int status, const char *where)
{
    if (status == LCE_OK) return;
    PyObject *e = PyObject_CallFunction(g_lce_error, "is", status, where);
    if (e) {
        PyErr_SetObject(g_lce_error, e);
        Py_DECREF(e);
    }
    throw Raised{};
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw Raised{};
    }
    return THPVariable_Unpack(o);
}

const char *dtype_name(at::ScalarType t)
{
    return t == at::kFloat ? "torch.float32" : t == at::kInt ? "torch.int32" : "torch.uint8";
}

void *device_pointer(const at::Tensor &t, at::ScalarType dtype, const char *name)
{
    if (!t.is_cuda()) value_error(std::string(name) + " must be a CUDA tensor (there is no CPU path)");
    if (t.scalar_type() != dtype || !t.is_contiguous()) value_error(std::string(name) + " must be contiguous " + dtype_name(dtype));
    return t.data_ptr();
}

void *device_pointer(PyObject *o, at::ScalarType dtype, const char *name)  // None -> null
{
    return o == Py_None ? nullptr : device_pointer(tensor(o, name), dtype, name);
}

void *host_pointer(PyObject *o, at::ScalarType dtype, const char *name)  // None -> null
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    if (t.is_cuda() || t.scalar_type() != dtype || !t.is_contiguous())
        value_error(std::string(name) + " must be a contiguous host " + dtype_name(dtype) + " tensor");
    return t.data_ptr();
}

void *current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

at::Tensor empty_like_device(at::IntArrayRef shape, at::ScalarType dtype, const at::Tensor &on)
{
    if (on.is_cuda()) return at::Tensor(at::detail::empty_cuda(shape, dtype, on.device(), c10::nullopt));
    return at::empty(shape, on.options().dtype(dtype));
}

// The descriptor is a ctypes structure with the layout of lce_bconv2d_desc.
struct Desc {
    Py_buffer view{};
    const lce_bconv2d_desc *d = nullptr;
    explicit Desc(PyObject *o)
    {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Raised{};
        if (view.len != (Py_ssize_t)sizeof(lce_bconv2d_desc)) {
            PyBuffer_Release(&view);
            PyErr_SetString(PyExc_TypeError, "desc must be a BConv2dDesc");
            throw Raised{};
        }
        d = static_cast<const lce_bconv2d_desc *>(view.buf);
    }
    ~Desc() { PyBuffer_Release(&view); }
    Desc(const Desc &) = delete;
};

int64_t words(int64_t c) { return (c + 31) / 32; }

template <typename Call>
int without_gil(Call call)
{
    int st;
    Py_BEGIN_ALLOW_THREADS;
    st = call();
    Py_END_ALLOW_THREADS;
    return st;
}

// Every entry point: fixed number of positional arguments, C++ exceptions turned into Python ones.
template <PyObject *(*Body)(PyObject *const *), Py_ssize_t N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return Body(args);
    } catch (const Raised &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject *returned(PyObject *given, const at::Tensor &made)
{
    if (given == Py_None) return THPVariable_Wrap(made);
    Py_INCREF(given);
    return given;
}

PyObject *bitpack(PyObject *const *a)  // x, out
{
    const at::Tensor &x = tensor(a[0], "x");
    if (x.dim() == 0) value_error("x must have a channel axis");
    const int64_t C = x.size(-1), rows = C ? x.numel() / C : 0;
    at::Tensor made;
    if (a[1] == Py_None) {
        c10::SmallVector<int64_t, 6> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = words(C);
        made = empty_like_device(shape, at::kInt, x);
    }
    const at::Tensor &out = a[1] == Py_None ? made : tensor(a[1], "out");
    auto *px = static_cast<const float *>(device_pointer(x, at::kFloat, "x"));
    auto *po = static_cast<uint32_t *>(device_pointer(out, at::kInt, "out"));
    void *s = current_stream();
    check(without_gil([&] { return lce_bitpack(px, po, rows, (int32_t)C, s); }), "lce_bitpack");
    return returned(a[1], made);
}

PyObject *unpack(PyObject *const *a)  // words, channels, out
{
    const at::Tensor &w = tensor(a[0], "words");
    const long C = PyLong_AsLong(a[1]);
    if (C == -1 && PyErr_Occurred()) throw Raised{};
    if (words(C) == 0) {  // the row count is the tensor's words divided by the words per row
        PyErr_SetString(PyExc_ZeroDivisionError, "integer division or modulo by zero");
        throw Raised{};
    }
    const int64_t rows = w.numel() / words(C);
    at::Tensor made;
    if (a[2] == Py_None) {
        c10::SmallVector<int64_t, 6> shape(w.sizes().begin(), w.sizes().end());
        if (shape.empty()) shape.push_back(C); else shape.back() = C;
        made = empty_like_device(shape, at::kFloat, w);
    }
    const at::Tensor &out = a[2] == Py_None ? made : tensor(a[2], "out");
    auto *pw = static_cast<const uint32_t *>(device_pointer(w, at::kInt, "words"));
    auto *po = static_cast<float *>(device_pointer(out, at::kFloat, "out"));
    void *s = current_stream();
    check(without_gil([&] { return lce_unpack(pw, po, rows, (int32_t)C, s); }), "lce_unpack");
    return returned(a[2], made);
}

// lce_bconv2d and lce_bconv2d_f32: desc, input, weights, multiplier, bias, thresholds, out
template <bool F32>
PyObject *bconv2d(PyObject *const *a)
{
    const Desc desc(a[0]);
    const lce_bconv2d_desc &d = *desc.d;
    int32_t oh = 0, ow = 0;
    check(lce_bconv2d_out_shape(&d, &oh, &ow), "lce_bconv2d_out_shape");
    const at::Tensor &input = tensor(a[1], "input"), &weights = tensor(a[2], "weights");
    const at::ScalarType out_dtype = d.out_type == LCE_OUT_FLOAT32 ? at::kFloat : at::kInt;
    at::Tensor made;
    if (a[6] == Py_None)
        made = empty_like_device({d.batch, oh, ow, d.out_type == LCE_OUT_BITPACKED ? words(d.out_c) : (int64_t)d.out_c}, out_dtype, input);
    const at::Tensor &out = a[6] == Py_None ? made : tensor(a[6], "out");
    const int64_t want_in = (int64_t)d.batch * d.in_h * d.in_w * (F32 ? (int64_t)d.in_c : words(d.in_c));
    const int64_t want_w = d.weights_packed ? (int64_t)(lce_bconv2d_packed_weights_bytes(&d) / 4)
                                            : (int64_t)d.out_c * d.kernel_h * d.kernel_w * words(d.in_c);
    if (input.numel() != want_in || weights.numel() != want_w) value_error("input / weights size does not match the descriptor");
    void *pi = device_pointer(input, F32 ? at::kFloat : at::kInt, "input");
    auto *pw = static_cast<const uint32_t *>(device_pointer(weights, at::kInt, "weights"));
    auto *pm = static_cast<const float *>(device_pointer(a[3], at::kFloat, "multiplier"));
    auto *pb = static_cast<const float *>(device_pointer(a[4], at::kFloat, "bias"));
    auto *pt = static_cast<const int32_t *>(device_pointer(a[5], at::kInt, "thresholds"));
    void *po = device_pointer(out, out_dtype, "out");
    void *s = current_stream();
    if (F32)
        check(without_gil([&] { return lce_bconv2d_f32(&d, static_cast<const float *>(pi), pw, pm, pb, pt, po, s); }), "lce_bconv2d_f32");
    else
        check(without_gil([&] { return lce_bconv2d(&d, static_cast<const uint32_t *>(pi), pw, pm, pb, pt, po, s); }), "lce_bconv2d");
    return returned(a[6], made);
}

PyObject *bconv2d_fused(PyObject *const *a)  // desc, input, weights, multiplier, bias, residual, out_float, out_packed
{
    const Desc desc(a[0]);
    auto *pi = static_cast<const uint32_t *>(device_pointer(tensor(a[1], "input"), at::kInt, "input"));
    auto *pw = static_cast<const uint32_t *>(device_pointer(tensor(a[2], "weights"), at::kInt, "weights"));
    auto *pm = static_cast<const float *>(device_pointer(tensor(a[3], "multiplier"), at::kFloat, "multiplier"));
    auto *pb = static_cast<const float *>(device_pointer(tensor(a[4], "bias"), at::kFloat, "bias"));
    auto *pr = static_cast<const float *>(device_pointer(a[5], at::kFloat, "residual"));
    auto *pf = static_cast<float *>(device_pointer(a[6], at::kFloat, "out_float"));
    auto *pp = static_cast<uint32_t *>(device_pointer(a[7], at::kInt, "out_packed"));
    void *s = current_stream();
    check(without_gil([&] { return lce_bconv2d_fused(desc.d, pi, pw, pm, pb, pr, pf, pp, s); }), "lce_bconv2d_fused");
    Py_RETURN_NONE;
}

PyObject *plan_run(PyObject *const *a)  // handle (int or None)
{
    void *h = a[0] == Py_None ? nullptr : PyLong_AsVoidPtr(a[0]);
    if (PyErr_Occurred()) throw Raised{};
    void *s = current_stream();
    check(without_gil([&] { return lce_plan_run(static_cast<const lce_plan *>(h), s); }), "lce_plan_run");
    Py_RETURN_NONE;
}

PyObject *bmaxpool(PyObject *const *a)  // words, channels, pool_h, pool_w, stride_h, stride_w, padding, out
{
    const at::Tensor &w = tensor(a[0], "words");
    int32_t v[6];
    for (int i = 0; i < 6; ++i) {
        const long x = PyLong_AsLong(a[1 + i]);
        if (x == -1 && PyErr_Occurred()) throw Raised{};
        v[i] = (int32_t)x;
    }
    if (w.dim() != 4) value_error("words must be [N, H, W, words per pixel]");
    const int64_t N = w.size(0), H = w.size(1), W = w.size(2), Cw = w.size(3);
    if (Cw != words(v[0])) value_error("last dimension does not match channels");
    at::Tensor made;
    if (a[7] == Py_None) {
        if (v[3] == 0 || v[4] == 0) {
            PyErr_SetString(PyExc_ZeroDivisionError, "integer division or modulo by zero");
            throw Raised{};
        }
        const auto extent = [&](int64_t size, int64_t k, int64_t s) {
            if (v[5] == LCE_PAD_VALID) return size >= k ? (size - k) / s + 1 : (int64_t)0;
            return (size + s - 1) / s;
        };
        made = empty_like_device({N, extent(H, v[1], v[3]), extent(W, v[2], v[4]), Cw}, at::kInt, w);
    }
    const at::Tensor &out = a[7] == Py_None ? made : tensor(a[7], "out");
    auto *pw = static_cast<const uint32_t *>(device_pointer(w, at::kInt, "words"));
    auto *po = static_cast<uint32_t *>(device_pointer(out, at::kInt, "out"));
    void *s = current_stream();
    check(without_gil([&] { return lce_bmaxpool(pw, po, (int32_t)N, (int32_t)H, (int32_t)W, v[0], v[1], v[2], v[3], v[4], v[5], s); }), "lce_bmaxpool");
    return returned(a[7], made);
}

PyObject *add_f32(PyObject *const *args)  // a, b, out
{
    const at::Tensor &a = tensor(args[0], "a"), &b = tensor(args[1], "b");
    at::Tensor made;
    if (args[2] == Py_None) made = empty_like_device(a.sizes(), a.scalar_type(), a);
    const at::Tensor &out = args[2] == Py_None ? made : tensor(args[2], "out");
    if (a.numel() != b.numel() || a.numel() != out.numel()) value_error("size mismatch");
    auto *pa = static_cast<const float *>(device_pointer(a, at::kFloat, "a"));
    auto *pb = static_cast<const float *>(device_pointer(b, at::kFloat, "b"));
    auto *po = static_cast<float *>(device_pointer(out, at::kFloat, "out"));
    const int64_t n = a.numel();
    void *s = current_stream();
    check(without_gil([&] { return lce_add_f32(pa, pb, po, n, s); }), "lce_add_f32");
    return returned(args[2], made);
}

// desc, input, weights, multiplier, bias, thresholds, out, workspace
template <bool ASYNC>
PyObject *bconv2d_host(PyObject *const *a)
{
    const Desc desc(a[0]);
    auto *pi = static_cast<const uint32_t *>(host_pointer(a[1], at::kInt, "input"));
    auto *pw = static_cast<const uint32_t *>(host_pointer(a[2], at::kInt, "weights"));
    auto *pm = static_cast<const float *>(host_pointer(a[3], at::kFloat, "multiplier"));
    auto *pb = static_cast<const float *>(host_pointer(a[4], at::kFloat, "bias"));
    auto *pt = static_cast<const int32_t *>(host_pointer(a[5], at::kInt, "thresholds"));
    void *po = host_pointer(a[6], desc.d->out_type == LCE_OUT_FLOAT32 ? at::kFloat : at::kInt, "out");
    const at::Tensor &ws = tensor(a[7], "workspace");
    void *pws = device_pointer(ws, at::kByte, "workspace");
    const size_t bytes = (size_t)ws.numel();
    void *s = current_stream();
    if (ASYNC)
        check(without_gil([&] { return lce_bconv2d_host_async(desc.d, pi, pw, pm, pb, pt, po, pws, bytes, s); }), "lce_bconv2d_host_async");
    else
        check(without_gil([&] { return lce_bconv2d_host(desc.d, pi, pw, pm, pb, pt, po, pws, bytes, s); }), "lce_bconv2d_host");
    Py_RETURN_NONE;
}

// --- key/value cache, attention, residual norm: three element types, rows with strides ------------------------

int32_t element_type(const at::Tensor &t, const char *name)
{
    switch (t.scalar_type()) {
        case at::kFloat: return LCE_TYPE_FLOAT32;
        case at::kHalf: return LCE_TYPE_FLOAT16;
        case at::kBFloat16: return LCE_TYPE_BFLOAT16;
        default: value_error(std::string(name) + " must be torch.float32, torch.float16 or torch.bfloat16");
    }
}

// These calls' tensors live on the device whose stream they are enqueued on.
void on_current_device(const at::Tensor &t, const char *name)
{
    if (!t.is_cuda()) value_error(std::string(name) + " must be a CUDA tensor (there is no CPU path)");
    if (t.device().index() != c10::cuda::current_device()) value_error(std::string(name) + " must be on the current CUDA device");
}

void *current_device_pointer(PyObject *o, at::ScalarType dtype, const char *name)  // None -> null
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    on_current_device(t, name);
    return device_pointer(t, dtype, name);
}

template <typename T>
struct Buffer {  // a ctypes structure with the layout of T
    Py_buffer view{};
    T d{};
    Buffer(PyObject *o, const char *what)
    {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Raised{};
        const bool fits = view.len == (Py_ssize_t)sizeof(T);
        if (fits) d = *static_cast<const T *>(view.buf);
        PyBuffer_Release(&view);
        if (!fits) {
            PyErr_Format(PyExc_TypeError, "desc must be a %s", what);
            throw Raised{};
        }
    }
};

struct Rows {  // [tokens][heads][channels], channels next to one another
    char *data;
    int64_t tokens, token_stride, head_stride;
};

Rows rows(const at::Tensor &t, int64_t heads, int64_t channels, const char *name)
{
    on_current_device(t, name);
    if (t.dim() != 3 || t.size(1) != heads || t.size(2) != channels || (channels > 1 && t.size(0) > 0 && t.stride(2) != 1))
        value_error(std::string(name) + " must be [tokens, " + std::to_string(heads) + ", " + std::to_string(channels) + "] with its channels next to one another");
    return {static_cast<char *>(t.data_ptr()), t.size(0), t.stride(0), t.stride(1)};
}

void cache_fits(const at::Tensor &cache, const lce_kv_desc &d)
{
    on_current_device(cache, "cache");
    if ((uint64_t)cache.numel() != (uint64_t)lce_kv_cache_bytes(&d)) value_error("cache size does not match the descriptor");
}

PyObject *kv_quantize(PyObject *const *a)  // desc, k, v, slots, cache
{
    const Buffer<lce_kv_desc> desc(a[0], "KvDesc");
    const lce_kv_desc &d = desc.d;
    const at::Tensor &tk = tensor(a[1], "k"), &tv = tensor(a[2], "v"), &slots = tensor(a[3], "slots"), &cache = tensor(a[4], "cache");
    const Rows k = rows(tk, d.kv_heads, d.head_dim, "k"), v = rows(tv, d.kv_heads, d.head_dim, "v");
    const int32_t type = element_type(tk, "k");
    if (element_type(tv, "v") != type || v.tokens != k.tokens) value_error("k and v must be alike");
    auto *ps = static_cast<const int32_t *>(current_device_pointer(a[3], at::kInt, "slots"));
    if (slots.numel() != k.tokens) value_error("slots must have one entry for each token");
    cache_fits(cache, d);
    void *pc = device_pointer(cache, at::kByte, "cache"), *s = current_stream();
    check(without_gil([&] {
              return lce_kv_quantize(&d, k.data, v.data, type, k.tokens, k.token_stride, k.head_stride, v.token_stride, v.head_stride, ps, pc, s);
          }), "lce_kv_quantize");
    Py_RETURN_NONE;
}

at::ScalarType scalar_type(int32_t type) { return type == LCE_TYPE_FLOAT32 ? at::kFloat : type == LCE_TYPE_FLOAT16 ? at::kHalf : at::kBFloat16; }

PyObject *kv_dequantize(PyObject *const *a)  // desc, cache, slots, type, k, v
{
    const Buffer<lce_kv_desc> desc(a[0], "KvDesc");
    const lce_kv_desc &d = desc.d;
    const at::Tensor &cache = tensor(a[1], "cache"), &slots = tensor(a[2], "slots");
    auto *ps = static_cast<const int32_t *>(current_device_pointer(a[2], at::kInt, "slots"));
    cache_fits(cache, d);
    const long type = PyLong_AsLong(a[3]);
    if (type == -1 && PyErr_Occurred()) throw Raised{};
    if (type < LCE_TYPE_FLOAT32 || type > LCE_TYPE_BFLOAT16) value_error("dtype must be torch.float32, torch.float16 or torch.bfloat16");
    const int64_t tokens = slots.numel();
    at::Tensor made[2];
    void *out[2];
    for (int i = 0; i < 2; ++i) {
        const char *name = i ? "v" : "k";
        if (a[4 + i] == Py_None) made[i] = empty_like_device({tokens, d.kv_heads, d.head_dim}, scalar_type((int32_t)type), cache);
        const at::Tensor &t = a[4 + i] == Py_None ? made[i] : tensor(a[4 + i], name);
        const Rows r = rows(t, d.kv_heads, d.head_dim, name);
        if (r.tokens != tokens || t.scalar_type() != scalar_type((int32_t)type) || !t.is_contiguous())
            value_error(std::string(name) + " must be contiguous, of the dtype asked for, with a row for each slot");
        out[i] = r.data;
    }
    void *pc = device_pointer(cache, at::kByte, "cache"), *s = current_stream();
    check(without_gil([&] { return lce_kv_dequantize(&d, pc, ps, tokens, (int32_t)type, out[0], out[1], s); }), "lce_kv_dequantize");
    PyObject *k = returned(a[4], made[0]), *v = returned(a[5], made[1]);
    PyObject *both = PyTuple_Pack(2, k, v);
    Py_XDECREF(k);
    Py_XDECREF(v);
    return both;
}

// desc (KvDesc), q, cache, page_table, lengths, q_starts, scale, causal, window, out, workspace
PyObject *kv_attention(PyObject *const *a)
{
    const Buffer<lce_kv_desc> desc(a[0], "KvDesc");
    lce_kv_attention_desc d{};
    d.cache = desc.d;
    const at::Tensor &tq = tensor(a[1], "q"), &cache = tensor(a[2], "cache"), &table = tensor(a[3], "page_table"), &lengths = tensor(a[4], "lengths");
    if (tq.dim() != 3) value_error("q must be [tokens, heads, head_dim]");
    d.heads = (int32_t)tq.size(1);
    const Rows q = rows(tq, d.heads, d.cache.head_dim, "q");
    d.type = element_type(tq, "q");
    cache_fits(cache, d.cache);
    auto *pt = static_cast<const int32_t *>(current_device_pointer(a[3], at::kInt, "page_table"));
    auto *pl = static_cast<const int32_t *>(current_device_pointer(a[4], at::kInt, "lengths"));
    auto *pq = static_cast<const int32_t *>(current_device_pointer(a[5], at::kInt, "q_starts"));
    if (table.dim() != 2 || lengths.numel() != table.size(0)) value_error("page_table must be [sequences, pages] and lengths have an entry for each sequence");
    if (pq && tensor(a[5], "q_starts").numel() != table.size(0) + 1) value_error("q_starts must have one entry more than there are sequences");
    if (!pq && q.tokens != table.size(0)) value_error("without q_starts q must have one row for each sequence");
    if (table.size(0) >= (1ll << 31) || table.size(1) >= (1ll << 31) || tq.size(1) >= (1ll << 31)) value_error("page_table or q is too large");
    d.batch = (int32_t)table.size(0);
    d.table_pages = (int32_t)table.size(1);
    d.tokens = q.tokens;
    const double scale = PyFloat_AsDouble(a[6]);
    const int causal = PyObject_IsTrue(a[7]);
    const long window = PyLong_AsLong(a[8]);
    if (PyErr_Occurred()) throw Raised{};
    if (window < 0 || window >= (1ll << 31)) value_error("window must not be negative");
    d.scale = (float)scale;
    d.causal = causal;
    d.window = (int32_t)window;
    at::Tensor made, room;
    if (a[9] == Py_None) made = empty_like_device({q.tokens, d.heads, d.cache.head_dim}, tq.scalar_type(), tq);
    const at::Tensor &to = a[9] == Py_None ? made : tensor(a[9], "out");
    const Rows out = rows(to, d.heads, d.cache.head_dim, "out");
    if (out.tokens != q.tokens || to.scalar_type() != tq.scalar_type()) value_error("out must be like q");
    d.q_token_stride = q.token_stride; d.q_head_stride = q.head_stride;
    d.out_token_stride = out.token_stride; d.out_head_stride = out.head_stride;
    if (d.batch == 0 || d.tokens == 0) return returned(a[9], made);
    if (a[10] == Py_None) room = empty_like_device({(int64_t)lce_kv_attention_workspace_bytes(&d)}, at::kByte, tq);
    const at::Tensor &ws = a[10] == Py_None ? room : tensor(a[10], "workspace");
    on_current_device(ws, "workspace");
    void *pw = device_pointer(ws, at::kByte, "workspace"), *pc = device_pointer(cache, at::kByte, "cache"), *s = current_stream();
    const size_t bytes = (size_t)ws.numel();
    check(without_gil([&] { return lce_kv_attention(&d, q.data, pc, pt, pl, pq, out.data, pw, bytes, s); }), "lce_kv_attention");
    return returned(a[9], made);
}

// Rows [sequences][heads][tokens] of fp32 numbers, a row's tokens next to one another; None -> null.
float *token_rows(PyObject *o, int64_t sequences, int64_t heads, int64_t tokens, int64_t *seq_stride, int64_t *head_stride, const char *name)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    on_current_device(t, name);
    if (t.scalar_type() != at::kFloat) value_error(std::string(name) + " must be torch.float32");
    if (t.dim() != 3 || t.size(0) != sequences || t.size(1) != heads || t.size(2) < tokens || (t.size(2) > 1 && t.stride(2) != 1))
        value_error(std::string(name) + " must be [" + std::to_string(sequences) + ", " + std::to_string(heads) + ", " + std::to_string(tokens) +
                    " or more] with a row's tokens next to one another");
    *seq_stride = t.stride(0);
    *head_stride = t.stride(1);
    return static_cast<float *>(t.data_ptr());
}

// A page table [sequences][pages] and an entry for each sequence.
const int32_t *page_table(PyObject *o, const char *name, int32_t *sequences, int32_t *pages)
{
    auto *p = static_cast<const int32_t *>(current_device_pointer(o, at::kInt, name));
    const at::Tensor &t = tensor(o, name);
    if (t.dim() != 2) value_error(std::string(name) + " must be [sequences, pages]");
    if (t.size(0) >= (1ll << 31) || t.size(1) >= (1ll << 31)) value_error(std::string(name) + " is too large");
    *sequences = (int32_t)t.size(0);
    *pages = (int32_t)t.size(1);
    return p;
}

int32_t int_argument(PyObject *o, const char *name)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    if (v < -(1ll << 31) || v >= (1ll << 31)) value_error(std::string(name) + " does not fit 32 bits");
    return (int32_t)v;
}

// desc, q, k, positions, steps, q_out, k_out
PyObject *rotary(PyObject *const *a)
{
    const Buffer<lce_rotary_desc> desc(a[0], "RotaryDesc");
    lce_rotary_desc d = desc.d;
    const at::Tensor &tq = tensor(a[1], "q");
    if (tq.dim() != 3) value_error("q must be [tokens, heads, head_dim]");
    if (tq.size(1) >= (1ll << 31)) value_error("q is too large");
    d.q_heads = (int32_t)tq.size(1);
    d.type = element_type(tq, "q");
    const Rows q = rows(tq, d.q_heads, d.head_dim, "q");
    d.tokens = q.tokens;
    auto *pp = static_cast<const int32_t *>(current_device_pointer(a[3], at::kInt, "positions"));
    if (a[3] == Py_None || tensor(a[3], "positions").numel() != d.tokens) value_error("positions must have one entry for each token");
    auto *ps = static_cast<const uint64_t *>(current_device_pointer(a[4], at::kLong, "steps"));
    if (a[4] == Py_None || tensor(a[4], "steps").numel() != d.rotary_dim / 2) value_error("steps must have one entry for each pair of channels");
    at::Tensor made[2];
    Rows in[2] = {q, {nullptr, 0, 0, 0}}, out[2] = {};
    const char *names[2] = {"q_out", "k_out"};
    if (a[2] != Py_None) {
        const at::Tensor &tk = tensor(a[2], "k");
        if (tk.dim() != 3) value_error("k must be [tokens, heads, head_dim]");
        if (tk.size(1) >= (1ll << 31)) value_error("k is too large");
        d.k_heads = (int32_t)tk.size(1);
        in[1] = rows(tk, d.k_heads, d.head_dim, "k");
        if (element_type(tk, "k") != d.type || in[1].tokens != d.tokens) value_error("k must be of q's type and have its tokens");
    } else if (a[6] != Py_None) {
        value_error("k_out without k");
    }
    for (int i = 0; i < 2; ++i) {
        const int64_t heads = i ? d.k_heads : d.q_heads;
        if (i && a[2] == Py_None) continue;
        if (a[5 + i] == Py_None) made[i] = empty_like_device({d.tokens, heads, d.head_dim}, tq.scalar_type(), tq);
        const at::Tensor &t = a[5 + i] == Py_None ? made[i] : tensor(a[5 + i], names[i]);
        out[i] = rows(t, heads, d.head_dim, names[i]);
        if (out[i].tokens != d.tokens || t.scalar_type() != tq.scalar_type()) value_error(std::string(names[i]) + " must be like what it is made from");
        if (out[i].data == in[i].data && d.tokens > 0 && ((d.tokens > 1 && out[i].token_stride != in[i].token_stride) || (heads > 1 && out[i].head_stride != in[i].head_stride)))
            value_error(std::string(names[i]) + " in place must have the strides of what it is made from");
    }
    d.q_token_stride = in[0].token_stride; d.q_head_stride = in[0].head_stride;
    d.k_token_stride = in[1].token_stride; d.k_head_stride = in[1].head_stride;
    d.q_out_token_stride = out[0].token_stride; d.q_out_head_stride = out[0].head_stride;
    d.k_out_token_stride = out[1].token_stride; d.k_out_head_stride = out[1].head_stride;
    void *s = current_stream();
    check(without_gil([&] { return lce_rotary(&d, in[0].data, in[1].data, pp, ps, out[0].data, out[1].data, s); }), "lce_rotary");
    PyObject *qo = returned(a[5], made[0]), *ko;
    if (a[2] == Py_None) {
        Py_INCREF(Py_None);
        ko = Py_None;
    } else {
        ko = returned(a[6], made[1]);
    }
    PyObject *both = PyTuple_Pack(2, qo, ko);
    Py_XDECREF(qo);
    Py_XDECREF(ko);
    return both;
}

// desc (KvDesc), q, cache, page_table, lengths, q_starts, previous, out, scale, causal, window, decay, workspace
PyObject *kv_attention_weights(PyObject *const *a)
{
    const Buffer<lce_kv_desc> desc(a[0], "KvDesc");
    lce_kv_attention_weights_desc d{};
    d.cache = desc.d;
    const at::Tensor &tq = tensor(a[1], "q"), &cache = tensor(a[2], "cache"), &lengths = tensor(a[4], "lengths");
    if (tq.dim() != 3) value_error("q must be [tokens, heads, head_dim]");
    if (tq.size(1) >= (1ll << 31)) value_error("q is too large");
    d.heads = (int32_t)tq.size(1);
    const Rows q = rows(tq, d.heads, d.cache.head_dim, "q");
    d.type = element_type(tq, "q");
    d.tokens = q.tokens;
    d.q_token_stride = q.token_stride; d.q_head_stride = q.head_stride;
    cache_fits(cache, d.cache);
    auto *pt = page_table(a[3], "page_table", &d.batch, &d.table_pages);
    auto *pl = static_cast<const int32_t *>(current_device_pointer(a[4], at::kInt, "lengths"));
    auto *pq = static_cast<const int32_t *>(current_device_pointer(a[5], at::kInt, "q_starts"));
    if (lengths.numel() != d.batch) value_error("lengths must have an entry for each sequence");
    if (pq && tensor(a[5], "q_starts").numel() != (int64_t)d.batch + 1) value_error("q_starts must have one entry more than there are sequences");
    if (!pq && q.tokens != d.batch) value_error("without q_starts q must have one row for each sequence");
    const int64_t room_for = (int64_t)d.table_pages * d.cache.page_size;
    at::Tensor made, room;
    const float *previous = token_rows(a[6], d.batch, d.cache.kv_heads, room_for, &d.previous_seq_stride, &d.previous_head_stride, "previous");
    float *out;
    if (a[7] == Py_None) {
        made = empty_like_device({d.batch, d.cache.kv_heads, room_for}, at::kFloat, tq);
        out = static_cast<float *>(made.data_ptr());
        d.out_seq_stride = made.stride(0);
        d.out_head_stride = made.stride(1);
    } else {
        out = token_rows(a[7], d.batch, d.cache.kv_heads, room_for, &d.out_seq_stride, &d.out_head_stride, "out");
    }
    if (previous == out && previous && (d.previous_seq_stride != d.out_seq_stride || d.previous_head_stride != d.out_head_stride))
        value_error("out in place must have the strides of previous");
    const double scale = PyFloat_AsDouble(a[8]), decay = PyFloat_AsDouble(a[11]);
    const int causal = PyObject_IsTrue(a[9]);
    if (PyErr_Occurred()) throw Raised{};
    const int32_t window = int_argument(a[10], "window");
    if (window < 0) value_error("window must not be negative");
    d.scale = (float)scale;
    d.decay = (float)decay;
    d.causal = causal;
    d.window = window;
    if (d.batch == 0 || room_for == 0) return returned(a[7], made);
    const lce::RowSet out_rows{out, d.batch, d.cache.kv_heads, d.out_seq_stride, d.out_head_stride, room_for, 4};
    if (!lce::rows_apart(out_rows)) value_error("out must have rows apart from one another");
    if (previous && previous != out && d.decay != 0.0f &&
        lce::rows_meet({previous, d.batch, d.cache.kv_heads, d.previous_seq_stride, d.previous_head_stride, room_for, 4}, out_rows))
        value_error("out must be previous itself, with its strides, or other memory");
    if (a[12] == Py_None) room = empty_like_device({(int64_t)lce_kv_attention_weights_workspace_bytes(&d)}, at::kByte, tq);
    const at::Tensor &ws = a[12] == Py_None ? room : tensor(a[12], "workspace");
    on_current_device(ws, "workspace");
    void *pw = device_pointer(ws, at::kByte, "workspace"), *pc = device_pointer(cache, at::kByte, "cache"), *s = current_stream();
    const size_t bytes = (size_t)ws.numel();
    check(without_gil([&] { return lce_kv_attention_weights(&d, q.data, pc, pt, pl, pq, previous, out, pw, bytes, s); }), "lce_kv_attention_weights");
    return returned(a[7], made);
}

// desc (KvDesc), cache, page_table, lengths, scores, kept_table, budget, first, recent, kept, kept_lengths, kept_scores
PyObject *kv_evict(PyObject *const *a)
{
    const Buffer<lce_kv_desc> desc(a[0], "KvDesc");
    lce_kv_evict_desc d{};
    d.cache = desc.d;
    const at::Tensor &cache = tensor(a[1], "cache"), &lengths = tensor(a[3], "lengths");
    cache_fits(cache, d.cache);
    auto *pt = page_table(a[2], "page_table", &d.batch, &d.table_pages);
    int32_t sequences;
    auto *pk = page_table(a[5], "kept_table", &sequences, &d.kept_pages);
    if (sequences != d.batch) value_error("kept_table must have a row for each sequence");
    auto *pl = static_cast<const int32_t *>(current_device_pointer(a[3], at::kInt, "lengths"));
    if (lengths.numel() != d.batch) value_error("lengths must have an entry for each sequence");
    d.budget = int_argument(a[6], "budget");
    d.first = int_argument(a[7], "first");
    d.recent = int_argument(a[8], "recent");
    if (d.budget <= 0) value_error("budget must be positive");
    const int64_t heads = d.cache.kv_heads, shape[3] = {d.batch, heads, d.budget};
    const float *ps = token_rows(a[4], d.batch, heads, (int64_t)d.table_pages * d.cache.page_size, &d.scores_seq_stride, &d.scores_head_stride, "scores");
    if (!ps && d.batch > 0) value_error("scores must be given");
    at::Tensor made[3];
    int32_t *whole[2];
    for (int i = 0; i < 2; ++i) {
        const at::IntArrayRef wanted(shape, i ? 1 : 3);
        const char *name = i ? "kept_lengths" : "kept";
        if (a[9 + i] == Py_None) made[i] = empty_like_device(wanted, at::kInt, cache);
        const at::Tensor &t = a[9 + i] == Py_None ? made[i] : tensor(a[9 + i], name);
        on_current_device(t, name);
        whole[i] = static_cast<int32_t *>(device_pointer(t, at::kInt, name));
        if (t.sizes() != wanted) value_error(std::string(name) + (i ? " must have an entry for each sequence" : " must be [sequences, kv_heads, budget]"));
    }
    float *pks;
    if (a[11] == Py_None) {
        made[2] = empty_like_device(at::IntArrayRef(shape, 3), at::kFloat, cache);
        pks = static_cast<float *>(made[2].data_ptr());
        d.kept_scores_seq_stride = made[2].stride(0);
        d.kept_scores_head_stride = made[2].stride(1);
    } else {
        pks = token_rows(a[11], d.batch, heads, d.budget, &d.kept_scores_seq_stride, &d.kept_scores_head_stride, "kept_scores");
        const lce::RowSet kept_rows{pks, d.batch, heads, d.kept_scores_seq_stride, d.kept_scores_head_stride, d.budget, 4};
        if (!lce::rows_apart(kept_rows)) value_error("kept_scores must have rows apart from one another");
        if (lce::rows_meet({ps, d.batch, heads, d.scores_seq_stride, d.scores_head_stride, (int64_t)d.table_pages * d.cache.page_size, 4}, kept_rows))
            value_error("kept_scores must not be memory of scores");
    }
    void *pc = device_pointer(cache, at::kByte, "cache"), *s = current_stream();
    if (d.batch > 0) check(without_gil([&] { return lce_kv_evict(&d, pc, pt, pl, ps, pk, whole[0], whole[1], pks, s); }), "lce_kv_evict");
    PyObject *out[3];
    for (int i = 0; i < 3; ++i) out[i] = returned(a[9 + i], made[i]);
    PyObject *all = PyTuple_Pack(3, out[0], out[1], out[2]);
    for (PyObject *o : out) Py_XDECREF(o);
    return all;
}

// Rows of `channels` elements next to one another: any tensor whose leading axes are one run of rows.
char *norm_rows(PyObject *o, const lce_residual_norm_desc &d, at::ScalarType dtype, bool one_row_for_all, int64_t *stride, const char *name)
{
    *stride = d.channels;
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    on_current_device(t, name);
    if (t.scalar_type() != dtype) value_error(std::string(name) + " has another dtype than its neighbours");
    if (t.dim() == 0 || t.size(-1) != d.channels || (d.channels > 1 && t.stride(-1) != 1)) value_error(std::string(name) + " must have its channels last and next to one another");
    const int64_t n = t.numel() / d.channels;
    if (one_row_for_all && n == 1) *stride = 0;
    else if (n != d.rows) value_error(std::string(name) + " has another number of rows than the descriptor");
    else if (t.dim() == 2) *stride = n == 1 ? d.channels : t.stride(0);
    else if (!t.is_contiguous()) value_error(std::string(name) + " must be [rows, channels] or contiguous");
    return static_cast<char *>(t.data_ptr());
}

// desc, x, branch, gate, post_weight, post_bias, pre_weight, pre_bias, y, normed, packed
PyObject *residual_norm(PyObject *const *a)
{
    const Buffer<lce_residual_norm_desc> desc(a[0], "ResidualNormDesc");
    lce_residual_norm_desc d = desc.d;
    if (d.channels <= 0) check(LCE_ERR_INVALID_ARG, "lce_residual_norm");
    const at::Tensor &x = tensor(a[1], "x");
    d.stream_type = element_type(x, "x");
    d.type = a[2] != Py_None ? element_type(tensor(a[2], "branch"), "branch") : a[9] != Py_None ? element_type(tensor(a[9], "normed"), "normed") : d.stream_type;
    const at::ScalarType stream_dtype = scalar_type(d.stream_type), dtype = scalar_type(d.type);
    const char *px = norm_rows(a[1], d, stream_dtype, false, &d.x_stride, "x"), *pb = norm_rows(a[2], d, dtype, false, &d.branch_stride, "branch"),
               *pg = norm_rows(a[3], d, dtype, true, &d.gate_stride, "gate");
    const float *w[4];
    const char *names[4] = {"post_weight", "post_bias", "pre_weight", "pre_bias"};
    for (int i = 0; i < 4; ++i) {
        w[i] = static_cast<const float *>(current_device_pointer(a[4 + i], at::kFloat, names[i]));
        if (w[i] && tensor(a[4 + i], names[i]).numel() != d.channels) value_error(std::string(names[i]) + " must have an entry for each channel");
    }
    char *py = norm_rows(a[8], d, stream_dtype, false, &d.y_stride, "y"), *pn = norm_rows(a[9], d, dtype, false, &d.normed_stride, "normed");
    auto *pp = static_cast<uint32_t *>(current_device_pointer(a[10], at::kInt, "packed"));
    if (pp && tensor(a[10], "packed").numel() != d.rows * words(d.channels)) value_error("packed must have a word for every 32 channels of each row");
    void *s = current_stream();
    check(without_gil([&] { return lce_residual_norm(&d, px, pb, pg, w[0], w[1], w[2], w[3], py, pn, pp, s); }), "lce_residual_norm");
    Py_RETURN_NONE;
}

PyObject *setup(PyObject *const *a)  // LceError
{
    Py_INCREF(a[0]);
    Py_XSETREF(g_lce_error, a[0]);
    Py_RETURN_NONE;
}

#define LCE_METHOD(name, body, n) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<body, n>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    LCE_METHOD("setup", setup, 1),
    LCE_METHOD("bitpack", bitpack, 2),
    LCE_METHOD("unpack", unpack, 3),
    LCE_METHOD("bconv2d", bconv2d<false>, 7),
    LCE_METHOD("bconv2d_f32", bconv2d<true>, 7),
    LCE_METHOD("bconv2d_fused", bconv2d_fused, 8),
    LCE_METHOD("plan_run", plan_run, 1),
    LCE_METHOD("bmaxpool", bmaxpool, 8),
    LCE_METHOD("add_f32", add_f32, 3),
    LCE_METHOD("bconv2d_host", bconv2d_host<false>, 8),
    LCE_METHOD("bconv2d_host_async", bconv2d_host<true>, 8),
    LCE_METHOD("kv_quantize", kv_quantize, 5),
    LCE_METHOD("kv_dequantize", kv_dequantize, 6),
    LCE_METHOD("kv_attention", kv_attention, 11),
    LCE_METHOD("rotary", rotary, 7),
    LCE_METHOD("kv_attention_weights", kv_attention_weights, 13),
    LCE_METHOD("kv_evict", kv_evict, 12),
    LCE_METHOD("residual_norm", residual_norm, 11),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_lce_host", "Native call path of the binding (see binding.py).", -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lce_host() { return PyModule_Create(&g_module); }
