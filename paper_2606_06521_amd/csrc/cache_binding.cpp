// Python module _cache_binding: the cache calls of attn_fp8_cache.h on torch
// tensors.  Checks the tensors' types, shapes and places, allocates outputs and the
// workspace with torch, passes the current stream; everything else is the
// library's.  Native because a short call is host time: the same in Python takes
// 9 to 12 us of it, the launch itself 3.
//
// A function returns its outputs, or the library's status if that is not 0.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>

#include <array>
#include <cmath>
#include <string>

#include "../../include/attn_fp8_cache.h"

namespace {

[[noreturn]] void raise(PyObject* type, const std::string& what)
{
    PyErr_SetString(type, what.c_str());
    throw python_error();
}

[[noreturn]] void value_error(const std::string& what) { raise(PyExc_ValueError, what); }
[[noreturn]] void type_error(const std::string& what) { raise(PyExc_TypeError, what); }

const at::Tensor& tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o))
        type_error(std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}

long long integer(PyObject* o)
{
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred())
        throw python_error();
    return x;
}

int narrow(long long x, const char* name)
{
    if (x < INT32_MIN || x > INT32_MAX)
        value_error(std::string(name) + " is out of range");
    return (int)x;
}

int int_arg(PyObject* o, const char* name) { return narrow(integer(o), name); }

float real(PyObject* o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred())
        throw python_error();
    return (float)x;
}

bool truth(PyObject* o)
{
    const int x = PyObject_IsTrue(o);
    if (x < 0)
        throw python_error();
    return x != 0;
}

// The device and stream of a call: the current ones, where the first tensor is.
struct Place {
    at::Device device;
    void* stream;
    explicit Place(const at::Tensor& t) : device(t.device()), stream(nullptr)
    {
        if (!t.is_cuda())
            value_error("tensors must be on the GPU");
        const c10::hip::HIPStream current = c10::hip::getCurrentHIPStream();
        if (current.device_index() != device.index())
            value_error("tensors are on " + device.str() + ", the current device is " + std::to_string(current.device_index()));
        stream = current.stream();
    }
    at::Tensor empty(at::IntArrayRef shape, at::ScalarType type) const
    {
        return at::empty(shape, at::TensorOptions().dtype(type).device(device));
    }
};

std::string shape_text(at::IntArrayRef s)
{
    std::string r = "[";
    for (size_t i = 0; i < s.size(); ++i)
        r += (i ? ", " : "") + std::to_string(s[i]);
    return r + "]";
}

// A contiguous tensor of this type and shape on the call's device.
template <typename T>
T* dense(const at::Tensor& t, const char* name, const Place& at, at::ScalarType type, at::IntArrayRef shape)
{
    if (t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous() || t.device() != at.device)
        value_error(std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor " + shape_text(shape) + " on " +
                    at.device.str());
    return static_cast<T*>(t.data_ptr());
}

int32_t* ints(PyObject* o, const char* name, const Place& at, at::IntArrayRef shape)
{
    return dense<int32_t>(tensor(o, name), name, at, at::kInt, shape);
}

bool is_codes(const at::Tensor& t) { return t.scalar_type() == at::kFloat8_e4m3fn || t.scalar_type() == at::kByte; }

attn_fp8_cache cache_of(PyObject* o, const Place& at)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4)
        type_error("a cache is a KVCache: k, v, k_scale, v_scale");
    const at::Tensor &k = tensor(PyTuple_GET_ITEM(o, 0), "k"), &v = tensor(PyTuple_GET_ITEM(o, 1), "v");
    const at::Tensor &ks = tensor(PyTuple_GET_ITEM(o, 2), "k_scale"), &vs = tensor(PyTuple_GET_ITEM(o, 3), "v_scale");
    if (k.dim() != 4 || v.sizes() != k.sizes() || ks.dim() != 2 || vs.sizes() != ks.sizes() || ks.size(0) != k.size(0) ||
        ks.size(1) != k.size(1))
        value_error("a cache has k, v [pages, Hkv, page, d] and k_scale, v_scale [pages, Hkv]");
    if (!is_codes(k) || !is_codes(v) || ks.scalar_type() != at::kByte || vs.scalar_type() != at::kByte)
        type_error("a cache has float8_e4m3fn (or uint8) codes and uint8 scales");
    for (const at::Tensor* t : {&k, &v, &ks, &vs})
        if (t->device() != at.device || !t->is_contiguous())
            value_error("a cache's tensors must be contiguous and on the inputs' device");
    return {k.data_ptr(),
            v.data_ptr(),
            static_cast<uint8_t*>(ks.data_ptr()),
            static_cast<uint8_t*>(vs.data_ptr()),
            narrow(k.size(0), "pages"),
            narrow(k.size(1), "Hkv"),
            narrow(k.size(2), "page"),
            narrow(k.size(3), "d")};
}

attn_fp8_batch batch_of(PyObject* pages, PyObject* lens, PyObject* cu, PyObject* max_q, int64_t T, const Place& at)
{
    const at::Tensor& p = tensor(pages, "pages");
    if (p.dim() != 2)
        value_error("pages must be [B, W]");
    const int64_t B = p.size(0);
    attn_fp8_batch bt{};
    bt.pages = ints(pages, "pages", at, p.sizes());
    bt.lens = ints(lens, "lens", at, {B});
    bt.B = narrow(B, "B");
    bt.W = narrow(p.size(1), "W");
    bt.T = narrow(T, "T");
    int64_t most = 0;
    if (cu == Py_None) {
        const int64_t n = B ? T / B : 0;
        if (B * n != T)
            value_error(std::to_string(T) + " tokens of " + std::to_string(B) + " sequences: give cu");
        most = max_q == Py_None ? n : integer(max_q);
        if (most < n)
            value_error("max_q = " + std::to_string(most) + ", but each sequence has " + std::to_string(n) + " new tokens");
    } else {
        if (max_q == Py_None)
            value_error("cu needs max_q, the most new tokens of a sequence");
        bt.cu = ints(cu, "cu", at, {B + 1});
        most = integer(max_q);
    }
    bt.max_q = narrow(most < 1 ? 1 : most, "max_q");
    return bt;
}

int type_of(at::ScalarType t)
{
    switch (t) {
    case at::kFloat:
        return ATTN_TYPE_F32;
    case at::kBFloat16:
        return ATTN_TYPE_BF16;
    case at::kHalf:
        return ATTN_TYPE_F16;
    case at::kFloat8_e4m3fn:
        return ATTN_TYPE_E4M3;
    default:
        return -1;
    }
}

bool is_input(at::ScalarType t) { return t == at::kFloat || t == at::kBFloat16 || t == at::kHalf; }

attn_fp8_heads heads_of(const at::Tensor& t, const char* name, const Place& at, bool right_type, const char* types)
{
    if (t.dim() != 3 || !right_type || t.device() != at.device || (t.size(2) > 1 && t.stride(2) != 1))
        value_error(std::string(name) + " must be [T, H, d] with contiguous channels on " + at.device.str() + ", of type " + types);
    // (a stride that no element is found by may be any number)
    return {t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0, t.size(1) > 1 ? t.stride(1) : 0, type_of(t.scalar_type())};
}

constexpr const char* kInputTypes = "float32, bfloat16 or float16";
constexpr const char* kQueryTypes = "bfloat16 or float8_e4m3fn";

attn_fp8_rotation rotation_of(PyObject* table, PyObject* positions, int layout, int64_t T, const Place& at)
{
    const at::Tensor& t = tensor(table, "table");
    if (t.dim() != 3 || t.size(2) != 2 || t.scalar_type() != at::kFloat || !t.is_contiguous() || t.device() != at.device)
        value_error("table must be a contiguous float32 tensor [positions, rot / 2, 2] on " + at.device.str());
    return {static_cast<const float*>(t.data_ptr()), positions == Py_None ? nullptr : ints(positions, "positions", at, {T}),
            narrow(t.size(0), "positions"), narrow(2 * t.size(1), "rot"), layout};
}

// `given`, or a new tensor of this shape and type.
at::Tensor out_heads(PyObject* given, const char* name, const Place& at, const at::Tensor& like, attn_fp8_heads& h)
{
    if (given == Py_None) {
        at::Tensor t = at.empty(like.sizes(), like.scalar_type());
        h = {t.data_ptr(), like.size(1) * like.size(2), like.size(2), type_of(like.scalar_type())};
        return t;
    }
    const at::Tensor& t = tensor(given, name);
    if (t.sizes() != like.sizes())
        value_error(std::string(name) + " must have the shape " + shape_text(like.sizes()));
    h = heads_of(t, name, at, t.scalar_type() == like.scalar_type(), c10::toString(like.scalar_type()));
    return t;
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

void count_args(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want)
        type_error("wrong number of arguments");
}

// rope(x, table, positions, layout, out)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_args(n, 5);
    const at::Tensor& x = tensor(a[0], "x");
    const Place at(x);
    const attn_fp8_heads hx = heads_of(x, "x", at, is_input(x.scalar_type()), kInputTypes);
    if (a[2] == Py_None)
        value_error("rope needs positions");
    const attn_fp8_rotation r = rotation_of(a[1], a[2], int_arg(a[3], "layout"), x.size(0), at);
    attn_fp8_heads ho;
    const at::Tensor out = out_heads(a[4], "out", at, x, ho);
    const int st = attn_fp8_rope(&hx, &ho, narrow(x.size(0), "T"), narrow(x.size(1), "H"), narrow(x.size(2), "d"), &r, at.stream);
    return st ? PyLong_FromLong(st) : wrap(out);
    END_HANDLE_TH_ERRORS
}

// append(cache, k, v, pages, lens, cu, max_q, table, positions, layout, q, q_out)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_args(n, 12);
    const at::Tensor &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    const Place at(k);
    const attn_fp8_cache c = cache_of(a[0], at);
    const attn_fp8_heads hk = heads_of(k, "k", at, is_input(k.scalar_type()), kInputTypes);
    const attn_fp8_heads hv = heads_of(v, "v", at, v.scalar_type() == k.scalar_type(), "k's");
    const int64_t T = k.size(0);
    if (k.sizes() != v.sizes() || k.size(1) != c.Hkv || k.size(2) != c.d)
        value_error("k, v must be [T, " + std::to_string(c.Hkv) + ", " + std::to_string(c.d) + "]");
    const attn_fp8_batch bt = batch_of(a[3], a[4], a[5], a[6], T, at);
    const bool rotates = a[7] != Py_None;
    attn_fp8_rotation r{};
    if (rotates)
        r = rotation_of(a[7], a[8], int_arg(a[9], "layout"), T, at);
    attn_fp8_heads hq{}, ho{};
    at::Tensor q_out;
    int Hq = 0;
    const bool with_q = a[10] != Py_None;
    if (with_q) {
        if (!rotates)
            value_error("q is rotated along: that needs a table");
        const at::Tensor& q = tensor(a[10], "q");
        hq = heads_of(q, "q", at, q.scalar_type() == k.scalar_type(), "k's");
        if (q.size(0) != T || q.size(2) != c.d)
            value_error("q must be [" + std::to_string(T) + ", Hq, " + std::to_string(c.d) + "]");
        Hq = narrow(q.size(1), "Hq");
        q_out = out_heads(a[11], "q_out", at, q, ho);
    }
    const int st = attn_fp8_cache_append(&c, &bt, &hk, &hv, rotates ? &r : nullptr, with_q ? &hq : nullptr, with_q ? &ho : nullptr, Hq,
                                         at.stream);
    if (st)
        return PyLong_FromLong(st);
    if (with_q)
        return wrap(q_out);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// What attention and weights share: q, cache, pages, lens, cu, max_q, sm_scale.
struct Queries {
    Place at;
    attn_fp8_cache c;
    attn_fp8_heads hq;
    attn_fp8_batch bt;
    int64_t T, Hq, d;
    float sm_scale;
    Queries(const at::Tensor& q, PyObject* cache, PyObject* pages, PyObject* lens, PyObject* cu, PyObject* max_q, PyObject* sm)
        : at(q), c(cache_of(cache, at)),
          hq(heads_of(q, "q", at, q.scalar_type() == at::kBFloat16 || q.scalar_type() == at::kFloat8_e4m3fn, kQueryTypes)),
          bt(batch_of(pages, lens, cu, max_q, q.size(0), at)), T(q.size(0)), Hq(q.size(1)), d(q.size(2))
    {
        if (d != c.d || c.Hkv < 1 || Hq % c.Hkv != 0)
            value_error("q must be [T, Hq, " + std::to_string(c.d) + "] with Hq a multiple of " + std::to_string(c.Hkv));
        narrow(Hq, "Hq");
        sm_scale = sm == Py_None ? (float)(1.0 / std::sqrt((double)d)) : real(sm);
    }
};

// fwd(q, cache, pages, lens, cu, max_q, causal, sm_scale, q_descale, max_len, out, out_type, lse, want_lse)
PyObject* fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_args(n, 14);
    const at::Tensor& q = tensor(a[0], "q");
    const Queries s(q, a[1], a[2], a[3], a[4], a[5], a[7]);
    const int max_len = int_arg(a[9], "max_len");
    at::Tensor out, lse, ws;
    if (a[10] == Py_None) {
        const int type = int_arg(a[11], "out_dtype");
        out = s.at.empty({s.T, s.Hq, s.d}, type == ATTN_TYPE_F32 ? at::kFloat : at::kBFloat16);
    } else {
        out = tensor(a[10], "out");
        if (out.sizes() != q.sizes() || !out.is_contiguous() || out.device() != s.at.device)
            value_error("out must be a contiguous tensor of q's shape on its device");
        if (out.scalar_type() != at::kBFloat16 && out.scalar_type() != at::kFloat)
            type_error("out is bfloat16 or float32");
    }
    if (a[12] != Py_None) {
        lse = tensor(a[12], "lse");
        dense<float>(lse, "lse", s.at, at::kFloat, {s.T, s.Hq});
    } else if (truth(a[13])) {
        lse = s.at.empty({s.T, s.Hq}, at::kFloat);
    }
    size_t bytes = 0;
    int st = attn_fp8_cache_workspace_bytes(&s.c, &s.bt, (int)s.Hq, max_len, &bytes);
    if (!st) {
        if (bytes)
            ws = s.at.empty({(int64_t)bytes}, at::kByte);
        st = attn_fp8_cache_fwd(&s.c, &s.bt, &s.hq, (int)s.Hq, out.data_ptr(), type_of(out.scalar_type()),
                                lse.defined() ? static_cast<float*>(lse.data_ptr()) : nullptr, truth(a[6]), s.sm_scale, real(a[8]),
                                max_len, ws.defined() ? ws.data_ptr() : nullptr, bytes, s.at.stream);
    }
    if (st)
        return PyLong_FromLong(st);
    PyObject* o = wrap(out);
    PyObject* l = lse.defined() ? wrap(lse) : Py_NewRef(Py_None);
    PyObject* both = o && l ? PyTuple_Pack(2, o, l) : nullptr;
    Py_XDECREF(o);
    Py_XDECREF(l);
    return both;
    END_HANDLE_TH_ERRORS
}

// FP32 [B][Hkv][at least `least`] whose rows do not overlap: address and strides.
float* weight_rows(const at::Tensor& w, int64_t B, int64_t Hkv, int64_t least, const Place& at, int64_t& sb, int64_t& sh)
{
    const bool fits = w.dim() == 3 && w.size(0) == B && w.size(1) == Hkv && w.size(2) >= least && w.scalar_type() == at::kFloat &&
                      w.device() == at.device && (w.size(2) <= 1 || w.stride(2) == 1) && (Hkv <= 1 || w.stride(1) >= w.size(2)) &&
                      (B <= 1 || w.stride(0) >= (Hkv - 1) * w.stride(1) + w.size(2));
    if (!fits)
        value_error("weights must be float32 " + shape_text({B, Hkv}) + " times at least " + std::to_string(least) +
                    " with contiguous rows that do not overlap, on " + at.device.str());
    sb = B > 1 ? w.stride(0) : 0;
    sh = Hkv > 1 ? w.stride(1) : w.size(2);
    return static_cast<float*>(w.data_ptr());
}

// weights(q, lse, cache, pages, lens, weights, cu, max_q, causal, sm_scale, q_descale, max_len)
PyObject* weights(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_args(n, 12);
    const Queries s(tensor(a[0], "q"), a[2], a[3], a[4], a[6], a[7], a[9]);
    const float* lse = dense<float>(tensor(a[1], "lse"), "lse", s.at, at::kFloat, {s.T, s.Hq});
    const int max_len = int_arg(a[11], "max_len");
    int64_t most = (int64_t)s.bt.W * s.c.page, sb, sh;
    if (max_len > 0 && max_len < most)
        most = max_len;
    float* w = weight_rows(tensor(a[5], "weights"), s.bt.B, s.c.Hkv, most, s.at, sb, sh);
    const int st = attn_fp8_cache_weights(&s.c, &s.bt, &s.hq, (int)s.Hq, lse, truth(a[8]), s.sm_scale, real(a[10]), max_len, w, sb, sh,
                                          s.at.stream);
    return st ? PyLong_FromLong(st) : Py_NewRef(a[5]);
    END_HANDLE_TH_ERRORS
}

// evict(cache, pages, lens, weights, to, new_pages, budget, n_sink, n_recent, kept, new_lens, new_weights)
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_args(n, 12);
    const Place at(tensor(a[2], "lens"));
    const attn_fp8_cache c = cache_of(a[0], at), to = cache_of(a[4], at);
    const at::Tensor& pages = tensor(a[1], "pages");
    if (pages.dim() != 2)
        value_error("pages must be [B, W]");
    const int64_t B = pages.size(0), W = pages.size(1), budget = integer(a[6]);
    if (to.Hkv != c.Hkv || to.page != c.page || to.d != c.d || budget < 1 || c.page < 1)
        value_error("both caches have the same heads, page and d, and budget is at least 1");
    attn_fp8_batch bt{};
    bt.pages = ints(a[1], "pages", at, pages.sizes());
    bt.lens = ints(a[2], "lens", at, {B});
    bt.B = narrow(B, "B");
    bt.W = narrow(W, "W");
    bt.max_q = 1;
    const int32_t* new_pages = ints(a[5], "new_pages", at, {B, (budget + c.page - 1) / c.page});
    int64_t sb, sh;
    const float* w = weight_rows(tensor(a[3], "weights"), B, c.Hkv, W * c.page, at, sb, sh);
    const std::array<int64_t, 3> shape = {B, c.Hkv, budget};
    const at::Tensor kept = a[9] == Py_None ? at.empty(shape, at::kInt) : tensor(a[9], "kept");
    const at::Tensor new_lens = a[10] == Py_None ? at.empty({B}, at::kInt) : tensor(a[10], "new_lens");
    const at::Tensor new_weights = a[11] == Py_None ? at.empty(shape, at::kFloat) : tensor(a[11], "new_weights");
    const int st = attn_fp8_cache_evict(&c, &bt, &to, new_pages, w, sb, sh, narrow(budget, "budget"), int_arg(a[7], "n_sink"),
                                        int_arg(a[8], "n_recent"), dense<int32_t>(kept, "kept", at, at::kInt, shape),
                                        dense<int32_t>(new_lens, "new_lens", at, at::kInt, {B}),
                                        dense<float>(new_weights, "new_weights", at, at::kFloat, shape), at.stream);
    if (st)
        return PyLong_FromLong(st);
    PyObject* r[3] = {wrap(kept), wrap(new_lens), wrap(new_weights)};
    PyObject* all = r[0] && r[1] && r[2] ? PyTuple_Pack(3, r[0], r[1], r[2]) : nullptr;
    for (PyObject* x : r)
        Py_XDECREF(x);
    return all;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&rope)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&append)), METH_FASTCALL, nullptr},
    {"fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&fwd)), METH_FASTCALL, nullptr},
    {"weights", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&weights)), METH_FASTCALL, nullptr},
    {"evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&evict)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cache_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cache_binding() { return PyModule_Create(&module); }
