// The hot calls' argument handling between torch tensors and the C ABI, in native code.
//
// A layer's pair of calls on a few hundred rows keeps the GPU busy for 12-16 us; checking the
// tensors, sizing and allocating the outputs and finding the stream took 23 us per pair as Python
// with ctypes, so the host set the pace of every small layer.  Each function below does one
// call's checks (the same errors with the same texts), allocates what the caller did not pass
// through torch's allocator on the current stream, and enqueues with the interpreter lock
// released (a launch may wait for room in the queue).  It keeps no state between calls.
#include <Python.h>

#include <optional>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "dgq.h"

namespace {

struct Raised {};  // a Python exception is set

PyObject *g_error = nullptr;  // the package's DgqError
PyObject *s_handle = nullptr, *s_out_channels = nullptr, *s_cuda_stream = nullptr;

[[noreturn]] void raise(PyObject *type, const char *text) {
    PyErr_SetString(type, text);
    throw Raised();
}
[[noreturn]] void raise_value(const char *text) { raise(PyExc_ValueError, text); }

const char *dtype_name(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return "torch.float32";
        case at::kChar: return "torch.int8";
        case at::kByte: return "torch.uint8";
        default: return "torch.int32";
    }
}

bool given(PyObject *o) { return o != Py_None; }

const at::Tensor &tensor(PyObject *o, at::ScalarType t, const char *name) {
    if (THPVariable_Check(o)) {
        const at::Tensor &v = THPVariable_Unpack(o);
        if (v.is_cuda() && v.scalar_type() == t && v.is_contiguous()) return v;
    }
    PyErr_Format(PyExc_TypeError, "%s must be a contiguous CUDA tensor of dtype %s", name, dtype_name(t));
    throw Raised();
}

// data pointer of an optional tensor
template <class T>
T *pointer(const at::Tensor &v) { return static_cast<T *>(v.data_ptr()); }

template <class T>
T *optional(PyObject *o, at::ScalarType t, const char *name) {
    return given(o) ? pointer<T>(tensor(o, t, name)) : nullptr;
}

void *handle_of(PyObject *o) {  // None: a handle that was freed (the C call reports the null)
    PyObject *h = PyObject_GetAttr(o, s_handle);
    if (!h) throw Raised();
    void *p = given(h) ? PyLong_AsVoidPtr(h) : nullptr;
    Py_DECREF(h);
    if (!p && PyErr_Occurred()) throw Raised();
    return p;
}
const dgq_groups_t *groups_of(PyObject *o) { return static_cast<const dgq_groups_t *>(handle_of(o)); }
const dgq_weight_t *weight_of(PyObject *o) { return static_cast<const dgq_weight_t *>(handle_of(o)); }

int64_t integer(PyObject *o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
// sizes of the C ABI are 32 bits wide; what does not fit is reported by the call as an empty tensor
int32_t integer32(PyObject *o) {
    const int64_t v = integer(o);
    return v >= INT32_MIN && v <= INT32_MAX ? (int32_t)v : -1;
}

int64_t out_channels_of(PyObject *weight) {
    PyObject *o = PyObject_GetAttr(weight, s_out_channels);
    if (!o) throw Raised();
    const int64_t v = PyLong_AsLongLong(o);
    Py_DECREF(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}

void *stream_of(PyObject *o) {
    if (!given(o)) return c10::hip::getCurrentHIPStream().stream();
    PyObject *s = PyObject_GetAttr(o, s_cuda_stream);
    if (!s) throw Raised();
    void *p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!p && PyErr_Occurred()) throw Raised();
    return p;
}

// A new tensor, straight from the allocator (the dispatcher's way there takes 0.5 us; a new tensor has no gradient).  Where torch is
// to fill what nobody writes (torch.use_deterministic_algorithms), it does so on the stream that the call enqueues on.
at::Tensor empty(at::IntArrayRef sizes, at::ScalarType t, const at::Tensor &like, PyObject *stream = Py_None) {
    const at::Context &torch = at::globalContext();
    if (!torch.deterministicAlgorithms() || !torch.deterministicFillUninitializedMemory())
        return at::detail::empty_cuda(sizes, t, like.device(), std::nullopt);
    std::optional<c10::hip::HIPStreamGuard> on;
    if (given(stream)) on.emplace(c10::hip::getStreamFromExternal(static_cast<hipStream_t>(stream_of(stream)), like.device().index()));
    at::AutoDispatchBelowADInplaceOrView below;
    return at::empty(sizes, like.options().dtype(t).requires_grad(false));
}

dgq_groups_info_t info_of(const dgq_groups_t *g) {
    dgq_groups_info_t i{};
    if (g) dgq_groups_info(g, &i);
    return i;
}

// Shape of the block-tiled code buffer: [row blocks, chunks, 1024].
struct CodesShape {
    int64_t n[3];
    CodesShape(const dgq_groups_t *g, int64_t rows) {
        const int64_t chunks = info_of(g).k_padded / DGQ_K_GRANULE;
        n[0] = chunks ? (int64_t)dgq_codes_bytes(g, rows) / (chunks * 1024) : 0;
        n[1] = chunks;
        n[2] = 1024;
    }
    at::IntArrayRef sizes() const { return at::IntArrayRef(n, 3); }
    bool is(const at::Tensor &t) const { return t.sizes() == sizes(); }
};

bool shape_is(const at::Tensor &t, std::initializer_list<int64_t> s) {
    return t.sizes() == at::IntArrayRef(s.begin(), s.size());
}

// The C ABI sees no sizes: a tensor it would read or write past the end of is refused here.
void holds(const at::Tensor &t, int64_t n, const char *name) {
    if (t.numel() >= n) return;
    PyErr_Format(PyExc_ValueError, "%s has %lld elements, the call needs %lld", name, (long long)t.numel(), (long long)n);
    throw Raised();
}
void holds_if_given(PyObject *o, int64_t n, const char *name) {
    if (given(o)) holds(THPVariable_Unpack(o), n, name);
}

template <class F>
void enqueue(F &&call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = call();
    Py_END_ALLOW_THREADS;
    if (rc == 0) return;
    if (PyObject *e = PyObject_CallFunction(g_error, "is", rc, dgq_last_error())) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw Raised();
}

PyObject *wrap(const at::Tensor &t) {
    PyObject *o = THPVariable_Wrap(t);
    if (!o) throw Raised();
    return o;
}
// (the caller's object where one was passed, else the new tensor), as a pair
PyObject *pair(PyObject *a_given, const at::Tensor &a, PyObject *b_given, const at::Tensor &b) {
    PyObject *t = PyTuple_New(2);
    if (!t) throw Raised();
    try {
        PyTuple_SET_ITEM(t, 0, given(a_given) ? (Py_INCREF(a_given), a_given) : wrap(a));
        PyTuple_SET_ITEM(t, 1, given(b_given) ? (Py_INCREF(b_given), b_given) : wrap(b));
    } catch (...) {
        Py_DECREF(t);
        throw;
    }
    return t;
}
PyObject *one(PyObject *a_given, const at::Tensor &a) {
    if (!given(a_given)) return wrap(a);
    Py_INCREF(a_given);
    return a_given;
}

using Args = PyObject *const *;

// (groups, x, codes, row_class, stream)
PyObject *quantize_act(Args a) {
    const dgq_groups_t *g = groups_of(a[0]);
    const at::Tensor &x = tensor(a[1], at::kFloat, "x");
    if (x.dim() != 2) raise_value("x must be [rows, channels]");
    const int64_t rows = x.size(0);
    const dgq_groups_info_t info = info_of(g);
    if (g && x.size(1) != info.channels) {
        PyErr_Format(PyExc_ValueError, "x has %lld channels, the groups have %d", (long long)x.size(1), info.channels);
        throw Raised();
    }
    const CodesShape shape(g, rows);
    const at::Tensor codes = given(a[2]) ? tensor(a[2], at::kChar, "codes") : empty(shape.sizes(), at::kChar, x, a[4]);
    const at::Tensor cls = given(a[3]) ? tensor(a[3], at::kByte, "row_class") : empty({rows}, at::kByte, x, a[4]);
    if (!shape.is(codes) || cls.numel() != rows) raise_value("codes / row_class have the wrong shape");
    void *st = stream_of(a[4]);
    const float *xp = pointer<float>(x);
    int8_t *cp = pointer<int8_t>(codes);
    uint8_t *rp = pointer<uint8_t>(cls);
    enqueue([&] { return dgq_quantize_act(g, xp, rows, cp, rp, st); });
    return pair(a[2], codes, a[3], cls);
}

struct LinearIn {
    const dgq_groups_t *g;
    const dgq_weight_t *w;
    const at::Tensor &codes, &cls;
    int64_t rows;
    LinearIn(PyObject *groups, PyObject *weight, PyObject *c, PyObject *r)
        : g(groups_of(groups)), w(weight_of(weight)), codes(tensor(c, at::kChar, "codes")),
          cls(tensor(r, at::kByte, "row_class")), rows(cls.numel()) {
        if (!CodesShape(g, rows).is(codes)) raise_value("codes / row_class have the wrong shape");
    }
};

// (groups, weight, codes, row_class, y, acc_dump, stream, workspace)
PyObject *linear(Args a) {
    const LinearIn in(a[0], a[1], a[2], a[3]);
    const int64_t O = out_channels_of(a[1]);
    const at::Tensor y = given(a[4]) ? tensor(a[4], at::kFloat, "y") : empty({in.rows, O}, at::kFloat, in.codes, a[6]);
    if (!shape_is(y, {in.rows, O})) raise_value("y has the wrong shape");
    int32_t *dump = nullptr;
    if (given(a[5])) {
        const at::Tensor &d = tensor(a[5], at::kInt, "acc_dump");
        if (!shape_is(d, {in.rows, O, info_of(in.g).n_groups})) raise_value("acc_dump has the wrong shape");
        dump = pointer<int32_t>(d);
    }
    void *ws = nullptr;
    size_t ws_bytes = 0;
    if (given(a[7])) {
        const at::Tensor &t = tensor(a[7], at::kByte, "workspace");
        ws = t.data_ptr();
        ws_bytes = (size_t)t.numel();
    }
    void *st = stream_of(a[6]);
    const int8_t *cp = pointer<int8_t>(in.codes);
    const uint8_t *rp = pointer<uint8_t>(in.cls);
    float *yp = pointer<float>(y);
    enqueue([&] { return dgq_linear(in.g, in.w, cp, rp, in.rows, yp, dump, ws, ws_bytes, st); });
    return one(a[4], y);
}

// (groups, weight, codes, row_class, y, stream)
PyObject *linear_geglu(Args a) {
    const LinearIn in(a[0], a[1], a[2], a[3]);
    const int64_t oh = out_channels_of(a[1]) / 2;
    const at::Tensor y = given(a[4]) ? tensor(a[4], at::kFloat, "y") : empty({in.rows, oh}, at::kFloat, in.codes, a[5]);
    if (!shape_is(y, {in.rows, oh})) raise_value("y has the wrong shape");
    void *st = stream_of(a[5]);
    const int8_t *cp = pointer<int8_t>(in.codes);
    const uint8_t *rp = pointer<uint8_t>(in.cls);
    float *yp = pointer<float>(y);
    enqueue([&] { return dgq_linear_geglu(in.g, in.w, cp, rp, in.rows, yp, st); });
    return one(a[4], y);
}

// (groups, weight, codes, row_class, next_groups, codes_next, row_class_next, stream)
PyObject *linear_geglu_requant(Args a) {
    const LinearIn in(a[0], a[1], a[2], a[3]);
    const CodesShape shape(groups_of(a[4]), in.rows);
    const at::Tensor codes2 = given(a[5]) ? tensor(a[5], at::kChar, "codes_next") : empty(shape.sizes(), at::kChar, in.codes, a[7]);
    const at::Tensor cls2 = given(a[6]) ? tensor(a[6], at::kByte, "row_class_next") : empty({in.rows}, at::kByte, in.codes, a[7]);
    if (!shape.is(codes2) || cls2.numel() != in.rows) raise_value("codes_next / row_class_next have the wrong shape");
    void *st = stream_of(a[7]);
    const int8_t *cp = pointer<int8_t>(in.codes);
    const uint8_t *rp = pointer<uint8_t>(in.cls);
    int8_t *c2 = pointer<int8_t>(codes2);
    uint8_t *r2 = pointer<uint8_t>(cls2);
    enqueue([&] { return dgq_linear_geglu_requant(in.g, in.w, cp, rp, in.rows, c2, r2, st); });
    return pair(a[5], codes2, a[6], cls2);
}

// (groups9, codes, B, H, W, codes9, stream)
PyObject *conv3x3_codes(Args a) {
    const dgq_groups_t *g9 = groups_of(a[0]);
    const at::Tensor &codes = tensor(a[1], at::kChar, "codes");
    const int32_t B = integer32(a[2]), H = integer32(a[3]), W = integer32(a[4]);
    const CodesShape shape(g9, (int64_t)B * H * W);
    if (codes.numel() * 9 != shape.n[0] * shape.n[1] * shape.n[2])
        raise_value("codes do not belong to a [B*H*W, C] map of this layer");
    const at::Tensor out = given(a[5]) ? tensor(a[5], at::kChar, "codes9") : empty(shape.sizes(), at::kChar, codes, a[6]);
    if (!shape.is(out)) raise_value("codes9 has the wrong shape");
    void *st = stream_of(a[6]);
    const int8_t *cp = pointer<int8_t>(codes);
    int8_t *op = pointer<int8_t>(out);
    enqueue([&] { return dgq_conv3x3_codes(g9, cp, B, H, W, op, st); });
    return one(a[5], out);
}

// (groups, groups9, x, B, H, W, codes3, row_class, stream)
PyObject *quantize_act_conv3x3(Args a) {
    const dgq_groups_t *g = groups_of(a[0]), *g9 = groups_of(a[1]);
    const at::Tensor &x = tensor(a[2], at::kFloat, "x");
    const int32_t B = integer32(a[3]), H = integer32(a[4]), W = integer32(a[5]);
    const int64_t rows = (int64_t)B * H * W;
    if (g && !shape_is(x, {rows, info_of(g).channels})) raise_value("x must be [B*H*W, C]");
    const int64_t nbytes = (int64_t)dgq_conv3x3_codes3_bytes(g9, B, H, W);
    const at::Tensor codes3 = given(a[6]) ? tensor(a[6], at::kChar, "codes3") : empty({nbytes}, at::kChar, x, a[8]);
    const at::Tensor cls = given(a[7]) ? tensor(a[7], at::kByte, "row_class") : empty({rows}, at::kByte, x, a[8]);
    if (codes3.numel() != nbytes || cls.numel() != rows) raise_value("codes3 / row_class have the wrong size");
    void *st = stream_of(a[8]);
    const float *xp = pointer<float>(x);
    int8_t *cp = pointer<int8_t>(codes3);
    uint8_t *rp = pointer<uint8_t>(cls);
    enqueue([&] { return dgq_quantize_act_conv3x3(g, g9, xp, B, H, W, cp, rp, st); });
    return pair(a[6], codes3, a[7], cls);
}

// (groups9, weight, codes3, row_class, B, H, W, y, stream)
PyObject *linear_conv3x3(Args a) {
    const dgq_groups_t *g9 = groups_of(a[0]);
    const dgq_weight_t *w = weight_of(a[1]);
    const at::Tensor &codes3 = tensor(a[2], at::kChar, "codes3"), &cls = tensor(a[3], at::kByte, "row_class");
    const int32_t B = integer32(a[4]), H = integer32(a[5]), W = integer32(a[6]);
    const int64_t rows = (int64_t)B * H * W, O = out_channels_of(a[1]);
    holds(codes3, (int64_t)dgq_conv3x3_codes3_bytes(g9, B, H, W), "codes3");
    holds(cls, rows, "row_class");
    const at::Tensor y = given(a[7]) ? tensor(a[7], at::kFloat, "y") : empty({rows, O}, at::kFloat, codes3, a[8]);
    if (!shape_is(y, {rows, O})) raise_value("y has the wrong shape");
    void *st = stream_of(a[8]);
    const int8_t *cp = pointer<int8_t>(codes3);
    const uint8_t *rp = pointer<uint8_t>(cls);
    float *yp = pointer<float>(y);
    enqueue([&] { return dgq_linear_conv3x3(g9, w, cp, rp, B, H, W, yp, st); });
    return one(a[7], y);
}

// The sizes of an attention call's queries.
struct AttnShape {
    int64_t B, N, H, d;
    explicit AttnShape(const at::Tensor &q) {
        if (q.dim() != 4) raise_value("q must be [B, N, H, d]");
        B = q.size(0), N = q.size(1), H = q.size(2), d = q.size(3);
        if (B > INT32_MAX || N > INT32_MAX || H > INT32_MAX || d > INT32_MAX) raise_value("q is too large");
    }
};

// (q, k, v, key_bias, attn_bits, out, scale_out, codes_dump, workspace, stream)
PyObject *xattn_logq(Args a) {
    const at::Tensor &q = tensor(a[0], at::kFloat, "q"), &k = tensor(a[1], at::kFloat, "k"), &v = tensor(a[2], at::kFloat, "v");
    const float *kb = optional<float>(a[3], at::kFloat, "key_bias");
    const AttnShape s(q);
    const int64_t nk = k.dim() > 1 ? k.size(1) : 0;
    if (nk > INT32_MAX || !shape_is(k, {s.B, nk, s.H, s.d}) || !shape_is(v, {s.B, nk, s.H, s.d}))
        raise_value("k / v have the wrong shape");
    if (kb && THPVariable_Unpack(a[3]).numel() != nk) raise_value("key_bias has the wrong shape");
    const int32_t bits = integer32(a[4]);
    const at::Tensor out = given(a[5]) ? tensor(a[5], at::kFloat, "out") : empty(q.sizes(), at::kFloat, q, a[9]);
    holds(out, q.numel(), "out");
    const at::Tensor scale = given(a[6]) ? tensor(a[6], at::kFloat, "scale_out") : empty({s.B}, at::kFloat, q, a[9]);
    holds(scale, s.B, "scale_out");
    uint8_t *dump = optional<uint8_t>(a[7], at::kByte, "codes_dump");
    if (dump && !shape_is(THPVariable_Unpack(a[7]), {s.B, s.H, s.N, nk - 1})) raise_value("codes_dump has the wrong shape");
    at::Tensor ws;
    if (given(a[8])) {
        if (!THPVariable_Check(a[8])) raise(PyExc_TypeError, "workspace must be a tensor");
        ws = THPVariable_Unpack(a[8]);
    } else if (const size_t need = dgq_xattn_workspace_bytes((int32_t)s.B, (int32_t)s.N, (int32_t)s.H, (int32_t)s.d, (int32_t)nk)) {
        ws = empty({(int64_t)need}, at::kByte, q, a[9]);
    }
    void *wp = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t wb = ws.defined() ? (size_t)ws.numel() * ws.element_size() : 0;
    void *st = stream_of(a[9]);
    const float *qp = pointer<float>(q), *kp = pointer<float>(k), *vp = pointer<float>(v);
    float *op = pointer<float>(out), *sp = pointer<float>(scale);
    enqueue([&] {
        return dgq_xattn_logq(qp, kp, vp, kb, (int32_t)s.B, (int32_t)s.N, (int32_t)s.H, (int32_t)s.d, (int32_t)nk, bits, op,
                              sp, dump, wp, wb, st);
    });
    return pair(a[5], out, a[6], scale);
}

// (q, k, v, key_bias, attn_bits, scale_in, out, scale_out, codes_dump, stream); scale_out None stays None
PyObject *xattn_logq_static(Args a) {
    const at::Tensor &q = tensor(a[0], at::kFloat, "q"), &k = tensor(a[1], at::kFloat, "k"), &v = tensor(a[2], at::kFloat, "v");
    const at::Tensor &sin = tensor(a[5], at::kFloat, "scale_in");
    const AttnShape s(q);
    const int64_t nk = k.dim() > 1 ? k.size(1) : 0;
    if (nk > INT32_MAX || k.numel() != s.B * nk * s.H * s.d || v.numel() != k.numel())
        raise_value("k / v have the wrong size");
    const float *kb = optional<float>(a[3], at::kFloat, "key_bias");
    holds_if_given(a[3], nk, "key_bias");
    holds(sin, s.B, "scale_in");
    const int32_t bits = integer32(a[4]);
    const at::Tensor out = given(a[6]) ? tensor(a[6], at::kFloat, "out") : empty(q.sizes(), at::kFloat, q, a[9]);
    holds(out, q.numel(), "out");
    float *so = optional<float>(a[7], at::kFloat, "scale_out");
    holds_if_given(a[7], s.B, "scale_out");
    uint8_t *dump = optional<uint8_t>(a[8], at::kByte, "codes_dump");
    holds_if_given(a[8], s.B * s.H * s.N * (nk - 1), "codes_dump");
    void *st = stream_of(a[9]);
    const float *qp = pointer<float>(q), *kp = pointer<float>(k), *vp = pointer<float>(v), *ip = pointer<float>(sin);
    float *op = pointer<float>(out);
    enqueue([&] {
        return dgq_xattn_logq_static(qp, kp, vp, kb, (int32_t)s.B, (int32_t)s.N, (int32_t)s.H, (int32_t)s.d, (int32_t)nk,
                                     bits, ip, op, so, dump, st);
    });
    PyObject *o = one(a[6], out);
    PyObject *t = PyTuple_Pack(2, o, a[7]);
    Py_DECREF(o);
    if (!t) throw Raised();
    return t;
}

// (q, k, v, attn_bits, scale_in, out, scale_out, codes_dump, workspace, stream)
PyObject *selfattn_logq(Args a) {
    const at::Tensor &q = tensor(a[0], at::kFloat, "q"), &k = tensor(a[1], at::kFloat, "k"), &v = tensor(a[2], at::kFloat, "v");
    const at::Tensor &sin = tensor(a[4], at::kFloat, "scale_in");
    const AttnShape s(q);
    if (k.sizes() != q.sizes() || v.sizes() != q.sizes() || sin.numel() != s.B)
        raise_value("q, k, v must share one shape [B,N,H,d] and scale_in have B entries");
    const int32_t bits = integer32(a[3]);
    const at::Tensor out = given(a[5]) ? tensor(a[5], at::kFloat, "out") : empty(q.sizes(), at::kFloat, q, a[9]);
    holds(out, q.numel(), "out");
    float *so = optional<float>(a[6], at::kFloat, "scale_out");
    holds_if_given(a[6], s.B, "scale_out");
    uint8_t *dump = optional<uint8_t>(a[7], at::kByte, "codes_dump");
    if (dump && !shape_is(THPVariable_Unpack(a[7]), {s.B, s.H, s.N, s.N})) raise_value("codes_dump must be [B,H,N,N]");
    at::Tensor ws;
    if (given(a[8])) {
        if (!THPVariable_Check(a[8])) raise(PyExc_TypeError, "workspace must be a tensor");
        ws = THPVariable_Unpack(a[8]);
    } else {
        const size_t need = dgq_selfattn_workspace_bytes((int32_t)s.B, (int32_t)s.N, (int32_t)s.H, (int32_t)s.d);
        ws = empty({(int64_t)(need > 16 ? need : 16)}, at::kByte, q, a[9]);
    }
    void *wp = ws.data_ptr(), *st = stream_of(a[9]);
    const size_t wb = (size_t)ws.numel();
    const float *qp = pointer<float>(q), *kp = pointer<float>(k), *vp = pointer<float>(v), *ip = pointer<float>(sin);
    float *op = pointer<float>(out);
    enqueue([&] {
        return dgq_selfattn_logq(qp, kp, vp, (int32_t)s.B, (int32_t)s.N, (int32_t)s.H, (int32_t)s.d, bits, ip, op, so, dump,
                                 wp, wb, st);
    });
    return one(a[5], out);
}

// ---- the 8-bit cache ----

// A call's device and stream: its tensors lie on one device, which is current while it runs; what it allocates belongs to
// the stream that it enqueues on, so a workspace that is dropped on return is not handed out before that work is done.
class Place {
public:
    Place(PyObject *stream, const at::Tensor &first) : device_(first.device()), guard_(device_) {
        if (given(stream)) on_.emplace(c10::hip::getStreamFromExternal(static_cast<hipStream_t>(stream_of(stream)), device_.index()));
        stream_ = c10::hip::getCurrentHIPStream(device_.index()).stream();
    }
    void *stream() const { return stream_; }
    void same(const at::Tensor &t, const char *name) const {
        if (t.device() == device_) return;
        PyErr_Format(PyExc_ValueError, "%s is on another device", name);
        throw Raised();
    }

private:
    const c10::Device device_;
    const c10::DeviceGuard guard_;
    std::optional<c10::hip::HIPStreamGuard> on_;  // the current stream needs none
    hipStream_t stream_;
};

int32_t kv_dtype(at::ScalarType t) {
    return t == at::kFloat ? DGQ_F32 : t == at::kHalf ? DGQ_F16 : t == at::kBFloat16 ? DGQ_BF16 : -1;
}

const at::Tensor &floats(PyObject *o, const char *name, int64_t dims) {
    if (THPVariable_Check(o)) {
        const at::Tensor &v = THPVariable_Unpack(o);
        if (v.is_cuda() && kv_dtype(v.scalar_type()) >= 0) {
            if (v.dim() != dims) {
                PyErr_Format(PyExc_ValueError, "%s must have %lld dimensions", name, (long long)dims);
                throw Raised();
            }
            if (v.numel() == 0 || v.size(-1) == 1 || v.stride(-1) == 1) return v;
        }
    }
    PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor of float32, float16 or bfloat16 with contiguous dims", name);
    throw Raised();
}
// the stride of a dimension of one entry says nothing
int64_t step(const at::Tensor &t, int64_t dim) { return t.size(dim) > 1 ? t.stride(dim) : 0; }

const at::Tensor &ints(PyObject *o, const char *name, std::initializer_list<int64_t> shape) {
    const at::Tensor &t = tensor(o, at::kInt, name);
    if (!shape_is(t, shape)) {
        PyErr_Format(PyExc_ValueError, "%s has the wrong shape", name);
        throw Raised();
    }
    return t;
}
// Small int32 results of one call: those the caller did not pass are parts of one allocation, 16-byte aligned (five of their
// own took 3.4 us of a planning call's 8.5).
class IntResults {
public:
    IntResults(const Place &place, const at::Tensor &like) : place_(place), like_(like) {}
    void add(PyObject *o, const char *name, std::initializer_list<int64_t> shape) {
        Result &r = results_[n_++];
        r.object = o;
        if (given(o)) {
            r.tensor = ints(o, name, shape);
            place_.same(r.tensor, name);
            return;
        }
        for (int64_t x : shape) r.shape[r.dims++] = x;
        r.offset = total_;
        total_ += ((r.dims == 2 ? r.shape[0] * r.shape[1] : r.shape[0]) + 3) & ~(int64_t)3;
    }
    void allocate() {
        if (!total_) return;
        const at::Tensor all = empty({total_}, at::kInt, like_);
        for (int i = 0; i < n_; ++i) {
            Result &r = results_[i];
            if (given(r.object)) continue;
            r.tensor = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), all.dtype());
            r.tensor.unsafeGetTensorImpl()->set_storage_offset(r.offset);
            r.tensor.unsafeGetTensorImpl()->set_sizes_contiguous(at::IntArrayRef(r.shape, r.dims));
        }
    }
    int32_t *operator[](int i) const { return pointer<int32_t>(results_[i].tensor); }
    PyObject *tuple() const {
        PyObject *t = PyTuple_New(n_);
        if (!t) throw Raised();
        try {
            for (int i = 0; i < n_; ++i) PyTuple_SET_ITEM(t, i, one(results_[i].object, results_[i].tensor));
        } catch (...) {
            Py_DECREF(t);
            throw;
        }
        return t;
    }

private:
    struct Result {
        PyObject *object;
        at::Tensor tensor;
        int64_t shape[2], offset;
        int dims = 0;
    };
    const Place &place_;
    const at::Tensor &like_;
    Result results_[5];
    int n_ = 0;
    int64_t total_ = 0;
};

// The block table and what goes with it; B and width from its shape.
struct KvTable {
    const at::Tensor &table;
    int32_t B = 0, width = 0;
    explicit KvTable(PyObject *o) : table(tensor(o, at::kInt, "table")) {
        if (table.dim() != 2 || table.size(0) > INT32_MAX || table.size(1) > INT32_MAX) raise_value("table must be [B, width]");
        B = (int32_t)table.size(0), width = (int32_t)table.size(1);
    }
};

// (data, n_blocks, block_size, heads, d) from a[0]
struct KvCacheIn {
    const at::Tensor &data;
    int32_t n_blocks, block_size, heads, d;
    explicit KvCacheIn(Args a)
        : data(tensor(a[0], at::kByte, "cache.data")), n_blocks(integer32(a[1])), block_size(integer32(a[2])),
          heads(integer32(a[3])), d(integer32(a[4])) {
        holds(data, (int64_t)dgq_kv_cache_bytes(n_blocks, block_size, heads, d), "cache.data");
    }
};

// (lengths, new_rows, table, free_blocks, n_free, block_size, rows, lengths_out, n_free_out, row_offsets, runs, counts, stream)
PyObject *kv_plan(Args a) {
    const KvTable t(a[2]);
    const Place place(a[12], t.table);
    const at::Tensor &lengths = ints(a[0], "lengths", {t.B}), &more = ints(a[1], "new_rows", {t.B});
    const at::Tensor &list = tensor(a[3], at::kInt, "free_blocks"), &n_free = ints(a[4], "n_free", {1});
    if (list.dim() != 1 || list.numel() > INT32_MAX) raise_value("free_blocks must be [capacity]");
    place.same(lengths, "lengths"), place.same(more, "new_rows"), place.same(list, "free_blocks"), place.same(n_free, "n_free");
    const int32_t S = integer32(a[5]);
    const int64_t rows = integer(a[6]);
    int64_t max_runs = 2 * (int64_t)t.B + (S > 0 && rows > 0 ? rows / S : 0);
    if (given(a[10])) {
        const at::Tensor &r = tensor(a[10], at::kInt, "runs");
        if (r.dim() != 2 || r.size(1) != 4) raise_value("runs must be [max_runs, 4]");
        max_runs = r.size(0);
    }
    if (max_runs > INT32_MAX) raise_value("rows is too large");
    IntResults out(place, lengths);
    out.add(a[7], "lengths_out", {t.B});
    out.add(a[8], "n_free_out", {1});
    out.add(a[9], "row_offsets", {t.B + (int64_t)1});
    out.add(a[10], "runs", {max_runs, 4});
    out.add(a[11], "counts", {4});
    out.allocate();
    const int32_t *lp = pointer<int32_t>(lengths), *mp = pointer<int32_t>(more), *fp = pointer<int32_t>(list), *np = pointer<int32_t>(n_free);
    int32_t *tp = pointer<int32_t>(t.table);
    enqueue([&] {
        return dgq_kv_plan(lp, mp, t.B, S, rows, tp, t.width, fp, (int32_t)list.numel(), np, out[0], out[1], out[2], out[3], max_runs,
                           out[4], place.stream());
    });
    return out.tuple();
}

// (done, lengths, table, free_blocks, n_free, block_size, lengths_out, n_free_out, stream)
PyObject *kv_release(Args a) {
    const KvTable t(a[2]);
    const Place place(a[8], t.table);
    const at::Tensor &done = tensor(a[0], at::kByte, "done"), &lengths = ints(a[1], "lengths", {t.B});
    if (!shape_is(done, {t.B})) raise_value("done has the wrong shape");
    const at::Tensor &list = tensor(a[3], at::kInt, "free_blocks"), &n_free = ints(a[4], "n_free", {1});
    if (list.dim() != 1 || list.numel() > INT32_MAX) raise_value("free_blocks must be [capacity]");
    place.same(done, "done"), place.same(lengths, "lengths"), place.same(list, "free_blocks"), place.same(n_free, "n_free");
    const int32_t S = integer32(a[5]);
    IntResults out(place, lengths);
    out.add(a[6], "lengths_out", {t.B});
    out.add(a[7], "n_free_out", {1});
    out.allocate();
    const uint8_t *dp = pointer<uint8_t>(done);
    const int32_t *lp = pointer<int32_t>(lengths), *tp = pointer<int32_t>(t.table), *np = pointer<int32_t>(n_free);
    int32_t *fp = pointer<int32_t>(list);
    enqueue([&] {
        return dgq_kv_release(dp, lp, tp, t.B, t.width, S, fp, (int32_t)list.numel(), np, out[0], out[1], place.stream());
    });
    return out.tuple();
}

// (k, v, runs, data, n_blocks, block_size, heads, d, stream)
PyObject *kv_store(Args a) {
    const KvCacheIn c(a + 3);
    const Place place(a[8], c.data);
    const at::Tensor &k = floats(a[0], "k", 3), &v = floats(a[1], "v", 3), &runs = tensor(a[2], at::kInt, "runs");
    if (k.scalar_type() != v.scalar_type()) raise_value("k and v differ in type");
    if (k.sizes() != v.sizes() || k.size(1) != c.heads || k.size(2) != c.d) raise_value("k / v must be [rows, heads, d] of the cache");
    if (runs.dim() != 2 || runs.size(1) != 4) raise_value("runs must be [n_runs, 4]");
    place.same(k, "k"), place.same(v, "v"), place.same(runs, "runs");
    const void *kp = k.data_ptr(), *vp = v.data_ptr();
    void *cp = c.data.data_ptr();
    const int32_t *rp = pointer<int32_t>(runs), t = kv_dtype(k.scalar_type());
    enqueue([&] {
        return dgq_kv_store(kp, vp, t, k.size(0), step(k, 0), step(k, 1), step(v, 0), step(v, 1), rp, runs.size(0), cp,
                            c.n_blocks, c.block_size, c.heads, c.d, place.stream());
    });
    Py_RETURN_NONE;
}

// (data, n_blocks, block_size, heads, d, table, lengths, max_rows, dtype, k, v, stream)
PyObject *kv_load(Args a) {
    const KvCacheIn c(a);
    const Place place(a[11], c.data);
    const KvTable t(a[5]);
    const at::Tensor &lengths = ints(a[6], "lengths", {t.B});
    place.same(t.table, "table"), place.same(lengths, "lengths");
    const int32_t max_rows = integer32(a[7]);
    if (max_rows < 0) raise_value("max_rows is below 0");
    at::ScalarType type = at::kFloat;
    if (given(a[8])) {
        if (!THPDtype_Check(a[8])) raise(PyExc_TypeError, "dtype must be a torch.dtype");
        type = reinterpret_cast<THPDtype *>(a[8])->scalar_type;
    } else if (given(a[9]) && THPVariable_Check(a[9])) {
        type = THPVariable_Unpack(a[9]).scalar_type();
    }
    if (kv_dtype(type) < 0) raise_value("dtype must be float32, float16 or bfloat16");
    at::Tensor out[2];
    for (int i = 0; i < 2; ++i) {
        const char *name = i ? "v" : "k";
        if (!given(a[9 + i])) {
            out[i] = empty({t.B, max_rows, c.heads, c.d}, type, c.data);
            continue;
        }
        out[i] = floats(a[9 + i], name, 4);
        place.same(out[i], name);
        if (!shape_is(out[i], {t.B, max_rows, c.heads, c.d}) || out[i].scalar_type() != type || !out[i].is_contiguous())
            raise_value("k / v must be contiguous [B, max_rows, heads, d] of dtype");
    }
    const void *cp = c.data.data_ptr();
    void *kp = out[0].data_ptr(), *vp = out[1].data_ptr();
    const int32_t *tp = pointer<int32_t>(t.table), *lp = pointer<int32_t>(lengths);
    enqueue([&] {
        return dgq_kv_load(cp, c.n_blocks, c.block_size, c.heads, c.d, tp, t.width, lp, t.B, max_rows, kv_dtype(type), kp, vp, place.stream());
    });
    return pair(a[9], out[0], a[10], out[1]);
}

// (q, data, n_blocks, block_size, heads, d, table, lengths, q_offsets, out, workspace, stream)
PyObject *xattn_kv(Args a) {
    const KvCacheIn c(a + 1);
    const Place place(a[11], c.data);
    const KvTable t(a[6]);
    const at::Tensor &lengths = ints(a[7], "lengths", {t.B});
    const bool packed = given(a[8]);
    const at::Tensor &q = floats(a[0], "q", packed ? 3 : 4);
    const int64_t N = q.size(packed ? 0 : 1), Hq = q.size(packed ? 1 : 2);
    if ((!packed && q.size(0) != t.B) || q.size(-1) != c.d || Hq > INT32_MAX || Hq < 1)
        raise_value("q must be [B, N, heads, d], or [rows, heads, d] with q_offsets");
    const int32_t *op = packed ? pointer<int32_t>(ints(a[8], "q_offsets", {t.B + (int64_t)1})) : nullptr;
    if (packed) place.same(THPVariable_Unpack(a[8]), "q_offsets");
    place.same(q, "q"), place.same(t.table, "table"), place.same(lengths, "lengths");
    at::Tensor out;
    if (given(a[9])) {
        out = floats(a[9], "out", packed ? 3 : 4);
        place.same(out, "out");
        if (out.sizes() != q.sizes() || out.scalar_type() != q.scalar_type() || !out.is_contiguous())
            raise_value("out must be contiguous, of q's shape and type");
    } else {
        out = empty(q.sizes(), q.scalar_type(), q);
    }
    at::Tensor ws;
    if (given(a[10])) {
        if (!THPVariable_Check(a[10])) raise(PyExc_TypeError, "workspace must be a tensor");
        ws = tensor(a[10], at::kByte, "workspace");
        place.same(ws, "workspace");
    } else if (const size_t need = dgq_xattn_kv_workspace_bytes(t.B, N, packed, (int32_t)Hq, c.heads, c.d, t.width, c.block_size)) {
        ws = empty({(int64_t)need}, at::kByte, q);
    }
    void *wp = ws.defined() ? ws.data_ptr() : nullptr, *yp = out.data_ptr();
    const size_t wb = ws.defined() ? (size_t)ws.numel() : 0;
    const void *qp = q.data_ptr(), *cp = c.data.data_ptr();
    const int32_t *tp = pointer<int32_t>(t.table), *lp = pointer<int32_t>(lengths), type = kv_dtype(q.scalar_type());
    const int64_t sb = packed ? 0 : step(q, 0), sn = step(q, packed ? 0 : 1), sh = step(q, packed ? 1 : 2);
    enqueue([&] {
        return dgq_xattn_kv(qp, type, op, sb, sn, sh, t.B, N, (int32_t)Hq, cp, c.n_blocks, c.block_size, c.heads, c.d, tp, t.width, lp,
                            yp, wp, wb, place.stream());
    });
    return one(a[9], out);
}

// ---- group norm, and weights in 4 bits ----

// The type named by a dtype argument, `otherwise` where none is given.
at::ScalarType dtype_of(PyObject *o, at::ScalarType otherwise) {
    if (!given(o)) return otherwise;
    if (!THPDtype_Check(o)) raise(PyExc_TypeError, "dtype must be a torch.dtype");
    const at::ScalarType t = reinterpret_cast<THPDtype *>(o)->scalar_type;
    if (kv_dtype(t) < 0) raise_value("dtype must be float32, float16 or bfloat16");
    return t;
}

// A contiguous output of `type`: the caller's, whose type stands for a dtype that is not given, or a new one.
at::Tensor output(PyObject *o, PyObject *dtype, at::ScalarType in, at::IntArrayRef sizes, const at::Tensor &like, const Place &place,
                  const char *name) {
    const bool mine = given(o);
    at::ScalarType type = in;
    if (mine && THPVariable_Check(o)) type = THPVariable_Unpack(o).scalar_type();
    type = dtype_of(dtype, type);
    if (!mine) return empty(sizes, type, like);
    const at::Tensor t = floats(o, name, (int64_t)sizes.size());
    place.same(t, name);
    if (t.sizes() != sizes || t.scalar_type() != type || !t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s has the wrong shape or type, or is not contiguous", name);
        throw Raised();
    }
    return t;
}

// fp32 [n], or null
const float *vector_of(PyObject *o, const char *name, int64_t n, const Place &place) {
    if (!given(o)) return nullptr;
    const at::Tensor &t = tensor(o, at::kFloat, name);
    if (!shape_is(t, {n})) {
        PyErr_Format(PyExc_ValueError, "%s has the wrong shape", name);
        throw Raised();
    }
    place.same(t, name);
    return pointer<float>(t);
}

// fp32 [B, C] with rows of any stride, or null
struct Rows {
    const float *data = nullptr;
    int64_t stride = 0;
    Rows(PyObject *o, const char *name, int64_t B, int64_t C, const Place &place) {
        if (!given(o)) return;
        const at::Tensor &t = floats(o, name, 2);
        if (t.scalar_type() != at::kFloat) {
            PyErr_Format(PyExc_TypeError, "%s must be of dtype torch.float32", name);
            throw Raised();
        }
        if (!shape_is(t, {B, C})) {
            PyErr_Format(PyExc_ValueError, "%s must be [images, channels]", name);
            throw Raised();
        }
        place.same(t, name);
        data = pointer<float>(t), stride = step(t, 0);
    }
};

// (x, num_groups, weight, bias, eps, act, add, scale, shift, offsets, dtype, out, workspace, stream)
PyObject *groupnorm(Args a) {
    const bool packed = given(a[9]);
    const at::Tensor &x = floats(a[0], "x", packed ? 2 : 3);
    const Place place(a[13], x);
    const int32_t *op = nullptr;
    int64_t B = x.size(0);
    if (packed) {
        const at::Tensor &offsets = tensor(a[9], at::kInt, "offsets");
        if (offsets.dim() != 1 || offsets.numel() < 1) raise_value("offsets must be [images + 1]");
        place.same(offsets, "offsets");
        op = pointer<int32_t>(offsets), B = offsets.numel() - 1;
    }
    int64_t N = x.size(packed ? 0 : 1);
    const int64_t channels = x.size(-1);
    if (B > INT32_MAX || channels > INT32_MAX) raise_value("x is too large");
    const int32_t C = (int32_t)channels, G = integer32(a[1]), act = integer32(a[5]), type = kv_dtype(x.scalar_type());
    const double eps = PyFloat_AsDouble(a[4]);
    if (eps == -1 && PyErr_Occurred()) throw Raised();
    const float *wp = vector_of(a[2], "weight", C, place), *bp = vector_of(a[3], "bias", C, place);
    const Rows add(a[6], "add", B, C, place), scale(a[7], "scale", B, C, place), shift(a[8], "shift", B, C, place);
    const at::Tensor out = output(a[11], a[10], x.scalar_type(), x.sizes(), x, place, "out");
    if (!packed && B == 0) B = 1, N = 0;  // no images are no work, like images of no rows
    at::Tensor ws;
    if (given(a[12])) {
        ws = tensor(a[12], at::kByte, "workspace");
        place.same(ws, "workspace");
    } else if (const size_t need = dgq_groupnorm_workspace_bytes((int32_t)B, N, packed, C, G, type)) {
        ws = empty({(int64_t)need}, at::kByte, x);
    }
    void *sp = ws.defined() ? ws.data_ptr() : nullptr, *yp = out.data_ptr();
    const size_t sb = ws.defined() ? (size_t)ws.numel() : 0;
    const void *xp = x.data_ptr();
    enqueue([&] {
        return dgq_groupnorm(xp, type, packed ? 0 : step(x, 0), step(x, packed ? 0 : 1), op, (int32_t)B, N, C, G, wp, bp, (float)eps,
                             add.data, add.stride, scale.data, scale.stride, shift.data, shift.stride, act, yp,
                             kv_dtype(out.scalar_type()), sp, sb, place.stream());
    });
    return one(a[11], out);
}

// (data, out_channels, in_channels, group) from a[0]
struct W4In {
    const at::Tensor &data;
    int32_t O, C, group;
    explicit W4In(Args a) : data(tensor(a[0], at::kByte, "weight.data")), O(integer32(a[1])), C(integer32(a[2])), group(integer32(a[3])) {
        holds(data, (int64_t)dgq_w4_bytes(O, C, group), "weight.data");
    }
};

// (w, data, out_channels, in_channels, group, stream)
PyObject *w4_pack(Args a) {
    const W4In m(a + 1);
    const Place place(a[5], m.data);
    const at::Tensor &w = floats(a[0], "w", 2);
    if (!shape_is(w, {m.O, m.C})) raise_value("w must be [out_channels, in_channels] of the weight");
    place.same(w, "w");
    const void *wp = w.data_ptr();
    void *dp = m.data.data_ptr();
    enqueue([&] { return dgq_w4_pack(wp, kv_dtype(w.scalar_type()), step(w, 0), m.O, m.C, m.group, dp, place.stream()); });
    Py_RETURN_NONE;
}

// (data, out_channels, in_channels, group, dtype, out, stream)
PyObject *w4_unpack(Args a) {
    const W4In m(a);
    const Place place(a[6], m.data);
    const at::Tensor out = output(a[5], a[4], at::kFloat, {m.O, m.C}, m.data, place, "out");
    const void *dp = m.data.data_ptr();
    void *wp = out.data_ptr();
    enqueue([&] { return dgq_w4_unpack(dp, m.O, m.C, m.group, kv_dtype(out.scalar_type()), wp, place.stream()); });
    return one(a[5], out);
}

// (x, data, out_channels, in_channels, group, bias, act, dtype, out, workspace, stream)
PyObject *w4_matvec(Args a) {
    const W4In m(a + 1);
    const Place place(a[10], m.data);
    const at::Tensor &x = floats(a[0], "x", 2);
    if (x.size(1) != m.C) raise_value("x must be [rows, in_channels] of the weight");
    if (x.size(0) > INT32_MAX) raise_value("x is too large");
    place.same(x, "x");
    const int32_t M = (int32_t)x.size(0), act = integer32(a[6]);
    const float *bp = vector_of(a[5], "bias", m.O, place);
    const at::Tensor out = output(a[8], a[7], x.scalar_type(), {M, m.O}, x, place, "out");
    at::Tensor ws;
    if (given(a[9])) {
        ws = tensor(a[9], at::kByte, "workspace");
        place.same(ws, "workspace");
    } else if (const size_t need = dgq_w4_matvec_workspace_bytes(M, m.O, m.C)) {
        ws = empty({(int64_t)need}, at::kByte, x);
    }
    const void *xp = x.data_ptr(), *dp = m.data.data_ptr();
    void *yp = out.data_ptr(), *wp = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t wb = ws.defined() ? (size_t)ws.numel() : 0;
    enqueue([&] {
        return dgq_w4_matvec(xp, kv_dtype(x.scalar_type()), step(x, 0), M, dp, m.O, m.C, m.group, bp, act, yp,
                             kv_dtype(out.scalar_type()), wp, wb, place.stream());
    });
    return one(a[8], out);
}

template <PyObject *(*F)(Args), int NARGS>
PyObject *call(PyObject *, Args a, Py_ssize_t n) {
    if (n != NARGS) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", NARGS, n);
        return nullptr;
    }
    HANDLE_TH_ERRORS  // torch's own errors (out of memory and the like) as its Python calls report them
    try {
        return F(a);
    } catch (const Raised &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyObject *set_error_class(PyObject *, PyObject *cls) {
    Py_INCREF(cls);
    Py_XSETREF(g_error, cls);
    Py_RETURN_NONE;
}

#define DGQ_METHOD(NAME, NARGS) {#NAME, (PyCFunction)(void (*)(void))call<NAME, NARGS>, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    DGQ_METHOD(quantize_act, 5),
    DGQ_METHOD(linear, 8),
    DGQ_METHOD(linear_geglu, 6),
    DGQ_METHOD(linear_geglu_requant, 8),
    DGQ_METHOD(conv3x3_codes, 7),
    DGQ_METHOD(quantize_act_conv3x3, 9),
    DGQ_METHOD(linear_conv3x3, 9),
    DGQ_METHOD(xattn_logq, 10),
    DGQ_METHOD(xattn_logq_static, 10),
    DGQ_METHOD(selfattn_logq, 10),
    DGQ_METHOD(kv_plan, 13),
    DGQ_METHOD(kv_release, 9),
    DGQ_METHOD(kv_store, 9),
    DGQ_METHOD(kv_load, 12),
    DGQ_METHOD(xattn_kv, 12),
    DGQ_METHOD(groupnorm, 14),
    DGQ_METHOD(w4_pack, 6),
    DGQ_METHOD(w4_unpack, 7),
    DGQ_METHOD(w4_matvec, 11),
    {"set_error_class", set_error_class, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_hot", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__hot(void) {
    s_handle = PyUnicode_InternFromString("handle");
    s_out_channels = PyUnicode_InternFromString("out_channels");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (!s_handle || !s_out_channels || !s_cuda_stream) return nullptr;
    return PyModule_Create(&kModule);
}
