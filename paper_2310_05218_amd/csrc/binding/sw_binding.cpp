// The short way from a Python call to the C ABI: checks, output extents, the output tensor and the call in one native function.
//
// run(op, x, w, bias, scale, integers and flags ...; layer norm and attention: their own arguments) returns the output tensor or a tuple of
// them, a status code other than SW_OK, or None for whatever
// it does not take (other types, layouts, devices, arguments out of range): the caller then goes the long way, which takes it or says
// why not.  Nothing is kept between calls but the entry points' addresses.
//
// Measured on one 256 x 256 image under a 3 x 3 filter, whose kernel takes 3.7 us in a graph, calls one after the other: 4.4 to 4.9 us a call,
// 7.05 in Python through ctypes (2.3 of which the checks, 1.4 torch.empty, 0.6 ctypes).  A layer norm of 4 rows of 2048, whose kernel takes 2.3:
// 5.0 us a call, 8.2 in Python; one token of linear attention on 16 heads of 128 x 128, whose kernel takes 4.1: 5.1.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <cmath>

#include "../../../include/swconv.h"

namespace {

enum Op { kConv1d, kPool1d, kPool2d, kConv2d, kBiasRelu, kDilated, kDepthwise, kDepthwiseBiasRelu, kDepthwiseBf16, kS8, kS8Requant, kS8Nhwc, kNhwc, kLayerNorm, kLayerNormBackward,
          kAttention, kAttentionBackward, kAttentionStep };

struct Entries {
    decltype(&sw_conv1d) conv1d;
    decltype(&sw_pool1d) pool1d;
    decltype(&sw_pool2d) pool2d;
    decltype(&sw_conv2d) conv2d;
    decltype(&sw_conv2d_bias_relu) bias_relu;
    decltype(&sw_conv2d_dilated) dilated;
    decltype(&sw_conv2d_depthwise) depthwise;
    decltype(&sw_conv2d_depthwise_bias_relu) depthwise_bias_relu;
    decltype(&sw_conv2d_depthwise_bf16) depthwise_bf16;
    decltype(&sw_conv2d_s8) s8;
    decltype(&sw_conv2d_s8_requant) s8_requant;
    decltype(&sw_conv2d_s8_nhwc) s8_nhwc;
    decltype(&sw_conv2d_s8_nhwc_requant) s8_nhwc_requant;
    decltype(&sw_conv2d_nhwc) nhwc;
    decltype(&sw_conv2d_bf16_nhwc) bf16_nhwc;
    decltype(&sw_conv2d_f16_nhwc) f16_nhwc;
    decltype(&sw_layer_norm) layer_norm;
    decltype(&sw_layer_norm_backward) layer_norm_backward;
    decltype(&sw_layer_norm_backward_workspace_bytes) layer_norm_backward_workspace;
    decltype(&sw_linear_attention) attention;
    decltype(&sw_linear_attention_workspace_bytes) attention_workspace;
    decltype(&sw_linear_attention_backward) attention_backward;
    decltype(&sw_linear_attention_backward_workspace_bytes) attention_backward_workspace;
    decltype(&sw_linear_attention_step) attention_step;
};
Entries g_entry;
constexpr int kEntries = sizeof(Entries) / sizeof(void*);
bool g_bound = false;
bool g_host = false;        // bound to entry points that work on host memory, without a stream

// a contiguous tensor on the GPU of that type and number of dimensions, or null
const at::Tensor* tensor(PyObject* o, at::ScalarType type, int dims)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return (g_host ? t.is_cpu() : t.is_cuda()) && t.scalar_type() == type && t.dim() == dims && t.is_contiguous() ? &t : nullptr;
}

// an exact Python integer within int
bool integer(PyObject* o, int* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long long l = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow || l < INT32_MIN || l > INT32_MAX) return false;
    *v = (int)l;
    return true;
}

bool flag(PyObject* o, int* v)
{
    if (o != Py_True && o != Py_False) return false;
    *v = o == Py_True;
    return true;
}

// output positions along one axis, 0 for what has none (as sw_out_dim_dilated)
int64_t extent(int64_t n, int64_t k, int stride, int pad, int dil)
{
    if (n <= 0 || k <= 0 || stride <= 0 || pad < 0 || dil <= 0) return 0;
    const int64_t span = n + 2 * (int64_t)pad - (dil * (k - 1) + 1);
    return span < 0 ? 0 : span / stride + 1;
}

bool fits(const at::Tensor& t)
{
    for (int64_t d : t.sizes())
        if (d > INT32_MAX) return false;
    return true;
}

// without the interpreter's lock, which is taken back however the scope ends
class Unlocked {
    PyThreadState* const state_ = PyEval_SaveThread();

public:
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state_); }
};

// f(output, stream): the entry point on addresses that were taken before (one that there is not, of a transformed tensor, raises as it is)
template <class F>
PyObject* call(const at::Tensor& x, at::IntArrayRef shape, at::ScalarType type, F&& f)
{
    for (int64_t d : shape)
        if (d <= 0) return nullptr;
    at::Tensor y = at::empty(shape, x.options().dtype(type));
    if (g_host ? !y.is_cpu() : !y.is_cuda()) return nullptr;
    void* const out = y.mutable_data_ptr();
    void* const stream = g_host ? nullptr : static_cast<void*>(c10::hip::getCurrentHIPStream().stream());
    int rc;
    {
        const Unlocked unlocked;
        rc = f(out, stream);
    }
    return rc == SW_OK ? THPVariable_Wrap(std::move(y)) : PyLong_FromLong(rc);
}

// the address of a tensor's memory, whatever an entry point takes it for
struct Address {
    const void* p;
    Address(const at::Tensor* t) : p(t ? t->const_data_ptr() : nullptr) {}
    template <class T>
    operator const T*() const { return static_cast<const T*>(p); }
};

// null: not taken
PyObject* run_op(int op, PyObject* const* a, Py_ssize_t n)
{
    constexpr auto f32 = at::kFloat, bf16 = at::kBFloat16, f16 = at::kHalf, s8 = at::kChar, s32 = at::kInt;
    // a: x, w, bias, scale (None where an op has none), then integers
    if (n < 6) return nullptr;
    PyObject *const px = a[0], *const pw = a[1], *const pb = a[2], *const ps = a[3];
    int i[5] = {0, 0, 0, 0, 0};
    const Py_ssize_t ni = n - 4;
    auto ints = [&](Py_ssize_t want) {
        if (ni < want) return false;
        for (Py_ssize_t k = 0; k < want; ++k)
            if (!integer(a[4 + k], &i[k])) return false;
        return true;
    };
    if (op == kConv1d) {
        const at::Tensor *x = tensor(px, f32, 2), *w = tensor(pw, f32, 1);
        if (!x || !w || !ints(2) || !fits(*w)) return nullptr;
        const int64_t rows = x->size(0), len = x->size(1);
        const int k = (int)w->size(0);
        const Address xa(x), wa(w);
        return call(*x, {rows, extent(len, k, i[0], i[1], 1)}, f32,
                    [&](void* y, void* st) { return g_entry.conv1d(xa, wa, (float*)y, rows, len, k, i[0], i[1], st); });
    }
    if (op == kPool1d) {
        const at::Tensor* x = tensor(px, f32, 2);
        if (!x || !ints(3)) return nullptr;
        const int64_t rows = x->size(0), len = x->size(1);
        const Address xa(x);
        return call(*x, {rows, extent(len, i[0], i[1], 0, 1)}, f32,
                    [&](void* y, void* st) { return g_entry.pool1d(xa, (float*)y, rows, len, i[0], i[1], i[2], st); });
    }
    if (op == kPool2d) {
        const at::Tensor* x = tensor(px, f32, 4);
        if (!x || !ints(5) || !fits(*x)) return nullptr;
        const auto d = x->sizes();
        const Address xa(x);
        return call(*x, {d[0], d[1], extent(d[2], i[0], i[2], i[3], 1), extent(d[3], i[1], i[2], i[3], 1)}, f32, [&](void* y, void* st) {
            return g_entry.pool2d(xa, (float*)y, (int)d[0], (int)d[1], (int)d[2], (int)d[3], i[0], i[1], i[2], i[3], i[4], st);
        });
    }
    if (op == kConv2d || op == kBiasRelu || op == kDilated || op == kS8 || op == kS8Requant) {
        // channel first: x [N,C,H,W], w [K,C,R,S]; integers stride, pad, then relu or dilation
        const bool q = op == kS8 || op == kS8Requant;
        const at::Tensor *x = tensor(px, q ? s8 : f32, 4), *w = tensor(pw, q ? s8 : f32, 4);
        if (!x || !w || !ints(2) || !fits(*x) || !fits(*w)) return nullptr;
        const auto d = x->sizes(), e = w->sizes();
        if (e[1] != d[1]) return nullptr;
        const int N = (int)d[0], C = (int)d[1], H = (int)d[2], W = (int)d[3], K = (int)e[0], R = (int)e[2], S = (int)e[3];
        int relu = 0, dil = 1;
        const at::Tensor *b = nullptr, *sc = nullptr;
        if (op == kDilated) {
            if (ni < 3 || !integer(a[6], &dil)) return nullptr;
        } else if (op != kConv2d && op != kS8) {
            if (ni < 3 || !flag(a[6], &relu)) return nullptr;
            if (pb != Py_None && (!(b = tensor(pb, q ? s32 : f32, 1)) || b->size(0) != K)) return nullptr;
            if (q && (!(sc = tensor(ps, f32, 1)) || sc->size(0) != K)) return nullptr;
        }
        const Address xa(x), wa(w), ba(b), sa(sc);
        return call(*x, {N, K, extent(H, R, i[0], i[1], dil), extent(W, S, i[0], i[1], dil)}, op == kS8 ? s32 : op == kS8Requant ? s8 : f32, [&](void* y, void* st) {
            switch (op) {
            case kConv2d: return g_entry.conv2d(xa, wa, (float*)y, N, C, K, H, W, R, S, i[0], i[1], st);
            case kBiasRelu: return g_entry.bias_relu(xa, wa, ba, (float*)y, N, C, K, H, W, R, S, i[0], i[1], relu, st);
            case kDilated: return g_entry.dilated(xa, wa, (float*)y, N, C, K, H, W, R, S, i[0], i[1], dil, st);
            case kS8: return g_entry.s8(xa, wa, (int32_t*)y, N, C, K, H, W, R, S, i[0], i[1], st);
            default: return g_entry.s8_requant(xa, wa, ba, sa, (int8_t*)y, N, C, K, H, W, R, S, i[0], i[1], relu, st);
            }
        });
    }
    if (op == kDepthwise || op == kDepthwiseBiasRelu || op == kDepthwiseBf16) {
        const auto type = op == kDepthwiseBf16 ? bf16 : f32;
        const at::Tensor *x = tensor(px, type, 4), *w = tensor(pw, f32, 4);
        if (!x || !w || !ints(2) || !fits(*x) || !fits(*w)) return nullptr;
        const auto d = x->sizes(), e = w->sizes();
        if (e[0] != d[1] || e[1] != 1) return nullptr;
        const int N = (int)d[0], C = (int)d[1], H = (int)d[2], W = (int)d[3], R = (int)e[2], S = (int)e[3];
        int relu = 0;
        const at::Tensor* b = nullptr;
        if (op == kDepthwiseBiasRelu) {
            if (ni < 3 || !flag(a[6], &relu)) return nullptr;
            if (pb != Py_None && (!(b = tensor(pb, f32, 1)) || b->size(0) != C)) return nullptr;
        }
        const Address xa(x), wa(w), ba(b);
        return call(*x, {N, C, extent(H, R, i[0], i[1], 1), extent(W, S, i[0], i[1], 1)}, type, [&](void* y, void* st) {
            switch (op) {
            case kDepthwise: return g_entry.depthwise(xa, wa, (float*)y, N, C, H, W, R, S, i[0], i[1], st);
            case kDepthwiseBiasRelu: return g_entry.depthwise_bias_relu(xa, wa, ba, (float*)y, N, C, H, W, R, S, i[0], i[1], relu, st);
            default: return g_entry.depthwise_bf16(xa, wa, (unsigned short*)y, N, C, H, W, R, S, i[0], i[1], st);
            }
        });
    }
    if (op == kS8Nhwc || op == kNhwc) {
        // channel last: x [N,H,W,C], w [K,R,S,C]; integers stride, pad, dilation, relu
        if (!THPVariable_CheckExact(px)) return nullptr;
        const auto type = op == kS8Nhwc ? s8 : THPVariable_Unpack(px).scalar_type();
        if (op == kNhwc && type != f32 && type != bf16 && type != f16) return nullptr;
        const at::Tensor *x = tensor(px, type, 4), *w = tensor(pw, type, 4);
        int relu = 0;
        if (!x || !w || !ints(3) || ni < 4 || !flag(a[7], &relu) || !fits(*x) || !fits(*w)) return nullptr;
        const auto d = x->sizes(), e = w->sizes();
        if (e[3] != d[3]) return nullptr;
        const int N = (int)d[0], H = (int)d[1], W = (int)d[2], C = (int)d[3], K = (int)e[0], R = (int)e[1], S = (int)e[2];
        const at::Tensor *b = nullptr, *sc = nullptr;
        const bool q = op == kS8Nhwc && ps != Py_None;
        if (q && (!(sc = tensor(ps, f32, 1)) || sc->size(0) != K)) return nullptr;
        if ((q || op == kNhwc) && pb != Py_None && (!(b = tensor(pb, q ? s32 : f32, 1)) || b->size(0) != K)) return nullptr;
        const Address xa(x), wa(w), ba(b), sa(sc);
        const auto out = op == kNhwc ? type : q ? s8 : s32;
        return call(*x, {N, extent(H, R, i[0], i[1], i[2]), extent(W, S, i[0], i[1], i[2]), K}, out, [&](void* y, void* st) {
            if (op == kS8Nhwc)
                return q ? g_entry.s8_nhwc_requant(xa, wa, ba, sa, (int8_t*)y, N, H, W, C, K, R, S, i[0], i[1], relu, st)
                         : g_entry.s8_nhwc(xa, wa, (int32_t*)y, N, H, W, C, K, R, S, i[0], i[1], st);
            if (type == f32) return g_entry.nhwc(xa, wa, ba, (float*)y, N, H, W, C, K, R, S, i[0], i[1], i[2], relu, st);
            if (type == bf16) return g_entry.bf16_nhwc(xa, wa, ba, y, N, H, W, C, K, R, S, i[0], i[1], i[2], relu, st);
            return g_entry.f16_nhwc(xa, wa, ba, y, N, H, W, C, K, R, S, i[0], i[1], i[2], relu, st);
        });
    }
    return nullptr;
}

// ---- layer norm and linear attention: several outputs, strided tensors, workspaces --------------------------------------------------

// the sw_type of a tensor on the GPU; false: none
bool type_of(const at::Tensor& t, int* type)
{
    const auto k = t.scalar_type();
    *type = k == at::kFloat ? SW_F32 : k == at::kBFloat16 ? SW_BF16 : SW_F16;
    return (g_host ? t.is_cpu() : t.is_cuda()) && (k == at::kFloat || k == at::kBFloat16 || k == at::kHalf);
}

const at::Tensor* any_tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

// a contiguous tensor of that type and shape, or None where that may be (*t null then)
bool plain(PyObject* o, at::ScalarType type, at::IntArrayRef shape, bool none, const at::Tensor** t)
{
    *t = nullptr;
    if (o == Py_None) return none;
    *t = tensor(o, type, (int)shape.size());
    return *t && (*t)->sizes() == shape;
}

// a Python number that a float holds, `none` for None
bool number(PyObject* o, double none, float* v)
{
    double d = none;
    if (PyFloat_CheckExact(o))
        d = PyFloat_AS_DOUBLE(o);
    else if (o != Py_None)
        return false;
    if (!(d >= -3e38 && d <= 3e38)) return false;
    *v = (float)d;
    return true;
}

// rows of the last dimension, evenly apart
struct Rows {
    int64_t rows, width, stride;
    bool set(const at::Tensor& t)
    {
        if (t.dim() < 1 || t.numel() == 0) return false;
        const auto n = t.sizes(), s = t.strides();
        const int last = (int)t.dim() - 1;
        width = n[last];
        rows = t.numel() / width, stride = width;
        if (t.is_contiguous()) return true;
        if (s[last] != 1 && width > 1) return false;
        int64_t done = 1;
        for (int i = last - 1; i >= 0; --i) {
            if (n[i] == 1) continue;
            if (done == 1)
                stride = s[i];
            else if (s[i] != done * stride)
                return false;
            done *= n[i];
        }
        return true;
    }
};

// f(stream) without the lock; then `count` tensors as a tuple (one as it is), or the status
template <class F>
PyObject* call_into(at::Tensor* const* out, int count, F&& f)
{
    void* const stream = g_host ? nullptr : static_cast<void*>(c10::hip::getCurrentHIPStream().stream());
    int rc;
    {
        const Unlocked unlocked;
        rc = f(stream);
    }
    if (rc != SW_OK) return PyLong_FromLong(rc);
    if (count == 1) return THPVariable_Wrap(*out[0]);
    PyObject* all = PyTuple_New(count);
    for (int i = 0; all && i < count; ++i) {
        PyObject* one = Py_None;
        if (out[i])
            one = THPVariable_Wrap(*out[i]);
        else
            Py_INCREF(one);
        if (!one) {
            Py_DECREF(all);
            return nullptr;
        }
        PyTuple_SET_ITEM(all, i, one);
    }
    return all;
}

float* floats(const at::Tensor* t) { return t ? static_cast<float*>(t->mutable_data_ptr()) : nullptr; }

// (x, weight, bias, eps, stats), (dy, x, weight, mean, rstd, params)
PyObject* run_norm(bool backward, PyObject* const* a, Py_ssize_t n)
{
    if (n != (backward ? 6 : 5)) return nullptr;
    const at::Tensor *x = any_tensor(a[backward ? 1 : 0]), *w, *b = nullptr;
    int type, flags;
    Rows rx;
    if (!x || !type_of(*x, &type) || !rx.set(*x)) return nullptr;
    const int64_t width[1] = {rx.width};
    if (!flag(a[n - 1], &flags) || !plain(a[backward ? 2 : 1], at::kFloat, width, true, &w)) return nullptr;
    const auto stats = x->sizes().slice(0, x->dim() - 1);
    const auto f32 = x->options().dtype(at::kFloat);
    if (!backward) {
        float eps;
        if (!plain(a[2], at::kFloat, width, true, &b) || a[3] == Py_None || !number(a[3], 0, &eps)) return nullptr;
        const Address xa(x), wa(w), ba(b);
        at::Tensor y = at::empty(x->sizes(), x->options()), mean, rstd;
        if (flags) mean = at::empty(stats, f32), rstd = at::empty(stats, f32);
        void* const yp = y.mutable_data_ptr();
        float *const mp = flags ? floats(&mean) : nullptr, *const rp = flags ? floats(&rstd) : nullptr;
        at::Tensor* const out[3] = {&y, &mean, &rstd};
        return call_into(out, flags ? 3 : 1, [&](void* st) {
            return g_entry.layer_norm(xa.p, wa, ba, yp, mp, rp, rx.rows, rx.width, rx.stride, rx.width, eps, type, st);
        });
    }
    const at::Tensor *dy = any_tensor(a[0]), *mean, *rstd;
    Rows rdy;
    int dtype;
    if (!dy || !type_of(*dy, &dtype) || dtype != type || dy->sizes() != x->sizes() || !rdy.set(*dy) || !plain(a[3], at::kFloat, stats, false, &mean) ||
        !plain(a[4], at::kFloat, stats, false, &rstd))
        return nullptr;
    const Address da(dy), xa(x), wa(w), ma(mean), ra(rstd);
    at::Tensor dx = at::empty(x->sizes(), x->options()), dw, db, work;
    int64_t need = 0;
    if (flags) {
        need = g_entry.layer_norm_backward_workspace(rx.rows, rx.width);
        dw = at::empty(width, f32), db = at::empty(width, f32), work = at::empty({need}, x->options().dtype(at::kByte));
    }
    void *const dxp = dx.mutable_data_ptr(), *const wp = need ? work.mutable_data_ptr() : nullptr;
    float *const dwp = flags ? floats(&dw) : nullptr, *const dbp = flags ? floats(&db) : nullptr;
    at::Tensor* const out[3] = {&dx, flags ? &dw : nullptr, flags ? &db : nullptr};
    return call_into(out, 3, [&](void* st) {
        return g_entry.layer_norm_backward(da.p, xa.p, wa, ma, ra, dxp, dwp, dbp, rx.rows, rx.width, rdy.stride, rx.stride, rx.width, type, wp, need, st);
    });
}

// [..., heads, width] of that type and shape, the innermost dimension contiguous
bool heads_of(PyObject* o, const at::Tensor& like, at::IntArrayRef shape, const at::Tensor** t, sw_strides* s)
{
    *t = any_tensor(o);
    if (!*t || (*t)->is_cuda() != like.is_cuda() || (*t)->scalar_type() != like.scalar_type() || (*t)->sizes() != shape) return false;
    const auto st = (*t)->strides();
    const size_t d = st.size();
    if (st[d - 1] != 1 && shape[d - 1] > 1) return false;
    *s = sw_strides{d == 4 ? st[0] : 0, st[d - 3], st[d - 2]};
    return true;
}

sw_strides strides_of(at::IntArrayRef shape)
{
    const size_t d = shape.size();
    return sw_strides{d == 4 ? shape[1] * shape[2] * shape[3] : 0, shape[d - 2] * shape[d - 1], shape[d - 1]};
}

// (q, k, v, log_decay, scale, starts, state, slots, final_state), (do, q, k, v, log_decay, scale, starts, state, slots, d_final_state, d_state)
// and (q, k, v, log_decay, scale, state, slots)
PyObject* run_attention(int op, PyObject* const* a, Py_ssize_t n)
{
    const bool step = op == kAttentionStep, backward = op == kAttentionBackward;
    if (n != (step ? 7 : backward ? 11 : 9)) return nullptr;
    PyObject* const pdo = backward ? *a++ : nullptr;
    PyObject *const pstarts = step ? Py_None : a[5], *const pstate = a[step ? 5 : 6], *const pslots = a[step ? 6 : 7];
    const at::Tensor *q = any_tensor(a[0]), *k = any_tensor(a[1]), *v = any_tensor(a[2]), *starts = nullptr, *slots, *decay;
    const bool packed = pstarts != Py_None;
    const int64_t dim = step || packed ? 3 : 4;
    sw_linear_attention_dims d{};
    if (!q || !k || !v || !type_of(*q, &d.type) || q->dim() != dim || k->dim() != dim || v->dim() != dim || q->numel() == 0 || k->numel() == 0 ||
        v->numel() == 0 || !fits(*q) || !fits(*k) || !fits(*v))
        return nullptr;
    if (packed && (!(starts = tensor(pstarts, at::kInt, 1)) || starts->size(0) < 2 || starts->size(0) > INT32_MAX)) return nullptr;
    d.heads = (int)q->size(dim - 2), d.kv_heads = (int)v->size(dim - 2), d.dk = (int)q->size(dim - 1), d.dv = (int)v->size(dim - 1);
    d.B = packed ? (int)starts->size(0) - 1 : (int)q->size(0);
    d.T = step ? 1 : q->size(dim - 3);
    if (d.heads % d.kv_heads || !number(a[4], std::pow((double)d.dk, -0.5), &d.scale)) return nullptr;
    // shapes [..., heads, width] on q's first dimensions
    int64_t sq[4], sk[4], sv[4], so[4];
    for (int i = 0; i < dim - 2; ++i) sq[i] = sk[i] = sv[i] = so[i] = q->size(i);
    sq[dim - 2] = so[dim - 2] = d.heads, sk[dim - 2] = sv[dim - 2] = d.kv_heads;
    sq[dim - 1] = sk[dim - 1] = d.dk, sv[dim - 1] = so[dim - 1] = d.dv;
    const at::IntArrayRef nq(sq, dim), nk(sk, dim), nv(sv, dim), no(so, dim);
    sw_strides tq, tk, tv, tdo;
    const int64_t heads[1] = {d.heads}, sequences[1] = {d.B};
    const at::Tensor* d_o = nullptr;
    if (!heads_of(a[0], *q, nq, &q, &tq) || !heads_of(a[1], *q, nk, &k, &tk) || !heads_of(a[2], *q, nv, &v, &tv) ||
        (backward && !heads_of(pdo, *q, no, &d_o, &tdo)) || !plain(a[3], at::kFloat, heads, false, &decay) ||
        !plain(pslots, at::kInt, sequences, true, &slots))
        return nullptr;
    auto states = [&](PyObject* o, int64_t count, const at::Tensor** t) {
        const int64_t shape[4] = {count, d.heads, d.dk, d.dv};
        return plain(o, at::kFloat, shape, true, t);
    };
    PyObject* const pfinal = step ? Py_None : a[8];         // (backward: d_final_state)
    const at::Tensor *held = any_tensor(pstate != Py_None || backward ? pstate : pfinal), *state, *last, *d_state = nullptr;
    if (held && (held->dim() != 4 || held->size(0) > INT32_MAX)) return nullptr;
    d.n_states = held ? (int)held->size(0) : 0;
    if (!states(pstate, d.n_states, &state) || !states(pfinal, backward ? d.B : d.n_states, &last) || (step && !state) ||
        (backward && !states(a[9], d.B, &d_state)))
        return nullptr;
    const Address qa(q), ka(k), va(v), ga(decay), sa(slots), ca(starts);
    const auto options = q->options();
    if (step) {
        float* const sp = floats(state);
        at::Tensor o = at::empty(no, options);
        void* const op = o.mutable_data_ptr();
        auto as_rows = [](sw_strides s) { return sw_strides{s.token, 0, s.head}; };
        tq = as_rows(tq), tk = as_rows(tk), tv = as_rows(tv);
        const sw_strides to = as_rows(strides_of(no));
        at::Tensor* const out[1] = {&o};
        return call_into(out, 1, [&](void* st) { return g_entry.attention_step(qa.p, ka.p, va.p, op, ga, sp, sa, &d, &tq, &tk, &tv, &to, st); });
    }
    at::Tensor work;
    const int64_t need = backward ? g_entry.attention_backward_workspace(&d, packed) : g_entry.attention_workspace(&d, packed);
    if (need) work = at::empty({need}, options.dtype(at::kByte));
    void* const wp = need ? work.mutable_data_ptr() : nullptr;
    const Address first(state);
    if (!backward) {
        float* const lp = floats(last);
        at::Tensor o = at::empty(no, options);
        void* const op = o.mutable_data_ptr();
        const sw_strides to = strides_of(no);
        at::Tensor* const out[1] = {&o};
        return call_into(out, 1, [&](void* st) {
            return g_entry.attention(qa.p, ka.p, va.p, op, ga, first, lp, sa, ca, &d, &tq, &tk, &tv, &to, wp, need, st);
        });
    }
    const Address da(d_o), fa(last);
    float* const gs = floats(d_state);
    at::Tensor dq = at::empty(nq, options), dk = at::empty(nk, options), dv = at::empty(nv, options);
    void *const gq = dq.mutable_data_ptr(), *const gk = dk.mutable_data_ptr(), *const gv = dv.mutable_data_ptr();
    const sw_strides uq = strides_of(nq), uk = strides_of(nk), uv = strides_of(nv);
    at::Tensor* const out[3] = {&dq, &dk, &dv};
    return call_into(out, 3, [&](void* st) {
        return g_entry.attention_backward(da.p, qa.p, ka.p, va.p, ga, first, fa, gq, gk, gv, gs, sa, ca, &d, &tdo, &tq, &tk, &tv, &uq, &uk, &uv, wp, need, st);
    });
}

PyObject* run(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    int op;
    if (g_bound && n >= 1 && integer(a[0], &op)) {
        try {
            PyObject* y;
            if (op == kLayerNorm || op == kLayerNormBackward)
                y = run_norm(op == kLayerNormBackward, a + 1, n - 1);
            else if (op >= kAttention && op <= kAttentionStep)
                y = run_attention(op, a + 1, n - 1);
            else
                y = run_op(op, a + 1, n - 1);
            if (y) return y;
        } catch (...) {
            // (a tensor without storage, memory that is not there: the long way says it as it always has)
        }
        if (PyErr_Occurred()) PyErr_Clear();
    }
    Py_RETURN_NONE;
}

// bind(addresses of the entry points in the order of Entries, host = False); host: entry points for tensors in host memory, as tests have them
PyObject* bind(PyObject*, PyObject* args)
{
    PyObject* addresses;
    int host = 0;
    if (!PyArg_ParseTuple(args, "O|p", &addresses, &host)) return nullptr;
    if (!PyTuple_CheckExact(addresses) || PyTuple_GET_SIZE(addresses) != kEntries) {
        PyErr_SetString(PyExc_ValueError, "one address per entry point");
        return nullptr;
    }
    void* p[kEntries];
    for (int k = 0; k < kEntries; ++k) {
        p[k] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, k));
        if (!p[k]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
            return nullptr;
        }
    }
    static_assert(sizeof p == sizeof g_entry, "entries are addresses");
    std::memcpy(&g_entry, p, sizeof g_entry);
    g_host = host != 0;
    g_bound = true;
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"run", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(run)), METH_FASTCALL, nullptr},
    {"bind", bind, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_swnative", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__swnative(void) { return PyModule_Create(&kModule); }
