// Gated linear recurrence: a thread a channel of a sequence, token after token.
#include "sw_gates.h"
#include "sw_sequence.h"

namespace swconv {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t clamped(int64_t v, int64_t most) { return v < 0 ? 0 : v > most ? most : v; }

struct Rows {
    int64_t first, last, left, right;       // of the sequence; zeros go to [left, first) and [last, right)
    int entry;                              // of state; -1: none
};
__device__ __forceinline__ Rows rows_of(const RecurrenceBatch& n, int b)
{
    Rows r;
    if (n.starts) {
        r.first = clamped(n.starts[b], n.T), r.last = clamped(n.starts[b + 1], n.T);
        r.left = b == 0 ? 0 : r.first, r.right = b == n.B - 1 ? n.T : r.last;
    } else {
        r.first = r.left = 0, r.last = r.right = n.T;
    }
    r.entry = n.slots ? n.slots[b] : b;
    if (r.entry < 0 || r.entry >= n.n_states) r.entry = -1;
    return r;
}

template <int EK>
__device__ __forceinline__ const typename ElemOf<EK>::type* at(const Channels& c, int64_t batch, int channel)
{
    return static_cast<const typename ElemOf<EK>::type*>(c.p) + batch * c.batch + channel;
}
template <int EK>
__device__ __forceinline__ typename ElemOf<EK>::type* to(const Channels& c, int64_t batch, int channel)
{
    return static_cast<typename ElemOf<EK>::type*>(const_cast<void*>(c.p)) + batch * c.batch + channel;
}

template <int EK>
__global__ __launch_bounds__(kThreads) void recurrence_kernel(RecurrenceArgs p, int groups)
{
    typedef typename ElemOf<EK>::type T;
    const int b = blockIdx.x / groups, c = blockIdx.x % groups * kThreads + threadIdx.x;
    if (c >= p.n.C) return;
    const Rows rows = rows_of(p.n, b);
    const int64_t batch = p.n.starts ? 0 : b;
    const T *x = at<EK>(p.x, batch, c), *r = at<EK>(p.decay_gate, batch, c), *i = at<EK>(p.input_gate, batch, c);
    T* h = to<EK>(p.h, batch, c);
    const float log_decay = finite_decay(p.n.log_decay[c]);
    float now = p.state && rows.entry >= 0 ? p.state[(int64_t)rows.entry * p.n.C + c] : 0.f;
    for (int64_t t = rows.left; t < rows.first; ++t) h[t * p.h.token] = (T)0.f;
    for (int64_t t = rows.first; t < rows.last; ++t) {
        const Gate<EK> g(log_decay, (float)r[t * p.decay_gate.token], (float)i[t * p.input_gate.token]);
        now = __builtin_fmaf(g.a, now, g.w * g.p * (float)x[t * p.x.token]);
        h[t * p.h.token] = (T)now;
    }
    for (int64_t t = rows.last; t < rows.right; ++t) h[t * p.h.token] = (T)0.f;
    if (p.final_state && rows.entry >= 0) p.final_state[(int64_t)rows.entry * p.n.C + c] = now;
}

template <int EK>
__global__ __launch_bounds__(kThreads) void recurrence_backward_kernel(RecurrenceBackwardArgs p, int groups)
{
    typedef typename ElemOf<EK>::type T;
    const int b = blockIdx.x / groups, c = blockIdx.x % groups * kThreads + threadIdx.x;
    if (c >= p.n.C) return;
    const Rows rows = rows_of(p.n, b);
    const int64_t batch = p.n.starts ? 0 : b;
    const T *dh = at<EK>(p.dh, batch, c), *x = at<EK>(p.x, batch, c), *r = at<EK>(p.decay_gate, batch, c), *i = at<EK>(p.input_gate, batch, c),
            *h = at<EK>(p.h, batch, c);
    T *dx = to<EK>(p.dx, batch, c), *dr = to<EK>(p.d_decay_gate, batch, c), *di = to<EK>(p.d_input_gate, batch, c);
    auto zeros = [&](int64_t first, int64_t last) {
        for (int64_t t = first; t < last; ++t) dx[t * p.dx.token] = dr[t * p.d_decay_gate.token] = di[t * p.d_input_gate.token] = (T)0.f;
    };
    zeros(rows.left, rows.first);
    zeros(rows.last, rows.right);
    const float log_decay = finite_decay(p.n.log_decay[c]);
    const float first = p.state && rows.entry >= 0 ? p.state[(int64_t)rows.entry * p.n.C + c] : 0.f;
    float later = p.d_final_state ? p.d_final_state[(int64_t)b * p.n.C + c] : 0.f, sum = 0.f;
    for (int64_t t = rows.last - 1; t >= rows.first; --t) {
        const float gr = (float)r[t * p.decay_gate.token], gi = (float)i[t * p.input_gate.token], xt = (float)x[t * p.x.token];
        const Gate<EK> g(log_decay, gr, gi);
        const float u = (float)dh[t * p.dh.token] + later, before = t > rows.first ? (float)h[(t - 1) * p.h.token] : first;
        const float dw = g.w > 0.f ? g.a * g.a * __builtin_amdgcn_rcpf(g.w) : 0.f;
        const float l = u * (g.a * before - g.p * xt * dw);
        dx[t * p.dx.token] = (T)(u * g.w * g.p);
        di[t * p.d_input_gate.token] = (T)(u * g.w * xt * g.p * g.shut_p(gi));
        dr[t * p.d_decay_gate.token] = (T)(l * g.L * g.shut_s(gr));
        sum = __builtin_fmaf(l, g.s, sum);
        later = g.a * u;
    }
    if (p.d_state) p.d_state[(int64_t)b * p.n.C + c] = later;
    if (p.d_log_decay) static_cast<float*>(p.work)[(int64_t)b * p.n.C + c] = sum;
}

__global__ __launch_bounds__(kThreads) void recurrence_fold_kernel(const float* partial, int parts, int C, float* sums)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= C) return;
    float s = 0.f;
    for (int k = 0; k < parts; ++k) s += partial[(int64_t)k * C + c];
    sums[c] = s;
}

template <int EK>
__global__ __launch_bounds__(kThreads) void recurrence_step_kernel(RecurrenceStepArgs p, int groups)
{
    typedef typename ElemOf<EK>::type T;
    const int b = blockIdx.x / groups, c = blockIdx.x % groups * kThreads + threadIdx.x;
    if (c >= p.n.C) return;
    T* h = to<EK>(p.h, b, c);
    const int entry = p.n.slots ? p.n.slots[b] : b;
    if (entry < 0 || entry >= p.n.n_states) {
        *h = (T)0.f;
        return;
    }
    float* state = p.state + (int64_t)entry * p.n.C + c;
    const Gate<EK> g(finite_decay(p.n.log_decay[c]), (float)*at<EK>(p.decay_gate, b, c), (float)*at<EK>(p.input_gate, b, c));
    const float now = __builtin_fmaf(g.a, *state, g.w * g.p * (float)*at<EK>(p.x, b, c));
    *state = now;
    *h = (T)now;
}

}  // namespace

int64_t recurrence_workspace(const RecurrenceBatch&, bool, int) { return 0; }
int64_t recurrence_backward_workspace(const RecurrenceBatch& n, bool, int) { return (int64_t)n.B * n.C * 4; }

hipError_t launch_recurrence(const RecurrenceArgs& a, int ek, hipStream_t st)
{
    const int groups = (a.n.C + kThreads - 1) / kThreads;
    return with_elem(ek, [&](auto e) {
        SW_NOTED_LAUNCH(note_kernel("recurrence_kernel", ek), recurrence_kernel<e()>, dim3(groups * a.n.B), dim3(kThreads), 0, st, a, groups);
        return hipGetLastError();
    });
}

hipError_t launch_recurrence_backward(const RecurrenceBackwardArgs& a, int ek, hipStream_t st)
{
    const int groups = (a.n.C + kThreads - 1) / kThreads;
    return with_elem(ek, [&](auto e) {
        SW_NOTED_LAUNCH(note_kernel("recurrence_backward_kernel", ek), recurrence_backward_kernel<e()>, dim3(groups * a.n.B), dim3(kThreads), 0, st, a, groups);
        if (const hipError_t err = hipGetLastError()) return err;
        if (a.d_log_decay)
            hipLaunchKernelGGL(recurrence_fold_kernel, dim3(groups), dim3(kThreads), 0, st, static_cast<const float*>(a.work), a.n.B, a.n.C, a.d_log_decay);
        return hipGetLastError();
    });
}

hipError_t launch_recurrence_step(const RecurrenceStepArgs& a, int ek, hipStream_t st)
{
    const int groups = (a.n.C + kThreads - 1) / kThreads;
    return with_elem(ek, [&](auto e) {
        SW_NOTED_LAUNCH(note_kernel("recurrence_step_kernel", ek), recurrence_step_kernel<e()>, dim3(groups * a.n.B), dim3(kThreads), 0, st, a, groups);
        return hipGetLastError();
    });
}

}  // namespace swconv
