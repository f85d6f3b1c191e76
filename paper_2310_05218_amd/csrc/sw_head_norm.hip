// Norms of the heads of queries and keys with their rotation: a wavefront a head.
#include "sw_sequence.h"

namespace swconv {

namespace {

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// cos and sin of position * frequency
__device__ __forceinline__ void angle(int position, float frequency, float* c, float* s)
{
    const double f = (double)position * (double)frequency;
    *c = (float)cos(f), *s = (float)sin(f);
}

constexpr int kMost = 4;        // elements of a lane: heads of up to 256

template <int EK, bool BACKWARD>
__global__ __launch_bounds__(256) void head_norm_kernel(HeadNormArgs p)
{
    typedef typename ElemOf<EK>::type T;
    __shared__ float lds[4][256];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, heads = p.side[0].heads + p.side[1].heads;
    const int64_t tasks = p.B * p.T * heads;
    float sums[2][kMost] = {};
    for (int64_t task = blockIdx.x * 4 + wave; task < tasks; task += gridDim.x * 4) {
        const int64_t row = task / heads, batch = row / p.T, token = row % p.T;
        const int all = (int)(task % heads), which = all >= p.side[0].heads, head = all - (which ? p.side[0].heads : 0);
        const HeadNormSide side = which ? p.side[1] : p.side[0];
        auto place = [&](const AttentionOperand& o) { return static_cast<const T*>(o.p) + batch * o.batch + token * o.token + (int64_t)head * o.head; };
        const T* x = place(side.x);
        const int position = p.positions ? p.positions[row] : (int)token;
        float v[kMost], w[kMost], other[kMost] = {}, c[kMost] = {}, s[kMost] = {}, sum = 0.f;
#pragma unroll
        for (int k = 0; k < kMost; ++k) {
            const int e = lane + 64 * k;
            v[k] = e < p.D ? (float)x[e] : 0.f;
            w[k] = e < p.D && side.weight ? side.weight[e] : 1.f;
            sum += v[k] * v[k];
        }
        const float r = 1.f / sqrtf(wave_sum(sum) / (float)p.D + p.eps);
        // what turns with element e: its partner, and the angle (the sign is that of the partner's term)
        int with[kMost];
#pragma unroll
        for (int k = 0; k < kMost; ++k) {
            const int e = lane + 64 * k;
            with[k] = e;
            if (e >= 2 * p.pairs) continue;
            const bool second = p.interleaved ? e % 2 : e >= p.pairs;
            const int pair = p.interleaved ? e / 2 : second ? e - p.pairs : e;
            with[k] = p.interleaved ? e ^ 1 : second ? e - p.pairs : e + p.pairs;
            angle(position, p.frequencies[pair], &c[k], &s[k]);
            if (!second) s[k] = -s[k];
            if (BACKWARD) s[k] = -s[k];
        }
        if constexpr (!BACKWARD) {
            T* y = const_cast<T*>(place(side.y));
#pragma unroll
            for (int k = 0; k < kMost; ++k)
                if (lane + 64 * k < p.D && with[k] != lane + 64 * k)
                    other[k] = (float)x[with[k]] * r * (side.weight ? side.weight[with[k]] : 1.f);
            // (y may be x: no lane stores before all have read)
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < kMost; ++k) {
                const int e = lane + 64 * k;
                const float n = v[k] * r * w[k];
                if (e < p.D) y[e] = (T)(with[k] == e ? n : n * c[k] + other[k] * s[k]);
            }
        } else {
            const T* dy = place(side.dy);
            T* dx = const_cast<T*>(place(side.y));
            float g[kMost], dot = 0.f;
#pragma unroll
            for (int k = 0; k < kMost; ++k) {
                const int e = lane + 64 * k;
                g[k] = e < p.D ? (float)dy[e] : 0.f;
                if (e < p.D && with[k] != e) g[k] = g[k] * c[k] + (float)dy[with[k]] * s[k];
                v[k] *= r;
                if (e < p.D) sums[which][k] += g[k] * v[k];
                g[k] *= w[k];
                dot += g[k] * v[k];
            }
            dot = wave_sum(dot) / (float)p.D;
#pragma unroll
            for (int k = 0; k < kMost; ++k)
                if (lane + 64 * k < p.D) dx[lane + 64 * k] = (T)(r * (g[k] - v[k] * dot));
        }
    }
    if constexpr (BACKWARD) {
        if (!p.work) return;
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kMost; ++k) lds[wave][lane + 64 * k] = sums[which][k];
            __syncthreads();
            if ((int)threadIdx.x < p.D)
                static_cast<float*>(p.work)[((int64_t)blockIdx.x * 2 + which) * p.D + threadIdx.x] =
                    lds[0][threadIdx.x] + lds[1][threadIdx.x] + lds[2][threadIdx.x] + lds[3][threadIdx.x];
        }
    }
}

__global__ __launch_bounds__(256) void head_norm_fold_kernel(const float* partial, int parts, int D, float* dq, float* dk)
{
    const int e = threadIdx.x;
    float* out = blockIdx.x ? dk : dq;
    if (e >= D || !out) return;
    float s = 0.f;
    for (int k = 0; k < parts; ++k) s += partial[((int64_t)k * 2 + blockIdx.x) * D + e];
    out[e] = s;
}

unsigned groups_of(int64_t tasks)
{
    const int64_t want = (tasks + 3) / 4;
    return (unsigned)(want < 2048 ? want : 2048);
}

}  // namespace

int64_t head_norm_backward_workspace(int64_t rows, int heads, int kv_heads, int D) { return (int64_t)groups_of(rows * (heads + kv_heads)) * 2 * D * 4; }

hipError_t launch_head_norm(const HeadNormArgs& a, int ek, hipStream_t st)
{
    return with_elem(ek, [&](auto e) {
        note_kernel("head_norm_kernel", ek);
        hipLaunchKernelGGL((head_norm_kernel<e(), false>), dim3(groups_of(a.B * a.T * (a.side[0].heads + a.side[1].heads))), dim3(256), 0, st, a);
        return hipGetLastError();
    });
}

hipError_t launch_head_norm_backward(const HeadNormArgs& args, int ek, hipStream_t st)
{
    HeadNormArgs a = args;
    if (!a.side[0].dweight && !a.side[1].dweight) a.work = nullptr;
    return with_elem(ek, [&](auto e) {
        const unsigned groups = groups_of(a.B * a.T * (a.side[0].heads + a.side[1].heads));
        note_kernel("head_norm_backward_kernel", ek);
        hipLaunchKernelGGL((head_norm_kernel<e(), true>), dim3(groups), dim3(256), 0, st, a);
        if (const hipError_t err = hipGetLastError()) return err;
        if (a.work)
            hipLaunchKernelGGL(head_norm_fold_kernel, dim3(2), dim3(256), 0, st, static_cast<const float*>(a.work), (int)groups, a.D, a.side[0].dweight, a.side[1].dweight);
        return hipGetLastError();
    });
}

}  // namespace swconv
