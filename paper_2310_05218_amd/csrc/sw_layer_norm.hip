// Layer norm over the channels of channel-last rows, and its backward pass.
#include "sw_layers.h"

namespace swconv {

namespace {

constexpr int kThreads = 256;

// The sum over a workgroup, in every thread.
__device__ __forceinline__ float block_sum(float v, float* lds)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    float s = 0.f;
    for (int i = 0; i < kThreads / 64; ++i) s += lds[i];
    return s;
}

template <int EK>
__global__ __launch_bounds__(kThreads) void layer_norm_kernel(LayerNormArgs p)
{
    typedef typename ElemOf<EK>::type T;
    __shared__ float lds[kThreads / 64];
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
        T* y = static_cast<T*>(p.y) + row * p.y_stride;
        float s = 0.f;
        for (int i = threadIdx.x; i < p.C; i += kThreads) s += (float)x[i];
        const float mean = block_sum(s, lds) / (float)p.C;
        s = 0.f;
        for (int i = threadIdx.x; i < p.C; i += kThreads) {
            const float d = (float)x[i] - mean;
            s += d * d;
        }
        const float rstd = 1.0f / sqrtf(block_sum(s, lds) / (float)p.C + p.eps);
        for (int i = threadIdx.x; i < p.C; i += kThreads) {
            const float h = ((float)x[i] - mean) * rstd;
            y[i] = (T)(h * (p.weight ? p.weight[i] : 1.0f) + (p.bias ? p.bias[i] : 0.0f));
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

template <int EK>
__global__ __launch_bounds__(kThreads) void layer_norm_dx_kernel(LayerNormBackwardArgs p)
{
    typedef typename ElemOf<EK>::type T;
    __shared__ float lds[kThreads / 64];
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
        const T* dy = static_cast<const T*>(p.dy) + row * p.dy_stride;
        T* dx = static_cast<T*>(p.dx) + row * p.dx_stride;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float sg = 0.f, sgh = 0.f;
        for (int i = threadIdx.x; i < p.C; i += kThreads) {
            const float g = (float)dy[i] * (p.weight ? p.weight[i] : 1.0f);
            sg += g;
            sgh += g * (((float)x[i] - mean) * rstd);
        }
        sg = block_sum(sg, lds) / (float)p.C;
        sgh = block_sum(sgh, lds) / (float)p.C;
        for (int i = threadIdx.x; i < p.C; i += kThreads) {
            const float g = (float)dy[i] * (p.weight ? p.weight[i] : 1.0f);
            const float h = ((float)x[i] - mean) * rstd;
            dx[i] = (T)(rstd * (g - sg - h * sgh));
        }
    }
}

// sums of a run of rows, a column per thread: partial[run] = {dweight[C], dbias[C]}
template <int EK>
__global__ __launch_bounds__(kThreads) void layer_norm_sums_kernel(LayerNormBackwardArgs p, int64_t run)
{
    typedef typename ElemOf<EK>::type T;
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= p.C) return;
    const int64_t first = blockIdx.y * run, last = first + run < p.rows ? first + run : p.rows;
    float sw = 0.f, sb = 0.f;
    for (int64_t row = first; row < last; ++row) {
        const float dy = (float)static_cast<const T*>(p.dy)[row * p.dy_stride + i];
        sw += dy * (((float)static_cast<const T*>(p.x)[row * p.x_stride + i] - p.mean[row]) * p.rstd[row]);
        sb += dy;
    }
    p.partial[(int64_t)blockIdx.y * 2 * p.C + i] = sw;
    p.partial[(int64_t)blockIdx.y * 2 * p.C + p.C + i] = sb;
}

__global__ __launch_bounds__(kThreads) void layer_norm_fold_kernel(const float* partial, int parts, int C, float* dweight, float* dbias)
{
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= C) return;
    float sw = 0.f, sb = 0.f;
    for (int k = 0; k < parts; ++k) {
        sw += partial[(int64_t)k * 2 * C + i];
        sb += partial[(int64_t)k * 2 * C + C + i];
    }
    if (dweight) dweight[i] = sw;
    if (dbias) dbias[i] = sb;
}

unsigned row_groups(int64_t rows) { return (unsigned)(rows < 65536 ? rows : 65536); }

}  // namespace

hipError_t launch_layer_norm(const LayerNormArgs& a, int ek, hipStream_t st)
{
    return with_elem(ek, [&](auto e) {
        SW_NOTED_LAUNCH(note_kernel("layer_norm_kernel", ek), layer_norm_kernel<e()>, dim3(row_groups(a.rows)), dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

int layer_norm_backward_parts(int64_t rows, int64_t C) { return (int)(rows < 256 ? rows : 256); }

hipError_t launch_layer_norm_backward(const LayerNormBackwardArgs& a, int ek, hipStream_t st)
{
    return with_elem(ek, [&](auto e) {
        // (the sums over rows first: dx may be written over dy or x)
        if (a.dweight || a.dbias) {
            const int parts = layer_norm_backward_parts(a.rows, a.C);
            const unsigned columns = (unsigned)((a.C + kThreads - 1) / kThreads);
            SW_NOTED_LAUNCH(note_kernel("layer_norm_sums_kernel", ek), layer_norm_sums_kernel<e()>, dim3(columns, parts), dim3(kThreads), 0, st, a,
                            (a.rows + parts - 1) / parts);
            if (const hipError_t err = hipGetLastError()) return err;
            hipLaunchKernelGGL(layer_norm_fold_kernel, dim3(columns), dim3(kThreads), 0, st, a.partial, parts, a.C, a.dweight, a.dbias);
            if (const hipError_t err = hipGetLastError()) return err;
        }
        if (a.dx) {
            SW_NOTED_LAUNCH(note_kernel("layer_norm_dx_kernel", ek), layer_norm_dx_kernel<e()>, dim3(row_groups(a.rows)), dim3(kThreads), 0, st, a);
            return hipGetLastError();
        }
        return hipSuccess;
    });
}

}  // namespace swconv
