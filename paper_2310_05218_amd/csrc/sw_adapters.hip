// Low-rank adapters: a wavefront a product of a row with a row of `a`, then a thread an output.
#include "sw_sequence.h"

namespace swconv {

namespace {

// The adapter of a row; -1: none.  With packed rows the sequence is the last one that begins at or before the row, if the row is before its end.
__device__ __forceinline__ int adapter_of(const AdapterArgs& p, int64_t row)
{
    int64_t b;
    if (p.starts) {
        int lo = 0, hi = p.B + 1;       // how many of the B + 1 starts are at or before the row
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            if (p.starts[mid] <= row) lo = mid + 1;
            else hi = mid;
        }
        b = lo - 1;
        if (b < 0 || b >= p.B) return -1;
    } else {
        b = row / p.T;
    }
    const int s = p.slots ? p.slots[b] : (int)b;
    return s >= 0 && s < p.n ? s : -1;
}

// low[row, k] = a[s, k] . x[row]
template <int EK>
__global__ __launch_bounds__(256) void adapters_low_kernel(AdapterArgs p, int64_t rows)
{
    typedef typename ElemOf<EK>::type T;
    const int lane = threadIdx.x % 64;
    const int64_t tasks = rows * p.rank;
    for (int64_t task = blockIdx.x * 4 + threadIdx.x / 64; task < tasks; task += gridDim.x * 4) {
        const int64_t row = task / p.rank;
        const int s = adapter_of(p, row);
        if (s < 0) continue;
        const T *x = static_cast<const T*>(p.x) + row * p.x_stride, *a = static_cast<const T*>(p.a) + ((int64_t)s * p.rank + task % p.rank) * p.C_in;
        float sum = 0.f;
        for (int c = lane; c < p.C_in; c += 64) sum = __builtin_fmaf((float)x[c], (float)a[c], sum);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
        if (lane == 0) static_cast<float*>(p.work)[task] = sum;
    }
}

template <int EK>
__global__ __launch_bounds__(256) void adapters_out_kernel(AdapterArgs p, int64_t rows)
{
    typedef typename ElemOf<EK>::type T;
    const int64_t tasks = rows * p.C_out;
    for (int64_t task = (int64_t)blockIdx.x * 256 + threadIdx.x; task < tasks; task += (int64_t)gridDim.x * 256) {
        const int64_t row = task / p.C_out, c = task % p.C_out;
        const int s = adapter_of(p, row);
        float sum = (float)static_cast<const T*>(p.y)[row * p.y_stride + c];
        if (s >= 0) {
            const T* b = static_cast<const T*>(p.b) + ((int64_t)s * p.C_out + c) * p.rank;
            const float* low = static_cast<const float*>(p.work) + row * p.rank;
            float more = 0.f;
            for (int k = 0; k < p.rank; ++k) more = __builtin_fmaf(low[k], (float)b[k], more);
            sum = __builtin_fmaf(p.scales ? p.scales[s] : 1.f, more, sum);
        }
        static_cast<T*>(p.out)[row * p.out_stride + c] = (T)sum;
    }
}

int64_t rows_of(const AdapterArgs& a) { return a.starts ? a.T : a.T * a.B; }
unsigned most(int64_t want) { return (unsigned)(want < 4096 ? want : 4096); }

}  // namespace

int64_t adapters_workspace(const AdapterArgs& a, int) { return rows_of(a) * a.rank * 4; }

hipError_t launch_adapters(const AdapterArgs& a, int ek, hipStream_t st)
{
    const int64_t rows = rows_of(a);
    return with_elem(ek, [&](auto e) {
        hipLaunchKernelGGL(adapters_low_kernel<e()>, dim3(most((rows * a.rank + 3) / 4)), dim3(256), 0, st, a, rows);
        if (const hipError_t err = hipGetLastError()) return err;
        SW_NOTED_LAUNCH(note_kernel("adapters_out_kernel", ek), adapters_out_kernel<e()>, dim3(most((rows * a.C_out + 255) / 256)), dim3(256), 0, st, a, rows);
        return hipGetLastError();
    });
}

}  // namespace swconv
