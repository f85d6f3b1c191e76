// Sums over the rows of partial sums that workgroups have written, in a fixed order: 32 columns a workgroup, a row of them eight lanes with a 16-byte vector
// each, so that a thread has few rows, all on their way at once.  4 to 5 us, of which a launch and a trip to memory are 3.
#include "sw_sequence.h"

namespace swconv {

namespace {

constexpr int kThreads = 1024, kRows = kThreads / 8;
__global__ __launch_bounds__(kThreads) void fold_kernel(FoldArgs p)
{
    typedef Row<kElemF32> R;
    __shared__ R::floats lds[kThreads / 64][8];
    const int lane = threadIdx.x % 8, first = threadIdx.x / 8;
    const int i = blockIdx.x * 32 + lane * 4;
    R::floats s = 0.f;
    const auto of = blockIdx.y ? p.of[1] : p.of[0];
    if (!of.out) return;
    for (int k = first; k < of.parts; k += 8 * kRows) {
        R::floats v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = 0.f;
            if (k + j * kRows < of.parts && i < p.width) v[j] = R::load(of.partial + (int64_t)(k + j * kRows) * p.width, i, p.width);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[j];
    }
#pragma unroll
    for (int d = 8; d < 64; d <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += __shfl_xor(s[e], d, 64);
    if (threadIdx.x % 64 < 8) lds[threadIdx.x / 64][lane] = s;
    __syncthreads();
    if (threadIdx.x >= 8) return;
    for (int k = 1; k < kThreads / 64; ++k) s += lds[k][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i + e < p.width) of.out[i + e] = s[e];
}

}  // namespace

hipError_t launch_fold(const FoldArgs& a, hipStream_t st)
{
    hipLaunchKernelGGL(fold_kernel, dim3((a.width + 31) / 32, a.of[1].out ? 2 : 1), dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace swconv
