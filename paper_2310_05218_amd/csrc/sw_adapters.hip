// Low-rank adapters beside a shared projection: low = a x for every row, then out = y + scale b low.
//
// Long sequences go in tiles of 32 rows on the matrix cores, single tokens a row at a time.  Both factors and x are matrix operands as they lie: 16
// consecutive bytes of a row are a lane's.  A tile that several sequences meet in does the product for each of their adapters and keeps
// the rows that are its own, so that tiles need no list of sequences.
//
// `low` is a sum of fp32 products and enters a product itself.  Of 16-bit tensors it goes on as three 16-bit parts, v = v1 + v2 + v3, each the rest of the ones
// before rounded: 24 bits in bf16, and in half, of the row's largest value scaled to 2^13 ... 2^14, all bits above 2^-24 of that.  Three instructions in place of
// one; in fp32, on the fp32 ones, the product alone would take 21 us of the 27 that 6100 rows (rank 64, 2048 to 4096 channels, half) take to be moved.
#include "sw_sequence.h"

namespace swconv {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---- the rows' adapters ------------------------------------------------------------------------------------------------------------------------

// From `row` to `end` (at most `limit`) rows have adapter `s`; -1: none.  (Uniform: by whole wavefronts.)
struct Part {
    int64_t end;
    int s;
};
__device__ __forceinline__ Part part_from(const AdapterArgs& p, int64_t row, int64_t limit)
{
    int64_t b, end;
    if (p.starts) {
        int lo = 0, hi = p.B + 1;       // how many of the B + 1 starts are at or before the row; the next one, where there is one, is past it
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            if (uniform_load(p.starts + mid) <= row) lo = mid + 1;
            else hi = mid;
        }
        b = lo - 1;
        end = lo <= p.B ? uniform_load(p.starts + lo) : limit;
        if (b < 0 || b >= p.B) return Part{end < limit ? end : limit, -1};
    } else {
        b = row / p.T;
        end = (b + 1) * p.T;
    }
    const int s = p.slots ? uniform_load(p.slots + b) : (int)b;
    return Part{end < limit ? end : limit, s >= 0 && s < p.n ? s : -1};
}

// ---- tiles of rows ----------------------------------------------------------------------------------------------------------------------------

constexpr int kTileRows = 32;

template <int EK>
struct Matrix {
    typedef Row<EK> R;
    typedef typename R::T T;
    typedef typename R::vec vec;
    static constexpr int STEP = 4 * R::VEC;             // of the summed dimension that a lane's vector is a quarter of
    static constexpr int PARTS = EK == kElemF32 ? 1 : 3;
    static __device__ __forceinline__ f32x4 multiply(vec a, vec b, f32x4 c)
    {
        if constexpr (EK == kElemBF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
        else if constexpr (EK == kElemF16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
        else {
            // (element j of all lanes: any order of the summed dimension that both operands have)
#pragma unroll
            for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
            return c;
        }
    }
};

// The rank as the second product has it.
constexpr int padded_rank(int rank, int ek) { return ek == kElemF32 ? (rank + 15) / 16 * 16 : (rank + 31) / 32 * 32; }

// low of a tile's rows for up to 16 NT ranks, the input channels shared out to W wavefronts.  work: [rows][PARTS][padded rank], then a factor for each row.
template <int EK, int NT, int W>
__global__ __launch_bounds__(64 * W) void adapters_low_kernel(AdapterArgs p, int64_t rows, int K)
{
    typedef Matrix<EK> M;
    typedef typename M::R R;
    typedef typename M::T T;
    constexpr int PITCH = 16 * NT + 1;
    extern __shared__ float sums[];                     // [W][32][PITCH]
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 16, q = lane / 16;
    const int64_t first = (int64_t)blockIdx.x * kTileRows, last = first + kTileRows < rows ? first + kTileRows : rows;
    float* const factor = reinterpret_cast<float*>(static_cast<T*>(p.work) + rows * M::PARTS * K);
    const T* x[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int64_t row = first + 16 * t + m;
        x[t] = static_cast<const T*>(p.x) + (row < rows ? row : rows - 1) * p.x_stride;
    }
    for (int64_t row = first; row < last;) {
        const Part part = part_from(p, row, last);
        if (part.s >= 0) {
            const T* const a = static_cast<const T*>(p.a) + (int64_t)part.s * p.rank * p.C_in;
            const T* rank_row[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) rank_row[n] = a + (int64_t)(16 * n + m < p.rank ? 16 * n + m : p.rank - 1) * p.C_in;
            f32x4 acc[2][NT];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[t][n] = 0.f;
            for (int c = wave * M::STEP; c < p.C_in; c += W * M::STEP) {
                const int at = c + q * R::VEC;
                typename R::vec xv[2], av[NT];
                if (c + M::STEP <= p.C_in) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) xv[t] = R::load(x[t] + at);
#pragma unroll
                    for (int n = 0; n < NT; ++n) av[n] = R::load(rank_row[n] + at);
                } else {
#pragma unroll
                    for (int t = 0; t < 2; ++t) xv[t] = R::load(x[t], at, p.C_in);
#pragma unroll
                    for (int n = 0; n < NT; ++n) av[n] = R::load(rank_row[n], at, p.C_in);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < 2; ++t) acc[t][n] = M::multiply(xv[t], av[n], acc[t][n]);
            }
            __syncthreads();            // (the sums of the part before have been read)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sums[(wave * kTileRows + 16 * t + 4 * q + i) * PITCH + 16 * n + m] = acc[t][n][i];
            __syncthreads();
            // 16 lanes a row
            for (int r = threadIdx.x / 16; r < kTileRows; r += 4 * W) {
                const int64_t to = first + r;
                if (to < row || to >= part.end) continue;
                float v[NT], scale = 1.f;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    v[n] = 0.f;
#pragma unroll
                    for (int w = 0; w < W; ++w) v[n] += sums[(w * kTileRows + r) * PITCH + 16 * n + m];
                    if (16 * n + m >= p.rank) v[n] = 0.f;
                }
                if constexpr (EK == kElemF16) {
                    float most = 0.f;
#pragma unroll
                    for (int n = 0; n < NT; ++n) most = fmaxf(most, fabsf(v[n]));
#pragma unroll
                    for (int d = 1; d < 16; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, 16));
                    // 2^e with 2^13 <= most 2^-e < 2^14; rows of zeros, and of what is not finite, as they are
                    const int e = most > 0.f && most < 3.4e38f ? __builtin_amdgcn_frexp_expf(most) - 14 : 0;
                    scale = __builtin_amdgcn_ldexpf(1.f, e < -100 ? -100 : e);
                    const float back = __builtin_amdgcn_ldexpf(1.f, e < -100 ? 100 : -e);
#pragma unroll
                    for (int n = 0; n < NT; ++n) v[n] *= back;
                }
                T* const low = static_cast<T*>(p.work) + to * M::PARTS * K;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (16 * n + m >= K) continue;
                    float rest = v[n];
#pragma unroll
                    for (int k = 0; k < M::PARTS; ++k) {
                        const T one = (T)rest;
                        low[k * K + 16 * n + m] = one;
                        rest -= (float)one;
                    }
                }
                for (int n = 16 * NT + m; n < K; n += 16)
#pragma unroll
                    for (int k = 0; k < M::PARTS; ++k) low[k * K + n] = (T)0.f;
                if (m == 0) factor[to] = scale * (p.scales ? p.scales[part.s] : 1.f);
            }
        }
        row = part.end;
    }
}

// out of a tile's rows and a run of output channels, 64 of them a wavefront at a time.  Output channels are the matrix's rows, in an order that gives a lane 16
// consecutive ones of a row of y.
constexpr int kOutWaves = 4;
template <int EK>
__global__ __launch_bounds__(64 * kOutWaves) void adapters_out_kernel(AdapterArgs p, int64_t rows, int K, int chunks, int chunk)
{
    typedef Matrix<EK> M;
    typedef typename M::R R;
    typedef typename M::T T;
    constexpr int VEC = R::VEC, PARTS = M::PARTS;
    extern __shared__ float shared[];
    T* const low = reinterpret_cast<T*>(shared);        // [PARTS][32][K + VEC]
    const int pitch = K + VEC;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), m = lane % 16, q = lane / 16;
    // (workgroups that follow each other have different chunks: with eight of them the workgroups of a die have one, and its caches that part of b)
    const int64_t first = blockIdx.x / chunks * (int64_t)kTileRows, last = first + kTileRows < rows ? first + kTileRows : rows;
    const int from = (int)(blockIdx.x % chunks) * chunk, to = from + chunk < p.C_out ? from + chunk : p.C_out;
    const float* const factor = reinterpret_cast<const float*>(static_cast<const T*>(p.work) + rows * PARTS * K);
    for (int k = threadIdx.x; k < kTileRows * PARTS * (K / VEC); k += 64 * kOutWaves) {
        const int r = k / (PARTS * (K / VEC)), rest = k % (PARTS * (K / VEC)), part = rest / (K / VEC), c = rest % (K / VEC) * VEC;
        const int64_t row = first + r < rows ? first + r : rows - 1;
        *reinterpret_cast<typename R::vec*>(low + (part * kTileRows + r) * pitch + c) =
            *reinterpret_cast<const typename R::vec*>(static_cast<const T*>(p.work) + (row * PARTS + part) * K + c);
    }
    __syncthreads();
    for (int64_t row = first; row < last;) {
        const Part part = part_from(p, row, last);
        if (part.s >= 0) {
            const T* const b = static_cast<const T*>(p.b) + (int64_t)part.s * p.C_out * p.rank;
            bool mine[2];
            float f[2];
            const T* y[2];
            T* out[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int64_t at = first + 16 * t + m;
                mine[t] = at >= row && at < part.end;
                const int64_t safe = mine[t] ? at : row;
                f[t] = factor[safe];
                y[t] = static_cast<const T*>(p.y) + safe * p.y_stride;
                out[t] = static_cast<T*>(p.out) + safe * p.out_stride;
            }
            for (int c0 = from + 64 * wave; c0 < to; c0 += 64 * kOutWaves) {
                const int at = c0 + 16 * q;             // the lane's 16 channels of y
                typename R::vec yv[2][16 / VEC];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int k = 0; k < 16 / VEC; ++k) yv[t][k] = R::load(y[t], at + k * VEC, to);
                const T* rows_of_b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = c0 + (m / 4) * 16 + j * 4 + m % 4;
                    rows_of_b[j] = b + (int64_t)(c < to ? c : to - 1) * p.rank;
                }
                f32x4 acc[4][2];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int t = 0; t < 2; ++t) acc[j][t] = 0.f;
                for (int k = 0; k < K; k += M::STEP) {
                    typename R::vec bv[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) bv[j] = k + M::STEP <= p.rank ? R::load(rows_of_b[j] + k + q * VEC) : R::load(rows_of_b[j], k + q * VEC, p.rank);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int n = 0; n < PARTS; ++n) {
                            const typename R::vec v = *reinterpret_cast<const typename R::vec*>(low + (n * kTileRows + 16 * t + m) * pitch + k + q * VEC);
#pragma unroll
                            for (int j = 0; j < 4; ++j) acc[j][t] = M::multiply(bv[j], v, acc[j][t]);
                        }
                }
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (mine[t])
#pragma unroll
                        for (int k = 0; k < 16 / VEC; ++k) {
                            typename R::floats v = __builtin_convertvector(yv[t][k], typename R::floats);
#pragma unroll
                            for (int e = 0; e < VEC; ++e) v[e] = __builtin_fmaf(f[t], acc[(k * VEC + e) / 4][t][e % 4], v[e]);
                            R::store(out[t], at + k * VEC, to, v);
                        }
            }
        } else if (p.out != p.y) {
            for (int64_t r = row + wave; r < part.end; r += kOutWaves)
                for (int c = from + lane * VEC; c < to; c += 64 * VEC)
                    R::store(static_cast<T*>(p.out) + r * p.out_stride, c, to,
                             __builtin_convertvector(R::load(static_cast<const T*>(p.y) + r * p.y_stride, c, to), typename R::floats));
        }
        row = part.end;
    }
}

// ---- single rows ------------------------------------------------------------------------------------------------------------------------------

// N ranks from `k` on of a row, by a wavefront
template <int EK, int N>
__device__ __forceinline__ void dots(const AdapterArgs& p, int64_t row, int s, int k, float (&sum)[N])
{
    typedef Row<EK> R;
    typedef typename R::T T;
    const T *x = static_cast<const T*>(p.x) + row * p.x_stride, *a[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        a[j] = static_cast<const T*>(p.a) + ((int64_t)s * p.rank + (k + j < p.rank ? k + j : p.rank - 1)) * p.C_in;
        sum[j] = 0.f;
    }
#pragma unroll 4
    for (int c = threadIdx.x % 64 * R::VEC; c < p.C_in; c += 64 * R::VEC) {
        const auto xv = __builtin_convertvector(R::load(x, c, p.C_in), typename R::floats);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const auto av = __builtin_convertvector(R::load(a[j], c, p.C_in), typename R::floats);
#pragma unroll
            for (int e = 0; e < R::VEC; ++e) sum[j] = __builtin_fmaf(xv[e], av[e], sum[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] = lanes_sum<64>(sum[j]);
}

constexpr int kRowRanks = 4, kRowThreads = 256;

template <int EK>
__global__ __launch_bounds__(kRowThreads) void adapters_row_low_kernel(AdapterArgs p, int64_t rows, int each)
{
    const int64_t task = (int64_t)blockIdx.x * (kRowThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = task / each;
    const int k = (int)(task % each) * kRowRanks;
    if (row >= rows) return;
    const int s = part_from(p, row, row + 1).s;
    if (s < 0) return;
    float sum[kRowRanks];
    dots<EK, kRowRanks>(p, row, s, k, sum);
    if (threadIdx.x % 64 == 0)
#pragma unroll
        for (int j = 0; j < kRowRanks; ++j)
            if (k + j < p.rank) static_cast<float*>(p.work)[row * p.rank + k + j] = sum[j];
}

// out of a run of a row's channels, a channel a thread; WHOLE: low is computed on the way, by every workgroup of the row.
template <int EK, bool WHOLE>
__global__ __launch_bounds__(kRowThreads) void adapters_row_out_kernel(AdapterArgs p, int chunks, int chunk)
{
    typedef Row<EK> R;
    typedef typename R::T T;
    __shared__ float low[256];
    const int64_t row = blockIdx.x / chunks;
    const int from = (int)(blockIdx.x % chunks) * chunk, to = from + chunk < p.C_out ? from + chunk : p.C_out;
    const int s = part_from(p, row, row + 1).s;
    const T* const y = static_cast<const T*>(p.y) + row * p.y_stride;
    T* const out = static_cast<T*>(p.out) + row * p.out_stride;
    if (s < 0) {
        if (p.out != p.y)
            for (int c = from + threadIdx.x; c < to; c += kRowThreads) out[c] = y[c];
        return;
    }
    if constexpr (WHOLE) {
        for (int k = threadIdx.x / 64 * kRowRanks; k < p.rank; k += kRowThreads / 64 * kRowRanks) {
            float sum[kRowRanks];
            dots<EK, kRowRanks>(p, row, s, k, sum);
            if (threadIdx.x % 64 == 0)
#pragma unroll
                for (int j = 0; j < kRowRanks; ++j)
                    if (k + j < p.rank) low[k + j] = sum[j];
        }
    } else {
        if ((int)threadIdx.x < p.rank) low[threadIdx.x] = static_cast<const float*>(p.work)[row * p.rank + threadIdx.x];
    }
    __syncthreads();
    const float scale = p.scales ? p.scales[s] : 1.f;
    for (int c = from + threadIdx.x; c < to; c += kRowThreads) {
        const T* const b = static_cast<const T*>(p.b) + ((int64_t)s * p.C_out + c) * p.rank;
        const float yc = (float)y[c];
        float sum = 0.f;
        for (int k = 0; k < p.rank; k += R::VEC) {
            const auto bv = __builtin_convertvector(R::load(b, k, p.rank), typename R::floats);
#pragma unroll
            for (int e = 0; e < R::VEC; ++e) sum = __builtin_fmaf(k + e < p.rank ? low[k + e] : 0.f, bv[e], sum);
        }
        out[c] = (T)__builtin_fmaf(scale, sum, yc);
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------------------------------------

int64_t rows_of(const AdapterArgs& a) { return a.starts ? a.T : a.T * a.B; }

// Tiles where a sequence has eight rows on average: a tile that many short ones meet in does its product once for each.
bool in_tiles(const AdapterArgs& a) { return rows_of(a) >= 8 * (int64_t)a.B; }

// Single rows in one launch where a factor `a` is small enough for every workgroup of a row to read it.
constexpr int64_t kWholeBytes = 128 << 10;
bool whole_rows(const AdapterArgs& a, int ek) { return (int64_t)a.rank * a.C_in * elem_size(ek) <= kWholeBytes; }

template <int EK, int NT, int W>
hipError_t launch_low(const AdapterArgs& a, int64_t rows, int K, hipStream_t st)
{
    const size_t lds = sizeof(float) * W * kTileRows * (16 * NT + 1);
    static const hipError_t allowed = hipFuncSetAttribute(reinterpret_cast<const void*>(adapters_low_kernel<EK, NT, W>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (allowed != hipSuccess) return allowed;
    hipLaunchKernelGGL((adapters_low_kernel<EK, NT, W>), dim3((unsigned)((rows + kTileRows - 1) / kTileRows)), dim3(64 * W), lds, st, a, rows, K);
    return hipGetLastError();
}

template <int EK>
hipError_t launch_tiles(const AdapterArgs& a, hipStream_t st)
{
    const int64_t rows = rows_of(a);
    const int K = padded_rank(a.rank, EK);
    hipError_t err;
    if (a.rank <= 16) err = launch_low<EK, 1, 8>(a, rows, K, st);
    else if (a.rank <= 32) err = launch_low<EK, 2, 8>(a, rows, K, st);
    else if (a.rank <= 64) err = launch_low<EK, 4, 8>(a, rows, K, st);
    else if (a.rank <= 128) err = launch_low<EK, 8, 8>(a, rows, K, st);
    else err = launch_low<EK, 16, 4>(a, rows, K, st);
    if (err != hipSuccess) return err;
    const int blocks = (a.C_out + 63) / 64, most = blocks < 8 ? blocks : 8, chunk = (blocks + most - 1) / most * 64, chunks = (a.C_out + chunk - 1) / chunk;
    const size_t lds = (size_t)kTileRows * Matrix<EK>::PARTS * (K + Row<EK>::VEC) * elem_size(EK);
    const int64_t groups = (rows + kTileRows - 1) / kTileRows * chunks;
    SW_NOTED_LAUNCH(note_kernel("adapters_out_kernel", EK, a.rank), adapters_out_kernel<EK>, dim3((unsigned)groups), dim3(64 * kOutWaves), lds, st, a, rows, K, chunks, chunk);
    return hipGetLastError();
}

template <int EK>
hipError_t launch_rows(const AdapterArgs& a, hipStream_t st)
{
    const int64_t rows = rows_of(a);
    const bool whole = whole_rows(a, EK);
    if (!whole) {
        const int each = (a.rank + kRowRanks - 1) / kRowRanks;
        hipLaunchKernelGGL(adapters_row_low_kernel<EK>, dim3((unsigned)((rows * each + kRowThreads / 64 - 1) / (kRowThreads / 64))), dim3(kRowThreads), 0, st, a, rows, each);
        if (const hipError_t err = hipGetLastError()) return err;
    }
    // workgroups for every CU, several a row where rows are few
    constexpr int kGroups = 512;
    const int64_t want = (kGroups + rows - 1) / rows, most = (a.C_out + kRowThreads - 1) / kRowThreads;
    const int per = (int)((most + (want < most ? want : most) - 1) / (want < most ? want : most)), chunk = per * kRowThreads, chunks = (a.C_out + chunk - 1) / chunk;
    const dim3 grid((unsigned)(rows * chunks)), block(kRowThreads);
    note_kernel("adapters_row_out_kernel", EK, whole);
    if (whole)
        hipLaunchKernelGGL((adapters_row_out_kernel<EK, true>), grid, block, 0, st, a, chunks, chunk);
    else
        hipLaunchKernelGGL((adapters_row_out_kernel<EK, false>), grid, block, 0, st, a, chunks, chunk);
    return hipGetLastError();
}

constexpr int64_t kThreadsMost = ((int64_t)1 << 32) - 1;

}  // namespace

bool adapters_fit(const AdapterArgs& a)
{
    const int64_t rows = rows_of(a);
    if (in_tiles(a)) return (rows + kTileRows - 1) / kTileRows <= kThreadsMost / (8 * 64 * kOutWaves);
    return rows <= kThreadsMost / kRowThreads / 2 && rows <= kThreadsMost / (64 * ((a.rank + kRowRanks - 1) / kRowRanks)) - kRowThreads;
}

int64_t adapters_workspace(const AdapterArgs& a, int ek)
{
    const int64_t rows = rows_of(a);
    if (in_tiles(a)) return rows * (padded_rank(a.rank, ek) * (ek == kElemF32 ? 4 : 6) + 4);
    return whole_rows(a, ek) ? 0 : rows * a.rank * 4;
}

hipError_t launch_adapters(const AdapterArgs& a, int ek, hipStream_t st)
{
    return with_elem(ek, [&](auto e) { return in_tiles(a) ? launch_tiles<e()>(a, st) : launch_rows<e()>(a, st); });
}

}  // namespace swconv
