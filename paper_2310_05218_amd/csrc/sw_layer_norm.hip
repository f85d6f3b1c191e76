// Layer norm over the channels of channel-last rows, and its backward pass.
//
// Both are bound by memory: a row is read once into registers, folded there, and written once.  A row of V 16-byte vectors has the
// fewest lanes that hold it in a few vectors each: 8, 16 or 32 lanes (several rows a wavefront), a wavefront, 256 to 1024 threads.
// Workgroups walk over rows a grid apart: a thread's columns never change, so weight and bias stay in its registers (they are 4 bytes an
// element, twice a 16-bit row), and the next row is on its way while this one is folded.  Rows of more than 2048 vectors are read again from
// memory instead.  16384 rows of 4096 bf16: 52 us forwards (5.2 TB/s), 80 backwards (5.0).
//
// Loads are 16 bytes at any element's address.  The lane at the end of a row that is no whole number of vectors has the row's last vector, whose
// first elements are another's too: it leaves them out of its sums and stores what the other stores.  (With single elements in their place the
// compiler waits for a row's every load before the next one: the backward pass of 3001 rows of 1999 bf16 took 31 us for 17.)
#include <initializer_list>

#include "sw_layers.h"

namespace swconv {

namespace {

// ---- sums over lanes ----------------------------------------------------------------------------------------------------------

// The sums over all LANES threads of a row, in every one of them.  `lds` holds a value for each wavefront and sum, and is written again
// two calls later: one barrier a call, as a thread that is a call ahead of another has passed the barrier that the other's reads precede.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*lds)[LANES / 64 + 1], int& turn)
{
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum<LANES < 64 ? LANES : 64>(v[k]);
    if constexpr (LANES > 64) {
        float(*at)[LANES / 64 + 1] = lds + turn * N;
        turn ^= 1;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) at[k][threadIdx.x / 64] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.f;
#pragma unroll
            for (int i = 0; i < LANES / 64; ++i) v[k] += at[k][i];
        }
    }
}

constexpr int threads_of(int lanes) { return lanes < 256 ? 256 : lanes; }

// ---- forward -----------------------------------------------------------------------------------------------------------------------

// How a row ends.
enum Tail {
    kWhole,         // C is LANES * NV vectors
    kLast,          // the last lanes share elements; the first NV / 2 vectors of a lane are within the row whatever C is (with_lanes)
    kBrief          // C is less than a vector
};

// A lane's vectors of a row of C elements.
template <int EK, int LANES, int NV, Tail TAIL>
struct Columns {
    typedef Row<EK> R;
    typedef typename R::T T;
    typedef typename R::floats floats;
    int lane, C;
    static constexpr bool within(int i) { return TAIL == kWhole || (TAIL == kLast && i < NV / 2); }
    __device__ __forceinline__ int at(int i) const { return (lane + i * LANES) * R::VEC; }
    // where a lane's vector i begins, and whether it is one of the row's
    __device__ __forceinline__ int start(int i) const { return within(i) || at(i) < C - R::VEC ? at(i) : C - R::VEC; }
    __device__ __forceinline__ bool mine(int i) const { return within(i) || at(i) < C; }
    __device__ __forceinline__ typename R::vec load(const T* row, int i) const
    {
        if constexpr (TAIL == kBrief)
            return R::load(row, at(i), C);
        else
            return R::load(row + start(i));
    }
    __device__ __forceinline__ void store(T* row, int i, floats f) const
    {
        if constexpr (TAIL == kBrief)
            R::store(row, at(i), C, f);
        else if (mine(i))
            R::store(row + start(i), f);
    }
    __device__ __forceinline__ floats load_floats(const float* p, int i, float without) const
    {
        if constexpr (TAIL == kBrief) return R::load_floats(p, at(i), C, without);
        floats f = without;
        return p ? R::load_floats(p + start(i)) : f;
    }
    __device__ __forceinline__ void store_floats(float* p, int i, floats f) const
    {
        if constexpr (TAIL == kBrief)
            R::store_floats(p, at(i), C, f);
        else if (mine(i))
            R::store_floats(p + start(i), f);
    }
    // the sum of those elements that are the lane's alone
    __device__ __forceinline__ float sum(floats f, int i) const
    {
        if constexpr (TAIL == kBrief)
            f = R::within(f, at(i), C);
        else if (!within(i))
#pragma unroll
            for (int e = 0; e < R::VEC; ++e) f[e] = start(i) + e >= at(i) ? f[e] : 0.f;
        return R::sum(f);
    }
};

template <int EK, int LANES, int NV, Tail TAIL>
__global__ __launch_bounds__(threads_of(LANES)) void layer_norm_kernel(LayerNormArgs p)
{
    typedef Row<EK> R;
    typedef typename R::T T;
    typedef typename R::floats floats;
    constexpr int kRows = threads_of(LANES) / LANES;        // rows that a workgroup has at a time
    __shared__ float lds[2][LANES / 64 + 1];
    int turn = 0;
    const int C = TAIL != kWhole ? p.C : LANES * NV * R::VEC;
    const Columns<EK, LANES, NV, TAIL> columns{(int)threadIdx.x % LANES, C};
    const float inv = 1.0f / (float)C;
    floats w[NV], b[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) w[i] = columns.load_floats(p.weight, i, 1.f), b[i] = columns.load_floats(p.bias, i, 0.f);
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    const int64_t step = (int64_t)gridDim.x * kRows;
    typename R::vec raw[NV];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i] = columns.load(static_cast<const T*>(p.x) + (r < p.rows ? r : p.rows - 1) * p.x_stride, i);
    };
    fetch(row);
    // (the rows of a workgroup end together: whole wavefronts and, where a row has several, all of them pass every barrier)
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < p.rows; first += step, row += step) {
        floats x[NV];
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            x[i] = __builtin_convertvector(raw[i], floats);
            s[0] += columns.sum(x[i], i);
        }
        fetch(row + step);
        row_sums<LANES>(s, lds, turn);
        const float mean = s[0] * inv;
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            x[i] -= mean;
            s[0] += columns.sum(x[i] * x[i], i);
        }
        row_sums<LANES>(s, lds, turn);
        const float rstd = 1.0f / sqrtf(s[0] * inv + p.eps);
        if (row < p.rows) {
#pragma unroll
            for (int i = 0; i < NV; ++i) columns.store(static_cast<T*>(p.y) + row * p.y_stride, i, x[i] * rstd * w[i] + b[i]);
            if (columns.lane == 0) {
                if (p.mean) p.mean[row] = mean;
                if (p.rstd) p.rstd[row] = rstd;
            }
        }
    }
}

// Rows beyond what registers hold: a workgroup a row, which is read three times (the second and third from the caches).
template <int EK>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(LayerNormArgs p)
{
    typedef Row<EK> R;
    typedef typename R::T T;
    __shared__ float lds[2][17];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
        float s[1] = {0.f};
        for (int i = threadIdx.x * R::VEC; i < p.C; i += 1024 * R::VEC) s[0] += R::sum(__builtin_convertvector(R::load(x, i, p.C), typename R::floats));
        row_sums<1024>(s, lds, turn);
        const float mean = s[0] / (float)p.C;
        s[0] = 0.f;
        for (int i = threadIdx.x * R::VEC; i < p.C; i += 1024 * R::VEC) {
            const auto d = R::within(__builtin_convertvector(R::load(x, i, p.C), typename R::floats) - mean, i, p.C);
            s[0] += R::sum(d * d);
        }
        row_sums<1024>(s, lds, turn);
        const float rstd = 1.0f / sqrtf(s[0] / (float)p.C + p.eps);
        for (int i = threadIdx.x * R::VEC; i < p.C; i += 1024 * R::VEC)
            R::store(static_cast<T*>(p.y) + row * p.y_stride, i, p.C,
                     (__builtin_convertvector(R::load(x, i, p.C), typename R::floats) - mean) * rstd * R::load_floats(p.weight, i, p.C, 1.f) +
                         R::load_floats(p.bias, i, p.C, 0.f));
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

// ---- backward ----------------------------------------------------------------------------------------------------------------------

// A thread adds dy * h and dy of its columns over its rows in registers; the rows of a workgroup meet in LDS, and a workgroup writes its
// sums as one row {dweight[C], dbias[C]} of `partial`.
template <int EK, int LANES, int NV, Tail TAIL>
__global__ __launch_bounds__(threads_of(LANES)) void layer_norm_backward_kernel(LayerNormBackwardArgs p)
{
    typedef Row<EK> R;
    typedef typename R::T T;
    constexpr int kRows = threads_of(LANES) / LANES;
    __shared__ float lds[4][LANES / 64 + 1];
    int turn = 0;
    const int lane = threadIdx.x % LANES;
    const int C = TAIL != kWhole ? p.C : LANES * NV * R::VEC;
    const Columns<EK, LANES, NV, TAIL> columns{lane, C};
    const float inv = 1.0f / (float)C;
    typename R::floats w[NV], sw[NV], sb[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        w[i] = columns.load_floats(p.weight, i, 1.f);
        sw[i] = 0.f, sb[i] = 0.f;
    }
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    const int64_t step = (int64_t)gridDim.x * kRows;
    typename R::vec raw_x[NV], raw_dy[NV];
    float next_mean, next_rstd;
    auto fetch = [&](int64_t r) {
        r = r < p.rows ? r : p.rows - 1;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw_x[i] = columns.load(static_cast<const T*>(p.x) + r * p.x_stride, i);
            raw_dy[i] = columns.load(static_cast<const T*>(p.dy) + r * p.dy_stride, i);
        }
        next_mean = p.mean[r], next_rstd = p.rstd[r];
    };
    fetch(row);
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < p.rows; first += step, row += step) {
        const float mean = next_mean, rstd = next_rstd;
        const bool mine = row < p.rows;
        typename R::floats h[NV], g[NV];
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            h[i] = (__builtin_convertvector(raw_x[i], typename R::floats) - mean) * rstd;
            g[i] = __builtin_convertvector(raw_dy[i], typename R::floats);
            if (mine) {
                sw[i] += g[i] * h[i];
                sb[i] += g[i];
            }
            g[i] *= w[i];
            s[0] += columns.sum(g[i], i);
            s[1] += columns.sum(g[i] * h[i], i);
        }
        fetch(row + step);
        row_sums<LANES>(s, lds, turn);
        if (mine && p.dx)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                columns.store(static_cast<T*>(p.dx) + row * p.dx_stride, i, rstd * (g[i] - s[0] * inv - h[i] * (s[1] * inv)));
    }
    if (!p.partial) return;
    float* out = p.partial + (int64_t)blockIdx.x * 2 * C;
    if constexpr (kRows > 1) {
        // (at most 64 lanes a row: their columns' sums of all rows of the workgroup fit 16 KB)
        __shared__ typename R::floats meet[2][kRows][LANES];
        static_assert(NV == 1 || kRows * LANES * NV * sizeof(meet[0][0][0]) <= 32768, "LDS");
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            __syncthreads();
            meet[0][threadIdx.x / LANES][lane] = sw[i];
            meet[1][threadIdx.x / LANES][lane] = sb[i];
            __syncthreads();
            if (threadIdx.x < 2 * LANES) {
                const int which = threadIdx.x / LANES;
                typename R::floats s = meet[which][0][lane];
                for (int r = 1; r < kRows; ++r) s += meet[which][r][lane];
                columns.store_floats(out + which * C, i, s);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            columns.store_floats(out, i, sw[i]);
            columns.store_floats(out + C, i, sb[i]);
        }
    }
}

// Rows beyond what registers hold: the sums of a run of rows a column per thread, then dx a workgroup a row (dx may be written over dy or x).
template <int EK>
__global__ __launch_bounds__(256) void layer_norm_long_sums_kernel(LayerNormBackwardArgs p, int64_t run)
{
    typedef typename ElemOf<EK>::type T;
    const int i = blockIdx.x * 256 + threadIdx.x;
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

template <int EK>
__global__ __launch_bounds__(1024) void layer_norm_long_dx_kernel(LayerNormBackwardArgs p)
{
    typedef Row<EK> R;
    typedef typename R::T T;
    __shared__ float lds[4][17];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
        const T* dy = static_cast<const T*>(p.dy) + row * p.dy_stride;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float s[2] = {0.f, 0.f};
        auto terms = [&](int i, typename R::floats& g, typename R::floats& h) {
            g = __builtin_convertvector(R::load(dy, i, p.C), typename R::floats) * R::load_floats(p.weight, i, p.C, 1.f);
            h = R::within((__builtin_convertvector(R::load(x, i, p.C), typename R::floats) - mean) * rstd, i, p.C);
        };
        typename R::floats g, h;
        for (int i = threadIdx.x * R::VEC; i < p.C; i += 1024 * R::VEC) {
            terms(i, g, h);
            s[0] += R::sum(g);
            s[1] += R::sum(g * h);
        }
        row_sums<1024>(s, lds, turn);
        for (int i = threadIdx.x * R::VEC; i < p.C; i += 1024 * R::VEC) {
            terms(i, g, h);
            R::store(static_cast<T*>(p.dx) + row * p.dx_stride, i, p.C, rstd * (g - s[0] / (float)p.C - h * (s[1] / (float)p.C)));
        }
    }
}

// The sums over the rows of `partial` ([parts, 2 C]), in a fixed order: 32 columns a workgroup, a row of eight 16-byte vectors eight lanes, so
// that a thread has few rows, all on their way at once (1024 rows of 2 x 4096: 20 us with a wavefront's 64 columns, one row after another).
constexpr int kFoldThreads = 1024, kFoldRows = kFoldThreads / 8;
__global__ __launch_bounds__(kFoldThreads) void layer_norm_fold_kernel(const float* partial, int parts, int C, float* dweight, float* dbias)
{
    typedef Row<kElemF32> R;
    __shared__ R::floats lds[kFoldThreads / 64][8];
    const int lane = threadIdx.x % 8, first = threadIdx.x / 8;
    const int i = blockIdx.x * 32 + lane * 4;
    R::floats s = 0.f;
    for (int k = first; k < parts; k += 8 * kFoldRows) {
        R::floats v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = 0.f;
            if (k + j * kFoldRows < parts && i < 2 * C) v[j] = R::load(partial + (int64_t)(k + j * kFoldRows) * 2 * C, i, 2 * C);
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
    for (int k = 1; k < kFoldThreads / 64; ++k) s += lds[k][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float* out = i + e < C ? dweight : dbias;
        if (i + e < 2 * C && out) out[i + e < C ? i + e : i + e - C] = s[e];
    }
}

// ---- which lanes ---------------------------------------------------------------------------------------------------------------------

// f(lanes, vectors a lane) for rows of C elements: integral constants, 0 lanes where registers do not hold a row.
template <int EK, bool BACKWARD, class F>
hipError_t with_lanes(int64_t C, F&& f)
{
    const int64_t v = (C + Row<EK>::VEC - 1) / Row<EK>::VEC;
#define SW_LANES(l, n) \
    if (v <= (l) * (n)) return f(std::integral_constant<int, l>(), std::integral_constant<int, n>())
    SW_LANES(8, 1);
    SW_LANES(16, 1);
    SW_LANES(32, 1);
    SW_LANES(64, 1);
    SW_LANES(64, 2);
    SW_LANES(256, 1);
    SW_LANES(256, 2);
    SW_LANES(512, 2);
    if constexpr (BACKWARD) {
        SW_LANES(512, 4);
    } else {
        SW_LANES(1024, 2);
    }
#undef SW_LANES
    return f(std::integral_constant<int, 0>(), std::integral_constant<int, 0>());
}

// f(how the row ends): an integral constant.
template <int EK, int LANES, int NV, class F>
void with_tail(int64_t C, F&& f)
{
    if (C == LANES * NV * Row<EK>::VEC) return f(std::integral_constant<Tail, kWhole>());
    if constexpr (LANES == 8)
        if (C < Row<EK>::VEC) return f(std::integral_constant<Tail, kBrief>());
    f(std::integral_constant<Tail, kLast>());
}

constexpr int kCUs = 256;

// Workgroups of a launch: `threads` for every CU, or the rows there are.
unsigned row_groups(int64_t rows, int lanes, int threads)
{
    const int64_t want = (rows * lanes + threads_of(lanes) - 1) / threads_of(lanes), most = kCUs * (threads / threads_of(lanes));
    return (unsigned)(want < most ? want : most);
}

constexpr int kForwardThreads = 2048;
// Backward, where every workgroup adds a row of 2 C sums to fold: rows of a workgroup two on a CU (16384 x 4096 bf16 with four: 81 -> 76 us, the
// fold 7.6 -> 5), rows of a wavefront or less, whose wavefronts wait for nothing but memory, four (70000 x 200 bf16 with two: 19 -> 29).
constexpr int kBackwardMost = 1024;
constexpr int backward_threads(int lanes) { return lanes > 64 ? 512 : kBackwardMost; }
constexpr int kLongParts = 64;

// Rows of sums that a backward launch writes.
unsigned backward_parts(int64_t rows, int lanes)
{
    if (lanes == 0) return (unsigned)(rows < kLongParts ? rows : kLongParts);
    return row_groups(rows, lanes, backward_threads(lanes));
}

}  // namespace

hipError_t launch_layer_norm(const LayerNormArgs& a, int ek, hipStream_t st)
{
    return with_elem(ek, [&](auto e) {
        return with_lanes<e(), false>(a.C, [&](auto lanes, auto nv) {
            if constexpr (lanes() == 0) {
                SW_NOTED_LAUNCH(note_kernel("layer_norm_long_kernel", ek), layer_norm_long_kernel<e()>, dim3(row_groups(a.rows, 1024, kForwardThreads)), dim3(1024), 0, st, a);
            } else {
                const dim3 grid(row_groups(a.rows, lanes(), kForwardThreads)), block(threads_of(lanes()));
                note_kernel("layer_norm_kernel", ek, lanes(), nv());
                with_tail<e(), lanes(), nv()>(a.C, [&](auto tail) { hipLaunchKernelGGL((layer_norm_kernel<e(), lanes(), nv(), tail()>), grid, block, 0, st, a); });
            }
            return hipGetLastError();
        });
    });
}

int layer_norm_backward_parts(int64_t rows, int64_t C)
{
    unsigned most = 0;          // of any format
    for (const int ek : {kElemF32, kElemBF16, kElemF16})
        (void)with_elem(ek, [&](auto e) {
            return with_lanes<e(), true>(C, [&](auto lanes, auto) {
                const unsigned parts = backward_parts(rows, lanes());
                if (parts > most) most = parts;
                return hipSuccess;
            });
        });
    return (int)most;
}

hipError_t launch_layer_norm_backward(const LayerNormBackwardArgs& args, int ek, hipStream_t st)
{
    LayerNormBackwardArgs a = args;
    if (!a.dweight && !a.dbias) a.partial = nullptr;
    return with_elem(ek, [&](auto e) {
        return with_lanes<e(), true>(a.C, [&](auto lanes, auto nv) {
            const unsigned parts = backward_parts(a.rows, lanes());
            if constexpr (lanes() == 0) {
                note_kernel("layer_norm_long_dx_kernel", ek);
                if (a.partial) {
                    hipLaunchKernelGGL(layer_norm_long_sums_kernel<e()>, dim3((a.C + 255) / 256, parts), dim3(256), 0, st, a, (a.rows + parts - 1) / parts);
                    if (const hipError_t err = hipGetLastError()) return err;
                }
                if (a.dx) hipLaunchKernelGGL(layer_norm_long_dx_kernel<e()>, dim3(row_groups(a.rows, 1024, kForwardThreads)), dim3(1024), 0, st, a);
            } else {
                const dim3 block(threads_of(lanes()));
                note_kernel("layer_norm_backward_kernel", ek, lanes(), nv());
                with_tail<e(), lanes(), nv()>(
                    a.C, [&](auto tail) { hipLaunchKernelGGL((layer_norm_backward_kernel<e(), lanes(), nv(), tail()>), dim3(parts), block, 0, st, a); });
            }
            if (const hipError_t err = hipGetLastError()) return err;
            if (a.partial)
                hipLaunchKernelGGL(layer_norm_fold_kernel, dim3((2 * a.C + 31) / 32), dim3(kFoldThreads), 0, st, a.partial, (int)parts, a.C, a.dweight, a.dbias);
            return hipGetLastError();
        });
    });
}

}  // namespace swconv
