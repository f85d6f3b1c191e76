// Linear attention with a decay for each head, token by token: the recurrence as it stands, for prompts, gradients and single tokens.
#include "sw_attention.h"

namespace swconv {

namespace {

constexpr int kColumns = 64, kGroups = 4;       // a workgroup has 64 columns of the state, a quarter of its rows a wavefront

template <int EK, int ROWS>
__global__ __launch_bounds__(kColumns * kGroups) void attention_recurrent_kernel(AttentionSum s, AttentionBatch n)
{
    typedef typename ElemOf<EK>::type T;
    __shared__ float la[2][ROWS * kGroups], lb[2][ROWS * kGroups], sums[2][kGroups][kColumns];
    const int lane = threadIdx.x % 64, group = threadIdx.x / 64;
    const int head = blockIdx.y, col = blockIdx.z * kColumns + lane;
    int64_t lo = 0, hi = n.T;
    int seq = blockIdx.x;
    int64_t batch = seq;
    bool rest = false;
    if (n.starts) {
        lo = attention::packed_first(n, blockIdx.x);
        hi = attention::packed_end(n, blockIdx.x, lo);
        rest = blockIdx.x == 0 || (int)blockIdx.x == n.B + 1;
        seq = (int)blockIdx.x - 1;
        batch = 0;
    }
    auto at = [&](const AttentionOperand& o, int64_t t) { return batch * o.batch + t * o.token + head / o.share * o.head; };
    auto put = [&](int64_t t, float v) {
        if (s.y_f32)
            const_cast<float*>(static_cast<const float*>(s.y.p))[at(s.y, t) + col] = v;
        else
            const_cast<T*>(static_cast<const T*>(s.y.p))[at(s.y, t) + col] = (T)v;
    };
    if (rest) {
        for (int64_t t = lo + group; t < hi; t += kGroups)
            if (col < s.DC) put(t, 0.f);
        return;
    }
    const int entry = s.first_slots ? s.first_slots[seq] : seq;
    const bool kept = !s.first_slots || (entry >= 0 && entry < n.n_states);
    const float decay = expf(n.log_decay[head]);
    const int own = s.DA - group * ROWS;            // rows of the state here (those beyond it would be zero times whatever c is)
    float state[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int row = group * ROWS + r;
        state[r] = s.first.p && kept && row < s.DA && col < s.DC
                       ? s.first.p[entry * s.first.entry + head * s.first.head + row * s.first.row + col * s.first.col]
                       : 0.f;
    }
    for (int64_t i = lo; i < hi; ++i) {
        const int64_t t = s.reverse ? hi - 1 - (i - lo) : i;
        const int buf = (int)((i - lo) & 1);
        for (int d = threadIdx.x; d < ROWS * kGroups; d += kColumns * kGroups) {
            la[buf][d] = d < s.DA ? (float)static_cast<const T*>(s.a.p)[at(s.a, t) + d] : 0.f;
            lb[buf][d] = d < s.DA ? (float)static_cast<const T*>(s.b.p)[at(s.b, t) + d] : 0.f;
        }
        const float c = col < s.DC ? (float)static_cast<const T*>(s.c.p)[at(s.c, t) + col] * s.alpha_s : 0.f;
        __syncthreads();
        float y = 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (r >= own) break;
            const float held = s.reverse ? state[r] : state[r] * decay;
            state[r] = held + lb[buf][group * ROWS + r] * c;
            y += state[r] * la[buf][group * ROWS + r];
            if (s.reverse) state[r] *= decay;
        }
        sums[buf][group][lane] = y;
        __syncthreads();
        if (group == 0 && col < s.DC) put(t, s.alpha_y * (sums[buf][0][lane] + sums[buf][1][lane] + sums[buf][2][lane] + sums[buf][3][lane]));
    }
    if (s.last.p && kept && col < s.DC) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int row = group * ROWS + r;
            if (row < s.DA) s.last.p[entry * s.last.entry + head * s.last.head + row * s.last.row + col * s.last.col] = state[r];
        }
    }
}

// The state before each segment from the segments' own sums, in place: a thread has VEC elements of a sequence's and head's, which lie in `first`
// as they do here.
constexpr int kScanAhead = 8;       // sums on their way at once
template <int VEC>
__global__ __launch_bounds__(256) void attention_scan_kernel(AttentionSums sums, AttentionBatch n, AttentionSegments g)
{
    typedef float floats __attribute__((ext_vector_type(VEC)));
    struct __attribute__((packed, aligned(4))) loose {
        floats v;
    };
    const AttentionSum& s = sums.of[blockIdx.y / (unsigned)n.H];
    const int i = (blockIdx.x * 256 + threadIdx.x) * VEC, head = blockIdx.y % (unsigned)n.H;
    if (i >= s.DA * s.DC) return;
    const float g2 = n.log_decay[head] * 1.44269504088896341f;
    // (an infinity does not fade: where l is above zero, so is its power, however small)
    const float decay = exp2f(g2 * (float)g.length), of_infinity = g2 > -INFINITY ? 1.f : 0.f;
    const int64_t step = (int64_t)n.H * s.DA * s.DC;
    for (int seq = blockIdx.z; seq < n.B; seq += gridDim.z) {
        int64_t len = n.T, slot;
        if (n.starts) {
            const int64_t lo = attention::packed_first(n, seq + 1);
            len = attention::packed_end(n, seq + 1, lo) - lo;
            slot = attention::packed_slot(g, lo, seq + 1);
        } else {
            slot = seq * ((n.T + g.length - 1) / g.length);
        }
        const int64_t segments = (len + g.length - 1) / g.length;
        if (segments < 2) continue;
        const float* first = attention::entry_of(s.first, s, n, seq, head);
        floats state = 0.f;
        if (first) state = reinterpret_cast<const loose*>(first + i)->v;
        float* p = s.states + slot * step + (int64_t)head * s.DA * s.DC + i;
        auto at = [&](int64_t k) { return reinterpret_cast<floats*>(p + k * step); };
        for (int64_t k = 0; k < segments; k += kScanAhead) {
            floats own[kScanAhead];
#pragma unroll
            for (int j = 0; j < kScanAhead; ++j) own[j] = *at(k + j + 1 < segments ? k + j : k);
#pragma unroll
            for (int j = 0; j < kScanAhead; ++j) {
                if (k + j < segments) *at(k + j) = state;
#pragma unroll
                for (int e = 0; e < VEC; ++e) state[e] = fmaf(state[e], fabsf(state[e]) == INFINITY ? of_infinity : decay, own[j][e]);
            }
        }
    }
}

// VEC elements of a row and group of heads a thread, dk's and dv's workgroups side by side (gradients of 4 x 2000 tokens, 16 heads on 4 of 128 bf16:
// 230 us, 23 more with a launch for each and an element a thread).
template <int EK, int VEC>
__global__ __launch_bounds__(256) void attention_fold_kernel(AttentionFold dk, AttentionFold dv, int H, int64_t T, int64_t rows)
{
    typedef typename ElemOf<EK>::type E;
    typedef float floats __attribute__((ext_vector_type(VEC)));
    typedef E elems __attribute__((ext_vector_type(VEC)));
    struct __attribute__((packed, aligned(sizeof(E)))) loose {
        elems v;
    };
    const AttentionFold& f = blockIdx.y ? dv : dk;
    const int heads = H / f.y.share, vectors = f.D / VEC, row_vectors = heads * vectors;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * row_vectors; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / row_vectors, batch = row / T;
        const int in_row = (int)(i - row * row_vectors), u = in_row / vectors, d = (in_row - u * vectors) * VEC;
        const float* part = f.part + (row * H + u * f.y.share) * f.D + d;
        floats sum = 0.f;
        for (int h = 0; h < f.y.share; ++h) sum += *reinterpret_cast<const floats*>(part + h * f.D);
        E* y = const_cast<E*>(static_cast<const E*>(f.y.p)) + batch * f.y.batch + (row - batch * T) * f.y.token + u * f.y.head + d;
        reinterpret_cast<loose*>(y)->v = __builtin_convertvector(sum, elems);
    }
}

// One token: the state is read and written once, 8 bytes an element that are all there is to move, and nothing else takes time.  A workgroup
// has LANES * VEC columns of a head, all their rows, so that no sums meet outside of it: LANES lanes a row, VEC columns each, the loads of
// several rows a thread on their way at once, before q and k are asked for.  One token of 128 requests on 16 heads of 128 x 128: 53.7 us, 5.0 TB/s
// of a state that is in no cache (6.4 of one that is).
template <int EK, int LANES, int VEC>
__global__ __launch_bounds__(256) void attention_step_kernel(AttentionStepArgs p)
{
    typedef typename ElemOf<EK>::type T;
    typedef float floats __attribute__((ext_vector_type(VEC)));
    typedef T elems __attribute__((ext_vector_type(VEC)));
    struct __attribute__((packed, aligned(sizeof(T)))) loose {
        elems v;
    };
    constexpr int G = 256 / LANES;          // rows side by side
    constexpr int ROWS = LANES < 32 ? 4 : 8;    // ... and one after another, on their way at once (with 8 for 4, of 8 lanes: 3 to 8 % more time)
    __shared__ float lq[256], lk[256];
    __shared__ floats sums[4][LANES];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int b = blockIdx.x, head = blockIdx.y, col = (blockIdx.z * LANES + lane) * VEC;
    const bool mine = col < p.DV;
    const int entry = p.slots ? p.slots[b] : b;
    T* o = const_cast<T*>(static_cast<const T*>(p.o.p)) + b * p.o.batch + head * p.o.head + col;
    if (entry < 0 || entry >= p.n_states) {
        if (group == 0 && mine) reinterpret_cast<loose*>(o)->v = (elems)(T)0.f;
        return;
    }
    // (lanes beyond the last column read the first one's)
    float* state = p.state + ((int64_t)entry * p.H + head) * p.DK * p.DV + (mine ? col : 0);
    floats s[ROWS];
    auto fetch = [&](int first) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = first + i * G;
            s[i] = *reinterpret_cast<const floats*>(state + (r < p.DK ? r : 0) * p.DV);
        }
    };
    fetch(group);
    const floats v = __builtin_convertvector(
        reinterpret_cast<const loose*>(static_cast<const T*>(p.v.p) + b * p.v.batch + head / p.v.share * p.v.head + (mine ? col : 0))->v, floats);
    const float decay = expf(p.log_decay[head]);
    if ((int)threadIdx.x < p.DK) {
        lq[threadIdx.x] = (float)static_cast<const T*>(p.q.p)[b * p.q.batch + head * p.q.head + threadIdx.x];
        lk[threadIdx.x] = (float)static_cast<const T*>(p.k.p)[b * p.k.batch + head / p.k.share * p.k.head + threadIdx.x];
    }
    __syncthreads();
    floats y = 0.f;
    for (int first = group; first < p.DK; first += ROWS * G) {
        if (first != group) fetch(first);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = first + i * G;
            if (r >= p.DK) break;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float now = fmaf(lk[r], v[e], s[i][e] * decay);
                s[i][e] = now;
                y[e] = fmaf(lq[r], now, y[e]);
            }
            if (mine) *reinterpret_cast<floats*>(state + r * p.DV) = s[i];
        }
    }
#pragma unroll
    for (int d = LANES; d < 64; d <<= 1)
#pragma unroll
        for (int e = 0; e < VEC; ++e) y[e] += __shfl_xor(y[e], d, 64);
    if (threadIdx.x % 64 < LANES) sums[threadIdx.x / 64][lane] = y;
    __syncthreads();
    if (group == 0 && mine)
        reinterpret_cast<loose*>(o)->v = __builtin_convertvector(p.scale * (sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane]), elems);
}

}  // namespace

hipError_t launch_attention_recurrent(const AttentionSum& s, const AttentionBatch& n, int ek, hipStream_t st)
{
    const dim3 grid((unsigned)(n.starts ? n.B + 2 : n.B), (unsigned)n.H, (unsigned)((s.DC + kColumns - 1) / kColumns));
    return with_elem(ek, [&](auto e) {
        note_kernel("attention_recurrent_kernel", ek, s.DA <= 64 ? 16 : s.DA <= 128 ? 32 : 64);
        if (s.DA <= 64)
            hipLaunchKernelGGL((attention_recurrent_kernel<e(), 16>), grid, dim3(kColumns * kGroups), 0, st, s, n);
        else if (s.DA <= 128)
            hipLaunchKernelGGL((attention_recurrent_kernel<e(), 32>), grid, dim3(kColumns * kGroups), 0, st, s, n);
        else
            hipLaunchKernelGGL((attention_recurrent_kernel<e(), 64>), grid, dim3(kColumns * kGroups), 0, st, s, n);
        return hipGetLastError();
    });
}

// (a translation unit for each format's kernels)
#define SW_ATTENTION_UNITS(what)                                                                                                        \
    hipError_t launch_attention_##what##_f32(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st);  \
    hipError_t launch_attention_##what##_bf16(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st); \
    hipError_t launch_attention_##what##_f16(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st);  \
    hipError_t launch_attention_##what(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, int ek, hipStream_t st) \
    {                                                                                                                                   \
        return ek == kElemF32    ? launch_attention_##what##_f32(s, n, g, st)                                                              \
               : ek == kElemBF16 ? launch_attention_##what##_bf16(s, n, g, st)                                                             \
                                 : launch_attention_##what##_f16(s, n, g, st);                                                             \
    }
SW_ATTENTION_UNITS(states)
SW_ATTENTION_UNITS(chunks)
#undef SW_ATTENTION_UNITS

// Sequences are cut where there are fewer heads than `want` workgroups, and where that gains more than the two launches that it takes. us:
// - equal ones of up to four chunks stay whole (256 tokens bf16, 8 x 16 heads of 64: 17.8 whole, 24.8 cut; 200 tokens fp32, gradients, 8 heads of
//   64: 24.5 and 22.9); so do packed ones that are short in the mean and 512 tokens together, which bounds what the longest of them takes (8 of
//   500 tokens bf16, 8 heads of 64: 15.1 and 24.1).
// - segments of one chunk of 64 while those of two would be fewer than 192 workgroups (1000 tokens fp32, 8 heads of 64: 25.4, with two 32.8; where
//   they would be 256, the states cost more: 2 x 1000 tokens half on 16 heads of 128 50 and 39), but for packed ones that are that short.
AttentionSegments attention_segments(const AttentionBatch& n, int DA, int DC, bool packed, int ek)
{
    const int64_t rows = packed ? n.T : n.T * n.B, columns = (DC + 127) / 128, two = 2 * kAttentionChunk;
    AttentionSegments g{(int64_t)1 << 62, 0};
    const int64_t want = 512;          // workgroups
    const bool brief = packed && n.T / n.B <= two;
    const bool whole = packed ? brief && n.T <= 4 * two : n.T <= (ek == kElemF32 ? two : 2 * two);
    if (!whole && (packed ? 1 : n.B) * n.H * columns < want) {
        const int64_t chunks = ((rows * n.H * columns + want - 1) / want + kAttentionChunk - 1) / kAttentionChunk;
        const int64_t least = !brief && rows * n.H * columns < 192 * two ? 1 : 2;
        g.length = (chunks < least ? least : chunks) * kAttentionChunk;
    }
    if (g.length >= n.T) g.length = (int64_t)1 << 62;
    g.count = packed ? n.T / g.length + n.B + 2 : n.B * ((n.T + g.length - 1) / g.length);
    return g;
}

hipError_t launch_attention_scan(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st)
{
    // Four elements a thread where single ones would be more than the chip has room for (the calls' us with one and with four: 24 packed sequences on
    // 8 heads of 64 x 64, 3072 workgroups, 38.8 and 33.2; 4096 tokens on 8 such heads, 128 workgroups, 27.2 and 28.1).
    const int elements = s.of[0].DA * s.of[0].DC;
    const int64_t single = (int64_t)((elements + 255) / 256) * n.H * s.count * n.B;
    const int vec = elements % 4 == 0 && single >= 2048 ? 4 : 1;
    const dim3 grid((unsigned)((elements / vec + 255) / 256), (unsigned)(n.H * s.count), (unsigned)(n.B < 65535 ? n.B : 65535));
    if (vec == 4)
        hipLaunchKernelGGL(attention_scan_kernel<4>, grid, dim3(256), 0, st, s, n, g);
    else
        hipLaunchKernelGGL(attention_scan_kernel<1>, grid, dim3(256), 0, st, s, n, g);
    return hipGetLastError();
}

hipError_t launch_attention_fold(const AttentionFold& dk, const AttentionFold& dv, const AttentionBatch& n, int ek, hipStream_t st)
{
    const int64_t rows = n.starts ? n.T : n.T * n.B, all = rows * (n.H / dk.y.share) * (dk.D > dv.D ? dk.D : dv.D);
    return with_elem(ek, [&](auto e) {
        auto with = [&](auto vec) {
            const int64_t groups = all / (256 * vec()) + 1;
            hipLaunchKernelGGL((attention_fold_kernel<e(), vec()>), dim3((unsigned)(groups < 8192 ? groups : 8192), 2), dim3(256), 0, st, dk, dv, n.H, n.T, rows);
            return hipGetLastError();
        };
        return dk.D % 4 || dv.D % 4 ? with(std::integral_constant<int, 1>()) : with(std::integral_constant<int, 4>());
    });
}

hipError_t launch_attention_step(const AttentionStepArgs& a, int ek, hipStream_t st)
{
    return with_elem(ek, [&](auto e) {
        auto with = [&](auto lanes, auto vec) {
            const dim3 grid((unsigned)a.B, (unsigned)a.H, (unsigned)((a.DV + lanes() * vec() - 1) / (lanes() * vec())));
            SW_NOTED_LAUNCH(note_kernel("attention_step_kernel", ek, lanes(), vec()), (attention_step_kernel<e(), lanes(), vec()>), grid, dim3(256), 0, st, a);
            return hipGetLastError();
        };
        typedef std::integral_constant<int, 4> four;
        if (a.DV % 4) return with(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
        // 32 columns a workgroup while there are fewer heads than four a CU (of 128 x 128, us with 128 columns and with 32: one request's 16 heads
        // 4.5 and 3.3, 512 heads 10.6 and 9.9, 1024 heads 21.8 and 22.0, 4096 heads 84.7 and 85.5)
        if (a.DV <= 32 || (int64_t)a.B * a.H < 1024) return with(std::integral_constant<int, 8>(), four());
        return a.DV <= 64 ? with(std::integral_constant<int, 16>(), four()) : with(std::integral_constant<int, 32>(), four());
    });
}

}  // namespace swconv
