// Linear attention in chunks of tokens on the matrix cores: 64 of bf16 and half, 32 of fp32.
//
// A chunk of n tokens (rows i, j of a, b, c; state S before it; l the head's decay; e0 = 1 forwards in time, 0 backwards):
//     y_i = alpha_y [ alpha_s sum_{j<=i} l^(i-j) (a_i . b_j) c_j  +  l^(i+e0) S^T a_i ],   S <- l^n S + alpha_s sum_j l^(n-e0-j) b_j c_j^T
// A wavefront has 16 or 32 columns of c and y and all rows of their state, in its accumulators: the state never leaves registers while a
// segment lasts.  Operands are arranged so that results become operands where they are: an accumulator's column is a lane's, its rows
// 4 (lane / 16) ... + 3 of sixteen; a product's K order is free as long as both operands have the same, so two tiles of S as they lie are
// the operand of S^T a, with a's values picked in that order.  Outputs are computed transposed (rows: columns of y), so that a lane holds
// four neighbouring columns of one token.  Pair products are shared: each 16 x 16 tile is computed by one wavefront and handed round in LDS.
//
// Operands derived in fp32 enter a product as sums of 16-bit values that hold fp32's bits: pair products, the state and its new terms are three
// bf16 values each, 25 bits.  In half the state and its new terms are two values scaled by a power of two, 22 bits, and pair products, whose range
// half may not have, are three bf16 values that meet c as two (which are all of it).  fp32 tensors stay fp32 throughout, on the fp32 matrix instructions.
// So a result is what sums in 32 bits make it before its one rounding.  (With two bf16 values each, 17 bits, 8192 tokens on 16 heads of 128 bf16 took 88 us
// for 94, gradients of 4 x 4096 tokens 318 for 359, and three times as many of their results were rounded the other way.)
//
// 8192 tokens on 16 heads of 128 bf16: 94 us; of one set of inputs 91, of which 63 without any of the computations (335 MB at 5.3 TB/s: the operands, those of
// the segments' own sums once more, and 134 MB of states); the rest are a chunk's phases, one after another in a workgroup, with two of these on a CU (76 KB of LDS each).
#pragma once

#include "sw_attention.h"

namespace swconv {

namespace {

using namespace attention;

// ---- operand formats -------------------------------------------------------------------------------------------------------------
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// c + a b, 16 x 16 over 32: a's row and b's column lane % 16, K 8 (lane / 16) ... + 7
__device__ __forceinline__ f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Two values rounded to 16 bits, packed, and two packed ones widened.
template <class V>
__device__ __forceinline__ unsigned pack(float a, float b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    const f32x2 p = {a, b};
    if constexpr (__is_same(V, bf16x8))
        return __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
    else
        return __builtin_bit_cast(unsigned, __builtin_convertvector(p, f16x2));
}
template <class V>
__device__ __forceinline__ f32x2 widen(unsigned p)
{
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    if constexpr (__is_same(V, bf16x8))
        return (f32x2){__uint_as_float(p << 16), __uint_as_float(p & 0xffff0000u)};
    else
        return __builtin_convertvector(__builtin_bit_cast(f16x2, p), f32x2);
}
template <class V>
__device__ __forceinline__ f32x8 widened(V v)
{
    const u32x4 u = __builtin_bit_cast(u32x4, v);
    f32x8 f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x2 w = widen<V>(u[j]);
        f[2 * j] = w[0], f[2 * j + 1] = w[1];
    }
    return f;
}

// v as a sum of N values of a format: v rounded, the rest rounded, ...  (In pairs: converted one by one the compiler converts each twice.)
template <class V, int N>
__device__ __forceinline__ void parts(f32x8 v, V (&p)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        u32x4 u;
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = pack<V>(v[2 * j], v[2 * j + 1]);
        p[k] = __builtin_bit_cast(V, u);
        const f32x8 w = widened<V>(p[k]);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] -= w[j];
    }
}

template <int EK>
struct Operand;
template <>
struct Operand<kElemBF16> {
    typedef bf16x8 vec;
    static constexpr int kState = 3, kTerm = 3;
};
template <>
struct Operand<kElemF16> {
    typedef f16x8 vec;
    static constexpr int kState = 2, kTerm = 2;
};
// fp32: K is 4, a value a lane; a vector holds the operands of four instructions, K in the order 4 (lane / 16) + element.
template <>
struct Operand<kElemF32> {
    typedef f32x4 vec;
};
__device__ __forceinline__ f32x4 multiply(f32x4 a, f32x4 b, f32x4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// Tokens of a chunk, and how many tiles of 16 and operand vectors of them there are.
constexpr int chunk_of(int ek) { return ek == kElemF32 ? kAttentionChunk / 2 : kAttentionChunk; }
constexpr int tiles_of(int ek) { return chunk_of(ek) / 16; }

// ---- tiles in LDS -------------------------------------------------------------------------------------------------------------------
// Rows of W values and 16 bytes more: sixteen rows' same 16 bytes (operands along a row) lie in different banks; the transposing reads of
// 16-bit values meet in twos, which costs less than an exchange of pieces, whose addresses are no constant apart.
template <int EK>
constexpr int pitch_of(int W) { return elem_size(EK) * W + 16; }

// Four rows' values of one column, from the addresses of four neighbouring columns of one row each: lane i of sixteen gives row i / 4, columns
// 4 (i % 4) ..., and gets column i.
__device__ __forceinline__ u32x2 turned_read(const unsigned char* p)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(p)));
}

template <class V>
__device__ __forceinline__ V joined(u32x2 a, u32x2 b)
{
    return __builtin_bit_cast(V, (u32x4){a[0], a[1], b[0], b[1]});
}

// The operand of a tile that lies row by row: column m0 + lane % 16, of the rows k0 and on those that are the lane's (8 (lane / 16) ... + 7;
// fp32: 4 (lane / 16) ... + 3), m0 and k0 constants.
template <int EK, int W>
__device__ __forceinline__ const unsigned char* turned_base(const unsigned char* tile, int lane)
{
    if constexpr (EK == kElemF32)
        return tile + 4 * (lane / 16) * pitch_of<EK>(W) + 4 * (lane % 16);
    else
        return tile + (8 * (lane / 16) + lane % 16 / 4) * pitch_of<EK>(W) + 8 * (lane % 4);
}
template <int EK, int W>
__device__ __forceinline__ typename Operand<EK>::vec turned(const unsigned char* base, int m0, int k0)
{
    typedef typename Operand<EK>::vec V;
    const unsigned char* p = base + k0 * pitch_of<EK>(W) + elem_size(EK) * m0;
    if constexpr (EK == kElemF32) {
        V v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const float*>(p + e * pitch_of<EK>(W));
        return v;
    } else {
        return joined<V>(turned_read(p), turned_read(p + 4 * pitch_of<EK>(W)));
    }
}

// A lane's number that the compiler takes for new: what is worked out from it is worked out again, not kept in registers from chunk to chunk.
__device__ __forceinline__ int renewed(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// A tile of a chunk's rows of W values on its way from memory to LDS: rows `from` and on, `width` elements, zeros elsewhere.
// Whole vectors are loaded by all threads without a branch, those that have none from a place that has one, and become zeros on their way
// into LDS: with loads in branches the compiler waits for each tile's before it begins the next one's.  Rows that are no whole number of
// vectors go element by element, when the tile is written.
template <int EK, int W, int THREADS>
struct Staged {
    typedef Row<EK> R;
    typedef typename R::T T;
    static constexpr int CH = chunk_of(EK), VEC = R::VEC, NCH = W / VEC, ALL = CH * NCH, N = (ALL + THREADS - 1) / THREADS, STEP = THREADS / NCH;
    static_assert(THREADS % NCH == 0 && (ALL % THREADS == 0 || ALL < THREADS), "whole rows, by all threads or each by one");
    typename R::vec v[N];
    // `tile`: the first of the rows in memory (its last, backwards in time), where there is one; `step`: from one to the next.  An element's
    // place is a 32-bit distance from it: rows that are further apart than that allows are no case for this kernel.
    static __device__ __forceinline__ unsigned place(int row, bool reverse, unsigned step) { return (reverse ? CH - 1 - row : row) * step; }
    __device__ __forceinline__ void fetch(const T* tile, unsigned step, bool reverse, int from, int width)
    {
        if (width % VEC) return;
        const int thread = renewed(threadIdx.x), c = thread % NCH * VEC;
        int row = thread / NCH;
        if (ALL < THREADS) row %= CH;
        const unsigned col = c < width ? c : 0;
        if (from == 0) {
            // (one distance for all of a thread's rows: what they are apart is the same for all threads)
            const unsigned own = (place(row, reverse, step) + col) * (unsigned)sizeof(T);
            const int64_t apart = (int64_t)STEP * (int)sizeof(T) * (reverse ? -(int64_t)step : (int64_t)step);
            const char* at = reinterpret_cast<const char*>(tile);
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = reinterpret_cast<const typename R::loose*>(at + k * apart + own)->v;
            return;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int r = row + k * STEP < from ? from : row + k * STEP;
            v[k] = reinterpret_cast<const typename R::loose*>(reinterpret_cast<const char*>(tile) + (place(r, reverse, step) + col) * (unsigned)sizeof(T))->v;
        }
    }
    __device__ __forceinline__ void put(unsigned char* to, const T* tile, unsigned step, bool reverse, int from, int width)
    {
        const int thread = renewed(threadIdx.x), c = thread % NCH * VEC, row = thread / NCH;
        if (width % VEC) {
#pragma unroll 1
            for (int i = thread; i < CH * W; i += THREADS) {
                const int r = i / W, d = i % W;
                *reinterpret_cast<T*>(to + r * pitch_of<EK>(W) + (int)sizeof(T) * d) = r >= from && d < width ? tile[place(r, reverse, step) + d] : (T)0.f;
            }
            return;
        }
        if (from > 0 || width < W)
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (row + k * STEP < from || c >= width) v[k] = (typename R::vec){};
        if (ALL < THREADS && thread >= ALL) return;
        unsigned char* p = to + row * pitch_of<EK>(W) + thread % NCH * 16;
#pragma unroll
        for (int k = 0; k < N; ++k) *reinterpret_cast<typename R::vec*>(p + k * STEP * pitch_of<EK>(W)) = v[k];
    }
};

// ---- the state as an operand -----------------------------------------------------------------------------------------------------------

// The largest of the lanes that have a column.
__device__ __forceinline__ float column_largest(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// The exponent that brings a magnitude to 2^13 ... 2^14, within what halves hold.  (Of a column far below 2^-30 some bits are lost; halves
// themselves end at 2^-24.)
__device__ __forceinline__ int half_exponent(float largest)
{
    const int e = __builtin_amdgcn_frexp_expf(largest);
    return (e < -30 ? -30 : e > 100 ? 100 : e) - 14;
}

// O = S^T a: rows, columns of y; columns, the chunk's tokens.  `a`: row lane % 16 of the tile, at the lane's place.
template <int EK, int MT, int CT>
__device__ __forceinline__ void state_times_a(const f32x4 (&S)[MT][CT], const float (&frame)[CT], const unsigned char* a, f32x4 (&O)[tiles_of(EK)][CT],
                                              const float (&reach)[tiles_of(EK)])
{
    typedef typename Operand<EK>::vec V;
    constexpr int TI = tiles_of(EK);
    float in[CT];
    f32x4 out[CT];
    if constexpr (EK == kElemF16) {
        // a scale for each column, which is a row of what is computed: those of a lane's four rows are other lanes'
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            float largest = 0.f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) largest = fmaxf(largest, fabsf(S[m][c][e]));
            const int exponent = half_exponent(column_largest(largest * frame[c]));
            in[c] = frame[c] * __builtin_amdgcn_ldexpf(1.f, -exponent);
#pragma unroll
            for (int e = 0; e < 4; ++e) out[c][e] = __builtin_amdgcn_ldexpf(1.f, __shfl(exponent, 4 * (threadIdx.x % 64 / 16) + e, 64));
        }
    }
    if constexpr (EK == kElemF32) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < TI; ++i) {
                const V x = *reinterpret_cast<const V*>(a + 16 * i * pitch_of<EK>(16 * MT) + 64 * m);
#pragma unroll
                for (int c = 0; c < CT; ++c) O[i][c] = multiply(S[m][c], x, O[i][c]);
            }
    } else {
#pragma unroll
        for (int m = 0; m < MT / 2; ++m) {
            V x[TI];
#pragma unroll
            for (int i = 0; i < TI; ++i) {
                const unsigned char* at = a + 16 * i * pitch_of<EK>(16 * MT) + 64 * m;
                x[i] = joined<V>(*reinterpret_cast<const u32x2*>(at), *reinterpret_cast<const u32x2*>(at + 32));
            }
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                f32x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = EK == kElemF16 ? S[2 * m + e / 4][c][e % 4] * in[c] : S[2 * m + e / 4][c][e % 4];
                V p[Operand<EK>::kState];
                parts(v, p);
#pragma unroll
                for (int k = Operand<EK>::kState; k-- > 0;)
#pragma unroll
                    for (int i = 0; i < TI; ++i) O[i][c] = multiply(p[k], x[i], O[i][c]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            O[i][c] *= reach[i];
            if (EK == kElemF16) O[i][c] *= out[c];
        }
}

// S <- whole S + sum over the chunk's tokens of b times weighted c (an operand vector's tokens: weights in `tables`, those of
// the first vector times shift).
template <int EK, int MT, int CT>
__device__ __forceinline__ void add_products(f32x4 (&S)[MT][CT], float (&frame)[CT], float whole, const typename Operand<EK>::vec (&cv)[2][CT],
                                             const float* tables, float shift, const unsigned char* b)
{
    typedef typename Operand<EK>::vec V;
    const f32x4 tail[2] = {*reinterpret_cast<const f32x4*>(tables), *reinterpret_cast<const f32x4*>(tables + 256)};
    if constexpr (EK == kElemF32) {
#pragma unroll
        for (int i = 0; i < MT * CT; ++i) S[i / CT][i % CT] *= whole;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            V w[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c) w[c] = cv[k][c] * tail[0] * (k == 0 ? shift : 1.f);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const V x = turned<EK, 16 * MT>(b, 16 * m, 16 * k);
#pragma unroll
                for (int c = 0; c < CT; ++c) S[m][c] = multiply(x, w[c], S[m][c]);
            }
        }
    } else {
        auto weighted = [&](int k, int c) {
            f32x8 w = widened<V>(cv[k][c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] *= tail[e / 4][e % 4];
            if (k == 0) w *= shift;
            return w;
        };
        float in[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            float fades = whole;
            if constexpr (EK == kElemF16) {
                float largest = 0.f;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const f32x8 w = weighted(k, c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) largest = fmaxf(largest, fabsf(w[e]));
                }
                largest = column_largest(largest);
                const float next = largest > 0.f ? __builtin_amdgcn_ldexpf(1.f, half_exponent(largest)) : frame[c];
                fades *= frame[c] / next;
                in[c] = 1.f / next;
                frame[c] = next;
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) S[m][c] *= fades;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            V p[CT][Operand<EK>::kTerm];
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                f32x8 w = weighted(k, c);
                if (EK == kElemF16) w *= in[c];
                parts(w, p[c]);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const V x = turned<EK, 16 * MT>(b, 16 * m, 32 * k);
#pragma unroll
                for (int q = Operand<EK>::kTerm; q-- > 0;)
#pragma unroll
                    for (int c = 0; c < CT; ++c) S[m][c] = multiply(x, p[c][q], S[m][c]);
            }
        }
    }
}

// ---- the kernel ---------------------------------------------------------------------------------------------------------------------

// Pair products in LDS: row i, column j, as three bf16 parts or as fp32.  16-bit rows are read in whole operand vectors of two tiles: those of the
// first two tiles end where the first vector does.
constexpr int kPairParts = 3;
template <int EK>
constexpr int pair_pitch(int tile) { return EK != kElemF32 && tile < 2 ? pitch_of<EK>(chunk_of(EK) / 2) : pitch_of<EK>(chunk_of(EK)); }
template <int EK>
constexpr int pair_row(int tile)                                        // where the rows of a tile begin
{
    return EK != kElemF32 && tile >= 2 ? 32 * pair_pitch<EK>(0) + 16 * (tile - 2) * pair_pitch<EK>(2) : 16 * tile * pair_pitch<EK>(0);
}
template <int EK>
constexpr int pair_bytes() { return pair_row<EK>(tiles_of(EK)); }           // of one part
template <int EK>
constexpr int pair_parts() { return EK == kElemF32 ? 1 : kPairParts; }
constexpr int kTables = 64 * 16 * 4;                // bytes of the lanes' weights

template <int EK, int DAP, int WC, bool OUTPUT>
constexpr int chunk_lds_bytes()
{
    return chunk_of(EK) * ((OUTPUT ? 2 : 1) * pitch_of<EK>(DAP) + pitch_of<EK>(WC)) + (OUTPUT ? pair_parts<EK>() * pair_bytes<EK>() : 0) + kTables;
}

__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }

// DAP: rows of the state (DA, padded); four wavefronts of CT tiles of 16 columns each.  OUTPUT false: only a segment's own sum.
//
// A chunk of fewer tokens (a sequence's last) lies in the last rows of its tiles: the weights of tokens are counted from a chunk's end.
template <int EK, int DAP, int CT, bool OUTPUT>
__global__ __launch_bounds__(256, DAP <= 128 ? 2 : 1) void attention_chunk_kernel(AttentionSums sums, AttentionBatch n, AttentionSegments g)
{
    typedef typename ElemOf<EK>::type T;
    typedef typename Operand<EK>::vec V;
    constexpr int CH = chunk_of(EK), TI = tiles_of(EK), ES = elem_size(EK), kPairs = pair_bytes<EK>(), NW = 4, WC = 16 * CT * NW, MT = DAP / 16, THREADS = 64 * NW;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    unsigned char *tb = smem, *tc = tb + CH * pitch_of<EK>(DAP), *ta = tc + CH * pitch_of<EK>(WC), *tp = ta + (OUTPUT ? CH * pitch_of<EK>(DAP) : 0);

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l16 = lane % 16, own = lane / 16;
    // Workgroups side by side: the sums of one segment and head, then its heads, whose rows lie side by side in memory.  The outputs go
    // through the segments from the last one, which the caches saw last.
    const unsigned block = OUTPUT ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    const AttentionSum& s = sums.of[block % (unsigned)sums.count];
    const int head = block / (unsigned)sums.count % (unsigned)n.H, col0 = blockIdx.y * WC, col = col0 + wave * 16 * CT + l16;
    const int width = s.DC - col0;                  // columns from here on
    if (width <= 0) return;                         // (of a sum with fewer than another of the launch)
    const Place at = locate(n, g, block / (unsigned)sums.count / (unsigned)n.H, s.reverse);
    if (at.none) return;
    if (at.rest) {
        if (OUTPUT) zero_rows<T>(s, at, head, col0, width < WC ? width : WC);
        return;
    }
    if (!OUTPUT && at.ends) return;                 // (nothing comes after the last segment)

    const int e0 = s.reverse ? 0 : 1;
    const float g2 = n.log_decay[head] * 1.44269504088896341f;
    const float chunk_decay = uniform(power(g2, CH)), shift = uniform(power(g2, CH / 2));
    // The lanes' weights, all wavefronts' the same, sixteen values a lane in fours:
    // 0, 1: of a chunk's tokens, the second operand vector's 8 own + e (fp32: 4 own + e): l^(CH - e0 - token)
    // 2, 3: of pair products (row j = 4 own + e, column i = l16 of a tile), on the diagonal and with i's tile the next after j's
    float* tables = reinterpret_cast<float*>(tp + (OUTPUT ? pair_parts<EK>() * kPairs : 0)) + 4 * lane;
    for (int k = wave; k < (OUTPUT ? 4 : 2); k += NW)
        for (int e = 0; e < 4; ++e) {
            const int gap = l16 - 4 * own - e;
            const int after = CH / 2 - e0 - (EK == kElemF32 ? 4 : 8) * own - 4 * k - e;
            const float v = k < 2 ? power(g2, after < 0 ? 0 : after) : gap < 0 && k == 2 ? 0.f : s.alpha_y * power(g2, k == 2 ? gap : 16 + gap);
            tables[256 * k + e] = s.alpha_s * v;
        }
    float further[3];
    const float near = s.alpha_y * power(g2, l16 + e0);         // ... and of the state in y, of a whole chunk's first tokens
    if constexpr (OUTPUT) {
#pragma unroll
        for (int k = 0; k < 3; ++k) further[k] = uniform(power(g2, 16 * (k + 1)));
        // (tiles above the diagonal that are read with their neighbours and never written)
        for (int i = threadIdx.x; EK != kElemF32 && i < kPairParts * 2 * 16 * 2; i += THREADS) {
            const int part = i / 64, tile = i / 32 % 2 * 2, row = i / 2 % 16, side = i % 2;
            *reinterpret_cast<u32x4*>(tp + part * kPairs + pair_row<EK>(tile) + row * pair_pitch<EK>(tile) + 32 * tile + 32 + 16 * side) = (u32x4){0, 0, 0, 0};
        }
    }
    // places in the tiles
    const unsigned char *along_b = tb + l16 * pitch_of<EK>(DAP) + 16 * own, *along_a = ta + l16 * pitch_of<EK>(DAP) + 16 * own;
    const unsigned char* picked_a = ta + l16 * pitch_of<EK>(DAP) + 4 * ES * own;
    const unsigned char *down_b = turned_base<EK, DAP>(tb, lane), *down_c = turned_base<EK, WC>(tc, lane) + 16 * ES * CT * wave;
    auto pairs = [&](int tile) { return tp + pair_row<EK>(tile) + l16 * pair_pitch<EK>(tile); };

    f32x4 S[MT][CT];
    float frame[CT];                                // half: S is in units of `frame`, a power of two a column
    auto begin = [&] {
        if constexpr (OUTPUT)
            load_state(S, s, n, at, head, col);
        else
#pragma unroll
            for (int i = 0; i < MT * CT; ++i) S[i / CT][i % CT] = 0.f;
#pragma unroll
        for (int c = 0; c < CT; ++c) frame[c] = 1.f;
    };
    begin();

    const int64_t dir = s.reverse ? -1 : 1;
    auto row_of = [&](const AttentionOperand& o, int64_t t) {
        return at.batch * o.batch + (at.lo + (s.reverse ? at.len - 1 - t : t)) * o.token + head / o.share * o.head;
    };
    Staged<EK, DAP, THREADS> sa, sb;
    Staged<EK, WC, THREADS> sc;
    // the first of a chunk's rows that is a token
    auto from_of = [&](int64_t t) { return at.last - t < CH ? CH - (int)(at.last - t) : 0; };
    // Where a chunk's tiles begin in memory, at the lowest of their rows: the first chunk's, moved on by `dir` CH rows with each chunk.
    auto begins = [&](const AttentionOperand& o) { return row_of(o, at.first + (s.reverse ? CH - 1 : 0)); };
    const T *pa = OUTPUT ? static_cast<const T*>(s.a.p) + begins(s.a) : nullptr, *pb = static_cast<const T*>(s.b.p) + begins(s.b),
            *pc = static_cast<const T*>(s.c.p) + begins(s.c) + col0;
    const int ys = s.y_f32 ? 4 : ES;
    char* py = OUTPUT ? static_cast<char*>(const_cast<void*>(s.y.p)) + (begins(s.y) + col0 + wave * 16 * CT) * ys : nullptr;
    bool bad = false;
    for (int64_t t = at.first; t < at.last; t += CH) {
        const int from = from_of(t);
        {
            // (a chunk of fewer rows: `from` of its tile's are before its first token)
            const int64_t back = dir * from;
            const T *xa = pa - back * s.a.token, *xb = pb - back * s.b.token, *xc = pc - back * s.c.token;
            if constexpr (OUTPUT) sa.fetch(xa, (unsigned)s.a.token, s.reverse, from, s.DA);
            sb.fetch(xb, (unsigned)s.b.token, s.reverse, from, s.DA);
            sc.fetch(xc, (unsigned)s.c.token, s.reverse, from, width);
            __syncthreads();
            if constexpr (OUTPUT) sa.put(ta, xa, (unsigned)s.a.token, s.reverse, from, s.DA);
            sb.put(tb, xb, (unsigned)s.b.token, s.reverse, from, s.DA);
            sc.put(tc, xc, (unsigned)s.c.token, s.reverse, from, width);
            __syncthreads();
            pa += dir * CH * s.a.token, pb += dir * CH * s.b.token, pc += dir * CH * s.c.token;
        }
        // c: columns a lane, eight tokens each
        V cv[2][CT];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < CT; ++c) cv[k][c] = turned<EK, WC>(down_c, 16 * c, CH / 2 * k);
        if constexpr (OUTPUT) {
            // pair products: the tiles on and below the diagonal, (0,0) (1,0) (1,1) (2,0) ..., a wavefront after another
            for (int tile = wave; tile < TI * (TI + 1) / 2; tile += NW) {
                const int i = (tile >= 1) + (tile >= 3) + (tile >= 6), j = tile - i * (i + 1) / 2;
                f32x4 p = 0.f;
#pragma unroll
                for (int k = 0; k < DAP * ES / 64; ++k)
                    p = multiply(*reinterpret_cast<const V*>(along_b + 16 * j * pitch_of<EK>(DAP) + 64 * k),
                                 *reinterpret_cast<const V*>(along_a + 16 * i * pitch_of<EK>(DAP) + 64 * k), p);
                p *= *reinterpret_cast<const f32x4*>(tables + (i == j ? 512 : 768)) * (i - j < 2 ? 1.f : further[i - j - 2]);
                unsigned char* to = pairs(i) + 16 * ES * j + 4 * ES * own;
                if constexpr (EK == kElemF32) {
                    *reinterpret_cast<f32x4*>(to) = p;
                } else {
#pragma unroll
                    for (int q = 0; q < kPairParts; ++q) {
                        const u32x2 h = {pack<bf16x8>(p[0], p[1]), pack<bf16x8>(p[2], p[3])};
                        const f32x2 h0 = widen<bf16x8>(h[0]), h1 = widen<bf16x8>(h[1]);
                        *reinterpret_cast<u32x2*>(to + q * kPairs) = h;
                        p -= (f32x4){h0[0], h0[1], h1[0], h1[1]};
                    }
                }
            }

            f32x4 O[TI][CT];
#pragma unroll
            for (int i = 0; i < TI * CT; ++i) O[i / CT][i % CT] = 0.f;
            float reach[TI];
#pragma unroll
            for (int i = 0; i < TI; ++i) reach[i] = i == 0 ? near : near * further[i - 1];
            if (from > 0)
#pragma unroll
                for (int i = 0; i < TI; ++i) {
                    const int token = 16 * i + l16 - from;
                    reach[i] = s.alpha_y * power(g2, (token < 0 ? 0 : token) + e0);
                }
            state_times_a<EK, MT, CT>(S, frame, picked_a, O, reach);
            __syncthreads();
            // pair products times c
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if constexpr (EK == kElemF32) {
#pragma unroll
                    for (int i = k; i < TI; ++i) {
                        const f32x4 p = *reinterpret_cast<const f32x4*>(pairs(i) + 64 * k + 16 * own);
#pragma unroll
                        for (int c = 0; c < CT; ++c) O[i][c] = multiply(cv[k][c], p, O[i][c]);
                    }
                } else {
                    bf16x8 c2[CT][2];
                    if constexpr (EK == kElemF16)
#pragma unroll
                        for (int c = 0; c < CT; ++c) parts(widened<V>(cv[k][c]), c2[c]);
#pragma unroll
                    for (int i = 2 * k; i < TI; ++i) {
#pragma unroll
                        for (int q = kPairParts; q-- > 0;) {
                            const bf16x8 p = *reinterpret_cast<const bf16x8*>(pairs(i) + q * kPairs + 64 * k + 16 * own);
#pragma unroll
                            for (int c = 0; c < CT; ++c)
                                if constexpr (EK == kElemF16) {
                                    // (the last parts' product is below what the others are rounded to)
                                    if (q < kPairParts - 1) O[i][c] = multiply(c2[c][1], p, O[i][c]);
                                    O[i][c] = multiply(c2[c][0], p, O[i][c]);
                                } else {
                                    O[i][c] = multiply(cv[k][c], p, O[i][c]);
                                }
                        }
                    }
                }
            }
            bad |= any_nonfinite(O);
            const int now = renewed(lane);
            auto place = [&](int row) { return (unsigned)((s.reverse ? CH - 1 - row : row) * (unsigned)s.y.token + 4 * (now / 16)) * (unsigned)ys; };
            auto put_all = [&](auto* as) {
                typedef std::remove_pointer_t<decltype(as)> Y;
                if (from == 0 && width - wave * 16 * CT >= 16 * CT) {
                    const unsigned mine = place(now % 16);
                    const int64_t apart = dir * 16 * (int)sizeof(Y) * s.y.token;
#pragma unroll
                    for (int i = 0; i < TI; ++i)
#pragma unroll
                        for (int c = 0; c < CT; ++c) store_four(reinterpret_cast<Y*>(py + i * apart + mine) + 16 * c, O[i][c], 4);
                    return;
                }
                char* to = py - dir * from * s.y.token * (int)sizeof(Y);
#pragma unroll
                for (int i = 0; i < TI; ++i)
#pragma unroll
                    for (int c = 0; c < CT; ++c)
                        if (16 * i + now % 16 >= from)
                            store_four(reinterpret_cast<Y*>(to + place(16 * i + now % 16)) + 16 * c, O[i][c], width - wave * 16 * CT - 4 * (now / 16) - 16 * c);
            };
            if (s.y_f32)
                put_all(static_cast<float*>(nullptr));
            else
                put_all(static_cast<T*>(nullptr));
            py += dir * CH * s.y.token * ys;
        }
        add_products<EK, MT, CT>(S, frame, from == 0 ? chunk_decay : power(g2, CH - from), cv, tables, shift, down_b);
    }
#pragma unroll
    for (int i = 0; i < MT * CT; ++i) S[i / CT][i % CT] *= frame[i % CT];
    float* const last = OUTPUT && at.ends ? entry_of(s.last, s, n, at.seq, head) : nullptr;
    // (outputs say nothing of the last chunk's new terms, nor of a half state that is too large for units of theirs)
    if (!OUTPUT || last) bad |= any_nonfinite(S);
    if (bad) {
        __builtin_amdgcn_s_waitcnt(0);              // (what has been stored is stored before it is stored again)
        begin();
        const T *a = OUTPUT ? static_cast<const T*>(s.a.p) + row_of(s.a, at.first) : nullptr, *b = static_cast<const T*>(s.b.p) + row_of(s.b, at.first);
#pragma unroll
        for (int i = 0; i < CT; ++i) {
            const T* c = static_cast<const T*>(s.c.p) + row_of(s.c, at.first) + col + 16 * i;
            const int64_t to = row_of(s.y, at.first) + col + 16 * i;
            void* y = s.y_f32 ? static_cast<void*>(const_cast<float*>(static_cast<const float*>(s.y.p)) + to)
                              : static_cast<void*>(const_cast<T*>(static_cast<const T*>(s.y.p)) + to);
            token_by_token(S, i, TokenByToken<T>{a, b, c, dir * s.a.token, dir * s.b.token, dir * s.c.token, dir * s.y.token, at.last - at.first, s.DA,
                                                 power(g2, 1), s.alpha_s, s.alpha_y, s.reverse, s.y_f32, col + 16 * i < s.DC, y});
        }
    }
    if constexpr (OUTPUT) {
        if (last) store_state(S, last, s.last.row, s.last.col, s, col);
    } else {
        store_state(S, s.states + (at.slot * n.H + head) * s.DA * s.DC, s.DC, 1, s, col);
    }
}

// The sums of one size in one launch; all of them where that does not fill the chip.
template <int EK, bool OUTPUT>
hipError_t launch_chunk(const AttentionSums& all, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st)
{
    auto padded = [](int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 128 ? 128 : 256; };
    auto columns = [](int d) { return d <= 64 ? 0 : (d + 127) / 128; };
    // At most two workgroups of 64 columns a CU: in one launch, with as many rows of the state as the most of them have (gradients of 500 tokens
    // on 8 heads of 64 x 128 bf16, us: 32.6 in two launches, 26.5 in one).  States of 256 rows have no room for two on a CU.
    int most_rows = 0, most_columns = 0;
    for (int i = 0; i < all.count; ++i) {
        most_rows = padded(all.of[i].DA) > most_rows ? padded(all.of[i].DA) : most_rows;
        most_columns = all.of[i].DC > most_columns ? all.of[i].DC : most_columns;
    }
    const bool together = most_rows <= 128 && g.count * n.H * all.count * ((most_columns + 63) / 64) <= 512;
    bool done[3] = {false, false, false};
    for (int i = 0; i < all.count; ++i) {
        if (done[i]) continue;
        AttentionSums s;
        s.count = 0;
        const int da = together ? most_rows : padded(all.of[i].DA);
        int dc = all.of[i].DC;                  // the most columns of them
        for (int j = i; j < all.count; ++j)
            if (!done[j] && (together || (padded(all.of[j].DA) == da && columns(all.of[j].DC) == columns(dc)))) {
                s.of[s.count++] = all.of[j], done[j] = true;
                dc = all.of[j].DC > dc ? all.of[j].DC : dc;
            }
        auto with = [&](auto dap, auto ct) {
            constexpr int lds = chunk_lds_bytes<EK, dap(), 64 * ct(), OUTPUT>();
            static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(attention_chunk_kernel<EK, dap(), ct(), OUTPUT>),
                                                               hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            if (attr != hipSuccess) return attr;
            const dim3 grid((unsigned)(g.count * n.H * s.count), (unsigned)((dc + 64 * ct() - 1) / (64 * ct())));
            note_kernel("attention_chunk_kernel", EK, dap(), ct(), OUTPUT);
            hipLaunchKernelGGL((attention_chunk_kernel<EK, dap(), ct(), OUTPUT>), grid, dim3(256), lds, st, s, n, g);
            return hipGetLastError();
        };
        auto rows = [&](auto ct) {
            switch (da) {
            case 32: return with(std::integral_constant<int, 32>(), ct);
            case 64: return with(std::integral_constant<int, 64>(), ct);
            case 128: return with(std::integral_constant<int, 128>(), ct);
            default: return with(std::integral_constant<int, 256>(), ct);
            }
        };
        // Wavefronts of 16 columns where workgroups of 128 columns would be no more than the CUs: twice as many, each through in less time (128
        // tokens, us with 32 and with 16 columns: 8 heads of 128 bf16 17.2 and 13.5, 192 heads 18.1 and 17.8, 288 heads 22.9 and 27.0).
        const bool few = g.count * n.H * s.count * ((dc + 127) / 128) <= 256;
        const hipError_t e = dc <= 64 || few ? rows(std::integral_constant<int, 1>()) : rows(std::integral_constant<int, 2>());
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

}  // namespace swconv
