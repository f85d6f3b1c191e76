// Linear attention in chunks of 64 tokens on the matrix cores: bf16 and half.
//
// A chunk of n tokens (rows i, j of a, b, c; state S before it; l the head's decay; e0 = 1 forwards in time, 0 backwards):
//     y_i = alpha_y [ alpha_s sum_{j<=i} l^(i-j) (a_i . b_j) c_j  +  l^(i+e0) S^T a_i ],   S <- l^n S + alpha_s sum_j l^(n-e0-j) b_j c_j^T
// A wavefront has 32 columns of c and y and all rows of their state, in its accumulators: the state never leaves registers while a
// segment lasts.  Operands are arranged so that results become operands where they are: an accumulator's column is a lane's, its rows
// {0-3, 8-11, 16-19, 24-27} + 4 (lane / 32); a product's K order is free as long as both operands have the same, so S as it lies is the
// operand of S^T a, with a's values picked in that order.  Outputs are computed transposed (rows: columns of y), so that a lane holds
// four neighbouring columns of one token.  Pair products are shared: each 32 x 32 tile is computed by one wavefront and handed round in LDS.
//
// Operands derived in fp32 enter a product as sums of 16-bit values, and which sums is a choice of precision: pair products two bf16
// values (17 bits; half, whose range they may leave, meets c as two bf16 values too), the state two bf16 values or one half scaled by a
// power of two (both finer than y's own rounding), the state's new terms three bf16 or two scaled half values (22 bits and more: the
// state is an fp32 result).
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

__device__ __forceinline__ f32x16 multiply(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// v as a sum of N values of a format: v rounded, the rest rounded, ...
template <class V, int N>
__device__ __forceinline__ void parts(f32x8 v, V (&p)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        p[k] = __builtin_convertvector(v, V);
        if (k + 1 < N) v -= __builtin_convertvector(p[k], f32x8);
    }
}

template <int EK>
struct Operand;
template <>
struct Operand<kElemBF16> {
    typedef bf16x8 vec;
    static constexpr int kState = 2, kTerm = 3;
};
template <>
struct Operand<kElemF16> {
    typedef f16x8 vec;
    static constexpr int kState = 1, kTerm = 2;
};

// ---- tiles in LDS -------------------------------------------------------------------------------------------------------------------
// Rows of W 16-bit values and 16 bytes more: sixteen rows' same 16 bytes (operands along a row) lie in different banks; the transposing
// reads meet in twos, which costs less than an exchange of pieces, whose addresses are no constant apart.
constexpr int pitch_of(int W) { return 2 * W + 16; }

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

// The operand (column m0 + lane % 32, rows k0 + 8 (lane / 32) ... + 7) of a tile that lies row by row, m0 and k0 constants.
template <int W>
__device__ __forceinline__ const unsigned char* turned_base(const unsigned char* tile, int lane)
{
    return tile + (8 * (lane / 32) + lane % 16 / 4) * pitch_of(W) + 2 * (16 * (lane / 16 % 2) + 4 * (lane % 4));
}
template <int W, class V>
__device__ __forceinline__ V turned(const unsigned char* base, int m0, int k0)
{
    return joined<V>(turned_read(base + k0 * pitch_of(W) + 2 * m0), turned_read(base + (k0 + 4) * pitch_of(W) + 2 * m0));
}

// A tile of kAttentionChunk rows of W values on its way from memory to LDS: rows `from` and on, `width` elements, zeros elsewhere.
template <int EK, int W, int THREADS>
struct Staged {
    typedef Row<EK> R;
    static constexpr int NCH = W / 8, N = kAttentionChunk * NCH / THREADS, STEP = THREADS / NCH;
    typename R::vec v[N];
    // offset: of row 0, where there is one
    __device__ __forceinline__ void fetch(const AttentionOperand& o, int64_t offset, int64_t stride, int from, int width)
    {
        const int c = threadIdx.x % NCH * 8, row = threadIdx.x / NCH;
        const typename R::T* p = static_cast<const typename R::T*>(o.p) + offset + row * stride;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = (typename R::vec){};
        if (width % 8 == 0) {
            if (c >= width) return;
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (row + k * STEP >= from) v[k] = reinterpret_cast<const typename R::loose*>(p + k * STEP * stride + c)->v;
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (row + k * STEP >= from && c < width) v[k] = R::load(p + k * STEP * stride, c, width);
        }
    }
    __device__ __forceinline__ void put(unsigned char* tile) const
    {
        unsigned char* p = tile + threadIdx.x / NCH * pitch_of(W) + threadIdx.x % NCH * 16;
#pragma unroll
        for (int k = 0; k < N; ++k) *reinterpret_cast<typename R::vec*>(p + k * STEP * pitch_of(W)) = v[k];
    }
};

// ---- the state as an operand -----------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float larger_half(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// The exponent that brings a magnitude to 2^13 ... 2^14, within what halves hold.  (Of a column, or a state, far below 2^-30 some bits are
// lost; halves themselves end at 2^-24.)
__device__ __forceinline__ int half_exponent(float largest)
{
    const int e = __builtin_amdgcn_frexp_expf(largest);
    return (e < -30 ? -30 : e > 100 ? 100 : e) - 14;
}

// O = S^T a: rows, columns of y; columns, the chunk's tokens.  `a`: row lane % 32 of the tile, at the half's place.
template <int EK, int MT>
__device__ __forceinline__ void state_times_a(const f32x16 (&S)[MT], float frame, const unsigned char* a, f32x16 (&O)[2], const float (&reach)[2])
{
    typedef typename Operand<EK>::vec V;
    float in = 1.f, out = 1.f;
    if constexpr (EK == kElemF16) {
        // one scale for the wavefront's columns: they are the rows of what is computed
        float largest = 0.f;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) largest = fmaxf(largest, fabsf(S[m][r]));
        largest *= frame;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d, 64));
        largest = larger_half(largest);
        const int e = half_exponent(largest);
        in = frame * __builtin_amdgcn_ldexpf(1.f, -e);
        out = __builtin_amdgcn_ldexpf(1.f, e);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            f32x8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = EK == kElemF16 ? S[m][8 * q + e] * in : S[m][8 * q + e];
            V p[Operand<EK>::kState];
            parts(v, p);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned char* at = a + 32 * i * pitch_of(32 * MT) + 64 * m + 32 * q;
                const V x = joined<V>(*reinterpret_cast<const u32x2*>(at), *reinterpret_cast<const u32x2*>(at + 16));
#pragma unroll
                for (int k = Operand<EK>::kState; k-- > 0;) O[i] = multiply(p[k], x, O[i]);
            }
        }
#pragma unroll
    for (int i = 0; i < 2; ++i) O[i] *= reach[i] * out;
}

// S <- whole S + sum over the chunk's tokens of b times w (w: weighted c, tokens 16 k + 8 (lane / 32) + e).
template <int EK, int MT>
__device__ __forceinline__ void add_products(f32x16 (&S)[MT], float& frame, float whole, f32x8 (&w)[4], const unsigned char* b)
{
    typedef typename Operand<EK>::vec V;
    if constexpr (EK == kElemF16) {
        float largest = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) largest = fmaxf(largest, fabsf(w[k][e]));
        largest = larger_half(largest);
        const float next = largest > 0.f ? __builtin_amdgcn_ldexpf(1.f, half_exponent(largest)) : frame;
        whole *= frame / next;
        const float in = 1.f / next;
        frame = next;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] *= in;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) S[m] *= whole;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        V p[Operand<EK>::kTerm];
        parts(w[k], p);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const V x = turned<32 * MT, V>(b, 32 * m, 16 * k);
#pragma unroll
            for (int q = Operand<EK>::kTerm; q-- > 0;) S[m] = multiply(x, p[q], S[m]);
        }
    }
}

// ---- the kernel ---------------------------------------------------------------------------------------------------------------------

constexpr int kPairPitch = pitch_of(kAttentionChunk), kPairs = kAttentionChunk * kPairPitch;       // bytes of one part of the pair products

template <int DAP, int NW, bool OUTPUT>
constexpr int chunk_lds_bytes() { return kAttentionChunk * ((OUTPUT ? 2 : 1) * pitch_of(DAP) + pitch_of(32 * NW)) + (OUTPUT ? 2 * kPairs : 0); }

__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }

// DAP: rows of the state (DA, padded); NW wavefronts of 32 columns each.  OUTPUT false: only a segment's own sum.
//
// A chunk of fewer tokens (a sequence's last) lies in the last rows of its tiles: the weights of tokens are counted from a chunk's end.
template <int EK, int DAP, int NW, bool OUTPUT>
__global__ __launch_bounds__(64 * NW, DAP <= 128 ? 2 : 1) void attention_chunk_kernel(AttentionSum s, AttentionBatch n, AttentionSegments g, bool turned_states)
{
    typedef typename ElemOf<EK>::type T;
    typedef typename Operand<EK>::vec V;
    constexpr int CH = kAttentionChunk, WC = 32 * NW, MT = DAP / 32, THREADS = 64 * NW;
    constexpr bool AHEAD = (OUTPUT ? 2 : 1) * Staged<EK, DAP, THREADS>::N + Staged<EK, WC, THREADS>::N <= 12;    // the next chunk in registers
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    unsigned char *tb = smem, *tc = tb + CH * pitch_of(DAP), *ta = tc + CH * pitch_of(WC), *tp = ta + (OUTPUT ? CH * pitch_of(DAP) : 0);

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, half = lane / 32, l32 = lane % 32;
    const int head = blockIdx.y, col0 = blockIdx.z * WC, col = col0 + wave * 32 + l32;
    const int width = s.DC - col0;                  // columns from here on
    const Place at = locate(n, g);
    if (at.none) return;
    if (at.rest) {
        if (OUTPUT) zero_rows<T>(s, at, head, col0, width < WC ? width : WC);
        return;
    }
    if (!OUTPUT && at.ends) return;                 // (nothing comes after the last segment)

    const int e0 = s.reverse ? 0 : 1;
    const float g2 = n.log_decay[head] * 1.44269504088896341f;
    const float chunk_decay = uniform(power(g2, CH));
    // weights of a chunk's tokens 16 k + 8 half + e: l^(CH - e0 - token) = shift[k] * tail[e]
    float tail[8], shift[4];
#pragma unroll
    for (int e = 0; e < 8; ++e) tail[e] = s.alpha_s * power(g2, 16 - e0 - 8 * half - e);
#pragma unroll
    for (int k = 0; k < 4; ++k) shift[k] = uniform(power(g2, 16 * (3 - k)));
    // pair products: tiles of 32 x 32 (rows j, columns i): (0,0) (1,0) (1,1) of four wavefronts, (0,0) and (1,1), (1,0) of two
    const int ti = NW >= 4 ? (wave + 1) / 2 : wave, tj = NW >= 4 ? wave / 2 : 0;
    float fade[16];
    if constexpr (OUTPUT)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int gap = 32 * (ti - tj) + l32 - tile_row(r, half);
            fade[r] = gap < 0 ? 0.f : s.alpha_y * s.alpha_s * power(g2, gap);
        }
    // places in the tiles
    const unsigned char *along_b = tb + (32 * tj + l32) * pitch_of(DAP) + 16 * half, *along_a = ta + (32 * ti + l32) * pitch_of(DAP) + 16 * half;
    const unsigned char *picked_a = ta + l32 * pitch_of(DAP) + 8 * half, *down_b = turned_base<DAP>(tb, lane), *down_c = turned_base<WC>(tc, lane) + 64 * wave;
    unsigned char* pairs = tp + l32 * kPairPitch;

    f32x16 S[MT];
    if constexpr (OUTPUT)
        load_state(S, s, n, g, at, head, col, turned_states);
    else
#pragma unroll
        for (int m = 0; m < MT; ++m) S[m] = 0.f;
    float frame = 1.f;                              // half: S is in units of `frame`, a power of two a column

    const int64_t dir = s.reverse ? -1 : 1;
    auto row_of = [&](const AttentionOperand& o, int64_t t) {
        return at.batch * o.batch + (at.lo + (s.reverse ? at.len - 1 - t : t)) * o.token + head / o.share * o.head;
    };
    Staged<EK, DAP, THREADS> sa, sb;
    Staged<EK, WC, THREADS> sc;
    // the first of a chunk's rows that is a token, and the token that row 0 would be
    auto from_of = [&](int64_t t) { return at.last - t < CH ? CH - (int)(at.last - t) : 0; };
    auto fetch = [&](int64_t t) {
        const int from = from_of(t);
        if constexpr (OUTPUT) sa.fetch(s.a, row_of(s.a, t - from), dir * s.a.token, from, s.DA);
        sb.fetch(s.b, row_of(s.b, t - from), dir * s.b.token, from, s.DA);
        sc.fetch(s.c, row_of(s.c, t - from) + col0, dir * s.c.token, from, width);
    };
    auto slowly = [&](int64_t t) {
        const int from = from_of(t);
        const int64_t to = row_of(s.y, t - from) + col;
        float held[16 * MT];
#pragma unroll
        for (int i = 0; i < 16 * MT; ++i) held[i] = S[i / 16][i % 16] * frame;
        void* y = s.y_f32 ? static_cast<void*>(const_cast<float*>(static_cast<const float*>(s.y.p)) + to)
                          : static_cast<void*>(const_cast<T*>(static_cast<const T*>(s.y.p)) + to);
        token_by_token<T, MT>(held, TokenByToken<T>{OUTPUT ? ta : nullptr, tb, tc + (wave * 32 + l32) * 2, pitch_of(DAP), pitch_of(WC), from, CH, s.DA,
                                                    power(g2, 1), s.alpha_s, s.alpha_y, s.reverse, s.y_f32, col < s.DC, y, dir * s.y.token});
#pragma unroll
        for (int i = 0; i < 16 * MT; ++i) S[i / 16][i % 16] = held[i];
        frame = 1.f;
    };
    if (AHEAD && at.first < at.last) fetch(at.first);
    for (int64_t t = at.first; t < at.last; t += CH) {
        const int from = from_of(t);
        if (!AHEAD) fetch(t);
        __syncthreads();
        if constexpr (OUTPUT) sa.put(ta);
        sb.put(tb);
        sc.put(tc);
        __syncthreads();
        if (AHEAD && t + CH < at.last) fetch(t + CH);
        // c: columns a lane, eight tokens each
        V cv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) cv[k] = turned<WC, V>(down_c, 0, 16 * k);
        if constexpr (OUTPUT) {
            auto pair_tile = [&](int di, int dj, int i, int j) {
                f32x16 p = 0.f;
#pragma unroll
                for (int k = 0; k < DAP / 16; ++k)
                    p = multiply(*reinterpret_cast<const V*>(along_b + dj * pitch_of(DAP) + 32 * k),
                                 *reinterpret_cast<const V*>(along_a + di * pitch_of(DAP) + 32 * k), p);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    f32x8 v;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = p[8 * q + e] * fade[8 * q + e];
                    bf16x8 w[2];
                    parts(v, w);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const u32x4 u = __builtin_bit_cast(u32x4, w[k]);
                        unsigned char* to = pairs + k * kPairs + 32 * i * kPairPitch + 64 * j + 32 * q + 8 * half;
                        *reinterpret_cast<u32x2*>(to) = (u32x2){u[0], u[1]};
                        *reinterpret_cast<u32x2*>(to + 16) = (u32x2){u[2], u[3]};
                    }
                }
            };
            if (NW < 4 || wave < 3) pair_tile(0, 0, ti, tj);
            if (NW < 4 && wave == 0) pair_tile(32, 32, 1, 1);

            f32x16 O[2] = {0.f, 0.f};
            float reach[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int token = 32 * i + l32 - from;
                reach[i] = s.alpha_y * power(g2, (token < 0 ? 0 : token) + e0);
            }
            state_times_a<EK, MT>(S, frame, picked_a, O, reach);
            __syncthreads();
            // pair products times c
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                bf16x8 c2[2];
                if constexpr (EK == kElemF16) parts(__builtin_convertvector(cv[k], f32x8), c2);
#pragma unroll
                for (int i = k / 2; i < 2; ++i) {
                    bf16x8 p[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q) p[q] = *reinterpret_cast<const bf16x8*>(pairs + q * kPairs + 32 * i * kPairPitch + 32 * k + 16 * half);
                    if constexpr (EK == kElemF16) {
                        O[i] = multiply(c2[1], p[0], O[i]);
                        O[i] = multiply(c2[0], p[1], O[i]);
                        O[i] = multiply(c2[0], p[0], O[i]);
                    } else {
                        O[i] = multiply(cv[k], p[1], O[i]);
                        O[i] = multiply(cv[k], p[0], O[i]);
                    }
                }
            }
            if (__builtin_expect(any_nonfinite(O), 0)) {
                slowly(t);
                continue;
            }
            const int64_t to = row_of(s.y, t - from);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (32 * i + l32 >= from) store_outputs<T>(O[i], s, to, dir * s.y.token, 32 * i + l32, col0 + wave * 32);
        }
        f32x8 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = __builtin_convertvector(cv[k], f32x8);
#pragma unroll
            for (int e = 0; e < 8; ++e) w[k][e] *= tail[e] * shift[k];
        }
        add_products<EK, MT>(S, frame, from == 0 ? chunk_decay : power(g2, CH - from), w, down_b);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) S[m] *= frame;
    if constexpr (OUTPUT) {
        float* p = at.ends ? entry_of(s.last, s, n, at.seq, head) : nullptr;
        if (p) store_state(S, p, s.last.row, s.last.col, s, col);
    } else {
        // a sum with an infinity or a NaN in it: once more, token by token
        if (__syncthreads_or(any_nonfinite(S))) {
            frame = 1.f;
#pragma unroll
            for (int m = 0; m < MT; ++m) S[m] = 0.f;
            for (int64_t t = at.first; t < at.last; t += CH) {
                fetch(t);
                __syncthreads();
                sb.put(tb);
                sc.put(tc);
                __syncthreads();
                slowly(t);
            }
        }
        store_state(S, g.states + (at.slot * n.H + head) * s.DA * s.DC, s.DC, 1, s, col);
    }
}

template <int EK, bool OUTPUT>
hipError_t launch_chunk(const AttentionSum& s, const AttentionBatch& n, const AttentionSegments& g, bool turned, hipStream_t st)
{
    auto with = [&](auto dap, auto nw) {
        constexpr int lds = chunk_lds_bytes<dap(), nw(), OUTPUT>();
        static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(attention_chunk_kernel<EK, dap(), nw(), OUTPUT>),
                                                           hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (attr != hipSuccess) return attr;
        const dim3 grid((unsigned)g.count, (unsigned)n.H, (unsigned)((s.DC + 32 * nw() - 1) / (32 * nw())));
        note_kernel("attention_chunk_kernel", EK, dap(), nw(), OUTPUT);
        hipLaunchKernelGGL((attention_chunk_kernel<EK, dap(), nw(), OUTPUT>), grid, dim3(64 * nw()), lds, st, s, n, g, turned);
        return hipGetLastError();
    };
    auto rows = [&](auto nw) {
        if (s.DA <= 32) return with(std::integral_constant<int, 32>(), nw);
        if (s.DA <= 64) return with(std::integral_constant<int, 64>(), nw);
        if (s.DA <= 128) return with(std::integral_constant<int, 128>(), nw);
        return with(std::integral_constant<int, 256>(), nw);
    };
    return s.DC <= 64 ? rows(std::integral_constant<int, 2>()) : rows(std::integral_constant<int, 4>());
}

}  // namespace

}  // namespace swconv
