// What the kernels of linear attention in chunks share: a workgroup's place among sequences and segments, the state on its way between
// memory and accumulators, outputs on theirs to memory.
#pragma once

#include "sw_layers.h"

namespace swconv {
namespace attention {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// l^n for n >= 0, from log2(l): 1 for n = 0, whatever l is; below 2^-126 in steps of 2^-149 (what it is multiplied with may be large)
__device__ __forceinline__ float power(float g2, int n) { return n == 0 ? 1.f : exp2f(g2 * (float)n); }

__device__ __forceinline__ int64_t clamped(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

// Rows [lo, hi) of a packed batch's sequence j - 1, j = 1 ... B; j = 0 and B + 1: the rows before the first and after the last one.
__device__ __forceinline__ int64_t packed_first(const AttentionBatch& n, int j) { return j == 0 ? 0 : clamped(n.starts[j - 1], 0, n.T); }
__device__ __forceinline__ int64_t packed_end(const AttentionBatch& n, int j, int64_t lo) { return j == n.B + 1 ? n.T : clamped(n.starts[j], lo, n.T); }

// Where a workgroup is: tokens first ... last - 1, in the order they are worked on, of a sequence of `len` rows from row `lo` of `batch`.
struct Place {
    int64_t lo, len, first, last, batch, slot;
    int seq;
    bool none;          // nothing here
    bool rest;          // rows in no sequence
    bool alone;         // the only segment
    bool ends;          // the last segment
};

// Segment places of a packed batch: sequence j's first one is lo / length + j, which leaves each at least one and all they need.
__device__ __forceinline__ int64_t packed_slot(const AttentionSegments& g, int64_t lo, int j) { return lo / g.length + j; }

// place: of a segment, in the rows' order; backwards in time a sequence's segments are worked on from its end, the first place is the last one's.
__device__ __forceinline__ Place locate(const AttentionBatch& n, const AttentionSegments& g, int64_t place, bool reverse)
{
    Place p;
    p.slot = place;
    int64_t segment;
    if (n.starts) {
        // the last j whose first place is not past this one: 64 of them at a time, a lane each
        int count = 0;
        for (int base = 0; base < n.B + 2; base += 64) {
            const int j = base + (int)(threadIdx.x % 64);
            const bool before = j < n.B + 2 && packed_slot(g, packed_first(n, j), j) <= p.slot;
            const int found = __popcll(__ballot(before));
            count += found;
            if (found < 64) break;
        }
        const int j = count - 1;
        p.lo = packed_first(n, j);
        p.len = packed_end(n, j, p.lo) - p.lo;
        p.rest = j == 0 || j == n.B + 1;
        p.seq = j - 1;
        p.batch = 0;
        segment = p.slot - packed_slot(g, p.lo, j);
    } else {
        const int64_t segments = (n.T + g.length - 1) / g.length;
        p.seq = (int)(p.slot / segments);
        p.batch = p.seq;
        segment = p.slot % segments;
        p.lo = 0;
        p.len = n.T;
        p.rest = false;
    }
    const int64_t segments = p.len <= g.length ? 1 : (p.len + g.length - 1) / g.length;
    p.none = segment < 0 || segment >= segments;    // (below zero: starts that decrease, whose places are in no order)
    if (reverse && !p.none && !p.rest) {
        p.slot += segments - 1 - 2 * segment;
        segment = segments - 1 - segment;
    }
    p.first = segment * g.length;
    p.last = p.first + g.length < p.len ? p.first + g.length : p.len;
    p.alone = p.len <= g.length;
    p.ends = p.last >= p.len;
    return p;
}

// An entry of `first` or `last`, or null: not given, or out of range
__device__ __forceinline__ float* entry_of(const AttentionState& st, const AttentionSum& s, const AttentionBatch& n, int seq, int head)
{
    if (!st.p) return nullptr;
    const int entry = s.first_slots ? s.first_slots[seq] : seq;
    if (s.first_slots && (entry < 0 || entry >= n.n_states)) return nullptr;
    return st.p + entry * st.entry + head * st.head;
}

// An accumulator tile is 16 x 16: a lane has column lane % 16, rows 4 (lane / 16) ... + 3.

// f(tile, element, offset) for the elements of a column of a lane that lie within DA rows: offset, their row's place in memory.  (Rows are
// counted from the lane's own first one: what is added for an element is the same in all lanes.)
template <int MT, class F>
__device__ __forceinline__ void each_row(int DA, int64_t row_stride, F&& f)
{
    const int own = 4 * (threadIdx.x % 64 / 16);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (16 * m + 16 <= DA) {
#pragma unroll
            for (int e = 0; e < 4; ++e) f(m, e, own * row_stride + (16 * m + e) * row_stride);
        } else if (16 * m < DA) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (16 * m + own + e < DA) f(m, e, own * row_stride + (16 * m + e) * row_stride);
        }
    }
}

// The state before a segment into the accumulators of the columns `col` and 16 further each.
template <int MT, int CT>
__device__ __forceinline__ void load_state(f32x4 (&S)[MT][CT], const AttentionSum& s, const AttentionBatch& n, const Place& at, int head, int col)
{
    const float* p;
    int64_t row_stride, col_stride;
    if (at.alone) {
        p = entry_of(s.first, s, n, at.seq, head);
        row_stride = s.first.row, col_stride = s.first.col;
    } else {
        p = s.states + (at.slot * n.H + head) * s.DA * s.DC;
        row_stride = s.turned ? 1 : s.DC, col_stride = s.turned ? s.DA : 1;
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
#pragma unroll
        for (int m = 0; m < MT; ++m) S[m][c] = 0.f;
        if (!p || col + 16 * c >= s.DC) continue;
        const float* own = p + (col + 16 * c) * col_stride;
        each_row<MT>(s.DA, row_stride, [&](int m, int e, int64_t offset) { S[m][c][e] = own[offset]; });
    }
}

template <int MT, int CT>
__device__ __forceinline__ void store_state(const f32x4 (&S)[MT][CT], float* p, int64_t row_stride, int64_t col_stride, const AttentionSum& s, int col)
{
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        if (col + 16 * c >= s.DC) continue;
        float* own = p + (col + 16 * c) * col_stride;
        each_row<MT>(s.DA, row_stride, [&](int m, int e, int64_t offset) { own[offset] = S[m][c][e]; });
    }
}

// Zeros in `width` columns from col0 of the rows of a place in no sequence.
template <class T>
__device__ __forceinline__ void zero_rows(const AttentionSum& s, const Place& at, int head, int col0, int width)
{
    const int64_t all = (at.last - at.first) * width;
    for (int64_t i = threadIdx.x; i < all; i += blockDim.x) {
        const int64_t to = at.batch * s.y.batch + (at.lo + at.first + i / width) * s.y.token + head / s.y.share * s.y.head + col0 + i % width;
        if (s.y_f32)
            const_cast<float*>(static_cast<const float*>(s.y.p))[to] = 0.f;
        else
            const_cast<T*>(static_cast<const T*>(s.y.p))[to] = (T)0.f;
    }
}

// Four neighbouring columns of one row, those below `width` of them.
template <class T>
__device__ __forceinline__ void store_four(T* p, f32x4 v, int width)
{
    typedef T vec __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(sizeof(T)))) loose {
        vec v;
    };
    const vec w = __builtin_convertvector(v, vec);
    if (width >= 4) {
        reinterpret_cast<loose*>(p)->v = w;
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < width) p[e] = w[e];
}

// Whether a wavefront's accumulators hold an infinity or a NaN anywhere.
template <int N, int CT>
__device__ __forceinline__ bool any_nonfinite(const f32x4 (&v)[N][CT])
{
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fmaf(v[i][c][e], 0.f, sum);
    return __any(sum != 0.f);
}

// The recurrence itself, straight from memory: what a wavefront does once more with a segment that has an infinity or a NaN about.  In the
// products of whole chunks these reach the tokens before theirs, as zero times infinity.  It is rare, and the state lies in (private)
// memory so that nothing here takes registers from the loop it stands behind.  The operands' row 0 is the segment's first token.
template <class T>
struct TokenByToken {
    const T *a, *b, *c;                 // c: at the lane's column; a: null without outputs
    int64_t step_a, step_b, step_c, step_y, tokens;
    int DA;
    float decay, alpha_s, alpha_y;
    bool reverse, y_f32, column;        // column: the lane's is one of c's and y's
    void* y;                            // at the lane's column
};
template <class T, int MT, int CT>
__device__ __forceinline__ void token_by_token(f32x4 (&S)[MT][CT], int tile, const TokenByToken<T>& p)
{
    const int own = 4 * (threadIdx.x % 64 / 16);
    float held[4 * MT];
#pragma unroll
    for (int i = 0; i < 4 * MT; ++i) held[i] = S[i / 4][tile][i % 4];
#pragma unroll 1
    for (int64_t t = 0; t < p.tokens; ++t) {
        const float c = p.column ? p.alpha_s * (float)p.c[t * p.step_c] : 0.f;
        float y = 0.f;
#pragma unroll 1
        for (int i = 0; i < 4 * MT; ++i) {
            const int d = i / 4 * 16 + own + i % 4;
            if (d >= p.DA) continue;
            const float v = fmaf((float)p.b[t * p.step_b + d], c, p.reverse ? held[i] : held[i] * p.decay);
            if (p.a) y = fmaf((float)p.a[t * p.step_a + d], v, y);
            held[i] = p.reverse ? v * p.decay : v;
        }
        if (!p.a) continue;
        y += __shfl_xor(y, 16, 64);
        y = p.alpha_y * (y + __shfl_xor(y, 32, 64));
        if (own || !p.column) continue;
        if (p.y_f32)
            static_cast<float*>(p.y)[t * p.step_y] = y;
        else
            static_cast<T*>(p.y)[t * p.step_y] = (T)y;
    }
#pragma unroll
    for (int i = 0; i < 4 * MT; ++i) S[i / 4][tile][i % 4] = held[i];
}

}  // namespace attention
}  // namespace swconv
