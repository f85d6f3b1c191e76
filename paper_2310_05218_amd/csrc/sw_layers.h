// Declarations shared by the layer norm and linear attention translation units: element formats, the operands of the
// attention's sums, launchers (validated arguments in, the HIP error of the launch out).
#pragma once

#include "swconv_internal.h"

namespace swconv {

// ---- element formats (Elem): loads widen exactly, stores round once to nearest even -----------------------------------------
template <int EK>
struct ElemOf;
template <>
struct ElemOf<kElemF32> {
    typedef float type;
};
template <>
struct ElemOf<kElemBF16> {
    typedef __bf16 type;
};
template <>
struct ElemOf<kElemF16> {
    typedef _Float16 type;
};

// Runs f(std::integral_constant<int, EK>) for the format; what an unknown one would be is refused before.
template <class F>
hipError_t with_elem(int ek, F&& f)
{
    switch (ek) {
    case kElemF32: return f(std::integral_constant<int, kElemF32>());
    case kElemBF16: return f(std::integral_constant<int, kElemBF16>());
    default: return f(std::integral_constant<int, kElemF16>());
    }
}

// ---- vectors of 16 bytes at any element's address --------------------------------------------------------------------------------

template <int EK>
struct Row {
    typedef typename ElemOf<EK>::type T;
    static constexpr int VEC = 16 / sizeof(T);
    typedef T vec __attribute__((ext_vector_type(VEC)));
    typedef float floats __attribute__((ext_vector_type(VEC)));
    struct __attribute__((packed, aligned(sizeof(T)))) loose {
        vec v;
    };
    struct __attribute__((packed, aligned(4))) loose_floats {
        floats v;
    };
    // elements first ... first + VEC - 1 of C, zeros beyond
    static __device__ __forceinline__ vec load(const T* row, int first, int C)
    {
        if (first + VEC <= C) return reinterpret_cast<const loose*>(row + first)->v;
        vec v = {};
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (first + e < C) v[e] = row[first + e];
        return v;
    }
    static __device__ __forceinline__ void store(T* row, int first, int C, floats f)
    {
        const vec v = __builtin_convertvector(f, vec);
        if (first + VEC <= C) {
            reinterpret_cast<loose*>(row + first)->v = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (first + e < C) row[first + e] = v[e];
    }
    static __device__ __forceinline__ floats load_floats(const float* p, int first, int C, float without)
    {
        floats f = without;
        if (!p) return f;
        if (first + VEC <= C) return reinterpret_cast<const loose_floats*>(p + first)->v;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (first + e < C) f[e] = p[first + e];
        return f;
    }
    static __device__ __forceinline__ void store_floats(float* p, int first, int C, floats f)
    {
        if (first + VEC <= C) {
            reinterpret_cast<loose_floats*>(p + first)->v = f;
            return;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (first + e < C) p[first + e] = f[e];
    }
    // zeros in place of what is beyond the row
    static __device__ __forceinline__ floats within(floats f, int first, int C)
    {
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = first + e < C ? f[e] : 0.f;
        return f;
    }
    // VEC elements, all there
    static __device__ __forceinline__ vec load(const T* p) { return reinterpret_cast<const loose*>(p)->v; }
    static __device__ __forceinline__ void store(T* p, floats f) { reinterpret_cast<loose*>(p)->v = __builtin_convertvector(f, vec); }
    static __device__ __forceinline__ floats load_floats(const float* p) { return reinterpret_cast<const loose_floats*>(p)->v; }
    static __device__ __forceinline__ void store_floats(float* p, floats f) { reinterpret_cast<loose_floats*>(p)->v = f; }
    static __device__ __forceinline__ float sum(floats f)
    {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += f[e];
        return s;
    }
};

// ---- layer norm ------------------------------------------------------------------------------------------------------------
struct LayerNormArgs {
    const void* x;
    const float *weight, *bias;         // null: ones, zeros
    void* y;
    float *mean, *rstd;                 // null: not kept
    int64_t rows, x_stride, y_stride;
    int C;
    float eps;
};
hipError_t launch_layer_norm(const LayerNormArgs& a, int ek, hipStream_t st);

struct LayerNormBackwardArgs {
    const void *dy, *x;
    const float *weight, *mean, *rstd;  // weight null: ones
    void* dx;                           // null: not wanted
    float *dweight, *dbias;             // null: not wanted
    int64_t rows, dy_stride, x_stride, dx_stride;
    int C;
    float* partial;                     // layer_norm_backward_parts(rows, C) rows of 2 C sums
};
int        layer_norm_backward_parts(int64_t rows, int64_t C);
hipError_t launch_layer_norm_backward(const LayerNormBackwardArgs& a, int ek, hipStream_t st);

// ---- linear attention ----------------------------------------------------------------------------------------------------------
// Prompts and all three gradients are one sum over operands a, b (rows of DA) and c, y (rows of DC) with a state [DA, DC]:
//   forwards in time    S_t = l S_{t-1} + alpha_s b_t c_t^T,  y_t = alpha_y S_t^T a_t
//   backwards in time   G_t = R_{t+1} + alpha_s b_t c_t^T,    y_t = alpha_y G_t^T a_t,  R_t = l G_t
// o: (q, k, v) forwards; dq: (d_o, v, k) forwards on the transposed state; dk: (v, d_o, q) and dv: (k, q, d_o) backwards.
struct AttentionOperand {
    const void* p;
    int64_t batch, token, head;         // strides in elements
    int share;                          // neighbouring heads that have one row
};
struct AttentionState {                 // null: zeros before the first token, not kept after the last
    float* p;
    int64_t entry, head, row, col;      // strides in elements (row: along DA, col: along DC)
};
struct AttentionSum {
    AttentionOperand a, b, c, y;        // y: written; of the operands' format, or fp32 (y_f32)
    AttentionState first, last;         // first: only read
    const int32_t* first_slots;         // entry of a sequence in `first` and `last`; null: its number
    int DA, DC;
    float alpha_s, alpha_y;
    bool reverse, y_f32;
    float* states = nullptr;            // [segments, H, DA, DC]: the state before each segment
    bool turned = false;                // ... of the sum with a's and c's widths exchanged: [segments, H, DC, DA]
};
struct AttentionSums {                  // that are worked on side by side
    AttentionSum of[3];
    int count;
};
struct AttentionBatch {
    const float* log_decay;
    const int32_t* starts;              // packed sequences: [B + 1]; null: B sequences of T rows
    int64_t T;
    int B, H, n_states;
};
// A long sequence is cut into segments of `length` tokens (a multiple of the chunk) that are worked on side by side: their own sums first
// (attention_states), the state before each from these (attention_scan), then the outputs (attention_chunks).  A length of 2^62: whole sequences.
struct AttentionSegments {
    int64_t length, count;              // count: places for segments in all
};
constexpr int kAttentionChunk = 64;
AttentionSegments attention_segments(const AttentionBatch& n, int DA, int DC, bool packed, int ek);
// a segment's own sum for all but the last of a sequence, into `states`
hipError_t launch_attention_states(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, int ek, hipStream_t st);
// ... from which the state before each segment of a sequence that has several
hipError_t launch_attention_scan(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st);
// the outputs and last states
hipError_t launch_attention_chunks(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, int ek, hipStream_t st);
hipError_t launch_attention_recurrent(const AttentionSum& s, const AttentionBatch& n, int ek, hipStream_t st);
// y[row, u] = sum over the heads of group u of part[row, head], rows of D fp32 each (16-byte aligned), rounded to the format
struct AttentionFold {
    const float* part;
    AttentionOperand y;
    int D;
};
hipError_t launch_attention_fold(const AttentionFold& dk, const AttentionFold& dv, const AttentionBatch& n, int ek, hipStream_t st);

struct AttentionStepArgs {
    AttentionOperand q, k, v, o;
    float* state;
    const float* log_decay;
    const int32_t* slots;
    int B, H, DK, DV, n_states;
    float scale;
};
hipError_t launch_attention_step(const AttentionStepArgs& a, int ek, hipStream_t st);

}  // namespace swconv
