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
};
struct AttentionBatch {
    const float* log_decay;
    const int32_t* starts;              // packed sequences: [B + 1]; null: B sequences of T rows
    int64_t T;
    int B, H, n_states;
};
hipError_t launch_attention_recurrent(const AttentionSum& s, const AttentionBatch& n, int ek, hipStream_t st);
// y[row, u] = sum over the heads of group u of part[row, head], rows of D fp32 each, rounded to the format
hipError_t launch_attention_fold(const float* part, const AttentionOperand& y, const AttentionBatch& n, int kv_heads, int D, int ek, hipStream_t st);

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
