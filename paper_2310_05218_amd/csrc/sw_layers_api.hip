// C entry points of layer norm and linear attention: host-side validation, then the launchers.  Every argument error is reported
// before anything is enqueued; scratch memory is the caller's.
#include "../../include/swconv.h"

#include <cmath>
#include <initializer_list>

#include "sw_layers.h"

using namespace swconv;

static_assert((int)SW_F32 == (int)kElemF32 && (int)SW_BF16 == (int)kElemBF16 && (int)SW_F16 == (int)kElemF16, "the formats' numbers");

namespace {

constexpr int64_t kMaxExtent = (int64_t)1 << 46;    // elements from a tensor's first to its last: offsets in bytes stay within int64
constexpr int kMaxHead = 256;
constexpr int kMaxChannels = 1 << 20;

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }

int launch_status(hipError_t e) { return e == hipSuccess ? SW_OK : SW_ERR_LAUNCH; }

// The memory from a tensor's first to its last element.
struct Span {
    uintptr_t at = 0;
    int64_t bytes = 0;
};
bool meet(const Span& a, const Span& b) { return a.bytes && b.bytes && a.at < b.at + (uintptr_t)b.bytes && b.at < a.at + (uintptr_t)a.bytes; }
Span span_of(const void* p, int64_t elements, int64_t size) { return Span{reinterpret_cast<uintptr_t>(p), p ? elements * size : 0}; }

int64_t align16(int64_t n) { return (n + 15) / 16 * 16; }

// rows of `width` elements, `stride` apart
bool row_extent(int64_t rows, int64_t width, int64_t stride, int64_t* elements)
{
    if (stride < width || stride > kMaxExtent || rows > kMaxExtent / stride) return false;
    *elements = (rows - 1) * stride + width;
    return true;
}

bool workspace_fits(const void* p, int64_t bytes, int64_t need) { return need == 0 || (p && bytes >= need && !misaligned(p, 16)); }

// [batch, token, heads, width] with strides; false: extents beyond what offsets hold, or, of a tensor that is written, rows that
// overlap.  Dimensions of one element have no stride.
struct Tensor4 {
    int64_t elements = 0;
    AttentionOperand op{nullptr, 0, 0, 0, 1};
    bool set(const void* p, const sw_strides* s, int64_t batches, int64_t tokens, int heads, int width, int share, bool written = false)
    {
        const int64_t count[3] = {batches, tokens, heads};
        int64_t stride[3] = {s->batch, s->token, s->head};
        elements = width;
        for (int i = 0; i < 3; ++i) {
            if (count[i] == 1) stride[i] = 0;
            if (stride[i] < 0 || (count[i] > 1 && stride[i] > kMaxExtent / (count[i] - 1))) return false;
            elements += stride[i] * (count[i] - 1);
            if (elements > kMaxExtent) return false;
        }
        op = AttentionOperand{p, stride[0], stride[1], stride[2], share};
        if (!written) return true;
        // from the narrowest stride to the widest, each is past all that the ones before it reach
        int order[3] = {0, 1, 2};
        for (int i = 1; i < 3; ++i)
            for (int j = i; j > 0 && stride[order[j]] < stride[order[j - 1]]; --j) {
                const int t = order[j];
                order[j] = order[j - 1], order[j - 1] = t;
            }
        int64_t reach = width;
        for (int i : order) {
            if (count[i] == 1) continue;
            if (stride[i] < reach) return false;
            reach += stride[i] * (count[i] - 1);
        }
        return true;
    }
};

// Extents that every attention call shares.
int check_dims(const sw_linear_attention_dims& d)
{
    if (d.T <= 0 || d.B <= 0 || d.heads <= 0 || d.kv_heads <= 0 || d.dk <= 0 || d.dv <= 0 || d.heads % d.kv_heads != 0 || d.n_states < 0 ||
        !std::isfinite(d.scale))
        return SW_ERR_SHAPE;
    if (d.T > kMaxExtent / d.B || (int64_t)d.B + 2 > 0x7fffffff) return SW_ERR_SHAPE;
    if (d.dk > kMaxHead || d.dv > kMaxHead || d.heads > 65535) return SW_ERR_UNSUPPORTED;
    if (d.type != SW_F32 && d.type != SW_BF16 && d.type != SW_F16) return SW_ERR_UNSUPPORTED;
    return SW_OK;
}

// Packed rows are counted in 32 bits by `starts`.
bool packed_too_long(const sw_linear_attention_dims& d, const int32_t* starts) { return starts && d.T > 0x7fffffff; }

AttentionSegments segments_of(const sw_linear_attention_dims& d, bool packed)
{
    return attention_segments(AttentionBatch{nullptr, nullptr, d.T, d.B, d.heads, d.n_states}, d.dk, d.dv, packed, d.type);
}

// The same of calls that work on `sums` at a time: a launch has fewer than 2^32 threads, 256 for every segment's place, head and sum.  (Heads' rows
// beyond a tensor's extent are refused before bytes are counted from them.)
int check_sums(const sw_linear_attention_dims& d, bool packed, int sums)
{
    if (const int rc = check_dims(d)) return rc;
    if (d.T * (packed ? 1 : d.B) > kMaxExtent / ((int64_t)d.heads * (d.dk > d.dv ? d.dk : d.dv))) return SW_ERR_SHAPE;
    return segments_of(d, packed).count > ((1 << 24) - 1) / ((int64_t)d.heads * sums) ? SW_ERR_SHAPE : SW_OK;
}

// Whether the chunk kernels' 32-bit distances within a chunk reach its rows; tensors that lie further apart go token by token.
bool near_rows(std::initializer_list<const Tensor4*> tensors)
{
    for (const Tensor4* t : tensors)
        if (t->op.token > ((int64_t)1 << 30) / kAttentionChunk) return false;
    return true;
}

// Bytes of the segments' states (0: whole sequences).
int64_t state_bytes(const sw_linear_attention_dims& d, bool packed)
{
    const AttentionSegments g = segments_of(d, packed);
    return g.length > d.T ? 0 : align16(g.count * d.heads * d.dk * d.dv * 4);
}

// Bytes of the fp32 rows of dk and of dv that heads sharing them are added from (0: not shared).
int64_t fold_bytes(const sw_linear_attention_dims& d, bool packed, int width)
{
    return d.heads == d.kv_heads ? 0 : align16(4 * d.T * (packed ? 1 : d.B) * d.heads * width);
}

}  // namespace

extern "C" {

int sw_layer_norm(const void* x, const float* weight, const float* bias, void* y, float* mean, float* rstd, int64_t rows, int64_t C,
                  int64_t x_stride, int64_t y_stride, float eps, int type, void* hip_stream)
{
    if (!x || !y) return SW_ERR_NULL;
    int64_t nx, ny;
    if (rows <= 0 || C <= 0 || !(eps >= 0.f) || !std::isfinite(eps) || !row_extent(rows, C, x_stride, &nx) || !row_extent(rows, C, y_stride, &ny))
        return SW_ERR_SHAPE;
    if (C > kMaxChannels || (type != SW_F32 && type != SW_BF16 && type != SW_F16)) return SW_ERR_UNSUPPORTED;
    const int size = elem_size(type);
    if (misaligned(x, size) || misaligned(y, size) || misaligned(weight, 4) || misaligned(bias, 4) || misaligned(mean, 4) || misaligned(rstd, 4))
        return SW_ERR_ALIGN;
    const Span in[3] = {span_of(x, nx, size), span_of(weight, C, 4), span_of(bias, C, 4)};
    const Span out[3] = {span_of(y, ny, size), span_of(mean, rows, 4), span_of(rstd, rows, 4)};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 3; ++i)
            if (meet(out[o], in[i]) && !(o == 0 && i == 0 && x == y && x_stride == y_stride)) return SW_ERR_ALIAS;
        for (int p = 0; p < o; ++p)
            if (meet(out[o], out[p])) return SW_ERR_ALIAS;
    }
    const LayerNormArgs a{x, weight, bias, y, mean, rstd, rows, x_stride, y_stride, (int)C, eps};
    return launch_status(launch_layer_norm(a, type, static_cast<hipStream_t>(hip_stream)));
}

int64_t sw_layer_norm_backward_workspace_bytes(int64_t rows, int64_t C)
{
    if (rows <= 0 || C <= 0 || C > kMaxChannels) return 0;
    return align16((int64_t)layer_norm_backward_parts(rows, C) * 2 * C * 4);
}

int sw_layer_norm_backward(const void* dy, const void* x, const float* weight, const float* mean, const float* rstd, void* dx, float* dweight,
                           float* dbias, int64_t rows, int64_t C, int64_t dy_stride, int64_t x_stride, int64_t dx_stride, int type,
                           void* workspace, int64_t workspace_bytes, void* hip_stream)
{
    if (!dy || !x || !mean || !rstd || (!dx && !dweight && !dbias)) return SW_ERR_NULL;
    int64_t ndy, nx, ndx = 0;
    if (rows <= 0 || C <= 0 || !row_extent(rows, C, dy_stride, &ndy) || !row_extent(rows, C, x_stride, &nx) ||
        (dx && !row_extent(rows, C, dx_stride, &ndx)))
        return SW_ERR_SHAPE;
    if (C > kMaxChannels || (type != SW_F32 && type != SW_BF16 && type != SW_F16)) return SW_ERR_UNSUPPORTED;
    const int size = elem_size(type);
    if (misaligned(dy, size) || misaligned(x, size) || misaligned(dx, size) || misaligned(weight, 4) || misaligned(mean, 4) ||
        misaligned(rstd, 4) || misaligned(dweight, 4) || misaligned(dbias, 4))
        return SW_ERR_ALIGN;
    const int64_t need = dweight || dbias ? sw_layer_norm_backward_workspace_bytes(rows, C) : 0;
    if (!workspace_fits(workspace, workspace_bytes, need)) return SW_ERR_WORKSPACE;
    const Span in[5] = {span_of(dy, ndy, size), span_of(x, nx, size), span_of(weight, C, 4), span_of(mean, rows, 4), span_of(rstd, rows, 4)};
    const Span out[4] = {span_of(dx, ndx, size), span_of(dweight, C, 4), span_of(dbias, C, 4), span_of(workspace, need, 1)};
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 5; ++i) {
            const bool same = o == 0 && ((i == 0 && dx == dy && dx_stride == dy_stride) || (i == 1 && dx == x && dx_stride == x_stride));
            if (meet(out[o], in[i]) && !same) return SW_ERR_ALIAS;
        }
        for (int p = 0; p < o; ++p)
            if (meet(out[o], out[p])) return SW_ERR_ALIAS;
    }
    const LayerNormBackwardArgs a{dy, x, weight, mean, rstd, dx, dweight, dbias, rows, dy_stride, x_stride, dx_stride, (int)C,
                                  static_cast<float*>(workspace)};
    return launch_status(launch_layer_norm_backward(a, type, static_cast<hipStream_t>(hip_stream)));
}

int64_t sw_linear_attention_workspace_bytes(const sw_linear_attention_dims* dims, int packed)
{
    if (!dims || check_sums(*dims, packed != 0, 1) != SW_OK) return 0;
    return state_bytes(*dims, packed != 0);
}

int sw_linear_attention(const void* q, const void* k, const void* v, void* o, const float* log_decay, const float* state, float* final_state,
                        const int32_t* slots, const int32_t* starts, const sw_linear_attention_dims* dims, const sw_strides* q_strides,
                        const sw_strides* k_strides, const sw_strides* v_strides, const sw_strides* o_strides, void* workspace,
                        int64_t workspace_bytes, void* hip_stream)
{
    if (!q || !k || !v || !o || !log_decay || !dims || !q_strides || !k_strides || !v_strides || !o_strides) return SW_ERR_NULL;
    const sw_linear_attention_dims d = *dims;
    if (const int rc = check_sums(d, starts != nullptr, 1)) return rc;
    const int64_t batches = starts ? 1 : d.B;
    const int share = d.heads / d.kv_heads;
    Tensor4 tq, tk, tv, to;
    if (!tq.set(q, q_strides, batches, d.T, d.heads, d.dk, 1) || !tk.set(k, k_strides, batches, d.T, d.kv_heads, d.dk, share) ||
        !tv.set(v, v_strides, batches, d.T, d.kv_heads, d.dv, share) || !to.set(o, o_strides, batches, d.T, d.heads, d.dv, 1, true) ||
        packed_too_long(d, starts) || ((state || final_state) && (d.n_states <= 0 || (!slots && d.n_states < d.B))))
        return SW_ERR_SHAPE;
    const int size = elem_size(d.type);
    if (misaligned(q, size) || misaligned(k, size) || misaligned(v, size) || misaligned(o, size) || misaligned(log_decay, 4) ||
        misaligned(state, 4) || misaligned(final_state, 4) || misaligned(slots, 4) || misaligned(starts, 4))
        return SW_ERR_ALIGN;
    const int64_t per_head = (int64_t)d.dk * d.dv, states = per_head * d.heads;
    if (states > kMaxExtent / ((int64_t)d.n_states + 1)) return SW_ERR_SHAPE;
    const int64_t need = sw_linear_attention_workspace_bytes(dims, starts != nullptr);
    if (!workspace_fits(workspace, workspace_bytes, need)) return SW_ERR_WORKSPACE;
    const Span in[7] = {span_of(q, tq.elements, size), span_of(k, tk.elements, size), span_of(v, tv.elements, size), span_of(log_decay, d.heads, 4),
                        span_of(state, states * d.n_states, 4), span_of(slots, d.B, 4), span_of(starts, d.B + 1, 4)};
    const Span out[3] = {span_of(o, to.elements, size), span_of(final_state, states * d.n_states, 4), span_of(workspace, need, 1)};
    for (int p = 0; p < 3; ++p) {
        for (int i = 0; i < 7; ++i)
            if (meet(out[p], in[i]) && !(p == 1 && i == 4 && state == final_state)) return SW_ERR_ALIAS;
        for (int r = 0; r < p; ++r)
            if (meet(out[p], out[r])) return SW_ERR_ALIAS;
    }
    const AttentionState first{const_cast<float*>(state), states, per_head, d.dv, 1}, last{final_state, states, per_head, d.dv, 1};
    AttentionSums s;
    s.count = 1;
    s.of[0] = AttentionSum{tq.op, tk.op, tv.op, to.op, first, last, slots, d.dk, d.dv, 1.0f, d.scale, false, false, static_cast<float*>(workspace)};
    const AttentionBatch n{log_decay, starts, d.T, d.B, d.heads, d.n_states};
    const AttentionSegments g = segments_of(d, starts != nullptr);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (!near_rows({&tq, &tk, &tv, &to})) return launch_status(launch_attention_recurrent(s.of[0], n, d.type, st));
    hipError_t e = hipSuccess;
    if (need) e = launch_attention_states(s, n, g, d.type, st);
    if (need && e == hipSuccess) e = launch_attention_scan(s, n, g, st);
    if (e == hipSuccess) e = launch_attention_chunks(s, n, g, d.type, st);
    return launch_status(e);
}

int64_t sw_linear_attention_backward_workspace_bytes(const sw_linear_attention_dims* dims, int packed)
{
    if (!dims || check_sums(*dims, packed != 0, 3) != SW_OK) return 0;
    return fold_bytes(*dims, packed != 0, dims->dk) + fold_bytes(*dims, packed != 0, dims->dv) + 2 * state_bytes(*dims, packed != 0);
}

int sw_linear_attention_backward(const void* d_o, const void* q, const void* k, const void* v, const float* log_decay, const float* state,
                                 const float* d_final_state, void* dq, void* dk, void* dv, float* d_state, const int32_t* slots,
                                 const int32_t* starts, const sw_linear_attention_dims* dims, const sw_strides* do_strides,
                                 const sw_strides* q_strides, const sw_strides* k_strides, const sw_strides* v_strides,
                                 const sw_strides* dq_strides, const sw_strides* dk_strides, const sw_strides* dv_strides, void* workspace,
                                 int64_t workspace_bytes, void* hip_stream)
{
    if (!d_o || !q || !k || !v || !log_decay || !dq || !dk || !dv || !dims || !do_strides || !q_strides || !k_strides || !v_strides ||
        !dq_strides || !dk_strides || !dv_strides)
        return SW_ERR_NULL;
    const sw_linear_attention_dims d = *dims;
    if (const int rc = check_sums(d, starts != nullptr, 3)) return rc;
    const int64_t batches = starts ? 1 : d.B;
    const int share = d.heads / d.kv_heads;
    Tensor4 tdo, tq, tk, tv, tdq, tdk, tdv;
    if (!tdo.set(d_o, do_strides, batches, d.T, d.heads, d.dv, 1) || !tq.set(q, q_strides, batches, d.T, d.heads, d.dk, 1) ||
        !tk.set(k, k_strides, batches, d.T, d.kv_heads, d.dk, share) || !tv.set(v, v_strides, batches, d.T, d.kv_heads, d.dv, share) ||
        !tdq.set(dq, dq_strides, batches, d.T, d.heads, d.dk, 1, true) || !tdk.set(dk, dk_strides, batches, d.T, d.kv_heads, d.dk, share, true) ||
        !tdv.set(dv, dv_strides, batches, d.T, d.kv_heads, d.dv, share, true) || packed_too_long(d, starts) ||
        (state && (d.n_states <= 0 || (!slots && d.n_states < d.B))))
        return SW_ERR_SHAPE;
    const int size = elem_size(d.type);
    for (const void* p : {d_o, q, k, v, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv)})
        if (misaligned(p, size)) return SW_ERR_ALIGN;
    if (misaligned(log_decay, 4) || misaligned(state, 4) || misaligned(d_final_state, 4) || misaligned(d_state, 4) || misaligned(slots, 4) ||
        misaligned(starts, 4))
        return SW_ERR_ALIGN;
    const int64_t per_head = (int64_t)d.dk * d.dv, states = per_head * d.heads;
    if (states > kMaxExtent / ((int64_t)d.n_states + 1) || states > kMaxExtent / d.B) return SW_ERR_SHAPE;
    const int64_t need = sw_linear_attention_backward_workspace_bytes(dims, starts != nullptr);
    if (!workspace_fits(workspace, workspace_bytes, need)) return SW_ERR_WORKSPACE;
    const Span in[9] = {span_of(d_o, tdo.elements, size), span_of(q, tq.elements, size), span_of(k, tk.elements, size),
                        span_of(v, tv.elements, size), span_of(log_decay, d.heads, 4), span_of(state, states * d.n_states, 4),
                        span_of(d_final_state, states * d.B, 4), span_of(slots, d.B, 4), span_of(starts, d.B + 1, 4)};
    // (gradients may lie interleaved in one tensor, as q, k and v may: their spans are not held against each other, but no two begin together)
    const Span out[5] = {span_of(dq, tdq.elements, size), span_of(dk, tdk.elements, size), span_of(dv, tdv.elements, size),
                         span_of(d_state, states * d.B, 4), span_of(workspace, need, 1)};
    for (int p = 0; p < 5; ++p) {
        for (int i = 0; i < 9; ++i)
            if (meet(out[p], in[i]) && !(p == 3 && i == 6 && d_state == d_final_state)) return SW_ERR_ALIAS;
        for (int r = 0; r < p; ++r)
            if (p >= 3 ? meet(out[p], out[r]) : out[p].at == out[r].at) return SW_ERR_ALIAS;
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const AttentionBatch n{log_decay, starts, d.T, d.B, d.heads, d.n_states};
    const AttentionState none{nullptr, 0, 0, 0, 0}, turned{const_cast<float*>(state), states, per_head, 1, d.dv},
        turned_final{const_cast<float*>(d_final_state), states, per_head, 1, d.dv}, first{const_cast<float*>(d_final_state), states, per_head, d.dv, 1},
        last{d_state, states, per_head, d.dv, 1};
    // where heads share rows of k and v their gradients are added from fp32 rows of each head
    float *part_k = static_cast<float*>(workspace), *part_v = part_k + fold_bytes(d, starts != nullptr, d.dk) / 4;
    auto part = [&](float* p, int width) { return AttentionOperand{p, d.T * d.heads * width, (int64_t)d.heads * width, width, 1}; };
    // the states before each segment, forwards (those of the forward call) and backwards in time
    const int64_t bytes = state_bytes(d, starts != nullptr);
    float *ahead = part_v + fold_bytes(d, starts != nullptr, d.dv) / 4, *back = ahead + bytes / 4;
    const AttentionSum of_q{tdo.op, tv.op, tk.op, tdq.op, turned, none, slots, d.dv, d.dk, 1.0f, d.scale, false, false, ahead, true};
    const AttentionSum of_k{tv.op, tdo.op, tq.op, share > 1 ? part(part_k, d.dk) : tdk.op, turned_final, none, nullptr, d.dv, d.dk, d.scale, 1.0f, true,
                            share > 1, back, true};
    const AttentionSum of_v{tk.op, tq.op, tdo.op, share > 1 ? part(part_v, d.dv) : tdv.op, first, last, nullptr, d.dk, d.dv, d.scale, 1.0f, true,
                            share > 1, back, false};
    const AttentionSums gradients{{of_q, of_k, of_v}, 3}, of_q_and_k{{of_q, of_k, of_k}, 2}, of_v_alone{{of_v, of_v, of_v}, 1};
    const AttentionSegments g = segments_of(d, starts != nullptr);
    hipError_t e = hipSuccess;
    if (near_rows({&tdo, &tq, &tk, &tv, &tdq, &tdk, &tdv})) {
        if (bytes) {
            const AttentionSum forward{tq.op, tk.op, tv.op, tdo.op, {const_cast<float*>(state), states, per_head, d.dv, 1}, none, slots, d.dk, d.dv, 1.0f,
                                       d.scale, false, false, ahead, false};
            const AttentionSums both{{forward, of_v, of_v}, 2};
            e = launch_attention_states(both, n, g, d.type, st);
            if (e == hipSuccess) e = launch_attention_scan(both, n, g, st);
        }
        // (where d_state replaces d_final_state, all of dk's sum has read it before dv's, which writes it, begins: workgroups of one launch have no order)
        const bool in_place = d_state && d_state == d_final_state;
        if (e == hipSuccess) e = launch_attention_chunks(in_place ? of_q_and_k : gradients, n, g, d.type, st);
        if (e == hipSuccess && in_place) e = launch_attention_chunks(of_v_alone, n, g, d.type, st);
    } else {
        // (dv's last, for the same reason)
        for (int i = 0; i < 3 && e == hipSuccess; ++i) e = launch_attention_recurrent(gradients.of[i], n, d.type, st);
    }
    if (e == hipSuccess && share > 1) e = launch_attention_fold(AttentionFold{part_k, tdk.op, d.dk}, AttentionFold{part_v, tdv.op, d.dv}, n, d.type, st);
    return launch_status(e);
}

int sw_linear_attention_step(const void* q, const void* k, const void* v, void* o, const float* log_decay, float* state, const int32_t* slots,
                             const sw_linear_attention_dims* dims, const sw_strides* q_strides, const sw_strides* k_strides,
                             const sw_strides* v_strides, const sw_strides* o_strides, void* hip_stream)
{
    if (!q || !k || !v || !o || !log_decay || !state || !dims || !q_strides || !k_strides || !v_strides || !o_strides) return SW_ERR_NULL;
    const sw_linear_attention_dims d = *dims;
    if (const int rc = check_dims(d)) return rc;
    const int share = d.heads / d.kv_heads;
    Tensor4 tq, tk, tv, to;
    if (d.T != 1 || d.B >= 1 << 24 || !tq.set(q, q_strides, d.B, 1, d.heads, d.dk, 1) || !tk.set(k, k_strides, d.B, 1, d.kv_heads, d.dk, share) ||
        !tv.set(v, v_strides, d.B, 1, d.kv_heads, d.dv, share) || !to.set(o, o_strides, d.B, 1, d.heads, d.dv, 1, true) || d.n_states <= 0 ||
        (!slots && d.n_states < d.B))
        return SW_ERR_SHAPE;
    const int size = elem_size(d.type);
    if (misaligned(q, size) || misaligned(k, size) || misaligned(v, size) || misaligned(o, size) || misaligned(log_decay, 4) ||
        misaligned(state, 16) || misaligned(slots, 4))
        return SW_ERR_ALIGN;
    const int64_t states = (int64_t)d.dk * d.dv * d.heads;
    if (states > kMaxExtent / d.n_states) return SW_ERR_SHAPE;
    const Span in[5] = {span_of(q, tq.elements, size), span_of(k, tk.elements, size), span_of(v, tv.elements, size), span_of(log_decay, d.heads, 4),
                        span_of(slots, d.B, 4)};
    const Span out[2] = {span_of(o, to.elements, size), span_of(state, states * d.n_states, 4)};
    for (const Span& p : out)
        for (const Span& i : in)
            if (meet(p, i)) return SW_ERR_ALIAS;
    if (meet(out[0], out[1])) return SW_ERR_ALIAS;
    const AttentionStepArgs a{tq.op, tk.op, tv.op, to.op, state, log_decay, slots, d.B, d.heads, d.dk, d.dv, d.n_states, d.scale};
    return launch_status(launch_attention_step(a, d.type, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
