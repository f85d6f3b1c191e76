// What the C entry points of the sequence operators share on the host: extents, alignment, overlaps, workspaces.
#pragma once

#include <cmath>
#include <initializer_list>

#include "sw_layers.h"

namespace {

using namespace swconv;

constexpr int64_t kMaxExtent = (int64_t)1 << 46;    // elements from a tensor's first to its last: offsets in bytes stay within int64
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

}  // namespace
