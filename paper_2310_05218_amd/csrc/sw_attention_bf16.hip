// Linear attention in chunks: the kernels of bf16 operands.
#include "sw_attention_chunk.h"

namespace swconv {

hipError_t launch_attention_states_bf16(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st)
{
    return launch_chunk<kElemBF16, false>(s, n, g, st);
}

hipError_t launch_attention_chunks_bf16(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st)
{
    return launch_chunk<kElemBF16, true>(s, n, g, st);
}

}  // namespace swconv
