// Linear attention in chunks: the kernels of fp32 operands.
#include "sw_attention_chunk.h"

namespace swconv {

hipError_t launch_attention_states_f32(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st)
{
    return launch_chunk<kElemF32, false>(s, n, g, st);
}

hipError_t launch_attention_chunks_f32(const AttentionSums& s, const AttentionBatch& n, const AttentionSegments& g, hipStream_t st)
{
    return launch_chunk<kElemF32, true>(s, n, g, st);
}

}  // namespace swconv
