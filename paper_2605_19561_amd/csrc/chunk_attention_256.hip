// torq_chunk_attention for head_dim over 128.  Compiled apart: O and Q take 192 registers of a lane, and O lies in the accumulators' half of them (the
// other kernels' results of products lie in ordinary ones).
#include "chunk_attention_body.h"

namespace torq {

void go_chunk_256(const ChunkArgs &a, int format, bool bent, unsigned groups, hipStream_t stream) { go_chunk<256>(a, format, bent, groups, stream); }

}  // namespace torq
