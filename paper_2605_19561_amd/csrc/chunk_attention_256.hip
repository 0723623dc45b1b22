// torq_chunk_attention for head_dim up to 256.
#include "chunk_attention_body.h"

namespace torq {

void go_chunk_256(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream) {
  go_chunk<256, 256>(a, format, bend, groups, stream);
}

}  // namespace torq
