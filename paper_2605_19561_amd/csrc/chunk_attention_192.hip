// torq_chunk_attention for head_dim up to 192.
#include "chunk_attention_body.h"

namespace torq {

void go_chunk_192(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream) {
  go_chunk<256, 192>(a, format, bend, groups, stream);
}

}  // namespace torq
