// torq_chunk_attention for head_dim up to 128.
#include "chunk_attention_body.h"

namespace torq {

void go_chunk_128(const ChunkArgs &a, int format, int bend, unsigned groups, hipStream_t stream) {
  go_chunk<128, 128>(a, format, bend, groups, stream);
}

}  // namespace torq
