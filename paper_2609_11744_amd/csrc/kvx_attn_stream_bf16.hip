// The streaming attention kernel for bf16 queries, blocks of whole runs of 16 tokens.
#include "kvx_attn_stream.h"

namespace kvx {

void launch_stream_bf16(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  stream_dim<Bf16, true>(a, c, stream);
}

}  // namespace kvx
