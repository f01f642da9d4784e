// The streaming attention kernel for f16 queries, blocks of whole runs of 16 tokens.
#include "kvx_attn_stream.h"

namespace kvx {

void launch_stream_f16(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  stream_dim<F16, true>(a, c, stream);
}

}  // namespace kvx
