// The streaming attention kernel for f16 queries, blocks of any number of tokens.
#include "kvx_attn_stream.h"

namespace kvx {

void launch_stream_f16_any(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  stream_dim<F16, false>(a, c, stream);
}

}  // namespace kvx
