// The streaming attention kernel for bf16 queries, blocks of any number of tokens.
#include "kvx_attn_stream.h"

namespace kvx {

void launch_stream_bf16_any(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  stream_dim<Bf16, false>(a, c, stream);
}

}  // namespace kvx
