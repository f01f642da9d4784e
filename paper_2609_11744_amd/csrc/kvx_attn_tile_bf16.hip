// The tiled attention kernel for bf16 queries.
#include "kvx_attn_tile.h"

namespace kvx {

void launch_tiles_bf16(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  tile_dim<Bf16>(a, c, stream);
}

}  // namespace kvx
