// The tiled attention kernel for f16 queries.
#include "kvx_attn_tile.h"

namespace kvx {

void launch_tiles_f16(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  tile_dim<F16>(a, c, stream);
}

}  // namespace kvx
