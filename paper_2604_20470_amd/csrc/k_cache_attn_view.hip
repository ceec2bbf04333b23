// The many-rows kernel of the attention over the paged cache, over a window of it, and over all of it with partial sums as the results.
#include "cache_attn_tile.h"

namespace dr {

void launch_cache_attn_tile_view(const stream::Args& a, bool window, hipStream_t st) {
    if (window) launch_tile<stream::kWindow>(a, st);
    else launch_tile<stream::kParts>(a, st);
}

}  // namespace dr
