// The many-rows kernel of the attention over the paged cache, over all of it.
#include "cache_attn_tile.h"

namespace dr {

void launch_cache_attn_tile(const stream::Args& a, hipStream_t st) { launch_tile<stream::kAll>(a, st); }

}  // namespace dr
