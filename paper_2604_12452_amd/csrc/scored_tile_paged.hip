// Scored attention of chunks of prompts over the paged 8-bit cache on the matrix cores (scored_tile.h).
#include "scored_tile.h"

namespace lca {

hipError_t launch_scored_tile_paged(const ScoredArgs &a, int least, hipStream_t st) { return launch<true>(a, least, st); }

}  // namespace lca
