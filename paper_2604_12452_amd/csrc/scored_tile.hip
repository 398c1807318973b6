// Scored attention of packed prompts on the matrix cores (scored_tile.h).
#include "scored_tile.h"

namespace lca {

bool scored_tile_supported(const ServeDims &d)
{
    // (64 rows of a tile lie within the 2^31 bytes of a buffer descriptor)
    return d.dtype != LCA_F32 && d.d_sel <= 256 && d.d_pool <= 256 && d.sel_row < (1u << 23) && d.pool_row < (1u << 23);
}

size_t scored_tile_workspace_bytes(const ServeDims &d, bool paged)
{
    const Plan p = make_plan(d, paged);
    const int dv = CLASS_DV[width_class(d.d_sel, d.d_pool)];
    return p.parts > 1 ? (size_t)((long)d.T * d.hps / SLOT + 1) * d.S * p.parts * 32 * wavefronts(paged, dv) * (dv + 2) * sizeof(float) : 0;
}

hipError_t launch_scored_tile(const ScoredArgs &a, hipStream_t st) { return launch<false>(a, 0, st); }

}  // namespace lca
