// The tiles form of bl_attn_paged for bf16 queries (bl_paged_tiles.hpp).
#include "bl_paged_tiles.hpp"

namespace bl {

hipError_t launch_paged_tiles_bf16(const PagedArgs& p, int64_t wgs, hipStream_t s) {
    return p.tile_rows == 128 ? launch_paged_tiles_width<1, 4>(p, wgs, s) : launch_paged_tiles_width<1, 2>(p, wgs, s);
}

}  // namespace bl
