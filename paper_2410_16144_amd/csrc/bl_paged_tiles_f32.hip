// The tiles form of bl_attn_paged for fp32 queries (bl_paged_tiles.hpp).
#include "bl_paged_tiles.hpp"

namespace bl {

hipError_t launch_paged_tiles_f32(const PagedArgs& p, int64_t wgs, hipStream_t s) {
    return launch_paged_tiles_width<3, 2>(p, wgs, s);
}

}  // namespace bl
