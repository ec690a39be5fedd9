// bl_attn_paged: which form takes a call, and how many workgroups it is meant for.
#include <algorithm>

#include "bl_paged.hpp"

namespace bl {

hipError_t launch_paged_rows(const PagedArgs& p, bool bf16, int64_t wgs, hipStream_t s);
hipError_t launch_paged_tiles_bf16(const PagedArgs& p, int64_t wgs, hipStream_t s);
hipError_t launch_paged_tiles_f32(const PagedArgs& p, int64_t wgs, hipStream_t s);

namespace {

constexpr int64_t kCounters = 1 << 14;     // of any call's: figures never lie where another call counts

struct PagedPlan {
    bool    rows_form, shallow;
    int     tile_rows, most, wanted;
    int64_t wgs, slots, slot_bytes;
    int64_t counter_bytes, figure_bytes;
    bool launchable() const { return wgs < (1 << 24) && slots <= kCounters; }    // 2^32 threads (and every walk has a counter: 1024 key heads)
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Counts on the host are upper bounds, the lengths are the device's.  With `wanted` workgroups in mind a part has per >= n_heads * cost / wanted positions, cost
// the sum of all tiles' mean walks (paged_cost).  A walk of `reach` positions has at most reach / per + 1 parts, and the sum of all
// tiles' longest walks is at most twice the cost (the cost itself, where every sequence has one row): at most 2 wanted / n_heads parts more than
// there are tiles.  A walk with several parts has reach > per, fewer than 2 reach / per parts: at most 4 wanted slots of figures.
PagedPlan paged_plan(int n_heads, int group, int head_dim, int sequences, int rows, int max_pos, bool single, bool bf16) {
    PagedPlan r{};
    const int found = compute_unit_count(), cus = found > 0 ? found : 256, width = paged_width(head_dim);
    const int64_t all = (int64_t)rows * group;
    r.rows_form = single && group <= kPagedFew;
    const auto tiles_of = [&](int tile_rows) { return single ? (int64_t)sequences * ceil_div(group, tile_rows) : all / tile_rows + std::min<int64_t>(sequences, rows); };
    // Workgroups that a call is meant for.  Rows: as many as keep enough requests under way, no more, since every part of a walk has to be joined (64
    // heads on 8 at 100 003 positions: one per compute unit 73.8 us, two 79.9; eight sequences of 32 heads, 584 MB: 104.4 and 113.6); but rows of 64 elements
    // and less have half the bytes under way, and many sequences of unlike lengths want smaller parts more than few of them (32 heads on 8 over 60 to
    // 4000 positions: 64 sequences 54.9 us with two per unit, 61.1 with one, 128 97 and 108; of like lengths the same, 88).
    // Tiles: one per unit, joining is dearer still (for one and for two: 600 rows behind 512 of 32 heads, tiles by two on a unit either way, 24.4 and 38.0 us; 512 behind
    // 512 19.8 and 33.1; 16 rows of 64 heads on 8 behind 30 000 39 and 57; 300 rows of 32 on 8 behind 8000 84 and 77; 2000 rows of 16 heads of 256 79 and 103).
    r.wanted = r.rows_form && (width <= 64 || (int64_t)sequences * n_heads >= 2 * cus) ? 2 * cus : cus;
    if (r.rows_form) {
        // 128, 256, 512, 1024 positions: 32 heads at 1000 positions 13.4, 14.3, 17.1, 19.0 us; 64 on 8 at 8000 23.7, 19.3, 18.7, 22.9.
        r.tile_rows = group;
        r.most = 256;
        r.slot_bytes = (int64_t)group * (4 + head_dim) * 4;
    } else {
        // 128 rows where nearly two such tiles come on every unit (32 heads, 1024 rows behind as many: 49.7 us, 64 rows 42.4; 1700: 70.4 and 77.3; 4096 on
        // 8 key heads: 153 and 218); tiles of 64 by two on a unit where there are more of them than units (1024 rows behind 4096: 97 us, by one 117), else
        // by one (512 behind 512: 23.4 and 21.4).  Starts are the device's, so the last goes by full tiles.
        r.tile_rows = !bf16 || 2 * tiles_of(128) * n_heads < (width <= 128 ? 3 : 2) * cus ? 64 : 128;
        r.shallow = (single ? tiles_of(64) : ceil_div(all, 64)) * n_heads > cus;
        // As 32, 64, 128 positions (paged_parts): 5 rows of 32 heads on 8 behind 1500 positions 13.7, 14.3, 15.4 us, behind 4000 16.7, 18.0, 19.1, behind
        // 16 000 24.8, 24.9, 26.7; 64 rows of 12 heads behind 16 000 39.4, 36.7, 35.9; 16 rows of 64 heads on 8 behind 3000 21.8, 20.1, 21.8.
        r.most = kPagedTileParts;
        r.slot_bytes = (int64_t)r.tile_rows * (ceil_div(width, 32) * 32 * 4 + 8);
    }
    r.most = (int)std::min<int64_t>(r.most, ceil_div(max_pos, kPagedLeast));
    const int64_t tiles = tiles_of(r.tile_rows), more = (single ? 1 : 2) * (int64_t)r.wanted / n_heads + 1;
    r.wgs = n_heads * std::min(tiles * r.most, tiles + more);
    r.slots = r.most > 1 ? 4 * ((int64_t)r.wanted + n_heads) : 0;
    r.counter_bytes = kCounters * 4;
    r.figure_bytes = r.slots * r.slot_bytes;
    return r;
}

}  // namespace

int64_t paged_scratch_bytes(int n_heads, int group, int head_dim, int sequences, int rows, int max_pos, bool single) {
    int64_t most = 0;
    for (const bool bf16 : {false, true}) {
        const PagedPlan plan = paged_plan(n_heads, group, head_dim, sequences, rows, max_pos, single, bf16);
        most = std::max(most, plan.counter_bytes + plan.figure_bytes);
    }
    return most;
}

hipError_t launch_attn_paged(const ::bl_attn_paged_args& a, hipStream_t s) {
    PagedArgs p{};
    p.c = paged_of(*a.cache, *a.rows);
    p.q = a.q_dev; p.out = a.out_dev;
    p.group = a.n_q_heads / p.c.n_heads;
    p.scale = 1.4426950408889634f / sqrtf((float)p.c.head_dim);
    const bool bf16 = a.dt == BL_BF16;
    const PagedPlan plan = paged_plan(p.c.n_heads, p.group, p.c.head_dim, p.c.sequences, p.c.rows, p.c.max_pos, p.c.start == nullptr, bf16);
    if (!plan.launchable()) return hipErrorInvalidConfiguration;
    p.tile_rows = plan.tile_rows; p.most = plan.most; p.tile_shift = __builtin_ctz(plan.tile_rows); p.join = 64.0f; p.shallow = plan.shallow; p.slots = (int32_t)plan.slots; p.slot_bytes = (int32_t)plan.slot_bytes;
    p.target = (float)p.c.n_heads / (float)plan.wanted;
    p.counters = static_cast<uint32_t*>(a.scratch_dev);
    p.figures = reinterpret_cast<float*>(static_cast<uint8_t*>(a.scratch_dev) + plan.counter_bytes);
    return plan.rows_form ? launch_paged_rows(p, bf16, plan.wgs, s) : (bf16 ? launch_paged_tiles_bf16 : launch_paged_tiles_f32)(p, plan.wgs, s);
}

}  // namespace bl
