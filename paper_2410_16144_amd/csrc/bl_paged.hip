// bl_attn_paged: which form takes which rows, how many workgroups share a walk, and the launch that adds the shares of a tile.
#include <algorithm>

#include "bl_paged_tiles.hpp"

namespace bl {

hipError_t launch_paged_rows(const PagedArgs& p, bool bf16, int64_t wgs, hipStream_t s);
hipError_t launch_paged_tiles_bf16(const PagedArgs& p, int64_t tiles, int tile_rows, hipStream_t s);
hipError_t launch_paged_tiles_f32(const PagedArgs& p, int64_t tiles, int tile_rows, hipStream_t s);

namespace {

// A tile's rows, each the sum of its parts' figures.
template <bool BF16>
__global__ __launch_bounds__(256) void paged_merge_kernel(const PagedArgs p, int tile_rows) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int pieces = tile_rows / 16;                     // of 16 rows, a workgroup each
    int index = blockIdx.x;
    const int piece = index % pieces;
    index /= pieces;
    const int which = index / p.c.n_heads, head = index - which * p.c.n_heads;
    PagedTileOf t;
    if (!paged_tile(p, lane, which, tile_rows, t)) return;
    const int parts = paged_tile_parts(p, t), quads = p.c.head_dim >> 2;
    if (parts == 1) return;
    for (int i = tid; i < 16 * quads; i += 256) {
        const int row = piece * 16 + i / quads, e = 4 * (i % quads);
        if (row >= t.rows) break;
        const float* first = paged_figures(p, t, head, 0, row, tile_rows);
        const int64_t step = paged_figures(p, t, head, 1, row, tile_rows) - first;
        float m = -INFINITY, l = 0.0f;
        for (int n = 0; n < parts; ++n) m = fmaxf(m, first[n * step]);
        const float ref = m == -INFINITY ? 0.0f : m * p.scale;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int n = 0; n < parts; ++n) {
            const float m_n = first[n * step], l_n = first[n * step + 1];
            // (a part of which the row sees nothing has no share, whatever it holds; NaN weights have one)
            if (m_n == -INFINITY && l_n == 0.0f) continue;
            const float f = m_n == -INFINITY ? NAN : __builtin_amdgcn_exp2f(fmaf(m_n, p.scale, -ref));
            l += f * l_n;
            sum += f * *reinterpret_cast<const f32x4*>(first + n * step + 4 + e);
        }
        paged_store<BF16>(p.out, paged_row_at(p, t, head, t.row0 + row) + e, sum / l);
    }
}

// What a call launches.  Counts on the host are upper bounds: lengths are the device's.
struct PagedPlan {
    bool    rows_form, tiles_form;
    int     few, slot_rows, tile_rows, splits, n_heads;
    int64_t rows_wgs, tiles;
    float   target;
    int64_t counter_bytes, rows_bytes, tiles_bytes;
    int64_t bytes() const { return counter_bytes + rows_bytes + tiles_bytes; }
    bool    launchable() const { return rows_wgs < (1 << 24) && tiles * splits * n_heads < (1 << 24) && tiles * n_heads * 8 < (1 << 24); }
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

PagedPlan paged_plan(int n_heads, int group, int head_dim, int sequences, int rows, int max_pos, bool one_each) {
    PagedPlan r{};
    r.n_heads = n_heads;
    const int found = compute_unit_count(), cus = found > 0 ? found : 256;
    const int width = paged_width(head_dim);
    const int64_t all = (int64_t)rows * group;
    // Sequences of few rows have a form of their own, where there are some as far as the host can tell.
    r.rows_form = one_each ? group <= kPagedFew : all <= (int64_t)4 * kPagedFew * sequences && group <= kPagedFew;
    r.tiles_form = one_each ? !r.rows_form : !r.rows_form || all > kPagedFew;
    r.few = r.rows_form ? kPagedFew : 0;
    if (r.rows_form) {
        const int resident = width >= 256 ? 1 : width >= 192 ? 1 : width >= 96 ? 2 : 4;   // workgroups of a compute unit, by their LDS
        const int wanted = cus * resident;
        r.target = (float)n_heads / (float)wanted;
        r.slot_rows = one_each ? group : kPagedFew;
        const int64_t most = std::min<int64_t>(kPagedMostSplits, ceil_div(max_pos, kPagedLeast));
        r.rows_wgs = n_heads * std::min<int64_t>(sequences * most, wanted / n_heads + 1 + sequences);
        r.rows_bytes = most > 1 ? r.rows_wgs * r.slot_rows * (1 + head_dim / 2) * 8 : 0;
    }
    r.tile_rows = 128;
    r.splits = 1;
    if (r.tiles_form) {
        const int64_t slots = (int64_t)cus * (width <= 128 ? 2 : 1);
        const auto tiles_of = [&](int tile_rows) { return all / tile_rows + std::min<int64_t>(sequences, rows); };
        if (tiles_of(128) * n_heads < slots) r.tile_rows = 64;
        r.tiles = tiles_of(r.tile_rows);
        const int64_t most = std::min<int64_t>(16, ceil_div(max_pos, kPagedLeast));
        r.splits = (int)std::max<int64_t>(1, std::min(most, slots / (r.tiles * n_heads)));
        if (r.splits > 1) r.tiles_bytes = r.tiles * r.splits * n_heads * r.tile_rows * (4 + head_dim) * 4;
    }
    r.rows_bytes = ceil_div(r.rows_bytes, 256) * 256;
    r.counter_bytes = (int64_t)BL_PAGED_MAX_SEQUENCES * n_heads * 4;   // (of any call's: figures never lie where another call counts)
    return r;
}

}  // namespace

int64_t paged_scratch_bytes(int n_heads, int group, int head_dim, int sequences, int rows, int max_pos, bool one_each) {
    return paged_plan(n_heads, group, head_dim, sequences, rows, max_pos, one_each).bytes();
}

hipError_t launch_attn_paged(const ::bl_attn_paged_args& a, hipStream_t s) {
    PagedArgs p{};
    p.c = paged_of(*a.cache, *a.rows);
    p.q = a.q_dev; p.out = a.out_dev;
    p.group = a.n_q_heads / p.c.n_heads;
    p.scale = 1.4426950408889634f / sqrtf((float)p.c.head_dim);
    const PagedPlan plan = paged_plan(p.c.n_heads, p.group, p.c.head_dim, p.c.sequences, p.c.rows, p.c.max_pos, p.c.start == nullptr);
    if (!plan.launchable()) return hipErrorInvalidConfiguration;
    const bool bf16 = a.dt == BL_BF16;
    p.few = plan.few; p.slot_rows = plan.slot_rows; p.splits = plan.splits; p.target = plan.target;
    uint8_t* scratch = static_cast<uint8_t*>(a.scratch_dev);
    p.counters = reinterpret_cast<uint32_t*>(scratch);
    hipError_t e = hipSuccess;
    if (plan.tiles_form) {
        p.figures = reinterpret_cast<float*>(scratch + plan.counter_bytes + plan.rows_bytes);
        e = (bf16 ? launch_paged_tiles_bf16 : launch_paged_tiles_f32)(p, plan.tiles, plan.tile_rows, s);
        if (e == hipSuccess && plan.splits > 1) {
            const unsigned wgs = (unsigned)(plan.tiles * p.c.n_heads * (plan.tile_rows / 16));
            if (bf16) paged_merge_kernel<true><<<dim3(wgs), dim3(256), 0, s>>>(p, plan.tile_rows);
            else paged_merge_kernel<false><<<dim3(wgs), dim3(256), 0, s>>>(p, plan.tile_rows);
            e = hipGetLastError();
        }
    }
    if (e == hipSuccess && plan.rows_form) {
        p.figures = reinterpret_cast<float*>(scratch + plan.counter_bytes);
        e = launch_paged_rows(p, bf16, plan.rows_wgs, s);
    }
    return e;
}

}  // namespace bl
