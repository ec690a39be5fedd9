// bl_attn8_decode and bl_attn8_prefill: the choice of form, and the kernel of the rows form.
//
// One token of each of several sequences, each behind a prefix that they share; a prompt's tokens behind a cache.  A launch has a shared part --
// all tokens' rows against the prefix, or a prompt's cache -- and an own part, each sequence's rows against its own cache; the workgroups of a row
// meet in scratch memory (attn8_finish).  The rows form (bl_attn8_rows.hpp) takes up to eight shared rows and all own ones, the tiles form
// (bl_attn8_tiles.hpp) more shared ones; both parts are in one launch.
#include "bl_attn8_rows.hpp"

namespace bl {

namespace {

template <int KB, int NQ, int W, bool STREAM>
__global__ __launch_bounds__(64 * W) void attn8_rows_kernel(const Attn8Args p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ Rows8Shared shared;
    __shared__ Attn8Rows rows;
    Attn8Walk walk;
    const int wg = blockIdx.x;   // uniform, like the walk
    if (!(wg < p.shared_wgs ? attn8_shared_walk(p, wg, 4 * NQ, walk) : attn8_own_walk(p, wg - p.shared_wgs, 4 * NQ, walk))) return;
    rows8_walk<KB, NQ, W, STREAM>(p, walk, lds, shared, rows);
}

template <int KB, int NQ, int W, bool STREAM>
hipError_t launch_form(const Attn8Args& p, int wgs, hipStream_t s) {
    using L = Rows8Lds<KB, NQ, W>;
    static_assert(L::kBytes <= kMaxDecodeLds, "fits the LDS ceiling");
    static LdsCeiling ceiling;   // per instantiation, i.e. per kernel
    const hipError_t e = ceiling.ensure(reinterpret_cast<const void*>(&attn8_rows_kernel<KB, NQ, W, STREAM>), L::kBytes);
    if (e != hipSuccess) return e;
    attn8_rows_kernel<KB, NQ, W, STREAM><<<dim3((unsigned)wgs), dim3(64 * W), L::kBytes, s>>>(p);
    return hipGetLastError();
}

template <int KB>
hipError_t launch_block(const Attn8Args& p, const Attn8Plan& plan, bool stream, int wgs, hipStream_t s) {
    static_assert(kRows8Waves == 8 && kRows8ManyWaves == 2 && kRows8FewWaves == 4, "waves as planned");
    // Rows in eights and sixteens always by streaming loads: half the kernels.  Ordinary and streaming, us: 64 heads on 8 at 300 positions 7.8 and 8.1, at
    // 8000 (16 MB) 12.7 and 13.5, at 30 000 (61 MB) 21.7 and 20.5; 64 on 4 at 20 000 (20 MB) 22.1 and 22.9.
    if (plan.block == 8) return plan.waves == 8 ? launch_form<KB, 2, 8, true>(p, wgs, s) : launch_form<KB, 2, 4, true>(p, wgs, s);
    if (plan.block == 16) {
        if constexpr (KB <= 2) {
            if (plan.waves == 8) return launch_form<KB, 4, 8, true>(p, wgs, s);
        }
        return launch_form<KB, 4, 4, true>(p, wgs, s);
    }
    if (plan.waves == 8) return stream ? launch_form<KB, 1, 8, true>(p, wgs, s) : launch_form<KB, 1, 8, false>(p, wgs, s);
    return stream ? launch_form<KB, 1, 2, true>(p, wgs, s) : launch_form<KB, 1, 2, false>(p, wgs, s);
}

hipError_t launch_rows(const Attn8Args& p, const Attn8Plan& plan, int wgs, hipStream_t s) {
    // Caches of 32 MiB and more (the dies' L2s together) by streaming loads.  32 heads of 128, ordinary and streaming, us: 500 positions 6.9 and 7.8, 4000
    // (33 MB) 12.7 and 12.9, 8000 19.2 and 17.6, 30 000 52.2 and 46.7.  (By the caches' size, which the host knows, not by the positions.)
    const int64_t positions = p.shared_wgs > 0 ? (p.prompt ? p.pos0 + p.tokens : p.shared_len) : 0;
    const bool stream = 2 * (positions + (int64_t)p.tokens * p.max_pos) * p.n_heads * p.size >= 32 << 20;
    static_assert(BL_ATTN_MAX_HEAD_DIM == 256, "head sizes up to four blocks of 64");
    switch ((p.head_dim + 63) / 64) {
        case 1: return launch_block<1>(p, plan, stream, wgs, s);
        case 2: return launch_block<2>(p, plan, stream, wgs, s);
        case 3: return launch_block<3>(p, plan, stream, wgs, s);
        case 4: return launch_block<4>(p, plan, stream, wgs, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch(Attn8Args& p, const Attn8Plan& plan, void* scratch, hipStream_t s) {
    p.rows = p.tokens * p.group;
    p.size = kv8_size(p.head_dim);
    p.unit = 1.4426950408889634f / sqrtf((float)p.head_dim);
    p.counters = static_cast<uint32_t*>(scratch);
    p.figures = reinterpret_cast<float2*>(p.counters + attn8_counters(p.n_heads, p.rows));
    p.shared_set = plan.shared_set; p.own_set = plan.own_set;
    p.shared_splits = plan.shared_splits; p.shared_blocks = plan.shared_blocks; p.shared_units = (int32_t)plan.shared_units; p.strips = plan.strips;
    p.own_splits = plan.own_splits; p.own_blocks = plan.own_blocks;
    p.shared_wgs = (int32_t)plan.shared_wgs;
    const int wgs = (int)(plan.shared_wgs + plan.own_wgs);
    p.by_heads = divider(p.n_heads); p.by_group = divider(p.group); p.by_half = divider(p.head_dim / 2); p.by_tokens = divider(p.tokens);
    p.by_own_blocks = divider(p.own_blocks); p.by_own_splits = divider(p.own_splits); p.by_shared_splits = divider(p.shared_splits);
    p.by_shared_units = divider((int)plan.shared_units); p.by_pieces = divider(p.n_heads * p.shared_splits);
    const int found = compute_unit_count(), cus = found > 0 ? found : 256;
    p.folded = plan.folded;
    p.paired = !plan.folded && wgs > cus && wgs <= 2 * cus;   // all resident: a unit's second block is as short as its first one is long
    if (!plan.tiles) return launch_rows(p, plan, wgs, s);
    p.merges = plan.slots() > 1;
    hipError_t e = launch_attn8_tiles(p, plan.apart ? p.shared_wgs : wgs, s);
    if (e == hipSuccess && plan.apart) {
        p.shared_wgs = 0;
        e = launch_rows(p, plan, (int)plan.own_wgs, s);
    }
    return e == hipSuccess && p.merges ? launch_attn8_merge(p, s) : e;
}

// A prompt's rows: the write clears the counters of the launch behind it.
Attn8Plan prompt_plan(int n_heads, int group, int head_dim, int pos0, int M) { return attn8_plan(n_heads, group, M, pos0 + M, 0, kv8_size(head_dim)); }

}  // namespace

int64_t attn8_scratch_bytes(int n_heads, int group, int head_dim, int max_pos, int sequences, int prefix_len) {
    return attn8_scratch(attn8_plan(n_heads, group, sequences, prefix_len, max_pos, kv8_size(head_dim)), n_heads, (int64_t)sequences * group, head_dim);
}

hipError_t launch_attn8_decode(const ::bl_attn8_args& a, hipStream_t s) {
    Attn8Args p{};
    p.q = a.q_lin_dev; p.k_new = a.k_lin_dev; p.v_new = a.v_lin_dev; p.pos = a.pos_dev;
    p.rope = reinterpret_cast<const float2*>(a.rope_table_dev);
    p.out = a.out_dev;
    p.own = kv8_of(a.cache, 0);
    if (a.prefix_len > 0) p.shared = kv8_of(a.prefix, 0);
    p.n_heads = a.cache.n_heads; p.group = a.n_q_heads / a.cache.n_heads; p.head_dim = a.cache.head_dim;
    p.tokens = a.cache.sequences; p.shared_len = a.prefix_len; p.max_pos = a.cache.max_pos;
    p.own_codes = p.own.head_bytes * p.n_heads;
    p.own_scales = p.own.head_scales * p.n_heads;
    const Attn8Plan plan = attn8_plan(p.n_heads, p.group, p.tokens, p.shared_len, p.max_pos, kv8_size(p.head_dim));
    return plan.launchable() ? launch(p, plan, a.scratch_dev, s) : hipErrorInvalidConfiguration;
}

int64_t attn8_prefill_scratch_bytes(int n_heads, int group, int head_dim, int pos0, int M) {
    return attn8_scratch(prompt_plan(n_heads, group, head_dim, pos0, M), n_heads, (int64_t)M * group, head_dim);
}

hipError_t launch_attn8_prefill(const ::bl_attn8_prefill_args& a, hipStream_t s) {
    Attn8Args p{};
    p.q = a.q_lin_dev;
    p.rope = reinterpret_cast<const float2*>(a.rope_table_dev);
    p.out = a.out_dev;
    p.shared = kv8_of(a.cache, a.sequence);
    p.n_heads = a.cache.n_heads; p.group = a.n_q_heads / a.cache.n_heads; p.head_dim = a.cache.head_dim;
    p.tokens = a.M; p.prompt = 1; p.pos0 = a.pos0;
    const Attn8Plan plan = prompt_plan(p.n_heads, p.group, p.head_dim, a.pos0, a.M);
    if (!plan.launchable()) return hipErrorInvalidConfiguration;
    const int64_t counters = plan.meets() ? attn8_counters(p.n_heads, (int64_t)a.M * p.group) : 0;
    const ::bl_kv8_write_args w{&a.cache, a.k_lin_dev, a.v_lin_dev, a.rope_table_dev, (int64_t)p.n_heads * p.head_dim, BL_F32, a.sequence, a.pos0, a.M};
    const hipError_t e = launch_kv8_write(w, static_cast<uint32_t*>(a.scratch_dev), counters, s);
    return e != hipSuccess ? e : launch(p, plan, a.scratch_dev, s);
}

}  // namespace bl
