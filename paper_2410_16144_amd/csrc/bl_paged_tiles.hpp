// bl_attn_paged for many rows: prompts, pieces of prompts, drafted tokens.
//
// One workgroup = a tile of 32 RW consecutive rows of one sequence and key head (a row is one query head of one token, token by token, so that
// the query heads of a key head share what is read of it) against the positions 0 .. its last row's, 64 at a time through LDS, two chunks deep: one
// barrier per chunk, behind which the next one is requested.  Its four waves are RW sets of 32 rows times 4 / RW shares of a chunk's keys.  Two
// workgroups fit a compute unit (head sizes up to 128): one is in its products while the other is in its softmax.
//
// Scores are formed transposed, S^T = K Q^T (v_mfma_f32_32x32x16_bf16): a lane has 16 of 32 keys' weights of ONE row, laid out as the operand of
// O^T += V^T P^T; V^T by the transposing LDS read (slots 0..3 of lane half g are keys 4 g .. 4 g + 3 of sixteen, slots 4..7 keys 8 + 4 g ..).
// bf16 queries enter as they are and weights rounded to bf16 (at most 2^-8 of a weight, as much as the output's own rounding); fp32 queries and
// weights as three bf16 numbers each, their sum, in three products.  Maxima, sums and outputs are fp32.  The running maximum is moved only when a
// score exceeds it by 2^8 or more: weights are then at most 2^8, and what they are relative to cancels in the division.
//
// Long walks of few tiles are shared by up to `splits` workgroups, which leave their sums in memory for a launch of their own that adds them.
#pragma once
#include "bl_paged.hpp"

namespace bl {

constexpr int kPagedChunk = 64;

template <int PIECES>
__device__ __forceinline__ f32x16 paged_mfma32(const s16x8& a, const s16x8 (&b)[PIECES], f32x16 c) {
#pragma unroll
    for (int i = PIECES - 1; i >= 0; --i)
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b[i]), c, 0, 0, 0);
    return c;
}

// A tile: rows row0 .. row0 + rows - 1 of sequence b's rows of one key head.
struct PagedTileOf {
    PagedSequence s;
    int b, row0, rows, low, reach;   // low: the last position that its first row sees; reach: positions that its last row sees
    int slot;                        // number of the tile among all
};
__device__ __forceinline__ int paged_tiles_of(const PagedArgs& p, const PagedSequence& s, int tile_rows) {
    const int64_t rows = (int64_t)s.rows * p.group;
    return rows > p.few ? (int)((rows + tile_rows - 1) / tile_rows) : 0;
}
__device__ __forceinline__ bool paged_tile(const PagedArgs& p, int lane, int item, int tile_rows, PagedTileOf& t) {
    int index, before;
    if (!paged_find(p.c, lane, item, [&](const PagedSequence& s) { return paged_tiles_of(p, s, tile_rows); }, t.b, index, before, t.s)) return false;
    t.slot = item;
    const int rows = t.s.rows * p.group;
    t.row0 = (paged_tiles_of(p, t.s, tile_rows) - 1 - index) * tile_rows;      // the longest walk first
    t.rows = min(tile_rows, rows - t.row0);
    t.low = t.s.pos + t.row0 / p.group;
    t.reach = t.s.pos + (t.row0 + t.rows - 1) / p.group + 1;
    return true;
}
// Workgroups that share the tile's walk.
__device__ __forceinline__ int paged_tile_parts(const PagedArgs& p, const PagedTileOf& t) { return min(p.splits, (t.reach + kPagedLeast - 1) / kPagedLeast); }
__device__ __forceinline__ int64_t paged_row_at(const PagedArgs& p, const PagedTileOf& t, int head, int row) {   // of q and out
    const int token = row / p.group;
    return (((int64_t)(t.s.first + token) * p.c.n_heads + head) * p.group + row - token * p.group) * p.c.head_dim;
}
// A part's figures of a tile's row: (maximum, sum), two words of padding, then the values.
__device__ __forceinline__ float* paged_figures(const PagedArgs& p, const PagedTileOf& t, int head, int part, int row, int tile_rows) {
    return p.figures + ((((int64_t)t.slot * p.splits + part) * p.c.n_heads + head) * tile_rows + row) * (4 + p.c.head_dim);
}

template <int KS, int PIECES, int RW>
__global__ __launch_bounds__(256, KS <= 8 ? 2 : 1) void paged_tiles_kernel(const PagedArgs p) {
    using T = PagedTile<KS>;
    constexpr bool kBf16 = PIECES == 1;
    constexpr int KW = 4 / RW, kTileRows = 32 * RW, DT = (KS + 1) / 2;
    constexpr int NB = kBf16 && KW == 1 ? 2 : 1;           // blocks of 32 keys that share a softmax step
    constexpr int kTurns = 2 / KW / NB;
    static_assert(RW == 4 || RW == 2, "forms");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ int odd_chunk, bad_page;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int rw = wave % RW, kw = wave / RW;
    const Paged& c = p.c;

    const int item = (int)blockIdx.x / c.n_heads, head = (int)blockIdx.x - item * c.n_heads;
    PagedTileOf t;
    const int which = item / p.splits, part = item - which * p.splits;
    if (!paged_tile(p, lane, which, kTileRows, t)) return;
    const int parts = paged_tile_parts(p, t);
    if (part >= parts) return;
    const int chunks = (t.reach + kPagedChunk - 1) / kPagedChunk;
    const int c0 = (int)((int64_t)chunks * part / parts), c1 = (int)((int64_t)chunks * (part + 1) / parts);
    const int32_t* line = c.table + (int64_t)t.b * c.table_width;
    if (tid == 0) odd_chunk = bad_page = 0;
    __syncthreads();

    // waves 0 and 1 bring a chunk's keys, 2 and 3 its values, 32 positions each
    const bool value = wave >= 2;
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address(lds) + wave * T::kBytes);
    PagedRequest<KS> req;
    if (value) req.template prepare<true>(lane);
    else req.template prepare<false>(lane);
    const auto request = [&](int chunk) {
        const int j0 = chunk * kPagedChunk + 32 * (wave & 1);
        const PagedBase base = paged_base<KS>(c, line, head, j0, t.reach - 1);
        if (base.bad && lane == 0) bad_page = 1;
        const int limit = max(t.reach - 1 - j0, 0);        // (no row at all: any)
        const uint32_t dst = to + (uint32_t)(chunk & 1) * (4 * T::kBytes);
        if (value) req.template send<true>(c.v, base, dst, limit, lane);
        else req.template send<false>(c.k, base, dst, limit, lane);
    };
    request(c0);

    // the wave's rows: operand column l32
    const int row = rw * 32 + l32;                         // of the tile
    const bool there = row < t.rows;
    const int limit = t.s.pos + (t.row0 + row) / p.group;  // the last position that the row sees
    const int wave_low = t.s.pos + (t.row0 + rw * 32) / p.group;
    const int wave_high = rw * 32 < t.rows ? t.s.pos + (t.row0 + min(rw * 32 + 31, t.rows - 1)) / p.group : -1;
    s16x8 q[KS][PIECES];
    {
        const int64_t row_at = there ? paged_row_at(p, t, head, t.row0 + row) : 0;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) paged_query<PIECES>(p.q, row_at, 16 * ks + 8 * g, c.head_dim, there, q[ks]);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) asm volatile("" : "+v"(q[ks][i]));   // (here they have arrived: no wait of theirs in the loop)

    f32x16 o[DT];
    float run_m = -INFINITY, run_l = 0.0f;                 // run_l: over this lane half's keys only
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
    int v_at[DT];                                          // of the transposing reads
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        const int key = 4 * g + ((lane & 15) >> 2);
        int piece = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        if (piece >= 2 * KS) piece = 0;                    // an odd KS: the last 16 elements are never stored
        v_at[d] = key * T::kRow + paged_v_place<KS>(key, piece) * 16 + (lane & 1) * 8;
    }

    for (int chunk = c0; chunk < c1; ++chunk) {
        const int j0 = chunk * kPagedChunk;
        const uint8_t* ring = lds + (chunk & 1) * (4 * T::kBytes);
        wait_vm<0>();
        __syncthreads();                                   // the chunk is here, and nobody reads the other one any more
        if (chunk + 1 < c1) request(chunk + 1);
        // Weights of zero may stand before values that a row does not see; infinities and NaN among those take the careful way.
        bool careful = false;
        if (j0 + kPagedChunk - 1 > t.low) {                // uniform
            uint32_t most = 0;
            for (int i = tid * 16; i < 2 * T::kBytes; i += 256 * 16) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(ring + 2 * T::kBytes + i);
#pragma unroll
                for (int j = 0; j < 4; ++j) most = paged_exponents(most, x[j]);
            }
            if (paged_not_finite(most)) odd_chunk = chunk + 1;
            __syncthreads();
            careful = odd_chunk == chunk + 1;
        }
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) {
            const int block = KW == 2 ? kw : turn * NB, j1 = j0 + 32 * block;
            if (j1 > wave_high) continue;                  // uniform
            const uint8_t* keys = ring + block * T::kBytes;
            const uint8_t* values = ring + (2 + block) * T::kBytes;
            f32x16 x[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) x[n][r] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int n = 0; n < NB; ++n)
                    x[n] = paged_mfma32<PIECES>(*reinterpret_cast<const s16x8*>(keys + n * T::kBytes + l32 * T::kRow + paged_k_place<KS>(l32, 2 * ks + g) * 16),
                                                q[ks], x[n]);
            if (j1 + 32 * NB - 1 > wave_low) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (j1 + 32 * n + 8 * (r >> 2) + 4 * g + (r & 3) > limit) x[n][r] = -INFINITY;
            }
            float most = x[0][0];
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, x[n][r]);
            most = over_blocks<32>(most, MaxOp());
            const bool moves = (most - run_m) * p.scale > 8.0f;   // (of each row for itself: no row's bits depend on another's)
            if (__any(moves)) {
                const float m_new = moves ? most : run_m;
                const float keep = !moves ? 1.0f : run_m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((run_m - m_new) * p.scale);
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[d][r] *= keep;
                run_l *= keep;
                run_m = m_new;
            }
            const float ref = run_m == -INFINITY ? 0.0f : run_m * p.scale;   // (a row that has seen nothing yet)
            s16x8 w[2 * NB][PIECES];                       // of 16 keys each
#pragma unroll
            for (int n = 0; n < 2 * NB; ++n) {
                uint32_t parts_of[PIECES][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float a = __builtin_amdgcn_exp2f(fmaf(x[n >> 1][8 * (n & 1) + 2 * j], p.scale, -ref));
                    const float b = __builtin_amdgcn_exp2f(fmaf(x[n >> 1][8 * (n & 1) + 2 * j + 1], p.scale, -ref));
                    run_l += a;
                    run_l += b;
                    uint32_t two[PIECES];
                    paged_split<PIECES>(a, b, two);
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) parts_of[i][j] = two[i];
                }
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
                    w[n][i] = __builtin_bit_cast(s16x8, (u32x4{parts_of[i][0], parts_of[i][1], parts_of[i][2], parts_of[i][3]}));
            }
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const auto read_v = [&](int n, int d) {        // 16 keys, 32 elements
                const uint8_t* at = values + v_at[d] + n * 16 * T::kRow;
                const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
                const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * T::kRow));
                return s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            };
            if (!careful) {
#pragma unroll
                for (int n = 0; n < 2 * NB; ++n)
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[d] = paged_mfma32<PIECES>(read_v(n, d), w[n], o[d]);
            } else {
#pragma unroll
                for (int n = 0; n < 2 * NB; ++n)
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        s16x8 finite, up, down;
                        paged_put_away(read_v(n, d), finite, up, down);
                        o[d] = paged_mfma32<PIECES>(finite, w[n], o[d]);
                        f32x16 n_up, n_down;
#pragma unroll
                        for (int r = 0; r < 16; ++r) n_up[r] = n_down[r] = 0.0f;
                        n_up = paged_mfma32<PIECES>(up, w[n], n_up);
                        n_down = paged_mfma32<PIECES>(down, w[n], n_down);
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            if (n_up[r] > 0.0f) o[d][r] += INFINITY;
                            if (n_down[r] > 0.0f) o[d][r] -= INFINITY;
                        }
                    }
            }
        }
    }

    run_l = over_blocks<32>(run_l, AddOp());
    __syncthreads();
    if (bad_page) run_l = NAN;                             // (rows of a sequence whose table names a page that is not there)
    if constexpr (KW == 2) {                               // the chunk's shares meet
        float* meet = reinterpret_cast<float*>(lds) + rw * (64 * 16 * DT);
        float2* meet_ml = reinterpret_cast<float2*>(reinterpret_cast<float*>(lds) + RW * 64 * 16 * DT) + rw * 64;
        if (kw == 1) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) meet[(d * 16 + r) * 64 + lane] = o[d][r];
            meet_ml[lane] = make_float2(run_m, run_l);
        }
        __syncthreads();
        if (kw == 1) return;
        const float2 other = meet_ml[lane];
        const float m = fmaxf(run_m, other.x), ref = m == -INFINITY ? 0.0f : m * p.scale;
        const float f0 = run_m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(fmaf(run_m, p.scale, -ref));
        const float f1 = other.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(fmaf(other.x, p.scale, -ref));
        run_l = run_l * f0 + other.y * f1;
        run_m = m;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] = o[d][r] * f0 + meet[(d * 16 + r) * 64 + lane] * f1;
    }
    if (!there) return;
    if (parts == 1) {
        const int64_t at = paged_row_at(p, t, head, t.row0 + row);
        const float inv = 1.0f / run_l;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int e = 32 * d + 8 * r + 4 * g;
                if (e < c.head_dim) paged_store<kBf16>(p.out, at + e, f32x4{o[d][4 * r] * inv, o[d][4 * r + 1] * inv, o[d][4 * r + 2] * inv, o[d][4 * r + 3] * inv});
            }
    } else {
        float* at = paged_figures(p, t, head, part, row, kTileRows);
        if (g == 0) *reinterpret_cast<float2*>(at) = make_float2(run_m, run_l);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int e = 32 * d + 8 * r + 4 * g;
                if (e < c.head_dim) *reinterpret_cast<f32x4*>(at + 4 + e) = f32x4{o[d][4 * r], o[d][4 * r + 1], o[d][4 * r + 2], o[d][4 * r + 3]};
            }
    }
}

template <int KS, int PIECES, int RW>
hipError_t launch_paged_tiles_form(const PagedArgs& p, int64_t tiles, hipStream_t s) {
    constexpr int kRing = 8 * PagedTile<KS>::kBytes, kMeet = RW == 4 ? 0 : RW * 64 * (16 * ((KS + 1) / 2) * 4 + 8);
    constexpr int kBytes = kRing > kMeet ? kRing : kMeet;
    static_assert(kBytes <= kMaxDecodeLds, "fits the LDS ceiling");
    static LdsCeiling ceiling;
    const hipError_t e = ceiling.ensure(reinterpret_cast<const void*>(&paged_tiles_kernel<KS, PIECES, RW>), kBytes);
    if (e != hipSuccess) return e;
    paged_tiles_kernel<KS, PIECES, RW><<<dim3((unsigned)(tiles * p.splits * p.c.n_heads)), dim3(256), kBytes, s>>>(p);
    return hipGetLastError();
}

template <int PIECES, int RW>
hipError_t launch_paged_tiles_width(const PagedArgs& p, int64_t tiles, hipStream_t s) {
    switch (paged_width(p.c.head_dim)) {
        case 32: return launch_paged_tiles_form<2, PIECES, RW>(p, tiles, s);
        case 48: return launch_paged_tiles_form<3, PIECES, RW>(p, tiles, s);
        case 64: return launch_paged_tiles_form<4, PIECES, RW>(p, tiles, s);
        case 96: return launch_paged_tiles_form<6, PIECES, RW>(p, tiles, s);
        case 128: return launch_paged_tiles_form<8, PIECES, RW>(p, tiles, s);
        case 192: return launch_paged_tiles_form<12, PIECES, RW>(p, tiles, s);
        case 256: return launch_paged_tiles_form<16, PIECES, RW>(p, tiles, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace bl
