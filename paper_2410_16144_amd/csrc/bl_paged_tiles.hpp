// bl_attn_paged for many rows: prompts, pieces of prompts, drafted tokens.
//
// One workgroup = a tile of 32 RW consecutive rows of one sequence and key head (a row is one query head of one token, token by token, so that
// the query heads of a key head share what is read of it) against the positions 0 .. its last row's, 64 at a time through a ring of chunks in LDS with one
// barrier a chunk.  Its four waves are RW sets of 32 rows times 4 / RW shares of a chunk's keys:
//   * RW = 4, tiles of 128 rows, two workgroups on a compute unit (head sizes up to 128): one is in its products while the other is in its softmax.
//     4096 rows of 32 heads on 8, 128 wide: 155 us, 890 TFLOP/s; without exponentials, requests and reads of LDS it would be 125,
//     which is what the products alone run at (a library product of 4096 cubed: 1150 TFLOP/s).
//   * RW = 2, tiles of 64 rows, for fewer, also by two on a unit with a ring of two chunks, or by one with a ring of four (kDepth).  One alone is bound by
//     the chain of its chunk -- scores, maximum, weights, sums, 0.66 us, of which the products are 0.21 -- with nobody to fill its gaps; eight waves on chunks
//     of 128 take 0.60 per 64 positions, but 2.5 us more for their longer start and end (512 rows behind 512: 22.7 us, with four 20.9, since then 19.6), so four it is.
// Which when: paged_plan.
//
// Scores are formed transposed, S^T = K Q^T (v_mfma_f32_32x32x16_bf16): a lane has 16 of 32 keys' weights of ONE row, laid out as the operand of
// O^T += V^T P^T; V^T by the transposing LDS read (slots 0..3 of lane half g are keys 4 g .. 4 g + 3 of sixteen, slots 4..7 keys 8 + 4 g ..).
// bf16 queries enter as they are and weights rounded to bf16 (at most 2^-8 of a weight, as much as the output's own rounding); fp32 queries and
// weights as three bf16 numbers each, their sum, in three products.  Maxima, sums and outputs are fp32.  The running maximum is moved only when a
// score exceeds it by 2^8 or more: weights are then at most 2^8, and what they are relative to cancels in the division.
//
// Long walks of few tiles are shared by several workgroups, the last of which adds up their sums (paged_last).
#pragma once
#include <type_traits>

#include "bl_paged.hpp"

namespace bl {

constexpr int kPagedChunk = 64;
constexpr float kPagedLargeScore = 1024.0f;   // exponents of two: up to here a maximum's rounding is 2^-15 of one at most

template <int PIECES>
__device__ __forceinline__ f32x16 paged_mfma32(const s16x8& a, const s16x8 (&b)[PIECES], f32x16 c) {
#pragma unroll
    for (int i = PIECES - 1; i >= 0; --i)
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b[i]), c, 0, 0, 0);
    return c;
}

template <int KS, int RW, int DEPTH>
struct PagedTilesLds {
    static constexpr int DT = (KS + 1) / 2;
    static constexpr int kRing = DEPTH * 4 * PagedTile<KS>::kBytes;                    // [chunk % depth][keys, values][32 positions]
    static constexpr int kMeet = RW == 4 ? 0 : RW * 64 * (16 * DT * 4 + 8);             // half of the waves' sums
    static constexpr int kBytes = kRing > kMeet ? kRing : kMeet;
    static_assert(kBytes <= kMaxDecodeLds, "fits the LDS ceiling");
};

template <int KS, int PIECES, int RW, int kDepth>
__global__ __launch_bounds__(256, KS <= 8 && (PIECES == 1 || KS <= 4) ? 2 : 1) void paged_tiles_kernel(const PagedArgs p) {
    using T = PagedTile<KS>;
    constexpr bool kBf16 = PIECES == 1;
    constexpr int KW = 4 / RW, DT = (KS + 1) / 2;
    constexpr int NB = 2 / KW;                             // a wave's blocks of 32 keys in a chunk
    constexpr bool kReload = !kBf16 && KS > 8;             // a second walk loads its rows step by step: they take more registers than there are
    static_assert(RW == 4 || RW == 2, "forms");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ int odd_chunk, odd_sums, bad_page, last_one;
    __shared__ uint32_t odd_values[2][kPagedChunk * DT];   // [up, down][key][32 elements]: where infinities and NaN were
    __shared__ uint32_t odd_seen[2 * DT][256];             // the same of the keys that a lane's row sees
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, g = lane >> 5;
    const int rw = wave % RW, kw = wave / RW;
    const Paged& c = p.c;

    PagedWork t;
    if (!paged_work<false>(p, lane, t)) return;
    const int head = t.head, chunks = (t.reach + kPagedChunk - 1) / kPagedChunk;
    const int c0 = paged_first(t, chunks, t.part), c1 = paged_first(t, chunks, t.part + 1);
    const int32_t* line = c.table + (int64_t)t.b * c.table_width;
    if (tid == 0) odd_chunk = odd_sums = bad_page = 0;
    __syncthreads();

    // the wave's rows: operand column l32
    const int row = rw * 32 + l32;                         // of the tile
    const bool there = row < t.rows;
    // The last position that the row sees.  (A column without a row sees what the last row sees: what lies behind that is no reason to walk again.)
    const int limit = min(t.s.pos + (t.row0 + row) / p.group, t.reach - 1);
    const int wave_low = t.s.pos + uniform((t.row0 + rw * 32) / p.group);
    const int wave_high = rw * 32 < t.rows ? t.s.pos + uniform((t.row0 + min(rw * 32 + 31, t.rows - 1)) / p.group) : -1;
    s16x8 q[KS][PIECES];
    const auto load_step = [&](int ks) __attribute__((always_inline)) {
        paged_query<PIECES>(p.q, there ? paged_row_at(p, t, row) : 0, 16 * ks + 8 * g, c.head_dim, there, q[ks]);
    };
    const auto load_rows = [&]() __attribute__((always_inline)) {
        const int64_t row_at = there ? paged_row_at(p, t, row) : 0;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            if constexpr (kReload) load_step(ks);
            else paged_query<PIECES>(p.q, row_at, 16 * ks + 8 * g, c.head_dim, there, q[ks]);
    };
    load_rows();

    // waves 0 and 1 bring a chunk's keys, 2 and 3 its values, 32 positions each
    const bool value = wave >= 2;
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address(lds) + wave * T::kBytes);
    PagedRequest<KS, false, !kBf16 && KS == 16> req;
    if (value) req.template prepare<true>(lane);
    else req.template prepare<false>(lane);
    const auto first_of = [&](int chunk) { return min(chunk, c1) * kPagedChunk + 32 * (wave & 1); };
    // The table is looked at once for 32 chunks: a lane has the address of one of the wave's sixteens, two a chunk.  (Word by word, each chunk waited
    // for its words and then computed 64-bit addresses in the only wave of its unit: 0.72 us a chunk.)
    uint32_t low = 0, high = 0;
    int held = c0;                                         // the first of the chunks
    const auto look = [&](int chunk) __attribute__((always_inline)) {
        held = chunk;
        const int j = min(first_of(chunk + (lane >> 1)) + 16 * (lane & 1), t.reach - 1);
        int page = line[j >> c.page_shift];
        if ((uint32_t)page >= (uint32_t)c.pages) {
            if (chunk + (lane >> 1) < c1) bad_page = 1;
            page = 0;
        }
        const int inside = j & ((1 << c.page_shift) - 1) & ~15;
        const uint64_t at = reinterpret_cast<uint64_t>(value ? c.v : c.k) + ((((int64_t)page * c.n_heads + head) << c.page_shift) + inside) * T::kRow;
        low = (uint32_t)at;
        high = (uint32_t)(at >> 32);
    };
    look(c0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < PIECES; ++i) asm volatile("" : "+v"(q[ks][i]));   // (here they have arrived, under the look at the table: no wait of theirs later)
    // A request is prepared, and goes out piece by piece between the products: all at once, the wave stands still until the last piece has found a
    // place (700 cycles a chunk, as many as the products of the scores).
    PagedSource next{{nullptr, nullptr}};
    uint32_t next_at = 0;
    uint64_t pieces = 0;                                   // the lanes that bring them: all or none
    const auto prepare = [&](int chunk) __attribute__((always_inline)) {   // (one after the other)
        if (__builtin_expect(chunk - held >= 32, 0)) look(chunk);
        const int i = 2 * (chunk - held);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            next.at[h] = reinterpret_cast<const uint8_t*>((uint64_t)(uint32_t)__builtin_amdgcn_readlane(high, i + h) << 32 | (uint32_t)__builtin_amdgcn_readlane(low, i + h));
        next_at = to + (uint32_t)(chunk & (kDepth - 1)) * (4 * T::kBytes);
        pieces = ~0ull;
    };
    const auto prepare_if = [&](int chunk) __attribute__((always_inline)) {
        pieces = 0;
        if (chunk < c1) prepare(chunk);
    };
    constexpr int kSlots = KS * NB + 2 * NB * DT;          // of a chunk, a read and PIECES products each
    const auto send_at = [&](int slot, auto sure) __attribute__((always_inline)) {
        const int s = (slot * KS + kSlots - 1) / kSlots;   // the piece whose place this is, if any
        if (s < KS && s * kSlots / KS == slot) req.template piece<!decltype(sure)::value>(s, next, next_at, pieces);
    };
    f32x16 o[DT];
    float run_m, run_l;                                    // run_l: over this lane half's keys only
    // Of the transposing reads: pieces 4 d .. 4 d + 3 trade places among kMoved times 32 elements, what lies beyond is a constant away.
    constexpr int kMoved = KS % 8 == 0 ? 4 : KS % 4 == 0 ? 2 : KS % 2 == 0 ? 1 : DT;
    int v_at[kMoved];
#pragma unroll
    for (int d = 0; d < kMoved; ++d) {
        const int key = 4 * g + ((lane & 15) >> 2);
        int piece = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        if (piece >= 2 * KS) piece = 0;                    // an odd KS: the last 16 elements are never stored
        v_at[d] = key * T::kRow + paged_v_place<KS>(key, piece) * 16 + (lane & 1) * 8;
    }

    // Chunks that every row of the tile sees whole, then those that end among the rows' own positions.  (The first kind's code lies side by side: a jump
    // costs as much as two products.)
    // `sure`: chunks whose request, kDepth - 1 chunks on, is there to be made, so that it is known how many requests are behind the chunk's own.
    // `again`: of the second kind, a walk that was not right the first time (below); code of its own, or the others would be 2 % slower for it.
    const auto walk = [&](int chunk, auto which, auto sure, auto again) __attribute__((always_inline)) {
        constexpr bool kMasked = decltype(which)::value, kSure = decltype(sure)::value, kAgain = decltype(again)::value;
        const int j0 = chunk * kPagedChunk;
        const uint8_t* ring = lds + (chunk & (kDepth - 1)) * (4 * T::kBytes);
        wait_vm<kSure ? (kDepth - 2) * KS : 0>();
        __syncthreads();                                   // the chunk is here, and nobody reads the one before it any more
        if constexpr (kSure) prepare(chunk + kDepth - 1);
        else prepare_if(chunk + kDepth - 1);
        // Weights of zero may stand before values that a row does not see.  What lies behind the sequence's last row is nobody's: zero.  Infinities and NaN elsewhere
        // make sums that are not finite, and the second walk puts them away and notes them.
        bool careful = false;
        if constexpr (kMasked) {
            uint8_t* values = lds + (ring - lds) + 2 * T::kBytes;
            const int end = min(kPagedChunk, t.reach - j0) * T::kRow;   // (uniform)
            if (end < 2 * T::kBytes) {
#pragma unroll 1
                for (int i = end + tid * 16; i < 2 * T::kBytes; i += 256 * 16) *reinterpret_cast<u32x4*>(values + i) = u32x4{0, 0, 0, 0};
                __syncthreads();
            }
        }
        if constexpr (kAgain) {
            uint8_t* values = lds + (ring - lds) + 2 * T::kBytes;
            uint32_t most = 0;
#pragma unroll 1
            for (int i = tid * 16; i < 2 * T::kBytes; i += 256 * 16) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(values + i);
#pragma unroll
                for (int j = 0; j < 4; ++j) most = paged_exponents(most, x[j]);
            }
            if (paged_not_finite(most)) odd_chunk = chunk + 1;
            for (int i = tid; i < kPagedChunk * DT; i += 256) odd_values[0][i] = odd_values[1][i] = 0;
            __syncthreads();
            careful = uniform(odd_chunk) == chunk + 1;
            if (careful) {
#pragma unroll 1
                for (int i = tid * 16; i < 2 * T::kBytes; i += 256 * 16) {
                    const int key = i / T::kRow, piece = paged_v_place<KS>(key, i % T::kRow / 16);
                    uint32_t up = 0, down = 0;
#pragma unroll 1
                    for (int j = 0; j < 8; ++j) {
                        uint16_t* at = reinterpret_cast<uint16_t*>(values + i) + j;
                        const uint32_t x = *at, size = x & 0x7fffu;
                        if (size < 0x7f80u) continue;
                        if (size > 0x7f80u || x < 0x8000u) up |= 1u << j;     // (NaN is both)
                        if (size > 0x7f80u || x >= 0x8000u) down |= 1u << j;
                        *at = 0;
                    }
                    if (up) atomicOr(&odd_values[0][key * DT + piece / 4], up << 8 * (piece % 4));
                    if (down) atomicOr(&odd_values[1][key * DT + piece / 4], down << 8 * (piece % 4));
                }
                __syncthreads();
            }
        }
        const int block = KW == 2 ? kw : 0, j1 = j0 + 32 * block;
        // (Uniform.  Wide heads: a branch would cost registers for a second set of sums, which these have to fetch from memory in every chunk.)
        if (KS > 8 || (kMasked ? j1 <= wave_high : wave_high >= 0)) {
            const uint8_t* keys = ring + block * T::kBytes;
            const uint8_t* values = ring + (2 + block) * T::kBytes;
            f32x16 x[NB];
            // (four key operands are on their way from LDS at any time)
            constexpr int kReads = KS * NB, kAhead = kReads < 4 ? kReads : 4;
            s16x8 k[kAhead];
            const auto read_k = [&](int i) __attribute__((always_inline)) {               // block i % NB, elements 16 (i / NB) ..
                return *reinterpret_cast<const s16x8*>(keys + i % NB * T::kBytes + l32 * T::kRow + paged_k_place<KS>(l32, 2 * (i / NB) + g) * 16);
            };
#pragma unroll
            for (int i = 0; i < kAhead; ++i) k[i] = read_k(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kReads; ++i) {
                const f32x16 zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (kAgain && !kBf16) {
                    if (kReload && i % NB == 0) load_step(i / NB);
                    s16x8 finite, odd;
                    paged_apart(k[i % kAhead], finite, odd);
                    x[i % NB] = paged_mfma32<PIECES>(finite, q[i / NB], i < NB ? zero : x[i % NB]);
                    const u32x4 any = __builtin_bit_cast(u32x4, odd);
                    if (__any((any[0] | any[1] | any[2] | any[3]) != 0)) {
                        const s16x8 signs[1] = {paged_signs<PIECES>(q[i / NB])};
                        x[i % NB] = paged_mfma32<1>(odd, signs, x[i % NB]);
                    }
                } else {
                    x[i % NB] = paged_mfma32<PIECES>(k[i % kAhead], q[i / NB], i < NB ? zero : x[i % NB]);
                }
                if (i + kAhead < kReads) k[i % kAhead] = read_k(i + kAhead);
                send_at(i, sure);
                __builtin_amdgcn_sched_barrier(0);
            }
            // the first sixteen keys' value operands travel under the softmax
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const auto read_v = [&](int n, int d) __attribute__((always_inline)) {        // 16 keys, 32 elements
                const uint8_t* at = values + v_at[d % kMoved] + d / kMoved * (64 * kMoved) + n * 16 * T::kRow;
                const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
                const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 8 * T::kRow));
                return s16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            };
            s16x8 v[DT];
#pragma unroll
            for (int d = 0; d < DT; ++d) v[d] = read_v(0, d);
            __builtin_amdgcn_sched_barrier(0);
            if (kMasked && j1 + 32 * NB - 1 > wave_low) {
                const int seen = limit - j1 - 4 * g;
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * n + 8 * (r >> 2) + (r & 3) > seen) x[n][r] = -INFINITY;
            }
            if (kAgain && careful) {                       // of the keys that the row sees; both, which is NaN, where the score is -infinity and the weight zero
                asm volatile("");                          // (a branch: else every chunk pays for it)
                const int seen = limit - j1 - 4 * g;
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    uint32_t up = 0, down = 0;
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int key = 32 * (block + n) + 8 * (r >> 2) + 4 * g + (r & 3);
                            if (32 * n + 8 * (r >> 2) + (r & 3) <= seen) {
                                const uint32_t u = odd_values[0][key * DT + d], w = odd_values[1][key * DT + d];
                                up |= x[n][r] == -INFINITY ? u | w : u;
                                down |= x[n][r] == -INFINITY ? u | w : w;
                            }
                            if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                        }
                    odd_seen[2 * d][tid] = up;
                    odd_seen[2 * d + 1][tid] = down;
                }
            }
            float most = x[0][0];
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, x[n][r]);
            most = over_blocks<32>(most, MaxOp());
            const bool moves = (most - run_m) * p.scale > 8.0f;   // (of each row for itself: no row's bits depend on another's)
            if (__builtin_expect(__any(moves), 0)) {
                const float m_new = moves ? most : run_m;
                const float keep = !moves ? 1.0f : run_m == -INFINITY ? 0.0f : paged_above_zero(__builtin_amdgcn_exp2f((run_m - m_new) * p.scale));
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[d][r] *= keep;
                run_l *= keep;
                run_m = m_new;
            }
            float ref = run_m == -INFINITY ? 0.0f : run_m * p.scale;         // (a row that has seen nothing yet)
            const float off = kAgain && fabsf(ref) > kPagedLargeScore ? run_m : 0.0f;
            if (kAgain && off != 0.0f) ref = 0.0f;
            const auto exponent = [&](float score) { return fmaf(kAgain ? score - off : score, p.scale, -ref); };
            const auto weights = [&](int n, s16x8 (&w)[PIECES]) __attribute__((always_inline)) {   // of 16 keys
                uint32_t words[PIECES][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float a = __builtin_amdgcn_exp2f(exponent(x[n >> 1][8 * (n & 1) + 2 * j]));
                    const float b = __builtin_amdgcn_exp2f(exponent(x[n >> 1][8 * (n & 1) + 2 * j + 1]));
                    uint32_t two[PIECES];
                    paged_split<PIECES>(a, b, two);
                    // (a sum of the weights that the values are multiplied by: where one weight outweighs the others, its rounding cancels)
                    if constexpr (kBf16) {
                        run_l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two[0]), __builtin_bit_cast(bf16x2, 0x3f803f80u), run_l, false);
                    } else {
                        run_l += a;
                        run_l += b;
                    }
#pragma unroll
                    for (int i = 0; i < PIECES; ++i) words[i][j] = two[i];
                }
#pragma unroll
                for (int i = 0; i < PIECES; ++i) w[i] = __builtin_bit_cast(s16x8, (u32x4{words[i][0], words[i][1], words[i][2], words[i][3]}));
            };
            s16x8 w[2][PIECES];
            weights(0, w[0]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < 2 * NB; ++n) {             // sixteen keys' products beside the next sixteen's weights
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    o[d] = paged_mfma32<PIECES>(v[d], w[n & 1], o[d]);
                    if (n + 1 < 2 * NB) v[d] = read_v(n + 1, d);
                    send_at(kReads + n * DT + d, sure);
                }
                if (n + 1 < 2 * NB) weights(n + 1, w[(n + 1) & 1]);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (kAgain && careful) {                       // (lane and lane + 32 have the row's keys between them)
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (each has read nothing yet of what the other wrote)
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const uint32_t up = (odd_seen[2 * d][tid] | odd_seen[2 * d][tid ^ 32]) >> 4 * g, down = (odd_seen[2 * d + 1][tid] | odd_seen[2 * d + 1][tid ^ 32]) >> 4 * g;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const uint32_t bit = 1u << (8 * (r >> 2) + (r & 3));
                        if (up & bit) o[d][r] += INFINITY;
                        if (down & bit) o[d][r] -= INFINITY;
                        if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        } else {
            req.template send<!kSure>(next, next_at, pieces);
        }
    };
    // A weight's pieces times an infinity add up to NaN, as a weight of zero does, and so do a query's.  So a walk whose sums are not finite is walked again with
    // such keys and values apart throughout.  So is one with a large maximum, whose product with the scale is rounded by as much as exponents count (from 2^31 on beyond fp32's
    // largest): there, row by row, the difference is formed first.  (In every chunk of the first walk that costs 2 % of a long prompt.)
    const auto attempt = [&](auto again) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kDepth - 1; ++i) {
            prepare_if(c0 + i);
            req.template send<true>(next, next_at, pieces);
        }
        run_m = -INFINITY;
        run_l = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
        int chunk = c0;
        if constexpr (!decltype(again)::value) {
            const int plain = min(max(uniform((t.low + 1) / kPagedChunk), c0), c1);
            for (const int sure = min(plain, c1 - (kDepth - 1)); chunk < sure; ++chunk) walk(chunk, std::false_type{}, std::true_type{}, again);
            for (; chunk < plain; ++chunk) walk(chunk, std::false_type{}, std::false_type{}, again);
        }
        for (; chunk < c1; ++chunk) walk(chunk, std::true_type{}, std::false_type{}, again);
    };
    attempt(std::false_type{});
    {
        f32x4 sums = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) sums[r & 3] = fmaf(o[d][r], 0.0f, sums[r & 3]);
        const float any = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        if (any != any || (run_m != -INFINITY && fabsf(run_m * p.scale) > kPagedLargeScore)) odd_sums = 1;
    }
    __syncthreads();
    if (__builtin_expect(uniform(odd_sums), 0)) {
        look(c0);
        if constexpr (KS <= 8) load_rows();                // (again: kept across the first walk they would cost its registers)
        attempt(std::true_type{});
        __syncthreads();
    }
    run_l = over_blocks<32>(run_l, AddOp());
    if (uniform(bad_page)) run_l = NAN;                             // (rows of a sequence whose table names a page that is not there)
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
        if (kw == 0) {
            const float2 other = meet_ml[lane];
            const float m = fmaxf(run_m, other.x);
            const float f0 = paged_factor(run_m, run_l, p.scale, m), f1 = paged_factor(other.x, other.y, p.scale, m);
            run_l = run_l * f0 + other.y * f1;
            run_m = m;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] = o[d][r] * f0 + meet[(d * 16 + r) * 64 + lane] * f1;
        }
    }
    if (t.parts == 1) {
        if (kw || !there) return;
        const int64_t at = paged_row_at(p, t, row);
        const float inv = 1.0f / run_l;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int e = 32 * d + 8 * r + 4 * g;
                if (e < c.head_dim) paged_store<kBf16>(p.out, at + e, f32x4{o[d][4 * r] * inv, o[d][4 * r + 1] * inv, o[d][4 * r + 2] * inv, o[d][4 * r + 3] * inv});
            }
        return;
    }
    // Figures as the lanes have them, a KiB side by side; (maximum, sum) of the rows behind them.
    const int mine = (rw * DT * 256 + lane) * 16, pair = RW * DT * 4096 + row * 8;
    const bool used = rw * 32 < t.rows;                    // uniform
    if (kw == 0 && used) {
        const __amdgpu_buffer_rsrc_t slot = paged_resource(paged_slot(p, t.slot + t.part));
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) paged_leave(slot, mine + (d * 4 + r) * 1024, f32x4{o[d][4 * r], o[d][4 * r + 1], o[d][4 * r + 2], o[d][4 * r + 3]});
        if (g == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(run_m), __float_as_uint(run_l)}, slot, pair, 0, kDeviceScope);
    }
    if (!paged_last(p, t, last_one)) return;               // uniform
    // Pieces of 32 rows by 32 elements, by all waves.  A read is a trip to memory: all parts' maxima in one, the figures of six parts in one
    // (of eight the registers do not hold, and what is fetched from memory waits for all of them: 16 rows of 64 heads on 8 behind 30 000 48.2 us, now 43.3).
    const __amdgpu_buffer_rsrc_t from = paged_resource(paged_slot(p, t.slot));
    constexpr int kSome = 8, kLots = kPagedTileParts / kSome, kFew = 6;
    static_assert(kPagedTileParts % kSome == 0, "whole lots");
    const int pieces_used = (t.rows + 31) / 32 * DT;
#pragma unroll 1
    for (int piece = wave; piece < pieces_used; piece += 4) {
        const int set = piece / DT, d = piece - set * DT, of = set * 32 + l32;
        const int figures = (piece * 256 + lane) * 16, pairs = RW * DT * 4096 + of * 8;
        float2 ml[kPagedTileParts];
#pragma unroll
        for (int b = 0; b < kLots; ++b)
            if (b * kSome < t.parts) {
#pragma unroll
                for (int n = b * kSome; n < (b + 1) * kSome; ++n) ml[n] = paged_read_pair(from, min(n, t.parts - 1) * p.slot_bytes + pairs);
            }
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int b = 0; b < kLots; ++b)
            if (b * kSome < t.parts) {
#pragma unroll
                for (int n = b * kSome; n < (b + 1) * kSome; ++n) m = fmaxf(m, ml[n].x);
            }
        f32x4 sum[4] = {};
#pragma unroll 1
        for (int n0 = 0; n0 < t.parts; n0 += kFew) {
            float2 part[kFew];
            f32x4 x[kFew][4];
#pragma unroll
            for (int n = 0; n < kFew; ++n) {
                const int of_part = min(n0 + n, t.parts - 1) * p.slot_bytes;
                part[n] = paged_read_pair(from, of_part + pairs);
#pragma unroll
                for (int r = 0; r < 4; ++r) x[n][r] = paged_read(from, of_part + figures + r * 1024);
            }
#pragma unroll
            for (int n = 0; n < kFew; ++n) {
                if (n0 + n >= t.parts) continue;
                const float f = paged_factor(part[n].x, part[n].y, p.scale, m);
                l += f * part[n].y;
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] += f * x[n][r];
            }
        }
        if (of >= t.rows) continue;
        const int64_t at = paged_row_at(p, t, of);
        const float inv = 1.0f / l;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int e = 32 * d + 8 * r + 4 * g;
            if (e < c.head_dim) paged_store<kBf16>(p.out, at + e, sum[r] * inv);
        }
    }
}

template <int KS, int PIECES, int RW, int DEPTH = (RW == 4 || KS > 8 ? 2 : 4)>
hipError_t launch_paged_tiles_form(const PagedArgs& p, int64_t wgs, hipStream_t s) {
    using L = PagedTilesLds<KS, RW, DEPTH>;
    static LdsCeiling ceiling;   // per instantiation, i.e. per kernel
    const hipError_t e = ceiling.ensure(reinterpret_cast<const void*>(&paged_tiles_kernel<KS, PIECES, RW, DEPTH>), L::kBytes);
    if (e != hipSuccess) return e;
    paged_tiles_kernel<KS, PIECES, RW, DEPTH><<<dim3((unsigned)wgs), dim3(256), L::kBytes, s>>>(p);
    return hipGetLastError();
}

template <int PIECES, int RW>
hipError_t launch_paged_tiles_width(const PagedArgs& p, int64_t wgs, hipStream_t s) {
    switch (paged_width(p.c.head_dim)) {
        case 32: return launch_paged_tiles_form<2, PIECES, RW>(p, wgs, s);
        case 48: return launch_paged_tiles_form<3, PIECES, RW>(p, wgs, s);
        case 64: return launch_paged_tiles_form<4, PIECES, RW>(p, wgs, s);
        case 96:
            if constexpr (PIECES == 1 && RW == 2)
                if (p.shallow) return launch_paged_tiles_form<6, PIECES, RW, 2>(p, wgs, s);
            return launch_paged_tiles_form<6, PIECES, RW>(p, wgs, s);
        case 128:
            if constexpr (PIECES == 1 && RW == 2)
                if (p.shallow) return launch_paged_tiles_form<8, PIECES, RW, 2>(p, wgs, s);
            return launch_paged_tiles_form<8, PIECES, RW>(p, wgs, s);
        case 192: return launch_paged_tiles_form<12, PIECES, RW>(p, wgs, s);
        case 256: return launch_paged_tiles_form<16, PIECES, RW>(p, wgs, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace bl
