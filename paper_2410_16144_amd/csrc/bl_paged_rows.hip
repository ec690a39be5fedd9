// bl_attn_paged for few rows: sequences with up to sixteen rows (tokens x query heads) per key head -- one token of every sequence, as a rule.
//
// Bound by the cache's bytes: 4 head_dim bytes per position and key head for at most 64 products each, a hundredth of what the matrix cores do
// meanwhile.  So the launch is about spreading the positions of all sequences evenly over the chip and keeping enough requests under way.
//   * Every sequence's walk is cut into equal parts of about (all positions) / (workgroups), 256 positions at least; which part a workgroup has
//     follows from the positions on the device (paged_work), so that a captured launch serves any lengths.  The grid is an upper bound;
//     workgroups without a part end at once.
//   * A workgroup's four waves take its 32-position chunks in turn, each with a tile of keys and one of values of its own in LDS that it fills
//     and waits for by itself: the next chunk's keys are requested when the scores are formed, its values when the sums are.  Streaming loads, since
//     nothing is read twice (32 heads of 128, ordinary and streaming, us: 8000 positions 33.1 and 30.4, 32 000 98.0 and 87.8, 5.4 and 6.0 TB/s;
//     500 to 4000 positions the same).
//   * Scores are formed transposed, S^T = K Q^T (v_mfma_f32_16x16x32_bf16): a lane has eight of the chunk's weights of ONE row, already laid out as
//     the operand of O^T += V^T P^T, V^T by the transposing LDS read.  The contraction index runs over the positions in the order of the
//     result registers: slots 0..3 of lane group g are positions 4 g .. 4 g + 3, slots 4..7 positions 16 + 4 g .. 16 + 4 g + 3.
//   * fp32 queries and weights enter as three bf16 numbers each, their sum (three products; the operator is bound by memory all the same); bf16
//     queries as they are, and their weights as two: off by at most 2^-16 of a weight, far below the output's rounding.
//   * Running maxima and sums are fp32; the parts of a walk meet in scratch memory in their order, and the workgroup that draws a row's last
//     ticket adds them up.  Nobody waits for anybody.
#include <type_traits>

#include "bl_paged.hpp"

namespace bl {

namespace {

constexpr int kWaves = 4;

constexpr int kMostParts = 256;

template <int KS>
struct RowsLds {
    static constexpr int kWidth = 16 * KS;
    static constexpr int kRing = kWaves * 2 * PagedTile<KS>::kBytes;
    static constexpr int kPitch = kWidth + 4;                           // floats of a row where the waves meet
    static constexpr int kMeet = kWaves * kPagedFew * (kPitch * 4 + 8);
    static constexpr int kJoin = kPagedFew * kMostParts * 8 + 256 * 16; // the parts' factors, and the teams' sums
    static constexpr int kMore = kMeet > kJoin ? kMeet : kJoin;
    static constexpr int kBytes = kRing > kMore ? kRing : kMore;
    static_assert(kBytes <= kMaxDecodeLds, "fits the LDS ceiling");
};

template <int PIECES>
__device__ __forceinline__ f32x4 mfma16(const s16x8& a, const s16x8 (&b)[PIECES], f32x4 c) {
#pragma unroll
    for (int i = PIECES - 1; i >= 0; --i)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b[i]), c, 0, 0, 0);
    return c;
}

// A slot's row: (maximum, sum), two words of padding, the weighted values.
__device__ __forceinline__ int figure_at(int head_dim, int row, int word) { return (row * (4 + head_dim) + word) * 4; }

// After every thread has left its figures.  factor: LDS of rows * parts pairs, sums of 256 quads; store(row, e, x): four outputs.
template <typename Store>
__device__ __forceinline__ void join_parts(const PagedArgs& p, const PagedWork& w, float2* factor, f32x4* sums, int& last_one, const Store& store) {
    constexpr int kThreads = 256, kAhead = 32;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (!paged_last(p, w, last_one)) return;               // uniform
    const int d = p.c.head_dim, quads = d >> 2, total = w.rows * quads, parts = w.parts;
    const __amdgpu_buffer_rsrc_t from = paged_resource(paged_slot(p, w.slot));
    const int teams = max(1, kThreads / total);            // that share an output's parts, where there are few outputs
    const int team = teams > 1 ? tid / total : 0;
    f32x4 a[kAhead];
    const auto read = [&](int i, int n0) {                 // output quad i of parts n0 + team, n0 + team + teams, ...
        const int row = i / quads, at = figure_at(d, row, 4 + 4 * (i - row * quads));
#pragma unroll
        for (int h = 0; h < kAhead; ++h)
            if (h % 4 || n0 + h * teams < parts)           // (by fours)
                a[h] = paged_read(from, min(n0 + team + h * teams, parts - 1) * p.slot_bytes + at);
            else
                break;
    };
    const int i0 = teams > 1 ? tid - team * total : tid;
    const int pairs = w.rows * parts;                      // [row][part]; most often a few each
    constexpr int kPairs = 4;
    float2 ml[kPairs];
#pragma unroll
    for (int h = 0; h < kPairs; ++h) {
        const int i = min(tid + h * kThreads, pairs - 1), row = i / parts;
        ml[h] = paged_read_pair(from, (i - row * parts) * p.slot_bytes + figure_at(d, row, 0));
    }
    read(min(i0, total - 1), 0);                           // (the first of the values travel with the maxima and sums)
#pragma unroll
    for (int h = 0; h < kPairs; ++h)
        if (tid + h * kThreads < pairs) factor[tid + h * kThreads] = ml[h];
    for (int i = tid + kPairs * kThreads; i < pairs; i += kThreads) {
        const int row = i / parts;
        factor[i] = paged_read_pair(from, (i - row * parts) * p.slot_bytes + figure_at(d, row, 0));
    }
    __syncthreads();
    for (int row = wave; row < w.rows; row += kThreads / 64) {
        float2* mine = factor + row * parts;
        float m = -INFINITY, l = 0.0f;
        for (int n = lane; n < parts; n += 64) m = fmaxf(m, mine[n].x);
        m = over_lanes<64>(m, MaxOp());
        for (int n = lane; n < parts; n += 64) l += paged_factor(mine[n].x, mine[n].y, p.scale, m) * mine[n].y;
        l = over_lanes<64>(l, AddOp());
        for (int n = lane; n < parts; n += 64) {
            const float f = paged_factor(mine[n].x, mine[n].y, p.scale, m), share = f / l;
            mine[n].x = f == 0.0f ? share : paged_above_zero(share);
        }
    }
    __syncthreads();
    for (int i = i0; i < total; i += kThreads) {
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        const int row = i / quads;
        if (team < teams)
            for (int n0 = 0; n0 < parts; n0 += kAhead * teams) {
                if (n0 || i != i0) read(i, n0);
#pragma unroll
                for (int h = 0; h < kAhead; ++h) {
                    if (h % 4 == 0 && n0 + h * teams >= parts) break;
                    const int n = n0 + team + h * teams;
                    if (n < parts) sum += factor[row * parts + n].x * a[h];
                }
            }
        if (teams > 1) {                                   // (all outputs in one turn)
            if (team < teams) sums[tid] = sum;
            break;
        }
        store(row, 4 * (i - row * quads), sum);
    }
    if (teams > 1) {                                       // uniform
        __syncthreads();
        if (tid < total) {
            f32x4 sum = sums[tid];
            for (int t = 1; t < teams; ++t) sum += sums[t * total + tid];
            const int row = tid / quads;
            store(row, 4 * (tid - row * quads), sum);
        }
    }
}

template <int KS, int PIECES>
__global__ __launch_bounds__(64 * kWaves) void paged_rows_kernel(const PagedArgs p) {
    using L = RowsLds<KS>;
    using T = PagedTile<KS>;
    constexpr bool kBf16 = PIECES == 1;
    constexpr int kWeight = kBf16 ? 2 : 3;                 // pieces of a weight
    constexpr int kSteps = (KS + 1) / 2;                   // of 32 elements
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ int last_one;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, g = lane >> 4;
    const Paged& c = p.c;

    PagedWork w;
    if (!paged_work<true>(p, lane, w)) return;
    const PagedSequence& s = w.s;
    const int reach = w.reach, chunks = (reach + 31) >> 5, head = w.head, rows = w.rows;
    const int c0 = paged_first(w, chunks, w.part), c1 = paged_first(w, chunks, w.part + 1);
    const int32_t* line = c.table + (int64_t)w.b * c.table_width;

    // ---- the rows: operand column i16
    const bool there = i16 < rows;
    const int64_t row_at = there ? paged_row_at(p, w, i16) : 0;
    const int limit = reach - 1;                           // the last position that is seen, by columns without a row too: what lies behind it is no reason to walk again
    s16x8 q[kSteps][PIECES];
#pragma unroll
    for (int t = 0; t < kSteps; ++t) paged_query<PIECES>(p.q, row_at, 32 * t + 8 * g, c.head_dim, there, q[t]);

    // ---- requests
    uint8_t* tile = lds + wave * 2 * T::kBytes;
    const uint32_t at_k = __builtin_amdgcn_readfirstlane(lds_address(tile)), at_v = at_k + T::kBytes;
    PagedRequest<KS, true> req_k, req_v;
    req_k.template prepare<false>(lane);
    req_v.template prepare<true>(lane);
    int chunk;
    PagedBase base{{0, 0}, false};
    PagedEntries entries{{0, 0}};
    f32x4 o[KS];
    float run_m, run_l;                                    // run_l: over this lane group's positions only
    const auto begin = [&]() __attribute__((always_inline)) {
        chunk = c0 + wave;
        if (chunk < c1) {
            const PagedEntries first = paged_entries(c, line, 32 * chunk, reach - 1);
#pragma unroll
            for (int t = 0; t < kSteps; ++t)
#pragma unroll
                for (int n = 0; n < PIECES; ++n) asm volatile("" : "+v"(q[t][n]));   // (the rows arrive while the table is looked at: no wait of theirs later)
            base = paged_base<KS>(c, first, head, 32 * chunk, reach - 1);
            entries = paged_entries(c, line, 32 * (chunk + kWaves), reach - 1);
            req_k.send(paged_source(c.k, base), at_k);
            req_v.send(paged_source(c.v, base), at_v);
        }
        run_m = -INFINITY;
        run_l = 0.0f;
#pragma unroll
        for (int t = 0; t < KS; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    };

    // Chunks that the sequence has whole, then its last one.  (The first kind's code lies side by side: jumps cost as much as products.)
    const auto walk = [&](auto which, bool careful) __attribute__((always_inline)) {
        constexpr bool kMasked = decltype(which)::value;
        const int j0 = 32 * chunk, next = chunk + kWaves;
        const bool bad = base.bad;                         // uniform
        wait_vm<KS>();                                     // keys are here; the values may be on their way
        f32x4 x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            x[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            const int row = 16 * h + i16;
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                s16x8 k = {0, 0, 0, 0, 0, 0, 0, 0};
                if (KS % 2 == 0 || t + 1 < kSteps || g < 2)
                    k = *reinterpret_cast<const s16x8*>(tile + row * T::kRow + paged_k_place<KS>(row, 4 * t + g) * 16);
                if (kMasked && !kBf16 && careful) {        // uniform
                    s16x8 finite, odd;
                    paged_apart(k, finite, odd);
                    x[h] = mfma16<PIECES>(finite, q[t], x[h]);
                    const u32x4 any = __builtin_bit_cast(u32x4, odd);
                    if (__any((any[0] | any[1] | any[2] | any[3]) != 0)) {
                        const s16x8 signs[1] = {paged_signs<PIECES>(q[t])};
                        x[h] = mfma16<1>(odd, signs, x[h]);
                    }
                } else {
                    x[h] = mfma16<PIECES>(k, q[t], x[h]);
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // every key has left the tile
        if (next < c1) {
            base = paged_base<KS>(c, entries, head, 32 * next, reach - 1);
            entries = paged_entries(c, line, 32 * (next + kWaves), reach - 1);
            req_k.send(paged_source(c.k, base), at_k);
            wait_vm<KS>();                                 // values are here
        } else {
            wait_vm<0>();
        }
        if constexpr (kMasked) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (j0 + 16 * h + 4 * g + r > limit) x[h][r] = -INFINITY;
        }
        if (__builtin_expect(bad, 0)) x[0] = x[1] = f32x4{NAN, NAN, NAN, NAN};
        float most = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
        most = over_blocks<32>(over_blocks<16>(most, MaxOp()), MaxOp());
        const float m_new = fmaxf(run_m, most);
        // (The difference first: a maximum of 2^31 or more, rounded after its product with the scale, makes exponents beyond fp32's of its own weight.)
        const float top = m_new == -INFINITY ? 0.0f : m_new;             // (a row that has seen nothing yet)
        float keep = run_m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((run_m - top) * p.scale);
        if (kMasked && careful) keep = paged_above_zero(keep);
        run_m = m_new;
        run_l *= keep;
        uint32_t words[kWeight][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                const float u = __builtin_amdgcn_exp2f((x[h][r] - top) * p.scale), v = __builtin_amdgcn_exp2f((x[h][r + 1] - top) * p.scale);
                run_l += u;
                run_l += v;
                uint32_t two[kWeight];
                paged_split<kWeight>(u, v, two);
#pragma unroll
                for (int i = 0; i < kWeight; ++i) words[i][2 * h + (r >> 1)] = two[i];
            }
        s16x8 weights[kWeight];
#pragma unroll
        for (int i = 0; i < kWeight; ++i) weights[i] = __builtin_bit_cast(s16x8, (u32x4{words[i][0], words[i][1], words[i][2], words[i][3]}));

        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const uint8_t* values = tile + T::kBytes;
        const auto read_v = [&](int t) {
            const int key = 4 * g + (i16 >> 2), piece = 2 * t + ((i16 >> 1) & 1);
            const uint8_t* at = values + key * T::kRow + paged_v_place<KS>(key, piece) * 16 + (i16 & 1) * 8;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
            const s16x4 e = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * T::kRow));
            return s16x8{a[0], a[1], a[2], a[3], e[0], e[1], e[2], e[3]};
        };
        if constexpr (!kMasked) {
#pragma unroll
            for (int t = 0; t < KS; ++t) o[t] = mfma16<kWeight>(read_v(t), weights, o[t] * keep);
        } else {
            // The end of the walk: what lies behind the sequence's last row is nobody's (zero here).
            s16x8 mine;                                    // of the operand: positions that the sequence has
#pragma unroll
            for (int r = 0; r < 8; ++r) mine[r] = j0 + (r < 4 ? 0 : 16) + 4 * g + (r & 3) < reach ? (short)-1 : (short)0;
            s16x8 seen[1], lost[1];                        // one where the row sees the position; where its score is -infinity
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                seen[0][r] = mine[r] & (short)0x3f80;
                lost[0][r] = x[r >> 2][r & 3] == -INFINITY ? seen[0][r] : (short)0;
            }
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                const s16x8 v = read_v(t) & mine;
                if (!careful) {                            // uniform
                    o[t] = mfma16<kWeight>(v, weights, o[t] * keep);
                    continue;
                }
                s16x8 finite, up, down;
                paged_put_away(v, finite, up, down);
                f32x4 x_t = mfma16<kWeight>(finite, weights, o[t] * keep);
                const s16x8 either = up | down;
                const u32x4 any = __builtin_bit_cast(u32x4, either);
                if (__any((any[0] | any[1] | any[2] | any[3]) != 0)) {
                    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                    const f32x4 n_up = mfma16<1>(up, seen, zero), n_down = mfma16<1>(down, seen, zero), n_lost = mfma16<1>(either, lost, zero);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (n_up[r] > 0.0f) x_t[r] += INFINITY;
                        if (n_down[r] > 0.0f) x_t[r] -= INFINITY;
                        if (n_lost[r] > 0.0f) x_t[r] = NAN;
                    }
                }
                o[t] = x_t;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (next < c1) req_v.send(paged_source(c.v, base), at_v);
        chunk = next;
    };
    // The pieces of a weight times an infinity add up to NaN, and so do a weight that is rounded to zero and the pieces of a query.  So a walk whose sums are not
    // finite is walked again with such keys and values apart throughout: a value counts by who sees it, not by what is left of its weight.
    for (bool again = false;; again = true) {
        begin();
        if (!again && chunk < c1 && 32 * chunk + 31 <= s.pos)
            do walk(std::false_type{}, false);
            while (chunk < c1 && 32 * chunk + 31 <= s.pos);
        while (chunk < c1) walk(std::true_type{}, again);
        if (again) break;
        f32x4 odd = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) odd[r] = fmaf(o[t][r], 0.0f, odd[r]);
        const float any = (odd[0] + odd[1]) + (odd[2] + odd[3]);
        if (!__any(any != any)) break;
    }

    // ---- the waves meet
    run_l = over_blocks<32>(over_blocks<16>(run_l, AddOp()), AddOp());
    __syncthreads();                                       // the tiles are done with
    float* meet = reinterpret_cast<float*>(lds);           // [wave][row][element]
    float2* meet_ml = reinterpret_cast<float2*>(meet + kWaves * kPagedFew * L::kPitch);
    if (g == 0) meet_ml[wave * kPagedFew + i16] = make_float2(run_m, run_l);
#pragma unroll
    for (int t = 0; t < KS; ++t) *reinterpret_cast<f32x4*>(meet + (wave * kPagedFew + i16) * L::kPitch + 16 * t + 4 * g) = o[t];
    __syncthreads();
    const int quads = c.head_dim >> 2;
    const __amdgpu_buffer_rsrc_t slot = paged_resource(paged_slot(p, w.slot + w.part));
    const auto store = [&](int r, int e, const f32x4& x) { paged_store<kBf16>(p.out, paged_row_at(p, w, r) + e, x); };
    for (int i = tid; i < rows * quads; i += 64 * kWaves) {
        const int r = i / quads, e = 4 * (i - r * quads);
        float2 ml[kWaves];
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int n = 0; n < kWaves; ++n) {
            ml[n] = meet_ml[n * kPagedFew + r];
            m = fmaxf(m, ml[n].x);
        }
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int n = 0; n < kWaves; ++n) {
            const float f = paged_factor(ml[n].x, ml[n].y, p.scale, m);
            l += f * ml[n].y;
            sum += f * *reinterpret_cast<const f32x4*>(meet + (n * kPagedFew + r) * L::kPitch + e);
        }
        if (w.parts == 1) {
            store(r, e, sum / l);
        } else {
            paged_leave(slot, figure_at(c.head_dim, r, 4 + e), sum);
            if (e == 0) paged_leave(slot, figure_at(c.head_dim, r, 0), f32x4{m, l, 0.0f, 0.0f});
        }
    }
    if (w.parts == 1) return;                              // uniform
    float2* factor = reinterpret_cast<float2*>(lds);
    join_parts(p, w, factor, reinterpret_cast<f32x4*>(factor + kPagedFew * kMostParts), last_one, store);
}

template <int KS, int PIECES>
hipError_t launch_rows(const PagedArgs& p, int64_t wgs, hipStream_t s) {
    using L = RowsLds<KS>;
    static LdsCeiling ceiling;
    const hipError_t e = ceiling.ensure(reinterpret_cast<const void*>(&paged_rows_kernel<KS, PIECES>), L::kBytes);
    if (e != hipSuccess) return e;
    paged_rows_kernel<KS, PIECES><<<dim3((unsigned)wgs), dim3(64 * kWaves), L::kBytes, s>>>(p);
    return hipGetLastError();
}

template <int PIECES>
hipError_t launch_width(const PagedArgs& p, int64_t wgs, hipStream_t s) {
    switch (paged_width(p.c.head_dim)) {
        case 32: return launch_rows<2, PIECES>(p, wgs, s);
        case 48: return launch_rows<3, PIECES>(p, wgs, s);
        case 64: return launch_rows<4, PIECES>(p, wgs, s);
        case 96: return launch_rows<6, PIECES>(p, wgs, s);
        case 128: return launch_rows<8, PIECES>(p, wgs, s);
        case 192: return launch_rows<12, PIECES>(p, wgs, s);
        case 256: return launch_rows<16, PIECES>(p, wgs, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_paged_rows(const PagedArgs& p, bool bf16, int64_t wgs, hipStream_t s) {
    return bf16 ? launch_width<1>(p, wgs, s) : launch_width<3>(p, wgs, s);
}

}  // namespace bl
