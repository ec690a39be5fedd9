// bl_attn_paged for few rows: sequences with up to sixteen rows (tokens x query heads) per key head -- one token of every sequence, as a rule.
//
// Bound by the cache's bytes: 4 head_dim bytes per position and key head for at most 64 products each, a hundredth of what the matrix cores do
// meanwhile.  So the launch is about spreading the positions of all sequences evenly over the chip and keeping enough requests under way.
//   * Every sequence's walk is cut into equal parts of about (all positions) / (workgroups), 256 positions at least; which part a workgroup has
//     follows from the positions on the device (paged_find), so that a captured launch serves any lengths.  The grid is an upper bound;
//     workgroups without a part end at once.
//   * A workgroup's four waves take its 32-position chunks in turn, each with a tile of keys and one of values of its own in LDS that it fills
//     and waits for by itself: the next chunk's keys are requested when the scores are formed, its values when the sums are.
//   * Scores are formed transposed, S^T = K Q^T (v_mfma_f32_16x16x32_bf16): a lane has eight of the chunk's weights of ONE row, already laid out as
//     the operand of O^T += V^T P^T, V^T by the transposing LDS read.  The contraction index runs over the positions in the order of the
//     result registers: slots 0..3 of lane group g are positions 4 g .. 4 g + 3, slots 4..7 positions 16 + 4 g .. 16 + 4 g + 3.
//   * fp32 queries and weights enter as three bf16 numbers each, their sum (three products; the operator is bound by memory all the same);
//     bf16 queries as they are, and their weights rounded to bf16: at most 2^-8 of a weight, as much as the output's own rounding.
//   * Running maxima and sums are fp32; the parts of a walk meet in scratch memory in their order, and the workgroup that draws a row's last
//     ticket adds them up.  Nobody waits for anybody.
#include "bl_paged.hpp"
#include "bl_figures.hpp"

namespace bl {

namespace {

constexpr int kWaves = 4;

template <int KS>
struct RowsLds {
    static constexpr int kWidth = 16 * KS;
    static constexpr int kRing = kWaves * 2 * PagedTile<KS>::kBytes;
    static constexpr int kPitch = kWidth + 4;                           // floats of a row where the waves meet
    static constexpr int kMeet = kWaves * kPagedFew * (kPitch * 4 + 8);
    static constexpr int kFactors = kPagedFew * kPagedMostSplits * 8;   // the parts' factors
    static constexpr int kBytes = kRing > kMeet ? (kRing > kFactors ? kRing : kFactors) : (kMeet > kFactors ? kMeet : kFactors);
    static_assert(kBytes <= kMaxDecodeLds, "fits the LDS ceiling");
};

template <int PIECES>
__device__ __forceinline__ f32x4 mfma16(const s16x8& a, const s16x8 (&b)[PIECES], f32x4 c) {
#pragma unroll
    for (int i = PIECES - 1; i >= 0; --i)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b[i]), c, 0, 0, 0);
    return c;
}

// The positions of a part of a walk, in chunks of 32: a walk of so many positions has so many parts.
__device__ __forceinline__ int rows_parts(int walked, int per) { return walked > 0 ? min((walked - 1) / per + 1, kPagedMostSplits) : 0; }

template <int KS, int PIECES>
__global__ __launch_bounds__(64 * kWaves) void paged_rows_kernel(const PagedArgs p) {
    using L = RowsLds<KS>;
    using T = PagedTile<KS>;
    constexpr bool kBf16 = PIECES == 1;
    constexpr int kSteps = (KS + 1) / 2;                   // of 32 elements
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ int last_one;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, g = lane >> 4;
    const Paged& c = p.c;

    // ---- whose part of which walk
    const int each = (int)blockIdx.x / c.n_heads, head = (int)blockIdx.x - each * c.n_heads;
    const auto walked = [&](const PagedSequence& s) { return s.rows > 0 && s.rows * (int64_t)p.group <= p.few ? s.pos + s.rows : 0; };
    float total = 0.0f;
    if (c.sequences == 1) {
        total = (float)walked(paged_sequence_uniform(c, 0));
    } else {
        const int lanes = (c.sequences + 63) >> 6;
        for (int i = 0; i < lanes; ++i)
            if (lane * lanes + i < c.sequences) total += (float)walked(paged_sequence(c, lane * lanes + i));
        total = over_lanes<64>(total, AddOp());
    }
    // (a little more than the quotient, so that the parts are never more than the grid: see paged_rows_grid)
    const int per = max(kPagedLeast, (int)fminf(total * p.target * 1.0001f, 2.0e9f) + 1);
    int b, part, before;
    PagedSequence s;
    if (!paged_find(c, lane, each, [&](const PagedSequence& q) { return rows_parts(walked(q), per); }, b, part, before, s)) return;
    const int reach = s.pos + s.rows, parts = rows_parts(reach, per), chunks = (reach + 31) >> 5;
    const int c0 = (int)((int64_t)chunks * part / parts), c1 = (int)((int64_t)chunks * (part + 1) / parts);
    const int rows = s.rows * p.group;
    const int32_t* line = c.table + (int64_t)b * c.table_width;

    // ---- requests
    uint8_t* tile = lds + wave * 2 * T::kBytes;
    const uint32_t at_k = __builtin_amdgcn_readfirstlane(lds_address(tile)), at_v = at_k + T::kBytes;
    PagedRequest<KS> req_k, req_v;
    req_k.template prepare<false>(lane);
    req_v.template prepare<true>(lane);
    int chunk = c0 + wave;
    PagedBase base{{0, 0}, false};
    if (chunk < c1) {
        base = paged_base<KS>(c, line, head, 32 * chunk, reach - 1);
        req_k.template send<false>(c.k, base, at_k, reach - 1 - 32 * chunk, lane);
        req_v.template send<true>(c.v, base, at_v, reach - 1 - 32 * chunk, lane);
    }

    // ---- the rows: operand column i16
    const int token = i16 / p.group;
    const bool there = i16 < rows;
    const int64_t row_at = ((int64_t)(s.first + token) * c.n_heads + head) * p.group * c.head_dim + (int64_t)(i16 - token * p.group) * c.head_dim;
    const int limit = s.pos + token;                       // the last position that the row sees
    s16x8 q[kSteps][PIECES];
#pragma unroll
    for (int t = 0; t < kSteps; ++t) paged_query<PIECES>(p.q, row_at, 32 * t + 8 * g, c.head_dim, there, q[t]);

    f32x4 o[KS];
    float run_m = -INFINITY, run_l = 0.0f;                 // run_l: over this lane group's positions only
#pragma unroll
    for (int t = 0; t < KS; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (; chunk < c1; chunk += kWaves) {
        const int j0 = 32 * chunk, next = chunk + kWaves;
        const bool bad = base.bad, masked = j0 + 31 > s.pos;     // uniform
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
                x[h] = mfma16<PIECES>(k, q[t], x[h]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // every key has left the tile
        if (next < c1) {
            base = paged_base<KS>(c, line, head, 32 * next, reach - 1);
            req_k.template send<false>(c.k, base, at_k, reach - 1 - 32 * next, lane);
            wait_vm<KS>();                                 // values are here
        } else {
            wait_vm<0>();
        }
        if (masked) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (j0 + 16 * h + 4 * g + r > limit) x[h][r] = -INFINITY;
        }
        if (bad) x[0] = x[1] = f32x4{NAN, NAN, NAN, NAN};
        float most = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
        most = over_blocks<32>(over_blocks<16>(most, MaxOp()), MaxOp());
        const float m_new = fmaxf(run_m, most);
        const float ref = m_new == -INFINITY ? 0.0f : m_new * p.scale;   // (a row that has seen nothing yet)
        const float keep = run_m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(fmaf(run_m, p.scale, -ref));
        run_m = m_new;
        run_l *= keep;
        uint32_t w[PIECES][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                const float u = __builtin_amdgcn_exp2f(fmaf(x[h][r], p.scale, -ref)), v = __builtin_amdgcn_exp2f(fmaf(x[h][r + 1], p.scale, -ref));
                run_l += u;
                run_l += v;
                uint32_t two[PIECES];
                paged_split<PIECES>(u, v, two);
#pragma unroll
                for (int i = 0; i < PIECES; ++i) w[i][2 * h + (r >> 1)] = two[i];
            }
        s16x8 weights[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) weights[i] = __builtin_bit_cast(s16x8, (u32x4{w[i][0], w[i][1], w[i][2], w[i][3]}));

        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const uint8_t* values = tile + T::kBytes;
        const auto read_v = [&](int t) {
            const int key = 4 * g + (i16 >> 2), piece = 2 * t + ((i16 >> 1) & 1);
            const uint8_t* at = values + key * T::kRow + paged_v_place<KS>(key, piece) * 16 + (i16 & 1) * 8;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
            const s16x4 e = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * T::kRow));
            return s16x8{a[0], a[1], a[2], a[3], e[0], e[1], e[2], e[3]};
        };
        if (!masked) {
#pragma unroll
            for (int t = 0; t < KS; ++t) o[t] = mfma16<PIECES>(read_v(t), weights, o[t] * keep);
        } else {
            // The end of the walk.  What lies behind the sequence's last row is nobody's (zero here); among several tokens' rows a weight of
            // zero may stand before a value that the row does not see: infinities and NaN are counted apart, by whom they weigh with.
            s16x8 mine;                                    // of the operand: positions that the sequence has
#pragma unroll
            for (int r = 0; r < 8; ++r) mine[r] = j0 + (r < 4 ? 0 : 16) + 4 * g + (r & 3) < reach ? (short)-1 : (short)0;
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                const s16x8 v = read_v(t) & mine;
                s16x8 finite, up, down;
                paged_put_away(v, finite, up, down);
                f32x4 x_t = mfma16<PIECES>(finite, weights, o[t] * keep);
                const s16x8 either = up | down;
                const u32x4 any = __builtin_bit_cast(u32x4, either);
                if (__any((any[0] | any[1] | any[2] | any[3]) != 0)) {
                    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                    const f32x4 n_up = mfma16<PIECES>(up, weights, zero), n_down = mfma16<PIECES>(down, weights, zero);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (n_up[r] > 0.0f) x_t[r] += INFINITY;
                        if (n_down[r] > 0.0f) x_t[r] -= INFINITY;
                    }
                }
                o[t] = x_t;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (next < c1) req_v.template send<true>(c.v, base, at_v, reach - 1 - 32 * next, lane);
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
    const auto out_at = [&](int r, int e) {
        const int of = r / p.group;
        return ((int64_t)(s.first + of) * c.n_heads + head) * p.group * c.head_dim + (int64_t)(r - of * p.group) * c.head_dim + e;
    };
    const int stride = 1 + c.head_dim / 2;                 // pairs of a row's figures: (maximum, sum), then the values
    const auto figures_of = [&](int n, int r) {            // part n of this walk
        return reinterpret_cast<float2*>(p.figures) + (((int64_t)(before + n) * c.n_heads + head) * p.slot_rows + r) * stride;
    };
    for (int i = tid; i < rows * quads; i += 64 * kWaves) {
        const int r = i / quads, e = 4 * (i - r * quads);
        float2 ml[kWaves];
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            ml[w] = meet_ml[w * kPagedFew + r];
            m = fmaxf(m, ml[w].x);
        }
        const float ref = m == -INFINITY ? 0.0f : m * p.scale;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = ml[w].x == -INFINITY ? (ml[w].y == 0.0f ? 0.0f : NAN) : __builtin_amdgcn_exp2f(fmaf(ml[w].x, p.scale, -ref));
            if (ml[w].y == 0.0f) continue;                 // (a wave that had no chunk, or none that the row sees)
            l += f * ml[w].y;
            sum += f * *reinterpret_cast<const f32x4*>(meet + (w * kPagedFew + r) * L::kPitch + e);
        }
        if (parts == 1) {
            paged_store<kBf16>(p.out, out_at(r, e), sum / l);
        } else {
            float2* dst = figures_of(part, r);
            leave_figure(dst + 1 + (e >> 1), sum[0], sum[1]);
            leave_figure(dst + 2 + (e >> 1), sum[2], sum[3]);
            if (e == 0) leave_figure(dst, m, l);
        }
    }
    if (parts == 1) return;                                // uniform

    // ---- the walk's parts meet: figures travel by device-scope stores, every thread waits until its own have been performed, then the ticket
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    uint32_t* counter = p.counters + (int64_t)b * c.n_heads + head;
    if (tid == 0) last_one = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(parts - 1);
    __syncthreads();
    if (!last_one) return;                                 // uniform
    float2* factor = reinterpret_cast<float2*>(lds);       // [row][part]: (maximum, sum), then (factor, -)
    for (int i = tid; i < rows * parts; i += 64 * kWaves) {
        const int r = i / parts;
        factor[i] = read_figure(figures_of(i - r * parts, r));
    }
    __syncthreads();
    for (int r = wave; r < rows; r += kWaves) {
        float2* mine = factor + r * parts;
        float m = -INFINITY, l = 0.0f;
        for (int n = lane; n < parts; n += 64) m = fmaxf(m, mine[n].x);
        m = over_lanes<64>(m, MaxOp());
        const float ref = m == -INFINITY ? 0.0f : m * p.scale;
        const auto factor_of = [&](const float2& f) {      // (a part that the row sees nothing of: nothing)
            return f.x == -INFINITY ? (f.y == 0.0f ? 0.0f : NAN) : __builtin_amdgcn_exp2f(fmaf(f.x, p.scale, -ref));
        };
        for (int n = lane; n < parts; n += 64) l += factor_of(mine[n]) * mine[n].y;
        l = over_lanes<64>(l, AddOp());
        for (int n = lane; n < parts; n += 64) mine[n].x = factor_of(mine[n]) / l;
    }
    __syncthreads();
    const int halves = c.head_dim >> 1, pairs = rows * halves;
    // threads in teams, a team's share of the parts each, where there are fewer outputs than threads
    const int teams = max(1, 64 * kWaves / pairs);
    float2* sums = factor + kPagedFew * kPagedMostSplits - 64 * kWaves;   // (teams > 1: few rows, whose factors end far ahead)
    for (int i0 = 0; i0 < pairs; i0 += 64 * kWaves) {
        const int team = teams > 1 ? tid / pairs : 0, i = teams > 1 ? tid - team * pairs : i0 + tid;
        const int r = min(i, pairs - 1) / halves, e = min(i, pairs - 1) - r * halves;
        float2 sum = make_float2(0.0f, 0.0f);
        if (team < teams && i < pairs) {
            constexpr int kAhead = 8;
            for (int n0 = team; n0 < parts; n0 += kAhead * teams) {
                float2 a[kAhead];
#pragma unroll
                for (int h = 0; h < kAhead; ++h) a[h] = read_figure(figures_of(min(n0 + h * teams, parts - 1), r) + 1 + e);
#pragma unroll
                for (int h = 0; h < kAhead; ++h) {
                    const int n = n0 + h * teams;
                    if (n >= parts) continue;
                    const float2 f = factor[r * parts + n];
                    if (f.y == 0.0f && f.x == f.x) continue;   // (a part that the row sees nothing of)
                    sum.x += f.x * a[h].x;
                    sum.y += f.x * a[h].y;
                }
            }
        }
        if (teams > 1) {
            __syncthreads();
            sums[tid] = sum;
            __syncthreads();
            if (tid >= pairs) break;
            sum = make_float2(0.0f, 0.0f);
            for (int t = 0; t < teams; ++t) {
                sum.x += sums[t * pairs + tid].x;
                sum.y += sums[t * pairs + tid].y;
            }
        }
        if (i < pairs && team == 0) {
            if constexpr (kBf16) *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + out_at(r, 2 * e)) = paged_bf16_pair(sum.x, sum.y);
            else *reinterpret_cast<float2*>(static_cast<float*>(p.out) + out_at(r, 2 * e)) = sum;
        }
    }
    if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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
