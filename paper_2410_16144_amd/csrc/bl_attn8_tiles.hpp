// The tiles form of the attention over 8-bit caches: 32 rows (token, query head) that read one key head, against 32 positions at a time.
//
// A workgroup's four waves share out the 32-position halves of chunks and merge their running maxima, sums and outputs at the end (SETS = 4), or
// have two or four tiles of 32 rows, with two waves or one for each: a long prompt has workgroups enough, and what a tile costs beside its
// halves -- its queries' way into the operands, the meeting -- is paid less often per half (32 heads of 128, 1024 tokens, one tile and two: 47.6 and
// 42.8 us).  A wave brings its own operands and waits for nobody.  Every operand comes from memory as it lies there (bl_kv8.hpp), 16 bytes per
// lane: no LDS, no transposition.
//
// Scores are formed transposed, S^T = K Q^T, by v_mfma_i32_32x32x32_i8 on the codes, with the queries as three signed bytes each (24-bit
// fixed point relative to a row's largest value, as in the rows form): the lowest byte's sums are rounded to units of the second's and go on
// as its accumulators (half a unit in sums of typically 2^22 of them), the third's are 256 of those units -- one integer, one conversion.  A
// lane (query l % 32, half g) then has 16 weights of one query, of positions 16 g .. 16 g + 15 in order: the rows of the K operand are
// taken from memory so that result register r is position 16 g + r, whose values are byte r of the 16 bytes that the lane with the
// same g loads for a dim.  So O^T += V^T P^T has its operands in place: 32x32x16 f16 products, codes converted (exactly) in registers, a
// weight w = p s^v as the sum of two f16 numbers (22 bits) -- relative to the row's own largest weight, see kTiles8Top.  fp32 accumulation
// throughout.
//
// A half is 28 matrix instructions (900 cycles) and some 290 vector instructions (1400): the vector ALU bounds a long walk, at 1.0 us per half and
// SIMD with two waves there (cycles with a vector instruction 67 %, with a matrix one 43 %).  A half's scores are formed beside the weights and
// outputs of the half before, so that either pipe has work in one wave's stream; by itself that changed nothing (512 tokens behind 16 000, 32 heads of 128:
// 285 us, in turn 281), with the wave's priority raised while the products are formed 270: the other wave then has the phase that this one has not.  Head
// sizes to 64 have half the products and do without (12 heads of 64, 2048 tokens 38.6 us, raised 41.5).
#pragma once
#include "bl_attn8.hpp"

namespace bl {

constexpr int kTiles8Keys = 32, kTiles8Waves = 4, kTiles8Threads = 64 * kTiles8Waves;
static_assert(1 << kTiles8Set == kTiles8Waves * kTiles8Keys, "a half chunk per wave");
// What keeps a row's weights within f16.  A row has a reference score, p = exp2(score - reference), and a wave an exponent E above those of all
// value scales that it has met; weights, and with them the outputs, are w = p s^v 2^(9 - E).  The reference is set so that the row's largest weight so far
// is between 2^6 and 2^7 (2^3 at least, see alike): weights down to 2^-3 then have 22 bits, smaller ones are rounded to 2^-25, 2^-28 of the largest.
// By the largest score alone, a value that a row does not see, or gives no weight, would take the bits of those that it does: E is all rows'.  The
// reference is looked at again where score and scales of a half would allow a weight of 2^15, and rises if a weight of the row's own is above 2^7
// by then: nearly every half has a new maximum for one of 32 queries, and the 64 products that rescale the outputs are a sixth of a half's
// instructions.  It is at most 118 below a half's largest score (a half's sum of p stays below 2^122, and the sums of 4 million positions, in units of
// 2^24, below 2^116): a row that weighs values 2^-120 times as large as what others see has all bits of them.  Where the scales are alike it is the
// largest score itself, and the exponents of what weighs much are small numbers (with 9 + 51 for the 9, their rounding alone gave 5e-7 of the output).
constexpr int kTiles8Top = 15, kTiles8Set0 = 7, kTiles8Far = 118;
constexpr int kTiles8Above = 2;            // E is set so far above a scale's exponent: the next, slightly larger ones leave it (2048 tokens 108.8 and 106.7 us)
constexpr int kTiles8Scale = kTiles8Set0 + kTiles8Above;
constexpr int kTiles8Unit = 24;            // sums of p are in units of 2^24
constexpr int kTiles8Sum = 100;            // ... and above 2^100 of them not scaled up any more
constexpr int kTiles8NoScale = -140;       // below every scale's exponent

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x16 tiles8_mfma(const v4i& a, const v4i& b, const i32x16& c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 tiles8_mfma16(const u32x4& a, const u32x4& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ int exponent_above(float x) { return (int)(__float_as_uint(x) >> 23) - 126; }   // x < 2^this, for x >= 0 (0: -126)
// Four codes as f16: 1024 + (code + 128) by its bits, less 1152 (both exact).
__device__ __forceinline__ void tiles8_widen(uint32_t codes, uint32_t& lo, uint32_t& hi) {
    const uint32_t u = codes ^ 0x80808080u;
    const f16x2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off);
}

// D32: head size in 32s (rounded up).
template <int D32>
struct Tiles8Lds {
    static constexpr int kDims = 32 * D32;
    static constexpr int kQPitch = 3 * kDims + 16;                    // bytes per row of queries: rows spread over the banks
    static constexpr int kOPitch = kDims + 4;                         // floats per row of outputs
    static constexpr int kMeet = kTiles8Waves * 32 * kOPitch * 4;     // (a tile's queries are no larger: four tiles' fit, too)
    static constexpr int kBytes = kMeet;
    static_assert(kTiles8Waves * 32 * kQPitch <= kMeet, "four tiles of queries");
};

struct Tiles8Shared {
    float  unit[kTiles8Waves * 32];
    float  scale[kTiles8Waves][2][2 * kTiles8Keys] __attribute__((aligned(16)));   // two halves' key scales, value scales
    float2 ml[kTiles8Waves][32];                                       // the waves' maxima and sums
};

template <int D32, int SETS>
__device__ __forceinline__ void tiles8_walk(const Attn8Args& p, const Attn8Walk& walk_of, uint8_t* lds, Tiles8Shared& shared, Attn8Rows& rows_of) {
    using L = Tiles8Lds<D32>;
    static_assert(SETS == 4 || SETS == 2 || SETS == 1, "waves of a tile");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = wave / SETS, set = wave % SETS;
    const int l32 = lane & 31, g = lane >> 5;
    const int d = p.head_dim, half = d >> 1, size = p.size;
    const int head = walk_of.head, split = walk_of.split, splits = walk_of.splits;
    // this wave's tile of the workgroup's rows (rows beyond the last repeat it)
    const int row0 = walk_of.row0 + 32 * tile, rows = min(32, walk_of.rows - 32 * tile);
    const auto row_of = [&](int r) { return walk_of.row0 + min(32 * tile + r, walk_of.rows - 1); };
    const int keys = p.prompt ? p.pos0 + divided(row_of(31), p.by_group) + 1 : walk_of.keys;
    const int lowest = p.prompt ? p.pos0 + divided(row_of(0), p.by_group) + 1 : keys;
    const int halves = (keys + kTiles8Keys - 1) / kTiles8Keys;
    const auto half_of = [&](int i) { return SETS * (split + splits * i) + set; };
    int mine = rows > 0 ? walk_of.mine : 0;                            // halves of this wave
    if (SETS < 4) mine = min(mine, (halves - set + SETS - 1) / SETS);  // (one split: a tile's own end)
    if (mine > 0 && half_of(mine - 1) >= halves) --mine;

    // ---- requests
    const float* scales = (g ? walk_of.c.v_scale : walk_of.c.k_scale) + l32;
    // K operand: lane l32 = 8 i + 4 g' + c has position 16 g' + 4 i + c of the half, row 16 c + 8 T + 4 g' + i of the chunk
    const int k_row = 16 * (l32 & 3) + (l32 & 4) + (l32 >> 3);
    uint32_t k_at[D32], v_at[D32];
#pragma unroll
    for (int s = 0; s < D32; ++s) {
        const int left = size - 64 * (s >> 1), width = min(left, 64);   // (a piece beyond the head size: any other; its queries are zero)
        const int piece = min(2 * (s & 1) + g, (width >> 4) - 1);
        k_at[s] = (uint32_t)((s >> 1) * 4096 + k_row * width + 16 * piece);
        v_at[s] = (uint32_t)(min(32 * s + l32, size - 1) * 64 + 16 * g);
    }
    v4i k[D32], v[D32];
    float scale;
    const auto request_keys = [&](int i) {
        const int h = half_of(i);
        const int8_t* base = walk_of.c.k + (int64_t)(h >> 1) * (kKv8Chunk * size);
#pragma unroll
        for (int s = 0; s < D32; ++s) {
            const int width = min(size - 64 * (s >> 1), 64);
            k[s] = *reinterpret_cast<const v4i*>(base + 8 * (h & 1) * width + k_at[s]);
        }
        scale = scales[h * kTiles8Keys];
    };
    const auto request_values = [&](int i) {
        const int h = half_of(i);
        const int8_t* base = walk_of.c.v + (int64_t)(h >> 1) * (kKv8Chunk * size) + 32 * (h & 1);
#pragma unroll
        for (int t = 0; t < D32; ++t) v[t] = *reinterpret_cast<const v4i*>(base + v_at[t]);
    };
    if (mine > 0) {
        request_keys(0);
        request_values(0);
    }

    // ---- the tile's queries: rotated, three bytes per element, through LDS.  Eight lanes share a row, two neighbouring elements and their
    // partners in the other half of the head at a time; the waves of a tile share its rows.
    uint8_t* queries = lds + tile * 32 * L::kQPitch;
    {
        constexpr int kTurns = D32, kPasses = 4 / SETS;    // 16 of at most 16 D32 elements of a half each; eight rows each
        typedef float f32x2_u __attribute__((ext_vector_type(2), aligned(4)));
        typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(8)));
        const int t8 = lane & 7;
#pragma unroll
        for (int pass = 0; pass < kPasses; ++pass) {
            const int r = 8 * (set * kPasses + pass) + (lane >> 3), row = row_of(r);
            const int pos = attn8_position(p, divided(row, p.by_group));
            const bool there = attn8_takes_part(p, pos);
            const float* src = p.q + attn8_row_at(p, head, row);
            const float* angles = reinterpret_cast<const float*>(p.rope + (int64_t)(there ? pos : 0) * half);
            f32x2 lo[kTurns], hi[kTurns];
            f32x4 cs[kTurns];
#pragma unroll
            for (int m = 0; m < kTurns; ++m) {
                const int i = 2 * (t8 + 8 * m);
                lo[m] = hi[m] = f32x2{0.0f, 0.0f};
                cs[m] = f32x4{1.0f, 0.0f, 1.0f, 0.0f};
                if (there && i < half) {
                    lo[m] = *reinterpret_cast<const f32x2_u*>(src + i);
                    hi[m] = *reinterpret_cast<const f32x2_u*>(src + half + i);
                    cs[m] = *reinterpret_cast<const f32x4_u*>(angles + 2 * i);
                }
            }
            float amax = 0.0f;
#pragma unroll
            for (int m = 0; m < kTurns; ++m)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float a = lo[m][x], b = hi[m][x], c = cs[m][2 * x], s = cs[m][2 * x + 1];
                    lo[m][x] = a * c - b * s;
                    hi[m][x] = a * s + b * c;
                    amax = MaxBitsOp()(amax, MaxBitsOp()(fabsf(lo[m][x]), fabsf(hi[m][x])));   // (a NaN becomes the row's unit)
                }
            amax = over_lanes<8>(amax, MaxBitsOp());
            const float inv = query_inv(amax);
            if (t8 == 0) shared.unit[32 * tile + r] = amax * (1.0f / kQueryFull) * 256.0f * p.unit;
            uint8_t* dst = queries + r * L::kQPitch;
            const auto put = [&](int e, const f32x2& x) {      // byte by byte, both elements' side by side
                const uint32_t a = query_bytes(x[0], inv), b = query_bytes(x[1], inv);
                *reinterpret_cast<uint16_t*>(dst + e) = (uint16_t)__builtin_amdgcn_perm(b, a, 0x0c0c0400u);
                *reinterpret_cast<uint16_t*>(dst + L::kDims + e) = (uint16_t)__builtin_amdgcn_perm(b, a, 0x0c0c0501u);
                *reinterpret_cast<uint16_t*>(dst + 2 * L::kDims + e) = (uint16_t)__builtin_amdgcn_perm(b, a, 0x0c0c0602u);
            };
#pragma unroll
            for (int m = 0; m < kTurns; ++m) {
                const int i = 2 * (t8 + 8 * m);
                if (i < half) {
                    put(i, lo[m]);
                    put(half + i, hi[m]);
                }
            }
            for (int e = d + 2 * t8; e < L::kDims; e += 16) put(e, f32x2{0.0f, 0.0f});
        }
    }
    if (SETS == 4 && tid < rows) attn8_count(p, rows_of, tid, row0 + tid, attn8_walked(p, walk_of));
    __syncthreads();
    v4i q[3][D32];   // B operands: column l32, dims 32 s + 16 g ...
#pragma unroll
    for (int b = 0; b < 3; ++b)
#pragma unroll
        for (int s = 0; s < D32; ++s) q[b][s] = *reinterpret_cast<const v4i*>(queries + l32 * L::kQPitch + b * L::kDims + 32 * s + 16 * g);
    const float unit = shared.unit[32 * tile + l32];
    const int limit = p.prompt ? min(keys, p.pos0 + divided(row_of(l32), p.by_group) + 1) : keys;   // positions that this lane's query sees

    f32x16 o[D32];
#pragma unroll
    for (int t = 0; t < D32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
    float run_m = -INFINITY, run_l = 0.0f;      // the reference score; run_l: over this lane half's positions only
    int run_e = kTiles8NoScale, next_e = run_e; // E (uniform); with the half under way
    bool alike = false;                         // the first half's value scales are within a factor of 16 (uniform)
    int next_room = 0;                          // of the half under way: how far its scores may be above the reference for weights below 2^15
    i32x16 low, high;                           // the scores under way: S^T, 32 positions x 32 queries, in units of 256 of the queries'

    // A half's scales go through LDS, lanes 0-31 the keys', lanes 32-63 the values', when its keys have arrived.
    const auto scales_in = [&](int i) {
        const int first = half_of(i) * kTiles8Keys;
        // What lies behind the last row may be anything.  A value's scale that is not finite becomes its key's NaN: that makes NaN of the queries that
        // see the row, and of no others, whose weight times it would be.
        const bool there = first + l32 < keys, finite = scale < INFINITY;
        const float own = g && there && finite ? scale : 0.0f, v_max = wave_max(own);
        const uint32_t bad = (uint32_t)(__ballot(there && !finite) >> 32);   // uniform
        next_room = kTiles8Far;
        if (__float_as_uint(v_max) != 0) {      // uniform
            const int e = exponent_above(v_max);
            if (e > next_e) next_e = e + kTiles8Above;
            next_room = min(kTiles8Top - kTiles8Scale + next_e - e, kTiles8Far);
        }
        float k_scale = scale;
        if (bad != 0 && (bad >> l32 & 1)) k_scale = __builtin_nanf("");
        shared.scale[wave][i & 1][lane] = g ? ldexpf(own, kTiles8Scale - next_e) : k_scale;
        __builtin_amdgcn_wave_barrier();        // (a wave's LDS operations are performed in order)
    };
    const auto scores_low_high = [&] {
#pragma unroll
        for (int r = 0; r < 16; ++r) low[r] = 64;   // (an operand that is a constant: a quarter of a unit below the middle)
#pragma unroll
        for (int r = 0; r < 16; ++r) high[r] = 0;
#pragma unroll
        for (int s = 0; s < D32; ++s) {
            low = tiles8_mfma(k[s], q[0][s], low);
            high = tiles8_mfma(k[s], q[2][s], high);
        }
    };
    const auto scores_middle = [&] {
#pragma unroll
        for (int r = 0; r < 16; ++r) low[r] >>= 8;
#pragma unroll
        for (int s = 0; s < D32; ++s) low = tiles8_mfma(k[s], q[1][s], low);
    };

    // One half: its scores are in low and high.  NEXT: another half follows, its keys are here; MORE: and another one behind it.  END: one of the
    // tile's last two halves, the only ones that some query may not see all of (32 rows).
    const auto walk = [&](int i, auto next, auto more, auto end) {
        constexpr bool NEXT = decltype(next)::value, MORE = decltype(more)::value, END = decltype(end)::value;
        const int first = half_of(i) * kTiles8Keys;
        const bool masked = END && first + kTiles8Keys > lowest;   // uniform
        const float* scales_of = shared.scale[wave][i & 1];
        const int e_new = next_e;
        const float room = (float)next_room;
        float x[16];
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const f32x4 ks = *reinterpret_cast<const f32x4*>(scales_of + 16 * g + 4 * r4);
#pragma unroll
            for (int c = 0; c < 4; ++c) x[4 * r4 + c] = (float)((high[4 * r4 + c] << 8) + low[4 * r4 + c]) * ks[c];
        }
        if (masked) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (first + 16 * g + r >= limit) x[r] = -INFINITY;
        }
        float mx = x[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
        mx = over_blocks<32>(mx, MaxOp());
        // (a query whose values are all zero has unit 0; it must not meet an infinity)
        const float top = END && mx == -INFINITY ? mx : mx * unit;
        if (__any(top > run_m + room) || e_new != run_e) {
            int left = 0;                                  // of a new exponent's bits, what the outputs take: the reference takes the others
            if (e_new != run_e) {
                const int more = e_new - run_e, taken = min(more, max(kTiles8Sum - exponent_above(over_blocks<32>(run_l, MaxOp())), 0));
                run_m -= (float)taken;
                run_l = ldexpf(run_l, taken);
                left = taken - more;
                run_e = e_new;
            }
            // The exponent of the row's largest weight relative to its largest score.  In a first half whose scales are alike, theirs: sixteen more
            // exponentials there, where nothing else is under way, cost short walks 0.2 us of 25.
            int w_exp = kTiles8Scale - kTiles8Above;
            if (!alike) {
                float w_max = 0.0f;
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                    const f32x4 vs = *reinterpret_cast<const f32x4*>(scales_of + kTiles8Keys + 16 * g + 4 * r4);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float at = x[4 * r4 + c];
                        w_max = fmaxf(w_max, __builtin_amdgcn_exp2f(END && at == -INFINITY ? at : fmaf(at, unit, -top)) * vs[c]);
                    }
                }
                w_exp = exponent_above(over_blocks<32>(w_max, MaxOp()));
            }
            alike = false;
            const float m_new = top > run_m + room ? fmaxf(run_m, top + (float)max(w_exp - kTiles8Set0, -kTiles8Far)) : run_m;
            const float apart = run_m - m_new;
            const int far = apart < -64.0f ? 64 : 0;       // (2^-126 is the least that exp2 gives; sums may be as large)
            const float f = m_new == run_m ? 1.0f : __builtin_amdgcn_exp2f(apart + (float)far);
            const float fo = ldexpf(f, left - far);
#pragma unroll
            for (int t = 0; t < D32; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t][r] *= fo;
            run_l = ldexpf(run_l * f, -far);
            run_m = m_new;
        }
        const float base = END && run_m == -INFINITY ? 0.0f : run_m;
        if constexpr (D32 > 2) __builtin_amdgcn_s_setprio(1);   // until the products are out
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (NEXT) {
            scales_in(i + 1);
            scores_low_high();
        }
        u32x4 w_hi[2], w_lo[2];
        float sum = 0.0f;
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            const f32x4 vs = *reinterpret_cast<const f32x4*>(scales_of + kTiles8Keys + 16 * g + 4 * r4);
            float w[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float at = x[4 * r4 + c];
                const float pj = __builtin_amdgcn_exp2f(END && at == -INFINITY ? at : fmaf(at, unit, -base));
                sum += pj;
                w[c] = pj * vs[c];
            }
#pragma unroll
            for (int c = 0; c < 4; c += 2) {
                const f16x2 hi = __builtin_convertvector((f32x2{w[c], w[c + 1]}), f16x2);
                const uint32_t both = __builtin_bit_cast(uint32_t, hi);
                f32x2 rest;                                // what the first parts leave: w - hi (exact)
                asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(rest[0]) : "v"(both), "v"(w[c]));
                asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(rest[1]) : "v"(both), "v"(w[c + 1]));
                const f16x2 lo = __builtin_convertvector(rest, f16x2);
                w_hi[r4 >> 1][2 * (r4 & 1) + (c >> 1)] = both;
                w_lo[r4 >> 1][2 * (r4 & 1) + (c >> 1)] = __builtin_bit_cast(uint32_t, lo);
            }
        }
        run_l = fmaf(sum, 1.0f / (1 << kTiles8Unit), run_l);
        if constexpr (NEXT) {
            __builtin_amdgcn_sched_barrier(0);
            scores_middle();
        }
#pragma unroll
        for (int t = 0; t < D32; ++t) {
            u32x4 a[2];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t lo, hi;
                tiles8_widen((uint32_t)v[t][w], lo, hi);
                a[w >> 1][2 * (w & 1)] = lo;
                a[w >> 1][2 * (w & 1) + 1] = hi;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                o[t] = tiles8_mfma16(a[h], w_lo[h], o[t]);
                o[t] = tiles8_mfma16(a[h], w_hi[h], o[t]);
            }
        }
        if constexpr (D32 > 2) __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (MORE) request_keys(i + 2);
        if constexpr (NEXT) request_values(i + 1);
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    if (mine > 0) {
        const float v_min = over_lanes<64>(g == 0 ? INFINITY : half_of(0) * kTiles8Keys + l32 >= keys ? 0.0f : scale, MinOp());
        scales_in(0);
        alike = exponent_above(__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v_min)))) > next_e - kTiles8Above - 4;
        scores_low_high();
        scores_middle();
        __builtin_amdgcn_sched_barrier(0);
        if (mine > 1) request_keys(1);
        __builtin_amdgcn_sched_barrier(0);
    }
    for (int i = 0; i + 2 < mine; ++i) walk(i, yes, yes, no);
    if (mine > 1) walk(mine - 2, yes, no, yes);
    if (mine > 0) walk(mine - 1, no, no, yes);

    // ---- the waves meet: references and sums first -- the references moved so that a sum is one of 0.5 to 1: by how much a wave has of a row --
    // then the outputs, each scaled by its own factor
    run_l = over_blocks<32>(run_l, AddOp());
    const int l_own = exponent_above(run_l), l_e = l_own + kTiles8Unit;
    run_m += (float)l_e;
    if (g == 0) shared.ml[wave][l32] = make_float2(run_m, ldexpf(run_l, -l_own));
    __syncthreads();
    const auto figure = [&](int at_tile, int r) {
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < SETS; ++w) m = fmaxf(m, shared.ml[at_tile * SETS + w][r].x);
        const float ref = m == -INFINITY ? 0.0f : m;       // (a prompt's row whose walk ends before this workgroup's halves)
#pragma unroll
        for (int w = 0; w < SETS; ++w) l += shared.ml[at_tile * SETS + w][r].y * __builtin_amdgcn_exp2f(shared.ml[at_tile * SETS + w][r].x - ref);
        return make_float2(m, l);
    };
    const float2 all = figure(tile, l32);
    float f = ldexpf(__builtin_amdgcn_exp2f(run_m - (all.x == -INFINITY ? 0.0f : all.x)), run_e - kTiles8Scale - l_e);
    if (SETS < 4) f = rows > 0 ? f / all.y : 0.0f;         // (one split: nobody else has figures)
    float* meet = reinterpret_cast<float*>(lds);   // (the barrier above: every wave has its queries)
#pragma unroll
    for (int t = 0; t < D32; ++t)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4)
            *reinterpret_cast<f32x4*>(meet + (wave * 32 + l32) * L::kOPitch + 32 * t + 8 * r4 + 4 * g) =
                f32x4{o[t][4 * r4] * f, o[t][4 * r4 + 1] * f, o[t][4 * r4 + 2] * f, o[t][4 * r4 + 3] * f};
    __syncthreads();
    const auto pair = [&](int at_tile, int r, int e) {
        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < SETS; ++w) {
            const float2 a = *reinterpret_cast<const float2*>(meet + ((at_tile * SETS + w) * 32 + r) * L::kOPitch + e);
            sum.x += a.x;
            sum.y += a.y;
        }
        return sum;
    };
    if constexpr (SETS == 4) {
        attn8_finish<32, 0, kTiles8Waves>(
            p, rows_of, lds, head, row0, rows, walk_of.slot, [&](int r, int e) { return pair(0, r, e); }, [&](int r) { return figure(0, r); });
    } else {
        for (int i = tid; i < walk_of.rows * half; i += kTiles8Threads) {
            const int r = divided(i, p.by_half), e = 2 * (i - r * half);
            *reinterpret_cast<float2*>(p.out + attn8_row_at(p, head, walk_of.row0 + r) + e) = pair(r >> 5, r & 31, e);
        }
    }
}

}  // namespace bl
