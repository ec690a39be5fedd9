// The rows form of the attention over 8-bit caches: few rows (up to 16) that read one key head.
//
// A workgroup walks sets of as many chunks of 64 positions as it has waves, each wave a chunk of its own with its own running maximum, sum and
// weighted values; the waves meet once, at the end.
// out = sum_j p_j s^v_j v_j / sum_j p_j,   p_j = exp(s^k_j q.k_j / sqrt(d) - max), over int8 codes k_j, v_j with scales s^k_j, s^v_j.
//
// Both products run on v_mfma_i32_16x16x64_i8 with the codes as they lie in memory -- no conversion, no LDS (bl_kv8.hpp).  What multiplies
// them is split into signed bytes instead: a query is the integer round(q * 8355584 / max|q|) = 65536 a + 256 b + c, its three bytes
// three rows of the operand (four queries make sixteen rows; the fourth row of each is not used), and the sums of the three are put together
// again behind the product.  A chunk's weights w_j = p_j s^v_j are integers of 23 bits relative to the row's largest in the chunk, cut the same
// way: fma(w, 2^n, 2^23 + 0x8080) has the integer in its low 23 bits, and the 0x8080 makes the two low bytes signed ones (xor 0x80).
// Integer sums are exact; a product's rounding is that of a 24-bit (23-bit) operand, as in fp32.
//
// A wave's next keys are requested when this chunk's scores are formed, its next values when the weighted values are: half a chunk is always
// on its way.  Memory bounds a long walk (32 heads of 128, rows in fours: every further byte at 6.96 TB/s; 64 heads on 8 at 100 000 positions, in
// eights: 41.7 us, 4.9 TB/s), waiting a short one: 17 positions of 12 heads of 64 take 5.2 us (in a cache of 18 rows and of 8192), a split walk 8 to 9 beside its bytes (start 2.1,
// position and queries 1.4, figures out 0.9, ticket 1.0, figures in 2.3).  The token's own row is quantized by the workgroup whose walk ends with it
// and put into the operands from LDS.
#pragma once
#include "bl_attn8.hpp"

namespace bl {

constexpr float kWeightZero = 8388608.0f + 32896.0f;   // 2^23 + 0x8080
constexpr float kWeightMost = 0.996f;             // 0.996 * 2^23 + 0x8080 < 2^23: the integer fits
constexpr int kWeightPitch = 80;                  // bytes per operand row of weights in LDS: the four queries' rows in different banks

__device__ __forceinline__ v4i rows8_mfma(const v4i& a, const v4i& b, const v4i& c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
// 65536 a + 256 b + c of a product's three sums
__device__ __forceinline__ float rows8_joined(const v4i& s) { return fmaf((float)s[2], 65536.0f, (float)((s[1] << 8) + s[0])); }

// A walk's bytes are read once.  From memory, streaming loads are faster, and leave a model's weights in the memory-side cache; a short cache that
// the token before left in the dies' caches is faster without (see launch_rows).
template <bool STREAM>
__device__ __forceinline__ v4i rows8_load(const int8_t* at) {
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const v4i*>(at));
    else return *reinterpret_cast<const v4i*>(at);
}

// KB: head size in blocks of 64 dims (rounded up).  NQ: rows of a workgroup in fours.  W: waves of a workgroup.  STREAM: by streaming loads.
template <int KB, int NQ, int W>
struct Rows8Lds {
    static constexpr int kRows = 4 * NQ, kDims = 64 * KB, kThreads = 64 * W;
    static constexpr int kQuery = 0;                                          // [row][byte][dims]
    static constexpr int kNew = kQuery + kRows * 3 * kDims;                   // the token's own key and value
    static constexpr int kWeights = kNew + 2 * kDims;                         // [wave][four rows][16][pitch]
    static constexpr int kWalk = kWeights + W * NQ * 16 * kWeightPitch;
    static constexpr int kPitch = kDims + 16;                                 // floats per row of weighted values
    static constexpr int kMeet = W * kRows * (kPitch * 4 + 8);      // [wave][row] values, then [wave][row] (maximum, sum)
    static constexpr int kMost = 2 * kAttn8MaxSplits;                         // figures of one row at most
    static constexpr int kMerge = kRows * kMost * 8 + kThreads * 8;
    static constexpr int kBytes = kWalk > kMeet ? (kWalk > kMerge ? kWalk : kMerge) : kMeet > kMerge ? kMeet : kMerge;
};

struct Rows8Shared {
    float unit[16];             // a query's unit times log2(e) / sqrt(head_dim)
    float new_scale[2];         // of the token's own key and value
};

template <int KB, int NQ, int W, bool STREAM>
__device__ __forceinline__ void rows8_walk(const Attn8Args& p, const Attn8Walk& walk_of, uint8_t* lds, Rows8Shared& shared, Attn8Rows& rows_of) {
    using L = Rows8Lds<KB, NQ, W>;
    constexpr int DT = 4 * KB, kRows = L::kRows, kDims = L::kDims, kThreads = L::kThreads;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 15, g = lane >> 4;     // an operand's column (row) and its sixteen of the contraction; of results: column, query
    const int d = p.head_dim, half = d >> 1, size = p.size;
    const Kv8& c = walk_of.c;
    const int head = walk_of.head, split = walk_of.split, splits = walk_of.splits, row0 = walk_of.row0, rows = walk_of.rows, keys = walk_of.keys,
              lowest = walk_of.lowest, sequence = walk_of.sequence, sets = walk_of.sets;
    const int chunks = kv8_chunks(keys);
    const int last_set = split + (walk_of.mine - 1) * splits;
    const int mine = walk_of.mine - (W * last_set + wave >= chunks ? 1 : 0);   // chunks of this wave
    const auto chunk_of = [&](int i) { return W * (split + i * splits) + wave; };
    const bool owner = sequence >= 0 && last_set == sets - 1;                         // this workgroup's walk ends with the token itself

    // ---- requests: operands of 16 bytes per lane, from consecutive memory
    v4i k[KB][4], v[DT];
    f32x4 k_scale, v_scale;
    const int tail = size - 64 * (KB - 1);                 // bytes of a key's row in its last block
    const uint32_t k_full = (uint32_t)(j * 64 + 16 * g), k_tail = (uint32_t)(j * tail + 16 * min(g, (tail >> 4) - 1));
    const auto request_keys = [&](int i) {
        const int8_t* base = c.k + (int64_t)chunk_of(i) * (kKv8Chunk * size);
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const bool last = b == KB - 1;             // (a full block's rows are 64 bytes apart, too)
                k[b][u] = rows8_load<STREAM>(base + b * 4096 + (last ? 16 * u * tail : 1024 * u) + (last ? k_tail : k_full));
            }
        k_scale = *reinterpret_cast<const f32x4*>(c.k_scale + chunk_of(i) * kKv8Chunk + 4 * j);
    };
    const auto request_values = [&](int i) {
        const int8_t* base = c.v + (int64_t)chunk_of(i) * (kKv8Chunk * size);
#pragma unroll
        for (int t = 0; t < DT; ++t)   // (beyond the head size: the last sixteen dims again; nobody stores what comes of them)
            v[t] = rows8_load<STREAM>(base + min(t, (size >> 4) - 1) * 1024 + k_full);
        v_scale = *reinterpret_cast<const f32x4*>(c.v_scale + chunk_of(i) * kKv8Chunk + 4 * j);
    };
    if (mine > 0) {
        request_keys(0);
        request_values(0);
    }


    // ---- the rows' queries, rotated, as three bytes per element; the token's own key and value as cached
    {
        constexpr int kPairs = (KB + 1) / 2;               // of a lane: elements i = lane + 64 n and i + half
        constexpr int kTasks = (kRows + 2 + W - 1) / W;    // of a wave: rows, then the key, then the value
        float lo[kTasks][kPairs], hi[kTasks][kPairs];
        float2 cs[kTasks][kPairs];
        const int tasks = owner ? rows + 2 : rows;         // (rows beyond the last have what LDS held: nobody looks at what comes of them)
        // (requests stand under no condition of a lane: an element beyond the half is another one, and what comes of a token that takes no
        // part is not written)
#pragma unroll
        for (int n = 0; n < kTasks; ++n) {
            const int t = wave + W * n;
            if (t >= tasks) break;                         // uniform
            const int row = row0 + min(t, rows - 1);
            const float* src = t < rows ? p.q + attn8_row_at(p, head, row) : (t == rows ? p.k_new : p.v_new) + ((int64_t)sequence * p.n_heads + head) * d;
            const int pos = sequence >= 0 ? walk_of.pos : attn8_position(p, divided(row, p.by_group));
            const float2* angles = p.rope + (int64_t)(attn8_takes_part(p, pos) ? pos : 0) * half;
#pragma unroll
            for (int m = 0; m < kPairs; ++m) {
                const int i = min(lane + 64 * m, half - 1);
                lo[n][m] = src[i];
                hi[n][m] = src[i + half];
                cs[n][m] = angles[i];
            }
        }
#pragma unroll
        for (int n = 0; n < kTasks; ++n) {
            const int t = wave + W * n;
            if (t >= tasks) break;                         // uniform
            float amax = 0.0f;
#pragma unroll
            for (int m = 0; m < kPairs; ++m) {
                if (t <= rows) {                           // (a value is not rotated)
                    const float a = lo[n][m], b = hi[n][m];
                    lo[n][m] = a * cs[n][m].x - b * cs[n][m].y;
                    hi[n][m] = a * cs[n][m].y + b * cs[n][m].x;
                }
                amax = MaxBitsOp()(amax, MaxBitsOp()(fabsf(lo[n][m]), fabsf(hi[n][m])));   // (a NaN becomes the row's unit)
            }
            amax = over_lanes<64>(amax, MaxBitsOp());
            if (t < rows) {
                const float inv = query_inv(amax);
                if (lane == 0) shared.unit[t] = amax * (1.0f / kQueryFull) * p.unit;
                uint8_t* dst = lds + L::kQuery + t * 3 * kDims;
                const auto put = [&](int e, uint32_t bytes) {
                    dst[e] = (uint8_t)bytes;
                    dst[kDims + e] = (uint8_t)(bytes >> 8);
                    dst[2 * kDims + e] = (uint8_t)(bytes >> 16);
                };
#pragma unroll
                for (int m = 0; m < kPairs; ++m) {
                    const int i = lane + 64 * m;
                    if (i < half) {
                        put(i, query_bytes(lo[n][m], inv));
                        put(i + half, query_bytes(hi[n][m], inv));
                    }
                }
                for (int e = d + lane; e < kDims; e += kWave) put(e, 0);
            } else {
                float inv, scale;
                kv8_scales(amax, inv, scale);
                if (lane == 0) shared.new_scale[t - rows] = scale;
                uint8_t* dst = lds + L::kNew + (t - rows) * kDims;
#pragma unroll
                for (int m = 0; m < kPairs; ++m) {
                    const int i = lane + 64 * m;
                    if (i < half) {
                        dst[i] = kv8_finite(amax) ? (uint8_t)kv8_code(lo[n][m], inv) : 0;
                        dst[i + half] = kv8_finite(amax) ? (uint8_t)kv8_code(hi[n][m], inv) : 0;
                    }
                }
                for (int e = d + lane; e < kDims; e += kWave) dst[e] = 0;
            }
        }
    }
    if (tid < rows) attn8_count(p, rows_of, tid, row0 + tid, attn8_walked(p, walk_of));
    __syncthreads();
    const int at = keys - 1;                               // of the token in its own cache
    if (owner && row0 == sequence * p.group) {             // its first block of rows stores the row
        const int64_t base = (int64_t)(chunks - 1) * (kKv8Chunk * size);
        for (int e = tid; e < size; e += kThreads) {
            c.k[base + kv8_key_at(at, e, size)] = (int8_t)lds[L::kNew + e];
            c.v[base + kv8_value_at(at, e)] = (int8_t)lds[L::kNew + kDims + e];
        }
        if (tid == 0) c.k_scale[at] = shared.new_scale[0];
        if (tid == 1) c.v_scale[at] = shared.new_scale[1];
    }

    // ---- the walk
    const int fours = (rows + 3) >> 2;                     // of rows that exist (uniform)
    float o[NQ][DT], run_m[NQ], run_l[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        run_m[n] = -INFINITY;
        run_l[n] = 0.0f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[n][t] = 0.0f;
    }
    v4i q[NQ][KB];                                         // operand rows 4 query + byte
    float unit[NQ];
    int limit[NQ];                                         // rows that this lane's query sees
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const uint8_t* src = lds + L::kQuery + ((4 * n + (j >> 2)) * 3 + min(j & 3, 2)) * kDims + 16 * g;
#pragma unroll
        for (int b = 0; b < KB; ++b) q[n][b] = *reinterpret_cast<const v4i*>(src + 64 * b);
        unit[n] = shared.unit[4 * n + g];
        limit[n] = p.prompt ? min(keys, p.pos0 + divided(row0 + 4 * n + g, p.by_group) + 1) : keys;
    }
    uint8_t* weights = lds + L::kWeights + wave * (NQ * 16 * kWeightPitch);

    const auto walk = [&](int i, auto which) {
        constexpr bool kLast = decltype(which)::value;
        const int first = chunk_of(i) * kKv8Chunk;
        if (kLast && owner && chunk_of(i) == chunks - 1) {   // uniform: the token's own row, as stored
            const int in = at & 63, u0 = in & 3, j0 = in >> 2, g0 = in >> 4, w0 = (in >> 2) & 3, shift = 8 * (in & 3);
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const v4i fresh = *reinterpret_cast<const v4i*>(lds + L::kNew + 64 * b + 16 * g);   // (padding: multiplied by zeros)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (u == u0 && j == j0) k[b][u] = fresh;
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const uint32_t fresh = lds[L::kNew + kDims + 16 * t + j];
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (w == w0 && g == g0) v[t][w] = (int)(((uint32_t)v[t][w] & ~(0xffu << shift)) | fresh << shift);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (u == u0 && j == j0) {
                    k_scale[u] = shared.new_scale[0];
                    v_scale[u] = shared.new_scale[1];
                }
        }
        // scores: lane (query g, j) has the four positions 4 j + u
        v4i s[NQ][4];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            if (n < fours) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    s[n][u] = rows8_mfma(q[n][0], k[0][u], v4i{0, 0, 0, 0});
#pragma unroll
                    for (int b = 1; b < KB; ++b) s[n][u] = rows8_mfma(q[n][b], k[b][u], s[n][u]);
                }
            }
        f32x4 ks = k_scale;
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!kLast) request_keys(i + 1);
        __builtin_amdgcn_sched_barrier(0);
        const bool masked = first + kKv8Chunk > lowest;    // uniform: a row's walk ends in this chunk
        f32x4 vs = v_scale;
        if (masked) {                                      // what lies behind the last row may be anything
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (first + 4 * j + u >= keys) ks[u] = vs[u] = 0.0f;
        }
        float keep[NQ], take[NQ];                          // factors of the walk so far and of this chunk
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            if (n < fours) {
                float x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    x[u] = rows8_joined(s[n][u]) * ks[u] * unit[n];
                    if (masked && first + 4 * j + u >= limit[n]) x[u] = -INFINITY;
                }
                float m_c = over_lanes<16>(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), MaxOp());
                const float base = m_c == -INFINITY ? 0.0f : m_c;      // (a row that sees nothing of this chunk: no weights)
                float w[4], sum = 0.0f;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float p_j = __builtin_amdgcn_exp2f(x[u] - base);
                    sum += p_j;
                    w[u] = p_j * vs[u];
                }
                if (masked && p.prompt) {                  // uniform; a later token's row may be anything, NaN and infinities included
                    asm volatile("");                      // (a branch: else every chunk pays for it)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (first + 4 * j + u >= limit[n]) w[u] = 0.0f;
                }
                // the weights' unit: a power of two with which the chunk's largest one has 23 bits (22 where 23 would not fit three bytes)
                const MaxBitsOp larger;                    // (of numbers without a sign, NaN above all)
                const float w_max = over_lanes<16>(larger(larger(w[0], w[1]), larger(w[2], w[3])), larger);
                int exponent = __builtin_amdgcn_frexp_expf(w_max) - (__builtin_amdgcn_frexp_mantf(w_max) < kWeightMost ? 23 : 22);
                if (__any(exponent < -100)) {              // (values of 1e-22 and less: relative to a score lower by 64 their unit is a normal number)
                    const int up = exponent < -100 ? 64 : 0;
#pragma unroll
                    for (int u = 0; u < 4; ++u) w[u] = ldexpf(w[u], up);
                    sum = ldexpf(sum, up);
                    m_c -= (float)up;
                    exponent += up;
                }
                const float per = ldexpf(1.0f, -exponent);
                uint32_t bits[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) bits[u] = __float_as_uint(fmaf(w[u], per, kWeightZero));
                const float m_new = fmaxf(run_m[n], m_c), ref = m_new == -INFINITY ? 0.0f : m_new;
                keep[n] = __builtin_amdgcn_exp2f(run_m[n] - ref);
                take[n] = __builtin_amdgcn_exp2f(m_c - ref);
                run_m[n] = m_new;
                run_l[n] = run_l[n] * keep[n] + sum * take[n];
                take[n] = fmaf(w_max, 0.0f, ldexpf(take[n], exponent));   // (a weight that is not finite: NaN)
                // byte k of the four words, side by side
                const uint32_t low01 = __builtin_amdgcn_perm(bits[1], bits[0], 0x05010400u), low23 = __builtin_amdgcn_perm(bits[3], bits[2], 0x05010400u);
                const uint32_t top01 = __builtin_amdgcn_perm(bits[1], bits[0], 0x0c0c0602u), top23 = __builtin_amdgcn_perm(bits[3], bits[2], 0x0c0c0602u);
                uint8_t* dst = weights + n * (16 * kWeightPitch) + 4 * g * kWeightPitch + 4 * j;
                *reinterpret_cast<uint32_t*>(dst) = __builtin_amdgcn_perm(low23, low01, 0x05040100u) ^ 0x80808080u;
                *reinterpret_cast<uint32_t*>(dst + kWeightPitch) = __builtin_amdgcn_perm(low23, low01, 0x07060302u) ^ 0x80808080u;
                *reinterpret_cast<uint32_t*>(dst + 2 * kWeightPitch) = __builtin_amdgcn_perm(top23, top01, 0x05040100u);
            }
        __builtin_amdgcn_wave_barrier();                   // (a wave's LDS operations are performed in order)
        // weighted values: lane (query g, j) has the dims 16 t + j
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            if (n < fours) {
                const v4i w = *reinterpret_cast<const v4i*>(weights + n * (16 * kWeightPitch) + j * kWeightPitch + 16 * g);
#pragma unroll
                for (int t = 0; t < DT; ++t) o[n][t] = fmaf(rows8_joined(rows8_mfma(w, v[t], v4i{0, 0, 0, 0})), take[n], o[n][t] * keep[n]);
            }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!kLast) request_values(i + 1);
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int i = 0; i + 1 < mine; ++i) walk(i, std::false_type{});
    if (mine > 0) walk(mine - 1, std::true_type{});

    // ---- the waves meet
    __syncthreads();                                       // the queries and weights in LDS are done with
    float* meet = reinterpret_cast<float*>(lds);
    float2* meet_ml = reinterpret_cast<float2*>(meet + W * kRows * L::kPitch);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float l = over_lanes<16>(run_l[n], AddOp());
        if (j == 0) meet_ml[wave * kRows + 4 * n + g] = make_float2(run_m[n], l);
#pragma unroll
        for (int t = 0; t < DT; ++t) meet[(wave * kRows + 4 * n + g) * L::kPitch + 16 * t + j] = o[n][t];
    }
    __syncthreads();
    const auto factors = [&](int r, float (&f)[W]) {   // of the waves' figures; returns their maximum
        float2 ml[W];
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            ml[w] = meet_ml[w * kRows + r];
            m = fmaxf(m, ml[w].x);
        }
        const float ref = m == -INFINITY ? 0.0f : m;       // (a prompt's row whose walk ends before this workgroup's chunks)
        float l = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            f[w] = __builtin_amdgcn_exp2f(ml[w].x - ref);
            l += f[w] * ml[w].y;
        }
        return make_float2(m, l);
    };
    attn8_finish<kRows, L::kMost, W>(
        p, rows_of, lds, head, row0, rows, walk_of.slot,
        [&](int r, int e) {
            float f[W], x = 0.0f, y = 0.0f;
            factors(r, f);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float2 a = *reinterpret_cast<const float2*>(meet + (w * kRows + r) * L::kPitch + e);
                x += f[w] * a.x;
                y += f[w] * a.y;
            }
            return make_float2(x, y);
        },
        [&](int r) {
            float f[W];
            return factors(r, f);
        });
}

}  // namespace bl
