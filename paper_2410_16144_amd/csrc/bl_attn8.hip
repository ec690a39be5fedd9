// Attention over the 8-bit cache for few rows at a time: one token of each of several sequences, with or without a shared
// prefix (bl_attn8_decode), and prompts that the kernel of bl_attn8_prompt.hip does not take (bl_attn8_prefill).
//
// A row is one query head of one token.  A workgroup has up to 16 rows that read the same key head and walks sets of four chunks of
// 64 positions, each wave a chunk of its own with its own running maximum, sum and weighted values; the waves meet once, at the end.
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
// on its way.  The token's own row is quantized by the workgroup whose walk ends with it and put into the operands from LDS.
//
// Workgroups of one row meet as bl_attn_decode's do: figures by device-scope stores, a wait until they have been performed, a barrier, a
// ticket per row; the workgroup with a row's last ticket reads all figures and merges them.
#include "bl_attn8_plan.hpp"
#include "bl_kv8.hpp"
#include "bl_lanes.hpp"
#include "bl_quant_device.hpp"

namespace bl {

namespace {

constexpr int kThreads = 64 * kRows8Waves;
constexpr float kQueryFull = 8355584.0f;          // 127 less than three signed bytes hold: the quotient's and the product's roundings
constexpr float kWeightZero = 8388608.0f + 32896.0f;   // 2^23 + 0x8080
constexpr float kWeightMost = 0.996f;             // 0.996 * 2^23 + 0x8080 < 2^23: the integer fits
constexpr int kWeightPitch = 80;                  // bytes per operand row of weights in LDS: the four queries' rows in different banks

struct Rows8Args {
    const float*   q;
    const float*   k_new;
    const float*   v_new;
    const int32_t* pos;         // one per token (not for a prompt)
    const float2*  rope;
    float*         out;
    uint32_t*      counters;    // [key head][rows8_padded(rows)]
    float2*        figures;     // [key head][row][slot][1 + head_dim / 2]: (maximum, sum), weighted values
    Kv8            own;
    Kv8            shared;      // the prefix, or a prompt's cache
    int64_t        own_codes, own_scales;   // from one sequence to the next
    int32_t        n_heads, group, head_dim, size, tokens;
    int32_t        rows;        // tokens * group
    int32_t        shared_len;  // rows of the prefix
    int32_t        max_pos;     // of a sequence's own cache
    int32_t        shared_wgs, shared_splits, shared_blocks, own_splits, own_blocks;
    int32_t        prompt;      // the shared walk is a prompt's: token m sees rows 0 .. pos0 + m
    int32_t        pos0;
};

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4i mfma8(const v4i& a, const v4i& b, const v4i& c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
// 65536 a + 256 b + c of a product's three sums
__device__ __forceinline__ float joined(const v4i& s) { return fmaf((float)s[2], 65536.0f, (float)((s[1] << 8) + s[0])); }

__device__ __forceinline__ float2 read_figure(float2* at) {
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
__device__ __forceinline__ void leave_figure(float2* at, float x, float y) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(at), (unsigned long long)__float_as_uint(x) | (unsigned long long)__float_as_uint(y) << 32,
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// KB: head size in blocks of 64 dims (rounded up).  NQ: rows of a workgroup in fours.
template <int KB, int NQ>
struct Rows8Lds {
    static constexpr int kRows = 4 * NQ, kDims = 64 * KB;
    static constexpr int kQuery = 0;                                          // [row][byte][dims]
    static constexpr int kNew = kQuery + kRows * 3 * kDims;                   // the token's own key and value
    static constexpr int kWeights = kNew + 2 * kDims;                         // [wave][four rows][16][pitch]
    static constexpr int kWalk = kWeights + kRows8Waves * NQ * 16 * kWeightPitch;
    static constexpr int kPitch = kDims + 16;                                 // floats per row of weighted values
    static constexpr int kMeet = kRows8Waves * kRows * (kPitch * 4 + 8);      // [wave][row] values, then [wave][row] (maximum, sum)
    static constexpr int kMost = 2 * kRows8MaxSplits;                         // figures of one row at most
    static constexpr int kTeams = kRows * kMost * 8;                          // behind the merge's factors: the teams' sums
    static constexpr int kMerge = kTeams + kThreads * 8;
    static constexpr int kBytes = kWalk > kMeet ? (kWalk > kMerge ? kWalk : kMerge) : kMeet > kMerge ? kMeet : kMerge;
};

template <int KB, int NQ>
__global__ __launch_bounds__(kThreads) void attn8_rows_kernel(const Rows8Args p) {
    using L = Rows8Lds<KB, NQ>;
    constexpr int DT = 4 * KB, kRows = L::kRows, kDims = L::kDims;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ float s_unit[kRows];             // a query's unit times log2(e) / sqrt(head_dim)
    __shared__ float s_new_scale[2];
    __shared__ int s_target[kRows];             // workgroups that a row's figures come from
    __shared__ int s_shared_used[kRows];        // ... and how many of them walk the shared rows
    __shared__ int s_active[kRows];
    __shared__ int s_list[kRows];
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 15, g = lane >> 4;     // an operand's column (row) and its sixteen of the contraction; of results: column, query
    const int d = p.head_dim, half = d >> 1, size = p.size;

    // ---- which rows, which walk
    int head, split, splits, slot, row0, rows, keys, lowest, sequence = -1, last_pos = 0;
    Kv8 c;
    const bool shared = (int)blockIdx.x < p.shared_wgs;   // uniform, like all of this
    if (shared) {
        const int per = 8 * p.shared_blocks, a = (int)blockIdx.x / per, rest = (int)blockIdx.x - a * per;
        const int block = rest >> 3, unit = a * 8 + (rest & 7);
        if (unit >= p.n_heads * p.shared_splits) return;   // the grid's padding
        split = unit / p.n_heads;
        head = unit - split * p.n_heads;
        splits = p.shared_splits;
        slot = split;
        row0 = block * kRows;
        rows = min(kRows, p.rows - row0);
        keys = p.prompt ? p.pos0 + (row0 + rows - 1) / p.group + 1 : p.shared_len;
        lowest = p.prompt ? p.pos0 + row0 / p.group + 1 : keys;
        c = p.shared;
    } else {
        int i = (int)blockIdx.x - p.shared_wgs;
        head = i % p.n_heads;
        i /= p.n_heads;
        const int block = i % p.own_blocks;
        i /= p.own_blocks;
        sequence = i % p.tokens;
        split = i / p.tokens;
        splits = p.own_splits;
        slot = p.shared_splits + split;
        row0 = sequence * p.group + block * kRows;
        rows = min(kRows, p.group - block * kRows);
        last_pos = p.pos[sequence];
        const int at = last_pos - p.shared_len;
        if (at < 0 || at >= p.max_pos) return;             // a sequence that takes no part
        keys = lowest = at + 1;
        c = p.own;
        c.k += sequence * p.own_codes;
        c.v += sequence * p.own_codes;
        c.k_scale += sequence * p.own_scales;
        c.v_scale += sequence * p.own_scales;
    }
    c.k += head * c.head_bytes;
    c.v += head * c.head_bytes;
    c.k_scale += head * c.head_scales;
    c.v_scale += head * c.head_scales;
    const int chunks = kv8_chunks(keys), sets = sets_of(keys);
    if (split >= sets) return;
    const int sets_mine = (sets - split + splits - 1) / splits;
    const int last_set = split + (sets_mine - 1) * splits;
    const int mine = sets_mine - (kRows8Waves * last_set + wave >= chunks ? 1 : 0);   // chunks of this wave
    const auto chunk_of = [&](int i) { return kRows8Waves * (split + i * splits) + wave; };
    const bool owner = !shared && last_set == sets - 1;                               // this workgroup's walk ends with the token itself

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
                k[b][u] = *reinterpret_cast<const v4i*>(base + b * 4096 + (last ? 16 * u * tail : 1024 * u) + (last ? k_tail : k_full));
            }
        k_scale = *reinterpret_cast<const f32x4*>(c.k_scale + chunk_of(i) * kKv8Chunk + 4 * j);
    };
    const auto request_values = [&](int i) {
        const int8_t* base = c.v + (int64_t)chunk_of(i) * (kKv8Chunk * size);
#pragma unroll
        for (int t = 0; t < DT; ++t)   // (beyond the head size: the last sixteen dims again; nobody stores what comes of them)
            v[t] = *reinterpret_cast<const v4i*>(base + min(t, (size >> 4) - 1) * 1024 + k_full);
        v_scale = *reinterpret_cast<const f32x4*>(c.v_scale + chunk_of(i) * kKv8Chunk + 4 * j);
    };
    if (mine > 0) {
        request_keys(0);
        request_values(0);
    }

    // ---- the rows' queries, rotated, as three bytes per element; the token's own key and value as cached
    const auto position_of = [&](int token) { return p.prompt ? p.pos0 + token : p.pos[token]; };
    const auto takes_part = [&](int pos) { return p.prompt || (pos >= p.shared_len && pos - p.shared_len < p.max_pos); };
    {
        constexpr int kPairs = (KB + 1) / 2;               // of a lane: elements i = lane + 64 n and i + half
        float lo[NQ + 1][kPairs], hi[NQ + 1][kPairs];
        float2 cs[NQ + 1][kPairs];
        const bool fresh = owner && wave < 2;              // wave 0: the key, wave 1: the value
#pragma unroll
        for (int n = 0; n <= NQ; ++n) {
            const int r = wave + 4 * n;
            const float* src = nullptr;
            int pos = -1;
            if (n < NQ && r < rows) {
                const int row = row0 + r, token = row / p.group;
                pos = position_of(token);
                src = p.q + ((int64_t)token * p.n_heads * p.group + head * p.group + row - token * p.group) * d;
            } else if (n == NQ && fresh) {
                pos = last_pos;
                src = (wave == 0 ? p.k_new : p.v_new) + ((int64_t)sequence * p.n_heads + head) * d;
            }
            const bool there = src != nullptr && takes_part(pos);   // uniform
#pragma unroll
            for (int m = 0; m < kPairs; ++m) {
                const int i = lane + 64 * m;
                lo[n][m] = hi[n][m] = 0.0f;
                cs[n][m] = make_float2(1.0f, 0.0f);
                if (there && i < half) {
                    lo[n][m] = src[i];
                    hi[n][m] = src[i + half];
                    cs[n][m] = p.rope[(int64_t)pos * half + i];
                }
            }
        }
#pragma unroll
        for (int n = 0; n <= NQ; ++n) {
            float amax = 0.0f;
#pragma unroll
            for (int m = 0; m < kPairs; ++m) {
                if (n < NQ || wave == 0) {                 // (a value is not rotated)
                    const float a = lo[n][m], b = hi[n][m];
                    lo[n][m] = a * cs[n][m].x - b * cs[n][m].y;
                    hi[n][m] = a * cs[n][m].y + b * cs[n][m].x;
                }
                amax = fmaxf(amax, fmaxf(fabsf(lo[n][m]), fabsf(hi[n][m])));
            }
            amax = wave_max(amax);
            if (n < NQ) {
                const int r = wave + 4 * n;
                float inv = kQueryFull / amax;
                if (!(inv < INFINITY)) inv = 0.0f;
                if (lane == 0) s_unit[r] = amax / kQueryFull * (1.4426950408889634f / sqrtf((float)d));
                uint8_t* dst = lds + L::kQuery + r * 3 * kDims;
                const auto put = [&](int e, float x) {
                    const uint32_t bytes = ((uint32_t)((int)rintf(x * inv) + 0x808080)) ^ 0x808080u;
                    dst[e] = (uint8_t)bytes;
                    dst[kDims + e] = (uint8_t)(bytes >> 8);
                    dst[2 * kDims + e] = (uint8_t)(bytes >> 16);
                };
#pragma unroll
                for (int m = 0; m < kPairs; ++m) {
                    const int i = lane + 64 * m;
                    if (i < half) {
                        put(i, lo[n][m]);
                        put(i + half, hi[n][m]);
                    }
                }
                for (int e = d + lane; e < kDims; e += kWave) put(e, 0.0f);
            } else if (fresh) {                            // uniform in the wave
                float inv, scale;
                kv8_scales(amax, inv, scale);
                if (lane == 0) s_new_scale[wave] = scale;
                uint8_t* dst = lds + L::kNew + wave * kDims;
#pragma unroll
                for (int m = 0; m < kPairs; ++m) {
                    const int i = lane + 64 * m;
                    if (i < half) {
                        dst[i] = (uint8_t)kv8_code(lo[n][m], inv);
                        dst[i + half] = (uint8_t)kv8_code(hi[n][m], inv);
                    }
                }
                for (int e = d + lane; e < kDims; e += kWave) dst[e] = 0;
            }
        }
    }
    if (tid < rows) {   // who else has figures of these rows
        const int row = row0 + tid, token = row / p.group;
        const int pos = position_of(token), at = pos - p.shared_len;
        const bool active = takes_part(pos);
        const int walked = p.prompt ? min(splits, sets) : p.shared_len > 0 ? min(p.shared_splits, sets_of(p.shared_len)) : 0;
        s_active[tid] = active;
        s_shared_used[tid] = walked;
        s_target[tid] = walked + (active && !p.prompt ? min(p.own_splits, sets_of(at + 1)) : 0);
    }
    __syncthreads();
    const int at = keys - 1;                               // of the token in its own cache
    if (owner && row0 == sequence * p.group) {             // its first block of rows stores the row
        const int64_t base = (int64_t)(chunks - 1) * (kKv8Chunk * size);
        for (int e = tid; e < size; e += kThreads) {
            c.k[base + kv8_key_at(at, e, size)] = (int8_t)lds[L::kNew + e];
            c.v[base + kv8_value_at(at, e)] = (int8_t)lds[L::kNew + kDims + e];
        }
        if (tid == 0) c.k_scale[at] = s_new_scale[0];
        if (tid == 1) c.v_scale[at] = s_new_scale[1];
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
        unit[n] = s_unit[4 * n + g];
        limit[n] = p.prompt ? min(keys, p.pos0 + (row0 + 4 * n + g) / p.group + 1) : keys;
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
                    k_scale[u] = s_new_scale[0];
                    v_scale[u] = s_new_scale[1];
                }
        }
        // scores: lane (query g, j) has the four positions 4 j + u
        v4i s[NQ][4];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            if (n < fours) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    s[n][u] = mfma8(q[n][0], k[0][u], v4i{0, 0, 0, 0});
#pragma unroll
                    for (int b = 1; b < KB; ++b) s[n][u] = mfma8(q[n][b], k[b][u], s[n][u]);
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
                    x[u] = joined(s[n][u]) * ks[u] * unit[n];
                    if (masked && first + 4 * j + u >= limit[n]) x[u] = -INFINITY;
                }
                const float m_c = over_lanes<16>(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), MaxOp());
                const float base = m_c == -INFINITY ? 0.0f : m_c;      // (a row that sees nothing of this chunk: no weights)
                float w[4], sum = 0.0f;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float p_j = __builtin_amdgcn_exp2f(x[u] - base);
                    sum += p_j;
                    w[u] = p_j * vs[u];
                }
                // the weights' unit: a power of two with which the chunk's largest one has 23 bits (22 where 23 would not fit three bytes)
                const float w_max = over_lanes<16>(fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])), MaxOp());
                const int exponent = max(__builtin_amdgcn_frexp_expf(w_max) - (__builtin_amdgcn_frexp_mantf(w_max) < kWeightMost ? 23 : 22), -120);
                const float per = ldexpf(1.0f, -exponent);
                uint32_t bits[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) bits[u] = __float_as_uint(fmaf(w[u], per, kWeightZero));
                const float m_new = fmaxf(run_m[n], m_c), ref = m_new == -INFINITY ? 0.0f : m_new;
                keep[n] = __builtin_amdgcn_exp2f(run_m[n] - ref);
                take[n] = __builtin_amdgcn_exp2f(m_c - ref);
                run_m[n] = m_new;
                run_l[n] = run_l[n] * keep[n] + sum * take[n];
                take[n] = ldexpf(take[n], exponent);
                // byte k of the four words, side by side
                const uint32_t low01 = __builtin_amdgcn_perm(bits[1], bits[0], 0x05010400u), low23 = __builtin_amdgcn_perm(bits[3], bits[2], 0x05010400u);
                const uint32_t top01 = __builtin_amdgcn_perm(bits[1], bits[0], 0x0c0c0602u), top23 = __builtin_amdgcn_perm(bits[3], bits[2], 0x0c0c0602u);
                uint8_t* dst = weights + n * (16 * kWeightPitch) + 4 * g * kWeightPitch + 4 * j;
                *reinterpret_cast<uint32_t*>(dst) = __builtin_amdgcn_perm(low23, low01, 0x05040100u) ^ 0x80808080u;
                *reinterpret_cast<uint32_t*>(dst + kWeightPitch) = __builtin_amdgcn_perm(low23, low01, 0x07060302u) ^ 0x80808080u;
                *reinterpret_cast<uint32_t*>(dst + 2 * kWeightPitch) = __builtin_amdgcn_perm(top23, top01, 0x05040100u);
            }
        // weighted values: lane (query g, j) has the dims 16 t + j
#pragma unroll
        for (int n = 0; n < NQ; ++n)
            if (n < fours) {
                const v4i w = *reinterpret_cast<const v4i*>(weights + n * (16 * kWeightPitch) + j * kWeightPitch + 16 * g);
#pragma unroll
                for (int t = 0; t < DT; ++t) o[n][t] = fmaf(joined(mfma8(w, v[t], v4i{0, 0, 0, 0})), take[n], o[n][t] * keep[n]);
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
    float2* meet_ml = reinterpret_cast<float2*>(meet + kRows8Waves * kRows * L::kPitch);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const float l = over_lanes<16>(run_l[n], AddOp());
        if (j == 0) meet_ml[wave * kRows + 4 * n + g] = make_float2(run_m[n], l);
#pragma unroll
        for (int t = 0; t < DT; ++t) meet[(wave * kRows + 4 * n + g) * L::kPitch + 16 * t + j] = o[n][t];
    }
    __syncthreads();
    const auto out_of = [&](int r) {                       // where row r of the block goes
        const int row = row0 + r, token = row / p.group;
        return p.out + ((int64_t)token * p.n_heads * p.group + head * p.group + row - token * p.group) * d;
    };
    const int stride = half + 1, slots = p.shared_splits + p.own_splits;
    const auto figures_of = [&](int r) { return p.figures + ((int64_t)head * p.rows + row0 + r) * slots * stride; };
    for (int i = tid; i < rows * half; i += kThreads) {
        const int r = i / half, e = 2 * (i - r * half);
        float m = -INFINITY, l = 0.0f, x = 0.0f, y = 0.0f;
        float2 ml[kRows8Waves];
#pragma unroll
        for (int w = 0; w < kRows8Waves; ++w) {
            ml[w] = meet_ml[w * kRows + r];
            m = fmaxf(m, ml[w].x);
        }
        const float ref = m == -INFINITY ? 0.0f : m;       // (a prompt's row whose walk ends before this workgroup's chunks)
#pragma unroll
        for (int w = 0; w < kRows8Waves; ++w) {
            const float f = __builtin_amdgcn_exp2f(ml[w].x - ref);
            const float2 a = *reinterpret_cast<const float2*>(meet + (w * kRows + r) * L::kPitch + e);
            l += f * ml[w].y;
            x += f * a.x;
            y += f * a.y;
        }
        if (s_target[r] == 1) {                            // the only workgroup: nothing is left for anybody
            if (s_active[r]) {
                float* dst = out_of(r) + e;
                dst[0] = x / l;
                dst[1] = y / l;
            }
        } else {
            float2* dst = figures_of(r) + (int64_t)slot * stride;
            leave_figure(dst + 1 + (e >> 1), x, y);
            if (e == 0) leave_figure(dst, m, l);
        }
    }
    // Every thread's figures have been performed before the workgroup draws its tickets: stores are outstanding vector memory operations
    // until they are acknowledged, and a barrier alone does not wait for them.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    uint32_t* counters = p.counters + (int64_t)head * rows8_padded(p.rows) + row0;
    if (wave == 0) {
        bool last = false;
        if (lane < rows && s_target[lane] > 1)
            last = __hip_atomic_fetch_add(counters + lane, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(s_target[lane] - 1);
        const unsigned long long which = __ballot(last);
        if (last) s_list[__popcll(which & ((1ull << lane) - 1))] = lane;
        if (lane == 0) s_count = __popcll(which);
    }
    __syncthreads();
    const int listed = s_count;
    if (listed == 0) return;                               // uniform

    // ---- this workgroup is the last of some rows: their figures become the output
    float2* factor = reinterpret_cast<float2*>(lds);       // [row of the list][figure]: (maximum, sum), then (factor, -)
    const auto slot_of = [&](int r, int f) { return f < s_shared_used[r] ? f : p.shared_splits + f - s_shared_used[r]; };
    for (int i = tid; i < listed * L::kMost; i += kThreads) {
        const int r = s_list[i / L::kMost], f = i % L::kMost;
        if (f < s_target[r]) factor[i] = read_figure(figures_of(r) + (int64_t)slot_of(r, f) * stride);
    }
    __syncthreads();
    for (int n = wave; n < listed; n += kRows8Waves) {
        const int target = s_target[s_list[n]];
        float2 a[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) a[h] = lane + 64 * h < target ? factor[n * L::kMost + lane + 64 * h] : make_float2(-INFINITY, 0.0f);
        const float m = over_lanes<64>(fmaxf(a[0].x, a[1].x), MaxOp());
        const float f0 = __builtin_amdgcn_exp2f(a[0].x - m), f1 = __builtin_amdgcn_exp2f(a[1].x - m);
        const float l = over_lanes<64>(f0 * a[0].y + f1 * a[1].y, AddOp());
        if (lane < target) factor[n * L::kMost + lane].x = f0 / l;
        if (lane + 64 < target) factor[n * L::kMost + lane + 64].x = f1 / l;
    }
    __syncthreads();
    const int pairs = listed * half;                       // of outputs
    const int teams = max(1, kThreads / pairs);            // that share a pair's figures
    float2* sums = reinterpret_cast<float2*>(lds + L::kTeams);
    for (int i = tid; i < pairs * teams; i += kThreads) {  // (more than one team: one turn)
        const int team = i / pairs, pair = i - team * pairs, n = pair / half, e = pair - n * half, r = s_list[n], target = s_target[r];
        float2* src = figures_of(r) + 1 + e;
        float x = 0.0f, y = 0.0f;
        for (int f = team; f < target; f += 8 * teams) {   // eight at a time: a read is a trip to memory
            float2 a[8];
#pragma unroll
            for (int h = 0; h < 8; ++h) a[h] = read_figure(src + (int64_t)slot_of(r, min(f + h * teams, target - 1)) * stride);
#pragma unroll
            for (int h = 0; h < 8; ++h) {
                const float w = f + h * teams < target ? factor[n * L::kMost + f + h * teams].x : 0.0f;
                x += w * a[h].x;
                y += w * a[h].y;
            }
        }
        if (teams > 1) sums[i] = make_float2(x, y);
        else if (s_active[r]) *reinterpret_cast<float2*>(out_of(r) + 2 * e) = make_float2(x, y);
    }
    if (teams > 1) {                                       // uniform
        __syncthreads();
        if (tid < pairs) {
            const int n = tid / half, e = tid - n * half, r = s_list[n];
            float x = 0.0f, y = 0.0f;
            for (int t = 0; t < teams; ++t) {
                x += sums[t * pairs + tid].x;
                y += sums[t * pairs + tid].y;
            }
            if (s_active[r]) {
                float* dst = out_of(r) + 2 * e;
                dst[0] = x;
                dst[1] = y;
            }
        }
    }
    if (tid < listed) __hip_atomic_store(counters + s_list[tid], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int KB, int NQ>
hipError_t launch_form(const Rows8Args& p, int64_t wgs, hipStream_t s) {
    using L = Rows8Lds<KB, NQ>;
    static_assert(L::kBytes <= kMaxDecodeLds, "fits the LDS ceiling");
    static LdsCeiling ceiling;   // per instantiation, i.e. per kernel
    const hipError_t e = ceiling.ensure(reinterpret_cast<const void*>(&attn8_rows_kernel<KB, NQ>), L::kBytes);
    if (e != hipSuccess) return e;
    attn8_rows_kernel<KB, NQ><<<dim3((unsigned)wgs), dim3(kThreads), L::kBytes, s>>>(p);
    return hipGetLastError();
}

template <int KB>
hipError_t launch_block(const Rows8Args& p, int block, int64_t wgs, hipStream_t s) {
    if (block == 4) return launch_form<KB, 1>(p, wgs, s);
    if (block == 8) return launch_form<KB, 2>(p, wgs, s);
    return launch_form<KB, 4>(p, wgs, s);
}

hipError_t launch_rows(Rows8Args& p, const Rows8Plan& plan, void* scratch, hipStream_t s) {
    p.rows = p.tokens * p.group;
    p.size = kv8_size(p.head_dim);
    p.counters = static_cast<uint32_t*>(scratch);
    p.figures = reinterpret_cast<float2*>(p.counters + rows8_counters(p.n_heads, p.rows));
    p.shared_wgs = (int32_t)plan.shared_wgs;
    p.shared_splits = plan.shared_splits; p.shared_blocks = plan.shared_blocks;
    p.own_splits = plan.own_splits; p.own_blocks = plan.own_blocks;
    const int64_t wgs = plan.shared_wgs + plan.own_wgs;
    if (wgs > INT32_MAX) return hipErrorInvalidValue;
    static_assert(BL_ATTN_MAX_HEAD_DIM == 256, "head sizes up to four blocks of 64");
    switch ((p.head_dim + 63) / 64) {
        case 1: return launch_block<1>(p, plan.block, wgs, s);
        case 2: return launch_block<2>(p, plan.block, wgs, s);
        case 3: return launch_block<3>(p, plan.block, wgs, s);
        case 4: return launch_block<4>(p, plan.block, wgs, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

int64_t attn8_scratch_bytes(int n_heads, int group, int head_dim, int max_pos, int sequences, int prefix_len) {
    const Rows8Plan plan = rows8_plan(n_heads, group, sequences, prefix_len, max_pos);
    return rows8_scratch_bytes(plan, n_heads, (int64_t)sequences * group, head_dim);
}

hipError_t launch_attn8_decode(const ::bl_attn8_args& a, hipStream_t s) {
    Rows8Args p{};
    p.q = a.q_lin_dev; p.k_new = a.k_lin_dev; p.v_new = a.v_lin_dev; p.pos = a.pos_dev;
    p.rope = reinterpret_cast<const float2*>(a.rope_table_dev);
    p.out = a.out_dev;
    p.own = kv8_of(a.cache, 0);
    if (a.prefix_len > 0) p.shared = kv8_of(a.prefix, 0);
    p.n_heads = a.cache.n_heads; p.group = a.n_q_heads / a.cache.n_heads; p.head_dim = a.cache.head_dim;
    p.tokens = a.cache.sequences; p.shared_len = a.prefix_len; p.max_pos = a.cache.max_pos;
    p.own_codes = p.own.head_bytes * p.n_heads;
    p.own_scales = p.own.head_scales * p.n_heads;
    return launch_rows(p, rows8_plan(p.n_heads, p.group, p.tokens, p.shared_len, p.max_pos), a.scratch_dev, s);
}

// A prompt's rows: the write clears the counters of the launch behind it.
static Rows8Plan prompt_plan(int n_heads, int group, int pos0, int M) { return rows8_plan(n_heads, group, M, pos0 + M, 0); }

int64_t attn8_prefill_scratch_bytes(int n_heads, int group, int head_dim, int pos0, int M) {
    return rows8_scratch_bytes(prompt_plan(n_heads, group, pos0, M), n_heads, (int64_t)M * group, head_dim);
}

hipError_t launch_attn8_prefill(const ::bl_attn8_prefill_args& a, hipStream_t s) {
    Rows8Args p{};
    p.q = a.q_lin_dev;
    p.rope = reinterpret_cast<const float2*>(a.rope_table_dev);
    p.out = a.out_dev;
    p.shared = kv8_of(a.cache, a.sequence);
    p.n_heads = a.cache.n_heads; p.group = a.n_q_heads / a.cache.n_heads; p.head_dim = a.cache.head_dim;
    p.tokens = a.M; p.prompt = 1; p.pos0 = a.pos0;
    const Rows8Plan plan = prompt_plan(p.n_heads, p.group, a.pos0, a.M);
    const ::bl_kv8_write_args w{&a.cache, a.k_lin_dev, a.v_lin_dev, a.rope_table_dev, (int64_t)p.n_heads * p.head_dim, BL_F32, a.sequence, a.pos0, a.M};
    const hipError_t e = launch_kv8_write(w, static_cast<uint32_t*>(a.scratch_dev), rows8_counters(p.n_heads, (int64_t)a.M * p.group), s);
    if (e != hipSuccess) return e;
    return launch_rows(p, plan, a.scratch_dev, s);
}

}  // namespace bl
