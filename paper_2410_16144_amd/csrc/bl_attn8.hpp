// What the kernels of the attention over 8-bit caches share: arguments, the operands' numbers, and how the workgroups of a row meet.
#pragma once
#include "bl_attn8_plan.hpp"
#include "bl_kv8.hpp"
#include "bl_lanes.hpp"
#include "bl_quant_device.hpp"

namespace bl {

struct Attn8Args {
    const float*   q;
    const float*   k_new;
    const float*   v_new;
    const int32_t* pos;         // one per token (not for a prompt)
    const float2*  rope;
    float*         out;
    uint32_t*      counters;    // [key head][attn8_padded(rows)]
    float2*        figures;     // [key head][row][slot][1 + head_dim / 2]: (maximum, sum), weighted values
    Kv8            own;
    Kv8            shared;      // the prefix, or a prompt's cache
    int64_t        own_codes, own_scales;   // from one sequence to the next
    int32_t        n_heads, group, head_dim, size, tokens;
    int32_t        rows;        // tokens * group: a row is one query head of one token, of one key head
    int32_t        shared_len;  // rows of the prefix
    int32_t        max_pos;     // of a sequence's own cache
    int32_t        shared_wgs, shared_splits, shared_blocks, shared_units, strips, own_splits, own_blocks;
    int32_t        shared_set, own_set;   // positions of a workgroup's sets: 1 << so much
    int32_t        prompt;      // the shared walk is a prompt's: token m sees rows 0 .. pos0 + m
    int32_t        pos0;
    int32_t        merges;      // a launch follows that merges the figures
    int32_t        folded;      // a workgroup takes two of a prompt's blocks, from both ends
    int32_t        paired;      // a prompt's blocks in the order last, ..., middle, first, ..., middle instead of last ... first
    float          unit;        // log2(e) / sqrt(head_dim)
    Divider        by_heads, by_group, by_half, by_tokens, by_own_blocks, by_own_splits, by_shared_splits, by_shared_units, by_pieces;   // (pieces: n_heads * shared_splits)
};

hipError_t launch_attn8_tiles(const Attn8Args& p, int wgs, hipStream_t s);   // bl_attn8_tiles.hip
hipError_t launch_attn8_merge(const Attn8Args& p, hipStream_t s);

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A query as a 24-bit fixed-point number: x inv = x * kQueryFull / max|x|, as three signed bytes (the xor makes the two low ones signed).
constexpr float kQueryFull = 8355584.0f;   // 127 less than three signed bytes hold: the quotient's and the product's roundings
__device__ __forceinline__ uint32_t query_bytes(float x, float inv) { return ((uint32_t)((int)rintf(x * inv) + 0x808080)) ^ 0x808080u; }
__device__ __forceinline__ float query_inv(float amax) {
    const float inv = kQueryFull / amax;
    return inv < INFINITY ? inv : 0.0f;
}

__device__ __forceinline__ int attn8_position(const Attn8Args& p, int token) { return p.prompt ? p.pos0 + token : p.pos[token]; }
__device__ __forceinline__ bool attn8_takes_part(const Attn8Args& p, int pos) { return p.prompt || (pos >= p.shared_len && pos - p.shared_len < p.max_pos); }
// a row's place in q and out
__device__ __forceinline__ int64_t attn8_row_at(const Attn8Args& p, int head, int row) {
    const int token = divided(row, p.by_group);
    return ((int64_t)token * p.n_heads * p.group + head * p.group + row - token * p.group) * p.head_dim;
}

__device__ __forceinline__ float2 read_figure(float2* at) {
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
__device__ __forceinline__ void leave_figure(float2* at, float x, float y) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(at), (unsigned long long)__float_as_uint(x) | (unsigned long long)__float_as_uint(y) << 32,
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ int attn8_sets(int positions, int set) { return (positions + (1 << set) - 1) >> set; }

// One workgroup's part of a launch.
struct Attn8Walk {
    Kv8 c;                      // the key head's cache
    int head, row0, rows;       // rows row0 .. row0 + rows - 1 (of one key head)
    int split, splits, slot;    // which of the workgroups that share the walk; where its figures go
    int keys, lowest;           // positions of the walk: the most that a row sees, and the fewest
    int sequence, pos;          // an own walk's sequence and its token's position; sequence -1: a shared walk
    int sets;                   // sets of positions of the walk
    int mine;                   // ... of this workgroup: split, split + splits, ...
};

__device__ __forceinline__ void attn8_to_head(const Attn8Args& p, Attn8Walk& w) {
    w.c.k += w.head * w.c.head_bytes;
    w.c.v += w.head * w.c.head_bytes;
    w.c.k_scale += w.head * w.c.head_scales;
    w.c.v_scale += w.head * w.c.head_scales;
}

// False: nothing to do for this workgroup.  The index goes by blocks of rows first, then by pieces of the cache (padded to whole rounds of the dies, so
// that a piece's workgroups are on one die); a prompt's later blocks walk more and are launched first.  again: the second of a folded prompt's
// blocks.  PROMPT: a prompt in tiles, whose blocks may go by strips (the index costs a batch's kernel half a microsecond).
template <bool PROMPT = false>
__device__ __forceinline__ bool attn8_shared_walk(const Attn8Args& p, int wg, int block_rows, Attn8Walk& w, bool again = false) {
    const int pieces = p.n_heads * p.shared_splits, round = divided(wg, p.by_shared_units);
    int piece = wg - round * p.shared_units, turn = round;
    if constexpr (PROMPT) {
        const int strip = divided(piece, p.by_pieces);
        piece -= strip * pieces;
        turn = round * p.strips + strip;
        if (strip >= p.strips || turn >= (p.folded ? (p.shared_blocks + 1) >> 1 : p.shared_blocks)) return false;
        if (again && 2 * turn == p.shared_blocks - 1) return false;   // (the block in the middle)
    } else if (piece >= pieces) {
        return false;
    }
    const int first_half = (p.shared_blocks + 1) >> 1;
    const int block = !p.prompt || again ? turn : p.paired && turn >= first_half ? turn - first_half : p.shared_blocks - 1 - turn;
    w.split = divided(piece, p.by_heads);
    w.head = piece - w.split * p.n_heads;
    w.splits = p.shared_splits;
    w.slot = w.split;
    w.row0 = block * block_rows;
    w.rows = min(block_rows, p.rows - w.row0);
    w.keys = p.prompt ? p.pos0 + divided(w.row0 + w.rows - 1, p.by_group) + 1 : p.shared_len;
    w.lowest = p.prompt ? p.pos0 + divided(w.row0, p.by_group) + 1 : w.keys;
    w.sequence = w.pos = -1;
    w.sets = attn8_sets(w.keys, p.shared_set);
    w.mine = divided(w.sets - w.split + w.splits - 1, p.by_shared_splits);
    w.c = p.shared;
    attn8_to_head(p, w);
    return w.split < w.sets;
}

__device__ __forceinline__ bool attn8_own_walk(const Attn8Args& p, int wg, int block_rows, Attn8Walk& w) {
    int i = divided(wg, p.by_heads);
    w.head = wg - i * p.n_heads;
    const int next = divided(i, p.by_own_blocks), block = i - next * p.own_blocks;
    i = next;
    w.split = divided(i, p.by_tokens);
    w.sequence = i - w.split * p.tokens;
    w.splits = p.own_splits;
    w.slot = p.shared_splits + w.split;
    w.row0 = w.sequence * p.group + block * block_rows;
    w.rows = min(block_rows, p.group - block * block_rows);
    w.pos = p.pos[w.sequence];
    const int at = w.pos - p.shared_len;
    if (at < 0 || at >= p.max_pos) return false;           // a sequence that takes no part
    w.keys = w.lowest = at + 1;
    w.sets = attn8_sets(w.keys, p.own_set);
    w.mine = divided(max(w.sets - w.split + w.splits - 1, 0), p.by_own_splits);
    w.c = p.own;
    w.c.k += w.sequence * p.own_codes;
    w.c.v += w.sequence * p.own_codes;
    w.c.k_scale += w.sequence * p.own_scales;
    w.c.v_scale += w.sequence * p.own_scales;
    attn8_to_head(p, w);
    return w.split < w.sets;
}

// Workgroups that walk the shared part of a row whose walk there has so many sets.
__device__ __forceinline__ int attn8_walked(const Attn8Args& p, const Attn8Walk& w) {
    return w.sequence < 0 ? min(w.splits, w.sets) : p.shared_len > 0 ? min(p.shared_splits, attn8_sets(p.shared_len, p.shared_set)) : 0;
}

// Of a workgroup's rows: how many workgroups have figures of each.
struct Attn8Rows {
    int target[32];        // workgroups that a row's figures come from
    int shared_used[32];   // ... and how many of them walk the shared rows
    int active[32];        // whether anybody wants the row
    int list[32];          // rows whose last workgroup this is
    int count, most;       // of them; the most figures that one of them has
};

// (thread tid of the first `rows`; barrier by the caller.)  walked: workgroups that walk these rows' shared part, if this is one of them.
__device__ __forceinline__ void attn8_count(const Attn8Args& p, Attn8Rows& s, int tid, int row, int walked) {
    const int pos = attn8_position(p, divided(row, p.by_group));
    const bool active = attn8_takes_part(p, pos);
    s.active[tid] = active;
    s.shared_used[tid] = walked;
    s.target[tid] = walked + (active && !p.prompt ? min(p.own_splits, attn8_sets(pos - p.shared_len + 1, p.own_set)) : 0);
}

// The end of every walk.  pair(r, e): the workgroup's weighted values of dims e, e + 1 of its row r; figure(r): their maximum and sum.  A row
// that only this workgroup has walked is written; else the figures are left in memory, and the workgroup that draws a row's last ticket
// reads all of them and writes the row.  Nobody waits for anybody: figures travel by device-scope stores, performed past the dies' caches;
// every thread waits until its own have been performed (stores are outstanding vector memory operations until they are acknowledged, and a
// barrier alone does not wait for them), then the barrier, then the tickets; the reads are device-scope loads.
// W: waves.  LDS: kRows * kMost pairs for the merge's factors and 64 W pairs behind them; pair() may read it until the barrier.
// Where a launch of attn8_merge_kernel follows (p.merges), it does the rest: the figures are left, and nobody draws a ticket.
template <int kRows, int kMost, int W, typename Pair, typename Figure>
__device__ __forceinline__ void attn8_finish(const Attn8Args& p, Attn8Rows& s, uint8_t* lds, int head, int row0, int rows, int slot, const Pair& pair,
                                             const Figure& figure) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = p.head_dim >> 1, stride = half + 1, slots = p.shared_splits + p.own_splits;
    const auto figures_of = [&](int r) { return p.figures + ((int64_t)head * p.rows + row0 + r) * slots * stride; };
    for (int i = tid; i < rows * half; i += (64 * W)) {
        const int r = divided(i, p.by_half), e = 2 * (i - r * half);
        const float2 x = pair(r, e);
        if (s.target[r] == 1) {                            // the only workgroup: nothing is left for anybody
            if (s.active[r]) {
                const float l = figure(r).y;
                *reinterpret_cast<float2*>(p.out + attn8_row_at(p, head, row0 + r) + e) = make_float2(x.x / l, x.y / l);
            }
        } else {
            float2* dst = figures_of(r) + (int64_t)slot * stride;
            leave_figure(dst + 1 + (e >> 1), x.x, x.y);
            if (e == 0) {
                const float2 f = figure(r);
                leave_figure(dst, f.x, f.y);
            }
        }
    }
    if constexpr (kMost == 0) return;                      // (tiles: always followed)
    if (p.merges) return;                                  // uniform
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    uint32_t* counters = p.counters + (int64_t)head * attn8_padded(p.rows) + row0;
    if (wave == 0) {
        bool last = false;
        if (lane < rows && s.target[lane] > 1)
            last = __hip_atomic_fetch_add(counters + lane, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(s.target[lane] - 1);
        const unsigned long long which = __ballot(last);
        if (last) s.list[__popcll(which & ((1ull << lane) - 1))] = lane;
        const float most = over_lanes<64>(last ? (float)s.target[lane] : 0.0f, MaxOp());
        if (lane == 0) {
            s.count = __popcll(which);
            s.most = (int)most;
        }
    }
    __syncthreads();
    const int listed = s.count;
    if (listed == 0) return;                               // uniform

    // ---- this workgroup is the last of some rows: their figures become the output.  A read is a trip to memory: a thread has up to 32 of them under way,
    // the first of them together with the maxima and sums.
    const int shift = 32 - __clz(s.most - 1);              // of a row's entries below (most >= 2)
    float2* factor = reinterpret_cast<float2*>(lds);       // [row of the list][figure]: (maximum, sum), then (factor, -)
    const auto slot_of = [&](int r, int f) { return f < s.shared_used[r] ? f : p.shared_splits + f - s.shared_used[r]; };
    const int pairs = listed * half;                       // of outputs
    const int teams = max(1, (64 * W) / pairs);            // that share a pair's figures
    const int team = teams > 1 ? tid / pairs : 0;
    constexpr int kTurns = kRows >= 4 * W ? 4 : kRows >= 2 * W ? 2 : 1, kFigures = 8;   // (of all pairs of a head size of 128, if they are few)
    const auto read = [&](float2 (&a)[kTurns][kFigures], int i0, int f0) {   // pairs i0, i0 + threads, ..., figures f0, f0 + teams, ...
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int at = min(i0 + t * (64 * W), pairs - 1), n = divided(at, p.by_half), r = s.list[n], last = s.target[r] - 1;
            float2* src = figures_of(r) + 1 + at - n * half;
            if (i0 + t * (64 * W) < pairs || t == 0)
#pragma unroll
                for (int h = 0; h < kFigures; ++h) a[t][h] = read_figure(src + (int64_t)slot_of(r, min(f0 + h * teams, last)) * stride);
        }
    };
    float2 a[kTurns][kFigures];
    read(a, tid - team * pairs, min(team, teams - 1));
    for (int i = tid; i < listed << shift; i += (64 * W)) {
        const int r = s.list[i >> shift], f = i & ((1 << shift) - 1);
        if (f < s.target[r]) factor[i] = read_figure(figures_of(r) + (int64_t)slot_of(r, f) * stride);
    }
    __syncthreads();
    for (int n = wave; n < listed; n += W) {
        const int target = s.target[s.list[n]];
        float2* mine = factor + (n << shift);
        float2 ml[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) ml[h] = lane + 64 * h < target ? mine[lane + 64 * h] : make_float2(-INFINITY, 0.0f);
        const float m = over_lanes<64>(fmaxf(ml[0].x, ml[1].x), MaxOp());
        const float f0 = __builtin_amdgcn_exp2f(ml[0].x - m), f1 = __builtin_amdgcn_exp2f(ml[1].x - m);
        const float l = over_lanes<64>(f0 * ml[0].y + f1 * ml[1].y, AddOp());
        if (lane < target) mine[lane].x = f0 / l;
        if (lane + 64 < target) mine[lane + 64].x = f1 / l;
    }
    __syncthreads();
    float2* sums = factor + kRows * kMost;
    for (int i0 = tid - team * pairs; i0 < pairs; i0 += kTurns * (64 * W)) {
        float2 sum[kTurns];
#pragma unroll
        for (int t = 0; t < kTurns; ++t) sum[t] = make_float2(0.0f, 0.0f);
        for (int f0 = team; f0 < s.most; f0 += kFigures * teams) {
            if (f0 != team || i0 != tid - team * pairs) read(a, i0, f0);
#pragma unroll
            for (int t = 0; t < kTurns; ++t) {
                const int at = min(i0 + t * (64 * W), pairs - 1), n = divided(at, p.by_half), target = s.target[s.list[n]];
                if (i0 + t * (64 * W) < pairs || t == 0)
#pragma unroll
                    for (int h = 0; h < kFigures; ++h) {
                        const int f = f0 + h * teams;
                        const float w = f < target ? factor[(n << shift) + f].x : 0.0f;
                        sum[t].x += w * a[t][h].x;
                        sum[t].y += w * a[t][h].y;
                    }
            }
        }
        if (teams > 1) {
            if (team < teams) sums[team * pairs + i0] = sum[0];   // (all pairs in one turn)
        } else {
#pragma unroll
            for (int t = 0; t < kTurns; ++t) {
                const int at = i0 + t * (64 * W), n = divided(min(at, pairs - 1), p.by_half), e = at - n * half, r = s.list[n];
                if (at < pairs && s.active[r]) *reinterpret_cast<float2*>(p.out + attn8_row_at(p, head, row0 + r) + 2 * e) = sum[t];
            }
        }
    }
    if (teams > 1) {                                       // uniform
        __syncthreads();
        if (tid < pairs) {
            const int n = divided(tid, p.by_half), e = tid - n * half, r = s.list[n];
            float2 sum = make_float2(0.0f, 0.0f);
            for (int t = 0; t < teams; ++t) {
                sum.x += sums[t * pairs + tid].x;
                sum.y += sums[t * pairs + tid].y;
            }
            if (s.active[r]) *reinterpret_cast<float2*>(p.out + attn8_row_at(p, head, row0 + r) + 2 * e) = sum;
        }
    }
    if (tid < listed) __hip_atomic_store(counters + s.list[tid], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace bl
