// How the launches of the attention over 8-bit caches are cut into workgroups: host arithmetic only.
#pragma once
#include <stdint.h>

namespace bl {

constexpr int kRows8Waves = 4;          // waves of a workgroup: a workgroup walks sets of four chunks, a wave one chunk of each
constexpr int kRows8MaxSplits = 64;     // workgroups that share a row's cache: the merge's lanes
constexpr int kRows8Workgroups = 512;   // that a launch aims at: two on each of 256 compute units

constexpr int sets_of(int positions) { return (positions + 64 * kRows8Waves - 1) / (64 * kRows8Waves); }

// A launch's parts: rows (tokens x query heads of a key head) that share a walk, in blocks of up to `block` rows.
struct Rows8Plan {
    int     block;            // rows of a workgroup: 4, 8 or 16
    int     shared_splits;    // workgroups that share the walk over the shared rows; 0: none
    int     shared_blocks;    // row blocks over all tokens
    int     own_splits;       // the same for a sequence's own rows; 0: none
    int     own_blocks;       // row blocks of one sequence's rows
    int64_t shared_wgs, own_wgs;
    int     slots() const { return shared_splits + own_splits; }   // figures that a row's workgroups leave
};

// shared_len: rows of the walk that all tokens share (a prefix, or a prompt's cache), own_len: of each token's own (0: none).
inline Rows8Plan rows8_plan(int n_heads, int group, int tokens, int shared_len, int own_len) {
    Rows8Plan p{};
    const int64_t rows = (int64_t)tokens * group, most = shared_len > 0 ? rows : group;
    p.block = most <= 4 ? 4 : most <= 8 ? 8 : 16;
    p.shared_blocks = shared_len > 0 ? (int)((rows + p.block - 1) / p.block) : 0;
    p.own_blocks = own_len > 0 ? (group + p.block - 1) / p.block : 0;
    const int64_t shared = (int64_t)n_heads * p.shared_blocks, own = (int64_t)n_heads * tokens * p.own_blocks;
    const int shared_sets = shared_len > 0 ? sets_of(shared_len) : 0, own_sets = own_len > 0 ? sets_of(own_len) : 0;
    // sets per workgroup: the fewest with which the launch has no more workgroups than it aims at
    int64_t quota = (shared * shared_sets + own * own_sets + kRows8Workgroups - 1) / kRows8Workgroups;
    const int most_sets = shared_sets > own_sets ? shared_sets : own_sets;
    for (;; quota += quota / 16 + 1) {
        if (quota < 1) quota = 1;
        p.shared_splits = (int)((shared_sets + quota - 1) / quota);
        p.own_splits = (int)((own_sets + quota - 1) / quota);
        if (p.shared_splits <= kRows8MaxSplits && p.own_splits <= kRows8MaxSplits &&
            (quota >= most_sets || shared * p.shared_splits + own * p.own_splits <= kRows8Workgroups))
            break;
    }
    // (the shared part's workgroups go around the dies in eights, all row blocks of a piece of the cache on one die)
    p.shared_wgs = ((int64_t)n_heads * p.shared_splits + 7) / 8 * 8 * p.shared_blocks;
    p.own_wgs = own * p.own_splits;
    return p;
}

// The scratch memory: a counter per (key head, row), a head's in lines of their own, then the figures.
constexpr int64_t rows8_padded(int64_t rows) { return (rows + 31) / 32 * 32; }
inline int64_t rows8_counters(int n_heads, int64_t rows) { return n_heads * rows8_padded(rows); }
inline int64_t rows8_scratch_bytes(const Rows8Plan& p, int n_heads, int64_t rows, int head_dim) {
    return rows8_counters(n_heads, rows) * 4 + n_heads * rows * p.slots() * (head_dim / 2 + 1) * 8;
}

}  // namespace bl
