// How the launches of the attention over 8-bit caches are cut into workgroups: host arithmetic only.
#pragma once
#include <stdint.h>

namespace bl {

constexpr int kAttn8Waves = 4;            // waves of a workgroup
constexpr int kRows8Set = 256;            // positions that a workgroup of the rows form walks at a time: a chunk of 64 per wave
constexpr int kTiles8Set = 128;           // ... of the tiles form: 32 per wave
constexpr int kTiles8Rows = 32;           // rows of a workgroup of the tiles form
constexpr int kAttn8MaxSplits = 64;       // workgroups that share a row's walk: the merge's lanes
#ifndef WGS
#define WGS 512
#endif
constexpr int kAttn8Workgroups = WGS;     // that a launch aims at: two on each of 256 compute units

// Division by a number that the host knows, for 0 <= n < 2^31: n m >> (31 + s) with 2^s >= d and m = 2^(31 + s) / d rounded up.  m d exceeds
// 2^(31 + s) by less than d <= 2^s, so n m / 2^(31 + s) exceeds n / d by less than 1 / d: the same whole number.  (A workgroup that divides
// its index by unknown numbers spends some forty instructions on each, one after another, ahead of its first request.)
struct Divider {
    uint32_t m, shift;   // m = 0: by one
};
constexpr Divider divider(int d) {
    if (d <= 1) return {0, 0};
    uint32_t s = 1;
    while ((1ll << s) < d) ++s;
    return {(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s - 1};
}
constexpr int divided(int n, Divider by) { return by.m ? (int)((uint32_t)(((uint64_t)(uint32_t)n * by.m) >> 32) >> by.shift) : n; }

constexpr int sets_of(int positions, int set) { return (positions + set - 1) / set; }

// A launch's parts.  Shared: the walk that all tokens share (a prefix, or a prompt's cache), in blocks of rows, all of them by each piece of the
// walk.  Own: each sequence's own rows.
struct Attn8Plan {
    int     tiles;            // the shared part in tiles of 32 rows; else (and the own part) rows in fours
    int     block;            // rows of a workgroup of the rows form: 4, 8 or 16
    int     shared_set;       // positions of a set of the shared part
    int     shared_splits;    // workgroups that share the walk over the shared rows; 0: none
    int     shared_blocks;    // row blocks over all tokens
    int     own_splits;       // the same for a sequence's own rows; 0: none
    int     own_blocks;       // row blocks of one sequence's rows
    int64_t shared_wgs, own_wgs;
    int     slots() const { return shared_splits + own_splits; }   // figures that a row's workgroups leave
};

// shared_len: positions of the shared walk, own_len: of each token's own (0: none).
inline Attn8Plan attn8_plan(int n_heads, int group, int tokens, int shared_len, int own_len) {
    Attn8Plan p{};
    const int64_t rows = (int64_t)tokens * group;
    p.tiles = shared_len > 0 && rows > 4;
    const int64_t most = p.tiles ? (own_len > 0 ? 4 : 0) : shared_len > 0 ? rows : group;   // (beside tiles: fours)
    p.block = most <= 4 ? 4 : most <= 8 ? 8 : 16;
    const int shared_block = p.tiles ? kTiles8Rows : p.block;
    p.shared_set = p.tiles ? kTiles8Set : kRows8Set;
    p.shared_blocks = shared_len > 0 ? (int)((rows + shared_block - 1) / shared_block) : 0;
    p.own_blocks = own_len > 0 ? (group + p.block - 1) / p.block : 0;
    const int64_t shared = (int64_t)n_heads * p.shared_blocks, own = (int64_t)n_heads * tokens * p.own_blocks;
    // positions per workgroup: the fewest with which the launch has no more workgroups than it aims at
    const auto splits = [](int len, int set, int64_t quota) {
        const int64_t sets = quota / set > 1 ? quota / set : 1;
        return len > 0 ? (int)((sets_of(len, set) + sets - 1) / sets) : 0;
    };
    const int longest = shared_len > own_len ? shared_len : own_len;
    for (int64_t quota = kTiles8Set;; quota += quota / 16 / kTiles8Set * kTiles8Set + kTiles8Set) {
        p.shared_splits = splits(shared_len, p.shared_set, quota);
        p.own_splits = splits(own_len, kRows8Set, quota);
        if (p.shared_splits <= kAttn8MaxSplits && p.own_splits <= kAttn8MaxSplits &&
            (quota >= longest + kRows8Set || shared * p.shared_splits + own * p.own_splits <= kAttn8Workgroups))
            break;
    }
    // (the shared part's workgroups go around the dies in eights, all row blocks of a piece of the cache on one die)
    p.shared_wgs = ((int64_t)n_heads * p.shared_splits + 7) / 8 * 8 * p.shared_blocks;
    p.own_wgs = own * p.own_splits;
    return p;
}

// The scratch memory: a counter per (key head, row), a head's in lines of their own, then the figures.
constexpr int64_t attn8_padded(int64_t rows) { return (rows + 31) / 32 * 32; }
inline int64_t attn8_counters(int n_heads, int64_t rows) { return n_heads * attn8_padded(rows); }
inline int64_t attn8_scratch(const Attn8Plan& p, int n_heads, int64_t rows, int head_dim) {
    return attn8_counters(n_heads, rows) * 4 + n_heads * rows * p.slots() * (head_dim / 2 + 1) * 8;
}

}  // namespace bl
