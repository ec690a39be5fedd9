// How the launches of the attention over 8-bit caches are cut into workgroups: host arithmetic only.
#pragma once
#include <stdint.h>

namespace bl {

constexpr int kAttn8Units = 256;          // compute units
// Rows that share a walk and go without tiles.  32 heads of 128, rows and tiles, us: 5 tokens behind 8000 22.9 and 26.8, 8 behind 500 13.4 and 14.2;
// 16 (in sixteens) 32.7 and 27.7, 21.6 and 15.6.
constexpr int kRows8Most = 8;
// Waves of a workgroup of the rows form, each with a chunk of 64 positions at a time: eight, with many heads and sequences fewer: more workgroups than
// compute units.  A unit holds one workgroup of eight waves (133 registers) and six of two, and what a short walk takes is waiting.  Rows in fours,
// 32 heads of 128, caches of 17 positions, eight waves and two, us: 16 sequences 10.2 and 7.2, 32 20.1 and 10.3, 64 37.4 and 17.5.  In eights, eight
// waves and four: a token at 100 000, 64 heads on 8, 41.6 and 49.2; 40 sequences of 64 on 8 at 300 positions 15.1 and 12.5.  In sixteens: 64 on 4 at
// 20 000 22.8 and 29.5, 96 sequences at 300 22.3 and 19.4; head sizes above 128 have no room for eight such waves' sums.
constexpr int kRows8Waves = 8;
constexpr int kRows8FewWaves = 4;         // in eights and sixteens, and beside tiles
constexpr int kRows8ManyWaves = 2;        // in fours
// Own walks beside tiles, in their kernel, share a unit two by two with them and run while the tiles do; more of them are launched by themselves.  32
// heads of 128 behind a prefix of 100, 300 own positions, in one launch and in two, us: 40 sequences 24.4 and 32.2, 64 36.6 and 41.4, 80 45.0 and 46.9, 128
// 66.0 and 63.2; 20 own positions: 40 21.3 and 23.7, 64 30.6 and 29.2, 128 49.5 and 41.9.
constexpr int kAttn8Beside = 8 * kAttn8Units;
constexpr int kTiles8Set = 7;             // positions that a workgroup of the tiles form walks at a time: 1 << 7, 32 per wave
constexpr int kTiles8Rows = 32;           // rows of a tile
constexpr int kAttn8MaxSplits = 64;       // workgroups that share a row's walk: the merge's lanes
constexpr int kAttn8Waves = 2048;         // that a launch aims at: two on each SIMD of 256 compute units
// ... and, where the own walks alone are as many, that the walk of the prefix has all the same.  Sixteen sequences of 32 heads behind 8000 positions, 20 of
// their own: 25.7 us, with half as many 32.0, without 84.
constexpr int kAttn8SharedWaves = 1024;
// A short walk that meets nobody else is not split: the meeting (figures performed, tickets, figures read: three trips to memory) takes 3.6 us, a
// set of 512 positions in one compute unit 1.0 us with a head size of 64 and 1.8 with 128.  One workgroup per head and one per set, us: 32 heads
// of 128 at 1000 positions 9.3 and 10.5, at 2000 12.9 and 10.9; 12 of 64 at 1000 6.7 and 9.0, at 2000 8.7 and 9.3.  (By the cache's size, which the host
// knows, not by the position: at 1000 of 8192 positions a token's walk is one workgroup per set.)
constexpr int kRows8Together = 256 << 10;   // bytes of codes

// What splitting a prompt's walk in tiles takes and saves, in tenths of a microsecond (32 heads of 128): a set of 128 positions with one wave on a SIMD and
// with two; the merging launch; 100 rows' figures, out and in.  As planned and in one piece, us: 256 tokens behind 600 32.8 and 25.1, 200 behind none 22.3
// and 16.6, behind 1500 35.6 and 32.0; the other way 20 tokens behind 1000 17.4 and 22.7, 40 behind 2000 22.4 and 32.7; 77 behind 1000 24.1 and 25.0.
constexpr int kTiles8SetAlone = 14, kTiles8SetBeside = 20, kTiles8Merge = 40;

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

constexpr int sets_of(int positions, int set) { return (int)(((int64_t)positions + (1 << set) - 1) >> set); }   // of 1 << set positions

// A launch's parts.  Shared: the walk that all tokens share (a prefix, or a prompt's cache), in blocks of rows, all of them by each piece of the
// walk.  Own: each sequence's own rows.
struct Attn8Plan {
    int     tiles;            // the shared part in tiles of 32 rows; else (and the own part) rows in fours
    int     tile_rows;        // rows of a workgroup of the tiles form: 32, 64 or 128
    int     folded;           // a workgroup takes two of a prompt's blocks, from both ends: all walk as much, to the launch's end
    int     block;            // rows of a workgroup of the rows form: 4, 8 or 16
    int     shared_set, own_set;   // 1 << so many positions are a workgroup's set
    int     waves;            // of a workgroup of the rows form
    int     apart;            // the own part is a launch of its own, behind the one of the tiles
    int     shared_splits;    // workgroups that share the walk over the shared rows; 0: none
    int     shared_blocks;    // row blocks over all tokens
    int     own_splits;       // the same for a sequence's own rows; 0: none
    int     own_blocks;       // row blocks of one sequence's rows
    int     strips;           // dies that a piece of the shared walk's row blocks go to
    int64_t shared_units;     // workgroups of one block in every strip of every piece, in whole rounds of the dies
    int64_t shared_wgs, own_wgs;
    int     slots() const { return shared_splits + own_splits; }   // figures that a row's workgroups leave
    bool    meets() const { return !tiles && slots() > 1; }        // the workgroups of a row meet by counters (else: one, or a merging launch)
    bool    launchable() const {                                   // fewer than 2^32 threads in each launch
        const int64_t rows_threads = 64 * waves, tiles_threads = tiles ? 64 * kRows8FewWaves : rows_threads;
        return (apart ? shared_wgs : shared_wgs + own_wgs) * tiles_threads < 1ll << 32 && own_wgs * rows_threads < 1ll << 32;
    }
};

// shared_len: positions of the shared walk, own_len: of each token's own (0: none).  size: bytes of a row of codes.
inline Attn8Plan attn8_plan(int n_heads, int group, int tokens, int shared_len, int own_len, int size) {
    Attn8Plan p{};
    const int64_t rows = (int64_t)tokens * group;
    p.tiles = shared_len > 0 && rows > kRows8Most;
    const int64_t most = p.tiles ? (own_len > 0 ? 4 : 0) : shared_len > 0 ? rows : group;   // (beside tiles: fours)
    p.block = most <= 4 ? 4 : most <= 8 ? 8 : 16;
    p.own_blocks = own_len > 0 ? (group + p.block - 1) / p.block : 0;
    const int64_t own = (int64_t)n_heads * tokens * p.own_blocks;
    p.apart = p.tiles && own > kAttn8Beside;
    const bool many = (own > 0 ? own : n_heads * ((rows + p.block - 1) / p.block)) > kAttn8Units;
    if (p.tiles && !p.apart) p.waves = kRows8FewWaves;
    else if (p.block == 4) p.waves = many ? kRows8ManyWaves : kRows8Waves;
    else p.waves = many || (p.block == 16 && size > 128) ? kRows8FewWaves : kRows8Waves;
    p.own_set = p.waves == kRows8Waves ? 9 : p.waves == kRows8FewWaves ? 8 : 7;
    // A prompt of many rows: two or four tiles per workgroup, and folded where that leaves enough of them: unfolded, a compute unit's last long
    // block runs alone.  32 heads of 128, unfolded and folded, us: 2048 tokens 114 and 106, behind 16 000 1107 and 1060, 4096 325 and 311; with one tile
    // per workgroup it cost (1024 tokens: two tiles unfolded 43, one folded 49).
    const auto enough = [&](int more, int fold) {
        const int64_t blocks = (rows + (kTiles8Rows << more) - 1) / (kTiles8Rows << more);
        return p.tiles && own_len == 0 && n_heads * ((blocks + fold - 1) / fold) * kRows8FewWaves >= kAttn8Waves;
    };
    p.folded = enough(1, 2);
    const int more = enough(2, 2) ? 2 : enough(1, 1) ? 1 : 0;
    p.tile_rows = kTiles8Rows << more;
    const int shared_block = p.tiles ? p.tile_rows : p.block;
    p.shared_set = p.tiles ? kTiles8Set - more : p.own_set;
    p.shared_blocks = shared_len > 0 ? (int)((rows + shared_block - 1) / shared_block) : 0;
    const int64_t shared = (int64_t)n_heads * p.shared_blocks;
    // positions per workgroup: the fewest with which the launch has no more workgroups than it aims at
    const auto splits = [](int len, int set, int64_t quota) {
        const int64_t sets = quota >> set > 1 ? quota >> set : 1;
        return len > 0 ? (int)((sets_of(len, set) + sets - 1) / sets) : 0;
    };
    const auto share = [&](int shared_now, int own_now) {   // the splits of one launch
        const int64_t longest = shared_now > own_now ? shared_now : own_now, unit = 1 << (own_now > 0 ? p.own_set : p.shared_set);
        const bool together = !p.tiles && (shared_now == 0 || own_now == 0) && sets_of((int)longest, p.own_set) * unit * 2 * size <= kRows8Together;
        for (int64_t quota = together || more ? longest + unit : unit;; quota += quota / 16 / unit * unit + unit) {
            const int a = splits(shared_now, p.shared_set, quota), b = splits(own_now, p.own_set, quota);
            if (a > kAttn8MaxSplits || b > kAttn8MaxSplits) continue;
            const int64_t shared_waves = shared * a * (p.tiles ? kRows8FewWaves : p.waves);
            const bool fits = shared_waves + own * b * p.waves <= kAttn8Waves || (b == 1 && shared_waves <= kAttn8SharedWaves);
            if (!more && quota < longest + unit && !fits) continue;
            if (shared_now > 0) p.shared_splits = a;
            if (own_now > 0) p.own_splits = b;
            return;
        }
    };
    if (p.apart) {
        share(shared_len, 0);
        share(0, own_len);
    } else {
        share(shared_len, own_len);
    }
    if (p.tiles && own_len == 0 && p.shared_splits > 1) {
        const int64_t sets = sets_of(shared_len, p.shared_set), most = (sets + p.shared_splits - 1) / p.shared_splits, wide = size > 128 ? size : 128;
        const int64_t set = shared * p.shared_splits > kAttn8Units ? kTiles8SetBeside : kTiles8SetAlone;
        if (sets * kTiles8SetAlone * wide / 128 <= most * set * wide / 128 + kTiles8Merge + n_heads * rows / 100 * wide / 128) p.shared_splits = 1;
    }
    // The shared part's workgroups go around the dies in eights, all row blocks of a piece of the cache to one die.  A prompt with few pieces, not a multiple
    // of eight, would leave dies without work: there two, four or eight dies take a piece's blocks in turn.  300 tokens, 16 heads of 256 on 2, us:
    // 64.5 and 32.4, 1500 404 and 114; 1500, 28 of 128 on 4 87.7 and 54.6; with 32 pieces and more it costs (100 behind 3000, 12 of 64, 19.6 and 20.5).
    const int64_t turns = p.folded ? (p.shared_blocks + 1) / 2 : p.shared_blocks, pieces = (int64_t)n_heads * p.shared_splits;
    p.strips = 1;
    if (p.tiles && own_len == 0 && pieces < 32)
        while (pieces * p.strips % 8 != 0) p.strips *= 2;
    if (turns < p.strips) p.strips = 1;
    p.shared_units = (pieces * p.strips + 7) / 8 * 8;
    p.shared_wgs = p.shared_units * ((turns + p.strips - 1) / p.strips);
    p.own_wgs = own * p.own_splits;
    return p;
}

// The scratch memory: a counter per (key head, row), a head's in lines of their own, then the figures (none where a row has one workgroup).  0: a batch or prompt too large
// for a launch.
constexpr int64_t attn8_padded(int64_t rows) { return (rows + 31) / 32 * 32; }
inline int64_t attn8_counters(int n_heads, int64_t rows) { return n_heads * attn8_padded(rows); }
inline int64_t attn8_scratch(const Attn8Plan& p, int n_heads, int64_t rows, int head_dim) {
    if (!p.launchable()) return 0;
    return attn8_counters(n_heads, rows) * 4 + (p.slots() > 1 ? n_heads * rows * p.slots() * (head_dim / 2 + 1) * 8 : 0);
}

}  // namespace bl
