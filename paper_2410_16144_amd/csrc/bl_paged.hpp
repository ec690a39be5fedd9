// The paged key/value cache (bl_paged_cache): its layout, the rows of a call, and how 32 positions get into LDS.
//
// A pool of pages; a page holds page_size positions of every key head, [page][key head][position][element], bf16, rows of paged_width(head_dim)
// elements.  Positions 16 n .. 16 n + 15 of a sequence lie behind each other whatever the page size (a power of two, 16 at least), so
// everything here goes by sixteens: one entry of the sequence's line of the table, one address.
#pragma once
#include "bl_internal.hpp"
#include "bl_lanes.hpp"

namespace bl {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Elements of a stored row: whole sixteens that the matrix instructions take without a remainder worth speaking of.
constexpr int paged_width(int head_dim) {
    return head_dim <= 32 ? 32 : head_dim <= 48 ? 48 : head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : head_dim <= 128 ? 128 : head_dim <= 192 ? 192 : 256;
}

// The cache and a call's rows as the kernels see them.
struct Paged {
    uint16_t*      k;
    uint16_t*      v;
    const int32_t* table;      // [sequences][table_width]
    const int32_t* pos;        // [sequences]
    const int32_t* start;      // [sequences + 1]; null: row b is sequence b's only one
    int32_t        n_heads, head_dim, page_shift, pages, table_width, sequences, rows, max_pos;
};

inline Paged paged_of(const ::bl_paged_cache& c, const ::bl_paged_rows& r) {
    Paged p;
    p.k = c.k_pages_dev; p.v = c.v_pages_dev;
    p.table = r.table_dev; p.pos = r.pos_dev; p.start = r.start_dev;
    p.n_heads = c.n_heads; p.head_dim = c.head_dim; p.page_shift = 0;
    while ((1 << p.page_shift) < c.page_size) ++p.page_shift;
    p.pages = c.pages; p.table_width = r.table_width; p.sequences = r.sequences; p.rows = r.rows; p.max_pos = r.max_pos;
    return p;
}

// Uniform numbers, in scalar registers: divisions leave them in vector ones.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Numbers that nothing in a launch writes, by scalar loads (the index is uniform).
__device__ __forceinline__ int32_t scalar_word(const int32_t* at, int64_t i) {
    return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)at)[i];
}

struct PagedSequence {
    int first, rows, pos;      // its rows of the call (0: it takes no part), and the position of the first
};
// What the device's words say is looked at before anything is addressed with it.
__device__ __forceinline__ PagedSequence paged_sequence(const Paged& p, int first, int end, int pos) {
    const bool takes_part = first >= 0 && end >= first && end <= p.rows && pos >= 0 && end - first <= p.max_pos && pos <= p.max_pos - (end - first);
    return takes_part ? PagedSequence{first, end - first, pos} : PagedSequence{0, 0, 0};
}
__device__ __forceinline__ PagedSequence paged_sequence(const Paged& p, int b) {   // any lane's own
    return p.start ? paged_sequence(p, p.start[b], p.start[b + 1], p.pos[b]) : paged_sequence(p, b, b + 1, p.pos[b]);
}
__device__ __forceinline__ PagedSequence paged_sequence_uniform(const Paged& p, int b) {
    const int pos = scalar_word(p.pos, b);
    return p.start ? paged_sequence(p, scalar_word(p.start, b), scalar_word(p.start, b + 1), pos) : paged_sequence(p, b, b + 1, pos);
}

// Sum over this lane and those before it, on the vector ALU's lane moves.
__device__ __forceinline__ int wave_inclusive_sum(int v) {
#define BL_BEFORE(ctrl, rows) __builtin_amdgcn_update_dpp(0, v, (ctrl), (rows), 0xf, false)
    v += BL_BEFORE(0x111, 0xf);    // row_shr 1, 2, 4, 8
    v += BL_BEFORE(0x112, 0xf);
    v += BL_BEFORE(0x114, 0xf);
    v += BL_BEFORE(0x118, 0xf);
    v += BL_BEFORE(0x142, 0xa);    // row 0's and 2's last lane to the row behind it
    v += BL_BEFORE(0x143, 0xc);    // lane 31 to the upper half
#undef BL_BEFORE
    return v;
}

// ---- 32 positions of one key head in LDS: rows of 32 KS bytes, their 16-byte pieces moved about so that the reads of the products meet
// all banks: keys by one piece of 16 or 32 rows, values by 32 bytes of four.  Every pattern repeats after 16 rows.
template <int KS>
__device__ __forceinline__ int paged_k_place(int row, int c) {
    return KS == 8 || KS == 16 ? c ^ (row & 15) : KS == 4 || KS == 12 ? c ^ ((row >> 1) & 7) : KS == 2 || KS == 6 ? c ^ ((row >> 2) & 3) : c;
}
template <int KS>
__device__ __forceinline__ int paged_v_place(int row, int c) {
    return KS == 8 || KS == 16 ? c ^ ((row & 3) << 2) : KS == 4 || KS == 12 ? c ^ (((row >> 1) & 1) << 2) : c;
}

// Addresses of the two sixteens of 32 positions of one key head, in the keys' pool or the values' (offsets in bytes).
struct PagedBase {
    int64_t at[2];
    bool    bad;     // the table names a page that is not there
};
// The table's words for 32 positions from j0 on: looked up a request ahead, since a scalar load that is waited for stands in everybody's way.  line: the
// sequence's line of the table; last: its last position.  Sixteens behind it are not looked up.
struct PagedEntries {
    int page[2];
};
__device__ __forceinline__ PagedEntries paged_entries(const Paged& p, const int32_t* line, int j0, int last) {
    return {scalar_word(line, min(j0, last) >> p.page_shift), scalar_word(line, min(j0 + 16, last) >> p.page_shift)};
}
template <int KS>
__device__ __forceinline__ PagedBase paged_base(const Paged& p, const PagedEntries& e, int head, int j0, int last) {
    PagedBase r;
    r.bad = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = min(j0 + 16 * h, last);
        int page = __builtin_amdgcn_readfirstlane(e.page[h]);
        if ((uint32_t)page >= (uint32_t)p.pages) {
            page = 0;
            r.bad = true;
        }
        const int inside = j & ((1 << p.page_shift) - 1) & ~15;
        r.at[h] = ((((int64_t)page * p.n_heads + head) << p.page_shift) + inside) * (32 * KS);
    }
    return r;
}

template <int KS>
struct PagedTile {
    static constexpr int kRow = 32 * KS;
    static constexpr int kBytes = 32 * kRow;                      // KS pieces of 1 KiB
    static constexpr bool kWhole = KS % 2 == 0;                   // a piece lies in one sixteen
    static constexpr int kKept = kWhole ? KS / 2 : KS;            // offsets of a lane
};

// A lane's place in piece s: row and byte offset in the row's memory.
template <int KS, bool VALUE>
__device__ __forceinline__ void paged_piece(int s, int lane, int& row, int& byte) {
    const int at = s * 64 + lane;
    row = at / (2 * KS);
    const int place = at % (2 * KS);
    byte = (VALUE ? paged_v_place<KS>(row, place) : paged_k_place<KS>(row, place)) * 16;
}

struct PagedSource {
    const uint8_t* at[2];   // of the two sixteens
};
__device__ __forceinline__ PagedSource paged_source(const uint16_t* pool, const PagedBase& base) {
    const uint8_t* at = reinterpret_cast<const uint8_t*>(pool);
    return {{at + base.at[0], at + base.at[1]}};
}

// Positions behind the sequence's last one come as they lie in their page, or as another sixteen: whatever they are, nobody sees them.  STREAM: by
// streaming (nontemporal) loads, for a cache that a launch reads once.  LEAN: a lane's offsets are worked out from one at each request, for kernels that have no
// registers for eight (from scratch memory each came behind the request before it: 655 rows of 16 heads of 256 on 2 behind 3316 positions, fp32, 395 us, like this 274).
template <int KS, bool STREAM, bool LEAN = false>
struct PagedRequest {
    static_assert(!LEAN || KS == 16, "forms in use");
    uint32_t off[LEAN ? 1 : PagedTile<KS>::kKept];   // in a sixteen
    bool     value;                                  // LEAN
    __device__ __forceinline__ uint32_t offset(int s) const {
        if constexpr (LEAN) {                              // piece s has rows 2 s and 2 s + 1; its places differ from piece 0's by what paged_k_place or paged_v_place make of 2 s
            uint32_t first = off[0];
            asm volatile("" : "+v"(first));
            s %= PagedTile<KS>::kKept;
            return (first ^ (value ? 128u * (s & 1) : 32u * s)) + 1024u * s;
        } else {
            return off[s % PagedTile<KS>::kKept];
        }
    }
    template <bool VALUE>
    __device__ __forceinline__ void prepare(int lane) {
        value = VALUE;
        if constexpr (LEAN) {
            int row, byte;
            paged_piece<KS, VALUE>(0, lane, row, byte);
            off[0] = (uint32_t)(row * PagedTile<KS>::kRow + byte);
            return;
        }
#pragma unroll
        for (int s = 0; s < (LEAN ? 0 : PagedTile<KS>::kKept); ++s) {
            int row, byte;
            paged_piece<KS, VALUE>(s, lane, row, byte);
            off[s] = (uint32_t)((row & 15) * PagedTile<KS>::kRow + byte);
        }
    }
    // One of KS pieces of 1 KiB on its way to LDS address dst (uniform, as everything here that is no lane's), by all lanes, which are active here.  ANY:
    // by the lanes of `who`: all or, where there is nothing to bring, none, without a branch between the products.
    template <bool ANY = false>
    __device__ __forceinline__ void piece(int s, const PagedSource& from, uint32_t dst, uint64_t who = ~0ull) const {
        const uint32_t to = __builtin_amdgcn_readfirstlane(dst + 1024 * s);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
        if constexpr (PagedTile<KS>::kWhole) {
            const uint8_t* src = uniform_ptr(from.at[2 * s / KS]);
            const uint32_t o = offset(s);
            static_assert(!(ANY && STREAM), "forms in use");
            if constexpr (STREAM)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(to), "v"(o), "s"(src) : "memory", "m0");
            else if constexpr (ANY)
                asm volatile("s_mov_b64 exec, %3\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1"
                             ::"s"(to), "v"(o), "s"(src), "s"(who) : "memory", "m0", "exec");
            else
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(o), "s"(src) : "memory", "m0");
        } else {   // a piece lies in both sixteens
            const int row = (s * 64 + (int)(threadIdx.x & 63)) / (2 * KS);
            const uint8_t *first = from.at[0], *second = from.at[1], *src = (row < 16 ? first : second) + off[s];
            if constexpr (ANY)
                asm volatile("s_mov_b64 exec, %2\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b64 exec, -1"
                             ::"s"(to), "v"(src), "s"(who) : "memory", "m0", "exec");
            else
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(src) : "memory", "m0");
        }
#pragma clang diagnostic pop
    }
    template <bool ANY = false>
    __device__ __forceinline__ void send(const PagedSource& from, uint32_t dst, uint64_t who = ~0ull) const {   // all of them
#pragma unroll
        for (int s = 0; s < KS; ++s) piece<ANY>(s, from, dst, who);
    }
};

__device__ __forceinline__ uint32_t lds_address(const void* at) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)at; }

// ---- operands

__device__ __forceinline__ uint32_t paged_bf16_pair(float a, float b) {   // rounded to nearest even, the first in the low half
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// Two numbers as PIECES bf16 numbers each, the first one's in the low halves: one, rounded; two, of which the second is the rounded rest (16 bits);
// three by cutting off 8 bits at a time, whose sum is the number itself (24 bits; nothing rounds up to an infinity).
template <int PIECES>
__device__ __forceinline__ void paged_split(float a, float b, uint32_t (&out)[PIECES]) {
    if constexpr (PIECES == 1) {
        out[0] = paged_bf16_pair(a, b);
    } else {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if (PIECES == 2 && i == 1) {
                out[i] = paged_bf16_pair(a, b);
                break;
            }
            const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
            out[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            a -= __uint_as_float(x & 0xffff0000u);
            b -= __uint_as_float(y & 0xffff0000u);
        }
    }
}

// Eight elements e .. e + 7 of a row's query (zeros from head_dim on and in rows that are not there, whose row_at is another's; head_dim is a multiple of
// four, e of eight) as operand pieces.  fp32 is loaded by every lane: in a branch, each load would be waited for by its cutting into pieces (12 heads of 64 at
// position 17: 7.2 us, so 6.7); bf16 has nothing to cut, and idle lanes' loads would cost it 0.3 us.
template <int PIECES>
__device__ __forceinline__ void paged_query(const void* q, int64_t row_at, int e, int head_dim, bool there, s16x8 (&out)[PIECES]) {
    uint32_t parts[PIECES][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const bool in = there && e + 4 * h < head_dim;
        if constexpr (PIECES == 1) {
            typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(2)));
            u32x2_u x = {0, 0};
            if (in) x = *reinterpret_cast<const u32x2_u*>(static_cast<const uint16_t*>(q) + row_at + e + 4 * h);
            parts[0][2 * h] = x[0];
            parts[0][2 * h + 1] = x[1];
        } else {
            const int64_t at = row_at + min(e + 4 * h, head_dim - 4);
            typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
            const f32x4_u x = *reinterpret_cast<const f32x4_u*>(static_cast<const float*>(q) + at);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t two[PIECES];
                paged_split<PIECES>(in ? x[2 * j] : 0.0f, in ? x[2 * j + 1] : 0.0f, two);
#pragma unroll
                for (int i = 0; i < PIECES; ++i) parts[i][2 * h + j] = two[i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) out[i] = __builtin_bit_cast(s16x8, (u32x4{parts[i][0], parts[i][1], parts[i][2], parts[i][3]}));
}

// Whether a bf16 number is an infinity or NaN, of the two in a word: the largest exponents seen, to be told at the end.
__device__ __forceinline__ uint32_t paged_exponents(uint32_t most, uint32_t word) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    const u16x2 a = __builtin_bit_cast(u16x2, most), b = __builtin_bit_cast(u16x2, word & 0x7f807f80u);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(a, b));
}
__device__ __forceinline__ bool paged_not_finite(uint32_t most) { return (most & 0xffffu) == 0x7f80u || most >> 16 == 0x7f80u; }

// Keys before queries of several pieces: a piece of zero times an infinity is NaN, where the query's element makes an infinity of it.  So the keys' numbers that
// are not finite are multiplied apart, by the elements' signs (of zero: zero).
__device__ __forceinline__ void paged_apart(const s16x8& k, s16x8& finite, s16x8& odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        odd[i] = (k[i] & 0x7f80) == 0x7f80 ? k[i] : (short)0;
        finite[i] = k[i] ^ odd[i];
    }
}
template <int PIECES>
__device__ __forceinline__ s16x8 paged_signs(const s16x8 (&q)[PIECES]) {
    s16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        short any = 0;
#pragma unroll
        for (int n = 0; n < PIECES; ++n) any |= q[n][i] & 0x7fff;
        r[i] = any ? (short)((q[0][i] & 0x8000) | 0x3f80) : (short)0;
    }
    return r;
}

// Values with infinities and NaN put away: the finite ones, and ones where +infinity (or NaN) and -infinity (or NaN) were.
__device__ __forceinline__ void paged_put_away(const s16x8& v, s16x8& finite, s16x8& up, s16x8& down) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t x = (uint16_t)v[i], size = x & 0x7fffu;
        const bool odd = size >= 0x7f80u, nan = size > 0x7f80u;
        finite[i] = odd ? (short)0 : v[i];
        up[i] = odd && (nan || x < 0x8000u) ? (short)0x3f80 : (short)0;
        down[i] = odd && (nan || x >= 0x8000u) ? (short)0x3f80 : (short)0;
    }
}

// A row's four outputs.
template <bool BF16>
__device__ __forceinline__ void paged_store(void* out, int64_t at, const f32x4& x) {
    if constexpr (BF16) {
        typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(2)));
        *reinterpret_cast<u32x2_u*>(static_cast<uint16_t*>(out) + at) = u32x2_u{paged_bf16_pair(x[0], x[1]), paged_bf16_pair(x[2], x[3])};
    } else {
        typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));
        *reinterpret_cast<f32x4_u*>(static_cast<float*>(out) + at) = x;
    }
}

// ---- who does what: the attention's launches
//
// A sequence's rows of one key head (tokens x query heads of the group, token by token) go by tiles; a tile's walk over the positions up to its last row's
// may be shared by several workgroups.  How many follows on the device from all positions that the call walks: each workgroup is meant to have
// an equal share of them, kPagedLeast at least.  The grid is an upper bound; workgroups beyond what there is to do end at once.

constexpr int kPagedTileParts = 32;   // workgroups that share a tile's walk at most
constexpr int kPagedLeast = 256;      // positions that are worth a workgroup
constexpr int kPagedFew = 16;         // rows of a sequence and key head up to which the rows form takes them

struct PagedArgs {
    Paged       c;
    const void* q;
    void*       out;
    uint32_t*   counters;      // [slot]: tickets of the walks whose first slot it is
    float*      figures;       // [slot]: maxima, sums and weighted values of a tile's rows, as each form has them
    int32_t     slot_bytes;
    int32_t     group;         // query heads per key head
    int32_t     tile_rows;     // a power of two, or (rows form) the group
    int32_t     tile_shift;
    int32_t     most;          // workgroups of a walk
    float       join;          // tiles: positions that are walked while a part is joined
    int32_t     slots;         // of figures
    int32_t     shallow;       // tiles of 64 rows: whether two workgroups are to share a compute unit
    float       target;        // key heads / workgroups that the call is meant for
    float       scale;         // log2(e) / sqrt(head_dim)
};

struct PagedWork {
    PagedSequence s;
    int b, head;
    int row0, rows;            // the tile's rows, of the sequence's
    int low, reach;            // the last position that its first row sees; positions that its last row sees
    int part, parts;           // which of the walk's workgroups this is
    int slot;                  // of the walk's first part; its others' behind it
};

// (Every workgroup passes all of this once: with 64-bit divisions, a hundred instructions each, a call took 0.5 us more, one in several parts 1.)
template <bool ROWS>
__device__ __forceinline__ int paged_tiles(const PagedArgs& p, int rows) { return ROWS ? rows : (rows * p.group + p.tile_rows - 1) >> p.tile_shift; }   // (2^30 at most)
// Parts of a walk with `per` positions each: rounded up, or (tiles, where joining a part takes as long as `join` positions) down and by no more than
// makes walking (reach / parts) and joining (parts * join) the shortest together.
template <bool ROWS>
__device__ __forceinline__ int paged_parts(const PagedArgs& p, const PagedSequence& s, int per) {
    const int reach = s.pos + s.rows;
    return min(ROWS ? (reach - 1) / per + 1 : max(reach / max(per, (int)sqrtf(p.join * (float)reach)), 1), p.most);
}

// What the call walks of a sequence, in positions (its tiles' mean).
template <bool ROWS>
__device__ __forceinline__ float paged_cost(const PagedArgs& p, const PagedSequence& s) {
    return s.rows ? (float)paged_tiles<ROWS>(p, s.rows) * ((float)(s.pos + s.rows) - 0.5f * (float)(s.rows - 1)) : 0.0f;
}

// By every wave for itself, a lane for every (sequences / 64) of them.  False: nothing to do.
template <bool ROWS>
__device__ __forceinline__ bool paged_work(const PagedArgs& p, int lane, PagedWork& w) {
    const Paged& c = p.c;
    const int item = uniform((int)blockIdx.x / c.n_heads), items = uniform((int)gridDim.x / c.n_heads);
    w.head = (int)blockIdx.x - item * c.n_heads;
    const int each = (c.sequences + 63) >> 6;
    int index = item, first_slot = 0, per;
    // (a little more than the quotient, so that there are never more parts than the grid has: see paged_plan)
    const auto share = [&](float cost) { return __builtin_amdgcn_readfirstlane(max(kPagedLeast, (int)fminf(cost * p.target * 1.0001f, 2.0e9f) + 1)); };
    if (c.sequences == 1) {
        w.b = 0;
        w.s = paged_sequence_uniform(c, 0);
        per = share(paged_cost<ROWS>(p, w.s));
    } else {
        PagedSequence mine{0, 0, 0};
        float cost = 0.0f;
        for (int i = 0; i < each; ++i)
            if (lane * each + i < c.sequences) {
                mine = paged_sequence(c, lane * each + i);
                cost += paged_cost<ROWS>(p, mine);
            }
        per = share(over_lanes<64>(cost, AddOp()));
        int sum = 0, shared = 0;
        const auto count = [&](const PagedSequence& s, int& n, int& shared_n) {
            const int parts = s.rows ? paged_parts<ROWS>(p, s, per) : 0;
            n = parts ? paged_tiles<ROWS>(p, s.rows) * parts : 0;
            shared_n = parts > 1 ? n : 0;
        };
        for (int i = 0; i < each; ++i)
            if (lane * each + i < c.sequences) {
                if (each > 1) mine = paged_sequence(c, lane * each + i);
                int n, shared_n;
                count(mine, n, shared_n);
                sum += n;
                shared += shared_n;
            }
        const int upto = wave_inclusive_sum(sum), shared_upto = wave_inclusive_sum(shared);
        const unsigned long long later = __ballot(item < upto);
        if (later == 0) return false;
        const int which = __builtin_ctzll(later);
        index = item - __builtin_amdgcn_readlane(upto - sum, which);
        first_slot = __builtin_amdgcn_readlane(shared_upto - shared, which);
        for (w.b = which * each;; ++w.b) {                 // (the item is one of this lane's sequences'; where rows overlap, sums may mean nothing)
            if (w.b >= c.sequences || index < 0) return false;
            w.s = paged_sequence_uniform(c, w.b);
            int n, shared_n;
            count(w.s, n, shared_n);
            if (index < n) break;
            index -= n;
            first_slot += shared_n;
        }
    }
    if (w.s.rows == 0) return false;
    const int tiles = uniform(paged_tiles<ROWS>(p, w.s.rows)), all = w.s.rows * p.group;
    w.parts = uniform(paged_parts<ROWS>(p, w.s, per));
    const int turn = uniform(index / w.parts);
    w.part = index - turn * w.parts;
    if (turn >= tiles || item - w.part + w.parts > items) return false;   // (a walk that the grid has no room for, as where sequences overlap: nobody's)
    w.row0 = (tiles - 1 - turn) * p.tile_rows;             // the longest walk first
    w.rows = min(p.tile_rows, all - w.row0);
    w.low = w.s.pos + uniform(w.row0 / p.group);
    w.reach = w.s.pos + uniform((w.row0 + w.rows - 1) / p.group) + 1;
    w.slot = (first_slot + turn * w.parts) * c.n_heads + w.head * w.parts;
    w.parts = min(w.parts, (w.reach + kPagedLeast - 1) / kPagedLeast);   // (a sequence's first tiles walk less than its last one)
    if (w.part >= w.parts) return false;
    if (w.parts > 1 && (uint32_t)w.slot > (uint32_t)(p.slots - w.parts)) {   // (never, see paged_plan)
        if (w.part) return false;
        w.parts = 1;
    }
    return true;
}

// The first of a walk's chunks that part n has (there are as many chunks as parts at least).
__device__ __forceinline__ int paged_first(const PagedWork& w, int chunks, int n) {
    const int each = uniform(chunks / w.parts);
    return n * each + min(n, chunks - each * w.parts);
}

__device__ __forceinline__ int64_t paged_row_at(const PagedArgs& p, const PagedWork& w, int row) {   // of q and out; row of the tile
    const int of = w.row0 + row, token = of / p.group;
    return (((int64_t)(w.s.first + token) * p.c.n_heads + w.head) * p.group + of - token * p.group) * p.c.head_dim;
}

// ---- the parts of a walk meet
//
// Every part's figures travel by device-scope stores of 16 bytes, performed past the dies' caches; every thread waits until its own have been
// performed, then the workgroup draws a ticket, and the one that draws the last reads all of them, by device-scope loads, and adds them up in the
// parts' order.  Nobody waits for anybody.

constexpr int kDeviceScope = 16;       // the buffer instructions' sc1
__device__ __forceinline__ __amdgpu_buffer_rsrc_t paged_resource(float* at) { return __builtin_amdgcn_make_buffer_rsrc(at, 0, -1, 0x00027000); }
__device__ __forceinline__ float* paged_slot(const PagedArgs& p, int slot) {
    return reinterpret_cast<float*>(const_cast<uint8_t*>(uniform_ptr(reinterpret_cast<const uint8_t*>(p.figures) + (int64_t)slot * p.slot_bytes)));
}
__device__ __forceinline__ void paged_leave(__amdgpu_buffer_rsrc_t slot, int byte, const f32x4& x) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), slot, byte, 0, kDeviceScope);
}
__device__ __forceinline__ f32x4 paged_read(__amdgpu_buffer_rsrc_t slot, int byte) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(slot, byte, 0, kDeviceScope));
}
__device__ __forceinline__ float2 paged_read_pair(__amdgpu_buffer_rsrc_t slot, int byte) {
    const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(slot, byte, 0, kDeviceScope);
    return make_float2(__uint_as_float(x[0]), __uint_as_float(x[1]));
}

// Whether this workgroup is the walk's last, all of whose figures are there now.
__device__ __forceinline__ bool paged_last(const PagedArgs& p, const PagedWork& w, int& last_one) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t* counter = p.counters + w.slot;
        last_one = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(w.parts - 1);
        if (last_one) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return uniform(last_one) != 0;
}

// The weight of a finite score is above zero, however small: what an infinite value is multiplied by must not be zero, or NaN comes of it, and only where
// one part of a walk, or one order of its chunks, has it so.  (The smallest number there is: of finite values nothing comes of it that counts.)
__device__ __forceinline__ float paged_above_zero(float x) { return x < 0x1p-149f ? 0x1p-149f : x; }   // (NaN stays)

// What a part's, or a wave's, figures are multiplied by to be relative to the maximum `top`: nothing where a row has seen nothing, or scores of -infinity alone
// (whose sums may be NaN, and stay it); NaN weights stay NaN.
__device__ __forceinline__ float paged_factor(float m, float l, float scale, float top) {
    return m == -INFINITY ? (l == 0.0f ? 0.0f : NAN) : paged_above_zero(__builtin_amdgcn_exp2f((m - top) * scale));
}

}  // namespace bl
