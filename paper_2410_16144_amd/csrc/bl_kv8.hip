// bl_kv8_write and bl_kv8_read: rows into the 8-bit cache and out of it (layout: bl_kv8.hpp).
//
// One workgroup per (chunk of 64 positions, key head, keys or values).  A write is a stream of projections in and a quarter of their bytes
// (half, from bf16) out: every row's largest value stays in the registers of the lanes that hold the row -- one read -- and the
// codes are put into the cache's order in LDS, since a value's neighbours in memory are the same dim's of other positions.  Four rows
// are a thread's, so that both orders are written and read by words (2000 bf16 rows, 32 heads of 128, written and read back, 49 MB each way: byte
// by byte 31.5 us, by words 24.6; copying as many bytes at the card's 5.2 TB/s: 19).  A chunk that the call covers in part is written row
// by row (keys) and byte by byte (values): the bytes between belong to other positions.
#include "bl_kv8.hpp"
#include "bl_lanes.hpp"

namespace bl {

namespace {

constexpr int kKv8Threads = 256;
// A chunk's values in LDS: the 64 positions of a dim, 80 bytes on from the next dim's, its four pieces of 16 moved about by the dim.  Sixteen
// lanes with a word of every fourth dim then meet sixteen banks (of four positions beside each other: all 64), and a piece stays whole.
constexpr int kValuePitch = 64 + 16;
__device__ __forceinline__ int value_piece(int dim, int piece) { return dim * kValuePitch + (piece ^ (dim >> 4 & 3)) * 16; }
__device__ __forceinline__ int value_word(int dim, int quad) { return value_piece(dim, quad >> 2) + (quad & 3) * 4; }   // positions 4 quad ..

struct WriteArgs {
    Kv8           cache;
    const void*   x[2];        // keys, values
    const float2* rope;        // may be null
    uint32_t*     clear;       // words that the launch sets to zero, for a launch behind it
    int64_t       clear_count;
    int64_t       ld;
    int32_t       n_heads, head_dim, size, pos0, M;
};

template <bool BF16, int V> struct RowVec;
template <> struct RowVec<false, 4> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct RowVec<false, 2> { typedef float type __attribute__((ext_vector_type(2), aligned(4))); };
template <> struct RowVec<true, 4> { typedef uint16_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct RowVec<true, 2> { typedef uint16_t type __attribute__((ext_vector_type(2), aligned(2))); };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// L lanes share a row, each with V elements of the head's lower half and their partners in the upper half (V divides half the head
// size, V L reaches it), of at least four rows in order: a dim's codes of four positions are a word.  All rows of a thread are requested before
// the first is used.
template <int L> constexpr int kWriteThreads = 16 * L < kKv8Threads ? 16 * L : kKv8Threads;

template <bool BF16, int V, int L>
__global__ __launch_bounds__(kWriteThreads<L>) void kv8_write_kernel(const WriteArgs p) {
    typedef typename RowVec<BF16, V>::type vec_t;
    constexpr int kThreads = kWriteThreads<L>, kTurns = kKv8Chunk / (kThreads / L);
    static_assert(kTurns % 4 == 0, "rows in fours");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int tid = threadIdx.x, l = tid % L, d = p.head_dim, half = d >> 1, size = p.size;
    const int head = blockIdx.y, chunk = p.pos0 / kKv8Chunk + (int)blockIdx.x, first = chunk * kKv8Chunk;
    const bool value = blockIdx.z != 0;
    const int lo = max(p.pos0, first), hi = min(p.pos0 + p.M, first + kKv8Chunk);   // rows of this workgroup
    if (p.clear) {
        const int64_t wgs = (int64_t)gridDim.x * gridDim.y * gridDim.z;
        for (int64_t i = ((int64_t)(blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x) * kThreads + tid; i < p.clear_count; i += wgs * kThreads)
            p.clear[i] = 0;
    }
    const int at = l * V, r0 = tid / L * kTurns;
    const bool mine = at < half;
    vec_t a[kTurns], b[kTurns];
    typedef float pair_t __attribute__((ext_vector_type(2 * V), aligned(8)));   // V pairs (cosine, sine)
    pair_t cs[kTurns];
    const bool rotate = !value && p.rope != nullptr;   // uniform
    const auto* x = static_cast<const typename std::conditional<BF16, uint16_t, float>::type*>(p.x[value]);
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int row = min(max(first + r0 + t, lo), hi - 1), e = mine ? at : 0;   // (any row of the call where there is none)
        const auto* src = x + (int64_t)(row - p.pos0) * p.ld + head * d + e;
        a[t] = *reinterpret_cast<const vec_t*>(src);
        b[t] = *reinterpret_cast<const vec_t*>(src + half);
        if (rotate) cs[t] = *reinterpret_cast<const pair_t*>(p.rope + (int64_t)row * half + e);
    }
#pragma unroll
    for (int t4 = 0; t4 < kTurns; t4 += 4) {
        uint32_t words[2][V] = {};   // of four positions
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = t4 + j, r = r0 + t, row = first + r;
            float u[V], w[V], amax = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                u[i] = widen(a[t][i]);
                w[i] = widen(b[t][i]);
                if (rotate) {   // each operation rounded on its own (the library is compiled without contraction)
                    const float c = cs[t][2 * i], s = cs[t][2 * i + 1], f = u[i], g = w[i];
                    u[i] = f * c - g * s;
                    w[i] = f * s + g * c;
                }
                if (mine) amax = MaxBitsOp()(amax, MaxBitsOp()(fabsf(u[i]), fabsf(w[i])));
            }
            amax = over_lanes<L>(amax, MaxBitsOp());
            if (!kv8_finite(amax)) {
#pragma unroll
                for (int i = 0; i < V; ++i) u[i] = w[i] = 0.0f;
            }
            float inv, scale;
            kv8_scales(amax, inv, scale);
            if (l == 0 && row >= lo && row < hi) (value ? p.cache.v_scale : p.cache.k_scale)[head * p.cache.head_scales + row] = scale;
            uint32_t row_u = 0, row_w = 0;   // a key row's bytes side by side
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t cu = (uint8_t)kv8_code(u[i], inv), cw = (uint8_t)kv8_code(w[i], inv);
                row_u |= cu << 8 * i;
                row_w |= cw << 8 * i;
                words[0][i] |= cu << 8 * j;
                words[1][i] |= cw << 8 * j;
            }
            if (!value && mine) {
                typedef typename std::conditional<V == 4, uint32_t, uint16_t>::type part_t;
                uint8_t* to = lds + kv8_key_row(r) * (size + 16) + at;
                *reinterpret_cast<part_t*>(to) = (part_t)row_u;
                *reinterpret_cast<part_t*>(to + half) = (part_t)row_w;   // (V divides half the head size)
            }
        }
        if (value && mine) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                *reinterpret_cast<uint32_t*>(lds + value_word(at + i, (r0 + t4) >> 2)) = words[0][i];
                *reinterpret_cast<uint32_t*>(lds + value_word(half + at + i, (r0 + t4) >> 2)) = words[1][i];
            }
        }
    }
    __syncthreads();
    int8_t* dst = (value ? p.cache.v : p.cache.k) + head * p.cache.head_bytes + (int64_t)chunk * kKv8Chunk * size;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    for (int piece = tid; piece < 4 * size; piece += kThreads) {   // of 16 bytes
        if (value) {
            const int e = piece >> 2, r = (piece & 3) * 16, from = value_piece(e, piece & 3);
            const u32x4 codes = e < d ? *reinterpret_cast<const u32x4*>(lds + from) : u32x4{0, 0, 0, 0};
            if (first + r >= lo && first + r + 16 <= hi) *reinterpret_cast<u32x4*>(dst + e * 64 + r) = codes;
            else
                for (int i = 0; i < 16; ++i)
                    if (first + r + i >= lo && first + r + i < hi) dst[e * 64 + r + i] = (int8_t)(e < d ? lds[from + i] : 0);
        } else {
            const int off = piece * 16, block = off >> 12, width = min(64, size - 64 * block), in = off & 4095;
            const int row = in / width, e = 64 * block + in % width, r = 4 * (row & 15) + (row >> 4);
            if (first + r < lo || first + r >= hi) continue;
            u32x4 codes = *reinterpret_cast<const u32x4*>(lds + row * (size + 16) + e);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (e + 4 * i >= d) codes[i] = 0;   // the padding (a multiple of four dims)
            *reinterpret_cast<u32x4*>(dst + off) = codes;
        }
    }
}

struct ReadArgs {
    Kv8     cache;
    void*   out[2];
    int64_t ld;
    int32_t head_dim, size, pos0, M;
    int32_t first;   // of blockIdx.z: 0 keys, 1 values
};

template <bool BF16>
__global__ __launch_bounds__(kKv8Threads) void kv8_read_kernel(const ReadArgs p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const int tid = threadIdx.x, d = p.head_dim, size = p.size;
    const int head = blockIdx.y, chunk = p.pos0 / kKv8Chunk + (int)blockIdx.x, first = chunk * kKv8Chunk;
    const bool value = p.first + (int)blockIdx.z != 0;
    const int lo = max(p.pos0, first), hi = min(p.pos0 + p.M, first + kKv8Chunk);
    const int8_t* src = (value ? p.cache.v : p.cache.k) + head * p.cache.head_bytes + (int64_t)chunk * kKv8Chunk * size;
    const float* scales = (value ? p.cache.v_scale : p.cache.k_scale) + head * p.cache.head_scales;
    for (int piece = tid; piece < 4 * size; piece += kKv8Threads) {
        const u32x4 codes = *reinterpret_cast<const u32x4*>(src + piece * 16);
        const int off = piece * 16;
        if (value) {
            *reinterpret_cast<u32x4*>(lds + value_piece(piece >> 2, piece & 3)) = codes;
        } else {
            const int block = off >> 12, width = min(64, size - 64 * block), in = off & 4095;
            *reinterpret_cast<u32x4*>(lds + in / width * (size + 16) + 64 * block + in % width) = codes;
        }
    }
    __syncthreads();
    // four positions by four dims at a time: words of the keys are rows', of the values dims'
    const int quads = d >> 2, group0 = (lo - first) >> 2, groups = ((hi - 1 - first) >> 2) - group0 + 1;
    for (int i = tid; i < groups * quads; i += kKv8Threads) {
        const int group = group0 + i / quads, e = 4 * (i % quads);
        uint32_t words[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            words[j] = *reinterpret_cast<const uint32_t*>(lds + (value ? value_word(e + j, group) : kv8_key_row(4 * group + j) * (size + 16) + e));
        if (value) {
            const uint32_t a = __builtin_amdgcn_perm(words[1], words[0], 0x05010400u), b = __builtin_amdgcn_perm(words[3], words[2], 0x05010400u);
            const uint32_t c = __builtin_amdgcn_perm(words[1], words[0], 0x07030602u), f = __builtin_amdgcn_perm(words[3], words[2], 0x07030602u);
            words[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
            words[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            words[2] = __builtin_amdgcn_perm(f, c, 0x05040100u);
            words[3] = __builtin_amdgcn_perm(f, c, 0x07060302u);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = first + 4 * group + j;
            if (row < lo || row >= hi) continue;
            const float scale = scales[row];
            float x[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) x[n] = (float)(int8_t)(words[j] >> 8 * n) * scale;
            const int64_t at = (int64_t)(row - p.pos0) * p.ld + head * d + e;
            if constexpr (BF16) {
                typedef __bf16 b4 __attribute__((ext_vector_type(4), aligned(2)));
                typedef float f4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<b4*>(static_cast<__bf16*>(p.out[value]) + at) = __builtin_convertvector((f4{x[0], x[1], x[2], x[3]}), b4);
            } else {
                typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
                *reinterpret_cast<f4*>(static_cast<float*>(p.out[value]) + at) = f4{x[0], x[1], x[2], x[3]};
            }
        }
    }
}

int lds_bytes(int size) { return max(64 * (size + 16), size * kValuePitch); }

dim3 chunk_grid(int pos0, int M, int n_heads, int sides) {
    const int chunks = (pos0 + M - 1) / kKv8Chunk - pos0 / kKv8Chunk + 1;
    return dim3((unsigned)chunks, (unsigned)n_heads, (unsigned)sides);
}

template <bool BF16, int V, int L>
hipError_t launch_write(const WriteArgs& p, hipStream_t s) {
    kv8_write_kernel<BF16, V, L><<<chunk_grid(p.pos0, p.M, p.n_heads, 2), dim3(kWriteThreads<L>), lds_bytes(p.size), s>>>(p);
    return hipGetLastError();
}

template <bool BF16>
hipError_t launch_write_form(const WriteArgs& p, hipStream_t s) {
    const int half = p.head_dim / 2;
    if (half % 4 == 0) {   // the widest rows: 128 elements in fours
        if (half <= 32) return launch_write<BF16, 4, 8>(p, s);
        if (half <= 64) return launch_write<BF16, 4, 16>(p, s);
        return launch_write<BF16, 4, 32>(p, s);
    }
    if (half <= 32) return launch_write<BF16, 2, 16>(p, s);
    if (half <= 64) return launch_write<BF16, 2, 32>(p, s);
    return launch_write<BF16, 2, 64>(p, s);
}

}  // namespace

hipError_t launch_kv8_write(const ::bl_kv8_write_args& a, uint32_t* clear, int64_t clear_count, hipStream_t s) {
    WriteArgs p;
    p.cache = kv8_of(*a.cache, a.sequence);
    p.x[0] = a.k_dev; p.x[1] = a.v_dev;
    p.rope = reinterpret_cast<const float2*>(a.rope_table_dev);
    p.clear = clear; p.clear_count = clear_count;
    p.ld = a.ld;
    p.n_heads = a.cache->n_heads; p.head_dim = a.cache->head_dim; p.size = kv8_size(p.head_dim); p.pos0 = a.pos0; p.M = a.M;
    return a.dt == BL_BF16 ? launch_write_form<true>(p, s) : launch_write_form<false>(p, s);
}

hipError_t launch_kv8_read(const ::bl_kv8_read_args& a, hipStream_t s) {
    ReadArgs p;
    p.cache = kv8_of(*a.cache, a.sequence);
    p.out[0] = a.k_out_dev; p.out[1] = a.v_out_dev;
    p.ld = a.ld;
    p.head_dim = a.cache->head_dim; p.size = kv8_size(p.head_dim); p.pos0 = a.pos0; p.M = a.M;
    p.first = a.k_out_dev ? 0 : 1;
    const dim3 grid = chunk_grid(a.pos0, a.M, a.cache->n_heads, a.k_out_dev && a.v_out_dev ? 2 : 1);
    if (a.dt == BL_BF16) kv8_read_kernel<true><<<grid, dim3(kKv8Threads), lds_bytes(p.size), s>>>(p);
    else kv8_read_kernel<false><<<grid, dim3(kKv8Threads), lds_bytes(p.size), s>>>(p);
    return hipGetLastError();
}

}  // namespace bl
