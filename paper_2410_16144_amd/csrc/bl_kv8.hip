// bl_kv8_write and bl_kv8_read: rows into the 8-bit cache and out of it (layout: bl_kv8.hpp).
//
// One workgroup per (chunk of 64 positions, key head, keys or values).  A write is a stream of projections in and a quarter of their bytes
// (half, from bf16) out: every row's largest value stays in the registers of the lanes that hold the row -- one read -- and the
// codes are put into the cache's order in LDS, since a value's neighbours in memory are the same dim's of other positions.  A chunk that the
// call covers in part is written row by row (keys) and byte by byte (values): the bytes between belong to other positions.
#include "bl_kv8.hpp"
#include "bl_lanes.hpp"

namespace bl {

namespace {

constexpr int kKv8Threads = 256;
constexpr int kValuePitch = 64 + 16;   // bytes of a dim's positions in LDS: the dims of a write spread over the banks

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
// size, V L reaches it).  All rows of a thread are requested before the first is used.
template <bool BF16, int V, int L>
__global__ __launch_bounds__(kKv8Threads) void kv8_write_kernel(const WriteArgs p) {
    typedef typename RowVec<BF16, V>::type vec_t;
    constexpr int kRows = kKv8Threads / L, kTurns = kKv8Chunk / kRows;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int tid = threadIdx.x, l = tid % L, d = p.head_dim, half = d >> 1, size = p.size;
    const int head = blockIdx.y, chunk = p.pos0 / kKv8Chunk + (int)blockIdx.x, first = chunk * kKv8Chunk;
    const bool value = blockIdx.z != 0;
    const int lo = max(p.pos0, first), hi = min(p.pos0 + p.M, first + kKv8Chunk);   // rows of this workgroup
    if (p.clear) {
        const int64_t wgs = (int64_t)gridDim.x * gridDim.y * gridDim.z;
        for (int64_t i = ((int64_t)(blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x) * kKv8Threads + tid; i < p.clear_count; i += wgs * kKv8Threads)
            p.clear[i] = 0;
    }
    const int at = l * V;
    const bool mine = at < half;
    vec_t a[kTurns], b[kTurns];
    typedef float pair_t __attribute__((ext_vector_type(2 * V), aligned(8)));   // V pairs (cosine, sine)
    pair_t cs[kTurns];
    const bool rotate = !value && p.rope != nullptr;   // uniform
    const auto* x = static_cast<const typename std::conditional<BF16, uint16_t, float>::type*>(p.x[value]);
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int row = min(max(first + tid / L + t * kRows, lo), hi - 1), e = mine ? at : 0;   // (any row of the call where there is none)
        const auto* src = x + (int64_t)(row - p.pos0) * p.ld + head * d + e;
        a[t] = *reinterpret_cast<const vec_t*>(src);
        b[t] = *reinterpret_cast<const vec_t*>(src + half);
        if (rotate) cs[t] = *reinterpret_cast<const pair_t*>(p.rope + (int64_t)row * half + e);
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int row = first + tid / L + t * kRows, r = row - first;
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
            if (mine) amax = fmaxf(amax, fmaxf(fabsf(u[i]), fabsf(w[i])));
        }
#pragma unroll
        for (int o = 1; o < L; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
        float inv, scale;
        kv8_scales(amax, inv, scale);
        if (row >= lo && row < hi) {
            if (l == 0) (value ? p.cache.v_scale : p.cache.k_scale)[head * p.cache.head_scales + row] = scale;
            if (mine) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const uint8_t cu = (uint8_t)kv8_code(u[i], inv), cw = (uint8_t)kv8_code(w[i], inv);
                    if (value) {
                        lds[(at + i) * kValuePitch + r] = cu;
                        lds[(half + at + i) * kValuePitch + r] = cw;
                    } else {
                        const int base = kv8_key_row(r) * (size + 16) + at + i;
                        lds[base] = cu;
                        lds[base + half] = cw;
                    }
                }
            }
        }
    }
    __syncthreads();
    int8_t* dst = (value ? p.cache.v : p.cache.k) + head * p.cache.head_bytes + (int64_t)chunk * kKv8Chunk * size;
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    for (int piece = tid; piece < 4 * size; piece += kKv8Threads) {   // of 16 bytes
        if (value) {
            const int e = piece >> 2, r = (piece & 3) * 16;
            const u32x4 codes = e < d ? *reinterpret_cast<const u32x4*>(lds + e * kValuePitch + r) : u32x4{0, 0, 0, 0};
            if (first + r >= lo && first + r + 16 <= hi) *reinterpret_cast<u32x4*>(dst + e * 64 + r) = codes;
            else
                for (int i = 0; i < 16; ++i)
                    if (first + r + i >= lo && first + r + i < hi) dst[e * 64 + r + i] = (int8_t)(e < d ? lds[e * kValuePitch + r + i] : 0);
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
            *reinterpret_cast<u32x4*>(lds + (piece >> 2) * kValuePitch + (piece & 3) * 16) = codes;
        } else {
            const int block = off >> 12, width = min(64, size - 64 * block), in = off & 4095;
            *reinterpret_cast<u32x4*>(lds + in / width * (size + 16) + 64 * block + in % width) = codes;
        }
    }
    __syncthreads();
    const int quads = d >> 2;
    for (int i = tid; i < (hi - lo) * quads; i += kKv8Threads) {
        const int row = lo + i / quads, e = 4 * (i % quads), r = row - first;
        const float scale = scales[row];
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int8_t code = (int8_t)(value ? lds[(e + j) * kValuePitch + r] : lds[kv8_key_row(r) * (size + 16) + e + j]);
            x[j] = (float)code * scale;
        }
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

int lds_bytes(int size) { return max(64 * (size + 16), size * kValuePitch); }

dim3 chunk_grid(int pos0, int M, int n_heads, int sides) {
    const int chunks = (pos0 + M - 1) / kKv8Chunk - pos0 / kKv8Chunk + 1;
    return dim3((unsigned)chunks, (unsigned)n_heads, (unsigned)sides);
}

template <bool BF16, int V, int L>
hipError_t launch_write(const WriteArgs& p, hipStream_t s) {
    kv8_write_kernel<BF16, V, L><<<chunk_grid(p.pos0, p.M, p.n_heads, 2), dim3(kKv8Threads), lds_bytes(p.size), s>>>(p);
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
