// The 8-bit key/value cache: where a row's codes lie, and what its kernels share.
//
// Per sequence and key head the positions are cut into chunks of 64, each one contiguous piece of 64 * S bytes of keys and as many of
// values (S: the head size rounded up to 16, the padding zero), in the order in which the int8 matrix instructions want their operands,
// so that every operand of the attention kernels is ONE 16-byte load per lane from consecutive memory, and nothing passes through LDS:
//   keys    [block of up to 64 dims][row][dims], the row of position p being 16 (p % 4) + p % 64 / 4.  The 16 rows of an operand
//           (v_mfma_i32_16x16x64_i8) are positions 4 j + u, j = 0 .. 15: a lane then holds the scores of the four positions 4 j .. 4 j + 3,
//           whose weights are one 32-bit word of the next product's operand;
//   values  [dim][64 positions]: a dim's positions side by side, since the second product contracts over them.
#pragma once
#include <type_traits>

#include "bl_internal.hpp"

namespace bl {

constexpr int kKv8Chunk = BL_KV8_CHUNK;
static_assert(kKv8Chunk == kWave, "one chunk's positions are a wave's lanes");

__host__ __device__ constexpr int kv8_size(int head_dim) { return (head_dim + 15) & ~15; }   // bytes per row of codes
__host__ __device__ constexpr int kv8_chunks(int positions) { return (positions + kKv8Chunk - 1) / kKv8Chunk; }
__host__ __device__ constexpr int kv8_key_row(int p) { return 16 * (p & 3) + ((p & 63) >> 2); }
// offsets inside a chunk of codes
__host__ __device__ constexpr int kv8_key_at(int p, int dim, int size) {
    const int block = dim >> 6, left = size - 64 * block, width = left < 64 ? left : 64;
    return block * 4096 + kv8_key_row(p) * width + (dim & 63);
}
__host__ __device__ constexpr int kv8_value_at(int p, int dim) { return dim * 64 + (p & 63); }

// One sequence's cache of one layer as the kernels see it.
struct Kv8 {
    int8_t* k;
    int8_t* v;
    float*  k_scale;
    float*  v_scale;
    int64_t head_bytes;     // codes of a key head
    int64_t head_scales;    // scales of a key head
};

inline Kv8 kv8_of(const ::bl_kv8_cache& c, int64_t sequence) {
    Kv8 r;
    const int64_t chunks = kv8_chunks(c.max_pos);
    r.head_bytes = chunks * kKv8Chunk * kv8_size(c.head_dim);
    r.head_scales = chunks * kKv8Chunk;
    r.k = c.k_codes_dev + sequence * c.n_heads * r.head_bytes;
    r.v = c.v_codes_dev + sequence * c.n_heads * r.head_bytes;
    r.k_scale = c.k_scale_dev + sequence * c.n_heads * r.head_scales;
    r.v_scale = c.v_scale_dev + sequence * c.n_heads * r.head_scales;
    return r;
}

// The quantizer's scalars of a row (bl_quant_act's: one division each; a row whose inv is infinite is a row of zeros).  amax with MaxBitsOp:
// of a row with a NaN or an infinity it is not finite; the row is one of zeros then, too, and its scale a NaN, so that whoever reads it sees that.
__device__ __forceinline__ bool kv8_finite(float amax) { return amax < INFINITY; }
__device__ __forceinline__ void kv8_scales(float amax, float& inv, float& scale) {
    inv = 127.0f / amax;
    scale = amax / 127.0f;
    if (!(inv < INFINITY)) inv = scale = 0.0f;
    if (!kv8_finite(amax)) {
        inv = 0.0f;
        scale = __builtin_nanf("");
    }
}
__device__ __forceinline__ int kv8_code(float x, float inv) { return (int)fminf(fmaxf(rintf(x * inv), -128.0f), 127.0f); }

}  // namespace bl
