// Reductions over neighbouring lanes of a wavefront, shared by the attention kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bl {

// Sum or maximum over groups of L neighbouring lanes (8 to 64), on the vector ALU's lane moves instead of a trip through LDS per
// step (ds_bpermute): lane ^ 1 and ^ 2 by quad permutation, the other half of eight and of sixteen lanes by their mirror images -- whose
// lanes all hold their quad's or half's result by then -- and the 16- and 32-lane blocks by the swaps of two registers.  Every step
// adds the two halves' figures (in either order the same bits), so every lane gets the same result.
#define BL_LANES(v, ctrl) __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), (ctrl), 0xf, 0xf, false))
template <int OFF, typename Op>
__device__ __forceinline__ float over_blocks(float v, Op op) {   // lane and lane ^ OFF
    static_assert(OFF == 16 || OFF == 32, "the two swaps");
    const uint32_t u = __float_as_uint(v);
    if constexpr (OFF == 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
    } else {
        const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
    }
}
template <int L, typename Op>
__device__ __forceinline__ float over_lanes(float v, Op op) {
    static_assert(L == 8 || L == 16 || L == 32 || L == 64, "half a row of sixteen lanes, or whole ones");
    v = op(v, BL_LANES(v, 0xb1));    // quad_perm [1, 0, 3, 2]
    v = op(v, BL_LANES(v, 0x4e));    // quad_perm [2, 3, 0, 1]
    v = op(v, BL_LANES(v, 0x141));   // row_half_mirror
    if constexpr (L >= 16) v = op(v, BL_LANES(v, 0x140));   // row_mirror
    if constexpr (L >= 32) v = over_blocks<16>(v, op);
    if constexpr (L >= 64) v = over_blocks<32>(v, op);
    return v;
}
#undef BL_LANES
struct AddOp { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
// Of numbers without a sign, a NaN above all others (their bits' order).
struct MaxBitsOp {
    __device__ __forceinline__ float operator()(float a, float b) const { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }
};
struct MinOp { __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); } };
struct MaxOp { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

}  // namespace bl
