// The kernel of the tiles form: the shared part of a launch in tiles of 32 rows, sequences' own parts beside it in rows.
#include "bl_attn8_rows.hpp"
#include "bl_attn8_tiles.hpp"

namespace bl {

namespace {

constexpr int max_of(int a, int b) { return a > b ? a : b; }

// OWN: whether there is an own part (a prompt has none; without it the kernel is smaller).
template <int D32, bool OWN>
__global__ __launch_bounds__(kAttn8Threads, D32 <= 4 ? 2 : 1) void attn8_tiles_kernel(const Attn8Args p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ Attn8Rows rows;
    Attn8Walk walk;
    const int wg = blockIdx.x;   // uniform, like the walk
    if (!OWN || wg < p.shared_wgs) {
        __shared__ Tiles8Shared shared;
        if (attn8_shared_walk(p, wg, kTiles8Rows, walk)) tiles8_walk<D32>(p, walk, lds, shared, rows);
    } else {
        __shared__ Rows8Shared shared;
        if (attn8_own_walk(p, wg - p.shared_wgs, 4, walk)) rows8_walk<(D32 + 1) / 2, 1>(p, walk, lds, shared, rows);
    }
}

template <int D32, bool OWN>
hipError_t launch_form(const Attn8Args& p, int wgs, hipStream_t s) {
    constexpr int kBytes = OWN ? max_of(Tiles8Lds<D32>::kBytes, Rows8Lds<(D32 + 1) / 2, 1>::kBytes) : Tiles8Lds<D32>::kBytes;
    static_assert(kBytes + 4096 <= 160 * 1024, "fits a compute unit");
    static LdsCeiling ceiling;   // per instantiation, i.e. per kernel
    const hipError_t e = ceiling.ensure(reinterpret_cast<const void*>(&attn8_tiles_kernel<D32, OWN>), kBytes);
    if (e != hipSuccess) return e;
    attn8_tiles_kernel<D32, OWN><<<dim3((unsigned)wgs), dim3(kAttn8Threads), kBytes, s>>>(p);
    return hipGetLastError();
}

template <int D32>
hipError_t launch_size(const Attn8Args& p, int wgs, hipStream_t s) {
    return wgs > p.shared_wgs ? launch_form<D32, true>(p, wgs, s) : launch_form<D32, false>(p, wgs, s);
}

}  // namespace

hipError_t launch_attn8_tiles(const Attn8Args& p, int wgs, hipStream_t s) {
    static_assert(BL_ATTN_MAX_HEAD_DIM == 256, "head sizes up to eight 32s");
    switch ((p.head_dim + 31) / 32) {
        case 1: return launch_size<1>(p, wgs, s);
        case 2: return launch_size<2>(p, wgs, s);
        case 3: return launch_size<3>(p, wgs, s);
        case 4: return launch_size<4>(p, wgs, s);
        case 5: return launch_size<5>(p, wgs, s);
        case 6: return launch_size<6>(p, wgs, s);
        case 7: return launch_size<7>(p, wgs, s);
        case 8: return launch_size<8>(p, wgs, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace bl
