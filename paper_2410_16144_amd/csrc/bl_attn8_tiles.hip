// The kernel of the tiles form: the shared part of a launch in tiles of 32 rows, sequences' own parts beside it in rows.
#include "bl_attn8_rows.hpp"
#include "bl_attn8_tiles.hpp"

namespace bl {

namespace {

constexpr int max_of(int a, int b) { return a > b ? a : b; }

// SETS: waves of a tile.  OWN: whether there is an own part (a prompt has none; without it the kernel is smaller).  FOLD: a prompt's blocks by twos
// (a form of its own: the loop costs seven registers more than there are).
template <int D32, int SETS, bool OWN, bool FOLD>
__global__ __launch_bounds__(kTiles8Threads, D32 <= 4 ? 2 : 1) void attn8_tiles_kernel(const Attn8Args p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ Attn8Rows rows;
    Attn8Walk walk;
    const int wg = blockIdx.x;   // uniform, like the walk
    if constexpr (!OWN) {
        __shared__ Tiles8Shared shared;
        for (int again = 0; again <= (FOLD ? 1 : 0); ++again) {
            if (again) __syncthreads();   // (everybody has what the first block left in LDS)
            if (attn8_shared_walk<true>(p, wg, kTiles8Rows * kTiles8Waves / SETS, walk, again)) tiles8_walk<D32, SETS>(p, walk, lds, shared, rows);
        }
    } else if (wg < p.shared_wgs) {
        __shared__ Tiles8Shared shared;
        if (attn8_shared_walk(p, wg, kTiles8Rows * kTiles8Waves / SETS, walk)) tiles8_walk<D32, SETS>(p, walk, lds, shared, rows);
    } else {
        // By ordinary loads whatever their size.  32 heads of 128 behind 500 positions, ordinary and streaming, us: 16 sequences of 100 positions 15.7 and 16.5,
        // 40 of 300 25.8 and 29.3; 16 of 2000 44.5 and 40.7, 60 of 1500 96.0 and 88.8.
        __shared__ Rows8Shared shared;
        if (attn8_own_walk(p, wg - p.shared_wgs, 4, walk)) rows8_walk<(D32 + 1) / 2, 1, kTiles8Waves, false>(p, walk, lds, shared, rows);
    }
}

template <int D32, int SETS, bool OWN, bool FOLD = false>
hipError_t launch_form(const Attn8Args& p, int wgs, hipStream_t s) {
    constexpr int kBytes = OWN ? max_of(Tiles8Lds<D32>::kBytes, Rows8Lds<(D32 + 1) / 2, 1, kTiles8Waves>::kBytes) : Tiles8Lds<D32>::kBytes;
    static_assert(kBytes + 4096 <= 160 * 1024, "fits a compute unit");
    static LdsCeiling ceiling;   // per instantiation, i.e. per kernel
    const hipError_t e = ceiling.ensure(reinterpret_cast<const void*>(&attn8_tiles_kernel<D32, SETS, OWN, FOLD>), kBytes);
    if (e != hipSuccess) return e;
    attn8_tiles_kernel<D32, SETS, OWN, FOLD><<<dim3((unsigned)wgs), dim3(kTiles8Threads), kBytes, s>>>(p);
    return hipGetLastError();
}

template <int D32>
hipError_t launch_size(const Attn8Args& p, int wgs, hipStream_t s) {
    if (wgs > p.shared_wgs) return launch_form<D32, 4, true>(p, wgs, s);
    if (p.folded) return p.shared_set == 5 ? launch_form<D32, 1, false, true>(p, wgs, s) : launch_form<D32, 2, false, true>(p, wgs, s);
    return p.shared_set == 6 ? launch_form<D32, 2, false>(p, wgs, s) : launch_form<D32, 4, false>(p, wgs, s);
}

// What the workgroups of a row left behind a launch of tiles: one workgroup per (row, key head), the row's figures shared out among its waves.
// A launch of its own, because the last workgroup of 32 rows reads their figures a trip to memory at a time: 77 tokens behind 1001, 32 heads of 120,
// five workgroups per row 31.5 us with tickets, of which the reading 10, 25.7 so; one token's rows are few, and meet without (attn8_finish).
__global__ __launch_bounds__(kTiles8Threads) void attn8_merge_kernel(const Attn8Args p) {
    __shared__ float2 s_sum[kTiles8Waves][kWave];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x, head = blockIdx.y, token = divided(row, p.by_group);
    const int pos = attn8_position(p, token);
    if (!attn8_takes_part(p, pos)) return;                 // uniform
    int keys = p.shared_len;
    if (p.prompt) {                                        // of the row's block
        const int last = min((row / kTiles8Rows + 1) * kTiles8Rows, p.rows) - 1;
        keys = p.pos0 + divided(last, p.by_group) + 1;
    }
    const int walked = min(p.shared_splits, attn8_sets(keys, p.shared_set));
    const int target = walked + (p.prompt ? 0 : min(p.own_splits, attn8_sets(pos - p.shared_len + 1, p.own_set)));
    if (target == 1) return;                               // written already
    const int half = p.head_dim >> 1, stride = half + 1, slots = p.shared_splits + p.own_splits;
    const float2* figures = p.figures + ((int64_t)head * p.rows + row) * slots * stride;
    const auto at = [&](int f) { return figures + (int64_t)(f < walked ? f : p.shared_splits + f - walked) * stride; };
    float2 ml[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) ml[h] = lane + 64 * h < target ? *at(lane + 64 * h) : make_float2(-INFINITY, 0.0f);
    const float m = over_lanes<64>(fmaxf(ml[0].x, ml[1].x), MaxOp());
    const float f0 = __builtin_amdgcn_exp2f(ml[0].x - m), f1 = __builtin_amdgcn_exp2f(ml[1].x - m);
    const float l = over_lanes<64>(f0 * ml[0].y + f1 * ml[1].y, AddOp());
    for (int e0 = 0; e0 < half; e0 += kWave) {             // (a second turn for head sizes above 128)
        const int e = min(e0 + lane, half - 1);
        float x = 0.0f, y = 0.0f;
        for (int f = wave; f < target; f += kTiles8Waves) {
            const float w = __shfl(f < 64 ? f0 : f1, f & 63);
            const float2 a = at(f)[1 + e];
            x += w * a.x;
            y += w * a.y;
        }
        s_sum[wave][lane] = make_float2(x, y);
        __syncthreads();
        if (wave == 0 && e0 + lane < half) {
            x = y = 0.0f;
#pragma unroll
            for (int w = 0; w < kTiles8Waves; ++w) {
                x += s_sum[w][lane].x;
                y += s_sum[w][lane].y;
            }
            *reinterpret_cast<float2*>(p.out + attn8_row_at(p, head, row) + 2 * e) = make_float2(x / l, y / l);
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_attn8_merge(const Attn8Args& p, hipStream_t s) {
    attn8_merge_kernel<<<dim3((unsigned)p.rows, (unsigned)p.n_heads), dim3(kTiles8Threads), 0, s>>>(p);
    return hipGetLastError();
}

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
