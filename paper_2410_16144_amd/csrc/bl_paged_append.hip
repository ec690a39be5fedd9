// bl_paged_append: queries and keys normed per head and rotated, keys and values into their pages.
//
// A stream: every projection is read once and written once, bound by memory (and by its launch for a single token).  Eight or sixteen lanes have one head's
// vector of one row, both elements of every rotated pair in one lane, so that the sum of squares is a few lane exchanges and nothing passes
// through LDS; a wave has some heads of one row, so that the row's sequence and page are found once per wave, by scalar loads, while
// the projections are on their way.
#include "bl_paged.hpp"

namespace bl {

namespace {

struct AppendArgs {
    Paged        c;
    const void*  x[3];         // queries, keys, values
    void*        q_out;
    const float* gamma[2];     // of queries and keys; may be null
    const float2* rope;        // may be null
    int64_t      ld[3];
    float        eps;
    int32_t      n_q_heads;
};

template <bool BF16, int V> struct AppendVec;
template <> struct AppendVec<true, 8> { typedef uint16_t type __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct AppendVec<false, 8> { typedef float type __attribute__((ext_vector_type(8), aligned(4))); };
template <> struct AppendVec<false, 4> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct AppendVec<false, 2> { typedef float type __attribute__((ext_vector_type(2), aligned(4))); };
template <> struct AppendVec<true, 4> { typedef uint16_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct AppendVec<true, 2> { typedef uint16_t type __attribute__((ext_vector_type(2), aligned(2))); };

__device__ __forceinline__ float widened(float x) { return x; }
__device__ __forceinline__ float widened(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// V elements, the address a multiple of V elements' size
template <bool BF16, int V>
__device__ __forceinline__ void append_store(void* to, int64_t at, const float (&x)[V]) {
    if constexpr (V == 8) {
        const float low[4] = {x[0], x[1], x[2], x[3]}, high[4] = {x[4], x[5], x[6], x[7]};
        if constexpr (BF16) {
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(to) + at) =
                u32x4{paged_bf16_pair(x[0], x[1]), paged_bf16_pair(x[2], x[3]), paged_bf16_pair(x[4], x[5]), paged_bf16_pair(x[6], x[7])};
        } else {
            append_store<BF16, 4>(to, at, low);
            append_store<BF16, 4>(to, at + 4, high);
        }
    } else if constexpr (BF16) {
        if constexpr (V == 4) *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(to) + at) = u32x2{paged_bf16_pair(x[0], x[1]), paged_bf16_pair(x[2], x[3])};
        else *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(to) + at) = paged_bf16_pair(x[0], x[1]);
    } else {
        if constexpr (V == 4) *reinterpret_cast<f32x4*>(static_cast<float*>(to) + at) = f32x4{x[0], x[1], x[2], x[3]};
        else *reinterpret_cast<f32x2*>(static_cast<float*>(to) + at) = f32x2{x[0], x[1]};
    }
}

// The sequence that row t belongs to; no rows if none has it.  (Uniform t.)  Where starts rise, as many end at t or before.  Starts that fall hide nobody's
// rows but their own: where that one does not have the row, everyone is asked (with up to 64 sequences nobody need be if all end at t or before).
__device__ __forceinline__ PagedSequence sequence_of(const Paged& c, int t, int lane, int& of) {
    const auto has = [&](const PagedSequence& s) { return t >= s.first && t < s.first + s.rows; };
    of = c.start ? 0 : t;
    if (!c.start || c.sequences == 1) return paged_sequence_uniform(c, of);
    const int each = (c.sequences + 63) >> 6;              // at most 16
    int b = 0;
    if (each > 1) b = each * __popcll(__ballot(c.start[min((lane + 1) * each, c.sequences)] <= t));
    const int i = b + lane;
    of = uniform(b + __popcll(__ballot((each == 1 || lane < each) && i < c.sequences && c.start[min(i, c.sequences - 1) + 1] <= t)));
    if (of < c.sequences) {
        const PagedSequence s = paged_sequence_uniform(c, of);
        if (has(s)) return s;
    } else if (each == 1) {
        return {0, 0, 0};
    }
#pragma unroll 1
    for (int from = 0; from < c.sequences; from += 256) {
        bool mine[4];                                      // (the loads of 256 travel together)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int n = from + 64 * u + lane, at = min(n, c.sequences - 1);
            const int first = c.start[at], end = c.start[at + 1];
            mine[u] = (n < c.sequences) & (t >= first) & (t < end);
        }
        if (!__any(mine[0] || mine[1] || mine[2] || mine[3])) continue;
#pragma unroll 1
        for (int n = from; n < min(from + 256, c.sequences); ++n) {
            const PagedSequence s = paged_sequence_uniform(c, n);
            if (has(s)) {
                of = n;
                return s;
            }
        }
    }
    return {0, 0, 0};
}

// L lanes have a head, NV times V elements and their partners each (V divides half the head size, NV V L reaches it).  bf16 by 16 bytes a lane: 2000 rows
// of 32 + 2 * 32 heads of 128 in 25.6 us (99 MB, 3.9 TB/s; a copy of as many bytes takes 20), by 8 bytes 30.7; two heads a lane instead of one 25.2 there
// and more where there are few rows.
template <bool IN16, bool OUT16, int L, int V, int NV>
__global__ __launch_bounds__(256) void paged_append_kernel(const AppendArgs p) {
    typedef typename AppendVec<IN16, V>::type vec_t;
    typedef typename std::conditional<IN16, uint16_t, float>::type in_t;
    const Paged& c = p.c;
    const int lane = threadIdx.x & 63, l = lane & (L - 1);
    constexpr int kHeads = 64 / L;                         // of a wave
    const int heads = p.n_q_heads + 2 * c.n_heads, units = (heads + kHeads - 1) / kHeads;   // of a row
    const int64_t unit = (int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6);
    const int t = (int)(unit / units);
    if (t >= c.rows) return;
    int head = kHeads * (int)(unit - (int64_t)t * units) + lane / L;
    const bool there = head < heads;
    const int kind = head < p.n_q_heads ? 0 : head < p.n_q_heads + c.n_heads ? 1 : 2;
    head = there ? head - (kind == 0 ? 0 : kind == 1 ? p.n_q_heads : p.n_q_heads + c.n_heads) : 0;
    const int d = c.head_dim, half = d >> 1;

    vec_t a[NV], b[NV];
    const in_t* src = static_cast<const in_t*>(p.x[kind]) + t * p.ld[kind] + (int64_t)head * d;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int e = (l + L * n) * V;
        if (e >= half) continue;
        a[n] = *reinterpret_cast<const vec_t*>(src + e);
        b[n] = *reinterpret_cast<const vec_t*>(src + half + e);
    }
    int of;
    const PagedSequence s = sequence_of(c, t, lane, of);
    if (t < s.first || t >= s.first + s.rows) return;
    const int at = s.pos + t - s.first;
    const int page = uniform(scalar_word(c.table, (int64_t)of * c.table_width + (at >> c.page_shift)));

    float u[NV][V], w[NV][V], ss = 0.0f;
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool in = (l + L * n) * V < half;
            u[n][i] = in ? widened(a[n][i]) : 0.0f;
            w[n][i] = in ? widened(b[n][i]) : 0.0f;
            ss += u[n][i] * u[n][i] + w[n][i] * w[n][i];
        }
    if (kind < 2 && p.gamma[kind]) {
        ss = over_lanes<L>(ss, AddOp());
        const float r = 1.0f / sqrtf(ss / (float)d + p.eps);
        typedef float g_t __attribute__((ext_vector_type(V), aligned(4)));
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int e = (l + L * n) * V;
            if (e >= half) continue;
            const g_t ga = *reinterpret_cast<const g_t*>(p.gamma[kind] + e), gb = *reinterpret_cast<const g_t*>(p.gamma[kind] + half + e);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                u[n][i] = u[n][i] * ga[i] * r;
                w[n][i] = w[n][i] * gb[i] * r;
            }
        }
    }
    if (kind < 2 && p.rope) {
        typedef float pair_t __attribute__((ext_vector_type(2 * V), aligned(8)));   // V pairs (cosine, sine)
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int e = (l + L * n) * V;
            if (e >= half) continue;
            const pair_t cs = *reinterpret_cast<const pair_t*>(p.rope + (int64_t)at * half + e);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float f = u[n][i], g = w[n][i];
                u[n][i] = f * cs[2 * i] - g * cs[2 * i + 1];
                w[n][i] = f * cs[2 * i + 1] + g * cs[2 * i];
            }
        }
    }
    if (!there) return;
    if (kind == 0) {
        const int64_t to = ((int64_t)t * p.n_q_heads + head) * d;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int e = (l + L * n) * V;
            if (e >= half) continue;
            append_store<OUT16, V>(p.q_out, to + e, u[n]);
            append_store<OUT16, V>(p.q_out, to + half + e, w[n]);
        }
    } else if ((uint32_t)page < (uint32_t)c.pages) {       // (a page that is not there: nobody's)
        const int width = paged_width(d), slot = at & ((1 << c.page_shift) - 1);
        uint16_t* pool = kind == 1 ? c.k : c.v;
        const int64_t to = ((((int64_t)page * c.n_heads + head) << c.page_shift) + slot) * width;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int e = (l + L * n) * V;
            if (e >= half) continue;
            append_store<true, V>(pool, to + e, u[n]);
            append_store<true, V>(pool, to + half + e, w[n]);
        }
        for (int e = d + 4 * l; e < width; e += 4 * L) *reinterpret_cast<u32x2*>(pool + to + e) = u32x2{0, 0};   // the padding
    }
}

template <bool IN16, bool OUT16, int L, int V, int NV>
hipError_t launch_append(const AppendArgs& p, hipStream_t s) {
    constexpr int kHeads = 64 / L;
    const int64_t units = (p.n_q_heads + 2 * p.c.n_heads + kHeads - 1) / kHeads, wgs = (p.c.rows * units + 3) / 4;
    if (wgs > (1 << 24) - 1) return hipErrorInvalidConfiguration;   // 2^32 threads
    paged_append_kernel<IN16, OUT16, L, V, NV><<<dim3((unsigned)wgs), dim3(256), 0, s>>>(p);
    return hipGetLastError();
}

template <bool IN16, bool OUT16>
hipError_t launch_append_form(const AppendArgs& p, hipStream_t s) {
    const int half = p.c.head_dim / 2;
    if constexpr (IN16) {
        if (half % 8 == 0) return half <= 64 ? launch_append<IN16, OUT16, 8, 8, 1>(p, s) : launch_append<IN16, OUT16, 16, 8, 1>(p, s);
    }
    if (half % 4 == 0) return half <= 64 ? launch_append<IN16, OUT16, 16, 4, 1>(p, s) : launch_append<IN16, OUT16, 16, 4, 2>(p, s);
    return half <= 32 ? launch_append<IN16, OUT16, 16, 2, 1>(p, s) : half <= 64 ? launch_append<IN16, OUT16, 16, 2, 2>(p, s) : launch_append<IN16, OUT16, 16, 2, 4>(p, s);
}

}  // namespace

hipError_t launch_paged_append(const ::bl_paged_append_args& a, hipStream_t s) {
    AppendArgs p;
    p.c = paged_of(*a.cache, *a.rows);
    p.x[0] = a.q_dev; p.x[1] = a.k_dev; p.x[2] = a.v_dev;
    p.q_out = a.q_out_dev;
    p.gamma[0] = a.gamma_q_dev; p.gamma[1] = a.gamma_k_dev;
    p.rope = reinterpret_cast<const float2*>(a.rope_table_dev);
    p.ld[0] = a.ld_q; p.ld[1] = a.ld_k; p.ld[2] = a.ld_v;
    p.eps = a.eps;
    p.n_q_heads = a.n_q_heads;
    if (a.dt == BL_BF16) return a.q_out_dt == BL_BF16 ? launch_append_form<true, true>(p, s) : launch_append_form<true, false>(p, s);
    return a.q_out_dt == BL_BF16 ? launch_append_form<false, true>(p, s) : launch_append_form<false, false>(p, s);
}

}  // namespace bl
