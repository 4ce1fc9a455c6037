// What the decoding steps share (the 8-bit cache's, sa_decode8.hip, and the paged one's,
// sa_paged_decode.hip): the query heads that read the same rows, the arithmetic of a
// partial softmax state, and the kernel that joins the states of a row's ranges.
#pragma once

#include <math.h>

#include "sa_internal.h"
#include "sa_mfma.h"

namespace sa {

constexpr int kCols = 16;             // query heads of a workgroup

// The query heads of a call in units that share rows: heads of one cache head with one
// set (Sec. 5.1: alternating heads have two, heads with summary subblocks one each;
// the set repeats every `period` heads), in tiles of kCols.
struct HeadUnits {
    int32_t group, period, classes, tiles, units;  // units: of all cache heads of a sequence
};
inline HeadUnits head_units(int mode, int32_t sub, int heads, int kv_heads) {
    HeadUnits u;
    u.group = heads / kv_heads;
    u.period = 1;
    if (mode == MODE_INTERLEAVED) u.period = sub == 0 ? 2 : (sub % 2 == 0 ? sub : 2 * sub);
    else if (mode != MODE_A1 && sub > 0) u.period = sub;
    u.classes = u.period < u.group ? u.period : u.group;
    u.tiles = ((u.group + u.period - 1) / u.period + kCols - 1) / kCols;
    u.units = kv_heads * u.classes * u.tiles;
    return u;
}

// Keys of the largest set that a position up to max_pos can have.
inline int64_t largest_set(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c) {
    const DivL dc = make_divl(c > 0 ? c : 1);
    // the largest set is max_pos's or (fixed) that of the last position of the l-block before
    const int32_t before = max_pos / l * l - 1;
    int64_t count = 0;
    for (int g = 0; g < layout_count(mode, sub); ++g) {
        const int32_t w = (int32_t)summary_start(l, c, subblock_of_layout(mode, sub, g));
        for (const int32_t pos : {max_pos, before < 0 ? max_pos : before}) {
            const DecodeSet S(pattern, part_of_layout(mode, g), pos, l, c, w, dc);
            count = S.count > count ? S.count : count;
        }
    }
    return count;
}

// Factor of a state with maximum m (a q . k, unscaled) in a sum relative to mx >= m; m = -inf
// is the empty state.
__device__ inline float weight(float m, float mx, float scale) {
    return m == -INFINITY ? 0.f : exp2_fast((m - mx) * scale);
}

// Whether a row's sum of weights (>= 0, or NaN) says that it has no key.  By its bits: the build lets comparisons
// assume that there is no NaN, and a NaN score must not pass for an empty row.
__device__ inline bool no_key(float total) { return __float_as_uint(total) == 0; }

__device__ inline void put_nan(uint16_t* dst) { *dst = 0x7fc0; }
__device__ inline void put_nan(float* dst) { *reinterpret_cast<uint32_t*>(dst) = 0x7fc00000u; }
template <typename T>
__device__ inline void put(T* dst, float x) {
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<__bf16*>(dst) = (__bf16)x;
    else
        *dst = x;
}

// Order of a wave's own LDS writes and reads across its lanes (the hardware keeps it).
__device__ inline void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// One workgroup per (batch, head).  Bound by the latency of reading the ranges' states, so
// they are read in one round: groups of D threads take every G-th range, eight at a time
// with a running maximum of their own, and the groups' states meet in LDS (four sequences
// of 1,048,576, the whole step: 7.4 us; with a common maximum taken first, 8.1).
template <int D, typename T, int NT, typename Args>
__global__ void __launch_bounds__(NT)
step_combine_kernel(Args a, const float* __restrict__ part, T* __restrict__ o, float* __restrict__ lse) {
    constexpr int G = NT / D, U = 8;
    __shared__ float s_x[G][D], s_l[G], s_m[G];
    const int64_t row = blockIdx.x, b = row / a.heads, h = row % a.heads;
    const int tid = threadIdx.x, g = tid / D, e = tid % D;
    int64_t first, step;  // the row's states: the first one, and from one to the next
    const int splits = a.ranges(b, h, &first, &step);
    const float* src = part + first * (D + 2);
    float m = -INFINITY, l = 0.f, x = 0.f;
    for (int s0 = g; s0 < splits; s0 += U * G) {
        float ms[U], ls[U], xs[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * G;
            const float* p = src + (s < splits ? s : s0) * step * (D + 2);
            xs[u] = p[e];
            ms[u] = p[D];
            ls[u] = p[D + 1];
        }
        float mx = m;
#pragma unroll
        for (int u = 0; u < U; ++u) mx = fmaxf(mx, ms[u]);
        const float old = weight(m, mx, a.scale_log2);
        l *= old;
        x *= old;
        m = mx;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float wt = s0 + u * G < splits ? weight(ms[u], mx, a.scale_log2) : 0.f;
            l = fmaf(ls[u], wt, l);
            x = fmaf(xs[u], wt, x);
        }
    }
    s_x[g][e] = x;
    if (e == 0) {
        s_m[g] = m;
        s_l[g] = l;
    }
    __syncthreads();
    if (tid < D) {
        m = s_m[0];
#pragma unroll
        for (int t = 1; t < G; ++t) m = fmaxf(m, s_m[t]);
        x = l = 0.f;
#pragma unroll
        for (int t = 0; t < G; ++t) {
            const float wt = weight(s_m[t], m, a.scale_log2);
            x = fmaf(s_x[t][tid], wt, x);
            l = fmaf(s_l[t], wt, l);
        }
        T* dst = o + b * a.osb + h * a.osh + tid;
        if (a.positions[b] > a.max_pos) {  // no position of this call
            put_nan(dst);
            if (tid == 0) put_nan(lse + row);
        } else {  // no key: o = 0, lse = -inf
            put(dst, x * (no_key(l) ? 0.f : 1.f / l));
            if (tid == 0) lse[row] = no_key(l) ? -INFINITY : (m * a.scale_log2 + __log2f(l)) / kLog2e;
        }
    }
}

// One thread for each of a row's D elements and up to 16 ranges (`most` of a row, about); more ranges, four times
// the threads (4 sequences of 8 cache heads of 64, 18 ranges of an 8-bit cache: 9.8 -> 9.1 us).
template <int D, typename T, typename Args>
hipError_t step_combine(const Args& a, int batch, int most, const float* part, void* o, float* lse, hipStream_t stream) {
    const dim3 rows((unsigned)(batch * a.heads));
    if (most > 16)
        hipLaunchKernelGGL((step_combine_kernel<D, T, 1024, Args>), rows, dim3(1024), 0, stream, a, part, (T*)o, lse);
    else
        hipLaunchKernelGGL((step_combine_kernel<D, T, 256, Args>), rows, dim3(256), 0, stream, a, part, (T*)o, lse);
    return hipGetLastError();
}

}  // namespace sa
