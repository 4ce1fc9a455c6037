// Rotary positions of several axes (sparse_attn_rotary).
//
// Element pair (x0, x1) of a token at place p of the pair's axis becomes
//     y0 = x0 cos(p f) - x1 sin(p f),  y1 = x0 sin(p f) + x1 cos(p f),
// f = base^(-2 t / s) for pair t of an axis of s elements.  The gradient is the
// rotation by -p f.  Nothing is reused but the angles, which all heads of a token
// share: the work is bound by reading and writing q and k once.  A thread owns W
// pairs of one token, takes their sines and cosines once, and walks heads with
// them.
//
// The angle in turns is p f / (2 pi) modulo 1.  With F = f / (2 pi) in units of
// 2^-64 turns, the low 64 bits of the integer product p F are that fraction, with
// an error of p 2^-65 turns at most and no range reduction: places of millions lose
// nothing.  Its upper 32 bits, read as signed, are the turn in [-1/2, 1/2).
#include <math.h>

#include "sa_internal.h"
#include "sa_mfma.h"

namespace sa {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocksX = 1 << 20;

struct RotaryArgs {
    RotaryTensor t[2];
    const int32_t* places;
    int64_t pb, pn;
    int64_t n, tokens;        // tokens of a sequence; of the call
    int32_t unit_shift;       // log2 of the units of a token
    int32_t heads_per_slice;  // heads that a thread walks
    int32_t rotated;          // elements that axes own
    int32_t axes, dims[kMaxAxes];
    float sign;
    uint64_t turn[64];        // F of every pair
};

template <int N>
__device__ inline void load(const float* p, float* x) {
    typedef float V __attribute__((ext_vector_type(N)));
    const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = v[e];
}
template <>
__device__ inline void load<1>(const float* p, float* x) {
    *x = *p;
}
template <int N>
__device__ inline void load(const __bf16* p, float* x) {
    typedef __bf16 V __attribute__((ext_vector_type(N)));
    const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (float)v[e];
}
template <>
__device__ inline void load<1>(const __bf16* p, float* x) {
    *x = (float)*p;
}
template <int N, typename T>
__device__ inline void store(T* p, const float* x) {
    if constexpr (N == 1) {
        *p = (T)*x;
    } else {
        typedef T V __attribute__((ext_vector_type(N)));
        V v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)x[e];
        *reinterpret_cast<V*>(p) = v;
    }
}

// HALVES: the W pairs are elements e0 .. e0 + W - 1 and the same half an axis further;
// else the 2 W elements from e0 on, pair by pair.
template <typename T, int W, bool HALVES>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a) {
    const int64_t idx = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kThreads + threadIdx.x;
    const int64_t tok = idx >> a.unit_shift;
    if (tok >= a.tokens) return;
    const int pair = ((int)idx & ((1 << a.unit_shift) - 1)) * W;  // the unit's first pair
    const int64_t b = tok < a.n ? 0 : tok / a.n, i = tok - b * a.n;

    // the axis of each pair (units of HALVES lie inside one axis), and where the unit's elements are
    const int32_t* place = a.places + b * a.pb + i * a.pn;
    float c[W], s[W];
    int e0 = 2 * pair, half = 0;
    bool turned = true;
    if constexpr (HALVES) {
        int at = 0, axis = 0;
        while (axis < a.axes && 2 * pair >= at + a.dims[axis]) at += a.dims[axis++];
        turned = axis < a.axes;
        half = (turned ? a.dims[axis] : 2 * (W << a.unit_shift) - at) / 2;
        e0 = pair + at / 2;
        const int64_t p = turned ? place[axis] : 0;
#pragma unroll
        for (int t = 0; t < W; ++t) {
            const int32_t f = (int32_t)(((uint64_t)p * a.turn[pair + t]) >> 32);
            sincospif((float)f * 0x1p-31f, &s[t], &c[t]);
        }
    } else {
        int at = 0, axis = 0;
#pragma unroll
        for (int t = 0; t < W; ++t) {
            while (axis < a.axes && 2 * (pair + t) >= at + a.dims[axis]) at += a.dims[axis++];
            const int64_t p = axis < a.axes ? place[axis] : 0;
            const int32_t f = (int32_t)(((uint64_t)p * a.turn[pair + t]) >> 32);
            sincospif((float)f * 0x1p-31f, &s[t], &c[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < W; ++t) s[t] *= a.sign;

    const int h0 = blockIdx.z * a.heads_per_slice, all = a.t[0].heads + a.t[1].heads;
    const int h1 = h0 + a.heads_per_slice < all ? h0 + a.heads_per_slice : all;
    for (int h = h0; h < h1; ++h) {
        const bool second = h >= a.t[0].heads;
        const RotaryTensor& r = a.t[second];
        const int hh = second ? h - a.t[0].heads : h;
        const T* x = (const T*)r.x + b * r.xb + hh * r.xh + i * r.xs + e0;
        T* y = (T*)r.y + b * r.yb + hh * r.yh + i * r.ys + e0;
        if constexpr (HALVES) {
            float x0[W], x1[W], y0[W], y1[W];
            load<W>(x, x0);
            load<W>(x + half, x1);
#pragma unroll
            for (int t = 0; t < W; ++t) {
                y0[t] = turned ? x0[t] * c[t] - x1[t] * s[t] : x0[t];
                y1[t] = turned ? x0[t] * s[t] + x1[t] * c[t] : x1[t];
            }
            store<W>(y, y0);
            store<W>(y + half, y1);
        } else {
            float v[2 * W];
            load<2 * W>(x, v);
#pragma unroll
            for (int t = 0; t < W; ++t) {
                const float x0 = v[2 * t], x1 = v[2 * t + 1];
                if (2 * (pair + t) < a.rotated) {
                    v[2 * t] = x0 * c[t] - x1 * s[t];
                    v[2 * t + 1] = x0 * s[t] + x1 * c[t];
                }
            }
            store<2 * W>(y, v);
        }
    }
}

template <typename T, int W, bool HALVES>
hipError_t launch(RotaryArgs& a, const RotaryCall& c, hipStream_t stream) {
    const int units = c.d / 2 / W;
    a.unit_shift = __builtin_ctz((unsigned)units);
    const int64_t blocks = (a.tokens * units + kThreads - 1) / kThreads;
    // a launch takes fewer than 2^32 threads along x
    const unsigned gx = (unsigned)(blocks < kMaxBlocksX ? blocks : kMaxBlocksX), gy = (unsigned)((blocks + gx - 1) / gx);
    const int all = a.t[0].heads + a.t[1].heads;
    a.heads_per_slice = all;
    hipLaunchKernelGGL((rotary_kernel<T, W, HALVES>), dim3(gx, gy), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

template <typename T, bool HALVES>
hipError_t launch_width(RotaryArgs& a, const RotaryCall& c, int w, hipStream_t stream) {
    switch (w) {
    case 8: return launch<T, 8, HALVES>(a, c, stream);
    case 4: return launch<T, 4, HALVES>(a, c, stream);
    case 2: return launch<T, 2, HALVES>(a, c, stream);
    default: return launch<T, 1, HALVES>(a, c, stream);
    }
}

}  // namespace

hipError_t rotary_launch(const RotaryCall& c, hipStream_t stream) {
    RotaryArgs a;
    a.t[0] = c.t[0];
    a.t[1] = c.t[1];
    a.places = c.places;
    a.pb = c.pb;
    a.pn = c.pn;
    a.n = c.n;
    a.tokens = c.n * c.batch;
    a.axes = c.axes;
    a.sign = c.inverse ? -1.f : 1.f;
    // F by repeated products in extended precision (64 bits of mantissa): a few units
    // of 2^-64 off at the last of 64 pairs.  No turn of a whole pair reaches 2^64: f <= 1.
    int pair = 0;
    int w = 8;
    for (int x = 0; x < kMaxAxes; ++x) {
        a.dims[x] = x < c.axes ? c.dims[x] : 0;
        if (x >= c.axes) continue;
        const long double step = powl((long double)c.base, -2.0L / c.dims[x]);
        long double f = 0x1p64L / 6.283185307179586476925286766559L;
        for (int t = 0; t < c.dims[x] / 2; ++t, f *= step) a.turn[pair++] = (uint64_t)(f + 0.5L);
        while ((c.dims[x] / 2) % w != 0) w /= 2;
    }
    a.rotated = 2 * pair;
    while (pair < 64) a.turn[pair++] = 0;
    if (!c.halves) w = 4;  // 8 neighbouring elements
    if (c.dtype == 1)
        return c.halves ? launch_width<__bf16, true>(a, c, w, stream) : launch_width<__bf16, false>(a, c, w, stream);
    return c.halves ? launch_width<float, true>(a, c, w, stream) : launch_width<float, false>(a, c, w, stream);
}

}  // namespace sa
