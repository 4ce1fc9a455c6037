// Rotary positions of several axes (sparse_attn_rotary).
//
// Element pair (x0, x1) of a token at place p of the pair's axis becomes
//     y0 = x0 cos(p f) - x1 sin(p f),  y1 = x0 sin(p f) + x1 cos(p f),
// f = base^(-2 t / s) for pair t of an axis of s elements.  The gradient is the
// rotation by -p f.  Nothing is reused but the angles, which all heads of a token
// share: the work is bound by reading and writing q and k once.  A thread owns W
// pairs of one token and makes their sines and cosines once for several heads.
//
// The angle in turns is p f / (2 pi) modulo 1.  With F = f / (2 pi) in units of
// 2^-64 turns, the low 64 bits of the integer product p F are that fraction, off by
// p times F's own error (sa_turns.h: 2^-29.9 turns at the furthest place) and with no range
// reduction: places of millions lose nothing.  Its upper 32 bits, read as signed, are the turn in [-1/2, 1/2).
#include "sa_internal.h"
#include "sa_mfma.h"
#include "sa_turns.h"

namespace sa {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocksX = 1 << 20;
// Heads that a thread turns, all of their loads on their way at once: up to 8 of bf16, 4 of
// fp32 (64 registers at the widest), fewer while there are not kEnoughBlocks workgroups
// (2 sequences of 12,288, 2 x 8 heads of 64, both directions: 4 heads a thread 46.4 us, 8
// 43.8, and 42.3 with 2,048 workgroups asked for in place of 1,024; fp32, 3 x 4,185 tokens, 16 heads of 128: 4 heads 85.6, 12 in three rounds 92.5; one
// token: 1 head 2.8, 8 5.5).
template <typename T>
constexpr int kBatch = 16 / sizeof(T);
constexpr int64_t kEnoughBlocks = 2048;

struct RotaryArgs {
    RotaryTensor t[2];
    const int32_t* places;
    int64_t pb, pn;
    int64_t n, tokens;        // tokens of a sequence; of the call
    int32_t unit_shift;       // log2 of the units of a token
    int32_t heads_per_slice;  // heads that a thread turns
    int32_t slices0;          // slices of the first tensor; the second one's follow
    int32_t axes, rotated;    // axes; elements that they own
    int32_t end[kMaxAxes];    // element behind each axis (behind the last one: d)
    float sign;
    uint64_t turn[64];        // F of every pair
};

template <typename T, int N>
struct Piece {
    typedef T type __attribute__((ext_vector_type(N)));
};
template <typename T>
struct Piece<T, 1> {
    typedef T type;
};
template <typename T, int N>
__device__ inline float element(const typename Piece<T, N>::type& v, int e) {
    if constexpr (N == 1) return (float)v;
    else return (float)v[e];
}
template <typename T, int N>
__device__ inline void set_element(typename Piece<T, N>::type& v, int e, float x) {
    if constexpr (N == 1) v = (T)x;
    else v[e] = (T)x;
}

// Sine and cosine of an angle in units of 2^-32 turns.  fp32 results take the library's, within
// a unit in the last place, of what is left of the angle behind its nearest quarter turn.  That is taken off
// in integers: as a float, a whole half turn is off by up to 2^-26 turns, more than the last place of its
// sine, and an eighth by 2^-28.  For bf16 results, which round to 2^-8, the hardware's instructions, whose
// argument is in turns: off by 2^-22.3 at most (measured over 3e7 angles; one token 3.4 -> 2.8 us;
// 2 sequences of 12,288, both directions, 45.5 -> 42.1).
__device__ inline void turn_sincos(int32_t turn, float* s, float* c, const float*) {
    const uint32_t quarter = ((uint32_t)turn + 0x20000000u) >> 30;
    float a, b;
    sincospif((float)(int32_t)((uint32_t)turn - (quarter << 30)) * 0x1p-31f, &a, &b);
    const float x = quarter & 1 ? b : a, y = quarter & 1 ? a : b;
    *s = quarter & 2 ? -x : x;
    *c = (quarter + 1) & 2 ? -y : y;
}
__device__ inline void turn_sincos(int32_t turn, float* s, float* c, const __bf16*) {
    const float x = (float)turn * 0x1p-32f;
    *s = __builtin_amdgcn_sinf(x);
    *c = __builtin_amdgcn_cosf(x);
}

// HALVES: the W pairs are elements e0 .. e0 + W - 1 and the same half an axis further;
// else the 2 W elements from e0 on, pair by pair.
template <typename T, int W, bool HALVES>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a) {
    constexpr int N = HALVES ? W : 2 * W, P = HALVES ? 2 : 1;  // elements of a piece; pieces of a unit
    typedef typename Piece<T, N>::type V;
    const int64_t idx = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kThreads + threadIdx.x;
    const int64_t tok = idx >> a.unit_shift;
    if (tok >= a.tokens) return;
    const int pair = ((int)idx & ((1 << a.unit_shift) - 1)) * W;  // the unit's first pair
    int64_t b = 0;
    if (tok >= a.n) b = a.tokens < ((int64_t)1 << 32) ? (uint32_t)tok / (uint32_t)a.n : tok / a.n;
    const int64_t i = tok - b * a.n;

    // where the unit's elements are (a unit of HALVES lies inside one axis or behind them);
    // axes are told apart by comparisons: an index into the arguments would be one more
    // read of memory on the way
    int e0 = 2 * pair, half = 0;
    if constexpr (HALVES) {
        int at = 0, size = a.end[0];
#pragma unroll
        for (int x = 0; x < kMaxAxes; ++x)
            if (2 * pair >= a.end[x]) {
                at = a.end[x];
                size = (x + 1 < kMaxAxes ? a.end[x + 1] : 2 * (W << a.unit_shift)) - at;
            }
        half = size / 2;
        e0 = pair + at / 2;
    }
    auto axis_of = [&](int p) {
        int x = 0;
#pragma unroll
        for (int k = 0; k < kMaxAxes; ++k) x += 2 * p >= a.end[k];
        return x < a.axes ? x : a.axes - 1;
    };

    // the heads' elements are on their way while the angles are made
    const bool second = (int)blockIdx.z >= a.slices0;
    const RotaryTensor r = second ? a.t[1] : a.t[0];
    const int h0 = ((int)blockIdx.z - (second ? a.slices0 : 0)) * a.heads_per_slice;
    const int h1 = h0 + a.heads_per_slice < r.heads ? h0 + a.heads_per_slice : r.heads;
    const T* x = (const T*)r.x + b * r.xb + i * r.xs + e0;
    T* y = (T*)r.y + b * r.yb + i * r.ys + e0;
    constexpr int B = kBatch<T>;
    V v[B][P];
#pragma unroll
    for (int u = 0; u < B; ++u)
        if (h0 + u < h1) {
#pragma unroll
            for (int k = 0; k < P; ++k) v[u][k] = *reinterpret_cast<const V*>(x + (h0 + u) * r.xh + k * half);
        }

    const int32_t* place = a.places + b * a.pb + i * a.pn;
    float c[W], s[W];
    const bool turned = 2 * pair < a.rotated;
    int64_t p = place[axis_of(pair)];
#pragma unroll
    for (int t = 0; t < W; ++t) {
        if (!HALVES && t > 0) p = place[axis_of(pair + t)];
        turn_sincos((int32_t)(((uint64_t)p * a.turn[pair + t]) >> 32), &s[t], &c[t], (const T*)nullptr);
    }
#pragma unroll
    for (int t = 0; t < W; ++t) s[t] *= a.sign;

#pragma unroll
    for (int u = 0; u < B; ++u)
        if (h0 + u < h1) {
#pragma unroll
            for (int t = 0; t < W; ++t) {
                V &z0 = v[u][0], &z1 = v[u][P - 1];
                const int i0 = HALVES ? t : 2 * t, i1 = HALVES ? t : 2 * t + 1;
                const float x0 = element<T, N>(z0, i0), x1 = element<T, N>(z1, i1);
                if (HALVES ? turned : 2 * (pair + t) < a.rotated) {
                    set_element<T, N>(z0, i0, x0 * c[t] - x1 * s[t]);
                    set_element<T, N>(z1, i1, x0 * s[t] + x1 * c[t]);
                }
            }
#pragma unroll
            for (int k = 0; k < P; ++k) *reinterpret_cast<V*>(y + (h0 + u) * r.yh + k * half) = v[u][k];
        }
}

template <typename T, int W, bool HALVES>
hipError_t launch(RotaryArgs& a, const RotaryCall& c, hipStream_t stream) {
    const int units = c.d / 2 / W;
    a.unit_shift = __builtin_ctz((unsigned)units);
    const int64_t blocks = (a.tokens * units + kThreads - 1) / kThreads;
    // a launch takes fewer than 2^32 threads along x
    const unsigned gx = (unsigned)(blocks < kMaxBlocksX ? blocks : kMaxBlocksX), gy = (unsigned)((blocks + gx - 1) / gx);
    auto slices = [&](int t) { return (a.t[t].heads + a.heads_per_slice - 1) / a.heads_per_slice; };
    a.heads_per_slice = kBatch<T>;
    while (a.heads_per_slice > 1 && blocks * (slices(0) + slices(1)) < kEnoughBlocks) a.heads_per_slice /= 2;
    a.slices0 = slices(0);
    const dim3 grid(gx, gy, (unsigned)(a.slices0 + slices(1)));
    hipLaunchKernelGGL((rotary_kernel<T, W, HALVES>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

// Pieces of at most 16 bytes, so that a lane's piece follows its neighbour's; for halves
// the widest that every axis' half is a multiple of (w, a power of two).
template <typename T>
hipError_t launch_width(RotaryArgs& a, const RotaryCall& c, int w, hipStream_t stream) {
    if (!c.halves) return launch<T, 8 / sizeof(T), false>(a, c, stream);
    if constexpr (sizeof(T) == 2)
        if (w == 8) return launch<T, 8, true>(a, c, stream);
    switch (w) {
    case 1: return launch<T, 1, true>(a, c, stream);
    case 2: return launch<T, 2, true>(a, c, stream);
    default: return launch<T, 4, true>(a, c, stream);
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
    int pair = 0;
    int w = 8;
    for (int x = 0; x < c.axes; ++x) {
        turn_units(c.base, c.dims[x], a.turn + pair);
        pair += c.dims[x] / 2;
        a.end[x] = 2 * pair;
        while ((c.dims[x] / 2) % w != 0) w /= 2;
    }
    for (int x = c.axes; x < kMaxAxes; ++x) a.end[x] = c.d;
    a.rotated = 2 * pair;
    while (pair < 64) a.turn[pair++] = 0;
    return c.dtype == 1 ? launch_width<__bf16>(a, c, w, stream) : launch_width<float>(a, c, w, stream);
}

}  // namespace sa
