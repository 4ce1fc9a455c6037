// One decoding step over an 8-bit cache (sparse_attn_decode8): for every (batch,
// head) the output of one query at its sequence's own position, attending
// S_position (Sec. 4.3) over codes with block scales.
//
// Bound by reading the rows of S_position, d bytes each for K and V.  Split-key as
// the step over an unquantised cache (sa_decode.hip): a workgroup walks one range of
// the set with a running maximum and sum, a second kernel joins the ranges.
#include <math.h>

#include "sa_e4m3.h"
#include "sa_internal.h"
#include "sa_mfma.h"

namespace sa {

namespace {

constexpr int kKeysPerSplit = 256;    // target keys per workgroup
constexpr int kMaxWorkgroups = 4096;  // splits are capped at this over all (batch, head)
constexpr int kWaves = 4;
constexpr int kCombineThreads = 256;

struct Decode8Args {
    Cache8 c;
    const int32_t* positions;
    int pattern, mode, heads, group, kv_heads, splits;  // group: query heads of a cache head
    int32_t sub, max_pos, l, sc;
    DivL dc;
    int64_t qsb, qsh;
    float scale_log2;
};

__device__ inline void load_q8(const uint16_t* p, float* x) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(u[e] << 16);
        x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
}
__device__ inline void load_q8(const float* p, float* x) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = a[e];
        x[4 + e] = b[e];
    }
}
// Factor of a state with maximum m in a sum relative to mx >= m; m = -inf is the empty state.
__device__ inline float weight(float m, float mx) { return m == -INFINITY ? 0.f : exp2_fast(m - mx); }

__device__ inline void put_nan(uint16_t* dst) { *dst = 0x7fc0; }
__device__ inline void put_nan(float* dst) { *reinterpret_cast<uint32_t*>(dst) = 0x7fc00000u; }
template <typename T>
__device__ inline void put(T* dst, float x) {
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<__bf16*>(dst) = (__bf16)x;
    else
        *dst = x;
}

// part: [batch * heads][splits][D + 2] fp32: D weighted V sums, running max, sum.
template <int D, typename T>
__global__ void __launch_bounds__(kWaves * 64)
decode8_split_kernel(Decode8Args a, const T* __restrict__ q, float* __restrict__ part) {
    constexpr int LPK = D / 8;     // lanes per key
    constexpr int KPW = 64 / LPK;  // keys per wave and pass
    __shared__ float s_m[kWaves], s_l[kWaves], s_acc[kWaves][D];
    const int tid = threadIdx.x, lane = tid % 64, w = tid / 64, slot = lane / LPK, ds = lane % LPK;
    int64_t id = blockIdx.x;
    const int split = (int)(id % a.splits);
    id /= a.splits;
    const int h = (int)(id % a.heads);
    const int64_t b = id / a.heads;
    const int64_t kvh = h / a.group;
    const int32_t pos = a.positions[b];
    const bool live = pos >= 0 && pos <= a.max_pos;
    const DecodeSet S(a.pattern, part_of_head(a.mode, h), live ? pos : 0, a.l, a.sc,
                      (int32_t)summary_start(a.l, a.sc, subblock_of_head(a.sub, h)), a.dc);
    const int64_t count = live ? S.count : 0;
    const int64_t per = (count + a.splits - 1) / a.splits;
    const int64_t t0 = split * per < count ? split * per : count, t1 = t0 + per < count ? t0 + per : count;

    float qv[8], acc[8], m = -INFINITY, l = 0.f;
    load_q8(q + b * a.qsb + h * a.qsh + 8 * ds, qv);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        qv[e] *= a.scale_log2;
        acc[e] = 0.f;
    }
    const int64_t base = b * a.c.sb + kvh * a.c.sh + 8 * ds, sbase = (b * a.kv_heads + kvh) * a.c.blocks;
    for (int64_t first = t0 + w * KPW; first < t1; first += kWaves * KPW) {
        const int64_t t = first + slot;
        const bool valid = t < t1;
        float vx[8], s = 0.f, sv = 0.f;
        if (valid) {
            const int32_t j = S.at(t);
            const int64_t row = base + (int64_t)j * a.c.ss, blk = sbase + (j >> a.c.block_shift);
            const u32x2 ku = *reinterpret_cast<const u32x2*>(a.c.k + row), vu = *reinterpret_cast<const u32x2*>(a.c.v + row);
            float kx[8];
            decode4(ku[0], kx);
            decode4(ku[1], kx + 4);
            decode4(vu[0], vx);
            decode4(vu[1], vx + 4);
            sv = a.c.vs[blk];
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(qv[e], kx[e], s);
            s *= a.c.ks[blk];
        }
#pragma unroll
        for (int off = 1; off < LPK; off <<= 1) s += __shfl_xor(s, off);
        if (valid) {
            const float mx = fmaxf(m, s), alpha = exp2_fast(m - mx), p = exp2_fast(s - mx);
            l = fmaf(l, alpha, p);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf(acc[e], alpha, p * (vx[e] * sv));
            m = mx;
        }
    }
#pragma unroll
    for (int off = LPK; off < 64; off <<= 1) {
        const float m2 = __shfl_xor(m, off), l2 = __shfl_xor(l, off), mx = fmaxf(m, m2);
        const float a1 = weight(m, mx), a2 = weight(m2, mx);
        l = l * a1 + l2 * a2;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = acc[e] * a1 + __shfl_xor(acc[e], off) * a2;
        m = mx;
    }
    if (slot == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s_acc[w][8 * ds + e] = acc[e];
        if (ds == 0) {
            s_m[w] = m;
            s_l[w] = l;
        }
    }
    __syncthreads();
    if (tid < D) {
        float mm = s_m[0], ll = 0.f, x = 0.f;
#pragma unroll
        for (int v = 1; v < kWaves; ++v) mm = fmaxf(mm, s_m[v]);
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            const float wt = weight(s_m[v], mm);
            ll = fmaf(s_l[v], wt, ll);
            x = fmaf(s_acc[v][tid], wt, x);
        }
        float* dst = part + ((b * a.heads + h) * a.splits + split) * (D + 2);
        dst[tid] = x;
        if (tid == 0) {
            dst[D] = mm;
            dst[D + 1] = ll;
        }
    }
}

// One workgroup per (batch, head): maximum first, one lane per range; then groups of D
// threads take every G-th range, and their sums are added in group order.
template <int D, typename T>
__global__ void __launch_bounds__(kCombineThreads)
decode8_combine_kernel(Decode8Args a, const float* __restrict__ part, T* __restrict__ o, float* __restrict__ lse) {
    constexpr int G = kCombineThreads / D;
    __shared__ float s_x[G][D], s_l[G];
    const int64_t row = blockIdx.x, b = row / a.heads, h = row % a.heads;
    const int tid = threadIdx.x, g = tid / D, e = tid % D;
    const float* src = part + row * a.splits * (D + 2);
    float m = -INFINITY;
    for (int s = tid % 64; s < a.splits; s += 64) m = fmaxf(m, src[(int64_t)s * (D + 2) + D]);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off));
    float l = 0.f, x = 0.f;
#pragma unroll 8
    for (int s = g; s < a.splits; s += G) {
        const float* p = src + (int64_t)s * (D + 2);
        const float wt = weight(p[D], m);
        l = fmaf(p[D + 1], wt, l);
        x = fmaf(p[e], wt, x);
    }
    s_x[g][e] = x;
    if (e == 0) s_l[g] = l;
    __syncthreads();
    if (tid < D) {
        x = l = 0.f;
#pragma unroll
        for (int t = 0; t < G; ++t) {
            x += s_x[t][tid];
            l += s_l[t];
        }
        T* dst = o + b * a.qsb + h * a.qsh + tid;
        if (a.positions[b] > a.max_pos) {  // no position of this call
            put_nan(dst);
            if (tid == 0) put_nan(lse + row);
        } else {  // no key: o = 0, lse = -inf
            put(dst, x * (l > 0.f ? 1.f / l : 0.f));
            if (tid == 0) lse[row] = l > 0.f ? (m + __log2f(l)) / kLog2e : -INFINITY;
        }
    }
}

template <int D, typename T>
hipError_t launch(const Decode8Args& a, int batch, const void* q, void* o, float* lse, float* part, hipStream_t stream) {
    const int64_t rows = (int64_t)batch * a.heads;
    hipLaunchKernelGGL((decode8_split_kernel<D, T>), dim3((unsigned)(rows * a.splits)), dim3(kWaves * 64), 0, stream, a,
                       (const T*)q, part);
    hipLaunchKernelGGL((decode8_combine_kernel<D, T>), dim3((unsigned)rows), dim3(kCombineThreads), 0, stream, a,
                       (const float*)part, (T*)o, lse);
    return hipGetLastError();
}

// Ranges per (batch, head): about kKeysPerSplit keys each for the largest set that a
// position up to max_pos can have, at most kMaxWorkgroups workgroups in all.
int splits_of(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c, int64_t rows) {
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
    int64_t splits = (count + kKeysPerSplit - 1) / kKeysPerSplit;
    const int64_t cap = kMaxWorkgroups / rows;
    if (splits > cap) splits = cap;
    return splits < 1 ? 1 : (int)splits;
}

}  // namespace

size_t decode8_workspace_bytes(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c,
                               int batch, int heads, int kv_heads, int d) {
    (void)kv_heads;
    const int64_t rows = (int64_t)batch * heads;
    return (size_t)rows * splits_of(pattern, mode, sub, max_pos, l, c, rows) * (d + 2) * sizeof(float);
}

hipError_t decode8_launch(const Cache8& cache, const int32_t* positions, int pattern, int mode, int32_t sub,
                          int32_t max_pos, int32_t l, int32_t c, int batch, int heads, int kv_heads, int d, int dtype,
                          const void* q, const int64_t* q_strides, float scale, void* o, float* lse, void* workspace,
                          hipStream_t stream) {
    Decode8Args a;
    a.c = cache;
    a.positions = positions;
    a.pattern = pattern;
    a.mode = mode;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.group = heads / kv_heads;
    a.splits = splits_of(pattern, mode, sub, max_pos, l, c, (int64_t)batch * heads);
    a.sub = sub;
    a.max_pos = max_pos;
    a.l = l;
    a.sc = c;
    a.dc = make_divl(c > 0 ? c : 1);
    a.qsb = q_strides[0];
    a.qsh = q_strides[1];
    a.scale_log2 = scale * kLog2eHost;
    float* part = static_cast<float*>(workspace);
    if (dtype == 1) {
        switch (d) {
        case 32: return launch<32, uint16_t>(a, batch, q, o, lse, part, stream);
        case 64: return launch<64, uint16_t>(a, batch, q, o, lse, part, stream);
        default: return launch<128, uint16_t>(a, batch, q, o, lse, part, stream);
        }
    }
    switch (d) {
    case 32: return launch<32, float>(a, batch, q, o, lse, part, stream);
    case 64: return launch<64, float>(a, batch, q, o, lse, part, stream);
    default: return launch<128, float>(a, batch, q, o, lse, part, stream);
    }
}

}  // namespace sa
