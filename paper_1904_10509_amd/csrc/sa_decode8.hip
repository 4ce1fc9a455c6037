// One decoding step over an 8-bit cache (sparse_attn_decode8): for every (batch,
// head) the output of one query at its sequence's own position, attending
// S_position (Sec. 4.3) over codes with block scales.
//
// Bound by reading the rows of S_position, d bytes each for K and V.  Split-key as
// the step over an unquantised cache (sa_decode.hip): a workgroup walks one range of
// the set with a running maximum and sum, a second kernel joins the ranges.
//
// The query heads that read one cache head with one set share every row read: up to
// 16 of them are the columns of the matrix products.  A code times its power-of-two
// scale is an exact bf16 (one conversion instruction, two elements, scale included),
// so bf16 matrix instructions lose nothing on K and V; a bf16 query goes in as it is,
// an fp32 one as three bf16 pieces (24 bits).  A wave takes 32 keys at a time:
//   S [32 keys x 16 heads] = K q^T   rows of K straight from memory as the A operand;
//   P = exp2(S - running maximum)    the D layout of S is the B layout of P;
//   O^T [d x 16] += V^T P            a lane holds 8 keys' bytes of D / 16 neighbouring
//                                    elements; pairs of keys are interleaved in registers.
// One head alone uses one column of 16 and pays for it in matrix time only, which the
// reads hide; what it would do with lanes on dot products is more than that.
#include <math.h>

#include "sa_e4m3.h"
#include "sa_internal.h"
#include "sa_mfma.h"

namespace sa {

namespace {

constexpr int kKeysPerSplit = 256;    // target keys per workgroup
constexpr int kMaxWorkgroups = 4096;  // splits are capped at this over all units
constexpr int kWaves = 4;
constexpr int kCombineThreads = 256;
constexpr int kCols = 16;             // query heads of a workgroup
constexpr int kChunk = 32;            // keys of a wave and step

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

struct Decode8Args {
    Cache8 c;
    uint32_t row16;  // token stride of the cache in 16-byte pieces
    const int32_t* positions;
    int pattern, mode, heads, kv_heads, splits;
    HeadUnits u;
    int32_t sub, max_pos, l, sc;
    DivL dc;
    int64_t qsb, qsh;
    float scale_log2;
};

__device__ inline float weight(float m, float mx, float scale) {
    return m == -INFINITY ? 0.f : exp2_fast((m - mx) * scale);
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

// Eight elements of a query as bf16 pieces that sum to them: one of bf16, three of fp32.
__device__ inline void query_pieces(const uint16_t* p, bf16x8* x) { x[0] = ld_bf16x8(p); }
__device__ inline void query_pieces(const float* p, bf16x8* x) {
    f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        x[i] = pack_bf16x8(a, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            a[e] -= (float)x[i][e];
            b[e] -= (float)x[i][4 + e];
        }
    }
}

// Row pieces of a chunk that a lane holds: D / 4 bytes of one key in each 16-key tile of K,
// D / 16 bytes of each of its 8 keys of V; and a key's scales (lane = key, lane mod 32).
template <int D>
struct Rows {
    uint32_t k[2][D / 16];
    uint32_t v[8][D < 64 ? 1 : D / 64];
    float ks, vs;
};

// Lane (g, r) = 16 g + r.  Key u of a chunk: row 4 g' + i of tile j for u = 8 g' + 4 j + i.
template <int D, typename T, int NWV, bool DIRECT>
__global__ void __launch_bounds__(NWV * 64)
decode8_split_kernel(Decode8Args a, const T* __restrict__ q, float* __restrict__ part, T* __restrict__ o,
                     float* __restrict__ lse) {
    constexpr int QP = sizeof(T) == 2 ? 1 : 3;   // pieces of a query
    constexpr int FK = D / 32, TV = D / 16;      // 32-deep products of K; 16-element tiles of V
    __shared__ __align__(16) uint32_t s_off[NWV][kChunk];
    __shared__ __align__(16) float s_ks[NWV][kChunk], s_vs[NWV][kChunk];
    __shared__ float s_m[NWV][kCols];
    __shared__ __align__(16) float s_acc[NWV / 2][kCols][D + 4];
    __shared__ float s_l[NWV / 2][kCols];

    const int tid = threadIdx.x, lane = tid % 64, w = __builtin_amdgcn_readfirstlane(tid / 64), g = lane / 16, r = lane % 16;
    int64_t id = blockIdx.x;
    const int split = (int)(id % a.splits);
    id /= a.splits;
    const int unit = (int)(id % a.u.units);
    const int64_t b = id / a.u.units;
    const int tile = unit % a.u.tiles, cls = unit / a.u.tiles % a.u.classes, kvh = unit / (a.u.tiles * a.u.classes);
    const int h0 = kvh * a.u.group + cls + tile * kCols * a.u.period;  // column c is head h0 + c * period
    const int left = (kvh + 1) * a.u.group - h0;
    const int cols = min(kCols, (left + a.u.period - 1) / a.u.period);  // < 1 for a class that has no such tile

    const int32_t pos = a.positions[b];
    const bool live = pos >= 0 && pos <= a.max_pos && cols > 0;
    const DecodeSet S(a.pattern, part_of_head(a.mode, h0), live ? pos : 0, a.l, a.sc,
                      (int32_t)summary_start(a.l, a.sc, subblock_of_head(a.sub, h0)), a.dc);
    const int64_t count = live ? S.count : 0;
    const int64_t per = (count + a.splits - 1) / a.splits;
    const int64_t t0 = split * per < count ? split * per : count, t1 = t0 + per < count ? t0 + per : count;

    bf16x8 qf[FK][QP];
#pragma unroll
    for (int f = 0; f < FK; ++f) {
#pragma unroll
        for (int i = 0; i < QP; ++i) qf[f][i] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        // product f, index 8 g + t stands for element 64 (f / 2) + 16 g + 8 (f mod 2) + t (D = 32: 8 g + t)
        const int e = D == 32 ? 8 * g : 64 * (f / 2) + 16 * g + 8 * (f % 2);
        if (r < cols) query_pieces(q + b * a.qsb + (int64_t)(h0 + r * a.u.period) * a.qsh + e, qf[f]);
    }
    const uint8_t* kb = a.c.k + b * a.c.sb + kvh * a.c.sh + (D == 32 ? 8 : 16) * g;
    const uint8_t* vb = a.c.v + b * a.c.sb + kvh * a.c.sh + D / 16 * r;
    const int64_t sbase = (b * a.kv_heads + kvh) * a.c.blocks;
    const float *ksb = a.c.ks + sbase, *vsb = a.c.vs + sbase;

    float m = -INFINITY, l = 0.f;  // running maximum of q . k (unscaled), this lane's part of the sum
    f32x4 acc[TV];
#pragma unroll
    for (int t = 0; t < TV; ++t) acc[t] = zero4();

    auto fetch = [&](int64_t first, Rows<D>& x) {
        // keys past the range repeat its last one (their weights become 0)
        const int64_t u = first + lane % kChunk;
        const int32_t j = S.at(u < t1 ? u : t1 - 1);
        s_off[w][lane % kChunk] = (uint32_t)j * a.row16;
        x.ks = ksb[j >> a.c.block_shift];
        x.vs = vsb[j >> a.c.block_shift];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint8_t* p = kb + ((uint64_t)s_off[w][8 * (r / 4) + 4 * t + r % 4] << 4);
            if constexpr (D == 32) {
                const u32x2 y = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
                x.k[t][0] = y[0];
                x.k[t][1] = y[1];
            } else {
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    const u32x4 y = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 64 * i));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.k[t][4 * i + e] = y[e];
                }
            }
        }
        const u32x4 o0 = *reinterpret_cast<const u32x4*>(&s_off[w][8 * g]), o1 = *reinterpret_cast<const u32x4*>(&s_off[w][8 * g + 4]);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint8_t* p = vb + ((uint64_t)(t < 4 ? o0[t % 4] : o1[t % 4]) << 4);
            if constexpr (D == 32) {
                x.v[t][0] = __builtin_nontemporal_load(reinterpret_cast<const uint16_t*>(p));
            } else if constexpr (D == 64) {
                x.v[t][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
            } else {
                const u32x2 y = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
                x.v[t][0] = y[0];
                x.v[t][1] = y[1];
            }
        }
        __builtin_amdgcn_wave_barrier();  // the offsets are read before the next chunk's are written
    };

    auto attend = [&](int64_t first, const Rows<D>& x) {
        s_ks[w][lane % kChunk] = x.ks;
        s_vs[w][lane % kChunk] = x.vs;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float ks = s_ks[w][8 * (r / 4) + 4 * t + r % 4];
            s[t] = zero4();
#pragma unroll
            for (int f = 0; f < FK; ++f) {
                const bf16x8 kf = scaled8(x.k[t][2 * f], x.k[t][2 * f + 1], ks);
#pragma unroll
                for (int i = QP - 1; i >= 0; --i) s[t] = mfma_16x16x32(kf, qf[f][i], s[t]);
            }
        }
        if (first + kChunk > t1) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (first + 8 * g + 4 * t + i >= t1) s[t][i] = -INFINITY;
        }
        float mx = m;
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(fmaxf(mx, s[0][i]), s[1][i]);
        mx = max_over_g(mx);
        if (__builtin_amdgcn_ballot_w64(mx > m)) {  // a new maximum of some head: bring the sums to it
            const float alpha = weight(m, mx, a.scale_log2);
            l *= alpha;
#pragma unroll
            for (int t = 0; t < TV; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][i] *= alpha;
            m = mx;
        }
        const float shift = m * a.scale_log2;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[t][i] = exp2_fast(fmaf(s[t][i], a.scale_log2, -shift));
                l += s[t][i];
            }
        // weights in bf16: a bf16 result is rounded no finer than each of them; an fp32 result takes a second
        // piece for the remainder (2^-17 of a weight)
        bf16x8 hi, lo;
        if constexpr (QP == 1)
            hi = pack_bf16x8(s[0], s[1]);
        else
            split_bf16x8(s[0], s[1], hi, lo);
        const f32x4 v0 = *reinterpret_cast<const f32x4*>(&s_vs[w][8 * g]), v1 = *reinterpret_cast<const f32x4*>(&s_vs[w][8 * g + 4]);
#pragma unroll
        for (int half = 0; half < TV / 2; ++half) {  // elements 2 half, 2 half + 1 of the lane's TV
            uint32_t pair[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const float vs = t < 4 ? v0[t % 4] : v1[t % 4];
                pair[t] = half % 2 ? scaled2<true>(x.v[t][half / 2], vs) : scaled2<false>(x.v[t][half / 2], vs);
            }
            u32x4 even, odd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                even[i] = __builtin_amdgcn_perm(pair[2 * i + 1], pair[2 * i], 0x05040100);
                odd[i] = __builtin_amdgcn_perm(pair[2 * i + 1], pair[2 * i], 0x07060302);
            }
            const bf16x8 fe = __builtin_bit_cast(bf16x8, even), fo = __builtin_bit_cast(bf16x8, odd);
            acc[2 * half] = mfma_16x16x32(fe, hi, acc[2 * half]);
            acc[2 * half + 1] = mfma_16x16x32(fo, hi, acc[2 * half + 1]);
            if constexpr (QP != 1) {
                acc[2 * half] = mfma_16x16x32(fe, lo, acc[2 * half]);
                acc[2 * half + 1] = mfma_16x16x32(fo, lo, acc[2 * half + 1]);
            }
        }
        __builtin_amdgcn_wave_barrier();  // the scales are read before the next chunk's are written
    };

    // the next chunk's rows are on their way while a chunk is worked on
    constexpr int64_t kStep = (int64_t)NWV * kChunk;
    int64_t first = t0 + (int64_t)w * kChunk;
    if (first < t1) {
        Rows<D> x, y;
        fetch(first, x);
        while (true) {
            const bool more = first + kStep < t1;
            if (more) fetch(first + kStep, y);
            attend(first, x);
            if (!more) break;
            first += kStep;
            const bool again = first + kStep < t1;
            if (again) fetch(first + kStep, x);
            attend(first, y);
            if (!again) break;
            first += kStep;
        }
    }
    l = sum_over_g(l);

    // join the waves: the common maximum, then sums in a fixed tree
    if (g == 0) s_m[w][r] = m;
    __syncthreads();
    float top = s_m[0][r];
#pragma unroll
    for (int v = 1; v < NWV; ++v) top = fmaxf(top, s_m[v][r]);
    const float wt = weight(m, top, a.scale_log2);
    l *= wt;
#pragma unroll
    for (int t = 0; t < TV; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] *= wt;
    // element TV (4 g + i) + t of head column r is acc[t][i]
#pragma unroll
    for (int half = NWV / 2; half >= 1; half /= 2) {
        if (w >= half && w < 2 * half) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < TV; ++t) s_acc[w - half][r][TV * (4 * g + i) + t] = acc[t][i];
            if (g == 0) s_l[w - half][r] = l;
        }
        __syncthreads();
        if (w < half) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < TV; ++t) acc[t][i] += s_acc[w][r][TV * (4 * g + i) + t];
            l += s_l[w][r];
        }
        __syncthreads();
    }
    if (w != 0 || r >= cols) return;
    const int64_t head = h0 + r * a.u.period, row = b * a.heads + head;
    if constexpr (DIRECT) {
        T* dst = o + b * a.qsb + head * a.qsh;
        const bool beyond = pos > a.max_pos;  // no position of this call: NaN; no key: o = 0, lse = -inf
        const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < TV; ++t) {
                if (beyond) put_nan(dst + TV * (4 * g + i) + t);
                else put(dst + TV * (4 * g + i) + t, acc[t][i] * inv);
            }
        if (g == 0) {
            if (beyond) put_nan(lse + row);
            else lse[row] = l > 0.f ? (top * a.scale_log2 + __log2f(l)) / kLog2e : -INFINITY;
        }
    } else {
        float* dst = part + (row * a.splits + split) * (D + 2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < TV; ++t) dst[TV * (4 * g + i) + t] = acc[t][i];
        if (g == 0) {
            dst[D] = top * a.scale_log2;
            dst[D + 1] = l;
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
    const dim3 grid((unsigned)((int64_t)batch * a.u.units * a.splits)), wg(kWaves * 64);
    if (a.splits == 1) {
        hipLaunchKernelGGL((decode8_split_kernel<D, T, kWaves, true>), grid, wg, 0, stream, a, (const T*)q, part, (T*)o, lse);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((decode8_split_kernel<D, T, kWaves, false>), grid, wg, 0, stream, a, (const T*)q, part, (T*)o, lse);
    hipLaunchKernelGGL((decode8_combine_kernel<D, T>), dim3((unsigned)(batch * a.heads)), dim3(kCombineThreads), 0, stream,
                       a, (const float*)part, (T*)o, lse);
    return hipGetLastError();
}

// Ranges per unit: about kKeysPerSplit keys each for the largest set that a
// position up to max_pos can have, at most kMaxWorkgroups workgroups in all.
int splits_of(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c, int64_t units) {
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
    const int64_t cap = kMaxWorkgroups / units;
    if (splits > cap) splits = cap;
    return splits < 1 ? 1 : (int)splits;
}

}  // namespace

size_t decode8_workspace_bytes(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c,
                               int batch, int heads, int kv_heads, int d) {
    const int64_t units = (int64_t)batch * head_units(mode, sub, heads, kv_heads).units;
    return (size_t)batch * heads * splits_of(pattern, mode, sub, max_pos, l, c, units) * (d + 2) * sizeof(float);
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
    a.row16 = (uint32_t)(cache.ss / 16);
    a.u = head_units(mode, sub, heads, kv_heads);
    a.splits = splits_of(pattern, mode, sub, max_pos, l, c, (int64_t)batch * a.u.units);
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
