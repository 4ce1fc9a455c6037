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
//   S [32 keys x 16 heads] = K q^T   K's scales in the conversion;
//   P = exp2(S - running maximum)    the D layout of S is the B layout of P; V's scales go
//                                    into P, where a lane holds the weights of 8 keys;
//   O^T [d x 16] += V^T P            transposing LDS reads give a lane 8 keys of one element.
// One head alone uses one column of 16 and pays for it in matrix time only, which the
// reads hide.
//
// The rows travel through registers into LDS, a key's row of K and its row of V by
// neighbouring lanes of one load: with both interleaved in memory a load reads whole
// lines of 128 bytes and a run of keys in one piece.  Loading the matrix layouts
// straight from memory instead, half a line for 16 scattered rows at a time, the
// same bytes took 57.5 us against 45.6 (32 sequences of 65,536, 8 heads of 64, loads alone).
#include <math.h>

#include "sa_e4m3.h"
#include "sa_internal.h"
#include "sa_mfma.h"

namespace sa {

namespace {

constexpr int kWaves = 4;
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
    int64_t qsb, qsh, osb, osh;  // strides of q and o
    float scale_log2;
};

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

// What a wave has in LDS: a chunk's rows (K, then V, of a key), their scales and their
// places in the cache.  The pitch of 16 bytes more than a row spreads the 16 rows that a
// read of K takes over the banks.
template <int D>
struct WaveLds {
    static constexpr int kPitch = 2 * D + 16;
    uint8_t rows[kChunk * kPitch];
    float ks[kChunk], vs[kChunk];
    uint32_t off[kChunk];
};

// The pieces of a chunk that a lane holds on their way to LDS, and a key's scales (lane = key, lane mod 32).
template <int D>
struct Rows {
    u32x4 x[D / 16];
    float ks, vs;
};

// Order of a wave's own LDS writes and reads across its lanes (the hardware keeps it).
__device__ inline void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Lane (g, r) = 16 g + r.  Key u of a chunk: row 4 g' + i of tile j for u = 8 g' + 4 j + i.
// (bf16 of d = 32 is one register over what six waves a SIMD may have: 256 units, 8,416 keys 33.7
// -> 31.9 us held to them.)
template <int D, typename T, int NWV, bool DIRECT>
__global__ void __launch_bounds__(NWV * 64, D == 32 && sizeof(T) == 2 ? 6 : 1)
decode8_split_kernel(Decode8Args a, const T* __restrict__ q, float* __restrict__ part, T* __restrict__ o,
                     float* __restrict__ lse) {
    constexpr int QP = sizeof(T) == 2 ? 1 : 3;   // pieces of a query
    constexpr int PP = sizeof(T) == 2 ? 2 : 3;   // pieces of a weight
    constexpr int FK = D / 32, TV = D / 16;      // 32-deep products of K; 16-element tiles of V
    constexpr int PR = D / 8;                    // 16-byte pieces of a key's rows
    union Lds {
        WaveLds<D> wave[NWV];
        struct {
            float acc[NWV][kCols][D + 4];
            float l[NWV][kCols];
        } join;
    };
    __shared__ __align__(16) Lds lds;
    __shared__ float s_m[NWV][kCols], s_top[kCols];

    const int tid = threadIdx.x, lane = tid % 64, w = __builtin_amdgcn_readfirstlane(tid / 64);
    const int g = lane / 16, r = lane % 16;
    // the same range of every unit in turn: the workgroups that run together read places far apart
    // (ranges of one unit side by side: 52.8 us against 45.6, loads alone)
    const uint32_t per_split = gridDim.x / a.splits;
    const int split = (int)(blockIdx.x / per_split);
    const uint32_t id = blockIdx.x % per_split;
    const int unit = (int)(id % a.u.units);
    const int64_t b = id / a.u.units;
    const int tile = unit % a.u.tiles, cls = unit / a.u.tiles % a.u.classes, kvh = unit / (a.u.tiles * a.u.classes);
    const int h0 = kvh * a.u.group + cls + tile * kCols * a.u.period;  // column c is head h0 + c * period
    const int left = (kvh + 1) * a.u.group - h0;
    const int cols = min(kCols, (left + a.u.period - 1) / a.u.period);  // < 1 for a class that has no such tile

    const int32_t pos = a.positions[b];
    const bool live = pos >= 0 && pos <= a.max_pos && cols > 0;
    const KeySet S(DecodeSet(a.pattern, part_of_head(a.mode, h0), live ? pos : 0, a.l, a.sc,
                             (int32_t)summary_start(a.l, a.sc, subblock_of_head(a.sub, h0)), a.dc));
    const uint32_t count = live ? S.count : 0, per = (count + a.splits - 1) / a.splits;
    const uint32_t t0 = min(split * per, count), t1 = min(t0 + per, count);

    WaveLds<D>& mine = lds.wave[w];
    // this lane's piece: of row 64 / PR * i + lane / PR in load i
    const int piece = lane % PR;
    const uint8_t* src = (piece < PR / 2 ? a.c.k : a.c.v) + b * a.c.sb + kvh * a.c.sh + 16 * (piece % (PR / 2));
    const int64_t sbase = (b * a.kv_heads + kvh) * a.c.blocks;
    const float *ksb = a.c.ks + sbase, *vsb = a.c.vs + sbase;

    float m = -INFINITY, l = 0.f;  // running maximum of q . k (unscaled), this lane's part of the sum
    f32x4 acc[TV];
#pragma unroll
    for (int t = 0; t < TV; ++t) acc[t] = zero4();

    auto fetch = [&](uint32_t first, Rows<D>& x) {
        // keys past the range repeat its last one (their weights become 0)
        const int32_t j = S.at(min(first + lane % kChunk, t1 - 1));
        mine.off[lane % kChunk] = (uint32_t)j * a.row16;
        x.ks = ksb[j >> a.c.block_shift];
        x.vs = vsb[j >> a.c.block_shift];
        wave_order();
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            x.x[i] = __builtin_nontemporal_load(
                reinterpret_cast<const u32x4*>(src + ((uint64_t)mine.off[64 / PR * i + lane / PR] << 4)));
        wave_order();
    };

    // the first rows are on their way before the query is taken apart
    constexpr uint32_t kStep = NWV * kChunk;
    uint32_t first = t0 + w * kChunk;
    Rows<D> x;
    if (first < t1) fetch(first, x);
    bf16x8 qf[FK][QP];
#pragma unroll
    for (int f = 0; f < FK; ++f) {
#pragma unroll
        for (int i = 0; i < QP; ++i) qf[f][i] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        // product f, index 8 g + t stands for element 64 (f / 2) + 16 g + 8 (f mod 2) + t (D = 32: 8 g + t)
        const int e = D == 32 ? 8 * g : 64 * (f / 2) + 16 * g + 8 * (f % 2);
        if (r < cols) query_pieces(q + b * a.qsb + (int64_t)(h0 + r * a.u.period) * a.qsh + e, qf[f]);
    }

    auto attend = [&](uint32_t first, const Rows<D>& x) {
        mine.ks[lane % kChunk] = x.ks;
        mine.vs[lane % kChunk] = x.vs;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
            *reinterpret_cast<u32x4*>(mine.rows + (64 / PR * i + lane / PR) * WaveLds<D>::kPitch + 16 * piece) = x.x[i];
        wave_order();
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int u = 8 * (r / 4) + 4 * t + r % 4;
            const uint8_t* row = mine.rows + u * WaveLds<D>::kPitch;
            const float ks = mine.ks[u];
            s[t] = zero4();
            // what the smaller pieces of an fp32 query add, summed apart: one by one into the whole sum, each of these
            // products would round it once more (8 of 12 at d = 128; error of o against 64 bits 2.9e-7 -> 1.5e-7, the
            // time the same)
            f32x4 low = zero4();
#pragma unroll
            for (int f = 0; f < FK; ++f) {
                const int e = D == 32 ? 8 * g : 64 * (f / 2) + 16 * g + 8 * (f % 2);
                const u32x2 k8 = *reinterpret_cast<const u32x2*>(row + e);
                const bf16x8 kf = scaled8(k8[0], k8[1], ks);
#pragma unroll
                for (int i = QP - 1; i > 0; --i) low = mfma_16x16x32(kf, qf[f][i], low);
                s[t] = mfma_16x16x32(kf, qf[f][0], s[t]);
            }
            if constexpr (QP > 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][i] += low[i];
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
        // (the difference first: the largest score has a weight of 1 and its neighbours' are right however
        // large both are; scaling before would lose 2^-24 of the scores themselves)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[t][i] = exp2_fast((s[t][i] - m) * a.scale_log2);
                l += s[t][i];
            }
        const f32x4 v0 = *reinterpret_cast<const f32x4*>(&mine.vs[8 * g]);
        const f32x4 v1 = *reinterpret_cast<const f32x4*>(&mine.vs[8 * g + 4]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[0][i] *= v0[i];
            s[1][i] *= v1[i];
        }
        // the weights as bf16 pieces that sum to them: two (2^-16 of a weight) for bf16 results, three (all 24 bits)
        // for fp32.  One piece would round a weight no finer than the result is: a set of a few keys
        // then came out a third further from the exact result, for 2% less time (32 sequences: 46.2 us, two
        // pieces 46.9, three 47.8); two pieces for fp32 were 2^-20 off, ten times its own rounding.
        bf16x8 pf[PP];
#pragma unroll
        for (int k = 0; k < PP; ++k) {
            pf[k] = pack_bf16x8(s[0], s[1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[0][i] -= (float)pf[k][i];
                s[1][i] -= (float)pf[k][4 + i];
            }
        }
#pragma unroll
        for (int t = 0; t < TV; ++t) {
            // lane i of a row of 16 gets element 16 t + i of keys 8 g .. 8 g + 7
            const u32x2 v8 = ld_tr8(mine.rows + (8 * g + r / 2) * WaveLds<D>::kPitch + D + 16 * t + 8 * (r % 2));
            const bf16x8 vf = scaled8(v8[0], v8[1], 1.f);
#pragma unroll
            for (int k = PP - 1; k >= 0; --k) acc[t] = mfma_16x16x32(vf, pf[k], acc[t]);
        }
        wave_order();  // read before the next chunk is written
    };

    if (first < t1) {
        if constexpr (D == 128) {
            // one chunk in registers: 4 KB more a wave on their way cost more in waves (a quarter of them) than they
            // gained (8 sequences, 4 cache heads, 8 query heads each: 23.4 -> 20.4 us)
            while (true) {
                attend(first, x);
                first += kStep;
                if (first >= t1) break;
                fetch(first, x);
            }
        } else {  // the next chunk's rows are on their way while a chunk is worked on
            Rows<D> y;
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
    }
    l = sum_over_g(l);

    // join the waves: the common maximum, then sums in the order of the waves; element
    // 16 t + 4 g + i of head column r is acc[t][i]
    if (g == 0) s_m[w][r] = m;
    __syncthreads();
    float top = s_m[0][r];
#pragma unroll
    for (int v = 1; v < NWV; ++v) top = fmaxf(top, s_m[v][r]);
    const float wt = weight(m, top, a.scale_log2);
    if (r < cols) {
#pragma unroll
        for (int t = 0; t < TV; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] *= wt;
            *reinterpret_cast<f32x4*>(&lds.join.acc[w][r][16 * t + 4 * g]) = acc[t];
        }
        if (g == 0) {
            lds.join.l[w][r] = l * wt;
            if (w == 0) s_top[r] = top;
        }
    }
    __syncthreads();
    const bool beyond = pos > a.max_pos;  // no position of this call: NaN; no key: o = 0, lse = -inf
    for (int i = tid; i < cols * D; i += NWV * 64) {
        const int c = i / D, e = i % D;
        float sum = 0.f, total = 0.f;
#pragma unroll
        for (int v = 0; v < NWV; ++v) {
            sum += lds.join.acc[v][c][e];
            total += lds.join.l[v][c];
        }
        const int64_t head = h0 + c * a.u.period, row = b * a.heads + head;
        if constexpr (DIRECT) {
            T* dst = o + b * a.osb + head * a.osh + e;
            if (beyond) put_nan(dst);
            else put(dst, sum * (no_key(total) ? 0.f : 1.f / total));
            if (e == 0) {
                if (beyond) put_nan(lse + row);
                else lse[row] = no_key(total) ? -INFINITY : (s_top[c] * a.scale_log2 + __log2f(total)) / kLog2e;
            }
        } else {
            float* dst = part + (row * a.splits + split) * (D + 2);
            dst[e] = sum;
            if (e == 0) {
                dst[D] = s_top[c];
                dst[D + 1] = total;
            }
        }
    }
}

// One workgroup per (batch, head).  Bound by the latency of reading the ranges' states, so
// they are read in one round: groups of D threads take every G-th range, eight at a time
// with a running maximum of their own, and the groups' states meet in LDS (four sequences
// of 1,048,576, the whole step: 7.4 us; with a common maximum taken first, 8.1).
template <int D, typename T, int NT>
__global__ void __launch_bounds__(NT)
decode8_combine_kernel(Decode8Args a, const float* __restrict__ part, T* __restrict__ o, float* __restrict__ lse) {
    constexpr int G = NT / D, U = 8;
    __shared__ float s_x[G][D], s_l[G], s_m[G];
    const int64_t row = blockIdx.x, b = row / a.heads, h = row % a.heads;
    const int tid = threadIdx.x, g = tid / D, e = tid % D;
    const float* src = part + row * a.splits * (D + 2);
    float m = -INFINITY, l = 0.f, x = 0.f;
    for (int s0 = g; s0 < a.splits; s0 += U * G) {
        float ms[U], ls[U], xs[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * G;
            const float* p = src + (int64_t)(s < a.splits ? s : s0) * (D + 2);
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
            const float wt = s0 + u * G < a.splits ? weight(ms[u], mx, a.scale_log2) : 0.f;
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

template <int D, typename T>
hipError_t launch(const Decode8Args& a, int batch, const void* q, void* o, float* lse, float* part, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)batch * a.u.units * a.splits)), wg(kWaves * 64);
    if (a.splits == 1) {
        hipLaunchKernelGGL((decode8_split_kernel<D, T, kWaves, true>), grid, wg, 0, stream, a, (const T*)q, part, (T*)o,
                           lse);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((decode8_split_kernel<D, T, kWaves, false>), grid, wg, 0, stream, a, (const T*)q, part, (T*)o,
                       lse);
    // one thread for each of a row's D elements and up to 16 ranges; more ranges, four times the threads (4
    // sequences of 8 cache heads of 64, 18 ranges: 9.8 -> 9.1 us)
    const dim3 rows((unsigned)(batch * a.heads));
    if (a.splits > 16)
        hipLaunchKernelGGL((decode8_combine_kernel<D, T, 1024>), rows, dim3(1024), 0, stream, a, (const float*)part,
                           (T*)o, lse);
    else
        hipLaunchKernelGGL((decode8_combine_kernel<D, T, 256>), rows, dim3(256), 0, stream, a, (const float*)part,
                           (T*)o, lse);
    return hipGetLastError();
}

// Ranges per unit, for the largest set that a position up to max_pos can have.
//   One range up to 256 keys, two chunks a wave: there is nothing to join (8 heads of 64, 206 keys: one
//   launch 4.8 us, two ranges 6.7).
//   Else 128 keys a range, one chunk a wave: the fewer serial steps the better, while there are few
//   workgroups (8 cache heads of 64, 736 keys: 256 keys a range 7.6 us, 128 7.2; d = 128 fp32, 2,272
//   keys 11.3 | 9.4).
//   From 512 workgroups on (1,024 for d <= 64, whose waves have less on their way; a quarter more before
//   a wave takes a second chunk) just so many, with longer ranges, as every range costs the join (8
//   sequences, 4 cache heads, d = 128, 8,416 keys: 2,112 workgroups 25.2, 1,024 20.4, 512 18.9), and at
//   most 128 ranges a unit (one unit, 65,760 keys: 512 ranges 15.1 us, 128 11.6).
//   Where that leaves more than 2,048 keys a range, ranges of about 1,024 (512 for d <= 64): walks of
//   different speed even out over more than one round (256 units of d = 128, 8,416 keys: 2 ranges
//   102 us, 8 92.5; 248 of d = 64, about 8,200 keys: 4 48.2, 16 46.6), up to 4,096 results to join or 512
//   a row, and whole rounds of the 1,024 workgroups that run at once (128 units of d = 64, 8,416 keys:
//   17 ranges 32.5, 8 29.2).
int splits_of(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c, int64_t units, int64_t rows,
              int d) {
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
    if (count <= 256) return 1;
    const int64_t finest = (count + 127) / 128, target = d == 128 ? 512 : 1024;
    const int64_t few = max64(min64(units * finest * 4 <= target * 5 ? finest : target / units, 128), 1);
    if (count <= 2048 * few) return (int)few;
    int64_t many = min64(min64(count / (d == 128 ? 1024 : 512), 4096 / rows), 512);
    const int64_t rounds = units * many / 1024;
    if (rounds > 0) many = rounds * 1024 / units;
    return (int)max64(few, many);
}

}  // namespace

size_t decode8_workspace_bytes(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c,
                               int batch, int heads, int kv_heads, int d) {
    const int64_t units = (int64_t)batch * head_units(mode, sub, heads, kv_heads).units;
    const int64_t rows = (int64_t)batch * heads;
    return (size_t)rows * splits_of(pattern, mode, sub, max_pos, l, c, units, rows, d) * (d + 2) * sizeof(float);
}

hipError_t decode8_launch(const Cache8& cache, const int32_t* positions, int pattern, int mode, int32_t sub,
                          int32_t max_pos, int32_t l, int32_t c, int batch, int heads, int kv_heads, int d, int dtype,
                          const void* q, const int64_t* q_strides, float scale, void* o, const int64_t* o_strides,
                          float* lse, void* workspace, hipStream_t stream) {
    Decode8Args a;
    a.c = cache;
    a.positions = positions;
    a.pattern = pattern;
    a.mode = mode;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.row16 = (uint32_t)(cache.ss / 16);
    a.u = head_units(mode, sub, heads, kv_heads);
    a.splits = splits_of(pattern, mode, sub, max_pos, l, c, (int64_t)batch * a.u.units, (int64_t)batch * heads, d);
    a.sub = sub;
    a.max_pos = max_pos;
    a.l = l;
    a.sc = c;
    a.dc = make_divl(c > 0 ? c : 1);
    a.qsb = q_strides[0];
    a.qsh = q_strides[1];
    a.osb = o_strides[0];
    a.osh = o_strides[1];
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
