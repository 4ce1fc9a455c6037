// One decoding step over a cache in pages (sparse_attn_paged_decode): for every (batch,
// head) the output of one query at its sequence's own position, attending S_position
// (Sec. 4.3) over keys and values in the elements' own type, page by page as the
// sequence's row of the page table says.
//
// Bound by reading the rows of S_position, d elements each for K and V, once for all query
// heads that share them.  Split-key: a workgroup walks one range of the set with a running
// maximum and sum, a second kernel joins the ranges (sa_step.h).
//
// The query heads that read one cache head with one set are the columns of the matrix
// products, up to 16.  A wave takes a chunk of keys at a time:
//   S [keys x 16 heads] = K q^T ;  P = exp2(S - running maximum) ;  O^T [d x 16] += V^T P
// in bf16 with 32 keys (16x16x32 products; P as two bf16 pieces, 2^-16 of a weight), in fp32
// with 16 keys (16x16x4 products, everything in fp32).  The D layout of S is the B layout of
// P, so the weights never leave their lane.  One head alone uses one column of 16 and pays
// for it in matrix time only, which the reads hide.
//
// The rows travel through registers into LDS, a key's row of K and its row of V by
// neighbouring lanes of one load: whole lines, and with both interleaved in memory one
// piece a key.  A key's page is a load that its rows depend on, so the pages of the chunk
// after next are asked for ahead of the next chunk's rows: loads return in order, and a
// wait for the pages then leaves the rows on their way.
#include "sa_step.h"

namespace sa {

namespace {

constexpr int kWaves = 4;

struct PagedArgs {
    PagedCache c;
    const int32_t* table;
    int64_t table_stride;
    const int32_t* positions;
    int32_t pages, shift;        // pages of the pool; log2 of a page's tokens
    int pattern, mode, heads, kv_heads, splits;
    HeadUnits u;
    int32_t sub, max_pos, l, sc;
    int32_t least;               // keys that a range is counted for, at least
    int32_t batch;
    int32_t each;                // ranges of every sequence at most; 0: `splits` of the whole batch (share_of)
    int2* cuts;                  // [batch, heads]: first range and ranges of a row
    DivL dc;
    int64_t qsb, qsh, osb, osh;  // strides of q and o
    float scale_log2;

    // The set of head h at a position.
    __device__ DecodeSet set(int h, int32_t pos) const {
        return DecodeSet(pattern, part_of_head(mode, h), pos, l, sc, (int32_t)summary_start(l, sc, subblock_of_head(sub, h)),
                         dc);
    }
    // Ranges of a row, and where their states lie: range i of the batch has one for each head.
    __device__ int ranges(int64_t b, int64_t h, int64_t* first, int64_t* step) const;
};

// How the sets of a batch are cut for one head: every sequence into equal ranges of at most `per` keys, all of
// them about `target` (PagedArgs::splits) ranges together, numbered through the batch.  Sequences of different
// lengths then take as long as each other: with a fixed number of ranges for each, 16 sequences between 866 and
// 32,767 keys (4 cache heads of 128, 8 query heads each) took 93.2 us, this way 53.8; of one length, 94.9 | 99.9, for
// the sums.  Every wave makes them by itself, a sequence a lane (64
// sequences at most).
struct Share {
    int64_t b;        // the sequence of a range (-1: there is none)
    int32_t base;     // ranges of the sequences before it
    int32_t ranges;   // its own
    uint32_t count;   // keys of its set
};
__device__ inline uint32_t keys_of(const PagedArgs& a, int h, int64_t b) {
    const int32_t pos = b < a.batch ? a.positions[b] : -1;
    return pos >= 0 && pos <= a.max_pos ? (uint32_t)a.set(h, pos).count : 0u;
}
// Sum over the lanes up to this one: within rows of 16 lanes, then across them, in registers.
__device__ inline int32_t sum_upto(int32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
    return x;
}
__device__ inline Share share_of(const PagedArgs& a, int h, int32_t range, int lane) {
    const uint32_t count = keys_of(a, h, lane);
    // in pieces of 64 keys, rounded up: all sequences' are within 32 bits
    const uint32_t total =
        (uint32_t)__builtin_amdgcn_readlane(sum_upto((int32_t)((count >> 6) + (count % 64 != 0))), 63);
    uint32_t per = max(min(total / a.splits + (total % a.splits != 0), 1u << 25) << 6, (uint32_t)a.least);
    int32_t n, upto;
    for (int i = 0;; ++i) {
        n = count == 0 ? 0 : (int32_t)((count - 1) / per + 1);
        upto = sum_upto(n);  // ranges up to this sequence
        const int32_t all = __builtin_amdgcn_readlane(upto, 63);
        if (all <= a.splits || i == 3) break;
        // rounded up for each sequence, they are more than `splits`: longer ones
        per = (uint32_t)min64(((int64_t)per * all / a.splits + 64) & ~63ll, (int64_t)1 << 31);
    }
    const uint64_t up = __builtin_amdgcn_ballot_w64(upto > range);
    if (!up) return {-1, 0, 0, 0};
    const int at = __builtin_ctzll(up);
    const int32_t ranges = __builtin_amdgcn_readlane(n, at);
    return {at, __builtin_amdgcn_readlane(upto, at) - ranges, ranges, (uint32_t)__builtin_amdgcn_readlane((int)count, at)};
}
// The row's first range leaves both numbers for the join (which forming the sums again took 1.8 us longer); a row
// without a key has none.
__device__ inline int PagedArgs::ranges(int64_t b, int64_t h, int64_t* first, int64_t* step) const {
    *step = heads;
    *first = 0;
    if (keys_of(*this, (int)h, b) == 0) return 0;
    const int2 at = cuts[b * heads + h];
    *first = (int64_t)at.x * heads + h;
    return at.y;
}

__device__ inline f32x4 mfma_f32(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// A NaN that the compiler does not know to be one (the build lets it assume that there is none).
__device__ inline float opaque_nan() {
    uint32_t x = 0x7fc00000u;
    asm volatile("" : "+v"(x));
    return __uint_as_float(x);
}

// Sizes of a wave's step.  The pitch of 16 bytes more than a key's two rows spreads the 16
// rows that a read of K takes over the banks.
template <int D, typename T>
struct Step {
    static constexpr int CH = sizeof(T) == 2 ? 32 : 16;          // keys
    static constexpr int RB = D * (int)sizeof(T);                // bytes of a row
    static constexpr int PITCH = 2 * RB + 16;
    static constexpr int PR = 2 * RB / 16;                       // 16-byte pieces of a key
    static constexpr int NL = CH * PR / 64;                      // loads of a lane
    static constexpr int TV = D / 16;                            // 16-element tiles of V
    static constexpr int V = D >= 64 ? 4 : 2, HB = D / (16 * V);  // fp32: neighbours in d per read of V, reads per row
};
template <int D, typename T>
struct WaveLds {
    uint8_t rows[Step<D, T>::CH * Step<D, T>::PITCH];
    int64_t off[Step<D, T>::CH];
};

// This lane's eight (bf16) or four (fp32) elements of a query, product by product.
template <int D, typename T>
struct Query;
template <int D>
struct Query<D, uint16_t> {
    bf16x8 x[D / 32];
    __device__ void zero() {
#pragma unroll
        for (int f = 0; f < D / 32; ++f) x[f] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
    }
    __device__ void load(const uint16_t* q, int g) {
#pragma unroll
        for (int f = 0; f < D / 32; ++f) x[f] = ld_bf16x8(q + 32 * f + 8 * g);
    }
};
template <int D>
struct Query<D, float> {
    f32x4 x[D / 16];
    __device__ void zero() {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) x[s] = zero4();
    }
    __device__ void load(const float* q, int g) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) x[s] = *reinterpret_cast<const f32x4*>(q + 16 * s + 4 * g);
    }
};

// Key u of a chunk is row r of tile j: bf16 u = 8 (r / 4) + 4 j + r mod 4 (two tiles, so that the
// D layout holds keys 8 g .. 8 g + 7 of a lane), fp32 u = r.  s[j][i] is key 8 g + 4 j + i (4 g + i).
template <int D>
__device__ inline void scores(const uint8_t* rows, const Query<D, uint16_t>& q, int g, int r, f32x4* s) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint16_t* row = reinterpret_cast<const uint16_t*>(rows + (8 * (r / 4) + 4 * j + r % 4) * Step<D, uint16_t>::PITCH);
        s[j] = zero4();
#pragma unroll
        for (int f = 0; f < D / 32; ++f) s[j] = mfma_16x16x32(ld_bf16x8(row + 32 * f + 8 * g), q.x[f], s[j]);
    }
}
template <int D>
__device__ inline void scores(const uint8_t* rows, const Query<D, float>& q, int g, int r, f32x4* s) {
    const float* row = reinterpret_cast<const float*>(rows + r * Step<D, float>::PITCH);
    f32x4 part[4] = {zero4(), zero4(), zero4(), zero4()};  // four short sums: half the rounding of one long one
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
        const f32x4 k = *reinterpret_cast<const f32x4*>(row + 16 * x + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i] = mfma_f32(k[i], q.x[x][i], part[i]);
    }
    s[0] = (part[0] + part[1]) + (part[2] + part[3]);
}

// acc += V^T P.  bf16: acc[t][i] is element 16 t + 4 g + i of head column r; fp32: acc[V hb + e][i]
// is element 16 V hb + V (4 g + i) + e.
template <int D>
__device__ inline void add_values(const uint8_t* rows, f32x4* p, int g, int r, f32x4* acc, uint16_t) {
    using S = Step<D, uint16_t>;
    bf16x8 hi, lo;  // the weights as two pieces that sum to them: one would round a weight no finer than the result is
    split_bf16x8(p[0], p[1], hi, lo);
#pragma unroll
    for (int t = 0; t < S::TV; ++t) {
        const uint8_t* at = rows + (8 * g + r / 4) * S::PITCH + S::RB + 2 * (16 * t + 4 * (r % 4));
        const u32x2 a = ld_tr16(reinterpret_cast<const uint16_t*>(at));
        const u32x2 b = ld_tr16(reinterpret_cast<const uint16_t*>(at + 4 * S::PITCH));
        const bf16x8 v = __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y});
        acc[t] = mfma_16x16x32(v, lo, acc[t]);
        acc[t] = mfma_16x16x32(v, hi, acc[t]);
    }
}
template <int D>
__device__ inline void add_values(const uint8_t* rows, f32x4* p, int g, int r, f32x4* acc, float) {
    using S = Step<D, float>;
    typedef float vec __attribute__((ext_vector_type(S::V)));
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int hb = 0; hb < S::HB; ++hb) {
            const vec v = *reinterpret_cast<const vec*>(rows + (4 * g + t) * S::PITCH + S::RB + 4 * (16 * S::V * hb + S::V * r));
#pragma unroll
            for (int e = 0; e < S::V; ++e) acc[S::V * hb + e] = mfma_f32(v[e], p[0][t], acc[S::V * hb + e]);
        }
}
template <int D, typename T>
__device__ inline int element(int t, int i, int g) {
    using S = Step<D, T>;
    if constexpr (sizeof(T) == 2) return 16 * t + 4 * g + i;
    else return 16 * S::V * (t / S::V) + S::V * (4 * g + i) + t % S::V;
}

template <int D, typename T, bool DIRECT>
__global__ void __launch_bounds__(kWaves * 64)
paged_split_kernel(PagedArgs a, const T* __restrict__ q, float* __restrict__ part, T* __restrict__ o,
                   float* __restrict__ lse) {
    using S = Step<D, T>;
    constexpr int CH = S::CH, NT = sizeof(T) == 2 ? 2 : 1;  // score tiles of a chunk
    union Lds {
        WaveLds<D, T> wave[kWaves];
        struct {
            float acc[kWaves][kCols][D + 4];
            float l[kWaves][kCols];
        } join;
    };
    __shared__ __align__(16) Lds lds;
    __shared__ float s_m[kWaves][kCols], s_top[kCols];

    const int tid = threadIdx.x, lane = tid % 64, w = __builtin_amdgcn_readfirstlane(tid / 64);
    const int g = lane / 16, r = lane % 16;
    const int unit = (int)(blockIdx.x % a.u.units);
    const int tile = unit % a.u.tiles, cls = unit / a.u.tiles % a.u.classes, kvh = unit / (a.u.tiles * a.u.classes);
    const int h0 = kvh * a.u.group + cls + tile * kCols * a.u.period;  // column c is head h0 + c * period
    const int left = (kvh + 1) * a.u.group - h0;
    const int cols = min(kCols, (left + a.u.period - 1) / a.u.period);  // < 1 for a class that has no such tile
    if (cols < 1) return;
    // the sequence and its keys t0 .. t1 - 1: all of them (one range a sequence), or the range of this workgroup
    int64_t b = blockIdx.x / a.u.units;
    const int32_t range = (int32_t)b;
    uint32_t t0 = 0, t1;
    if constexpr (DIRECT) {
        t1 = keys_of(a, h0, b);
    } else {
        Share s;
        if (a.each > 0) {
            s.b = range / a.each;
            s.base = (int32_t)s.b * a.each;
            s.count = keys_of(a, h0, s.b);
            if (s.count == 0) return;
            const uint32_t per = max((s.count + a.each - 1) / a.each, (uint32_t)a.least);
            s.ranges = (int32_t)((s.count - 1) / per + 1);
            if (range - s.base >= s.ranges) return;
        } else {
            s = share_of(a, h0, range, lane);
            if (s.b < 0) return;
        }
        b = s.b;
        // equal ranges of the sequence
        const uint32_t per = (s.count + s.ranges - 1) / s.ranges;
        t0 = min((range - s.base) * per, s.count);
        if (range == s.base && tid < cols) a.cuts[b * a.heads + h0 + tid * a.u.period] = make_int2(s.base, s.ranges);
        t1 = min(t0 + per, s.count);
    }
    const int32_t pos = a.positions[b];
    const KeySet set(a.set(h0, max(0, min(pos, a.max_pos))));

    WaveLds<D, T>& mine = lds.wave[w];
    // this lane's piece: of row 64 / PR * i + lane / PR in load i
    const int piece = lane % S::PR;
    const uint8_t* src = (piece < S::PR / 2 ? a.c.k : a.c.v) + kvh * a.c.sh + 16 * (piece % (S::PR / 2));
    const int32_t* table = a.table + b * a.table_stride;

    float m = -INFINITY, l = 0.f;  // running maximum of q . k (unscaled), this lane's part of the sum
    f32x4 acc[S::TV];
#pragma unroll
    for (int t = 0; t < S::TV; ++t) acc[t] = zero4();
    bool missing = false;  // a key of this wave whose page the pool does not have

    struct Key {
        int32_t at, page;
    };
    // keys past the range repeat its last one (their weights become 0)
    auto find = [&](uint32_t first) {
        const int32_t j = set.at(min(first + lane % CH, t1 - 1));
        return Key{j & ((1 << a.shift) - 1), table[j >> a.shift]};
    };
    auto fetch = [&](Key k, u32x4* x) {
        const bool there = (uint32_t)k.page < (uint32_t)a.pages;
        missing = missing || !there;
        mine.off[lane % CH] = (there ? k.page : 0) * a.c.sp + k.at * a.c.st;
        wave_order();
#pragma unroll
        for (int i = 0; i < S::NL; ++i)
            x[i] = __builtin_nontemporal_load(
                reinterpret_cast<const u32x4*>(src + mine.off[64 / S::PR * i + lane / S::PR]));
        wave_order();
    };

    constexpr uint32_t kStep = kWaves * CH;
    uint32_t first = t0 + w * CH;
    u32x4 x[S::NL];
    Key next{0, 0};
    if (first < t1) {
        const Key k = find(first);
        if (first + kStep < t1) next = find(first + kStep);
        fetch(k, x);
    }
    Query<D, T> qf;
    qf.zero();
    if (r < cols) qf.load(q + b * a.qsb + (int64_t)(h0 + r * a.u.period) * a.qsh, g);

    auto attend = [&](uint32_t first, const u32x4* x) {
#pragma unroll
        for (int i = 0; i < S::NL; ++i)
            *reinterpret_cast<u32x4*>(mine.rows + (64 / S::PR * i + lane / S::PR) * S::PITCH + 16 * piece) = x[i];
        wave_order();
        f32x4 s[NT];
        scores<D>(mine.rows, qf, g, r, s);
        if (first + CH > t1) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (first + 4 * NT * g + 4 * t + i >= t1) s[t][i] = -INFINITY;
        }
        float mx = m;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[t][i]);
        mx = max_over_g(mx);
        if (__builtin_amdgcn_ballot_w64(mx > m)) {  // a new maximum of some head: bring the sums to it
            const float alpha = weight(m, mx, a.scale_log2);
            l *= alpha;
#pragma unroll
            for (int t = 0; t < S::TV; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][i] *= alpha;
            m = mx;
        }
        // while every score so far is -inf, m is too: 0 as reference gives them the weight 0 that they have elsewhere
        const float m_ref = m == -INFINITY ? 0.f : m;
        // (the difference first: scaling before would lose 2^-24 of the scores themselves)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[t][i] = exp2_fast((s[t][i] - m_ref) * a.scale_log2);
                l += s[t][i];
            }
        add_values<D>(mine.rows, s, g, r, acc, T{});
        wave_order();  // read before the next chunk is written
    };

    if (first < t1) {
        if constexpr (S::NL > 8) {  // one chunk in registers
            while (true) {
                attend(first, x);
                first += kStep;
                if (first >= t1) break;
                const Key k = next;
                if (first + kStep < t1) next = find(first + kStep);
                fetch(k, x);
            }
        } else {  // the next chunk's rows are on their way while a chunk is worked on
            u32x4 y[S::NL];
            auto ahead = [&](u32x4* to) {  // the rows of the chunk after `first`, the pages of the one behind it
                if (first + kStep >= t1) return false;
                const Key k = next;
                if (first + 2 * kStep < t1) next = find(first + 2 * kStep);
                fetch(k, to);
                return true;
            };
            while (true) {
                const bool more = ahead(y);
                attend(first, x);
                if (!more) break;
                first += kStep;
                const bool again = ahead(x);
                attend(first, y);
                if (!again) break;
                first += kStep;
            }
        }
    }
    l = sum_over_g(l);
    if (__builtin_amdgcn_ballot_w64(missing)) l = opaque_nan();

    // join the waves: the common maximum, then sums in the order of the waves
    if (g == 0) s_m[w][r] = m;
    __syncthreads();
    float top = s_m[0][r];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) top = fmaxf(top, s_m[v][r]);
    const float wt = weight(m, top, a.scale_log2);
    if (r < cols) {
#pragma unroll
        for (int t = 0; t < S::TV; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) lds.join.acc[w][r][element<D, T>(t, i, g)] = acc[t][i] * wt;
        if (g == 0) {
            lds.join.l[w][r] = l * wt;
            if (w == 0) s_top[r] = top;
        }
    }
    __syncthreads();
    const bool beyond = pos > a.max_pos;  // no position of this call: NaN; no key: o = 0, lse = -inf
    for (int i = tid; i < cols * D; i += kWaves * 64) {
        const int c = i / D, e = i % D;
        float sum = 0.f, total = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
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
            float* dst = part + ((int64_t)range * a.heads + head) * (D + 2);
            dst[e] = sum;
            if (e == 0) {
                dst[D] = s_top[c];
                dst[D + 1] = total;
            }
        }
    }
}

// How a call's sets are cut.
struct Cut {
    int32_t splits;  // ranges of the batch, one more for each sequence at most; 0: every sequence is one range
    int32_t each;    // > 0: so many of every sequence instead
    int64_t ranges(int64_t batch) const { return each > 0 ? batch * each : splits + batch; }
};
//   One range a sequence up to 256 keys: there is nothing to join.
//   Up to 64 sequences: as many ranges as fill the workgroups that run at once (2 a compute unit for d = 128, whose
//   rows take 68 KB of LDS, 3 for d = 64, 5 for d = 32), so that they end together (one sequence of 32,768, 4 cache
//   heads of 128: 21.3 us, twice as many 29.2; 16 sequences of 866 to 32,767: 53.8 | 63.4), or four for each sequence.
//   More sequences, whose sums every workgroup would form at length: a number for each, four or what leaves a range
//   2,048 keys within 32,768 workgroups; short ranges even out over several rounds.  Ragged dense batches, us, at least
//   1 | 2 | 4 | 8 ranges: 96 of up to 4,096 (8 heads of 64) 44.7 | 44.7 | 42.8 | 46.9, 128 of up to 32,768 (32 on 4 of 128) 256 |
//   257 | 255 | 253, but 512 of up to 1,024 (8 of 64), which fill the chip by themselves, 62.6 | 76.1 | 109 | 140; ranges
//   of 1,024 | 2,048 | 4,096 keys at four: 128 of up to 32,768 293 | 255 | 257, 80 of up to 65,536 (8 of 64) 289 | 275 | 271.
// Ranges are counted for 128 keys each at least, one chunk a wave (two of fp32), and then made equal, the last with what
// is left (129 keys: 65 and 64); a shorter set is one range.
constexpr int32_t kLeastKeys = 128;
Cut cut_of(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c, int64_t batch, int64_t units, int d) {
    const int64_t count = largest_set(pattern, mode, sub, max_pos, l, c);
    if (count <= 256) return {0, 0};
    const int64_t finest = (count + kLeastKeys - 1) / kLeastKeys;
    if (batch > 64) {
        const int64_t each = max64(4, min64((count + 2047) / 2048, 32768 / (batch * units)));
        return {1, (int32_t)min64(each, finest)};
    }
    const int64_t places = 256 * (d == 128 ? 2 : d == 64 ? 3 : 5) / units;  // of one unit
    const int64_t n = places >= 2 * batch ? places : 4 * batch;
    return {(int32_t)max64(1, min64(n, batch * finest)), 0};
}

template <int D, typename T>
hipError_t launch(const PagedArgs& a, const void* q, void* o, float* lse, float* part, hipStream_t stream) {
    const dim3 wg(kWaves * 64);
    if (a.splits == 0) {
        hipLaunchKernelGGL((paged_split_kernel<D, T, true>), dim3((unsigned)((int64_t)a.batch * a.u.units)), wg, 0, stream, a,
                           (const T*)q, part, (T*)o, lse);
        return hipGetLastError();
    }
    const int64_t ranges = Cut{a.splits, a.each}.ranges(a.batch);
    hipLaunchKernelGGL((paged_split_kernel<D, T, false>), dim3((unsigned)(ranges * a.u.units)), wg, 0, stream, a,
                       (const T*)q, part, (T*)o, lse);
    return step_combine<D, T>(a, a.batch, a.each > 0 ? a.each : 2 * a.splits / a.batch, part, o, lse, stream);
}

}  // namespace

size_t paged_decode_workspace_bytes(int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l, int32_t c,
                                    int batch, int heads, int kv_heads, int d) {
    const Cut cut = cut_of(pattern, mode, sub, max_pos, l, c, batch, head_units(mode, sub, heads, kv_heads).units, d);
    if (cut.splits == 0) return 0;
    return (size_t)cut.ranges(batch) * heads * (d + 2) * sizeof(float) + (size_t)batch * heads * sizeof(int2);
}

hipError_t paged_decode_launch(const PagedStep& p, int pattern, int mode, int32_t sub, int32_t max_pos, int32_t l,
                               int32_t c, int batch, int heads, int kv_heads, int d, int dtype, const void* q,
                               const int64_t* q_strides, float scale, void* o, const int64_t* o_strides, float* lse,
                               void* workspace, hipStream_t stream) {
    PagedArgs a;
    a.c = p.cache;
    a.table = p.table;
    a.table_stride = p.table_stride;
    a.positions = p.positions;
    a.pages = p.pages;
    a.shift = p.shift;
    a.pattern = pattern;
    a.mode = mode;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.u = head_units(mode, sub, heads, kv_heads);
    a.batch = batch;
    const Cut cut = cut_of(pattern, mode, sub, max_pos, l, c, batch, a.u.units, d);
    a.splits = cut.splits;
    a.each = cut.each;
    a.least = kLeastKeys;
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
    a.cuts = reinterpret_cast<int2*>(part + cut.ranges(batch) * heads * (d + 2));  // (d + 2 is even)
    if (dtype == 1) {
        switch (d) {
        case 32: return launch<32, uint16_t>(a, q, o, lse, part, stream);
        case 64: return launch<64, uint16_t>(a, q, o, lse, part, stream);
        default: return launch<128, uint16_t>(a, q, o, lse, part, stream);
        }
    }
    switch (d) {
    case 32: return launch<32, float>(a, q, o, lse, part, stream);
    case 64: return launch<64, float>(a, q, o, lse, part, stream);
    default: return launch<128, float>(a, q, o, lse, part, stream);
    }
}

}  // namespace sa
