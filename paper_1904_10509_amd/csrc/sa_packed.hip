// Attention over prompts packed one behind the other (sparse_attn_packed_fwd): every row
// attends its set (Sec. 4.3) within its own sequence, query heads sharing key heads.
//
// No layout and no block grid: a workgroup takes a tile of query rows of one sequence and
// walks the tile's keys as an index space, 64 (fp32: 32) at a time, with the softmax of
// sa_fwd.hip (running maximum and sum in registers, S^T = K Q^T, O^T += V^T P^T):
//   strided A1     the band from the first row's first key to the last row; l >= n is dense causal;
//   strided A2     a tile holds rows of one residue class (rows l apart): dense causal among them;
//   strided merged the classes first, their state (maximum, sum, O in fp32) into the workspace of
//                  the rows that have one (i >= 2 l), then the band, which goes on from that state;
//   fixed A1       the keys from the start of the first row's l-block;
//   fixed A2       the summary columns, gathered: column u is position (u / c) l + w + u mod c;
//   fixed merged   the summary columns of earlier l-blocks, gathered, then the keys of the own one.
// So every key that is read is attended by some row of the tile, but for what tiles round off.
//
// Where a tile lies follows from `starts` alone: sequence s owns the tile places from
// floor(starts[s] / Q) + s on (Q rows a tile), which leaves each at least ceil(n / Q) of them
// and takes at most tokens / Q + sequences in all.  Places behind a sequence's last tile are
// empty.
//
// What bounds it: long walks the matrix products and the exponentials beside them, which share a SIMD's time (32
// heads of 128, 4 x 4,096 dense: 680-694 us, 792-809 TFLOP/s; by the counters the products keep a SIMD busy for 40% of
// it and vector instructions issue for 46%; heads of 64, 65,536 fixed: 37% and 68%), short ones the steps' latency (two
// sequences of 12,288, strided merged: waves wait 53% of their time) and, strided merged, the states' way through memory.
#include "sa_finite.h"
#include "sa_internal.h"
#include "sa_mask.h"
#include "sa_mfma.h"
#include "sa_step.h"
#include "sa_tile.h"

namespace sa {

namespace {

constexpr int kNoBand = 0x7fffffff;

struct PackedArgs {
    const int32_t* starts;
    int32_t sequences, tokens;
    int64_t qt, qh, kt, kh, vt, vh, ot, oh;
    int32_t group;                     // query heads of a key head
    int32_t head0, head_step, run_heads;  // heads of this launch: head0, head0 + head_step, ...
    int32_t mode, sub, l, c;
    DivL dl, dc;
    int32_t step;                      // rows from one of a tile to the next: 1, or l for residue classes
    int32_t band;                      // strided: furthest key behind a row (kNoBand: none)
    int32_t shift;                     // strided: nearest one
    bool by_rows;                      // classes: one place a row of the batch, live where a tile begins
    int64_t places;                    // tile places of one head
    bool turn_heads;                   // heads of one launch have sets of different sizes
    float scale_log2;
    float *state_o, *state_ml;         // states of the classes, [heads, tokens, d] and [heads, tokens, 2]
    bool put_state;                    // write them, in place of o and lse
    int32_t state_from;                // rows from here on have one to go on from (0x7fffffff: none)
    float* lse;
};

// Tile of a place: rows i0, i0 + 1, ... (counted in steps) below n of the sequence (or class) whose first
// row is `base`.  n = 0: an empty place.
struct TilePlace {
    int32_t base, n, i0;
};

// The last sequence whose places begin at `place` or before.  Every wave finds it by itself.  More than 128 sequences
// are cut into 64 runs, whose first ones a round compares, until a run has no more; those are compared 64 a round, all
// loads of a round at once, up to the first that begins behind the place.  2^20 sequences take four rounds.  (8,000
// prompts of one token, 8 heads of 64, bf16: 1,545 us with 64 after 64 from the first one on, 402 so.)
struct Found {
    int32_t s, start, end;  // s < 0: none
};
__device__ inline Found sequence_of(const PackedArgs& a, uint32_t rows, uint32_t place, int lane) {
    auto clamped = [&](int32_t s) { return max(0, min(a.starts[s], a.tokens)); };
    auto first_place = [&](int32_t s, int32_t start) { return a.by_rows ? (uint32_t)start : (uint32_t)start / rows + s; };
    int32_t lo = 0, hi = a.sequences;
    while (hi - lo > 128) {
        const int32_t run = (hi - lo + 63) / 64, s = lo + lane * run;
        const bool below = s < hi && first_place(s, clamped(s)) <= place;
        const int found = __builtin_popcountll(__builtin_amdgcn_ballot_w64(below));  // (places ascend with s)
        if (found == 0) return {-1, 0, 0};
        lo += (found - 1) * run;
        hi = min(hi, lo + run);
    }
    Found f{-1, 0, 0};
    for (int32_t s0 = lo; s0 < hi; s0 += 64) {
        const int32_t s = s0 + lane;
        int32_t start = 0, end = 0;
        bool below = false;
        if (s < hi) {
            start = clamped(s);
            end = clamped(s + 1);
            below = first_place(s, start) <= place;
        }
        const uint64_t m = __builtin_amdgcn_ballot_w64(below);
        const int found = __builtin_popcountll(m);
        if (found > 0) {
            f.s = s0 + found - 1;
            f.start = __builtin_amdgcn_readlane(start, found - 1);
            f.end = __builtin_amdgcn_readlane(end, found - 1);
        }
        if (~m) break;
    }
    return f;
}

template <int ROWS>
__device__ inline TilePlace tile_place(const PackedArgs& a, uint32_t place, int lane) {
    uint32_t cls = 0;
    if (a.step > 1 && !a.by_rows) {
        const uint32_t block = place / (uint32_t)a.l;
        cls = place - block * a.l;
        place = block;
    }
    const uint32_t per = (uint32_t)min64((int64_t)ROWS * a.step, 0x7fffffff);
    const Found f = sequence_of(a, per, place, lane);
    const int32_t n = f.end - f.start;
    if (f.s < 0 || n <= 0) return {0, 0, 0};
    uint32_t tile;
    if (a.by_rows) {
        const uint32_t i = place - f.start;
        if (i >= (uint32_t)n) return {0, 0, 0};
        const uint32_t m = (uint32_t)div_l(a.dl, (int32_t)i);
        if (m % ROWS != 0) return {0, 0, 0};
        cls = i - m * a.l;
        tile = m / ROWS;
    } else {
        tile = place - ((uint32_t)f.start / per + f.s);
    }
    if ((uint32_t)n <= cls) return {0, 0, 0};
    const int32_t rows = a.step == 1 ? n : div_l(a.dl, n - 1 - (int32_t)cls) + 1;
    if (tile > (uint32_t)(rows - 1) / ROWS) return {0, 0, 0};
    return {f.start + (int32_t)cls, rows, (int32_t)(tile * ROWS)};
}

// Consecutive workgroups go to the 8 XCDs in turn: with heads in eighths, an XCD takes neighbouring heads, which
// share key heads, and their keys stay in its L2.  Places from the last one down: a sequence's longest walks first.
__device__ inline bool place_of(const PackedArgs& a, uint32_t* place, int* head) {
    const uint32_t id = blockIdx.x + gridDim.x * blockIdx.y, run = (uint32_t)a.run_heads;
    if (id >= (uint32_t)a.places * run) return false;
    uint32_t p, h;
    if (run % 8 == 0) {
        const uint32_t each = run / 8;
        p = id / 8 / each;
        h = id % 8 * each + (id / 8 - p * each);
        // heads that alternate between a short and a long set: every XCD takes both in turn
        if (a.turn_heads) h = (h + p) % run;
    } else {
        p = id / run;
        h = id - p * run;
    }
    *place = (uint32_t)a.places - 1 - p;
    *head = a.head0 + (int)h * a.head_step;
    return true;
}

// The walk of a tile of rows i0 .. i1: `far` gathered columns, then the keys lo .. hi.
struct Walk {
    int32_t far, lo, hi;
    int32_t far_steps, steps;
};
template <bool FIXED_, int ROWS, int KEYS>
__device__ inline Walk tile_walk(const PackedArgs& a, int part, int32_t w, const TilePlace& t) {
    Walk k{0, 0, -1, 0, 0};
    const int32_t i1 = min(t.i0 + ROWS, t.n) - 1;
    if constexpr (FIXED_) {
        const int32_t blk = div_l(a.dl, t.i0);
        if (part == PART_A2) {
            const int32_t last = div_l(a.dl, i1), past = i1 - last * a.l - w + 1;
            k.far = last * a.c + max(0, min(past, a.c));
        } else {
            k.far = part == PART_MERGED ? blk * a.c : 0;
            k.lo = blk * a.l;
            k.hi = i1;
        }
    } else {
        k.lo = a.band == kNoBand ? 0 : max(0, t.i0 - a.band) / KEYS * KEYS;
        k.hi = i1 - a.shift;
    }
    k.far_steps = (k.far + KEYS - 1) / KEYS;
    k.steps = k.far_steps + (k.hi >= k.lo ? (k.hi - k.lo) / KEYS + 1 : 0);
    return k;
}

// What a row of this lane attends.
struct Row {
    int32_t i;        // its index, the last valid one at most
    int32_t blk0;     // fixed: first key of its l-block
    int32_t columns;  // fixed: gathered columns that it attends
};
template <bool FIXED_>
__device__ inline Row packed_row(const PackedArgs& a, int part, int32_t w, const Walk& k, int32_t i) {
    Row x{i, 0, k.far};
    if constexpr (FIXED_) {
        const int32_t blk = div_l(a.dl, i);
        x.blk0 = blk * a.l;
        if (part == PART_A2) x.columns = blk * a.c + max(0, min(i - x.blk0 - w + 1, a.c));
    }
    return x;
}

// Attended keys of step e of a row, as bits.  `sum`: the summary columns among a near step's keys.
template <bool FIXED_, int KEYS>
__device__ inline uint64_t row_bits(const PackedArgs& a, int part, const Walk& k, const Row& x, int e, uint64_t sum) {
    uint64_t m;
    if (FIXED_ && e < k.far_steps) {
        m = bit_range(0, x.columns - 1 - KEYS * e);
    } else {
        const int32_t j0 = k.lo + KEYS * (e - k.far_steps);
        if constexpr (FIXED_) {
            m = bit_range(x.blk0 - j0, 63);
            if (part == PART_MERGED) m |= sum;
            m &= bit_range(0, x.i - j0);
        } else {
            m = bit_range(a.band == kNoBand ? 0 : x.i - a.band - j0, x.i - a.shift - j0);
        }
    }
    return KEYS == 64 ? m : m & ((1ull << (KEYS & 63)) - 1);
}

// Whether rows r0 .. r1 attend every key of step e.
template <bool FIXED_, int KEYS>
__device__ inline bool step_full(const PackedArgs& a, int part, const Walk& k, int e, const Row& first, const Row& last) {
    if (FIXED_ && e < k.far_steps) return KEYS * (e + 1) <= first.columns;
    const int32_t j0 = k.lo + KEYS * (e - k.far_steps);
    if constexpr (FIXED_) return j0 >= last.blk0 && j0 + KEYS - 1 <= first.i;
    else return (a.band == kNoBand || last.i - a.band <= j0) && j0 + KEYS - 1 <= first.i - a.shift;
}

// Row of a sequence that key `at` of step e is (at < KEYS; past the walk's last key it repeats that one).
template <bool FIXED_, int KEYS>
__device__ inline int32_t key_row(const PackedArgs& a, int32_t w, const Walk& k, int e, int at) {
    if (FIXED_ && e < k.far_steps) {
        const int32_t u = min(KEYS * e + at, k.far - 1), blk = div_l(a.dc, u);
        return blk * a.l + w + (u - blk * a.c);
    }
    return min(k.lo + KEYS * (e - k.far_steps) + at, k.hi);
}

// ---------------------------------------------------------------------------
// bf16: waves of 32 rows, 64 keys a step, v_mfma_f32_32x32x16_bf16
// ---------------------------------------------------------------------------
// With lane = 32 h + r: A operand A[r][8h .. 8h+7], B operand B[8h .. 8h+7][r], D result element i is
// D[8 (i / 4) + 4 h + i mod 4][r].  S^T = K Q^T leaves a lane 16 of 32 keys of its one query row, and the
// elements 8 n .. 8 n + 7 are the B operand of P^T for the 16 keys 16 n .. 16 n + 15, if the contraction
// index 8 h + t stands for key 16 n + 8 (t / 4) + 4 h + t mod 4: V^T is read that way.
typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ inline f32x16 mfma_32x32x16(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 zero16() { return f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0}; }
__device__ inline bf16x8 pack_half(const f32x16& s, int n) {
    return n == 0 ? pack_bf16x8(f32x4{s[0], s[1], s[2], s[3]}, f32x4{s[4], s[5], s[6], s[7]})
                  : pack_bf16x8(f32x4{s[8], s[9], s[10], s[11]}, f32x4{s[12], s[13], s[14], s[15]});
}
// Max / sum over the two lanes that share r.
__device__ inline float max_over_h(float x) {
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float sum_over_h(float x) {
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ inline bool non_finite16(const f32x16& x) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint32_t v = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        top = v > top ? v : top;
    }
    return top >= 0x7F800000u;
}

// acc += the products of 16 keys (operands a, b) with this lane's row, which attends the keys whose bit is set
// (bits from the first of the 16 on): where a value is an infinity or a NaN, 0 times it would not be 0.
template <int DB>
__device__ inline void accumulate_bits(const bf16x8* a, bf16x8 b, uint32_t bits, int h, f32x16* acc) {
    const u32x4 bw = __builtin_bit_cast(u32x4, b);
#pragma unroll 1
    for (int x = 0; x < 16; ++x) {  // one key at a time
        const int t = (x >> 3) * 4 + (x & 3);
        u32x4 keep;
#pragma unroll
        for (int y = 0; y < 4; ++y) keep[y] = h == ((x >> 2) & 1) && y == (t >> 1) ? ((t & 1) ? 0xFFFF0000u : 0xFFFFu) : 0u;
        const bf16x8 bx = __builtin_bit_cast(bf16x8, bw & keep);
        const bool on = (bits >> x) & 1u;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const bf16x8 ax = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, a[db]) & keep);
            const f32x16 sum = mfma_32x32x16(ax, bx, acc[db]);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] = on ? sum[i] : acc[db][i];
            __builtin_amdgcn_sched_barrier(0);  // one sum in flight: registers
        }
    }
}

template <int D, int NW, bool FIXED_>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(D == 128 || (D == 64 && NW == 2) ? 2 : 3)))
packed_bf16_kernel(PackedArgs a, const uint16_t* __restrict__ q, const uint16_t* __restrict__ k,
                   const uint16_t* __restrict__ v, uint16_t* __restrict__ o) {
    constexpr int KEYS = 64, ROWS = 32 * NW, KS = D / 16, DB = D / 32, PRE = D == 128 ? 8 : 2 * KS;
    __shared__ __attribute__((aligned(16))) uint16_t sK[2][KEYS * D];
    __shared__ __attribute__((aligned(16))) uint16_t sV[2][KEYS * D];
    constexpr uint32_t kTileBytes = KEYS * D * 2;
    const uint32_t sK_base = lds_addr(&sK[0][0]), sV_base = lds_addr(&sV[0][0]);
    const int tid = threadIdx.x, lane = tid % 64, hh = lane / 32, r = lane % 32;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64);
    const float c2 = a.scale_log2;
    // byte offsets of this lane's operand reads in a tile; row blocks of 16 leave the swizzle as it is
    uint32_t row_off[KS], tr_off[2][DB];
#pragma unroll
    for (int x = 0; x < KS; ++x) row_off[x] = 2u * Swz<D>::off(r, 16 * x + 8 * hh);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int db = 0; db < DB; ++db)
            tr_off[e][db] = 2u * Swz<D>::off(8 * e + 4 * hh + lane % 16 / 4, 32 * db + 16 * (lane / 16 % 2) + 4 * (lane % 4));
    // a 1 KiB window of a tile is WR rows; the windows of a wave lie a multiple of 16 rows apart, so that a lane
    // fetches the same chunk of its row in all of them
    constexpr int WR = 512 / D, PER = KEYS / WR / NW;
    static_assert(PER >= 1 && (NW * WR) % 16 == 0, "windows of a wave");
    const int wrow = lane / (64 / WR), chunk = (lane % (64 / WR)) ^ Swz<D>::perm(w * WR + wrow);

    uint32_t place;
    int h;
    if (!place_of(a, &place, &h)) return;
    const TilePlace t = tile_place<ROWS>(a, place, lane);
    if (t.n == 0) return;  // the same for the whole workgroup
    const int part = FIXED_ ? part_of_head(a.mode, h) : PART_A1;
    const int32_t win = FIXED_ ? (int32_t)summary_start(a.l, a.c, subblock_of_head(a.sub, h)) : 0;
    const Walk walk = tile_walk<FIXED_, ROWS, KEYS>(a, part, win, t);
    if (a.put_state && walk.steps == 0) return;
    MaskParams mp{FIXED, part, a.l, a.c, 0, 0, 0, win};
    if (FIXED_ && part == PART_MERGED && a.l <= 64) summary_words(a.l, a.c, win, &mp.sum_lo, &mp.sum_hi);
    const int row0 = t.i0 + w * 32;  // first row of this wave
    const Row head_row = packed_row<FIXED_>(a, part, win, walk, min(row0, t.n - 1)),
              tail_row = packed_row<FIXED_>(a, part, win, walk, min(row0 + 32, t.n) - 1);
    const uint16_t* kh = k + (int64_t)(h / a.group) * a.kh + (int64_t)t.base * a.kt;
    const uint16_t* vh = v + (int64_t)(h / a.group) * a.vh + (int64_t)t.base * a.vt;
    const int64_t ks = a.kt * a.step, vs = a.vt * a.step;

    const Row row = packed_row<FIXED_>(a, part, win, walk, min(row0 + r, t.n - 1));
    const int64_t token = t.base + (int64_t)row.i * a.step, at_row = (int64_t)h * a.tokens + token;
    bf16x8 qf[KS];
    f32x16 acc[DB];
    float m_run, l_run;
    // the state that the rows begin with: nothing, or what the classes left
    auto begin = [&] {
        m_run = -INFINITY;
        l_run = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = zero16();
        if (!FIXED_ && row.i >= a.state_from) {
            m_run = a.state_ml[2 * at_row];
            l_run = hh == 0 ? a.state_ml[2 * at_row + 1] : 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const f32x4 x = *reinterpret_cast<const f32x4*>(a.state_o + at_row * D + 32 * db + 8 * y + 4 * hh);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[db][4 * y + i] = x[i];
                }
        }
    };
    // One step's K and V rows to a ring stage.  Steps whose rows lie at the same distances from their first one (keys
    // one behind the other; columns in runs of c that divide 64) take their addresses from a scalar that moves on by a
    // constant; in the others, and where rows would lie behind the sequence, every lane forms its row's.  (32 heads of
    // 128, 4 x 4,096 dense: 685 us; the scalar formed anew for every step 728, per 1 KiB window 740.)
    const bool even = ks == vs && 64 * ks < (int64_t)1 << 30;
    const bool even_far = FIXED_ && even && KEYS % a.c == 0 && (KEYS / a.c) * (int64_t)a.l * ks < (int64_t)1 << 30;
    uint32_t off[PER];
    const uint16_t *kp = kh, *vp = vh;
    int64_t forward = 0;
    auto load_step = [&](int e, int stage) {
        const bool far = FIXED_ && e < walk.far_steps;
        const int32_t first = far ? KEYS * e : walk.lo + KEYS * (e - walk.far_steps);
        if (e == 0 || (FIXED_ && e == walk.far_steps)) {
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int at = WR * (w + NW * x) + wrow;
                const int32_t rows = far && even_far ? at / a.c * a.l + at % a.c : at;
                off[x] = (uint32_t)((rows * ks + 8 * chunk) * 2);
            }
            const int64_t j = far ? win : walk.lo;
            forward = (far ? (int64_t)(KEYS / a.c) * a.l : KEYS) * ks;  // (0 and unused where c > KEYS)
            kp = kh + j * ks;
            vp = vh + j * vs;
        }
        const uint32_t kdst = sK_base + stage * kTileBytes, vdst = sV_base + stage * kTileBytes;
        if (far ? even_far && first + KEYS <= walk.far : even && first + KEYS <= t.n) {
            const void *kb = uniform_ptr(kp), *vb = uniform_ptr(vp);
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int window = w + NW * x;
                dma_b128(kb, off[x], kdst + 1024 * window);
                dma_b128(vb, off[x], vdst + 1024 * window);
            }
        } else {
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int window = w + NW * x;
                const int64_t j = key_row<FIXED_, KEYS>(a, win, walk, e, WR * window + wrow);
                dma_b128_at(kh + j * ks + 8 * chunk, kdst + 1024 * window);
                dma_b128_at(vh + j * vs + 8 * chunk, vdst + 1024 * window);
            }
        }
        kp += forward;
        vp += forward;
    };

    // V^T operand of 16 keys: columns 32 db + r
    auto values = [&](const char* at, int db) {
        const u32x2 lo = ld_tr16(reinterpret_cast<const uint16_t*>(at + tr_off[0][db]));
        const u32x2 hi = ld_tr16(reinterpret_cast<const uint16_t*>(at + tr_off[1][db]));
        return __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
    };
    if (walk.steps > 0) load_step(0, 0);
    {
        const uint16_t* p = q + token * a.qt + h * a.qh;
#pragma unroll
        for (int x = 0; x < KS; ++x) qf[x] = ld_bf16x8(p + 16 * x + 8 * hh);
    }
    begin();
    // (no load is left inside the loop: a wait for one would drain the ring.  Where registers run out the compiler puts
    // some there all the same: fixed sets at d = 128 have two of the query's operands in scratch and reload them in every
    // step behind the next step's loads, so that a wave waits for those too.  65,536, 8 heads of 128 on 4, l = 256, c = 32:
    // 1,361 us, 830 TFLOP/s, waves wait 38% of their time; strided ones, whose scratch is touched outside the loop, 20%)
    wait_loads_upto<0>();
    int e = 0;
    two_stage_while([&](auto stage) {
        constexpr int st = decltype(stage)::value;
        if (e >= walk.steps) return false;
        wait_loads_upto<0>();
        __syncthreads();  // this step is in LDS everywhere; the other stage is free
        if (e + 1 < walk.steps) load_step(e + 1, st ^ 1);
        const char* tK = reinterpret_cast<const char*>(sK[st]);
        const char* tV = reinterpret_cast<const char*>(sV[st]);
        auto compute = [&](auto full) {
            uint64_t bits = ~0ull;
            int cls[2] = {CHUNK_ALL, CHUNK_ALL};
            if constexpr (!decltype(full)::value) {
                const int32_t j0 = walk.lo + KEYS * (e - walk.far_steps);
                uint64_t sum = 0;
                if (FIXED_ && part == PART_MERGED && e >= walk.far_steps) sum = summary_bits(mp, mod_l(a.dl, j0));
                bits = row_bits<FIXED_, KEYS>(a, part, walk, row, e, sum);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const uint32_t b = (uint32_t)(bits >> (32 * kb));
                    cls[kb] = __builtin_amdgcn_ballot_w64(b != 0u) == 0ull    ? CHUNK_NONE
                              : __builtin_amdgcn_ballot_w64(b != ~0u) == 0ull ? CHUNK_ALL
                                                                              : CHUNK_PART;
                }
                if (cls[0] == CHUNK_NONE && cls[1] == CHUNK_NONE) return;
            }
            f32x16 s[2];
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                s[kb] = zero16();
                if (cls[kb] == CHUNK_NONE) continue;
                bf16x8 kf[KS];
#pragma unroll
                for (int x = 0; x < KS; ++x)
                    kf[x] = ld_bf16x8(reinterpret_cast<const uint16_t*>(tK + row_off[x] + kb * 32 * D * 2));
#pragma unroll
                for (int x = 0; x < KS; ++x) s[kb] = mfma_32x32x16(kf[x], qf[x], s[kb]);
            }
            if constexpr (decltype(full)::value) {
                // the operands of 32 keys ahead of the first product, the other 32 keys' with them
                __builtin_amdgcn_sched_group_barrier(0x100, PRE, 0);
#pragma unroll
                for (int x = 0; x < 2 * KS - PRE; ++x) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, PRE, 0);
            }
            __builtin_amdgcn_s_setprio(0);
            float mloc = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                if (cls[kb] == CHUNK_NONE) continue;
                if (cls[kb] == CHUNK_PART) {
                    const uint32_t b = (uint32_t)(bits >> (32 * kb)) >> (4 * hh);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[kb][i] = select_or_neg_inf(bit_lane_mask(b, 8 * (i / 4) + i % 4), s[kb][i]);
                }
#pragma unroll
                for (int i = 0; i < 16; i += 2) mloc = fmaxf(fmaxf(mloc, s[kb][i]), s[kb][i + 1]);
            }
            mloc = max_over_h(mloc);
            const float m_new = fmaxf(m_run, mloc);
            // rows with nothing attended so far keep m = -inf; 0 as reference gives p = 0
            const float m_ref = m_new == -INFINITY ? 0.f : m_new;
            const float neg = -m_ref * c2;
            const float alpha = exp2_fast((m_run - m_ref) * c2);
            m_run = m_new;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] *= alpha;
            f32x4 psum = zero4();  // four chains (d = 64, 2 x 8,192 dense, 16 heads: 399 -> 392 us)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                if (cls[kb] == CHUNK_NONE) continue;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[kb][i] = exp2_fast(fmaf(s[kb][i], c2, neg));
                    psum[i % 4] += s[kb][i];
                }
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    // Weights rounded to bf16 for the matrix product, off by up to 2^-8 each; the sum takes them whole.
                    // The attention over a layout rounds them so too, and the two are to agree.  Two pieces would take
                    // the error against 64 bits from 0.0019-0.0021 to the output's own rounding, 0.0016, for half as
                    // many products again (9 prompts dense 579 -> 782 us, audio 1,185 -> 1,651).
                    const bf16x8 pf = pack_half(s[kb], n);
                    bf16x8 vt[DB];
#pragma unroll
                    for (int db = 0; db < DB; ++db) vt[db] = values(tV + (32 * kb + 16 * n) * D * 2, db);
#pragma unroll
                    for (int db = 0; db < DB; ++db) acc[db] = mfma_32x32x16(vt[db], pf, acc[db]);
                }
            }
            l_run = fmaf(l_run, alpha, (psum[0] + psum[1]) + (psum[2] + psum[3]));
        };
        if (step_full<FIXED_, KEYS>(a, part, walk, e, head_row, tail_row)) compute(std::true_type{});
        else compute(std::false_type{});
        ++e;
        return true;
    });
    // An infinity or a NaN in a key that a row does not attend must not reach it, but 0 times it is not 0: sums that
    // come out non-finite are formed a second time, with the products of partly attended chunks kept apart by row.
    bool bad = false;
#pragma unroll
    for (int db = 0; db < DB; ++db) bad = bad || non_finite16(acc[db]);
    if (__syncthreads_or(bad)) {
        begin();
#pragma unroll 1
        for (int e = 0; e < walk.steps; ++e) {
            load_step(e, 0);
            wait_loads_upto<0>();
            __syncthreads();
            const int32_t j0 = walk.lo + KEYS * (e - walk.far_steps);
            uint64_t sum = 0;
            if (FIXED_ && part == PART_MERGED && e >= walk.far_steps) sum = summary_bits(mp, mod_l(a.dl, j0));
            const uint64_t bits = row_bits<FIXED_, KEYS>(a, part, walk, row, e, sum);
            if (__builtin_amdgcn_ballot_w64(bits != 0ull) != 0ull) {
                f32x16 s[2];
                float mloc = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const char* tK = reinterpret_cast<const char*>(sK[0]) + kb * 32 * D * 2;
                    s[kb] = zero16();
#pragma unroll
                    for (int x = 0; x < KS; ++x)
                        s[kb] = mfma_32x32x16(ld_bf16x8(reinterpret_cast<const uint16_t*>(tK + row_off[x])), qf[x], s[kb]);
                    const uint32_t b = (uint32_t)(bits >> (32 * kb)) >> (4 * hh);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s[kb][i] = select_or_neg_inf(bit_lane_mask(b, 8 * (i / 4) + i % 4), s[kb][i]);
                        mloc = fmaxf(mloc, s[kb][i]);
                    }
                }
                const float m_new = fmaxf(m_run, max_over_h(mloc)), m_ref = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = exp2_fast((m_run - m_ref) * c2);
                m_run = m_new;
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] *= alpha;
                f32x4 psum = zero4();
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const uint32_t b = (uint32_t)(bits >> (32 * kb));
                    const bool all = __builtin_amdgcn_ballot_w64(b != ~0u) == 0ull;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s[kb][i] = exp2_fast(fmaf(s[kb][i], c2, -m_ref * c2));
                        psum[i % 4] += s[kb][i];
                    }
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const bf16x8 pf = pack_half(s[kb], n);
                        bf16x8 vt[DB];
#pragma unroll
                        for (int db = 0; db < DB; ++db)
                            vt[db] = values(reinterpret_cast<const char*>(sV[0]) + (32 * kb + 16 * n) * D * 2, db);
                        if (all) {
#pragma unroll
                            for (int db = 0; db < DB; ++db) acc[db] = mfma_32x32x16(vt[db], pf, acc[db]);
                        } else {
                            accumulate_bits<DB>(vt, pf, b >> (16 * n), hh, acc);
                        }
                    }
                }
                l_run = fmaf(l_run, alpha, (psum[0] + psum[1]) + (psum[2] + psum[3]));
            }
            __syncthreads();  // read before the next step is written
        }
    }

    const float l_tot = sum_over_h(l_run);
    if (row0 + r < t.n) {
        if (!a.put_state) {
            const bool none = no_key(l_tot);
            const float inv = none ? 0.f : 1.f / l_tot;
            uint16_t* orow = o + token * a.ot + h * a.oh;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    *reinterpret_cast<uint2*>(orow + 32 * db + 8 * y + 4 * hh) = pack_bf16x4_bits(
                        f32x4{acc[db][4 * y], acc[db][4 * y + 1], acc[db][4 * y + 2], acc[db][4 * y + 3]} * inv);
            if (hh == 0) a.lse[at_row] = none ? -INFINITY : (m_run * c2 + __log2f(l_tot)) / kLog2e;
        } else if (row.i >= a.shift) {  // (no key before: the band begins with nothing there)
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    *reinterpret_cast<f32x4*>(a.state_o + at_row * D + 32 * db + 8 * y + 4 * hh) =
                        f32x4{acc[db][4 * y], acc[db][4 * y + 1], acc[db][4 * y + 2], acc[db][4 * y + 3]};
            if (hh == 0) {
                a.state_ml[2 * at_row] = m_run;
                a.state_ml[2 * at_row + 1] = l_tot;
            }
        }
    }
}

// ---------------------------------------------------------------------------
// fp32: 16 rows and 16 of a step's 32 keys a wave, 16x16x4 products (see sa_f32.hip for their operands).  Two waves
// share the keys of 16 rows and join their states at the end, so that a tile's walk is spread over the four SIMDs: a
// ragged batch waits for its longest (2,777 tokens at most, 8 heads of 128, alternating factors: 113 us with four
// groups of 16 rows and a wave for each, 104 so; dense 4 x 2,048, 8 heads: 423 us, 81 TFLOP/s, the products 57% of it).
// ---------------------------------------------------------------------------
__device__ inline f32x4 mfma_f32(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// A tile of rows of D floats in LDS: 16-byte piece p of row R sits at p ^ (R mod 16) (8 where a row has 8
// pieces), which spreads the 16 rows that a read of K takes over the banks (reads of V take one row).
template <int D>
__device__ inline int swz32(int row, int piece) {
    return piece ^ (row & (D / 4 < 16 ? D / 4 - 1 : 15));
}

constexpr int kGroups = 2;  // groups of 16 rows of a tile: their waves and the keys' halves fill the four SIMDs

template <int D, bool FIXED_>
__global__ void __launch_bounds__(128 * kGroups) __attribute__((amdgpu_waves_per_eu(2)))
packed_f32_kernel(PackedArgs a, const float* __restrict__ q, const float* __restrict__ k, const float* __restrict__ v,
                  float* __restrict__ o) {
    constexpr int KEYS = 32, ROWS = 16 * kGroups, DB = D / 16;
    constexpr int V = D >= 64 ? 4 : 2, HB = D / (16 * V);  // neighbours in d per read of V, reads per row
    typedef float vec __attribute__((ext_vector_type(V)));
    __shared__ __attribute__((aligned(16))) float sK[2][KEYS * D];
    __shared__ __attribute__((aligned(16))) float sV[2][KEYS * D];
    __shared__ float s_m[kGroups][16], s_l[kGroups][16];
    constexpr uint32_t kTileBytes = KEYS * D * 4;
    const uint32_t sK_base = lds_addr(&sK[0][0]), sV_base = lds_addr(&sV[0][0]);
    const int tid = threadIdx.x, lane = tid % 64, g = lane / 16, r = lane % 16;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64) % kGroups;     // its 16 rows of the tile
    const int half = __builtin_amdgcn_readfirstlane(tid / 64) / kGroups;  // its 16 keys of a step
    const float c2 = a.scale_log2;

    uint32_t place;
    int h;
    if (!place_of(a, &place, &h)) return;
    const TilePlace t = tile_place<ROWS>(a, place, lane);
    if (t.n == 0) return;  // the same for the whole workgroup
    const int part = FIXED_ ? part_of_head(a.mode, h) : PART_A1;
    const int32_t win = FIXED_ ? (int32_t)summary_start(a.l, a.c, subblock_of_head(a.sub, h)) : 0;
    const Walk walk = tile_walk<FIXED_, ROWS, KEYS>(a, part, win, t);
    if (a.put_state && walk.steps == 0) return;
    MaskParams mp{FIXED, part, a.l, a.c, 0, 0, 0, win};
    if (FIXED_ && part == PART_MERGED && a.l <= 64) summary_words(a.l, a.c, win, &mp.sum_lo, &mp.sum_hi);
    const int row0 = t.i0 + w * 16;
    const Row head_row = packed_row<FIXED_>(a, part, win, walk, min(row0, t.n - 1)),
              tail_row = packed_row<FIXED_>(a, part, win, walk, min(row0 + 16, t.n) - 1);
    const float* kh = k + (int64_t)(h / a.group) * a.kh + (int64_t)t.base * a.kt;
    const float* vh = v + (int64_t)(h / a.group) * a.vh + (int64_t)t.base * a.vt;
    const int64_t ks = a.kt * a.step, vs = a.vt * a.step;

    const Row row = packed_row<FIXED_>(a, part, win, walk, min(row0 + r, t.n - 1));
    const int64_t token = t.base + (int64_t)row.i * a.step, at_row = (int64_t)h * a.tokens + token;
    f32x4 qf[DB], acc[DB];
    float m_run, l_run;
    // acc[V hb + e][i] is element 16 V hb + V (4 g + i) + e
    auto begin = [&] {
        m_run = -INFINITY;
        l_run = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = zero4();
        if (!FIXED_ && half == 0 && row.i >= a.state_from) {
            m_run = a.state_ml[2 * at_row];
            l_run = g == 0 ? a.state_ml[2 * at_row + 1] : 0.f;
#pragma unroll
            for (int hb = 0; hb < HB; ++hb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const vec x = *reinterpret_cast<const vec*>(a.state_o + at_row * D + 16 * V * hb + V * (4 * g + i));
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[V * hb + e][i] = x[e];
                }
        }
    };
    constexpr int PER = KEYS * D / 256 / kGroups;
    // the waves of the first half load K, the others V
    const float* src = half == 0 ? kh : vh;
    const int64_t stride = half == 0 ? ks : vs;
    const uint32_t ring = half == 0 ? sK_base : sV_base;
    auto load_step = [&](int e, int stage) {
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            const int window = w + kGroups * x, oe = 256 * window + 4 * lane;
            const int at = oe / D, piece = swz32<D>(at, (oe % D) / 4);
            const int64_t j = key_row<FIXED_, KEYS>(a, win, walk, e, at);
            dma_b128_at(src + j * stride + 4 * piece,
                        __builtin_amdgcn_readfirstlane(ring + stage * kTileBytes + 1024 * window));
        }
    };

    bool careful = false;
    while (true) {
        if (walk.steps > 0) load_step(0, 0);
        if (!careful) {
            const float* p = q + token * a.qt + h * a.qh;
#pragma unroll
            for (int x = 0; x < DB; ++x) qf[x] = *reinterpret_cast<const f32x4*>(p + 16 * x + 4 * g);
        }
        begin();
        wait_loads_upto<0>();
        int e = 0;
        two_stage_while([&](auto stage) {
            constexpr int st = decltype(stage)::value;
            if (e >= walk.steps) return false;
            wait_loads_upto<0>();
            __syncthreads();
            if (e + 1 < walk.steps) load_step(e + 1, st ^ 1);
            const float* tK = sK[st];
            const float* tV = sV[st];
            uint32_t bits = ~0u;
            if (!step_full<FIXED_, KEYS>(a, part, walk, e, head_row, tail_row)) {
                const int32_t j0 = walk.lo + KEYS * (e - walk.far_steps);
                uint64_t sum = 0;
                if (FIXED_ && part == PART_MERGED && e >= walk.far_steps) sum = summary_bits(mp, mod_l(a.dl, j0));
                bits = (uint32_t)row_bits<FIXED_, KEYS>(a, part, walk, row, e, sum);
            }
            bits = bits >> (16 * half) & 0xFFFFu;  // this wave's keys 16 half + 4 g + i
            if (__builtin_amdgcn_ballot_w64(bits != 0u) != 0ull) {
                f32x4 c0 = zero4(), c1 = zero4();
                const int at = 16 * half + r;
#pragma unroll
                for (int x = 0; x < DB; ++x) {
                    const f32x4 kf = *reinterpret_cast<const f32x4*>(tK + at * D + 4 * swz32<D>(at, 4 * x + g));
                    c0 = mfma_f32(kf[0], qf[x][0], c0);
                    c1 = mfma_f32(kf[1], qf[x][1], c1);
                    c0 = mfma_f32(kf[2], qf[x][2], c0);
                    c1 = mfma_f32(kf[3], qf[x][3], c1);
                }
                f32x4 s = c0 + c1;
                float mx = m_run;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[i] = select_or_neg_inf(bit_lane_mask(bits >> (4 * g), i), s[i]);
                    mx = fmaxf(mx, s[i]);
                }
                mx = max_over_g(mx);
                const float m_ref = mx == -INFINITY ? 0.f : mx;
                const float alpha = exp2_fast((m_run - m_ref) * c2);
                float psum = 0.f;
                // (the difference first: scaling before would lose 2^-24 of the scores themselves)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[i] = exp2_fast((s[i] - m_ref) * c2);
                    psum += s[i];
                }
                l_run = fmaf(l_run, alpha, psum);
                m_run = mx;
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] *= alpha;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = 16 * half + 4 * g + i;
#pragma unroll
                    for (int hb = 0; hb < HB; ++hb) {
                        const int col = 16 * V * hb + V * r;
                        const vec x = *reinterpret_cast<const vec*>(tV + key * D + 4 * swz32<D>(key, col / 4) + col % 4);
                        if (careful) {  // one key at a time, for the rows that attend it
#pragma unroll 1
                            for (int gk = 0; gk < 4; ++gk) {
                                const bool on = (bits >> (4 * gk + i)) & 1u;
#pragma unroll
                                for (int e = 0; e < V; ++e) {
                                    const f32x4 sum =
                                        mfma_f32(g == gk ? x[e] : 0.f, g == gk ? s[i] : 0.f, acc[V * hb + e]);
                                    if (on) acc[V * hb + e] = sum;
                                }
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < V; ++e) acc[V * hb + e] = mfma_f32(x[e], s[i], acc[V * hb + e]);
                        }
                    }
                }
            }
            ++e;
            return true;
        });
        const bool bad = non_finite<DB>(acc);
        if (!__syncthreads_or(bad) || careful) break;
        careful = true;
    }

    // the two states of a row, the first half's first
    float l_tot = sum_over_g(l_run);
    float* other = &sK[0][0];  // (what the ring holds has been read)
    static_assert(sizeof(sK) >= ROWS * D * sizeof(float), "a state of every row");
    if (half == 1) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
            *reinterpret_cast<f32x4*>(other + ((w * DB + db) * 64 + lane) * 4) = acc[db];
        if (g == 0) {
            s_m[w][r] = m_run;
            s_l[w][r] = l_tot;
        }
    }
    __syncthreads();
    if (half == 1 || row0 + r >= t.n) return;
    {
        const float m1 = s_m[w][r], top = fmaxf(m_run, m1);
        const float w0 = weight(m_run, top, c2), w1 = weight(m1, top, c2);
        l_tot = l_tot * w0 + s_l[w][r] * w1;
        m_run = top;
#pragma unroll
        for (int db = 0; db < DB; ++db)
            acc[db] = acc[db] * w0 + *reinterpret_cast<const f32x4*>(other + ((w * DB + db) * 64 + lane) * 4) * w1;
    }
    const bool none = no_key(l_tot);
    const float inv = a.put_state ? 1.f : none ? 0.f : 1.f / l_tot;
    if (a.put_state && row.i < a.shift) return;
    float* dst = a.put_state ? a.state_o + at_row * D : o + token * a.ot + h * a.oh;
#pragma unroll
    for (int hb = 0; hb < HB; ++hb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vec x;
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = acc[V * hb + e][i] * inv;
            *reinterpret_cast<vec*>(dst + 16 * V * hb + V * (4 * g + i)) = x;
        }
    if (g != 0) return;
    if (a.put_state) {
        a.state_ml[2 * at_row] = m_run;
        a.state_ml[2 * at_row + 1] = l_tot;
    } else {
        a.lse[at_row] = none ? -INFINITY : (m_run * c2 + __log2f(l_tot)) / kLog2e;
    }
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------
constexpr int64_t kMaxGridX = 1 << 20;     // workgroups along x; along y the rest
// Tiles of 128 rows from so many workgroups on, which fill the chip; below, tiles of 64 (d = 128: always 128, as
// two waves a workgroup would leave its 64 KB of LDS half used).  Heads of 64, us, 128 rows | 64: 2 x 8,192 dense of 16
// heads 400 | 444, 65,536 + 57,026 fixed 1,175 | 1,345; 2 x 12,288 strided merged of 8 heads 76 | 74, six ragged ones 88 |
// 78.  The count takes in the places that stay empty, so many short prompts of 8 heads have tiles of 128 rows too, which
// they fill less: 200 of 20 tokens 16.0 | 11.7, 1,000 of 20 61.5 | 43.3, 100 of 1,000 strided merged 862 | 608.
constexpr int64_t kWidePlaces = 1024;

dim3 grid_of(const PackedArgs& a) {
    const int64_t n = a.places * a.run_heads;
    return dim3((unsigned)min64(n, kMaxGridX), (unsigned)((n + kMaxGridX - 1) / kMaxGridX));
}

int64_t tile_places(int64_t tokens, int64_t sequences, int32_t step, int rows) {
    if (step == 1) return tokens / rows + sequences;
    const int64_t per = (int64_t)rows * step;
    return min64((int64_t)step * (tokens / min64(per, 0x7fffffff) + sequences), tokens);
}
int64_t tile_places(const PackedArgs& a, int rows) { return tile_places(a.tokens, a.sequences, a.step, rows); }

template <int D, int NW, bool FIXED_>
hipError_t run_bf16(PackedArgs& a, const PackedCall& p, hipStream_t stream) {
    a.places = tile_places(a, 32 * NW);
    a.by_rows = a.step > 1 && a.places == a.tokens;
    hipLaunchKernelGGL((packed_bf16_kernel<D, NW, FIXED_>), grid_of(a), dim3(64 * NW), 0, stream, a, (const uint16_t*)p.q,
                       (const uint16_t*)p.k, (const uint16_t*)p.v, (uint16_t*)p.o);
    return hipGetLastError();
}

template <int D, bool FIXED_>
hipError_t run(PackedArgs& a, const PackedCall& p, hipStream_t stream) {
    if (p.dtype == 1) {
        if (D == 128 || tile_places(a, 128) * a.run_heads >= kWidePlaces) return run_bf16<D, 4, FIXED_>(a, p, stream);
        if constexpr (D < 128) return run_bf16<D, 2, FIXED_>(a, p, stream);
    }
    a.places = tile_places(a, 16 * kGroups);
    a.by_rows = a.step > 1 && a.places == a.tokens;
    hipLaunchKernelGGL((packed_f32_kernel<D, FIXED_>), grid_of(a), dim3(128 * kGroups), 0, stream, a, (const float*)p.q,
                       (const float*)p.k, (const float*)p.v, (float*)p.o);
    return hipGetLastError();
}

template <bool FIXED_>
hipError_t run_d(PackedArgs& a, const PackedCall& p, hipStream_t stream) {
    switch (p.d) {
    case 32: return run<32, FIXED_>(a, p, stream);
    case 64: return run<64, FIXED_>(a, p, stream);
    default: return run<128, FIXED_>(a, p, stream);
    }
}

// Whether a strided merged call has rows with keys beyond the band.
bool has_classes(int64_t tokens, int32_t pattern, int32_t mode, int32_t l) {
    return pattern == STRIDED && mode == MODE_MERGED && tokens > 2 * (int64_t)l;
}

}  // namespace

size_t packed_workspace_bytes(int64_t tokens, int32_t pattern, int32_t mode, int32_t l, int32_t heads, int32_t d) {
    return has_classes(tokens, pattern, mode, l) ? (size_t)tokens * heads * (d + 2) * sizeof(float) : 0;
}

bool packed_fits(const PackedCall& p) {
    const bool classes = p.pattern == STRIDED && p.mode != MODE_A1;
    const int64_t places = max64(tile_places(p.tokens, p.sequences, 1, 32),
                                 classes ? tile_places(p.tokens, p.sequences, p.l, 32) : 0);
    return places * p.heads < (int64_t)1 << 31;
}

hipError_t packed_launch(const PackedCall& p, hipStream_t stream) {
    PackedArgs a{};
    a.starts = p.starts;
    a.sequences = p.sequences;
    a.tokens = (int32_t)p.tokens;
    a.qt = p.qt, a.qh = p.qh, a.kt = p.kt, a.kh = p.kh, a.vt = p.vt, a.vh = p.vh, a.ot = p.ot, a.oh = p.oh;
    a.group = p.heads / p.kv_heads;
    a.head_step = 1;
    a.run_heads = p.heads;
    a.mode = p.mode;
    a.sub = p.sub;
    a.l = p.l;
    a.c = p.c;
    a.dl = make_divl(p.l);
    a.dc = make_divl(p.c > 0 ? p.c : 1);
    a.step = 1;
    a.state_from = kNoBand;
    a.scale_log2 = p.scale * kLog2eHost;
    a.lse = p.lse;
    a.turn_heads = p.pattern == FIXED && p.mode == MODE_INTERLEAVED;
    if (p.pattern == FIXED) return run_d<true>(a, p, stream);

    PackedArgs band = a, cls = a;
    band.band = p.l >= p.tokens ? kNoBand : p.l;
    cls.band = kNoBand;
    cls.step = p.l;
    if (p.mode == MODE_A1) return run_d<false>(band, p, stream);
    if (p.mode == MODE_A2) return run_d<false>(cls, p, stream);
    hipError_t e = hipSuccess;
    if (p.mode == MODE_INTERLEAVED) {  // even heads the band, odd ones the classes
        band.head_step = cls.head_step = 2;
        band.run_heads = (p.heads + 1) / 2;
        cls.head0 = 1;
        cls.run_heads = p.heads / 2;
        e = run_d<false>(band, p, stream);
        if (e == hipSuccess && cls.run_heads > 0) e = run_d<false>(cls, p, stream);
        return e;
    }
    if (has_classes(p.tokens, p.pattern, p.mode, p.l)) {
        cls.shift = 2;
        cls.put_state = true;
        cls.state_o = band.state_o = p.workspace;
        cls.state_ml = band.state_ml = p.workspace + (size_t)p.tokens * p.heads * p.d;
        band.state_from = 2 * p.l;
        e = run_d<false>(cls, p, stream);
        if (e != hipSuccess) return e;
    }
    return run_d<false>(band, p, stream);
}

}  // namespace sa
