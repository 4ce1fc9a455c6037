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
// What bounds it: long walks the matrix products and the exponentials beside them, short ones
// (a prompt of hundreds of tokens) the steps' latency.
#include "sa_finite.h"
#include "sa_internal.h"
#include "sa_mask.h"
#include "sa_mfma.h"
#include "sa_step.h"
#include "sa_tile.h"

namespace sa {

namespace {

constexpr int kPackedWaves = 4, kPackedThreads = 64 * kPackedWaves;
constexpr int kNoBand = 0x7fffffff;

struct PackedArgs {
    const int32_t* starts;
    int32_t sequences, tokens;
    int64_t qt, qh, kt, kh, vt, vh, ot, oh;
    int32_t heads, group;              // query heads; of one key head
    int32_t head0, head_step, run_heads;  // heads of this launch: head0, head0 + head_step, ...
    int32_t mode, sub, l, c;
    DivL dl, dc;
    int32_t step;                      // rows from one of a tile to the next: 1, or l for residue classes
    int32_t band;                      // strided: furthest key behind a row (kNoBand: none)
    int32_t shift;                     // strided: nearest one
    bool by_rows;                      // classes: one place a row of the batch, live where a tile begins
    int64_t places;                    // tile places of one head
    float scale, scale_log2;
    float *state_o, *state_ml;         // states of the classes, [heads, tokens, d] and [heads, tokens, 2]
    bool put_state;                    // write them, in place of o and lse
    int32_t state_from;                // rows from here on have one to go on from (0x7fffffff: none)
    float* lse;
};

// Tile of a place: rows i0, i0 + 1, ... (counted in steps) below n of the sequence (or class) whose first
// row is `base`.
struct TilePlace {
    int32_t base, n, i0;
    int32_t offset;  // of the first row in its sequence
};

// Every wave finds its sequence by itself: 64 candidates a round, all loads of a round at once.
__device__ inline int sequence_of(const PackedArgs& a, int rows, int64_t place, int lane) {
    int found = 0;
    for (int s0 = 0; s0 < a.sequences; s0 += 64) {
        const int s = s0 + lane;
        bool below = false;
        if (s < a.sequences) {
            const int32_t start = max(0, min(a.starts[s], a.tokens));
            below = a.by_rows ? start <= place : (int64_t)(start / rows) + s <= place;
        }
        const uint64_t m = __builtin_amdgcn_ballot_w64(below);
        found += __builtin_popcountll(m);
        if (~m) break;
    }
    return found - 1;  // (the first sequence's places begin at its start; found = 0 lies before it)
}

template <int ROWS>
__device__ inline TilePlace tile_place(const PackedArgs& a, int64_t place, int lane) {
    int32_t cls = 0;
    const int64_t rows = (int64_t)ROWS * a.step;
    if (a.step > 1 && !a.by_rows) {
        const int64_t block = place / a.l;
        cls = (int32_t)(place - block * a.l);
        place = block;
    }
    const int32_t per = (int32_t)min64(rows, 0x7fffffff);
    const int s = __builtin_amdgcn_readfirstlane(sequence_of(a, per, place, lane));
    if (s < 0) return {0, 0, 0, 0};
    const int32_t start = __builtin_amdgcn_readfirstlane(max(0, min(a.starts[s], a.tokens)));
    const int32_t end = __builtin_amdgcn_readfirstlane(max(0, min(a.starts[s + 1], a.tokens)));
    const int32_t n = end - start;
    int64_t tile;
    if (a.by_rows) {
        const int64_t i = place - start;
        if (i >= n) return {0, 0, 0, 0};
        const int32_t m = div_l(a.dl, (int32_t)i);
        if (m % ROWS != 0) return {0, 0, 0, 0};
        cls = (int32_t)i - m * a.l;
        tile = m / ROWS;
    } else {
        tile = place - ((int64_t)(start / per) + s);
    }
    if (n <= cls || tile < 0) return {0, 0, 0, 0};
    const int32_t rows_here = a.step == 1 ? n : div_l(a.dl, n - 1 - cls) + 1;
    const int64_t i0 = tile * ROWS;
    if (i0 >= rows_here) return {0, 0, 0, 0};
    return {start + cls, rows_here, (int32_t)i0, cls};
}

// Consecutive workgroups go to the 8 XCDs in turn: with heads in eighths, an XCD takes neighbouring heads, which
// share key heads, and their keys stay in its L2.  Places from the last one down: a sequence's longest walks first.
__device__ inline void place_of(const PackedArgs& a, int64_t id, int64_t* place, int* head) {
    int h;
    int64_t p;
    if (a.run_heads % 8 == 0) {
        const int each = a.run_heads / 8;
        const int64_t s = id / 8;
        p = s / each;
        h = (int)(id % 8) * each + (int)(s - p * each);
    } else {
        p = id / a.run_heads;
        h = (int)(id - p * a.run_heads);
    }
    *place = a.places - 1 - p;
    *head = a.head0 + h * a.head_step;
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
// bf16
// ---------------------------------------------------------------------------
// acc += the products of one chunk (operands a, b, see pack_bf16x8) with this lane's row, which attends the
// rows of the chunk whose bit is set: where a value is an infinity or a NaN, 0 times it would not be 0.
template <int DB>
__device__ inline void accumulate_bits(const bf16x8* a, bf16x8 b, uint32_t bits, int g, f32x4* acc) {
    const u32x4 bw = __builtin_bit_cast(u32x4, b);
#pragma unroll 1
    for (int x = 0; x < 32; ++x) {  // one row at a time
        const int e = (x >> 4) * 4 + (x & 3);
        u32x4 keep;
#pragma unroll
        for (int y = 0; y < 4; ++y)
            keep[y] = g == ((x >> 2) & 3) && y == (e >> 1) ? ((e & 1) ? 0xFFFF0000u : 0xFFFFu) : 0u;
        const bf16x8 bx = __builtin_bit_cast(bf16x8, bw & keep);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const bf16x8 ax = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, a[db]) & keep);
            const f32x4 sum = mfma_16x16x32(ax, bx, acc[db]);
            if ((bits >> x) & 1u) acc[db] = sum;
            __builtin_amdgcn_sched_barrier(0);  // one sum in flight: registers
        }
    }
}

template <int D, bool WIDE>
struct PackedCfg {
    static constexpr int QBW = WIDE ? 2 : 1;         // 16-row blocks of a wave
    static constexpr int RW = 16 * QBW;              // rows of a wave
    static constexpr int ROWS = RW * kPackedWaves;   // rows of a tile
    static constexpr int KS = D / 32, DB = D / 16;
    static constexpr int KB = 4, KC = 2;             // 16-key blocks and 32-key chunks of a step
    static constexpr int EU = D == 128 ? 2 : 3;      // waves per SIMD
};

template <int D, bool WIDE, bool FIXED_>
__global__ void __launch_bounds__(kPackedThreads) __attribute__((amdgpu_waves_per_eu(PackedCfg<D, WIDE>::EU)))
packed_bf16_kernel(PackedArgs a, const uint16_t* __restrict__ q, const uint16_t* __restrict__ k,
                   const uint16_t* __restrict__ v, uint16_t* __restrict__ o) {
    using C = PackedCfg<D, WIDE>;
    constexpr int KEYS = 64;
    __shared__ __attribute__((aligned(16))) uint16_t sK[2][KEYS * D];
    __shared__ __attribute__((aligned(16))) uint16_t sV[2][KEYS * D];
    constexpr uint32_t kTileBytes = KEYS * D * 2;
    const uint32_t sK_base = lds_addr(&sK[0][0]), sV_base = lds_addr(&sV[0][0]);
    const int tid = threadIdx.x, lane = tid % 64, g = lane / 16, r = lane % 16;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64);
    TileReader<D> rd;
    rd.init(g, r);
    const float c2 = a.scale_log2;

    for (int64_t id = blockIdx.x; id < a.places * a.run_heads; id += gridDim.x) {
        int64_t place;
        int h;
        place_of(a, id, &place, &h);
        const TilePlace t = tile_place<C::ROWS>(a, place, lane);
        if (t.n == 0) continue;  // the same for the whole workgroup
        const int part = FIXED_ ? part_of_head(a.mode, h) : PART_A1;
        const int32_t win = FIXED_ ? (int32_t)summary_start(a.l, a.c, subblock_of_head(a.sub, h)) : 0;
        const Walk walk = tile_walk<FIXED_, C::ROWS, KEYS>(a, part, win, t);
        if (a.put_state && walk.steps == 0) continue;
        MaskParams mp{FIXED, part, a.l, a.c, 0, 0, 0, win};
        if (FIXED_ && part == PART_MERGED && a.l <= 64) summary_words(a.l, a.c, win, &mp.sum_lo, &mp.sum_hi);
        const int row0 = t.i0 + w * C::RW;  // first row of this wave
        const Row head_row = packed_row<FIXED_>(a, part, win, walk, min(row0, t.n - 1)),
                  tail_row = packed_row<FIXED_>(a, part, win, walk, min(row0 + C::RW, t.n) - 1);
        const uint16_t* kh = k + (int64_t)(h / a.group) * a.kh + (int64_t)t.base * a.kt;
        const uint16_t* vh = v + (int64_t)(h / a.group) * a.vh + (int64_t)t.base * a.vt;
        const int64_t ks = a.kt * a.step, vs = a.vt * a.step;

        bf16x8 qf[C::QBW][C::KS];
        f32x4 oacc[C::QBW][C::DB];
        float m_run[C::QBW], l_run[C::QBW];
        Row rows[C::QBW];
#pragma unroll
        for (int u = 0; u < C::QBW; ++u) {
            rows[u] = packed_row<FIXED_>(a, part, win, walk, min(row0 + 16 * u + r, t.n - 1));
            const uint16_t* p = q + (t.base + (int64_t)rows[u].i * a.step) * a.qt + h * a.qh;
#pragma unroll
            for (int x = 0; x < C::KS; ++x) qf[u][x] = ld_bf16x8(p + 32 * x + 8 * g);
        }
        // the state that the rows begin with: nothing, or what the classes left
        auto begin = [&] {
#pragma unroll
            for (int u = 0; u < C::QBW; ++u) {
                m_run[u] = -INFINITY;
                l_run[u] = 0.f;
#pragma unroll
                for (int db = 0; db < C::DB; ++db) oacc[u][db] = zero4();
                if (!FIXED_ && rows[u].i >= a.state_from) {
                    const int64_t at = (int64_t)h * a.tokens + t.base + rows[u].i;
                    m_run[u] = a.state_ml[2 * at];
                    l_run[u] = g == 0 ? a.state_ml[2 * at + 1] : 0.f;
#pragma unroll
                    for (int db = 0; db < C::DB; ++db)
                        oacc[u][db] = *reinterpret_cast<const f32x4*>(a.state_o + at * D + 16 * db + 4 * g);
                }
            }
        };
        // one step's K and V rows to a ring stage: lane L of window `win` fetches the chunk that belongs at its slot
        constexpr int PER = KEYS * D / 512 / kPackedWaves;  // 1 KiB windows of a wave and tile
        auto load_step = [&](int e, int stage) {
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int window = w + kPackedWaves * x, oe = 512 * window + 8 * lane;
                const int at = oe / D, chunk = ((oe % D) / 8) ^ Swz<D>::perm(at);
                const int64_t j = key_row<FIXED_, KEYS>(a, win, walk, e, at);
                dma_b128_at(kh + j * ks + 8 * chunk, sK_base + stage * kTileBytes + 1024 * window);
                dma_b128_at(vh + j * vs + 8 * chunk, sV_base + stage * kTileBytes + 1024 * window);
            }
        };

        bool careful = false;
        while (true) {
            begin();
            // (no load that the compiler tracks is left inside the loop: a wait for one would drain the ring)
            wait_loads_upto<0>();
            if (walk.steps > 0) load_step(0, 0);
            int e = 0;
            two_stage_while([&](auto stage) {
                constexpr int st = decltype(stage)::value;
                if (e >= walk.steps) return false;
                wait_loads_upto<0>();
                __syncthreads();  // this step is in LDS everywhere; the other stage is free
                if (e + 1 < walk.steps) load_step(e + 1, st ^ 1);
                const uint16_t* tK = sK[st];
                const uint16_t* tV = sV[st];
                auto compute = [&](auto full) {
                    uint64_t bits[C::QBW];
                    int cls[C::QBW][C::KC];
#pragma unroll
                    for (int u = 0; u < C::QBW; ++u) {
                        bits[u] = ~0ull;
#pragma unroll
                        for (int kc = 0; kc < C::KC; ++kc) cls[u][kc] = CHUNK_ALL;
                    }
                    if constexpr (!decltype(full)::value) {
                        const int32_t j0 = walk.lo + KEYS * (e - walk.far_steps);
                        uint64_t sum = 0;
                        if (FIXED_ && part == PART_MERGED && e >= walk.far_steps) sum = summary_bits(mp, mod_l(a.dl, j0));
#pragma unroll
                        for (int u = 0; u < C::QBW; ++u) {
                            bits[u] = row_bits<FIXED_, KEYS>(a, part, walk, rows[u], e, sum);
#pragma unroll
                            for (int kc = 0; kc < C::KC; ++kc)
                                cls[u][kc] = chunk_class(chunk_bits(bits[u] >> (4 * g), kc, true), true);
                        }
                    }
                    bool live[C::KC];
#pragma unroll
                    for (int kc = 0; kc < C::KC; ++kc) {
                        live[kc] = false;
#pragma unroll
                        for (int u = 0; u < C::QBW; ++u) live[kc] = live[kc] || cls[u][kc] != CHUNK_NONE;
                    }
                    // V^T operands, read now: their latency hides behind the products and the softmax
                    bf16x8 vt[C::KC][C::DB];
#pragma unroll
                    for (int kc = 0; kc < C::KC; ++kc) {
                        if (!live[kc]) continue;
#pragma unroll
                        for (int db = 0; db < C::DB; ++db) vt[kc][db] = rd.tr(tV, kc * 32, kc * 32 + 16, db);
                    }
                    __builtin_amdgcn_s_setprio(1);
                    f32x4 s[C::QBW][C::KB];
#pragma unroll
                    for (int kb = 0; kb < C::KB; ++kb) {
#pragma unroll
                        for (int u = 0; u < C::QBW; ++u) s[u][kb] = zero4();
                        if (!live[kb / 2]) continue;
                        bf16x8 kf[C::KS];
#pragma unroll
                        for (int x = 0; x < C::KS; ++x) kf[x] = rd.row(tK, kb * 16, x);
#pragma unroll
                        for (int u = 0; u < C::QBW; ++u) {
                            if (cls[u][kb / 2] == CHUNK_NONE) continue;
#pragma unroll
                            for (int x = 0; x < C::KS; ++x) s[u][kb] = mfma_16x16x32(kf[x], qf[u][x], s[u][kb]);
                        }
                    }
                    __builtin_amdgcn_s_setprio(0);
#pragma unroll
                    for (int u = 0; u < C::QBW; ++u) {
                        float mloc = -INFINITY;
#pragma unroll
                        for (int kc = 0; kc < C::KC; ++kc) {
                            if (cls[u][kc] == CHUNK_NONE) continue;
                            if (cls[u][kc] == CHUNK_PART) {
#pragma unroll
                                for (int hk = 0; hk < 2; ++hk)
#pragma unroll
                                    for (int y = 0; y < 4; ++y)
                                        s[u][2 * kc + hk][y] = select_or_neg_inf(
                                            bit_lane_mask(bits[u] >> (4 * g), 16 * (2 * kc + hk) + y), s[u][2 * kc + hk][y]);
                            }
#pragma unroll
                            for (int hk = 0; hk < 2; ++hk) {
                                const f32x4 x = s[u][2 * kc + hk];
                                mloc = fmaxf(fmaxf(mloc, x[0]), x[1]);
                                mloc = fmaxf(fmaxf(mloc, x[2]), x[3]);
                            }
                        }
                        mloc = max_over_g(mloc);
                        const float m_new = fmaxf(m_run[u], mloc);
                        // rows with nothing attended so far keep m = -inf; 0 as reference gives p = 0
                        const float m_ref = m_new == -INFINITY ? 0.f : m_new;
                        const float neg = -m_ref * c2;
                        float psum = 0.f;
                        bf16x8 pf[C::KC];
#pragma unroll
                        for (int kc = 0; kc < C::KC; ++kc) {
                            if (cls[u][kc] != CHUNK_NONE) {
#pragma unroll
                                for (int hk = 0; hk < 2; ++hk)
#pragma unroll
                                    for (int y = 0; y < 4; ++y) {
                                        const float p = exp2_fast(fmaf(s[u][2 * kc + hk][y], c2, neg));
                                        s[u][2 * kc + hk][y] = p;
                                        psum += p;
                                    }
                            }
                            // weights rounded to bf16 for the matrix product, 2^-9 of each; the sum takes them whole
                            pf[kc] = pack_bf16x8(s[u][2 * kc], s[u][2 * kc + 1]);
                        }
                        const float alpha = exp2_fast((m_run[u] - m_ref) * c2);
                        l_run[u] = fmaf(l_run[u], alpha, psum);
                        m_run[u] = m_new;
#pragma unroll
                        for (int db = 0; db < C::DB; ++db) oacc[u][db] *= alpha;
#pragma unroll
                        for (int kc = 0; kc < C::KC; ++kc) {
                            if (cls[u][kc] == CHUNK_NONE) continue;
                            if (!decltype(full)::value && careful && cls[u][kc] == CHUNK_PART) {
                                accumulate_bits<C::DB>(vt[kc], pf[kc], (uint32_t)(bits[u] >> (32 * kc)), g, oacc[u]);
                                continue;
                            }
#pragma unroll
                            for (int db = 0; db < C::DB; ++db) oacc[u][db] = mfma_16x16x32(vt[kc][db], pf[kc], oacc[u][db]);
                        }
                    }
                };
                if (step_full<FIXED_, KEYS>(a, part, walk, e, head_row, tail_row)) compute(std::true_type{});
                else compute(std::false_type{});
                ++e;
                return true;
            });
            // an infinity or a NaN in a key that a row does not attend must not reach it: such sums are formed
            // a second time, with the products of partly attended chunks kept apart by row
            bool bad = false;
#pragma unroll
            for (int u = 0; u < C::QBW; ++u) bad = bad || non_finite<C::DB>(oacc[u]);
            if (!__syncthreads_or(bad) || careful) break;
            careful = true;
        }

#pragma unroll
        for (int u = 0; u < C::QBW; ++u) {
            const float l_tot = sum_over_g(l_run[u]);
            if (row0 + 16 * u + r >= t.n) continue;
            const int64_t token = t.base + (int64_t)rows[u].i * a.step, at = (int64_t)h * a.tokens + token;
            if (a.put_state) {
                if (rows[u].i < a.shift) continue;  // no key: the band begins with nothing there
#pragma unroll
                for (int db = 0; db < C::DB; ++db)
                    *reinterpret_cast<f32x4*>(a.state_o + at * D + 16 * db + 4 * g) = oacc[u][db];
                if (g == 0) {
                    a.state_ml[2 * at] = m_run[u];
                    a.state_ml[2 * at + 1] = l_tot;
                }
                continue;
            }
            const bool none = no_key(l_tot);
            const float inv = none ? 0.f : 1.f / l_tot;
            uint16_t* orow = o + token * a.ot + h * a.oh;
#pragma unroll
            for (int db = 0; db < C::DB; ++db)
                *reinterpret_cast<uint2*>(orow + db * 16 + 4 * g) = pack_bf16x4_bits(oacc[u][db] * inv);
            if (g == 0) a.lse[at] = none ? -INFINITY : (m_run[u] * c2 + __log2f(l_tot)) / kLog2e;
        }
    }
}

// ---------------------------------------------------------------------------
// fp32: four waves of 16 rows, 32 keys a step, 16x16x4 products (see sa_f32.hip for their operands)
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

template <int D, bool FIXED_>
__global__ void __launch_bounds__(kPackedThreads) __attribute__((amdgpu_waves_per_eu(2)))
packed_f32_kernel(PackedArgs a, const float* __restrict__ q, const float* __restrict__ k, const float* __restrict__ v,
                  float* __restrict__ o) {
    constexpr int KEYS = 32, ROWS = 16 * kPackedWaves, DB = D / 16;
    constexpr int V = D >= 64 ? 4 : 2, HB = D / (16 * V);  // neighbours in d per read of V, reads per row
    typedef float vec __attribute__((ext_vector_type(V)));
    __shared__ __attribute__((aligned(16))) float sK[2][KEYS * D];
    __shared__ __attribute__((aligned(16))) float sV[2][KEYS * D];
    constexpr uint32_t kTileBytes = KEYS * D * 4;
    const uint32_t sK_base = lds_addr(&sK[0][0]), sV_base = lds_addr(&sV[0][0]);
    const int tid = threadIdx.x, lane = tid % 64, g = lane / 16, r = lane % 16;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64);
    const float c2 = a.scale_log2;

    for (int64_t id = blockIdx.x; id < a.places * a.run_heads; id += gridDim.x) {
        int64_t place;
        int h;
        place_of(a, id, &place, &h);
        const TilePlace t = tile_place<ROWS>(a, place, lane);
        if (t.n == 0) continue;
        const int part = FIXED_ ? part_of_head(a.mode, h) : PART_A1;
        const int32_t win = FIXED_ ? (int32_t)summary_start(a.l, a.c, subblock_of_head(a.sub, h)) : 0;
        const Walk walk = tile_walk<FIXED_, ROWS, KEYS>(a, part, win, t);
        if (a.put_state && walk.steps == 0) continue;
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
        {
            const float* p = q + token * a.qt + h * a.qh;
#pragma unroll
            for (int x = 0; x < DB; ++x) qf[x] = *reinterpret_cast<const f32x4*>(p + 16 * x + 4 * g);
        }
        // acc[V hb + e][i] is element 16 V hb + V (4 g + i) + e
        auto begin = [&] {
            m_run = -INFINITY;
            l_run = 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = zero4();
            if (!FIXED_ && row.i >= a.state_from) {
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
        constexpr int PER = KEYS * D / 256 / kPackedWaves;
        auto load_step = [&](int e, int stage) {
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int window = w + kPackedWaves * x, oe = 256 * window + 4 * lane;
                const int at = oe / D, piece = swz32<D>(at, (oe % D) / 4);
                const int64_t j = key_row<FIXED_, KEYS>(a, win, walk, e, at);
                dma_b128_at(kh + j * ks + 4 * piece, sK_base + stage * kTileBytes + 1024 * window);
                dma_b128_at(vh + j * vs + 4 * piece, sV_base + stage * kTileBytes + 1024 * window);
            }
        };

        bool careful = false;
        while (true) {
            begin();
            wait_loads_upto<0>();
            if (walk.steps > 0) load_step(0, 0);
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
                if (__builtin_amdgcn_ballot_w64(bits != 0u) != 0ull) {
                    f32x4 s[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {  // key 16 y + 4 g + i
                        f32x4 c0 = zero4(), c1 = zero4();
#pragma unroll
                        for (int x = 0; x < DB; ++x) {
                            const f32x4 kf =
                                *reinterpret_cast<const f32x4*>(tK + (16 * y + r) * D + 4 * swz32<D>(16 * y + r, 4 * x + g));
                            c0 = mfma_f32(kf[0], qf[x][0], c0);
                            c1 = mfma_f32(kf[1], qf[x][1], c1);
                            c0 = mfma_f32(kf[2], qf[x][2], c0);
                            c1 = mfma_f32(kf[3], qf[x][3], c1);
                        }
                        s[y] = c0 + c1;
                    }
                    float mx = m_run;
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            s[y][i] = select_or_neg_inf(bit_lane_mask(bits >> (4 * g), 16 * y + i), s[y][i]);
                            mx = fmaxf(mx, s[y][i]);
                        }
                    mx = max_over_g(mx);
                    const float m_ref = mx == -INFINITY ? 0.f : mx;
                    const float alpha = exp2_fast((m_run - m_ref) * c2);
                    float psum = 0.f;
                    // (the difference first: scaling before would lose 2^-24 of the scores themselves)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            s[y][i] = exp2_fast((s[y][i] - m_ref) * c2);
                            psum += s[y][i];
                        }
                    l_run = fmaf(l_run, alpha, psum);
                    m_run = mx;
#pragma unroll
                    for (int db = 0; db < DB; ++db) acc[db] *= alpha;
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = 16 * y + 4 * g + i;
#pragma unroll
                            for (int hb = 0; hb < HB; ++hb) {
                                const int col = 16 * V * hb + V * r;
                                const vec x = *reinterpret_cast<const vec*>(tV + key * D + 4 * swz32<D>(key, col / 4) + col % 4);
                                if (careful) {  // one key at a time, for the rows that attend it
#pragma unroll 1
                                    for (int gk = 0; gk < 4; ++gk) {
                                        const bool on = (bits >> (16 * y + 4 * gk + i)) & 1u;
#pragma unroll
                                        for (int e = 0; e < V; ++e) {
                                            const f32x4 sum =
                                                mfma_f32(g == gk ? x[e] : 0.f, g == gk ? s[y][i] : 0.f, acc[V * hb + e]);
                                            if (on) acc[V * hb + e] = sum;
                                        }
                                    }
                                } else {
#pragma unroll
                                    for (int e = 0; e < V; ++e) acc[V * hb + e] = mfma_f32(x[e], s[y][i], acc[V * hb + e]);
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

        const float l_tot = sum_over_g(l_run);
        if (row0 + r >= t.n) continue;
        const bool none = no_key(l_tot);
        const float inv = a.put_state ? 1.f : none ? 0.f : 1.f / l_tot;
        if (a.put_state && row.i < a.shift) continue;
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
        if (g != 0) continue;
        if (a.put_state) {
            a.state_ml[2 * at_row] = m_run;
            a.state_ml[2 * at_row + 1] = l_tot;
        } else {
            a.lse[at_row] = none ? -INFINITY : (m_run * c2 + __log2f(l_tot)) / kLog2e;
        }
    }
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------
constexpr int64_t kMaxGrid = 1 << 20;      // workgroups; each takes every kMaxGrid-th place
constexpr int64_t kWidePlaces = 1024;      // tiles of 128 rows from so many workgroups on

int64_t tile_places(const PackedArgs& a, int rows) {
    if (a.step == 1) return a.tokens / rows + a.sequences;
    const int64_t per = (int64_t)rows * a.step;
    return min64((int64_t)a.step * (a.tokens / min64(per, 0x7fffffff) + a.sequences), a.tokens);
}

template <int D, bool WIDE, bool FIXED_>
hipError_t run_bf16(PackedArgs& a, const PackedCall& p, hipStream_t stream) {
    constexpr int ROWS = PackedCfg<D, WIDE>::ROWS;
    a.places = tile_places(a, ROWS);
    a.by_rows = a.step > 1 && a.places == a.tokens;
    const dim3 grid((unsigned)min64(a.places * a.run_heads, kMaxGrid));
    hipLaunchKernelGGL((packed_bf16_kernel<D, WIDE, FIXED_>), grid, dim3(kPackedThreads), 0, stream, a,
                       (const uint16_t*)p.q, (const uint16_t*)p.k, (const uint16_t*)p.v, (uint16_t*)p.o);
    return hipGetLastError();
}

template <int D, bool FIXED_>
hipError_t run(PackedArgs& a, const PackedCall& p, hipStream_t stream) {
    if (p.dtype == 1) {
        if (tile_places(a, PackedCfg<D, true>::ROWS) * a.run_heads >= kWidePlaces) return run_bf16<D, true, FIXED_>(a, p, stream);
        return run_bf16<D, false, FIXED_>(a, p, stream);
    }
    a.places = tile_places(a, 16 * kPackedWaves);
    a.by_rows = a.step > 1 && a.places == a.tokens;
    const dim3 grid((unsigned)min64(a.places * a.run_heads, kMaxGrid));
    hipLaunchKernelGGL((packed_f32_kernel<D, FIXED_>), grid, dim3(kPackedThreads), 0, stream, a, (const float*)p.q,
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

hipError_t packed_launch(const PackedCall& p, hipStream_t stream) {
    PackedArgs a{};
    a.starts = p.starts;
    a.sequences = p.sequences;
    a.tokens = (int32_t)p.tokens;
    a.qt = p.qt, a.qh = p.qh, a.kt = p.kt, a.kh = p.kh, a.vt = p.vt, a.vh = p.vh, a.ot = p.ot, a.oh = p.oh;
    a.heads = p.heads;
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
    a.scale = p.scale;
    a.scale_log2 = p.scale * kLog2eHost;
    a.lse = p.lse;
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
