// Storing keys and values into an 8-bit cache (sparse_attn_cache8_store).
//
// A block of 2^block_shift tokens of one (batch, head) has one scale 2^e, so the block
// is the unit of work: one workgroup reads the block's new rows once, keeps them in
// registers, takes their largest magnitude, and writes codes and scale.  No other
// workgroup touches that block.  Where it holds earlier tokens and the scale grows,
// the workgroup moves their codes to the new scale as well.  Bound by reading the new
// rows (2 or 4 bytes an element) and writing a byte each.
//
// Magnitudes are compared as integers (two bf16 at a time), and a conversion takes two
// elements with the scale.  Neither knows of infinities and NaN: a workgroup that meets one
// (its largest magnitude says so) goes over its registers again, element by element.
// Doing that for every element cost 15 instructions each and 63.5 us for 252 MB (8 prompts
// of up to 12,288 tokens, 8 heads of 64), as it is 43.4, 5.8 TB/s.
#include "sa_e4m3.h"
#include "sa_internal.h"
#include "sa_mfma.h"

namespace sa {

namespace {

// Up to here K and V of a block go to workgroups of their own, as a call of few blocks is bound by the
// latency of one (one token, 32 sequences, 8 heads: 3.6 -> 3.2 us; 1,501 tokens, 2 x 4 heads of 128, fp32, 104 blocks:
// 6.9 -> 5.1).  From there on one workgroup writes both, so that where they interleave a line's two halves
// meet in one L2 (520 blocks: the same; 776 of d = 128 15.8 -> 15.1; 49,216 of 16 tokens 69.0 -> 56.5).
constexpr int64_t kFewGroups = 512;

struct StoreArgs {
    Cache8 c;
    int32_t kv_heads, n_new, reach;  // reach: blocks that the new tokens of a sequence can lie in
    int32_t row_shift;               // log2 of the pieces of a row
    int64_t xb, xh, xs;              // element strides of k and v
    const int32_t* start;
    const int32_t* counts;
};

// The 16 bytes of k or v that a lane takes at a time, as loaded: words of two bf16, or floats.
template <typename T>
struct Piece {
    static constexpr int kElements = 16 / sizeof(T);
    typedef typename std::conditional<sizeof(T) == 2, u32x2, uint32_t>::type Codes;
    u32x4 u;
    // read once: marked so, a prompt's rows do not displace the cache's lines (50.9 -> 43.4 us for 252 MB)
    __device__ void load(const T* p) { u = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
    __device__ uint32_t bits(int e) const {  // element e as a float's
        if constexpr (sizeof(T) == 4) return u[e];
        else return e % 2 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16;
    }
    __device__ Codes encode(float scale) const {
        if constexpr (sizeof(T) == 4) return encode_word(u[0], u[1], u[2], u[3], scale);
        else return u32x2{encode_word(u[0], u[1], scale), encode_word(u[2], u[3], scale)};
    }
};

// Code e of a lane's codes set to NaN; codes moved to a scale 1 / factor as large.
__device__ inline uint32_t nan_code(uint32_t c, int e) { return (c & ~(0xffu << 8 * e)) | 0x7fu << 8 * e; }
__device__ inline void set_nan(uint32_t& c, int e) { c = nan_code(c, e); }
__device__ inline void set_nan(u32x2& c, int e) { c[e / 4] = nan_code(c[e / 4], e % 4); }
__device__ inline uint32_t rescaled(uint32_t c, float factor) {
    float y[4];
    decode4(c, y);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] *= factor;
    return encode4(y);
}
__device__ inline u32x2 rescaled(u32x2 c, float factor) { return u32x2{rescaled(c[0], factor), rescaled(c[1], factor)}; }

__device__ inline bool finite_bits(uint32_t x) { return (x & 0x7fffffffu) < 0x7f800000u; }

// Largest magnitudes so far, as a running word that `largest` turns into a float's bits.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ inline void grow(uint32_t& top, const Piece<uint16_t>& x) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                                      __builtin_bit_cast(u16x2, x.u[i] & 0x7fff7fffu)));
}
__device__ inline void grow(uint32_t& top, const Piece<float>& x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, x.u[i] & 0x7fffffffu);
}
__device__ inline uint32_t largest(uint32_t top, const uint16_t*) { return max(top << 16, top & 0xffff0000u); }
__device__ inline uint32_t largest(uint32_t top, const float*) { return top; }

// The largest over the workgroup.
template <int NT>
__device__ inline uint32_t group_max(uint32_t x, uint32_t* s) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, off));
    if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) x = max(x, s[w]);
    return x;
}

// NT threads, CH pieces each: NT * CH = the pieces of a block.  TENSORS: 2, or 1 with blockIdx.y for which.
template <typename T, int NT, int CH, int TENSORS>
__global__ void __launch_bounds__(NT)
store_kernel(StoreArgs a, const T* __restrict__ k, const T* __restrict__ v) {
    constexpr int E = Piece<T>::kElements;
    typedef typename Piece<T>::Codes Codes;
    __shared__ uint32_t s_max[2 * TENSORS][NT / 64], s_old[TENSORS];
    const int tid = threadIdx.x;
    const uint32_t id = blockIdx.x, row = id / (uint32_t)a.reach;
    const int r = (int)(id - row * (uint32_t)a.reach);
    const int64_t b = row / (uint32_t)a.kv_heads, h = row % (uint32_t)a.kv_heads;
    const int64_t start = a.start ? a.start[b] : 0;
    int64_t count = a.counts ? a.counts[b] : a.n_new;
    count = count < 0 ? 0 : (count > a.n_new ? a.n_new : count);
    const int64_t end = start + count < a.c.capacity ? start + count : a.c.capacity;
    const int64_t blk = (start >> a.c.block_shift) + r, first = blk << a.c.block_shift;
    if (start < 0 || first >= end || start >= end) return;  // the same for the whole workgroup

    // rows of the block as numbers from its first: new ones are lo .. hi - 1
    const int lo = (int)max64(start - first, 0), hi = (int)min64(end - first, (int64_t)1 << a.c.block_shift);
    // of the block's first row (in front of k where lo > 0: never read)
    const int64_t from = b * a.xb + h * a.xh + (first - start) * a.xs;
    const int mask = (1 << a.row_shift) - 1;
    Piece<T> x[TENSORS][CH];
    auto is_v = [](int t) { return TENSORS == 1 ? blockIdx.y == 1 : t == 1; };
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int piece = i * NT + tid, at = piece >> a.row_shift;
        const int64_t off = from + at * a.xs + (piece & mask) * E;
#pragma unroll
        for (int t = 0; t < TENSORS; ++t) {
            if (at >= lo && at < hi) x[t][i].load((is_v(t) ? v : k) + off);
            else x[t][i].u = u32x4{0, 0, 0, 0};
        }
    }
    const int64_t at_scale = (int64_t)row * a.c.blocks + blk;
    if (tid < TENSORS) s_old[tid] = lo > 0 ? __float_as_uint((is_v(tid) ? a.c.vs : a.c.ks)[at_scale]) : 0u;
    uint32_t top[TENSORS];
#pragma unroll
    for (int t = 0; t < TENSORS; ++t) {
        top[t] = 0;
#pragma unroll
        for (int i = 0; i < CH; ++i) grow(top[t], x[t][i]);
        top[t] = group_max<NT>(largest(top[t], k), s_max[t]);
    }
#pragma unroll
    for (int t = 0; t < TENSORS; ++t) {
        const bool fine = finite_bits(top[t]);
        if (!fine) {  // (the same for the whole workgroup) an infinity or a NaN: the largest of the others
            top[t] = 0;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t m = x[t][i].bits(e) & 0x7fffffffu;
                    if (finite_bits(m)) top[t] = max(top[t], m);
                }
            top[t] = group_max<NT>(top[t], s_max[TENSORS + t]);
        }
        int e_new = scale_exponent(top[t]);
        int growth = 0;  // of the scale of earlier tokens
        if (lo > 0) {
            const int e_old = exponent_of(s_old[t]);
            if (e_old > e_new) e_new = e_old;
            growth = e_new - e_old;
        }
        const float unit = __uint_as_float(power_bits(e_new));
        uint8_t* codes = (is_v(t) ? a.c.v : a.c.k) + b * a.c.sb + h * a.c.sh + first * a.c.ss;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int piece = i * NT + tid, at = piece >> a.row_shift;
            Codes* dst = reinterpret_cast<Codes*>(codes + at * a.c.ss + (piece & mask) * E);
            if (at >= lo && at < hi) {
                Codes u = x[t][i].encode(unit);
                if (!fine) {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (!finite_bits(x[t][i].bits(e))) set_nan(u, e);
                }
                *dst = u;
            } else if (at < lo && growth > 0) {
                *dst = rescaled(*dst, __uint_as_float(power_bits(growth < 126 ? -growth : -126)));
            }
        }
        if (tid == 0) (is_v(t) ? a.c.vs : a.c.ks)[at_scale] = unit;
    }
}

template <typename T, int NT, int CH>
hipError_t launch(const StoreArgs& a, int64_t groups, const void* k, const void* v, hipStream_t stream) {
    const T *kt = (const T*)k, *vt = (const T*)v;
    // (1,024 threads with both would have a compute unit to themselves: 8 x 3,000 tokens, 8 heads of 128, fp32, blocks
    // of 128 59.8 us, apart 47.6)
    if constexpr (NT < 1024) {
        if (groups >= kFewGroups) {
            hipLaunchKernelGGL((store_kernel<T, NT, CH, 2>), dim3((unsigned)groups), dim3(NT), 0, stream, a, kt, vt);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((store_kernel<T, NT, CH, 1>), dim3((unsigned)groups, 2), dim3(NT), 0, stream, a, kt, vt);
    return hipGetLastError();
}

// A block is 64 to 2,048 pieces of bf16, 128 to 4,096 of fp32: one a thread up to 256 threads, then up
// to 4 (32 registers for k and v).
template <typename T>
hipError_t launch_pieces(const StoreArgs& a, int64_t groups, int pieces, const void* k, const void* v,
                         hipStream_t stream) {
    if constexpr (sizeof(T) == 2)
        if (pieces == 64) return launch<T, 64, 1>(a, groups, k, v, stream);
    if constexpr (sizeof(T) == 4)
        if (pieces == 4096) return launch<T, 1024, 4>(a, groups, k, v, stream);
    switch (pieces) {
    case 128: return launch<T, 128, 1>(a, groups, k, v, stream);
    case 256: return launch<T, 256, 1>(a, groups, k, v, stream);
    case 512: return launch<T, 256, 2>(a, groups, k, v, stream);
    case 1024: return launch<T, 256, 4>(a, groups, k, v, stream);
    default: return launch<T, 512, 4>(a, groups, k, v, stream);
    }
}

}  // namespace

hipError_t cache8_store_launch(const Cache8& cache, int batch, int kv_heads, int64_t n_new, int d, int dtype,
                               const void* k, const void* v, const int64_t* kv_strides, const int32_t* start,
                               const int32_t* counts, hipStream_t stream) {
    StoreArgs a;
    a.c = cache;
    a.kv_heads = kv_heads;
    a.n_new = (int32_t)n_new;
    const int64_t T = (int64_t)1 << cache.block_shift;
    a.reach = (int32_t)((n_new + T - 2) / T + 1);
    const int elements = dtype == 1 ? Piece<uint16_t>::kElements : Piece<float>::kElements;
    a.row_shift = __builtin_ctz((unsigned)(d / elements));
    a.xb = kv_strides[0];
    a.xh = kv_strides[1];
    a.xs = kv_strides[2];
    a.start = start;
    a.counts = counts;
    const int64_t groups = (int64_t)a.reach * kv_heads * batch;
    const int pieces = (int)(T * d / elements);
    return dtype == 1 ? launch_pieces<uint16_t>(a, groups, pieces, k, v, stream)
                      : launch_pieces<float>(a, groups, pieces, k, v, stream);
}

}  // namespace sa
