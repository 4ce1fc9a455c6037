// Storing keys and values into an 8-bit cache (sparse_attn_cache8_store).
//
// A block of 2^block_shift tokens of one (batch, head) has one scale 2^e, so the block
// is the unit of work: one workgroup reads the block's new rows once, keeps them in
// registers, takes their largest magnitude, and writes codes and scale.  No other
// workgroup touches that block.  Where it holds earlier tokens and the scale grows,
// the workgroup moves their codes to the new scale as well.  Bound by reading the new
// rows (2 or 4 bytes an element) and writing a byte each.
#include "sa_e4m3.h"
#include "sa_internal.h"
#include "sa_mfma.h"

namespace sa {

namespace {

struct StoreArgs {
    Cache8 c;
    int32_t kv_heads, n_new, reach;  // reach: blocks that the new tokens of a sequence can lie in
    int32_t row_shift;               // log2 of the 8-element chunks of a row
    int64_t xb, xh, xs;              // element strides of k and v
    const int32_t* start;
    const int32_t* counts;
};

// Eight elements as the bits of floats.
__device__ inline void load_bits(const uint16_t* p, uint32_t* x) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = u[e] << 16;
        x[2 * e + 1] = u[e] & 0xffff0000u;
    }
}
__device__ inline void load_bits(const float* p, uint32_t* x) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(p), b = *reinterpret_cast<const u32x4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = a[e];
        x[4 + e] = b[e];
    }
}

__device__ inline bool finite_bits(uint32_t x) { return (x & 0x7fffffffu) < 0x7f800000u; }

// NT threads, CH chunks of 8 elements each: NT * CH = the chunks of a block.
template <typename T, int NT, int CH>
__global__ void __launch_bounds__(NT)
store_kernel(StoreArgs a, const T* __restrict__ k, const T* __restrict__ v) {
    __shared__ uint32_t s_max[2][NT / 64];
    const int tid = threadIdx.x;
    int64_t id = blockIdx.x;
    const int r = (int)(id % a.reach);
    id /= a.reach;
    const int h = (int)(id % a.kv_heads);
    const int64_t b = id / a.kv_heads;
    const int64_t start = a.start ? a.start[b] : 0;
    int64_t count = a.counts ? a.counts[b] : a.n_new;
    count = count < 0 ? 0 : (count > a.n_new ? a.n_new : count);
    if (start < 0) return;
    const int64_t end = start + count < a.c.capacity ? start + count : a.c.capacity;
    const int64_t blk = (start >> a.c.block_shift) + r, first = blk << a.c.block_shift;
    if (first >= end || start >= end) return;  // the same for the whole workgroup

    const int64_t base = b * a.xb + h * a.xh - start * a.xs;  // of position 0
    const int64_t head = b * a.kv_heads + h;
    uint32_t x[2][CH][8];
    uint32_t top[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int chunk = i * NT + tid;
        const int64_t pos = first + (chunk >> a.row_shift);
        const int e0 = (chunk & ((1 << a.row_shift) - 1)) * 8;
        const bool fresh = pos >= start && pos < end;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (fresh) {
                load_bits((t ? v : k) + base + pos * a.xs + e0, x[t][i]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[t][i][e] = 0;
            }
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t m = x[t][i][e] & 0x7fffffffu;
                if (finite_bits(m) && m > top[t]) top[t] = m;
            }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t o = (uint32_t)__shfl_xor((int)top[t], off);
            top[t] = o > top[t] ? o : top[t];
        }
        if (tid % 64 == 0) s_max[t][tid / 64] = top[t];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) m = s_max[t][w] > m ? s_max[t][w] : m;
        float* scale = (t ? a.c.vs : a.c.ks) + head * a.c.blocks + blk;
        uint8_t* codes = (t ? a.c.v : a.c.k) + b * a.c.sb + h * a.c.sh;
        int e_new = scale_exponent(m);
        int grow = 0;  // by how much the scale of earlier tokens grows
        if (first < start) {
            const int e_old = exponent_of(__float_as_uint(*scale));
            if (e_old > e_new) e_new = e_old;
            grow = e_new - e_old;
        }
        const float inv = __uint_as_float(power_bits(-e_new));
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int chunk = i * NT + tid;
            const int64_t pos = first + (chunk >> a.row_shift);
            u32x2* dst = reinterpret_cast<u32x2*>(codes + pos * a.c.ss + (chunk & ((1 << a.row_shift) - 1)) * 8);
            if (pos >= start && pos < end) {
                float y[8];
                bool fine = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = __uint_as_float(finite_bits(x[t][i][e]) ? x[t][i][e] : 0u) * inv;
                    fine = fine && finite_bits(x[t][i][e]);
                }
                u32x2 u{encode4(y), encode4(y + 4)};
                if (!fine) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!finite_bits(x[t][i][e])) u[e / 4] = (u[e / 4] & ~(0xffu << 8 * (e % 4))) | 0x7fu << 8 * (e % 4);
                }
                *dst = u;
            } else if (pos < start && grow > 0) {
                const float factor = __uint_as_float(power_bits(grow < 126 ? -grow : -126));
                u32x2 u = *dst;
                float y[8];
                decode4(u[0], y);
                decode4(u[1], y + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= factor;
                *dst = u32x2{encode4(y), encode4(y + 4)};
            }
        }
        __syncthreads();  // every wave has read the old scale
        if (tid == 0) *scale = __uint_as_float(power_bits(e_new));
    }
}

template <typename T>
hipError_t launch(const StoreArgs& a, int64_t groups, int chunks, const void* k, const void* v, hipStream_t stream) {
    const T *kt = (const T*)k, *vt = (const T*)v;
    const dim3 grid((unsigned)groups);
    switch (chunks) {
    case 64: hipLaunchKernelGGL((store_kernel<T, 64, 1>), grid, dim3(64), 0, stream, a, kt, vt); break;
    case 128: hipLaunchKernelGGL((store_kernel<T, 128, 1>), grid, dim3(128), 0, stream, a, kt, vt); break;
    case 256: hipLaunchKernelGGL((store_kernel<T, 256, 1>), grid, dim3(256), 0, stream, a, kt, vt); break;
    case 512: hipLaunchKernelGGL((store_kernel<T, 256, 2>), grid, dim3(256), 0, stream, a, kt, vt); break;
    case 1024: hipLaunchKernelGGL((store_kernel<T, 256, 4>), grid, dim3(256), 0, stream, a, kt, vt); break;
    default: hipLaunchKernelGGL((store_kernel<T, 256, 8>), grid, dim3(256), 0, stream, a, kt, vt); break;
    }
    return hipGetLastError();
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
    a.row_shift = __builtin_ctz((unsigned)d / 8);
    a.xb = kv_strides[0];
    a.xh = kv_strides[1];
    a.xs = kv_strides[2];
    a.start = start;
    a.counts = counts;
    const int64_t groups = (int64_t)a.reach * kv_heads * batch;
    const int chunks = (int)(T * d / 8);
    return dtype == 1 ? launch<uint16_t>(a, groups, chunks, k, v, stream) : launch<float>(a, groups, chunks, k, v, stream);
}

}  // namespace sa
