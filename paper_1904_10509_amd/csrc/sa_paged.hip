// The bookkeeping of a paged key / value cache (sparse_attn_page_tables) and storing new
// keys and values in it (sparse_attn_paged_store).
//
// Tables.  With h held and f fresh tokens of a sequence and pages of P tokens, everything
// is a sum over the sequences before it: of f for the first row, of ceil((h + f) / P) -
// ceil(h / P) for its first new page in the free list.  A call is bound by latency (one
// sequence is 16 bytes), so there is one launch: every workgroup forms both sums for all
// sequences by itself, in LDS, and then writes its share of the rows and of the new pages.
// A token finds its sequence by a search in LDS, and its page without reading what another
// workgroup writes: a held page from the table, a new one from the free list.
//
// Store.  Bound by reading and writing every row once: 16 bytes a thread and load.
#include "sa_internal.h"
#include "sa_mfma.h"

namespace sa {

namespace {

constexpr int kTableThreads = 1024;
constexpr int kTableRows = 4 * kTableThreads;  // rows of a workgroup
constexpr int kMaxTableGroups = 512;

__device__ inline int32_t pages_of(int64_t tokens, int shift) { return (int32_t)((tokens + (1 << shift) - 1) >> shift); }

// Last s of [0, n) with first[s] <= x (first ascends, first[0] <= x).
__device__ inline int last_at_most(const int32_t* first, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct Sums {
    uint32_t rows, pages;
};

// Sum of a and b with at most `most` rows (associative, as both are no more than that).
__device__ inline Sums add(Sums a, Sums b, uint32_t most) { return {min(a.rows + b.rows, most), a.pages + b.pages}; }

__global__ void __launch_bounds__(kTableThreads) page_tables_kernel(PageTables a) {
    extern __shared__ int32_t lds[];
    __shared__ Sums s_wave[kTableThreads / 64];
    int32_t* first_row = lds;                     // [sequences + 1]
    int32_t* first_page = lds + a.sequences + 1;  // [sequences + 1]
    const int tid = threadIdx.x, lane = tid % 64, w = tid / 64;
    const uint32_t most = (uint32_t)a.tokens;
    const int64_t places = (int64_t)a.max_pages << a.shift;
    auto held = [&](int s) { return (int64_t)max(0, min((int64_t)a.held[s], places)); };
    // rows first: a thread's own run of sequences, then a sum over the workgroup.  The pages of a
    // sequence depend on how many of its rows the call has room for, so they follow in a second turn.
    const int per = (a.sequences + kTableThreads - 1) / kTableThreads, s0 = min(tid * per, a.sequences),
              s1 = min(s0 + per, a.sequences);
    auto before = [&](Sums mine) {  // of the threads before this one; first_*[sequences] gets the whole
        Sums x = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const Sums y{(uint32_t)__shfl_up((int)x.rows, d), (uint32_t)__shfl_up((int)x.pages, d)};
            if (lane >= d) x = add(x, y, most);
        }
        __syncthreads();  // the sums of the turn before are read
        if (lane == 63) s_wave[w] = x;
        __syncthreads();
        Sums up{0, 0};
        for (int v = 0; v < w; ++v) up = add(up, s_wave[v], most);
        // (rows are capped, so the exclusive sum is formed from the lane before, not by taking `mine` off)
        const Sums left{(uint32_t)__shfl_up((int)x.rows, 1), (uint32_t)__shfl_up((int)x.pages, 1)};
        return lane == 0 ? up : add(up, left, most);
    };
    Sums mine{0, 0};
    for (int s = s0; s < s1; ++s) mine.rows = min(mine.rows + (uint32_t)max(0, a.fresh[s]), most);
    uint32_t rows = before(mine).rows;
    for (int s = s0; s < s1; ++s) {
        const int64_t h = held(s);
        const uint32_t begin = rows;
        first_row[s] = (int32_t)begin;
        rows = min(rows + (uint32_t)max(0, a.fresh[s]), most);
        const int64_t both = min(h + (int64_t)(rows - begin), places);
        first_page[s] = pages_of(both, a.shift) - pages_of(h, a.shift);  // its new pages, for now
        mine.pages += (uint32_t)first_page[s];
        if (blockIdx.x == 0) {
            a.starts[s] = (int32_t)begin;
            a.last[s] = (int32_t)(both - 1);
        }
    }
    uint32_t pages = before(Sums{0, mine.pages}).pages;
    for (int s = s0; s < s1; ++s) {
        const uint32_t n = (uint32_t)first_page[s];
        first_page[s] = (int32_t)pages;
        pages += n;
    }
    if (tid == kTableThreads - 1) {  // (its runs end at the last sequence, empty ones too)
        first_row[a.sequences] = (int32_t)rows;
        first_page[a.sequences] = (int32_t)pages;
        if (blockIdx.x == 0) {
            a.starts[a.sequences] = (int32_t)rows;
            a.taken[0] = (int32_t)pages;
        }
    }
    __syncthreads();
    const int32_t total_rows = first_row[a.sequences], total_pages = first_page[a.sequences];
    auto page_at = [&](int32_t n) { return n < a.free_count ? a.free_pages[n] : -1; };  // n-th new page of the call
    const int all = gridDim.x * kTableThreads, me = blockIdx.x * kTableThreads + tid;
    for (int32_t n = me; n < total_pages; n += all) {
        const int s = last_at_most(first_page, a.sequences, n);
        a.table[(int64_t)s * a.table_stride + pages_of(held(s), a.shift) + n - first_page[s]] = page_at(n);
    }
    for (int64_t t0 = 4 * (int64_t)me; t0 < a.tokens; t0 += 4 * (int64_t)all) {
        int s = t0 < total_rows ? last_at_most(first_row, a.sequences, (int32_t)t0) : a.sequences;
        int64_t h = 0;
        int32_t had = 0;
        if (s < a.sequences) {
            h = held(s);
            had = pages_of(h, a.shift);
        }
        int32_t position[4], slot[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t t = (int32_t)t0 + i;
            position[i] = slot[i] = -1;
            if (t0 + i >= total_rows) continue;
            while (t >= first_row[s + 1]) {  // the next sequence that has rows
                ++s;
                h = held(s);
                had = pages_of(h, a.shift);
            }
            const int64_t p = h + (t - first_row[s]);
            if (p >= places) continue;
            const int32_t at = (int32_t)(p >> a.shift);
            const int32_t page = at < had ? a.table[(int64_t)s * a.table_stride + at] : page_at(first_page[s] + at - had);
            position[i] = (int32_t)p;
            if (page >= 0 && page <= (0x7fffffff >> a.shift)) slot[i] = (page << a.shift) + (int32_t)(p & ((1 << a.shift) - 1));
        }
        if (a.wide && t0 + 4 <= a.tokens) {
            *reinterpret_cast<int4*>(a.positions + t0) = make_int4(position[0], position[1], position[2], position[3]);
            *reinterpret_cast<int4*>(a.slots + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
        } else {
            for (int i = 0; i < 4 && t0 + i < a.tokens; ++i) {
                a.positions[t0 + i] = position[i];
                a.slots[t0 + i] = slot[i];
            }
        }
    }
}

constexpr int kStoreThreads = 256;
constexpr int64_t kMaxStoreGroups = 1 << 22;

// Piece n of the call: 16 bytes of one row of K and of V, pieces fastest, then heads, then tokens.
__global__ void __launch_bounds__(kStoreThreads) paged_store_kernel(PagedStore a) {
    const int64_t total = a.tokens * a.heads << a.piece_shift;
    const int64_t each = (int64_t)gridDim.x * kStoreThreads;
    for (int64_t n = (int64_t)blockIdx.x * kStoreThreads + threadIdx.x; n < total; n += each) {
        const int64_t row = n >> a.piece_shift, piece = n & ((1 << a.piece_shift) - 1);
        const int64_t t = row / a.heads, h = row - t * a.heads;
        const int32_t slot = a.slots[t];
        const int32_t page = slot >> a.shift;
        if (slot < 0 || page >= a.pages) continue;
        const u32x4 k = *reinterpret_cast<const u32x4*>(a.k + t * a.kt + h * a.kh + piece * 16);
        const u32x4 v = *reinterpret_cast<const u32x4*>(a.v + t * a.vt + h * a.vh + piece * 16);
        const int64_t to = page * a.cache.sp + h * a.cache.sh + (slot & ((1 << a.shift) - 1)) * a.cache.st + piece * 16;
        *reinterpret_cast<u32x4*>(a.cache.k + to) = k;
        *reinterpret_cast<u32x4*>(a.cache.v + to) = v;
    }
}

}  // namespace

hipError_t page_tables_launch(const PageTables& a, hipStream_t stream) {
    const int64_t groups = max64(1, min64((a.tokens + kTableRows - 1) / kTableRows, kMaxTableGroups));
    const size_t lds = 2 * ((size_t)a.sequences + 1) * sizeof(int32_t);
    hipLaunchKernelGGL(page_tables_kernel, dim3((unsigned)groups), dim3(kTableThreads), lds, stream, a);
    return hipGetLastError();
}

hipError_t paged_store_launch(const PagedStore& a, hipStream_t stream) {
    const int64_t total = a.tokens * a.heads << a.piece_shift;
    const int64_t groups = max64(1, min64((total + kStoreThreads - 1) / kStoreThreads, kMaxStoreGroups));
    hipLaunchKernelGGL(paged_store_kernel, dim3((unsigned)groups), dim3(kStoreThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sa
