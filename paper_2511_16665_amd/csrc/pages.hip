// Pages of a paged cache, taken and given back on the device: block tables, slots and positions of the rows that a step adds.
#include <algorithm>

#include "dev_common.h"
#include "kernels.h"

namespace tlt {

constexpr int kPageThreads = 1024;

// Exclusive sums over the sequences, every workgroup for itself: thread t owns sequences t * per .. t * per + per - 1, whose totals are passed in and whose
// starts come back; `all` is the sum over all.
__device__ __forceinline__ int64_t block_excl(int64_t v, int64_t* tmp, int64_t& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    if (lane == 63) tmp[wave] = incl;
    __syncthreads();
    int64_t base = 0;
    all = 0;
    for (int w = 0; w < kPageThreads / 64; ++w) {
        if (w < wave) base += tmp[w];
        all += tmp[w];
    }
    __syncthreads();
    return base + incl - v;
}

struct GrowOut {
    const int32_t* depth = nullptr;
    int32_t *row_start = nullptr, *row_seq = nullptr, *position = nullptr;
    int64_t* slot = nullptr;
    int32_t* granted = nullptr;
};

struct SeqNeed {
    int64_t rows, want;   // new rows; pages to take if they are free (0 where the sequence is refused)
    int len, held;
    bool ok;              // page_count makes sense and the table is wide enough
};
__device__ __forceinline__ SeqNeed need_of(const PageState& pg, const int32_t* seq_len, const int32_t* n_new, int b) {
    SeqNeed s;
    s.len = max(seq_len[b], 0);
    s.rows = max(n_new[b], 0);
    s.held = pg.page_count[b];
    const int64_t need = ((int64_t)s.len + s.rows + pg.page_size - 1) / pg.page_size;
    s.ok = s.held >= 0 && s.held <= pg.max_pages && need <= pg.max_pages;
    s.want = s.ok ? max(need - s.held, (int64_t)0) : 0;
    return s;
}

// first index of 0 .. n - 1 whose value exceeds x (n: none); values do not fall
__device__ __forceinline__ int above(const int32_t* v, int n, int64_t x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Every workgroup forms the sums over the sequences for itself (their lengths are a few cached kilobytes), then takes its share of the popped pages and
// of the rows.  `done`: the only workgroup, which also moves the stack's end and the counts; otherwise pages_grow_end_k does, after all have read them.
__global__ __launch_bounds__(kPageThreads) void pages_grow_k(int B, int max_rows, int done, const int32_t* __restrict__ seq_len, const int32_t* __restrict__ n_new,
                                                             PageState pg, GrowOut out) {
    extern __shared__ int32_t page_lds[];
    __shared__ int64_t tmp[kPageThreads / 64];
    int32_t* row_end = page_lds;       // [B] rows of the sequences up to b
    int32_t* pop_end = page_lds + B;   // [B] pages popped for them
    const int tid = threadIdx.x, per = (B + kPageThreads - 1) / kPageThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int64_t n_free = min(max((int64_t)*pg.n_free, (int64_t)0), pg.n_pages);
    int64_t rows = 0, want = 0;
    for (int b = b0; b < b1; ++b) {
        const SeqNeed s = need_of(pg, seq_len, n_new, b);
        rows += s.rows, want += s.want;
    }
    int64_t all_rows, all_want;
    int64_t r0 = block_excl(rows, tmp, all_rows), w0 = block_excl(want, tmp, all_want);
    constexpr int64_t kMost = 0x7fffffff;
    int64_t taken = 0;
    for (int b = b0; b < b1; ++b) {
        const SeqNeed s = need_of(pg, seq_len, n_new, b);
        const bool granted = s.ok && (s.want == 0 || w0 + s.want <= n_free);
        if (blockIdx.x == 0) {
            if (out.granted) out.granted[b] = granted;
            if (out.row_start) out.row_start[b] = (int32_t)min(r0, kMost);
        }
        r0 += s.rows, w0 += s.want;
        row_end[b] = (int32_t)min(r0, kMost);
        taken += granted ? s.want : 0;
        pop_end[b] = granted && s.want > 0 ? 1 : 0;   // (for now: takes pages)
    }
    if (blockIdx.x == 0 && tid == 0 && out.row_start) out.row_start[B] = (int32_t)min(all_rows, kMost);
    int64_t all_taken;
    int64_t t0 = block_excl(taken, tmp, all_taken);
    for (int b = b0; b < b1; ++b) {
        if (pop_end[b]) t0 += need_of(pg, seq_len, n_new, b).want;
        pop_end[b] = (int32_t)t0;
    }
    __syncthreads();
    auto popped = [&](int64_t q) {
        const int64_t at = n_free - 1 - q;
        return at >= 0 ? pg.free_page[at] : -1;
    };
    const int64_t t = (int64_t)blockIdx.x * kPageThreads + tid, stride = (int64_t)gridDim.x * kPageThreads;
    for (int64_t q = t; q < all_taken; q += stride) {
        const int b = above(pop_end, B, q);
        pg.block_table[(int64_t)b * pg.max_pages + pg.page_count[b] + (q - (b ? pop_end[b - 1] : 0))] = popped(q);
    }
    for (int64_t r = t; r < max_rows; r += stride) {
        const int b = above(row_end, B, r);
        int32_t position = 0;
        int64_t slot = -1;
        if (b < B) {
            const SeqNeed s = need_of(pg, seq_len, n_new, b);
            const int i = (int)(r - (b ? row_end[b - 1] : 0));
            const int64_t at = (int64_t)s.len + i;
            position = s.len + (out.depth ? out.depth[r] : i);
            const int first = b ? pop_end[b - 1] : 0;
            const int64_t page_at = at / pg.page_size;
            if (s.ok && page_at < s.held + (pop_end[b] - first) && (s.want == 0 || pop_end[b] > first)) {
                const int page = page_at < s.held ? pg.block_table[(int64_t)b * pg.max_pages + page_at] : popped(first + page_at - s.held);
                if (page >= 0 && page < pg.n_pages) slot = (int64_t)page * pg.page_size + at % pg.page_size;
            }
        }
        if (out.row_seq) out.row_seq[r] = b < B ? b : -1;
        if (out.position) out.position[r] = position;
        if (out.slot) out.slot[r] = slot;
    }
    if (!done) return;
    __syncthreads();
    for (int b = tid; b < B; b += kPageThreads) {
        const int more = pop_end[b] - (b ? pop_end[b - 1] : 0);
        if (more) pg.page_count[b] += more;
    }
    if (tid == 0) *pg.n_free = (int32_t)(n_free - all_taken);
}

__global__ __launch_bounds__(kPageThreads) void pages_grow_end_k(int B, const int32_t* __restrict__ seq_len, const int32_t* __restrict__ n_new, PageState pg) {
    __shared__ int64_t tmp[kPageThreads / 64];
    const int tid = threadIdx.x, per = (B + kPageThreads - 1) / kPageThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int64_t n_free = min(max((int64_t)*pg.n_free, (int64_t)0), pg.n_pages);
    int64_t want = 0, all, taken = 0;
    for (int b = b0; b < b1; ++b) want += need_of(pg, seq_len, n_new, b).want;
    int64_t w0 = block_excl(want, tmp, all);
    for (int b = b0; b < b1; ++b) {
        const SeqNeed s = need_of(pg, seq_len, n_new, b);
        w0 += s.want;
        if (s.want > 0 && w0 <= n_free) {
            pg.page_count[b] = s.held + (int)s.want;
            taken += s.want;
        }
    }
    block_excl(taken, tmp, all);
    if (tid == 0) *pg.n_free = (int32_t)(n_free - all);
}

__device__ __forceinline__ int64_t gives(const PageState& pg, const int32_t* keep_len, int b) {
    const int held = pg.page_count[b];
    if (held < 0 || held > pg.max_pages) return 0;
    const int64_t keep = keep_len ? ((int64_t)max(keep_len[b], 0) + pg.page_size - 1) / pg.page_size : 0;
    return max(held - keep, (int64_t)0);
}

// Pushed in the reverse of the order in which growing pops: page q of those given back, counted by sequence and table entry, goes to n_free + total - 1 - q.
__global__ __launch_bounds__(kPageThreads) void pages_release_k(int B, int done, const int32_t* __restrict__ keep_len, PageState pg) {
    extern __shared__ int32_t page_lds[];
    __shared__ int64_t tmp[kPageThreads / 64];
    int32_t* end = page_lds;   // [B] pages given back by the sequences up to b
    const int tid = threadIdx.x, per = (B + kPageThreads - 1) / kPageThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int64_t n_free = min(max((int64_t)*pg.n_free, (int64_t)0), pg.n_pages);
    int64_t mine = 0, all;
    for (int b = b0; b < b1; ++b) mine += gives(pg, keep_len, b);
    int64_t e = block_excl(mine, tmp, all);
    if (n_free + all > pg.n_pages) return;   // (uniform, and the same in every workgroup)
    for (int b = b0; b < b1; ++b) {
        e += gives(pg, keep_len, b);
        end[b] = (int32_t)e;
    }
    __syncthreads();
    const int64_t stride = (int64_t)gridDim.x * kPageThreads;
    for (int64_t q = (int64_t)blockIdx.x * kPageThreads + tid; q < all; q += stride) {
        const int b = above(end, B, q);
        // (its last page is the last of the sequence's share)
        int32_t* entry = pg.block_table + (int64_t)b * pg.max_pages + pg.page_count[b] - (end[b] - q);
        pg.free_page[n_free + all - 1 - q] = *entry;
        *entry = -1;
    }
    if (!done) return;
    __syncthreads();
    for (int b = tid; b < B; b += kPageThreads) {
        const int less = end[b] - (b ? end[b - 1] : 0);
        if (less) pg.page_count[b] -= less;
    }
    if (tid == 0) *pg.n_free = (int32_t)(n_free + all);
}

__global__ __launch_bounds__(kPageThreads) void pages_release_end_k(int B, const int32_t* __restrict__ keep_len, PageState pg) {
    __shared__ int64_t tmp[kPageThreads / 64];
    const int tid = threadIdx.x, per = (B + kPageThreads - 1) / kPageThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int64_t n_free = min(max((int64_t)*pg.n_free, (int64_t)0), pg.n_pages);
    int64_t mine = 0, all;
    for (int b = b0; b < b1; ++b) mine += gives(pg, keep_len, b);
    block_excl(mine, tmp, all);
    if (n_free + all > pg.n_pages) return;
    for (int b = b0; b < b1; ++b) pg.page_count[b] -= (int)gives(pg, keep_len, b);
    if (tid == 0) *pg.n_free = (int32_t)(n_free + all);
}

// One workgroup that does everything in one launch, or several and a launch for the counts.
constexpr int64_t kPageOneGroup = 16 * kPageThreads;

hipError_t pages_grow(hipStream_t s, int B, const PageState& pg, const int32_t* seq_len, const int32_t* n_new, const int32_t* depth, int max_rows,
                      int32_t* row_start, int32_t* row_seq, int32_t* position, int64_t* slot, int32_t* granted) {
    GrowOut out;
    out.depth = depth, out.row_start = row_start, out.row_seq = row_seq, out.position = position, out.slot = slot, out.granted = granted;
    const int groups = max_rows <= kPageOneGroup ? 1 : (int)std::min<int64_t>(512, (max_rows + kPageThreads - 1) / kPageThreads);
    hipLaunchKernelGGL(pages_grow_k, dim3(groups), dim3(kPageThreads), (size_t)B * 8, s, B, max_rows, (int)(groups == 1), seq_len, n_new, pg, out);
    if (groups > 1) hipLaunchKernelGGL(pages_grow_end_k, dim3(1), dim3(kPageThreads), 0, s, B, seq_len, n_new, pg);
    return hipGetLastError();
}

hipError_t pages_release(hipStream_t s, int B, const PageState& pg, const int32_t* keep_len) {
    const int64_t most = std::min<int64_t>((int64_t)B * pg.max_pages, pg.n_pages);
    const int groups = most <= 8 * kPageOneGroup ? 1 : (int)std::min<int64_t>(256, most / (4 * kPageThreads));
    hipLaunchKernelGGL(pages_release_k, dim3(groups), dim3(kPageThreads), (size_t)B * 4, s, B, (int)(groups == 1), keep_len, pg);
    if (groups > 1) hipLaunchKernelGGL(pages_release_end_k, dim3(1), dim3(kPageThreads), 0, s, B, keep_len, pg);
    return hipGetLastError();
}

}  // namespace tlt
