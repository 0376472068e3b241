// Pages of a paged cache, taken and given back on the device: block tables, slots and positions of the rows that a step adds.
//
// Every workgroup forms the sums over the sequences for itself (their lengths are a few cached kilobytes), so that one launch does for the common call; all quantities are whole numbers, and every
// page and row has a place of its own, so nothing depends on the order of anything.
#include <algorithm>

#include "dev_common.h"
#include "kernels.h"

namespace tlt {

constexpr int kPageThreads = 1024, kPageWaves = kPageThreads / 64;
constexpr int kAtOnce = 4;   // pages or rows a thread works on at a time: their loads overlap

// The sums of (a, b) over the threads before this one, and over all.
__device__ __forceinline__ void block_excl2(int64_t& a, int64_t& b, int64_t (*tmp)[kPageWaves], int64_t& all_a, int64_t& all_b) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t ia = a, ib = b;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t ua = __shfl_up(ia, o, 64), ub = __shfl_up(ib, o, 64);
        if (lane >= o) ia += ua, ib += ub;
    }
    if (lane == 63) tmp[0][wave] = ia, tmp[1][wave] = ib;
    __syncthreads();
    all_a = all_b = 0;
    a = ia - a, b = ib - b;
#pragma unroll
    for (int w = 0; w < kPageWaves; ++w) {
        const int64_t va = tmp[0][w], vb = tmp[1][w];
        a += w < wave ? va : 0, b += w < wave ? vb : 0;
        all_a += va, all_b += vb;
    }
}

struct GrowOut {
    const int32_t* depth = nullptr;
    int32_t *row_start = nullptr, *row_seq = nullptr, *position = nullptr;
    int64_t* slot = nullptr;
    int32_t* granted = nullptr;
};

struct SeqNeed {
    int rows, len, held, want;   // new rows, committed ones, pages held, pages to take if they are free (0 where the sequence is refused)
    bool ok;                     // page_count makes sense and the table is wide enough
};
__device__ __forceinline__ SeqNeed need_of(const PageState& pg, const int32_t* seq_len, const int32_t* n_new, int b) {
    SeqNeed s;
    s.len = max(seq_len[b], 0);
    s.rows = max(n_new[b], 0);
    s.held = pg.page_count[b];
    const uint32_t tokens = (uint32_t)s.len + (uint32_t)s.rows, page = (uint32_t)pg.page_size, whole = tokens / page, need = whole + (whole * page != tokens);
    s.ok = s.held >= 0 && s.held <= pg.max_pages && need <= (uint32_t)pg.max_pages;
    s.want = s.ok ? max((int)need - s.held, 0) : 0;
    return s;
}

// first index of 0 .. n - 1 whose value exceeds x (n: none); values do not fall
__device__ __forceinline__ int above(const int32_t* v, int n, int32_t x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// `done`: the only workgroup, which also moves the stack's end and the counts; otherwise pages_grow_end_k does, after all have read them.  Bound by the chain lengths, sums, page, stack of
// dependent loads: 32 sequences of 48 rows 6.5 us, 256 sequences with 180000 rows and 11000 pages 7.5 us on 180 workgroups (and 2.6 for the counts).
__global__ __launch_bounds__(kPageThreads) void pages_grow_k(int B, int max_rows, int done, const int32_t* __restrict__ seq_len, const int32_t* __restrict__ n_new,
                                                             PageState pg, GrowOut out) {
    extern __shared__ int32_t page_lds[];
    __shared__ int64_t tmp[2][kPageWaves], limit;
    int32_t *row_end = page_lds, *pop_end = page_lds + B, *len_of = page_lds + 2 * B;   // [B] rows and pages popped of the sequences up to b; committed tokens
    const int tid = threadIdx.x, per = (B + kPageThreads - 1) / kPageThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int64_t n_free = min(max((int64_t)*pg.n_free, (int64_t)0), pg.n_pages);
    SeqNeed first{0, 0, 0, 0, false};   // (a thread has one sequence in most calls)
    if (b0 < B) first = need_of(pg, seq_len, n_new, b0);
    int64_t r0 = first.rows, w0 = first.want, all_rows, all_want;
    for (int b = b0 + 1; b < b1; ++b) {
        const SeqNeed s = need_of(pg, seq_len, n_new, b);
        r0 += s.rows, w0 += s.want;
    }
    if (tid == 0) limit = -1;
    block_excl2(r0, w0, tmp, all_rows, all_want);
    // what is popped ends where the first sequence that does not fit would begin
    constexpr int64_t kMost = 0x7fffffff;
    {
        int64_t w = w0;
        for (int b = b0; b < b1; ++b) {
            const int want = b == b0 ? first.want : need_of(pg, seq_len, n_new, b).want;
            if (w <= n_free && n_free < w + want) limit = w;
            w += want;
        }
    }
    __syncthreads();
    const int64_t taken = limit >= 0 ? limit : all_want;
    for (int b = b0; b < b1; ++b) {
        const SeqNeed s = b == b0 ? first : need_of(pg, seq_len, n_new, b);
        const bool granted = s.ok && (s.want == 0 || w0 + s.want <= n_free);
        if (blockIdx.x == 0) {
            if (out.granted) out.granted[b] = granted;
            if (out.row_start) out.row_start[b] = (int32_t)min(r0, kMost);
        }
        r0 += s.rows, w0 += s.want;
        row_end[b] = (int32_t)min(r0, kMost);
        pop_end[b] = (int32_t)min(w0, taken);
        len_of[b] = granted ? s.len : -1 - s.len;   // (negative: no slots)
    }
    if (blockIdx.x == 0 && tid == 0 && out.row_start) out.row_start[B] = (int32_t)min(all_rows, kMost);
    __syncthreads();
    const int32_t* top = pg.free_page + n_free - 1;   // (popped page q is top[-q])
    const uint32_t page = (uint32_t)pg.page_size;
    const int64_t t = (int64_t)blockIdx.x * kPageThreads + tid, stride = (int64_t)gridDim.x * kPageThreads;
    for (int64_t q = t; q < taken; q += stride * kAtOnce) {
        int32_t* to[kAtOnce];
        int32_t id[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t at = q + k * stride;
            to[k] = nullptr;
            if (at >= taken) continue;
            const int b = above(pop_end, B, (int32_t)at);
            id[k] = top[-at];
            to[k] = pg.block_table + (int64_t)b * pg.max_pages + pg.page_count[b] + (at - (b ? pop_end[b - 1] : 0));
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (to[k]) *to[k] = id[k];
    }
    for (int64_t r = t; r < max_rows; r += stride * kAtOnce) {
        int32_t seq[kAtOnce], position[kAtOnce], id[kAtOnce], in_page[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t at_row = r + k * stride;
            seq[k] = -1, position[k] = 0, id[k] = -1, in_page[k] = 0;
            if (at_row >= max_rows) continue;
            const int b = above(row_end, B, (int32_t)at_row);
            if (b >= B) continue;
            const int i = (int)(at_row - (b ? row_end[b - 1] : 0)), l = len_of[b], len = l < 0 ? -1 - l : l;
            seq[k] = b;
            position[k] = len + (out.depth ? out.depth[at_row] : i);
            if (l < 0) continue;
            const int held = pg.page_count[b], before = b ? pop_end[b - 1] : 0, fresh = pop_end[b] - before;
            const uint32_t at = (uint32_t)len + (uint32_t)i, n = at / page;
            in_page[k] = (int)(at - n * page);
            if ((int)n < held + fresh) id[k] = (int)n < held ? pg.block_table[(int64_t)b * pg.max_pages + n] : top[-(before + (int64_t)n - held)];
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t at_row = r + k * stride;
            if (at_row >= max_rows) continue;
            if (out.row_seq) out.row_seq[at_row] = seq[k];
            if (out.position) out.position[at_row] = position[k];
            if (out.slot) out.slot[at_row] = id[k] >= 0 && id[k] < pg.n_pages ? (int64_t)id[k] * pg.page_size + in_page[k] : -1;
        }
    }
    if (!done) return;
    __syncthreads();
    for (int b = tid; b < B; b += kPageThreads) {
        const int more = pop_end[b] - (b ? pop_end[b - 1] : 0);
        if (more) pg.page_count[b] += more;
    }
    if (tid == 0) *pg.n_free = (int32_t)(n_free - taken);
}

__global__ __launch_bounds__(kPageThreads) void pages_grow_end_k(int B, const int32_t* __restrict__ seq_len, const int32_t* __restrict__ n_new, PageState pg) {
    __shared__ int64_t tmp[2][kPageWaves], limit;
    const int tid = threadIdx.x, per = (B + kPageThreads - 1) / kPageThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int64_t n_free = min(max((int64_t)*pg.n_free, (int64_t)0), pg.n_pages);
    int64_t w0 = 0, none = 0, all, all_none;
    for (int b = b0; b < b1; ++b) w0 += need_of(pg, seq_len, n_new, b).want;
    if (tid == 0) limit = -1;
    block_excl2(w0, none, tmp, all, all_none);
    for (int b = b0; b < b1; ++b) {
        const SeqNeed s = need_of(pg, seq_len, n_new, b);
        if (w0 <= n_free && n_free < w0 + s.want) limit = w0;
        w0 += s.want;
        if (s.want > 0 && w0 <= n_free) pg.page_count[b] = s.held + s.want;
    }
    __syncthreads();
    if (tid == 0) *pg.n_free = (int32_t)(n_free - (limit >= 0 ? limit : all));
}

__device__ __forceinline__ int gives(const PageState& pg, const int32_t* keep_len, int b) {
    const int held = pg.page_count[b];
    const uint32_t tokens = keep_len ? (uint32_t)max(keep_len[b], 0) : 0u, page = (uint32_t)pg.page_size, whole = tokens / page, keep = whole + (whole * page != tokens);
    return held >= 0 && held <= pg.max_pages && (uint32_t)held > keep ? held - (int)keep : 0;
}

// Pushed in the reverse of the order in which growing pops: page q of those given back, counted by sequence and table entry, goes to n_free + total - 1 - q.  32 sequences 3.2 us,
// 256 sequences with 11000 pages 9.2.
__global__ __launch_bounds__(kPageThreads) void pages_release_k(int B, int done, const int32_t* __restrict__ keep_len, PageState pg) {
    extern __shared__ int32_t page_lds[];
    __shared__ int64_t tmp[2][kPageWaves];
    int32_t *end = page_lds, *held = page_lds + B;   // [B] pages given back by the sequences up to b; pages held so far
    const int tid = threadIdx.x, per = (B + kPageThreads - 1) / kPageThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int64_t n_free = min(max((int64_t)*pg.n_free, (int64_t)0), pg.n_pages);
    const int first = b0 < B ? gives(pg, keep_len, b0) : 0;   // (a thread has one sequence in most calls)
    int64_t e = first, none = 0, all, all_none;
    for (int b = b0 + 1; b < b1; ++b) e += gives(pg, keep_len, b);
    block_excl2(e, none, tmp, all, all_none);
    if (n_free + all > pg.n_pages) return;   // (uniform, and the same in every workgroup)
    for (int b = b0; b < b1; ++b) {
        e += b == b0 ? first : gives(pg, keep_len, b);
        end[b] = (int32_t)e, held[b] = pg.page_count[b];
    }
    __syncthreads();
    const int64_t stride = (int64_t)gridDim.x * kPageThreads;
    for (int64_t q = (int64_t)blockIdx.x * kPageThreads + tid; q < all; q += stride * kAtOnce) {
        int32_t *entry[kAtOnce], id[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t at = q + k * stride;
            entry[k] = nullptr;
            if (at >= all) continue;
            const int b = above(end, B, (int32_t)at);
            entry[k] = pg.block_table + (int64_t)b * pg.max_pages + held[b] - (end[b] - at);   // (its last page is the last of the sequence's share)
            id[k] = *entry[k];
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (entry[k]) pg.free_page[n_free + all - 1 - (q + k * stride)] = id[k], *entry[k] = -1;
    }
    if (!done) return;
    __syncthreads();
    for (int b = tid; b < B; b += kPageThreads) {
        const int less = end[b] - (b ? end[b - 1] : 0);
        if (less) pg.page_count[b] = held[b] - less;
    }
    if (tid == 0) *pg.n_free = (int32_t)(n_free + all);
}

__global__ __launch_bounds__(kPageThreads) void pages_release_end_k(int B, const int32_t* __restrict__ keep_len, PageState pg) {
    __shared__ int64_t tmp[2][kPageWaves];
    const int tid = threadIdx.x, per = (B + kPageThreads - 1) / kPageThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int64_t n_free = min(max((int64_t)*pg.n_free, (int64_t)0), pg.n_pages);
    int64_t e = 0, none = 0, all, all_none;
    for (int b = b0; b < b1; ++b) e += gives(pg, keep_len, b);
    block_excl2(e, none, tmp, all, all_none);
    if (n_free + all > pg.n_pages) return;
    for (int b = b0; b < b1; ++b) pg.page_count[b] -= gives(pg, keep_len, b);
    if (tid == 0) *pg.n_free = (int32_t)(n_free + all);
}

// One workgroup does everything in one launch; where there may be much to do, several and a launch for the counts.  Growing and giving back, 4096 rows 11.6 us in one workgroup, 17.4 in two launches; 8192 rows 15.1
// and 17.4, 16384 rows 24.7 and 17.3.  Pages given back: what the call cannot know is how many of a pool's pages they are.  A step's are few: taken and given back, 1024 of a pool of 131072 are 10.8 us in
// one launch, 13.1 in two; 4096 pages 12.1 and 12.9, all of them 171 and 108.
constexpr int64_t kRowsOfOne = 8 * kPageThreads, kPagesOfOne = 128 * kPageThreads;

hipError_t pages_grow(hipStream_t s, int B, const PageState& pg, const int32_t* seq_len, const int32_t* n_new, const int32_t* depth, int max_rows,
                      int32_t* row_start, int32_t* row_seq, int32_t* position, int64_t* slot, int32_t* granted) {
    GrowOut out;
    out.depth = depth, out.row_start = row_start, out.row_seq = row_seq, out.position = position, out.slot = slot, out.granted = granted;
    const int groups = max_rows <= kRowsOfOne ? 1 : (int)std::min<int64_t>(512, (max_rows + kPageThreads - 1) / kPageThreads);
    hipLaunchKernelGGL(pages_grow_k, dim3(groups), dim3(kPageThreads), (size_t)B * 12, s, B, max_rows, (int)(groups == 1), seq_len, n_new, pg, out);
    if (groups > 1) hipLaunchKernelGGL(pages_grow_end_k, dim3(1), dim3(kPageThreads), 0, s, B, seq_len, n_new, pg);
    return hipGetLastError();
}

hipError_t pages_release(hipStream_t s, int B, const PageState& pg, const int32_t* keep_len) {
    const int64_t most = std::min<int64_t>((int64_t)B * pg.max_pages, pg.n_pages);
    const int groups = most <= kPagesOfOne ? 1 : (int)std::min<int64_t>(256, most / (4 * kPageThreads));
    hipLaunchKernelGGL(pages_release_k, dim3(groups), dim3(kPageThreads), (size_t)B * 8, s, B, (int)(groups == 1), keep_len, pg);
    if (groups > 1) hipLaunchKernelGGL(pages_release_end_k, dim3(1), dim3(kPageThreads), 0, s, B, keep_len, pg);
    return hipGetLastError();
}

}  // namespace tlt
