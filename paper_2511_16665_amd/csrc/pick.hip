// Sampling from rows of logits behind top-k, top-p and min-p: one token per row, or the row with all other tokens at -infinity.
//
// Weights are the acceptance rules' whole numbers W = floor(exp(l / tau - max / tau) * 2^32), so sums do not depend on their order; they are held as doubles, which are exact
// up to 2^53 (2^20 tokens, 2^52).  What is kept is a prefix of the order (logit falling, index rising), given by the logit it ends in and the last index kept of those equal to it
// (cut, last below), and of that what weighs enough.  Equal logits have equal weights.
//
// A row is cut into segments, a workgroup each, and read two or three times:
//   pick_max_k     the largest logit, and 256 to 1024 sample maxima, which show how far down the most likely few hundred tokens reach
//   pick_weigh_k   all weights; the likely few hundred tokens go to a list, and weights go to a histogram over the distance to the largest logit where the list may not reach the
//                  prefix's end.  The last workgroup of a row orders the list and finds that end, or the histogram's bin that holds it
//   pick_gather_k  only where the list did not reach: the tokens of that bin (or all down to it) go to a list, what is above is summed up
//   pick_mask_k    for filtered rows
#include <algorithm>
#include <cfloat>

#include "dev_common.h"
#include "kernels.h"

namespace tlt {

typedef unsigned long long u64;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kWeighThreads = 256, kGatherThreads = 512;
constexpr int kSegsMost = 32, kSamples = 1024;
constexpr int kBins = 512;
constexpr int kList = 2048, kLocalList = 1024;   // entries of a row's list of likely tokens, and of what a segment may add
constexpr int kGather = 8192;                    // entries of the second list
constexpr int kBatchRows = 256;                  // rows of one round: their logits stay in the last-level cache between the readings
constexpr u64 kNoEntry = ~0ull;

// order of logits as whole numbers; -0 and +0 are equal
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t kKeyNothing = 0x007fffffu;   // of -infinity
// a token in a list: ascending numbers are the order
__device__ __forceinline__ u64 entry_of(float l, int j) { return (u64)(~key_of(l)) << 32 | (uint32_t)j; }
__device__ __forceinline__ float entry_logit(u64 e) { return logit_of(~(uint32_t)(e >> 32)); }

// what a request asks for, of one row
struct Asked {
    double tau;
    int top_k;         // 0: off
    uint32_t top_p;    // units of 2^-31; 2^31: off
    double least;      // weight; 0: off
    __device__ __forceinline__ bool by_p() const { return top_p < (1u << 31); }
    __device__ __forceinline__ bool prefix() const { return top_k > 0 || by_p(); }
};
__device__ __forceinline__ Asked asked_of(const PickFilter& f, int seq, int V) {
    Asked a{1.0, 0, 1u << 31, 0.0};
    const float tau = f.temperature ? f.temperature[seq] : 1.f;
    if (!(tau > 0.f)) {
        a.top_k = 1;
        return a;
    }
    a.tau = (double)tau;
    if (f.top_k) a.top_k = f.top_k[seq] < V ? max(f.top_k[seq], 0) : 0;
    if (f.top_p) {
        const float p = f.top_p[seq];
        if (p < 1.f) a.top_p = (uint32_t)(fmax((double)p, 0.0) * 2147483648.0);
    }
    if (f.min_p) {
        const float m = f.min_p[seq];
        if (m > 0.f) a.least = floor(fmin((double)m, 1.0) * 4294967296.0);
    }
    return a;
}
// ceil(share * S / 2^31), at least 1
__device__ __forceinline__ double share_of(uint32_t share, double S) {
    const unsigned __int128 x = (unsigned __int128)share * (u64)S + 0x7fffffffu;
    return fmax((double)(u64)(x >> 31), 1.0);
}
// (u * S) >> 32
__device__ __forceinline__ double aim_of(uint32_t u, double S) { return (double)(u64)(((unsigned __int128)u * (u64)S) >> 32); }

// A row's weights: 2^32 times 2^t, t = (l - max) * log2(e) / tau (good to 2^-51 of the distance), as 2^n * 2^r with |r| <= 1/2 and a polynomial of degree 10 in r that interpolates
// (2^r - 1) / r at Chebyshev's nodes, 2^-50.6 off at most.  Nineteen operations in double: the library's exponential and a division are five times as many, and reading a
// row costs as long as 16 operations per element.  t = 0 gives 2^32 exactly.
struct Weigh {
    double top, scale, tau;
    float top_f;
    bool inf;   // the largest is +infinity: those tokens weigh 2^32, all others nothing
    __device__ __forceinline__ Weigh(float largest, double tau_) : tau(tau_) {
        inf = largest == INFINITY;
        top_f = inf ? 0.f : largest;
        top = (double)top_f;
        scale = 1.4426950408889634074 / tau_;
    }
    __device__ __forceinline__ float fix(float x) const { return inf ? (x == INFINITY ? 0.f : -INFINITY) : x; }
    __device__ __forceinline__ double operator()(float x) const {
        const double t = fmax(((double)fix(x) - top) * scale, -40.0);   // (-infinity, and what infinities leave undefined, weigh nothing)
        constexpr double kMagic = 6755399441055744.0 + 32.0;             // 1.5 * 2^52: the sum's low bits are n + 32
        const double s = t + kMagic;
        const double r = t - (s - kMagic);
        double p = 7.070977866508138e-09;
        p = fma(p, r, 1.0205905413765595e-07);
        p = fma(p, r, 1.3215451633221434e-06);
        p = fma(p, r, 1.5252672924850737e-05);
        p = fma(p, r, 0.00015403530424776529);
        p = fma(p, r, 0.0013333558200794592);
        p = fma(p, r, 0.009618129107618665);
        p = fma(p, r, 0.05550410866465167);
        p = fma(p, r, 0.24022650695910075);
        p = fma(p, r, 0.6931471805599462);
        p = fma(p, r, 1.0);
        const int n = __double2loint(s);
        return floor(__hiloint2double(__double2hiint(p) + (n << 20), __double2loint(p)));
    }
    // l / tau - max / tau
    __device__ __forceinline__ double below(float x) const { return fix(x) == top_f ? 0.0 : (double)fix(x) / tau - top / tau; }
    __device__ __forceinline__ u64 whole(double w) const { return (u64)__double_as_longlong(w + 0x1p52) & 0xfffffffffffffull; }
};

// ---- reading a row: 16-byte pieces, the first and last of which may lie partly outside
template <typename T>
struct RowView {
    static constexpr int VEC = 16 / sizeof(T);
    const T* row;
    int V, off;   // off: elements of the first piece that are in front of the row
    __device__ __forceinline__ RowView(const T* row_, int V_) : row(row_), V(V_), off((int)(((uintptr_t)row_ & 15) / sizeof(T))) {}
    __device__ __forceinline__ int pieces() const { return (V + off + VEC - 1) / VEC; }
    __device__ __forceinline__ int first(int c) const { return c * VEC - off; }   // index of piece c's first element
    // elements outside the row are -infinity
    __device__ __forceinline__ void load(int c, float (&x)[VEC]) const {
        const int j = first(c);
        if (j >= 0 && j + VEC <= V) {
            const u32x4_t w = *(const u32x4_t*)(row + j);
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(w[e] << 16), x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = j + e >= 0 && j + e < V ? to_float(row[j + e]) : -INFINITY;
        }
    }
};

// ---- sums over a workgroup
__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
template <int NT>
__device__ __forceinline__ double block_sum(double v, double* tmp) {
    v = wave_sum_d(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) all += tmp[w];
    return all;
}
// sum over the threads before this one
template <int NT>
__device__ __forceinline__ double block_excl_d(double v, double* tmp) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 63) tmp[wave] = incl;
    __syncthreads();
    double base = 0.0;
    for (int w = 0; w < wave; ++w) base += tmp[w];
    return base + incl - v;
}

// a[0 .. n - 1] in ascending order; n a power of two
template <int NT>
__device__ void sort_entries(u64* a, int n) {
    for (int k = 2; k <= n; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (int i = threadIdx.x; i < n / 2; i += NT) {
                const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
                const u64 x = a[lo], y = a[hi];
                if ((x > y) == ((lo & k) == 0)) a[lo] = y, a[hi] = x;
            }
        }
    __syncthreads();
}
__device__ __forceinline__ int power_above(int n) {
    int p = 1;
    while (p < n) p <<= 1;
    return p;
}

// ---- what the workgroups of a row share
enum { kOpen = 0, kDone = 1, kBinAlone = 2, kAllDownTo = 3, kStepwise = 4 };
struct PickRow {
    uint32_t list_n, gather_n, seen_weigh, seen_gather;
    int32_t state;
    int32_t bin;                // kBinAlone: the bin that holds the end; kAllDownTo: the last one to take
    uint32_t cut;               // the result: kept are keys above it and those equal to it up to index `last`; 0: the row is copied
    int32_t last;
    double before_w, before_n;  // of the tokens above the gathered ones
    double whole;
};
struct PickWs {
    PickRow* row;
    float *top, *sample;     // [rows][segs], [rows][samples]
    double *whole, *part;    // [rows][segs], [rows][segs * 8]: sums of kept weights over the ranges of waves
    uint32_t* part_n;        // their counts
    u64 *list, *gather;      // [rows][kList], [rows][kGather]
    u64* bin_w;              // [rows][segs][kBins]
    uint32_t* bin_n;
};
struct PickGeo {
    int V, segs, pieces, per;   // pieces of a segment, and of a row at most
    int samples;                // per segment
    int rows_per_seq, row0;     // row0: first row of this round
};

// The workgroup that is the last of `total` of a row to come here sees what all of them wrote (every wave waits for its stores, then one thread releases them).
__device__ __forceinline__ bool last_here(uint32_t* seen, int total, int* flag) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) *flag = __hip_atomic_fetch_add(seen, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)total - 1u;
    __syncthreads();
    return *flag != 0;
}

// the bin of a logit, for rows whose bins span `reach` (nats times tau); at or past kBins: below them
__device__ __forceinline__ float bins_per_logit(const Asked& ask, int V) {
    // tokens whose weight is below (1 - p) 2^32 / V cannot be in the shortest prefix of weight p S, as S >= 2^32 and together they are less than (1 - p) S; otherwise
    // down to where weights are 0
    double reach = 23.0;
    if (ask.top_k == 0) reach = fmin(reach, 0.01 + log((double)V / fmax(1.0 - (double)ask.top_p * 0x1p-31, 1e-10)));
    return (float)fmin((double)kBins / (reach * ask.tau), 1e30);
}
__device__ __forceinline__ int bin_of(const Weigh& w, float x, float per_logit) { return (int)fminf((w.top_f - w.fix(x)) * per_logit, 1e6f); }

// ---- outputs
__device__ __forceinline__ void put_nothing(const PickOut& out, int r, bool nan) {
    if (out.token) out.token[r] = -1;
    if (out.logprob) out.logprob[2 * r] = out.logprob[2 * r + 1] = nan ? NAN : -INFINITY;
    if (out.kept) out.kept[r] = 0;
}
__device__ __forceinline__ void put_token(const PickOut& out, int r, const Weigh& w, int j, float x, double S, double whole) {
    out.token[r] = j;
    if (out.logprob) {
        const double z = w.below(x);
        out.logprob[2 * r] = (float)(z - log(S * 0x1p-32));
        out.logprob[2 * r + 1] = (float)(z - log(whole * 0x1p-32));
    }
}

struct Kept {
    uint32_t cut;
    int last;
    double least;
    __device__ __forceinline__ bool operator()(const Weigh& w, int j, float x) const {
        const uint32_t k = key_of(x);
        return (k > cut || (k == cut && j <= last)) && (least == 0.0 || w(x) >= least);
    }
};

// The first token of pieces [c0, c1) whose running sum, from `base` on, of kept weights exceeds `aim`; returns the sum over the pieces.
template <int NT, typename T, typename F>
__device__ double draw_from(const RowView<T>& row, int c0, int c1, const Weigh& w, const Kept& kept, double base, F aim_of_sum, double* tmp, const PickOut& out, int r, double whole) {
    constexpr int VEC = RowView<T>::VEC;
    const int per = (c1 - c0 + NT - 1) / NT, a = min(c1, c0 + (int)threadIdx.x * per), b = min(c1, a + per);
    double mine = 0.0;
    for (int c = a; c < b; ++c) {
        float x[VEC];
        row.load(c, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (kept(w, row.first(c) + e, x[e])) mine += w(x[e]);
    }
    const double all = block_sum<NT>(mine, tmp);
    double run = base + block_excl_d<NT>(mine, tmp), S;
    const double aim = aim_of_sum(all, S);
    if (run <= aim && aim < run + mine) {
        bool found = false;
        for (int c = a; c < b && !found; ++c) {
            float x[VEC];
            row.load(c, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (found || !kept(w, row.first(c) + e, x[e])) continue;
                run += w(x[e]);
                if (run > aim) {
                    put_token(out, r, w, row.first(c) + e, x[e], S, whole);
                    found = true;
                }
            }
        }
    }
    return all;
}

// Where the prefix ends in an ordered list whose entries follow on before_n tokens of weight before_w: how many entries are in, or -1 if it ends behind them.
// complete: no token above -infinity follows.  S: the weight that top_p is a share of, for rows without top_k.
template <int NT>
__device__ int end_in_list(const u64* a, int n, const Asked& ask, const Weigh& w, double before_w, double before_n, double S, bool complete, double* tmp, int* found) {
    const double most = ask.top_k > 0 ? (double)ask.top_k - before_n : 1e18;
    if (most > n && !complete && ask.top_k > 0) return -1;
    const int nk = (int)fmin((double)n, most);
    if (!ask.by_p()) return nk;
    const int per = (nk + NT - 1) / NT, i0 = min(nk, (int)threadIdx.x * per), i1 = min(nk, i0 + per);
    double mine = 0.0;
    for (int i = i0; i < i1; ++i) mine += w(entry_logit(a[i]));
    if (ask.top_k > 0) S = before_w + block_sum<NT>(mine, tmp);
    const double aim = share_of(ask.top_p, S);
    double run = before_w + block_excl_d<NT>(mine, tmp);
    if (threadIdx.x == 0) *found = -1;
    __syncthreads();
    if (run < aim && aim <= run + mine)
        for (int i = i0; i < i1; ++i) {
            run += w(entry_logit(a[i]));
            if (run >= aim) {
                *found = i + 1;
                break;
            }
        }
    __syncthreads();
    return *found;
}

// Draws from the first n entries of an ordered list, which are all that is kept but for `least`.
template <int NT>
__device__ void draw_from_list(u64* a, int n, const Asked& ask, const Weigh& w, double* tmp, const PickOut& out, int r, double whole) {
    // by index: entries too light, and those behind the end, go last
    const int size = power_above(n);
    double S = 0.0, count = 0.0;
    for (int i = threadIdx.x; i < size; i += NT) {
        u64 e = kNoEntry;
        if (i < n) {
            e = a[i];
            const double x = w(entry_logit(e));
            const bool in = ask.least == 0.0 || x >= ask.least;
            S += in ? x : 0.0, count += in;
            e = in ? e << 32 | e >> 32 : kNoEntry;
        }
        a[i] = e;
    }
    S = block_sum<NT>(S, tmp), count = block_sum<NT>(count, tmp);
    if (threadIdx.x == 0 && out.kept) out.kept[r] = (int32_t)count;
    sort_entries<NT>(a, size);
    const int m = (int)count, per = (m + NT - 1) / NT, i0 = min(m, (int)threadIdx.x * per), i1 = min(m, i0 + per);
    auto logit = [&](u64 e) { return logit_of(~(uint32_t)e); };
    double mine = 0.0;
    for (int i = i0; i < i1; ++i) mine += w(logit(a[i]));
    double run = block_excl_d<NT>(mine, tmp);
    const double aim = aim_of(out.u[r], S);
    if (run <= aim && aim < run + mine)
        for (int i = i0; i < i1; ++i) {
            run += w(logit(a[i]));
            if (run > aim) {
                put_token(out, r, w, (int)(a[i] >> 32), logit(a[i]), S, whole);
                break;
            }
        }
}

// ---- the largest logit and the samples
template <typename T>
__global__ __launch_bounds__(kWeighThreads) void pick_max_k(PickGeo geo, const T* logits, int64_t row_stride, PickWs ws, PickOut out) {
    constexpr int VEC = RowView<T>::VEC;
    __shared__ float wave_top[kWeighThreads / 64];
    const int lr = blockIdx.x / geo.segs, g = blockIdx.x - lr * geo.segs, tid = threadIdx.x;
    const RowView<T> row(logits + (int64_t)(geo.row0 + lr) * row_stride, geo.V);
    const int c1 = min(row.pieces(), (g + 1) * geo.per);
    float top = -INFINITY;
    bool nan = false;
    for (int c = g * geo.per + tid; c < c1; c += kWeighThreads) {
        float x[VEC];
        row.load(c, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) nan |= x[e] != x[e], top = fmaxf(top, x[e]);
    }
    const int lanes = kWeighThreads / geo.samples;   // that share a sample
    float s = top;
    for (int o = 1; o < lanes; o <<= 1) s = fmaxf(s, __shfl_xor(s, o, 64));
    if (tid % lanes == 0) ws.sample[(int64_t)lr * kSamples + g * geo.samples + tid / lanes] = s;
    top = wave_max(top);
    if (__any(nan)) top = NAN;
    if ((tid & 63) == 0) wave_top[tid >> 6] = top;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int w = 0; w < kWeighThreads / 64; ++w) top = top != top || wave_top[w] != wave_top[w] ? NAN : fmaxf(top, wave_top[w]);
        ws.top[lr * geo.segs + g] = top;
        if (g == 0) {
            PickRow z{};
            ws.row[lr] = z;
            if (out.rows && out.kept) out.kept[geo.row0 + lr] = 0;
        }
    }
}

// the row's largest logit; NaN if there is one
__device__ __forceinline__ float row_top(const PickGeo& geo, const PickWs& ws, int lr) {
    const int lane = threadIdx.x & 63;
    const float t = lane < geo.segs ? ws.top[lr * geo.segs + lane] : -INFINITY;
    return __any(t != t) ? NAN : wave_max(t);
}

// A logit that at least `rank` of the row's samples, and so at least as many tokens, reach: from a histogram of the samples between the smallest and the largest.
__device__ __forceinline__ float reached_by(int rank, int n, const float* sample, float top, uint32_t* bins, float* tmp) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float lo = INFINITY;
    for (int i = tid; i < n; i += kWeighThreads) {
        const float s = sample[i];
        if (s > -INFINITY) lo = fminf(lo, s);
    }
    lo = -wave_max(-lo);
    for (int i = tid; i < 1024; i += kWeighThreads) bins[i] = 0;
    if (lane == 0) tmp[wave] = lo;
    __syncthreads();
    lo = fminf(fminf(tmp[0], tmp[1]), fminf(tmp[2], tmp[3]));
    const float width = (top - lo) / 1023.f, per = width > 0.f ? 1.f / width : 0.f;   // (infinite distances: every token is in)
    for (int i = tid; i < n; i += kWeighThreads) {
        const float s = sample[i];
        if (s > -INFINITY) atomicAdd(&bins[min((int)fminf((top - s) * per, 1023.f), 1023)], 1u);
    }
    __syncthreads();
    // the first bin down to which `rank` samples lie; all of them if there are fewer
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) mine += bins[4 * tid + k];
    uint32_t incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    uint32_t* sums = (uint32_t*)tmp + 8;
    if (lane == 63) sums[wave] = incl;
    if (tid == 0) sums[4] = 1024;
    __syncthreads();
    for (int w = 0; w < wave; ++w) incl += sums[w];
    uint32_t run = incl - mine;
    if (run < (uint32_t)rank && incl >= (uint32_t)rank)
        for (int k = 0; k < 4; ++k) {
            run += bins[4 * tid + k];
            if (run >= (uint32_t)rank) {
                sums[4] = 4 * tid + k;
                break;
            }
        }
    __syncthreads();
    const int bin = (int)sums[4];
    __syncthreads();
    return bin >= 1023 ? -FLT_MAX : fmaxf(top - (float)(bin + 1) * width * 1.0001f, -FLT_MAX);
}

__device__ __forceinline__ int list_rank(const Asked& ask, int samples) {
    const int want = ask.top_k > 0 ? max(ask.top_k + ask.top_k / 4, 64) : 256;
    return min(want, samples * 3 / 4);
}

// ---- weights, list, histogram
template <typename T>
__global__ __launch_bounds__(kWeighThreads) void pick_weigh_k(PickGeo geo, const T* logits, int64_t row_stride, PickFilter filter, PickWs ws, PickOut out) {
    constexpr int VEC = RowView<T>::VEC, NT = kWeighThreads, NW = NT / 64;
    __shared__ u64 buf[kList];          // first: histogram (weights, counts) and the segment's list; then the row's list
    __shared__ double tmp[16];
    __shared__ uint32_t local_n, base_n;
    __shared__ int flag;
    u64* bin_w = buf;
    uint32_t* bin_n = (uint32_t*)(buf + kBins);
    u64* local = buf + kBins + kBins / 2;
    const int lr = blockIdx.x / geo.segs, g = blockIdx.x - lr * geo.segs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = geo.row0 + lr;
    const RowView<T> row(logits + (int64_t)r * row_stride, geo.V);
    PickRow* pr = ws.row + lr;
    const float top = row_top(geo, ws, lr);
    if (top != top || top == -INFINITY) {   // (uniform over the row's workgroups)
        if (g == 0 && tid == 0) {
            if (out.token) put_nothing(out, r, top != top);
            pr->state = kDone, pr->cut = 0, pr->last = -1;
        }
        return;
    }
    const Asked ask = asked_of(filter, r / geo.rows_per_seq, geo.V);
    const Weigh w(top, ask.tau);
    const bool prefix = ask.prefix();
    const int n_samples = geo.samples * geo.segs;
    // tokens from `from` on go to the list
    float from = INFINITY;
    bool use_bins = false, count_bins = false;
    if (prefix) {
        const int rank = list_rank(ask, n_samples);
        from = reached_by(rank, n_samples, ws.sample + (int64_t)lr * kSamples, top, (uint32_t*)buf, (float*)tmp);
        count_bins = ask.top_k > rank;
        use_bins = count_bins || ask.top_k == 0;
    }
    const float per_logit = use_bins ? bins_per_logit(ask, geo.V) : 0.f;
    for (int i = tid; i < kBins; i += NT) bin_w[i] = 0, bin_n[i] = 0;
    if (tid == 0) local_n = 0;
    __syncthreads();
    const int seg_end = min(row.pieces(), (g + 1) * geo.per), wper = (geo.per + NW - 1) / NW;
    const int c0 = min(seg_end, g * geo.per + wave * wper), c1 = min(seg_end, c0 + wper);
    double whole = 0.0, kept = 0.0;
    uint32_t kept_n = 0;
    for (int c = c0 + lane; c - lane < c1; c += 64) {   // (whole waves: the list is appended to together)
        float x[VEC];
        if (c < c1) row.load(c, x);
        else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = -INFINITY;
        }
        double weight[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            weight[e] = w(x[e]);
            whole += weight[e];
        }
        if (!prefix) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const bool in = x[e] > -INFINITY && weight[e] >= ask.least;
                kept += in ? weight[e] : 0.0, kept_n += in;
            }
            continue;
        }
        float best = x[0];
#pragma unroll
        for (int e = 1; e < VEC; ++e) best = fmaxf(best, x[e]);
        if (__any(best >= from)) {
            uint32_t n = 0;
#pragma unroll
            for (int e = 0; e < VEC; ++e) n += x[e] >= from;
            uint32_t at = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t up = __shfl_up(at, o, 64);
                if (lane >= o) at += up;
            }
            uint32_t start = 0;
            if (lane == 63) start = atomicAdd(&local_n, at);
            at += __shfl(start, 63, 64) - n;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (x[e] >= from) {
                    if (at < (uint32_t)kLocalList) local[at] = entry_of(x[e], row.first(c) + e);
                    ++at;
                }
        }
        if (use_bins) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int b = bin_of(w, x[e], per_logit);
                if (b < kBins) {
                    atomicAdd(&bin_w[b], w.whole(weight[e]));
                    if (count_bins) atomicAdd(&bin_n[b], 1u);
                }
            }
        }
    }
    whole = block_sum<NT>(whole, tmp);
    if (tid == 0) ws.whole[lr * geo.segs + g] = whole;
    if (!prefix) {
        kept = wave_sum_d(kept);
        for (int o = 32; o > 0; o >>= 1) kept_n += __shfl_xor(kept_n, o, 64);
        if (lane == 0) ws.part[(lr * geo.segs + g) * 8 + wave] = kept, ws.part_n[(lr * geo.segs + g) * 8 + wave] = kept_n;
    } else {
        if (tid == 0) base_n = atomicAdd(&pr->list_n, local_n > (uint32_t)kLocalList ? 1u << 20 : local_n);
        __syncthreads();
        const uint32_t n = min(local_n, (uint32_t)kLocalList), base = base_n;
        for (uint32_t i = tid; i < n; i += NT)
            if (base + i < (uint32_t)kList) ws.list[(int64_t)lr * kList + base + i] = local[i];
        if (use_bins)
            for (int i = tid; i < kBins; i += NT) {
                ws.bin_w[((int64_t)lr * geo.segs + g) * kBins + i] = bin_w[i];
                if (count_bins) ws.bin_n[((int64_t)lr * geo.segs + g) * kBins + i] = bin_n[i];
            }
    }
    if (!last_here(&pr->seen_weigh, geo.segs, &flag)) return;

    // ---- the row's last workgroup
    whole = 0.0;
    for (int i = 0; i < geo.segs; ++i) whole += ws.whole[lr * geo.segs + i];
    if (tid == 0) pr->whole = whole;
    if (!prefix) {
        if (tid == 0) pr->state = kDone, pr->cut = kKeyNothing, pr->last = -1;
        if (!out.token) return;
        // the wave's range that holds the draw
        const int ranges = geo.segs * 8;
        double S = 0.0, count = 0.0;
        for (int i = 0; i < ranges; ++i)
            if ((i & 7) < NW) S += ws.part[lr * ranges + i], count += ws.part_n[lr * ranges + i];
        const double aim = aim_of(out.u[r], S);
        double base = 0.0;
        int at = -1;
        for (int i = 0; i < ranges && at < 0; ++i) {
            if ((i & 7) >= NW) continue;
            const double add = ws.part[lr * ranges + i];
            if (base + add > aim) at = i;
            else base += add;
        }
        if (tid == 0 && out.kept) out.kept[r] = (int32_t)count;
        if (at < 0) return;   // (cannot be: S is the sum of the parts)
        const int end = min(row.pieces(), ((at >> 3) + 1) * geo.per), p0 = min(end, (at >> 3) * geo.per + (at & 7) * wper), p1 = min(end, p0 + wper);
        const Kept in{kKeyNothing, -1, ask.least};
        draw_from<NT>(row, p0, p1, w, in, base, [&](double, double& sum) { sum = S; return aim; }, tmp, out, r, whole);
        return;
    }
    const uint32_t n = pr->list_n;
    int end = -1;
    if (n <= (uint32_t)kList) {
        const int size = power_above((int)n);
        for (int i = tid; i < size; i += NT) buf[i] = i < (int)n ? ws.list[(int64_t)lr * kList + i] : kNoEntry;
        sort_entries<NT>(buf, size);
        end = end_in_list<NT>(buf, (int)n, ask, w, 0.0, 0.0, whole, from == -FLT_MAX, tmp, &flag);
    }
    if (end > 0) {
        if (tid == 0) {
            const u64 e = buf[end - 1];
            pr->state = kDone, pr->cut = ~(uint32_t)(e >> 32), pr->last = (int32_t)(uint32_t)e;
        }
        __syncthreads();
        if (out.token) draw_from_list<NT>(buf, end, ask, w, tmp, out, r, whole);
        return;
    }
    if (!use_bins) {
        if (tid == 0) pr->state = kStepwise;
        return;
    }
    // the bin that holds the end: thread t owns bins 2t and 2t + 1
    __syncthreads();
    u64 bw[2] = {0, 0};
    uint32_t bn[2] = {0, 0};
    for (int i = 0; i < geo.segs; ++i) {
        const int64_t at = ((int64_t)lr * geo.segs + i) * kBins + 2 * tid;
        bw[0] += ws.bin_w[at], bw[1] += ws.bin_w[at + 1];
        if (count_bins) bn[0] += ws.bin_n[at], bn[1] += ws.bin_n[at + 1];
    }
    const double aim = count_bins ? (double)ask.top_k : share_of(ask.top_p, whole);
    const double m0 = count_bins ? (double)bn[0] : (double)bw[0], m1 = count_bins ? (double)bn[1] : (double)bw[1];
    const double run = block_excl_d<NT>(m0 + m1, tmp);
    if (tid == 0) pr->state = kStepwise;   // (unless a bin is found)
    __syncthreads();
    if (run < aim && aim <= run + m0 + m1) {
        const bool second = run + m0 < aim;
        const double before = second ? run + m0 : run;
        pr->bin = 2 * tid + second;
        pr->before_w = count_bins ? 0.0 : before, pr->before_n = count_bins ? before : 0.0;
        // one limit: the bin's own tokens are enough.  Two: all tokens down to it, if a list holds them
        if (!count_bins || !ask.by_p()) pr->state = kBinAlone;
        else if (before + (second ? m1 : m0) <= (double)kGather) pr->state = kAllDownTo, pr->before_n = 0.0;
    }
}

// ---- rows that neither list nor bins settle: digit by digit over the keys, one workgroup, every step a pass over the row
template <int NT, typename T>
__device__ void cut_stepwise(const RowView<T>& row, const Asked& ask, const Weigh& w, u64* lds, double* tmp, uint32_t& cut, int& last) {
    constexpr int VEC = RowView<T>::VEC;
    u64 *bins = lds, *counts = lds + 256, *found = lds + 512;
    const int tid = threadIdx.x, pieces = row.pieces();
    auto each = [&](auto f) {
        for (int c = tid; c < pieces; c += NT) {
            float x[VEC];
            row.load(c, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f(row.first(c) + e, x[e]);
        }
    };
    uint32_t lim_key = kKeyNothing;   // among tokens above it, and lim_n of those equal to it
    u64 lim_n = 0;
    // Where a prefix ends: with by_weight when what it weighs reaches `aim` (>= 1), otherwise after `aim` tokens.
    auto prefix = [&](double aim, bool by_weight, uint32_t& key, u64& n, u64& before, u64& group) {
        key = 0, before = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            for (int i = tid; i < 256; i += NT) bins[i] = counts[i] = 0;
            __syncthreads();
            each([&](int, float x) {
                const uint32_t k = key_of(x);
                if (k <= lim_key || (shift < 24 && k >> (shift + 8) != key >> (shift + 8))) return;
                atomicAdd(&counts[k >> shift & 255], 1ull);
                if (by_weight) atomicAdd(&bins[k >> shift & 255], w.whole(w(x)));
            });
            __syncthreads();
            if (tid == 0) {
                if (lim_n && (shift == 24 || lim_key >> (shift + 8) == key >> (shift + 8))) {
                    counts[lim_key >> shift & 255] += lim_n;
                    if (by_weight) bins[lim_key >> shift & 255] += lim_n * w.whole(w(logit_of(lim_key)));
                }
                u64 sum = before;
                int at = -1, lowest = 0;
                for (int d = 255; d >= 0; --d) {
                    const u64 add = by_weight ? bins[d] : counts[d];
                    if (counts[d]) lowest = d;
                    if (add && (double)(sum + add) >= aim) {
                        at = d;
                        break;
                    }
                    sum += add;
                }
                if (at < 0) at = lowest, sum -= by_weight ? bins[lowest] : counts[lowest];   // (all of them)
                found[0] = sum, found[1] = counts[at], found[2] = bins[at], found[3] = at;
            }
            __syncthreads();
            before = found[0], n = found[1], group = found[2];
            key |= (uint32_t)found[3] << shift;
        }
        __syncthreads();
    };
    u64 ties = 0, n = 0, before = 0, group = 0;
    cut = kKeyNothing;
    if (ask.top_k > 0) {
        prefix((double)ask.top_k, false, cut, n, before, group);
        ties = min(n, (u64)max((int64_t)ask.top_k - (int64_t)before, (int64_t)0));
        lim_key = cut, lim_n = ties;
    }
    if (ask.by_p()) {
        double S = 0.0;
        each([&](int, float x) { S += key_of(x) > lim_key ? w(x) : 0.0; });
        S = block_sum<NT>(S, tmp);
        if (lim_n) S += (double)lim_n * w(logit_of(lim_key));
        const double aim = share_of(ask.top_p, S);
        prefix(aim, true, cut, n, before, group);
        const u64 one = group / max(n, 1ull);
        ties = one ? min(n, ((u64)aim - before + one - 1) / one) : n;
    }
    // the index of the last equal logit that is in, threads owning ranges of pieces
    const int per = (pieces + NT - 1) / NT, a = min(pieces, tid * per), b = min(pieces, a + per);
    if (tid == 0) found[0] = kNoEntry;
    double mine = 0.0;
    for (int c = a; c < b; ++c) {
        float x[VEC];
        row.load(c, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) mine += key_of(x[e]) == cut && x[e] > -INFINITY;
    }
    u64 at = (u64)block_excl_d<NT>(mine, tmp);
    if (cut != kKeyNothing && at < ties && ties <= at + (u64)mine)
        for (int c = a; c < b; ++c) {
            float x[VEC];
            row.load(c, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (key_of(x[e]) == cut && x[e] > -INFINITY && ++at == ties) found[0] = (u64)(row.first(c) + e);
        }
    __syncthreads();
    last = (int)(uint32_t)found[0];
    __syncthreads();
}

// ---- the second list
template <typename T>
__global__ __launch_bounds__(kGatherThreads) void pick_gather_k(PickGeo geo, const T* logits, int64_t row_stride, PickFilter filter, PickWs ws, PickOut out) {
    constexpr int VEC = RowView<T>::VEC, NT = kGatherThreads, NW = NT / 64;
    __shared__ u64 buf[kGather];
    __shared__ double tmp[16], part[kSegsMost * 8];
    __shared__ int flag;
    const int lr = blockIdx.x / geo.segs, g = blockIdx.x - lr * geo.segs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = geo.row0 + lr;
    PickRow* pr = ws.row + lr;
    const int state = pr->state;
    if (state == kDone || (state == kStepwise && g != 0)) return;
    const RowView<T> row(logits + (int64_t)r * row_stride, geo.V);
    const Asked ask = asked_of(filter, r / geo.rows_per_seq, geo.V);
    const Weigh w(row_top(geo, ws, lr), ask.tau);
    const double whole = pr->whole;
    const int wper = (geo.per + NW - 1) / NW, ranges = geo.segs * 8;
    if (state != kStepwise) {
        const float per_logit = bins_per_logit(ask, geo.V);
        const int hi = pr->bin, lo = state == kBinAlone ? hi : 0;
        const int seg_end = min(row.pieces(), (g + 1) * geo.per), c0 = min(seg_end, g * geo.per + wave * wper), c1 = min(seg_end, c0 + wper);
        double kept = 0.0;
        uint32_t kept_n = 0;
        for (int c = c0 + lane; c < c1; c += 64) {
            float x[VEC];
            row.load(c, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int b = bin_of(w, x[e], per_logit);
                if (b < lo) {
                    if (out.token) {
                        const double weight = w(x[e]);
                        const bool in = weight >= ask.least;
                        kept += in ? weight : 0.0, kept_n += in;
                    }
                } else if (b <= hi && x[e] > -INFINITY) {
                    const uint32_t at = atomicAdd(&pr->gather_n, 1u);
                    if (at < (uint32_t)kGather) ws.gather[(int64_t)lr * kGather + at] = entry_of(x[e], row.first(c) + e);
                }
            }
        }
        kept = wave_sum_d(kept);
        for (int o = 32; o > 0; o >>= 1) kept_n += __shfl_xor(kept_n, o, 64);
        if (lane == 0) ws.part[lr * ranges + g * 8 + wave] = kept, ws.part_n[lr * ranges + g * 8 + wave] = kept_n;
        if (!last_here(&pr->seen_gather, geo.segs, &flag)) return;
        const uint32_t n = pr->gather_n;
        int end = -1;
        if (n <= (uint32_t)kGather) {
            const int size = power_above((int)n);
            for (int i = tid; i < size; i += NT) buf[i] = i < (int)n ? ws.gather[(int64_t)lr * kGather + i] : kNoEntry;
            sort_entries<NT>(buf, size);
            end = end_in_list<NT>(buf, (int)n, ask, w, pr->before_w, pr->before_n, whole, false, tmp, &flag);
        }
        if (end > 0) {
            const u64 e = buf[end - 1];
            const Kept in{~(uint32_t)(e >> 32), (int)(uint32_t)e, ask.least};
            if (tid == 0) pr->cut = in.cut, pr->last = in.last;
            __syncthreads();
            if (!out.token) return;
            if (state == kAllDownTo) {
                draw_from_list<NT>(buf, end, ask, w, tmp, out, r, whole);
                return;
            }
            // the listed ones join the sums of their ranges
            for (int i = tid; i < ranges; i += NT) part[i] = ws.part[lr * ranges + i];
            double count = 0.0;
            for (int i = tid; i < ranges; i += NT) count += ws.part_n[lr * ranges + i];
            __syncthreads();
            for (int i = tid; i < end; i += NT) {
                const double x = w(entry_logit(buf[i]));
                if (x < ask.least) continue;
                const int c = ((int)(uint32_t)buf[i] + row.off) / VEC, seg = c / geo.per;
                atomicAdd(&part[seg * 8 + (c - seg * geo.per) / wper], x);
                count += 1.0;
            }
            count = block_sum<NT>(count, tmp);
            if (tid == 0 && out.kept) out.kept[r] = (int32_t)count;
            double S = 0.0, base = 0.0;
            for (int i = 0; i < ranges; ++i) S += part[i];
            const double aim = aim_of(out.u[r], S);
            int at = -1;
            for (int i = 0; i < ranges && at < 0; ++i) {
                if (base + part[i] > aim) at = i;
                else base += part[i];
            }
            if (at < 0) return;   // (cannot be)
            const int stop = min(row.pieces(), ((at >> 3) + 1) * geo.per), p0 = min(stop, (at >> 3) * geo.per + (at & 7) * wper), p1 = min(stop, p0 + wper);
            draw_from<NT>(row, p0, p1, w, in, base, [&](double, double& sum) { sum = S; return aim; }, tmp, out, r, whole);
            return;
        }
        __syncthreads();
    }
    Kept in{0, 0, ask.least};
    cut_stepwise<NT>(row, ask, w, buf, tmp, in.cut, in.last);
    if (tid == 0) pr->cut = in.cut, pr->last = in.last;
    if (!out.token) return;
    if (out.kept) {
        double count = 0.0;
        for (int c = tid; c < row.pieces(); c += NT) {
            float x[VEC];
            row.load(c, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) count += in(w, row.first(c) + e, x[e]) && x[e] > -INFINITY;
        }
        count = block_sum<NT>(count, tmp);
        if (tid == 0) out.kept[r] = (int32_t)count;
    }
    draw_from<NT>(row, 0, row.pieces(), w, in, 0.0, [&](double all, double& sum) { sum = all; return aim_of(out.u[r], all); }, tmp, out, r, whole);
}

// ---- filtered rows
template <typename T>
__global__ __launch_bounds__(kWeighThreads) void pick_mask_k(PickGeo geo, const T* logits, int64_t row_stride, PickFilter filter, PickWs ws, PickOut out) {
    constexpr int VEC = RowView<T>::VEC, NT = kWeighThreads;
    __shared__ double tmp[16];
    const int lr = blockIdx.x / geo.segs, g = blockIdx.x - lr * geo.segs, tid = threadIdx.x, r = geo.row0 + lr;
    const RowView<T> row(logits + (int64_t)r * row_stride, geo.V);
    const Asked ask = asked_of(filter, r / geo.rows_per_seq, geo.V);
    const PickRow& pr = ws.row[lr];
    const bool copy = pr.cut == 0;
    const Weigh w(row_top(geo, ws, lr), ask.tau);
    const Kept in{pr.cut, pr.last, ask.least};
    T* o = (T*)out.rows + (int64_t)r * out.rows_stride;
    const bool wide = ((uintptr_t)o & 15) == ((uintptr_t)row.row & 15);
    const int c1 = min(row.pieces(), (g + 1) * geo.per);
    uint32_t count = 0;
    for (int c = g * geo.per + tid; c < c1; c += NT) {
        float x[VEC];
        row.load(c, x);
        const int j = row.first(c);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (!copy) {
                const bool keep = x[e] > -INFINITY && in(w, j + e, x[e]);
                count += keep;
                if (!keep) x[e] = -INFINITY;
            }
        if (wide && j >= 0 && j + VEC <= geo.V) {
            u32x4_t v;
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(x[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(x[2 * e]) >> 16 | (__float_as_uint(x[2 * e + 1]) & 0xffff0000u);   // (values of T: exact)
            }
            *(u32x4_t*)(o + j) = v;
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (j + e >= 0 && j + e < geo.V) o[j + e] = from_float<T>(x[e]);
        }
    }
    if (!out.kept) return;
    const double all = block_sum<NT>((double)count, tmp);
    if (tid == 0 && all > 0.0) atomicAdd(&out.kept[r], (int32_t)all);
}

// ---- host
static int pick_segs(int rows, int vocab) {
    // some 1024 workgroups, of 2048 tokens at least
    return std::max(1, std::min({kSegsMost, 1024 / std::min(rows, kBatchRows), vocab / 2048}));
}
static size_t pick_carve(int rows, int vocab, char* base, PickWs* ws) {
    const size_t R = (size_t)std::min(rows, kBatchRows), S = (size_t)pick_segs(rows, vocab);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* p = base + at;
        at += (bytes + 255) / 256 * 256;
        return (void*)p;
    };
    PickWs w;
    w.row = (PickRow*)take(R * sizeof(PickRow));
    w.top = (float*)take(R * S * 4);
    w.sample = (float*)take(R * kSamples * 4);
    w.whole = (double*)take(R * S * 8);
    w.part = (double*)take(R * S * 64);
    w.part_n = (uint32_t*)take(R * S * 32);
    w.list = (u64*)take(R * kList * 8);
    w.gather = (u64*)take(R * kGather * 8);
    w.bin_w = (u64*)take(R * S * kBins * 8);
    w.bin_n = (uint32_t*)take(R * S * kBins * 4);
    if (ws) *ws = w;
    return at;
}
size_t pick_workspace_bytes(int rows, int vocab) { return pick_carve(rows, vocab, nullptr, nullptr); }

template <typename T>
static void pick_rounds(hipStream_t s, int rows, int rows_per_seq, int vocab, const T* logits, int64_t row_stride, const PickFilter& filter, const PickOut& out, char* base) {
    PickWs ws;
    pick_carve(rows, vocab, base, &ws);
    PickGeo geo;
    geo.V = vocab;
    geo.segs = pick_segs(rows, vocab);
    constexpr int VEC = RowView<T>::VEC;
    geo.pieces = (vocab + 2 * VEC - 2) / VEC;
    geo.per = (geo.pieces + geo.segs - 1) / geo.segs;
    geo.samples = kWeighThreads;
    while (geo.samples * geo.segs > kSamples) geo.samples >>= 1;
    geo.rows_per_seq = rows_per_seq;
    for (int r0 = 0; r0 < rows; r0 += kBatchRows) {
        geo.row0 = r0;
        const dim3 grid((unsigned)(std::min(kBatchRows, rows - r0) * geo.segs));
        hipLaunchKernelGGL(pick_max_k<T>, grid, dim3(kWeighThreads), 0, s, geo, logits, row_stride, ws, out);
        hipLaunchKernelGGL(pick_weigh_k<T>, grid, dim3(kWeighThreads), 0, s, geo, logits, row_stride, filter, ws, out);
        hipLaunchKernelGGL(pick_gather_k<T>, grid, dim3(kGatherThreads), 0, s, geo, logits, row_stride, filter, ws, out);
        if (out.rows) hipLaunchKernelGGL(pick_mask_k<T>, grid, dim3(kWeighThreads), 0, s, geo, logits, row_stride, filter, ws, out);
    }
}

hipError_t pick(hipStream_t s, int dtype, int rows, int rows_per_seq, int vocab, const void* logits, int64_t row_stride, const PickFilter& filter,
                const PickOut& out, void* ws, size_t ws_bytes) {
    if (ws_bytes < pick_workspace_bytes(rows, vocab)) return hipErrorInvalidValue;
    if (dtype == F32)
        pick_rounds<float>(s, rows, rows_per_seq, vocab, (const float*)logits, row_stride, filter, out, (char*)ws);
    else
        pick_rounds<bf16>(s, rows, rows_per_seq, vocab, (const bf16*)logits, row_stride, filter, out, (char*)ws);
    return hipGetLastError();
}

}  // namespace tlt
