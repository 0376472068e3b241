// Sampling from rows of logits behind top-k, top-p and min-p: one token per row, or the row with all other tokens at -infinity.
//
// Weights are whole numbers W = floor(exp(l / tau - max / tau) * 2^32), so sums do not depend on their order; they are held as doubles, which are exact up to 2^53 (2^20 tokens,
// 2^52).  (The acceptance rules form them by another formula; a few in a million at most differ by one.)  What is kept is a prefix of the order (logit falling, index rising), given by the logit it ends in
// and the last index kept of those equal to it (cut, last below), and of that what weighs enough.  Equal logits have equal weights.
//
// A row is cut into segments, a workgroup each, and read two or three times:
//   pick_max_k     the largest logit, and how far down the most likely few hundred tokens reach
//   pick_weigh_k   all weights; the likely few hundred tokens go to a list, and weights go to a histogram over the distance to the largest logit where the list may not reach the
//                  prefix's end.  The last workgroup of a row finds that end in the list, or the histogram's bin that holds it
//   pick_gather_k  only where the list did not reach: the tokens of that bin (or all down to it) go to a list, what is above is summed up
//   pick_mask_k    for filtered rows
// What has to be read and written once would take 35 us for 256 rows of 152064 in fp32 (156 MB); here they take 31 us for the maximum (5.0 TB/s), 66 for the weights (42 vector instructions per
// element, half of them in double, 83 % of the cycles; 16 instructions an element take as long as reading it), 41 for the second list.  One row is a chain of about 25 us: three launches, in the second 2.5 us of sums over the segments, 5 of reading, 2 of
// meeting, 9 of searches in LDS.  Many filtered rows (pick_row_k) and vocabularies up to 4096 (pick_small_k) have kernels of their own.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "dev_common.h"
#include "kernels.h"

namespace tlt {

typedef unsigned long long u64;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kWeighThreads = 256, kGatherThreads = 512, kRowThreads = 1024;
// Rows that the segments' kernels take at a time, for which the workspace has room (0.1 MB a row).  1024 rows of 152064 with top-p: 437 us at once, 474 in two halves, 549 in quarters; a workgroup per row 528.
constexpr int kPassRows = 1024;
// From there on filtered rows are a workgroup's each: a row is read again while it is near.  Of 152064 tokens, by segments and by a workgroup each: 128 rows with top-k and top-p 80 and 73 us, with top-p 100 and
// 124, of mixed settings 98 and 156; 192 rows 115 and 99, 147 and 146, 150 and 175; 256 rows 149 and 129, 186 and 164, 182 and 190; 1536 rows of mixed settings 852 and 712.
constexpr int kFewRows = 192;
constexpr int kSegsMost = 32;                        // (a power of two)
constexpr int kBins = 512;                           // of a row's histogram
constexpr int kFindBins = 256, kFindFew = 64;        // of a search in a list, and tokens that are compared with each other
constexpr int kList = 4096, kWaveList = 1024;        // entries of a row's list of likely tokens, and of what a wave may add (4096 in all: the row's list lies in their place)
constexpr int kGather = 8192;                        // entries of the second list
// vocabularies up to here are one list: one row of 4096 15.7 us, 20.9 by segments; 256 rows 22.5 and 38.3; of 1025 10.1 and 18.4, 12.0 and 34.0
constexpr int kSmall = 4096;
// numbers of groups whose largest logits show how far the likely tokens reach: 64 << k
constexpr int kGroups = 3, kListed = 64 << (kGroups - 1);   // and the largest top_k that lists are made for
// 16-byte pieces a lane asks for at once: in kernels that mostly move data (filtered rows 32 x 48 712 us, 740 with 2), and in those that compute, where they are asked for ahead (64 rows of 152064 62 us, 66 with 4)
constexpr int kInFlight = 4, kAhead = 2;
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
// the request's numbers as they are (loaded before they are needed)
struct Wish {
    float tau, p, m;
    int k;
    __device__ __forceinline__ Wish(const PickFilter& f, int seq)
        : tau(f.temperature ? f.temperature[seq] : 1.f), p(f.top_p ? f.top_p[seq] : 1.f), m(f.min_p ? f.min_p[seq] : 0.f), k(f.top_k ? f.top_k[seq] : 0) {}
    // tokens: of the row, above -infinity
    __device__ __forceinline__ Asked asked(int tokens) const {
        Asked a{1.0, 1, 1u << 31, 0.0};
        if (!(tau > 0.f)) return a;
        a.tau = (double)tau;
        a.top_k = k < tokens ? max(k, 0) : 0;
        if (p < 1.f) a.top_p = (uint32_t)(fmax((double)p, 0.0) * 2147483648.0);
        if (m > 0.f) a.least = floor(fmin((double)m, 1.0) * 4294967296.0);
        return a;
    }
};
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
    // (the largest is +infinity: 2^128 in its place, from which those tokens are cut to distance 0 and all others are far)
    __device__ __forceinline__ Weigh(float largest, double tau_) : tau(tau_) {
        const bool inf = largest == INFINITY;
        top_f = inf ? FLT_MAX : largest;
        top = inf ? 0x1p128 : (double)largest;
        scale = inf ? 1.0 : 1.4426950408889634074 / tau_;
    }
    // how far below the largest, for bins: does not fall from a token to one with a smaller logit
    __device__ __forceinline__ float distance(float x) const { return fmaxf(top_f - x, 0.f); }
    __device__ __forceinline__ double operator()(float x) const {
        const double t = fmin(fmax(((double)x - top) * scale, -40.0), 0.0);   // (-infinity, and what infinities leave undefined, weigh nothing)
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
    __device__ __forceinline__ double below(float x) const { return (double)x >= top ? 0.0 : (double)x / tau - top / tau; }
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
    __device__ __forceinline__ bool inside(int c) const { return first(c) >= 0 && first(c) + VEC <= V; }
    __device__ __forceinline__ u32x4_t raw(int c) const { return *(const u32x4_t*)(row + first(c)); }
    static __device__ __forceinline__ void values(u32x4_t w, float (&x)[VEC]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) x[e] = __uint_as_float(w[e]);
            else x[2 * e] = __uint_as_float(w[e] << 16), x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4_t packed(const float (&x)[VEC]) {   // (values of T: exact)
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(x[e]);
            else w[e] = __float_as_uint(x[2 * e]) >> 16 | (__float_as_uint(x[2 * e + 1]) & 0xffff0000u);
        }
        return w;
    }
    // elements outside the row are -infinity
    __device__ __forceinline__ void load(int c, float (&x)[VEC]) const {
        if (inside(c)) {
            values(raw(c), x);
        } else {
            const int j = first(c);
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = j + e >= 0 && j + e < V ? to_float(row[j + e]) : -INFINITY;
        }
    }
    // f(piece, values) for pieces `from`, from + step, .. below `end`, N of them loaded at once (AHEAD: before the ones in front of them are worked on); pieces at `end` and behind it come as -infinity (f is called by whole
    // waves, whose lanes hold consecutive pieces).  The row has a piece that lies inside.
    template <bool AHEAD = false, typename F>
    __device__ __forceinline__ void each(int from, int step, int end, F f) const {
        constexpr int N = AHEAD ? kAhead : kInFlight;
        const int lane = threadIdx.x & 63, in0 = off ? 1 : 0, in1 = (V + off) / VEC;   // pieces in0 .. in1 - 1 lie inside
        u32x4_t w[N], next[N];
        auto ask = [&](int c, u32x4_t (&w)[N]) {
#pragma unroll
            for (int u = 0; u < N; ++u) w[u] = raw(min(max(c + u * step, in0), in1 - 1));
        };
        if (AHEAD) ask(from, next);
        for (int c = from; c - lane < end; c += N * step) {
            if (AHEAD) {
#pragma unroll
                for (int u = 0; u < N; ++u) w[u] = next[u];
                ask(c + N * step, next);   // (held inside the row)
            } else {
                ask(c, w);
            }
            if (c - lane < in0 || c - lane + (N - 1) * step + 63 >= min(end, in1)) {   // (uniform over the wave)
                const int behind = in1 * VEC < V + off ? in1 : -1;   // the piece behind the last whole one
                u32x4_t part = {};
                if (c == 0 && in0) w[0] = partly(0);
                bool is = false;
#pragma unroll
                for (int u = 0; u < N; ++u) is |= c + u * step == behind;
                if (is) part = partly(behind);
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    const int at = c + u * step;
                    const bool in = at < end && (at < in1 || at == behind);
                    float x[VEC];
                    values(at == behind ? part : w[u], x);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[e] = in ? x[e] : -INFINITY;
                    w[u] = packed(x);
                }
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                float x[VEC];
                values(w[u], x);
                f(c + u * step, x);
            }
        }
    }
    // a piece of which a part lies outside
    __device__ __forceinline__ u32x4_t partly(int c) const {
        float x[VEC];
        load(c, x);
        return packed(x);
    }
};

// Places in a list for the wave's lanes with `is`, from a counter in LDS
__device__ __forceinline__ uint32_t place(bool is, uint32_t* n) {
    const uint64_t all = __ballot(is);
    if (all == 0) return 0;
    uint32_t first = 0;
    if ((threadIdx.x & 63) == 0) first = atomicAdd(n, (uint32_t)__popcll(all));
    return __builtin_amdgcn_readfirstlane(first) + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
}

// Weights of a wave's scattered tokens: their logits are put side by side first, 64 at a time, so that the lanes of the arithmetic are full (buf: 128 floats of LDS).
struct SparseSum {
    float* buf;
    double least, sum = 0.0;   // of this lane: to be added up over the wave
    uint32_t count = 0, n = 0;
    __device__ __forceinline__ void take(const Weigh& w, uint32_t many) {
        const int lane = threadIdx.x & 63;
        const double x = (uint32_t)lane < many ? w(buf[lane]) : -1.0;
        const bool in = x >= least && x >= 0.0;
        sum += in ? x : 0.0, count += in;
    }
    __device__ __forceinline__ void add(const Weigh& w, bool is, float x) {
        const uint64_t all = __ballot(is);
        if (all == 0) return;
        const int lane = threadIdx.x & 63;
        if (is) buf[n + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0))] = x;
        n += (uint32_t)__popcll(all);
        if (n < 64) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        take(w, 64);
        const float rest = buf[64 + lane];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        buf[lane] = rest;
        n -= 64;
    }
    __device__ __forceinline__ void finish(const Weigh& w) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (n) take(w, n);
    }
};

// ---- sums over a workgroup of NT threads, or over one wave (NT = 64), which needs no barrier
template <int NT>
__device__ __forceinline__ void together() {
    if constexpr (NT == 64) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}
// sum over the lanes up to this one: within rows of 16 lanes by shifts, then from row to row (data-parallel moves; a shuffle is a trip through LDS)
__device__ __forceinline__ double wave_incl(double v) {
    auto add = [&](auto ctrl, auto rows) {
        const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
        v += __hiloint2double(hi, lo);
    };
    add(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr:1
    add(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast:15
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast:31
    return v;
}
__device__ __forceinline__ double lane_63(double v) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63), __builtin_amdgcn_readlane(__double2loint(v), 63));
}
__device__ __forceinline__ double wave_sum_d(double v) { return lane_63(wave_incl(v)); }
template <int NT>
__device__ __forceinline__ double block_sum(double v, double* tmp) {
    v = wave_sum_d(v);
    if constexpr (NT == 64) return v;
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
    const double incl = wave_incl(v);
    if constexpr (NT == 64) return incl - v;
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) tmp[wave] = incl;
    __syncthreads();
    double base = 0.0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) base += w < wave ? tmp[w] : 0.0;
    return base + incl - v;
}

// ---- tokens in a list in LDS: entry_of, and the weights where there is room for them (they are formed when they are asked for otherwise): S double, or uint32_t, which holds half as many bytes, all
// weights but the largest two, and costs a comparison
template <typename S>
struct TokenList {
    const u64* e;
    const S* stored;
    Weigh w;
    int n;
    static constexpr uint32_t kFull = 0xffffffffu;   // this, or the one weight above it
    __device__ __forceinline__ double weight(int i) const {
        if constexpr (std::is_same<S, double>::value) return stored ? stored[i] : w(entry_logit(e[i]));
        const uint32_t x = stored ? (uint32_t)stored[i] : kFull;
        return x != kFull ? (double)x : w(entry_logit(e[i]));
    }
    static __device__ __forceinline__ S held(double weight) { return std::is_same<S, double>::value ? (S)weight : (S)fmin(weight, 4294967295.0); }
};
struct FindLds {
    u64 bins[kFindBins], order[kFindFew];
    double value[kFindFew], base;
    u64 found;
    uint32_t n;
    int bin;
};
// The first of the list's active tokens, in ascending order of `order` (all different), with which the running sum of `value` (whole numbers) reaches `aim`; kNoEntry: none.
// Bins by `bin` (which does not fall in that order), then evenly over the orders of the bin in which it happens, until that holds few tokens, which are compared with each other.
template <int NT, typename O, typename A, typename F, typename G>
__device__ u64 locate(int n, O order, A active, F value, G bin, double aim, FindLds& s, double* tmp) {
    const int tid = threadIdx.x;
    constexpr int B = NT < kFindBins ? kFindBins / NT : 1;
    double base = 0.0, per = 0.0;
    u64 lo = 0, hi = kNoEntry - 1;
    auto bin_at = [&](int i, u64 o) { return per == 0.0 ? bin(i) : (int)((double)(o - lo) * per); };
    for (;;) {
        for (int i = tid; i < kFindBins; i += NT) s.bins[i] = 0;
        if (tid == 0) s.n = 0, s.found = kNoEntry, s.bin = -1;
        together<NT>();
        for (int i = tid; i < n; i += NT) {
            const u64 o = order(i);
            if (o >= lo && o <= hi && active(i)) atomicAdd(&s.bins[bin_at(i, o)], (u64)__double_as_longlong(value(i) + 0x1p52) & 0xfffffffffffffull);
        }
        together<NT>();
        double mine[B], sum = 0.0;
#pragma unroll
        for (int k = 0; k < B; ++k) mine[k] = tid * B + k < kFindBins ? (double)s.bins[tid * B + k] : 0.0, sum += mine[k];
        double run = base + block_excl_d<NT>(sum, tmp);
#pragma unroll
        for (int k = 0; k < B; ++k) {
            if (run < aim && aim <= run + mine[k]) s.bin = tid * B + k, s.base = run;
            run += mine[k];
        }
        together<NT>();
        const int at = s.bin;
        if (at < 0) return kNoEntry;   // (uniform)
        base = s.base;
        for (int i = tid; i < n; i += NT) {
            const u64 o = order(i);
            if (o >= lo && o <= hi && active(i) && bin_at(i, o) == at) {
                const uint32_t m = atomicAdd(&s.n, 1u);
                if (m < (uint32_t)kFindFew) s.order[m] = o, s.value[m] = value(i);
            }
        }
        together<NT>();
        const uint32_t m = s.n;
        if (m <= (uint32_t)kFindFew) {
            if ((uint32_t)tid < m) {
                const u64 mine_at = s.order[tid];
                double before = base;
#pragma unroll 4
                for (uint32_t j = 0; j < m; ++j) before += s.order[j] < mine_at ? s.value[j] : 0.0;
                if (before < aim && aim <= before + s.value[tid]) s.found = mine_at;
            }
            together<NT>();
            const u64 found = s.found;
            together<NT>();
            return found;
        }
        // the range of the bin's tokens
        if (tid == 0) s.order[0] = kNoEntry, s.order[1] = 0;
        together<NT>();
        u64 first = kNoEntry, last = 0;
        for (int i = tid; i < n; i += NT) {
            const u64 o = order(i);
            if (o >= lo && o <= hi && active(i) && bin_at(i, o) == at) first = min(first, o), last = max(last, o);
        }
        if (first != kNoEntry) atomicMin(&s.order[0], first), atomicMax(&s.order[1], last);   // (not `last`: in the order of indices token 0 is 0)
        together<NT>();
        lo = s.order[0], hi = s.order[1];
        per = (double)kFindBins / ((double)(hi - lo) + 1.0) * (1.0 - 0x1p-40);
        together<NT>();
    }
}

// ---- what the workgroups of a row share
enum { kOpen = 0, kDone = 1, kByWeight = 2, kByNumber = 3, kAllDownTo = 4, kStepwise = 5 };
struct PickRow {
    uint32_t list_n, gather_n, seen_weigh, seen_gather;
    int32_t state;
    int32_t bin_lo, bin_hi;     // bins to gather: the one that the end lies in (kByWeight: of top_p; kByNumber: of top_k), or all down to it (kAllDownTo)
    uint32_t cut;               // the result: kept are keys above it and those equal to it up to index `last`; 0: the row is copied
    int32_t last;
    double before, whole;       // weight (kByWeight) or number (kByNumber) of the tokens above those bins
};
struct PickWs {
    PickRow* row;
    float *top, *reach;      // [rows][segs], [rows][segs][kGroups]: the least of the largest logits of a segment's groups
    uint32_t* groups;        // [rows][segs][kGroups]: how many of them have a token
    uint32_t* tokens;        // [rows][segs]: tokens above -infinity
    double *whole, *part;    // [rows][segs], [rows][segs * 8]: sums of kept weights over the ranges of waves
    uint32_t* part_n;        // their counts
    u64 *list, *gather;      // [rows][kList], [rows][kGather]
    u64* bins;               // [rows][segs][kBins]
};
struct PickGeo {
    int V, segs, per;         // per: pieces of a segment
    int rows_per_seq, row0;   // row0: first row of this launch
};

// What one workgroup of a row leaves for another of the same launch goes past the caches of an XCD, both ways, so that nothing has to be written back or dropped where they meet: a meeting takes 0.7 us of the
// last workgroup, 4.1 with ordinary stores and a release that writes the cache back, and its list is there after 1.3 us instead of 5.8 (64 rows of 152064).
template <typename V>
__device__ __forceinline__ void leave(V* to, V v) { __hip_atomic_store(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename V>
__device__ __forceinline__ V left(const V* from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// The workgroup that is the last of `total` of a row to come here sees what all of them left (every wave waits until its stores are done, then one thread counts).
__device__ __forceinline__ bool last_here(uint32_t* seen, int total, int* flag) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) *flag = __hip_atomic_fetch_add(seen, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)total - 1u;
    __syncthreads();
    return *flag != 0;
}

// bins per logit, downwards from the largest one; at or past kBins a token is below them.  likely: how far down a thousand or two of the tokens reach.
__device__ __forceinline__ float bins_per_logit(const Asked& ask, int V, float likely) {
    // tokens whose weight is below (1 - p) 2^32 / V cannot be in the shortest prefix of weight p S, as S >= 2^32 and together they are less than (1 - p) S; otherwise
    // down to where weights are 0, and for a number of tokens, which may be many of those, to where most tokens are (four times as far as the likely ones, in a bell)
    double reach = 23.0 * ask.tau;
    if (ask.top_k == 0) reach = fmin(reach, ask.tau * (0.01 + log((double)V / fmax(1.0 - (double)ask.top_p * 0x1p-31, 1e-10))));
    else if (likely > 0.f) reach = fmax(reach, 4.0 * (double)likely);
    return (float)fmin((double)kBins / reach, 1e30);
}
// Is every token that weighs anything in a bin?  (In front of which the bins end where weights are 0; a difference that fp32 does not hold is in none, and at such a temperature it may weigh.)
__device__ __forceinline__ bool bins_hold_all(const Asked& ask) { return 23.0 * ask.tau <= (double)FLT_MAX; }
__device__ __forceinline__ float bin_of(const Weigh& w, float x, float per_logit) { return w.distance(x) * per_logit; }   // (its whole part; NaN: below them)

// ---- outputs
__device__ __forceinline__ void put_nothing(const PickOut& out, int r, bool nan) {
    if (out.token) out.token[r] = -1;
    if (out.logprob) out.logprob[2 * r] = out.logprob[2 * r + 1] = nan ? NAN : -INFINITY;
    if (out.kept) out.kept[r] = 0;
}
// what a draw has found (in LDS), written out once
struct Drawn {
    double S;
    int token;
    float logit;
};
__device__ __forceinline__ void put_token(int32_t* token, float* logprob, const Weigh w, const Drawn& d, double whole) {
    *token = d.token;
    if (logprob) {
        const double z = w.below(d.logit);
        logprob[0] = (float)(z - log(d.S * 0x1p-32));
        logprob[1] = (float)(z - log(whole * 0x1p-32));
    }
}

struct Kept {
    uint32_t cut;
    int last;
    double least;
    __device__ __forceinline__ bool operator()(const Weigh& w, int j, float x) const {
        const uint32_t k = key_of(x);
        bool in = (k > cut) | ((k == cut) & (j <= last));
        if (least != 0.0) in &= w(x) >= least;   // (the same for all lanes)
        return in;
    }
};

// The first token of pieces [c0, c1) whose running sum, from `base` on, of kept weights exceeds (u * S) >> 32.  S < 0: the sum over the pieces.
template <int NT, typename T>
__device__ __forceinline__ void draw_from(const RowView<T> row, int c0, int c1, const Weigh w, const Kept kept, double base, double S, uint32_t u, double* tmp, Drawn* drawn) {
    constexpr int VEC = RowView<T>::VEC;
    const int per = (c1 - c0 + NT - 1) / NT, a = min(c1, c0 + (int)threadIdx.x * per), b = min(c1, a + per);
    double mine = 0.0;
    for (int c = a; c < b; ++c) {
        float x[VEC];
        row.load(c, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) mine += kept(w, row.first(c) + e, x[e]) ? w(x[e]) : 0.0;
    }
    if (S < 0.0) S = block_sum<NT>(mine, tmp);
    double run = base + block_excl_d<NT>(mine, tmp);
    const double aim = aim_of(u, S);
    if (run <= aim && aim < run + mine) {
        bool found = false;
        for (int c = a; c < b && !found; ++c) {
            float x[VEC];
            row.load(c, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const double add = !found && kept(w, row.first(c) + e, x[e]) ? w(x[e]) : 0.0;
                run += add;
                if (add > 0.0 && run > aim) drawn->S = S, drawn->token = row.first(c) + e, drawn->logit = x[e], found = true;
            }
        }
    }
    __syncthreads();
}

// Where the prefix ends in a list whose tokens follow on before_n others of weight before_w: its last token, or kNoEntry if it ends behind them.  n of the list's entries are
// tokens, nearly all between the logits `best` and `least`.  S: the weight that top_p is a share of, for rows without top_k.  all: what is not in the list weighs nothing (a
// top_k that reaches behind it, with top_p, then leaves the share of the whole list).
template <int NT, typename L>
__device__ __forceinline__ u64 end_in_list(const L l, int n, const Asked ask, double before_w, double before_n, double S, float best, float least, bool all, FindLds& s, double* tmp) {
    u64 end = kNoEntry - 1;   // (above every entry)
    auto order = [&](int i) { return l.e[i]; };
    // evenly over the distances from `best`
    const float near = l.w.distance(best), per = fminf((float)(kFindBins - 1) / (l.w.distance(least) - near), 1e30f);
    auto bin = [&](int i) { return min((int)fminf(fmaxf(l.w.distance(entry_logit(l.e[i])) - near, 0.f) * per, 1e6f), kFindBins - 1); };
    if (ask.top_k > 0) {
        const double aim = (double)ask.top_k - before_n;
        if (aim <= (double)n) end = locate<NT>(l.n, order, [](int) { return true; }, [](int) { return 1.0; }, bin, aim, s, tmp);
        else if (!all) return kNoEntry;
        if (ask.by_p()) {
            double mine = 0.0;
            for (int i = threadIdx.x; i < l.n; i += NT) mine += l.e[i] <= end ? l.weight(i) : 0.0;
            S = before_w + block_sum<NT>(mine, tmp);
        }
    }
    if (ask.by_p()) return locate<NT>(l.n, order, [&](int i) { return l.e[i] <= end; }, [&](int i) { return l.weight(i); }, bin, share_of(ask.top_p, S) - before_w, s, tmp);
    return end;
}

// Draws from the list's tokens up to `end`, which are all that is kept but for `least`.
template <int NT, typename L>
__device__ __forceinline__ void draw_from_list(const L l, u64 end, double least, int V, FindLds& s, double* tmp, int32_t* kept, uint32_t u, Drawn* drawn) {
    auto in = [&](int i) { return l.e[i] <= end && l.weight(i) >= least; };
    double S = 0.0, count = 0.0;
    for (int i = threadIdx.x; i < l.n; i += NT) {
        const bool k = in(i);
        S += k ? l.weight(i) : 0.0, count += k;
    }
    S = block_sum<NT>(S, tmp);
    count = block_sum<NT>(count, tmp);
    if (threadIdx.x == 0) {
        if (kept) *kept = (int32_t)count;
        drawn->S = 1.0, drawn->token = -1, drawn->logit = -INFINITY;   // (a search that finds nothing draws nothing)
    }
    const double per = (double)kFindBins / ((double)V + 1.0);
    const u64 token = locate<NT>(l.n, [&](int i) { return l.e[i] & 0xffffffffull; }, in, [&](int i) { return l.weight(i); }, [&](int i) { return (int)((double)(uint32_t)l.e[i] * per); },
                                 aim_of(u, S) + 1.0, s, tmp);
    for (int i = threadIdx.x; i < l.n; i += NT)
        if (in(i) && (l.e[i] & 0xffffffffull) == token) drawn->S = S, drawn->token = (int)token, drawn->logit = entry_logit(l.e[i]);
    together<NT>();
}

// The range of a wave, of those that a row's segments are cut into, in which the running sum of `part` passes aim (NT threads, at most one range each); -1: none.
template <int NT>
__device__ int range_of(double mine, double aim, double& base, FindLds& s, double* tmp) {
    const double run = block_excl_d<NT>(mine, tmp);
    if (threadIdx.x == 0) s.bin = -1;
    __syncthreads();
    if (run <= aim && aim < run + mine) s.bin = threadIdx.x, s.base = run;
    __syncthreads();
    base = s.base;
    return s.bin;
}

// ---- the largest logit, and how far down the likely tokens reach: of 64, 128 or 256 groups of a row's tokens each has one that is not below the least of the groups' largest, so at least so many
// tokens reach that (some 300, 620 or 1600, if they are spread evenly).
template <typename T>
__global__ __launch_bounds__(kWeighThreads) void pick_max_k(PickGeo geo, const T* logits, int64_t row_stride, PickWs ws, PickOut out) {
    constexpr int VEC = RowView<T>::VEC, NW = kWeighThreads / 64;
    __shared__ float wave_top[NW], wave_reach[kGroups][NW];
    __shared__ uint32_t wave_groups[kGroups][NW], wave_tokens[NW];
    const int lr = blockIdx.x / geo.segs, g = blockIdx.x - lr * geo.segs, tid = threadIdx.x, wave = tid >> 6, r = geo.row0 + lr;
    const RowView<T> row(logits + (int64_t)r * row_stride, geo.V);
    float top = -INFINITY;
    bool nan = false;
    uint32_t tokens = 0;
    // (pieces of all parts of the row: where likely tokens have low indices, every group has its share of them)
    row.each(g * kWeighThreads + tid, geo.segs * kWeighThreads, row.pieces(), [&](int, const float (&x)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) nan |= x[e] != x[e], top = fmaxf(top, x[e]), tokens += x[e] > -INFINITY;
    });
    float s = top;
    int have = 1;   // lanes that share s
#pragma unroll
    for (int k = kGroups - 1; k >= 0; --k) {
        const int lanes = min(64, kWeighThreads * geo.segs / (64 << k));   // (a power of two; 128 lanes are two waves, joined below)
        for (; have < lanes; have <<= 1) s = fmaxf(s, __shfl_xor(s, have, 64));
        const uint64_t full = __ballot(s > -INFINITY);
        const float least = -wave_max(s > -INFINITY ? -s : -INFINITY);
        if ((tid & 63) == 0) wave_reach[k][wave] = least, wave_groups[k][wave] = (uint32_t)(__popcll(full) / lanes);
    }
    top = wave_max(top);
    if (__any(nan)) top = NAN;
    tokens = (uint32_t)wave_sum_d((double)tokens);
    if ((tid & 63) == 0) wave_top[wave] = top, wave_tokens[wave] = tokens;
    __syncthreads();
    if (tid < kGroups) {
        float least = INFINITY;
        uint32_t n = 0;
        const bool pairs = kWeighThreads * geo.segs / (64 << tid) > 64;
        for (int v = 0; v < NW; v += pairs ? 2 : 1) {
            float x = wave_reach[tid][v];
            uint32_t m = wave_groups[tid][v];
            if (pairs) x = wave_groups[tid][v + 1] == 0 ? x : (m == 0 ? wave_reach[tid][v + 1] : fmaxf(x, wave_reach[tid][v + 1])), m = max(m, wave_groups[tid][v + 1]);
            if (m) least = fminf(least, x), n += m;
        }
        ws.reach[(lr * geo.segs + g) * kGroups + tid] = least, ws.groups[(lr * geo.segs + g) * kGroups + tid] = n;
    }
    if (tid == 0) {
#pragma unroll
        for (int v = 1; v < NW; ++v) tokens += wave_tokens[v];
        ws.tokens[lr * geo.segs + g] = tokens;
#pragma unroll
        for (int v = 0; v < NW; ++v) top = top != top || wave_top[v] != wave_top[v] ? NAN : fmaxf(top, wave_top[v]);
        ws.top[lr * geo.segs + g] = top;
        if (g == 0) {
            PickRow z{};
            ws.row[lr] = z;
            if (out.rows && out.kept) out.kept[r] = 0;
        }
    }
}

// the row's largest logit; NaN if there is one
__device__ __forceinline__ float row_top(const PickGeo& geo, const PickWs& ws, int lr) {
    const int lane = threadIdx.x & 63;
    const float t = lane < geo.segs ? ws.top[lr * geo.segs + lane] : -INFINITY;
    return __any(t != t) ? NAN : wave_max(t);
}

__device__ __forceinline__ Asked asked_of_row(const PickGeo& geo, const PickWs& ws, int lr, const PickFilter& filter) {
    const Wish wish(filter, (geo.row0 + lr) / geo.rows_per_seq);
    const int lane = threadIdx.x & 63;
    const float n = wave_sum(lane < geo.segs ? (float)ws.tokens[lr * geo.segs + lane] : 0.f);   // (2^20 at most: exact)
    return wish.asked((int)n);
}

// A logit that at least `rank` tokens reach, by the groups that fit what is asked for.
__device__ __forceinline__ int level_of(const Asked& ask) { return ask.top_k <= 64 ? 0 : ask.top_k <= 128 ? 1 : 2; }
__device__ __forceinline__ float reached(const PickGeo& geo, const PickWs& ws, int lr, int level, int& rank) {
    const int lane = threadIdx.x & 63, at = (lr * geo.segs + lane) * kGroups + level;
    const float least = lane < geo.segs ? ws.reach[at] : INFINITY;
    rank = (int)wave_sum(lane < geo.segs ? (float)ws.groups[at] : 0.f);
    return fmaxf(-wave_max(-least), -FLT_MAX);
}

// ---- weights, list, histogram
template <typename T>
__global__ __launch_bounds__(kWeighThreads) void pick_weigh_k(PickGeo geo, const T* logits, int64_t row_stride, PickFilter filter, PickWs ws, PickOut out) {
    constexpr int VEC = RowView<T>::VEC, NT = kWeighThreads, NW = NT / 64;
    __shared__ u64 local[kList];          // the segment's list, then the row's
    __shared__ union {
        u64 bins[kBins];                  // while the segment is read
        FindLds find;                     // then
    } lds;
    __shared__ double tmp[16];
    __shared__ Drawn drawn;
    __shared__ int flag;
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
    const Asked ask = asked_of_row(geo, ws, lr, filter);
    const Weigh w(top, ask.tau);
    const bool prefix = ask.prefix();
    // tokens from `from` on go to the list
    int rank = 0;
    float from = prefix ? reached(geo, ws, lr, level_of(ask), rank) : INFINITY;
    const bool count_bins = ask.top_k > min(rank, kListed), use_bins = prefix && (count_bins || ask.top_k == 0);
    const float per_logit = use_bins ? bins_per_logit(ask, geo.V, w.distance(from)) : 0.f;
    if (count_bins) from = INFINITY;   // (no list reaches that far)
    const bool weigh_all = out.token ? !prefix || use_bins || out.logprob : use_bins;
    if (!prefix && !weigh_all) {   // (a filtered row without a prefix: what it keeps is known)
        if (g == 0 && tid == 0) pr->state = kDone, pr->cut = kKeyNothing, pr->last = -1;
        return;
    }
    if (use_bins)
        for (int i = tid; i < kBins; i += NT) lds.bins[i] = 0;
    __syncthreads();
    const int seg_end = min(row.pieces(), (g + 1) * geo.per), wper = (geo.per + NW - 1) / NW;
    const int c0 = min(seg_end, g * geo.per + wave * wper), c1 = min(seg_end, c0 + wper);
    double whole = 0.0, kept = 0.0;
    uint32_t kept_n = 0;
    u64* listing = local + wave * kWaveList;   // the wave's own list: no counter is shared while the segment is read
    uint32_t listed = 0;
    row.template each<true>(c0 + lane, 64, c1, [&](int c, const float (&x)[VEC]) {
        double weight[VEC];
        if (weigh_all) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                weight[e] = w(x[e]);
                whole += weight[e];
            }
        }
        if (!prefix) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const bool in = x[e] > -INFINITY && weight[e] >= ask.least;
                kept += in ? weight[e] : 0.0, kept_n += in;
            }
            return;
        }
        float best = x[0];
#pragma unroll
        for (int e = 1; e < VEC; ++e) best = fmaxf(best, x[e]);
        if (__any(best >= from)) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const bool in = x[e] >= from;
                const uint64_t all = __ballot(in);
                if (all == 0) continue;
                const uint32_t at = listed + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
                if (in && at < (uint32_t)kWaveList) listing[at] = entry_of(x[e], row.first(c) + e);
                listed += (uint32_t)__popcll(all);
            }
        }
        if (use_bins) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float b = bin_of(w, x[e], per_logit);
                if (b < (float)kBins) atomicAdd(&lds.bins[(int)b], count_bins ? 1ull : w.whole(weight[e]));
            }
        }
    });
    whole = block_sum<NT>(whole, tmp);
    if (tid == 0) leave(ws.whole + lr * geo.segs + g, whole);
    if (!prefix) {
        kept = wave_sum_d(kept);
        for (int o = 32; o > 0; o >>= 1) kept_n += __shfl_xor(kept_n, o, 64);
        if (lane == 0) leave(ws.part + (lr * geo.segs + g) * 8 + wave, kept), leave(ws.part_n + (lr * geo.segs + g) * 8 + wave, kept_n);
    } else {
        uint32_t base = 0;
        if (lane == 0) base = atomicAdd(&pr->list_n, listed > (uint32_t)kWaveList ? 1u << 20 : listed);
        base = __builtin_amdgcn_readfirstlane(base);
        listed = min(listed, (uint32_t)kWaveList);
        for (uint32_t i = lane; i < listed; i += 64)
            if (base + i < (uint32_t)kList) leave(ws.list + (int64_t)lr * kList + base + i, listing[i]);
        __syncthreads();   // (the bins)
        if (use_bins)
            for (int i = tid; i < kBins; i += NT) leave(ws.bins + ((int64_t)lr * geo.segs + g) * kBins + i, lds.bins[i]);
    }
    if (!last_here(&pr->seen_weigh, geo.segs, &flag)) return;

    // ---- the row's last workgroup.  (The list's beginning is asked for together with its length.)
    constexpr int kEarly = 8;
    u64 early[kEarly];
    if (prefix) {
#pragma unroll
        for (int i = 0; i < kEarly; ++i) early[i] = left(ws.list + (int64_t)lr * kList + i * NT + tid);
    }
    whole = wave_sum_d(lane < geo.segs ? left(ws.whole + lr * geo.segs + lane) : 0.0);
    if (tid == 0) pr->whole = whole;
    FindLds& find = lds.find;
    if (!prefix) {
        if (tid == 0) pr->state = kDone, pr->cut = kKeyNothing, pr->last = -1;
        if (!out.token) return;
        // the wave's range that holds the draw
        static_assert(kSegsMost * 8 <= NT, "a range per thread");
        const bool is = tid < geo.segs * 8 && (tid & 7) < NW;
        const double mine = is ? left(ws.part + lr * geo.segs * 8 + tid) : 0.0;
        const double S = block_sum<NT>(mine, tmp), count = block_sum<NT>(is ? (double)left(ws.part_n + lr * geo.segs * 8 + tid) : 0.0, tmp);
        if (tid == 0 && out.kept) out.kept[r] = (int32_t)count;
        const double aim = aim_of(out.u[r], S);
        double base;
        const int at = range_of<NT>(mine, aim, base, find, tmp);
        if (at < 0) return;   // (cannot be: S is the sum of the parts)
        const int end = min(row.pieces(), ((at >> 3) + 1) * geo.per), p0 = min(end, (at >> 3) * geo.per + (at & 7) * wper), p1 = min(end, p0 + wper);
        draw_from<NT, T>(row, p0, p1, w, Kept{kKeyNothing, -1, ask.least}, base, S, out.u[r], tmp, &drawn);
        if (tid == 0) put_token(out.token + r, out.logprob ? out.logprob + 2 * r : nullptr, w, drawn, whole);
        return;
    }
    const uint32_t n = left(&pr->list_n);
    if (n > 0 && n <= (uint32_t)kList) {
        double* stored = n <= kList / 2 ? (double*)(local + kList / 2) : nullptr;
#pragma unroll
        for (int i = 0; i < kEarly; ++i) {
            if ((uint32_t)(i * NT + tid) < n) local[i * NT + tid] = early[i];
            if (stored && (uint32_t)(i * NT + tid) < n) stored[i * NT + tid] = w(entry_logit(early[i]));
        }
        static_assert(kList <= 2 * kEarly * NT, "weights are stored for early ones alone");
#pragma unroll 4
        for (uint32_t i = kEarly * NT + tid; i < n; i += NT) local[i] = left(ws.list + (int64_t)lr * kList + i);
        __syncthreads();
        const TokenList<double> l{local, stored, w, (int)n};
        const u64 end = end_in_list<NT>(l, (int)n, ask, 0.0, 0.0, whole, top, from, false, find, tmp);
        if (end != kNoEntry) {
            if (tid == 0) pr->state = kDone, pr->cut = ~(uint32_t)(end >> 32), pr->last = (int32_t)(uint32_t)end;
            if (out.token) {
                draw_from_list<NT>(l, end, ask.least, geo.V, find, tmp, out.kept ? out.kept + r : nullptr, out.u[r], &drawn);
                if (tid == 0) put_token(out.token + r, out.logprob ? out.logprob + 2 * r : nullptr, w, drawn, whole);
            }
            return;
        }
    }
    if (!use_bins) {
        if (tid == 0) pr->state = kStepwise;
        return;
    }
    // The bin that the end lies in: thread t owns bins 2t and 2t + 1.
    constexpr int OWN = kBins / NT;
    u64 own[OWN] = {};
#pragma unroll 8
    for (int i = 0; i < geo.segs; ++i) {
        const u64* from_seg = ws.bins + ((int64_t)lr * geo.segs + i) * kBins + OWN * tid;
#pragma unroll
        for (int k = 0; k < OWN; ++k) own[k] += left(from_seg + k);
    }
    double mine = 0.0;
#pragma unroll
    for (int k = 0; k < OWN; ++k) mine += (double)own[k];
    const double all = block_sum<NT>(mine, tmp), aim = count_bins ? (double)ask.top_k : share_of(ask.top_p, whole);
    double run = block_excl_d<NT>(mine, tmp);
    if (tid == 0) find.bin = -1;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        if (run < aim && aim <= run + (double)own[k]) find.bin = OWN * tid + k, find.base = run, find.value[0] = run + (double)own[k];
        run += (double)own[k];
    }
    __syncthreads();
    if (tid == 0) {
        const bool found = find.bin >= 0;
        int state = found ? (count_bins ? kByNumber : kByWeight) : kStepwise;
        pr->bin_lo = pr->bin_hi = find.bin, pr->before = find.base;
        // two limits: all tokens down to the bin of the first, if a list holds them (all that weigh anything, if they are fewer than top_k)
        if (count_bins && ask.by_p()) {
            state = (found || bins_hold_all(ask)) && (found ? find.value[0] : all) <= (double)kGather ? kAllDownTo : kStepwise;
            pr->before = 0.0, pr->bin_lo = 0, pr->bin_hi = found ? find.bin : kBins - 1;
        }
        pr->state = state;
    }
}

// ---- rows that neither list nor bins settle (thousands of equal logits, or a great top_k far down): digit by digit over the keys, one workgroup, every step a pass over the row; 280 us for a row of 152064
template <int NT, typename T>
__device__ __forceinline__ u64 cut_stepwise(const RowView<T> row, const Asked ask, const Weigh w, u64* lds, double* tmp) {
    uint32_t cut;
    int last;
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
    return (u64)cut << 32 | (uint32_t)last;
}

// ---- the second list
template <typename T>
__global__ __launch_bounds__(kGatherThreads) void pick_gather_k(PickGeo geo, const T* logits, int64_t row_stride, PickFilter filter, PickWs ws, PickOut out) {
    constexpr int VEC = RowView<T>::VEC, NT = kGatherThreads, NW = NT / 64;
    __shared__ u64 local[kGather];        // the segment's list, then the row's
    __shared__ FindLds find;
    __shared__ Drawn drawn;
    __shared__ double tmp[16], part[kSegsMost * 8];
    __shared__ float sparse[NW][128];
    __shared__ uint32_t local_n, base_n;
    __shared__ int flag;
    const int lr = blockIdx.x / geo.segs, g = blockIdx.x - lr * geo.segs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = geo.row0 + lr;
    PickRow* pr = ws.row + lr;
    const int state = pr->state;
    if (state == kDone || (state == kStepwise && g != 0)) return;
    const RowView<T> row(logits + (int64_t)r * row_stride, geo.V);
    Asked ask = asked_of_row(geo, ws, lr, filter);
    const float top = row_top(geo, ws, lr);
    const Weigh w(top, ask.tau);
    const double whole = pr->whole;
    const int wper = (geo.per + NW - 1) / NW, ranges = geo.segs * 8;
    if (state != kStepwise) {
        int rank;
        const float per_logit = bins_per_logit(ask, geo.V, w.distance(reached(geo, ws, lr, level_of(ask), rank)));
        const int lo = pr->bin_lo, hi = pr->bin_hi;
        const int seg_end = min(row.pieces(), (g + 1) * geo.per), c0 = min(seg_end, g * geo.per + wave * wper), c1 = min(seg_end, c0 + wper);
        if (tid == 0) local_n = 0;
        __syncthreads();
        SparseSum above{sparse[wave], ask.least};
        row.template each<true>(c0 + lane, 64, c1, [&](int c, const float (&x)[VEC]) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float b = bin_of(w, x[e], per_logit);
                if (out.token) above.add(w, b < (float)lo, x[e]);
                const bool is = b >= (float)lo && b < (float)(hi + 1);
                const uint32_t at = place(is, &local_n);
                if (is && at < (uint32_t)kGather) local[at] = entry_of(x[e], row.first(c) + e);
            }
        });
        above.finish(w);
        const double kept = wave_sum_d(above.sum), kept_n = wave_sum_d((double)above.count);
        if (lane == 0) leave(ws.part + lr * ranges + g * 8 + wave, kept), leave(ws.part_n + lr * ranges + g * 8 + wave, (uint32_t)kept_n);
        __syncthreads();
        if (tid == 0) base_n = atomicAdd(&pr->gather_n, local_n > (uint32_t)kGather ? 1u << 20 : local_n);
        __syncthreads();
        const uint32_t mine_n = min(local_n, (uint32_t)kGather), at = base_n;
        for (uint32_t i = tid; i < mine_n; i += NT)
            if (at + i < (uint32_t)kGather) leave(ws.gather + (int64_t)lr * kGather + at + i, local[i]);
        if (!last_here(&pr->seen_gather, geo.segs, &flag)) return;
        constexpr int kEarly = 2;   // (asked for together with the list's length)
        u64 early[kEarly];
#pragma unroll
        for (int i = 0; i < kEarly; ++i) early[i] = left(ws.gather + (int64_t)lr * kGather + i * NT + tid);
        const uint32_t n = left(&pr->gather_n);
        if (n > 0 && n <= (uint32_t)kGather) {
            uint32_t* stored = n <= kGather / 3 * 2 ? (uint32_t*)(local + kGather / 3 * 2) : nullptr;   // (8 and 4 bytes a token)
#pragma unroll
            for (int i = 0; i < kEarly; ++i)
                if ((uint32_t)(i * NT + tid) < n) {
                    local[i * NT + tid] = early[i];
                    if (stored) stored[i * NT + tid] = TokenList<uint32_t>::held(w(entry_logit(early[i])));
                }
#pragma unroll 4
            for (uint32_t i = kEarly * NT + tid; i < n; i += NT) {
                const u64 e = left(ws.gather + (int64_t)lr * kGather + i);
                local[i] = e;
                if (stored) stored[i] = TokenList<uint32_t>::held(w(entry_logit(e)));
            }
            __syncthreads();
            const TokenList<uint32_t> l{local, stored, w, (int)n};
            if (state == kByNumber) ask.top_p = 1u << 31;
            const double before = pr->before;
            const u64 end = end_in_list<NT>(l, (int)n, ask, state == kByWeight ? before : 0.0, state == kByNumber ? before : 0.0, whole, top - (float)lo / per_logit, top - (float)(hi + 1) / per_logit,
                                            state == kAllDownTo, find, tmp);
            if (end != kNoEntry) {
                const Kept in{~(uint32_t)(end >> 32), (int)(uint32_t)end, ask.least};
                if (tid == 0) pr->cut = in.cut, pr->last = in.last;
                if (!out.token) return;
                if (state == kAllDownTo) {
                    draw_from_list<NT>(l, end, ask.least, geo.V, find, tmp, out.kept ? out.kept + r : nullptr, out.u[r], &drawn);
                    if (tid == 0) put_token(out.token + r, out.logprob ? out.logprob + 2 * r : nullptr, w, drawn, whole);
                    return;
                }
                // the listed ones join the sums of their ranges
                static_assert(kSegsMost * 8 <= NT, "a range per thread");
                if (tid < ranges) part[tid] = left(ws.part + lr * ranges + tid);
                double count = tid < ranges ? (double)left(ws.part_n + lr * ranges + tid) : 0.0;
                __syncthreads();
                for (uint32_t i = tid; i < n; i += NT)
                    if (local[i] <= end && l.weight(i) >= ask.least) {
                        const int c = ((int)(uint32_t)local[i] + row.off) / VEC, seg = c / geo.per;
                        atomicAdd(&part[seg * 8 + (c - seg * geo.per) / wper], l.weight(i));
                        count += 1.0;
                    }
                count = block_sum<NT>(count, tmp);
                if (tid == 0 && out.kept) out.kept[r] = (int32_t)count;
                const double mine = tid < ranges ? part[tid] : 0.0, S = block_sum<NT>(mine, tmp), aim = aim_of(out.u[r], S);
                double base;
                const int range = range_of<NT>(mine, aim, base, find, tmp);
                if (range < 0) return;   // (cannot be)
                const int stop = min(row.pieces(), ((range >> 3) + 1) * geo.per), p0 = min(stop, (range >> 3) * geo.per + (range & 7) * wper), p1 = min(stop, p0 + wper);
                draw_from<NT, T>(row, p0, p1, w, in, base, S, out.u[r], tmp, &drawn);
                if (tid == 0) put_token(out.token + r, out.logprob ? out.logprob + 2 * r : nullptr, w, drawn, whole);
                return;
            }
        }
        ask = asked_of_row(geo, ws, lr, filter);
        __syncthreads();
    }
    u64* buf = local;
    Kept in{0, 0, ask.least};
    const u64 found = cut_stepwise<NT, T>(row, ask, w, buf, tmp);
    in.cut = (uint32_t)(found >> 32), in.last = (int)(uint32_t)found;
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
    draw_from<NT, T>(row, 0, row.pieces(), w, in, 0.0, -1.0, out.u[r], tmp, &drawn);
    if (tid == 0) put_token(out.token + r, out.logprob ? out.logprob + 2 * r : nullptr, w, drawn, whole);
}

// ---- filtered rows: read and written once, bound by memory (256 rows of 152064 in 55 us, 5.7 TB/s)
// Pieces first, first + step, .. of a row below `end`, with what is not kept at -infinity (copy: as they are); returns this thread's number of kept tokens.
template <typename T>
__device__ __forceinline__ uint32_t mask_row(const RowView<T>& row, T* o, int first, int step, int end, const Weigh& w, const Kept& in, bool copy) {
    constexpr int VEC = RowView<T>::VEC;
    const bool wide = ((uintptr_t)o & 15) == ((uintptr_t)row.row & 15);
    uint32_t count = 0;
    row.each(first, step, end, [&](int c, const float (&x)[VEC]) {
        const int j = row.first(c);
        float y[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const bool keep = in(w, j + e, x[e]);
            count += keep & !copy & (x[e] > -INFINITY);
            y[e] = (keep | copy) ? x[e] : -INFINITY;
        }
        if (c >= end) return;
        if (wide && row.inside(c)) {
            *(u32x4_t*)(o + j) = RowView<T>::packed(y);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (j + e >= 0 && j + e < row.V) o[j + e] = from_float<T>(y[e]);
        }
    });
    return count;
}

template <typename T>
__global__ __launch_bounds__(kWeighThreads) void pick_mask_k(PickGeo geo, const T* logits, int64_t row_stride, PickFilter filter, PickWs ws, PickOut out) {
    constexpr int NT = kWeighThreads;
    __shared__ double tmp[16];
    const int lr = blockIdx.x / geo.segs, g = blockIdx.x - lr * geo.segs, r = geo.row0 + lr;
    const RowView<T> row(logits + (int64_t)r * row_stride, geo.V);
    const Asked ask = Wish(filter, r / geo.rows_per_seq).asked(geo.V);   // (its least weight)
    const PickRow& pr = ws.row[lr];
    const Weigh w(row_top(geo, ws, lr), ask.tau);
    const uint32_t count = mask_row<T>(row, (T*)out.rows + (int64_t)r * out.rows_stride, g * geo.per + threadIdx.x, NT, min(row.pieces(), (g + 1) * geo.per), w,
                                       Kept{pr.cut, pr.last, ask.least}, pr.cut == 0);
    if (!out.kept) return;
    const double all = block_sum<NT>((double)count, tmp);
    if (threadIdx.x == 0 && all > 0.0) atomicAdd(&out.kept[r], (int32_t)all);
}

// The same, as functions of their own: inlined they would cost pick_row_k's loops their registers (32 x 48 rows of 152064 770 us when it was first measured, 975
// with them inlined; the kernels with fewer threads are better off inlined).
template <int NT>
__device__ __attribute__((noinline)) u64 end_in_list_apart(const TokenList<double> l, int n, const Asked ask, double before_w, double before_n, double S, float best, float least, bool all,
                                                             FindLds& s, double* tmp) {
    return end_in_list<NT>(l, n, ask, before_w, before_n, S, best, least, all, s, tmp);
}
template <int NT, typename T>
__device__ __attribute__((noinline)) u64 cut_stepwise_apart(const RowView<T> row, const Asked ask, const Weigh w, u64* lds, double* tmp) {
    return cut_stepwise<NT, T>(row, ask, w, lds, tmp);
}

// Many rows: a workgroup each, which does everything without meeting another one.  Rows are read three times and written once: 1536 rows of 152064 (0.93 GB each
// time) in 712 us, 5.2 TB/s.
template <typename T>
__global__ __launch_bounds__(kRowThreads) void pick_row_k(int V, int rows_per_seq, const T* logits, int64_t row_stride, PickFilter filter, PickOut out) {
    constexpr int VEC = RowView<T>::VEC, NT = kRowThreads, NW = NT / 64, kWaveList = kGather / NW;
    __shared__ u64 list[kGather];         // waves' lists of likely tokens, put together; then the bin's tokens
    __shared__ u64 bins[kBins];
    __shared__ FindLds find;
    __shared__ double tmp[16];
    __shared__ float wave_top[NW], wave_reach[kGroups][NW];
    __shared__ uint32_t wave_groups[kGroups][NW], wave_n[NW], count_n;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const RowView<T> row(logits + (int64_t)r * row_stride, V);
    T* o = (T*)out.rows + (int64_t)r * out.rows_stride;
    const int pieces = row.pieces();
    const Wish wish(filter, r / rows_per_seq);
    // the largest logit, the number of tokens, and how far the likely ones reach
    float top = -INFINITY;
    bool nan = false;
    uint32_t tokens = 0;
    row.each(tid, NT, pieces, [&](int, const float (&x)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) nan |= x[e] != x[e], top = fmaxf(top, x[e]), tokens += x[e] > -INFINITY;
    });
    float s = top;
    int have = 1;
#pragma unroll
    for (int k = kGroups - 1; k >= 0; --k) {
        constexpr int most = NT / 64;
        const int lanes = most >> k;   // of a group
        for (; have < lanes; have <<= 1) s = fmaxf(s, __shfl_xor(s, have, 64));
        const uint64_t full = __ballot(s > -INFINITY);
        const float least = -wave_max(s > -INFINITY ? -s : -INFINITY);
        if (lane == 0) wave_reach[k][wave] = least, wave_groups[k][wave] = (uint32_t)(__popcll(full) / lanes);
    }
    top = wave_max(top);
    if (__any(nan)) top = NAN;
    tokens = (uint32_t)wave_sum_d((double)tokens);
    if (lane == 0) wave_top[wave] = top, wave_n[wave] = tokens;
    __syncthreads();
    top = wave_top[0], tokens = wave_n[0];
#pragma unroll
    for (int v = 1; v < NW; ++v) top = top != top || wave_top[v] != wave_top[v] ? NAN : fmaxf(top, wave_top[v]), tokens += wave_n[v];
    if (top != top || top == -INFINITY) {   // (uniform)
        if (o != row.row) mask_row<T>(row, o, tid, NT, pieces, Weigh(0.f, 1.0), Kept{0, 0, 0.0}, true);
        if (tid == 0) put_nothing(out, r, top != top);
        return;
    }
    const Asked ask = wish.asked((int)tokens);
    const Weigh w(top, ask.tau);
    Kept in{kKeyNothing, -1, ask.least};   // (all, unless a prefix is asked for)
    if (ask.prefix()) {
        const int level = level_of(ask);
        int rank = 0;
        float from = INFINITY;
#pragma unroll
        for (int v = 0; v < NW; ++v) rank += wave_groups[level][v], from = fminf(from, wave_reach[level][v]);
        from = fmaxf(from, -FLT_MAX);
        const bool count_bins = ask.top_k > min(rank, kListed), use_bins = count_bins || ask.top_k == 0, weigh_all = ask.top_k == 0;
        const float per_logit = use_bins ? bins_per_logit(ask, V, w.distance(from)) : 0.f;
        if (count_bins) from = INFINITY;
        if (use_bins)
            for (int i = tid; i < kBins; i += NT) bins[i] = 0;
        __syncthreads();
        u64* listing = list + wave * kWaveList;
        uint32_t listed = 0;
        double whole = 0.0;
        row.each(tid, NT, pieces, [&](int c, const float (&x)[VEC]) {   // (waves take turns, so that neighbouring tokens go to several lists)
            double weight[VEC];
            if (weigh_all) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    weight[e] = w(x[e]);
                    whole += weight[e];
                }
            }
            float best = x[0];
#pragma unroll
            for (int e = 1; e < VEC; ++e) best = fmaxf(best, x[e]);
            if (__any(best >= from)) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const bool is = x[e] >= from;
                    const uint64_t all = __ballot(is);
                    if (all == 0) continue;
                    const uint32_t at = listed + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
                    if (is && at < (uint32_t)kWaveList) listing[at] = entry_of(x[e], row.first(c) + e);
                    listed += (uint32_t)__popcll(all);
                }
            }
            if (use_bins) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float b = bin_of(w, x[e], per_logit);
                    if (b < (float)kBins) atomicAdd(&bins[(int)b], count_bins ? 1ull : w.whole(weight[e]));
                }
            }
        });
        if (lane == 0) wave_n[wave] = listed > (uint32_t)kWaveList ? 1u << 20 : listed;
        whole = block_sum<NT>(whole, tmp);   // (the lists are whole, too)
        uint32_t n = 0, at = 0;
#pragma unroll
        for (int v = 0; v < NW; ++v) at += v < wave ? wave_n[v] : 0, n += wave_n[v];
        if (n <= (uint32_t)kGather) {
            u64 held[kWaveList / 64];
#pragma unroll
            for (int i = 0; i < kWaveList / 64; ++i) held[i] = listing[i * 64 + lane];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kWaveList / 64; ++i)
                if ((uint32_t)(i * 64 + lane) < listed) list[at + i * 64 + lane] = held[i];
            __syncthreads();
        }
        TokenList<double> l{list, nullptr, w, (int)n};
        u64 end = kNoEntry;
        if (n > 0 && n <= (uint32_t)kGather) end = end_in_list_apart<NT>(l, (int)n, ask, 0.0, 0.0, whole, top, from, false, find, tmp);
        if (end == kNoEntry && use_bins) {
            // the bin that the end lies in
            static_assert(kBins <= NT, "a bin per thread");
            const double mine = tid < kBins ? (double)bins[tid] : 0.0;
            const double all = block_sum<NT>(mine, tmp), aim = count_bins ? (double)ask.top_k : share_of(ask.top_p, whole), run = block_excl_d<NT>(mine, tmp);
            if (tid == 0) find.bin = -1, count_n = 0;
            __syncthreads();
            if (run < aim && aim <= run + mine) find.bin = tid, find.base = run, find.value[0] = run + mine;
            __syncthreads();
            // two limits: all tokens down to the bin of the first, if a list holds them (all that weigh anything, if they are fewer than top_k)
            const bool found = find.bin >= 0, down_to = count_bins && ask.by_p();
            const int lo = down_to ? 0 : find.bin, hi = found ? find.bin : kBins - 1;
            const double before = down_to ? 0.0 : find.base;
            if (down_to ? (found || bins_hold_all(ask)) && (found ? find.value[0] : all) <= (double)kGather : found) {   // (uniform)
                row.each(tid, NT, pieces, [&](int c, const float (&x)[VEC]) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float b = bin_of(w, x[e], per_logit);
                        const bool is = b >= (float)lo && b < (float)(hi + 1);
                        const uint32_t to = place(is, &count_n);
                        if (is && to < (uint32_t)kGather) list[to] = entry_of(x[e], row.first(c) + e);
                    }
                });
                __syncthreads();
                n = count_n;
                if (n > 0 && n <= (uint32_t)kGather) {
                    l.n = (int)n;
                    Asked one = ask;
                    if (count_bins && !down_to) one.top_p = 1u << 31;
                    end = end_in_list_apart<NT>(l, (int)n, one, count_bins ? 0.0 : before, count_bins ? before : 0.0, whole, top - (float)lo / per_logit, top - (float)(hi + 1) / per_logit, down_to, find, tmp);
                }
            }
        }
        if (end != kNoEntry) {
            in.cut = ~(uint32_t)(end >> 32), in.last = (int)(uint32_t)end;
        } else {
            __syncthreads();
            const u64 cut = cut_stepwise_apart<NT, T>(row, ask, w, list, tmp);
            in.cut = (uint32_t)(cut >> 32), in.last = (int)(uint32_t)cut;
        }
    }
    const uint32_t mine = mask_row<T>(row, o, tid, NT, pieces, w, in, false);
    const double all = block_sum<NT>((double)mine, tmp);
    if (tid == 0 && out.kept) out.kept[r] = (int32_t)all;
}

// ---- small vocabularies: a row is one list, and one workgroup does everything.  2 x 1024 in 10 us, a chain: the row, its weights, two or three searches of about 2 us in LDS.
template <typename T>
__global__ __launch_bounds__(kGatherThreads) void pick_small_k(int V, int rows_per_seq, const T* logits, int64_t row_stride, PickFilter filter, PickOut out) {
    constexpr int NT = kGatherThreads;
    __shared__ u64 entry[kSmall];
    __shared__ double weight[kSmall], tmp[16];
    __shared__ FindLds find;
    __shared__ Drawn drawn;
    const int r = blockIdx.x, tid = threadIdx.x;
    const T* row = logits + (int64_t)r * row_stride;
    T* o = out.rows ? (T*)out.rows + (int64_t)r * out.rows_stride : nullptr;
    const Wish wish(filter, r / rows_per_seq);
    const uint32_t u = out.token ? out.u[r] : 0u;
    float top = -INFINITY, least = INFINITY;
    bool nan = false;
    double tokens = 0.0;
    for (int j = tid; j < V; j += NT) {
        const float x = to_float(row[j]);
        const bool is = x > -INFINITY;
        nan |= x != x, top = fmaxf(top, x), tokens += is;
        if (is) least = fminf(least, x);
        entry[j] = is ? entry_of(x, j) : kNoEntry;
    }
    top = wave_max(top);
    if (__any(nan)) top = NAN;
    if ((tid & 63) == 0) tmp[tid >> 6] = (double)top;
    __syncthreads();
    top = (float)tmp[0];
#pragma unroll
    for (int v = 1; v < NT / 64; ++v) top = top != top || tmp[v] != tmp[v] ? NAN : fmaxf(top, (float)tmp[v]);
    if (top != top || top == -INFINITY) {   // (uniform)
        if (o && o != row)
            for (int j = tid; j < V; j += NT) o[j] = row[j];
        if (tid == 0) put_nothing(out, r, top != top);
        return;
    }
    tokens = block_sum<NT>(tokens, tmp);
    least = -wave_max(-least);
    __syncthreads();
    if ((tid & 63) == 0) tmp[tid >> 6] = (double)least;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < NT / 64; ++v) least = fminf(least, (float)tmp[v]);
    const Asked ask = wish.asked((int)tokens);
    const Weigh w(top, ask.tau);
    double whole = 0.0;
    for (int j = tid; j < V; j += NT) {
        const double x = entry[j] != kNoEntry ? w(entry_logit(entry[j])) : 0.0;
        weight[j] = x, whole += x;
    }
    whole = block_sum<NT>(whole, tmp);   // (and all of both lists is there)
    const TokenList<double> l{entry, weight, w, V};
    const u64 end = end_in_list<NT>(l, (int)tokens, ask, 0.0, 0.0, whole, top, least, true, find, tmp);
    if (out.token) {
        draw_from_list<NT>(l, end, ask.least, V, find, tmp, out.kept ? out.kept + r : nullptr, u, &drawn);
        if (tid == 0) put_token(out.token + r, out.logprob ? out.logprob + 2 * r : nullptr, w, drawn, whole);
        return;
    }
    double count = 0.0;
    for (int j = tid; j < V; j += NT) {
        const bool keep = entry[j] <= end && weight[j] >= ask.least;
        count += keep;
        const T x = row[j];
        o[j] = keep ? x : from_float<T>(-INFINITY);
    }
    count = block_sum<NT>(count, tmp);
    if (tid == 0 && out.kept) out.kept[r] = (int32_t)count;
}

// ---- host
constexpr int kMostGroups = 1448;   // segments of all rows, or one of each
static int pick_most_segs(int vocab) { return std::min(kSegsMost, std::max(1, vocab / 4096)); }
static int pick_segs(int rows, int vocab) {
    // 1024 workgroups (four on each CU), or up to 1448 where the next fewer would be half of that, of 4096 tokens at least (so that each of a segment's threads has some).  With top-p over 152064 tokens
    // 1024, 512 and 2048 workgroups: 64 rows 69, 76 and 83 us, 90 rows 84, 103 and 81, 32 rows 60, 58 and 60.  The rounding: 320 rows as 1280 workgroups 167 us, as 640 193; 700 rows as 1400 305, as 700 368; but 45 rows as
    // 1440 63, as 720 56.
    const int most = pick_most_segs(vocab);
    int segs = 1;
    while (2 * segs <= std::min(most, 1024 / rows)) segs *= 2;
    return segs < 8 && 2 * segs <= std::min(most, kMostGroups / rows) ? 2 * segs : segs;
}
static int pick_pass(int rows) { return (rows + (rows + kPassRows - 1) / kPassRows - 1) / ((rows + kPassRows - 1) / kPassRows); }
// R rows with RS segments
static size_t pick_carve(size_t R, size_t RS, char* base, PickWs* ws) {
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* p = base + at;
        at += (bytes + 255) / 256 * 256;
        return (void*)p;
    };
    PickWs w;
    w.row = (PickRow*)take(R * sizeof(PickRow));
    w.top = (float*)take(RS * 4);
    w.reach = (float*)take(RS * kGroups * 4);
    w.groups = (uint32_t*)take(RS * kGroups * 4);
    w.tokens = (uint32_t*)take(RS * 4);
    w.whole = (double*)take(RS * 8);
    w.part = (double*)take(RS * 64);
    w.part_n = (uint32_t*)take(RS * 32);
    w.list = (u64*)take(R * kList * 8);
    w.gather = (u64*)take(R * kGather * 8);
    w.bins = (u64*)take(RS * kBins * 8);
    if (ws) *ws = w;
    return at;
}
// (no smaller for more rows or a larger vocabulary: a caller sizes it once, for the largest call)
size_t pick_workspace_bytes(int rows, int vocab) {
    if (vocab <= kSmall) return 256;
    const size_t R = (size_t)std::min(rows, kPassRows);
    return pick_carve(R, std::max(R, std::min((size_t)kMostGroups, R * pick_most_segs(vocab))), nullptr, nullptr);
}

template <typename T>
static void pick_rounds(hipStream_t s, int rows, int rows_per_seq, int vocab, const T* logits, int64_t row_stride, const PickFilter& filter, const PickOut& out, char* base) {
    if (vocab <= kSmall) {
        hipLaunchKernelGGL(pick_small_k<T>, dim3(rows), dim3(kGatherThreads), 0, s, vocab, rows_per_seq, logits, row_stride, filter, out);
        return;
    }
    if (out.rows && rows > kFewRows) {
        hipLaunchKernelGGL(pick_row_k<T>, dim3(rows), dim3(kRowThreads), 0, s, vocab, rows_per_seq, logits, row_stride, filter, out);
        return;
    }
    const int pass = pick_pass(rows);
    PickWs ws;
    PickGeo geo;
    geo.V = vocab;
    geo.segs = pick_segs(pass, vocab);
    pick_carve((size_t)pass, (size_t)pass * geo.segs, base, &ws);
    constexpr int VEC = RowView<T>::VEC;
    geo.per = ((vocab + 2 * VEC - 2) / VEC + geo.segs - 1) / geo.segs;
    geo.rows_per_seq = rows_per_seq;
    for (geo.row0 = 0; geo.row0 < rows; geo.row0 += pass) {
        const dim3 grid((unsigned)(std::min(pass, rows - geo.row0) * geo.segs));
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
