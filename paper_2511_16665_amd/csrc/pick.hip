// Sampling from rows of logits behind top-k, top-p and min-p: one token per row, or the row with all other tokens at -infinity.
//
// Weights are the acceptance rules' whole numbers W = floor(exp(l / tau - max / tau) * 2^32), so sums do not depend on their order.  What is kept is a
// prefix of the order (logit falling, index rising), so it is given by a logit, the last index kept of those equal to it, and a least weight: (key, last,
// least) below.  Equal logits have equal weights, so both limits of the prefix are found on keys alone, and only the last group of equal logits is counted
// by index.
#include <algorithm>

#include "dev_common.h"
#include "kernels.h"

namespace tlt {

typedef unsigned long long u64;

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64;

// order of logits as whole numbers; -0 and +0 are equal
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
constexpr uint32_t kKeyNothing = 0x007fffffu;   // of -infinity

// what a request asks for, of one row
struct Asked {
    double tau;
    int top_k;         // 0: off
    uint32_t top_p;    // units of 2^-31; 2^31: off
    u64 least;         // weight; 0: off
};
__device__ __forceinline__ Asked asked_of(const PickFilter& f, int seq) {
    Asked a{1.0, 0, 1u << 31, 0ull};
    const float tau = f.temperature ? f.temperature[seq] : 1.f;
    if (!(tau > 0.f)) {
        a.top_k = 1;
        return a;
    }
    a.tau = (double)tau;
    if (f.top_k) a.top_k = max(f.top_k[seq], 0);
    if (f.top_p) {
        const float p = f.top_p[seq];
        if (p < 1.f) a.top_p = (uint32_t)(fmax((double)p, 0.0) * 2147483648.0);
    }
    if (f.min_p) {
        const float m = f.min_p[seq];
        if (m > 0.f) a.least = (u64)(fmin((double)m, 1.0) * 4294967296.0);
    }
    return a;
}
// ceil(share * S / 2^31), at least 1
__device__ __forceinline__ u64 share_of(uint32_t share, u64 S) {
    const unsigned __int128 x = (unsigned __int128)share * S + 0x7fffffffu;
    return max((u64)(x >> 31), 1ull);
}

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ u64 pick_block_sum(u64 v, u64* tmp) {
    v = wave_sum_u64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 all = 0;
    for (int w = 0; w < kPickWaves; ++w) all += tmp[w];
    return all;
}
// sum over the threads before this one
__device__ __forceinline__ u64 pick_block_excl(u64 v, u64* tmp) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const u64 up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 63) tmp[wave] = incl;
    __syncthreads();
    u64 base = 0;
    for (int w = 0; w < wave; ++w) base += tmp[w];
    return base + incl - v;
}

// A workgroup per row; every quantity is found by passes over the row.
template <typename T>
__global__ __launch_bounds__(kPickThreads) void pick_row_k(int V, int rows_per_seq, const T* logits, int64_t row_stride, PickFilter filter, PickOut out) {
    __shared__ u64 tmp[kPickWaves], bins[256], counts[256];
    __shared__ u64 found[3];
    __shared__ int found_i;
    const int r = blockIdx.x, tid = threadIdx.x;
    const T* l = logits + (int64_t)r * row_stride;
    const Asked ask = asked_of(filter, r / rows_per_seq);
    // the largest logit, and whether there is a NaN
    float top = -INFINITY;
    int nan = 0;
    for (int j = tid; j < V; j += kPickThreads) {
        const float x = to_float(l[j]);
        nan |= x != x;
        top = fmaxf(top, x);
    }
    top = wave_max(top);
    if (__any(nan)) top = NAN;
    float* ft = (float*)tmp;
    if ((tid & 63) == 0) ft[tid >> 6] = top;
    __syncthreads();
    top = ft[0];
    nan = top != top;
    for (int w = 1; w < kPickWaves; ++w) {
        nan |= ft[w] != ft[w];
        top = fmaxf(top, ft[w]);
    }
    __syncthreads();
    if (nan || top == -INFINITY) {   // (uniform)
        if (out.rows)
            for (int j = tid; j < V; j += kPickThreads) ((T*)out.rows)[(int64_t)r * out.rows_stride + j] = l[j];
        if (tid == 0) {
            if (out.token) out.token[r] = -1;
            if (out.logprob) out.logprob[2 * r] = out.logprob[2 * r + 1] = nan ? NAN : -INFINITY;
            if (out.kept) out.kept[r] = 0;
        }
        return;
    }
    const double scaled_top = (double)top / ask.tau;
    auto below = [&](float x) { return x == top ? 0.0 : (double)x / ask.tau - scaled_top; };
    auto weight = [&](float x) {   // (below e^-23 it is 0, and so it is where infinities leave nothing to compare)
        const double z = below(x);
        return x > -INFINITY && z > -23.0 ? (u64)floor(exp(z) * 4294967296.0) : 0ull;
    };
    // Where a prefix of the order ends: with `by_weight` after the weights before it reach `aim` (>= 1), otherwise after `aim` tokens; among those above
    // lim_key, and lim_n of those equal to it.  Digit by digit from the top; gives the key, how many equal to it are in, and what the ones above it add up to.
    uint32_t lim_key = kKeyNothing;
    u64 lim_n = 0;
    auto prefix = [&](u64 aim, bool by_weight, uint32_t& key, u64& n, u64& before, u64& group) {
        key = 0, before = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) bins[tid] = counts[tid] = 0;
            __syncthreads();
            for (int j = tid; j < V; j += kPickThreads) {
                const float x = to_float(l[j]);
                const uint32_t k = key_of(x);
                if (k <= lim_key || (shift < 24 && k >> (shift + 8) != key >> (shift + 8))) continue;
                atomicAdd(&counts[k >> shift & 255], 1ull);
                if (by_weight) atomicAdd(&bins[k >> shift & 255], weight(x));
            }
            __syncthreads();
            if (tid == 0) {
                if (lim_n && (shift == 24 || lim_key >> (shift + 8) == key >> (shift + 8))) {
                    const uint32_t bits = lim_key & 0x80000000u ? lim_key ^ 0x80000000u : ~lim_key;
                    counts[lim_key >> shift & 255] += lim_n;
                    if (by_weight) bins[lim_key >> shift & 255] += lim_n * weight(__uint_as_float(bits));
                }
                u64 sum = before;
                int at = -1, last = 0;
                for (int d = 255; d >= 0; --d) {
                    const u64 add = by_weight ? bins[d] : counts[d];
                    if (counts[d]) last = d;
                    if (add && sum + add >= aim) {
                        at = d;
                        break;
                    }
                    sum += add;
                }
                if (at < 0) at = last, sum -= by_weight ? bins[last] : counts[last];   // (all of them)
                found[0] = sum, found_i = at;
                found[1] = counts[at], found[2] = bins[at];
            }
            __syncthreads();
            before = found[0];
            key |= (uint32_t)found_i << shift;
            n = found[1], group = found[2];
        }
        __syncthreads();
    };
    uint32_t cut = kKeyNothing;   // kept: keys above it and the first `ties` of those equal to it
    u64 ties = 0, group_n = 0, before = 0, group = 0;
    if (ask.top_k > 0) {
        prefix((u64)ask.top_k, false, cut, group_n, before, group);
        ties = min(group_n, (u64)max((int64_t)ask.top_k - (int64_t)before, (int64_t)0));
        lim_key = cut, lim_n = ties;
    }
    if (ask.top_p < (1u << 31)) {
        u64 S = 0;
        for (int j = tid; j < V; j += kPickThreads) {
            const float x = to_float(l[j]);
            if (key_of(x) > lim_key) S += weight(x);
        }
        S = pick_block_sum(S, tmp);
        const uint32_t bits = lim_key & 0x80000000u ? lim_key ^ 0x80000000u : ~lim_key;
        if (lim_n) S += lim_n * weight(__uint_as_float(bits));
        const u64 aim = share_of(ask.top_p, S);
        prefix(aim, true, cut, group_n, before, group);
        const u64 each = group / max(group_n, 1ull);
        ties = each ? min(group_n, (aim - before + each - 1) / each) : group_n;
    }
    // the index of the last of the equal logits that is kept, threads owning ranges of indices
    const int per = (V + kPickThreads - 1) / kPickThreads, j0 = min(V, tid * per), j1 = min(V, j0 + per);
    if (tid == 0) found_i = -1;
    {
        u64 mine = 0;
        for (int j = j0; j < j1; ++j) mine += key_of(to_float(l[j])) == cut;
        u64 at = pick_block_excl(mine, tmp);
        if (cut != kKeyNothing && at < ties && ties <= at + mine)
            for (int j = j0; j < j1; ++j)
                if (key_of(to_float(l[j])) == cut && ++at == ties) found_i = j;
    }
    __syncthreads();
    const int last = found_i;
    auto kept = [&](int j, float x) {
        const uint32_t k = key_of(x);
        return (k > cut || (k == cut && j <= last)) && (ask.least == 0 || weight(x) >= ask.least);
    };
    u64 local = 0, whole = 0, count = 0;
    for (int j = j0; j < j1; ++j) {
        const float x = to_float(l[j]);
        const bool in = kept(j, x);
        count += in;
        if (out.token) {
            const u64 w = weight(x);
            whole += w, local += in ? w : 0;
        }
    }
    count = pick_block_sum(count, tmp);
    if (tid == 0 && out.kept) out.kept[r] = (int32_t)count;
    if (out.rows) {
        T* o = (T*)out.rows + (int64_t)r * out.rows_stride;
        for (int j = tid; j < V; j += kPickThreads) {
            const T x = l[j];
            o[j] = kept(j, to_float(x)) ? x : from_float<T>(-INFINITY);
        }
        return;
    }
    const u64 S = pick_block_sum(local, tmp);
    whole = pick_block_sum(whole, tmp);
    const u64 aim = (u64)(((unsigned __int128)out.u[r] * S) >> 32);
    u64 run = pick_block_excl(local, tmp);
    if (run <= aim && aim < run + local) {
        for (int j = j0; j < j1; ++j) {
            const float x = to_float(l[j]);
            if (!kept(j, x)) continue;
            run += weight(x);
            if (run > aim) {
                out.token[r] = j;
                if (out.logprob) {
                    out.logprob[2 * r] = (float)(below(x) - log((double)S * 0x1p-32));
                    out.logprob[2 * r + 1] = (float)(below(x) - log((double)whole * 0x1p-32));
                }
                break;
            }
        }
    }
}

size_t pick_workspace_bytes(int rows, int vocab) { return 256; }

hipError_t pick(hipStream_t s, int dtype, int rows, int rows_per_seq, int vocab, const void* logits, int64_t row_stride, const PickFilter& filter,
                const PickOut& out, void* ws, size_t ws_bytes) {
    if (ws_bytes < pick_workspace_bytes(rows, vocab)) return hipErrorInvalidValue;
    if (dtype == F32)
        hipLaunchKernelGGL(pick_row_k<float>, dim3(rows), dim3(kPickThreads), 0, s, vocab, rows_per_seq, (const float*)logits, row_stride, filter, out);
    else
        hipLaunchKernelGGL(pick_row_k<bf16>, dim3(rows), dim3(kPickThreads), 0, s, vocab, rows_per_seq, (const bf16*)logits, row_stride, filter, out);
    return hipGetLastError();
}

}  // namespace tlt
