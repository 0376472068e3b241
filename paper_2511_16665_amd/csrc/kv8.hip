// The 8-bit paged KV cache: writing rows, attention over them, keeping the accepted path, reading rows back.
//
// A row (one token of one kv head, d elements) is d codes in e4m3 (OCP: 4 exponent bits, bias 7, largest value 448, no infinities) and one
// exponent byte E; its values are code * 2^(E - 127).  E - 127 is the smallest e >= -126 with max|x| <= 448 * 2^e, so scaling by it is exact, the one
// rounding is that to e4m3 and a value has four significant bits (bf16 holds them all from 2^-130 up).  A row with an element that is not finite keeps E = 255 and codes of zero, and all of it
// reads as NaN.  One code of one exponent has no value in fp32 and bf16: rows from 248 * 2^120 on have E = 247 and the code 256, which would be 2^128;
// every reader takes the code below it instead (finite4).
#include <algorithm>

#include "dev_common.h"
#include "kernels.h"

namespace tlt {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;

// ---- format
// exponent byte of a row from the largest bit pattern of its magnitudes: 448 = 1.75 * 2^8
__device__ __forceinline__ uint32_t exponent_of(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return 255u;
    const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 1);
}
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23); }          // 2^(e - 127)
// 2^(127 - e): e is 248 at most for finite rows, so this is a normal number, and 0 for e = 255 (rows that are not finite: see encode4)
__device__ __forceinline__ float inverse_scale_of(uint32_t e) { return __uint_as_float(e == 255u ? 0u : (254u - e) << 23); }
// four codes: round to nearest, ties to even
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv) {
    if (inv == 0.f) return 0u;
    uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, (int)w, true);
}
__device__ __forceinline__ void decode4(uint32_t w, float scale, float* out) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    out[0] = lo[0] * scale, out[1] = lo[1] * scale, out[2] = hi[0] * scale, out[3] = hi[1] * scale;
}
// Four codes of a row whose exponent byte is kTopExp, the largest of a finite row, or above it (not finite: zeros stay zeros): 256, four exponent bits of one, becomes 240.
constexpr uint32_t kTopExp = 247;
__device__ __forceinline__ uint32_t finite4(uint32_t w) { return w - ((w & w >> 1 & w >> 2 & w >> 3 & 0x08080808u) >> 3); }
__device__ __forceinline__ u32x4_t finite16(u32x4_t w) { return u32x4_t{finite4(w[0]), finite4(w[1]), finite4(w[2]), finite4(w[3])}; }

// row number of a slot in the pools' rows of kv head 0 (kv head kh: + kh * page_size), -1: the block table does not back it
__device__ __forceinline__ int64_t row_of(const KV8Layer& kv, int b, int slot) {
    PageRef pr;
    if (!locate(kv.block_table, kv.max_pages, kv.n_pages, kv.page_size, b, slot, pr)) return -1;
    return pr.page * kv.n_kv * kv.page_size + pr.row;
}

// ---- write
// One workgroup per row (b, i).  A head (of q, k or v) belongs to a group of `lanes` lanes (a power of two); a lane holds VEC pairs (j, j + d/2) of it, one
// 16-byte piece of either half.  The largest magnitude of a k or v head is taken over its group.  Angles are formed in double (positions reach
// 32K, where an fp32 product position * frequency is 1e-3 rad off), once per row, and shared by the heads.  1536 rows of 28 and 4 heads of 128, 27 MB, 9.9 us
// (2.7 TB/s): all workgroups are on the chip at once, and a row's chain of length, angle, projection, maximum, table and store is exposed once with nothing behind it (0.7 us of
// it the angles; the row's loads in front of the angles change nothing).  One row 3.4 us, a launch and three dependent loads.
template <typename T>
__global__ __launch_bounds__(512) void kv8_write_k(const T* qkv, const T* __restrict__ bias, T* q_out, int64_t q_stride,   // (q_out may be qkv)
                                                   const int32_t* __restrict__ depth, int n, int n_q_heads, int lanes, double log2_theta, KV8Layer kv) {
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float cs[128], sn[128];
    const int r = blockIdx.x, b = r / n, i = r - b * n, d = kv.d, half = d >> 1, n_kv = kv.n_kv;
    const int heads = n_q_heads + 2 * n_kv;
    const T* row = qkv + (int64_t)r * heads * d;
    const int ctx = min(max(kv.seq_len[b], 0), 0x7fffffff - n);   // (so that no slot number overflows, whatever stands there)
    if ((int)threadIdx.x < half) {
        const int64_t pos = (int64_t)ctx + (depth ? depth[r] : i);
        double s, c;
        sincos((double)pos * exp2(-2.0 * (double)threadIdx.x / (double)d * log2_theta), &s, &c);
        cs[threadIdx.x] = (float)c, sn[threadIdx.x] = (float)s;
    }
    const int64_t at = row_of(kv, b, ctx + i);
    __syncthreads();
    const int group = threadIdx.x / lanes, p = threadIdx.x - group * lanes, per = blockDim.x / lanes;
    const int j = p * VEC;
    const bool on = j < half;
    for (int h0 = 0; h0 < heads; h0 += per) {   // (uniform: the shuffles below need every lane)
        const int h = h0 + group;
        const bool mine = on && h < heads;
        float lo[VEC], hi[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) lo[e] = hi[e] = 0.f;
        if (mine) {
            T a[VEC], c[VEC];
            *(u32x4_t*)a = *(const u32x4_t*)(row + h * d + j);
            *(u32x4_t*)c = *(const u32x4_t*)(row + h * d + half + j);
#pragma unroll
            for (int e = 0; e < VEC; ++e) lo[e] = to_float(a[e]), hi[e] = to_float(c[e]);
            if (bias) {
                *(u32x4_t*)a = *(const u32x4_t*)(bias + h * d + j);
                *(u32x4_t*)c = *(const u32x4_t*)(bias + h * d + half + j);
#pragma unroll
                for (int e = 0; e < VEC; ++e) lo[e] += to_float(a[e]), hi[e] += to_float(c[e]);
            }
            if (h < n_q_heads + n_kv) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float x = lo[e], y = hi[e], c1 = cs[j + e], s1 = sn[j + e];
                    lo[e] = x * c1 - y * s1, hi[e] = y * c1 + x * s1;
                }
            }
        }
        uint32_t amax = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            amax = max(amax, __float_as_uint(lo[e]) & 0x7fffffffu);
            amax = max(amax, __float_as_uint(hi[e]) & 0x7fffffffu);
        }
        for (int o = 1; o < lanes; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, 64));
        if (!mine) continue;
        if (h < n_q_heads) {
            T a[VEC], c[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) a[e] = from_float<T>(lo[e]), c[e] = from_float<T>(hi[e]);
            T* o = q_out + (int64_t)r * q_stride + h * d;
            *(u32x4_t*)(o + j) = *(const u32x4_t*)a;
            *(u32x4_t*)(o + half + j) = *(const u32x4_t*)c;
        } else if (at >= 0) {
            const bool is_k = h < n_q_heads + n_kv;
            const int64_t to = at + (int64_t)(h - n_q_heads - (is_k ? 0 : n_kv)) * kv.page_size;
            const uint32_t e8 = exponent_of(amax);
            const float inv = inverse_scale_of(e8);
            uint8_t* o = (is_k ? kv.k : kv.v) + to * d;
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                *(uint32_t*)(o + j + e) = encode4(lo[e], lo[e + 1], lo[e + 2], lo[e + 3], inv);
                *(uint32_t*)(o + half + j + e) = encode4(hi[e], hi[e + 1], hi[e + 2], hi[e + 3], inv);
            }
            if (p == 0) (is_k ? kv.k_exp : kv.v_exp)[to] = (uint8_t)e8;
        }
    }
}

hipError_t kv8_write(hipStream_t s, int dtype, int B, int n, const KV8Layer& kv, const void* qkv, const void* bias, const int32_t* depth, int n_q_heads,
                     float theta, void* q_out, int64_t q_stride) {
    const int vec = dtype == F32 ? 4 : 8, pieces = kv.d / 2 / vec, heads = n_q_heads + 2 * kv.n_kv;
    int lanes = 1;
    while (lanes < pieces) lanes <<= 1;
    int threads = (heads * lanes + 63) / 64 * 64;
    threads = threads < 128 ? 128 : (threads > 512 ? 512 : threads);
    const double log2_theta = log2((double)theta);
    const dim3 grid((unsigned)(B * n)), block(threads);
    if (dtype == F32)
        hipLaunchKernelGGL(kv8_write_k<float>, grid, block, 0, s, (const float*)qkv, (const float*)bias, (float*)q_out, q_stride, depth, n, n_q_heads, lanes, log2_theta, kv);
    else
        hipLaunchKernelGGL(kv8_write_k<bf16>, grid, block, 0, s, (const bf16*)qkv, (const bf16*)bias, (bf16*)q_out, q_stride, depth, n, n_q_heads, lanes, log2_theta, kv);
    return hipGetLastError();
}

// ---- read
// One wave per (layer, sequence, 16 rows, kv head): a row's d / 16 pieces of 16 codes go to d / 16 lanes.  Bound by memory, mostly what it writes: 4 layers of 7 sequences
// of 4001 rows, 345 MB, 74 us (4.6 TB/s; a large copy reaches 5.0).
template <typename T>
__global__ __launch_bounds__(256) void kv8_read_k(int n_layers, int B, int n, const int32_t* __restrict__ first, const int32_t* __restrict__ count,
                                                  T* __restrict__ out_k, T* __restrict__ out_v, KV8Layer kv) {
    const int lane = threadIdx.x & 63, chunks = (n + 15) / 16, d = kv.d, lpr = d / 16, per = 64 / lpr;
    int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (u >= (int64_t)n_layers * B * chunks * kv.n_kv) return;
    const int kh = (int)(u % kv.n_kv);
    u /= kv.n_kv;
    const int chunk = (int)(u % chunks);
    u /= chunks;
    const int b = (int)(u % B), layer = (int)(u / B);
    const int64_t rows_per_layer = kv.n_pages * kv.n_kv * kv.page_size;
    const int from = first[b], cnt = count ? min(count[b], n) : n;
    const int grp = lane / lpr, piece = (lane - grp * lpr) * 16;
    if (grp >= per) return;
    for (int t = grp; t < 16; t += per) {
        const int j = chunk * 16 + t;
        if (j >= cnt) return;
        const int64_t slot = (int64_t)from + j, at0 = from >= 0 && slot <= 0x7fffffff ? row_of(kv, b, (int)slot) : -1;
        const int64_t at = at0 + layer * rows_per_layer + (int64_t)kh * kv.page_size;
        const int64_t to = ((((int64_t)layer * B + b) * n + j) * kv.n_kv + kh) * d + piece;
        u32x4_t w[2] = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
        uint32_t e[2] = {127u, 127u};
        if (at0 >= 0) {
            w[0] = *(const u32x4_t*)(kv.k + at * d + piece), w[1] = *(const u32x4_t*)(kv.v + at * d + piece);
            e[0] = kv.k_exp[at], e[1] = kv.v_exp[at];
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (e[x] >= kTopExp) w[x] = finite16(w[x]);
            T* o = (x == 0 ? out_k : out_v) + to;
            float f[16];
#pragma unroll
            for (int q = 0; q < 4; ++q) decode4(w[x][q], scale_of(e[x]), f + 4 * q);
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int q = 0; q < 4; ++q) *(f32x4_t*)(o + 4 * q) = f32x4_t{f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]};
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    *(u32x4_t*)(o + 8 * q) = u32x4_t{pack_bf16x2(f[8 * q], f[8 * q + 1]), pack_bf16x2(f[8 * q + 2], f[8 * q + 3]),
                                                     pack_bf16x2(f[8 * q + 4], f[8 * q + 5]), pack_bf16x2(f[8 * q + 6], f[8 * q + 7])};
            }
        }
    }
}

hipError_t kv8_read(hipStream_t s, int dtype, int n_layers, int B, int n, const KV8Layer& kv, const int32_t* first, const int32_t* count, void* out_k,
                    void* out_v) {
    const int64_t units = (int64_t)n_layers * B * ((n + 15) / 16) * kv.n_kv;
    const dim3 grid((unsigned)((units + 3) / 4)), block(256);
    if (dtype == F32)
        hipLaunchKernelGGL(kv8_read_k<float>, grid, block, 0, s, n_layers, B, n, first, count, (float*)out_k, (float*)out_v, kv);
    else
        hipLaunchKernelGGL(kv8_read_k<bf16>, grid, block, 0, s, n_layers, B, n, first, count, (bf16*)out_k, (bf16*)out_v, kv);
    return hipGetLastError();
}

// ---- commit
// Row seq_len + path[j] -> row seq_len + j, j = 1 .. accept_len.  A thread owns one 16-byte column of a (layer, kv head)'s K or V rows, or the exponent
// bytes of either, for all j, and walks j upward in batches of 8 (8 loads in flight, then 8 stores).  A row that is written can only be the source
// of an earlier j (path[j] >= j), which the same thread has read by then.  ONE: a workgroup has all columns of its sequence and advances the length too;
// else workgroups of a sequence may still have to read it, and a second kernel does.
__device__ __forceinline__ int accepted(const int32_t* __restrict__ accept_len, int b, int stride) { return max(min(accept_len[b], min(stride - 1, 63)), 0); }

template <bool ONE>
__global__ __launch_bounds__(1024) void kv8_commit_k(int n_layers, KV8Layer kv, int32_t* __restrict__ seq_len, const int32_t* __restrict__ accept_len,
                                                     const int32_t* __restrict__ path_idx, int stride) {
    __shared__ int64_t s_src[64], s_dst[64];
    const int b = blockIdx.y, tid = threadIdx.x;
    // (the path does not wait for the length of what was accepted: on cold memory each step of this chain costs 1 to 2 us)
    const int ctx = seq_len[b], p = tid < min(stride, 64) ? path_idx[(int64_t)b * stride + tid] : 0;
    const int a = accepted(accept_len, b, stride);
    if (!ONE && a == 0) return;
    if (tid < 64) {
        int64_t src = -1, dst = -1;
        if (tid >= 1 && tid <= a) {
            if (p > tid && p < 64 && ctx >= 0 && ctx < 0x7fffffff - 64) src = row_of(kv, b, ctx + p), dst = row_of(kv, b, ctx + tid);
        }
        s_src[tid] = dst < 0 ? -1 : src, s_dst[tid] = dst;
        if (ONE && tid == 0) seq_len[b] = ctx + a + 1;
    }
    __syncthreads();
    const int cols = kv.d / 16, per_head = 2 * cols + 2, units = a > 0 ? n_layers * kv.n_kv * per_head : 0;
    const int64_t rows_per_layer = kv.n_pages * kv.n_kv * kv.page_size;
    for (int u = blockIdx.x * blockDim.x + tid; u < units; u += gridDim.x * blockDim.x) {
        const int head = u / per_head, c = u - head * per_head, layer = head / kv.n_kv, kh = head - layer * kv.n_kv;
        const int64_t base = layer * rows_per_layer + (int64_t)kh * kv.page_size;
        if (c < 2 * cols) {
            uint8_t* pool = (c < cols ? kv.k : kv.v) + base * kv.d + (c < cols ? c : c - cols) * 16;
            for (int j0 = 1; j0 <= a; j0 += 8) {
                u32x4_t t[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j0 + e <= a && s_src[j0 + e] >= 0) t[e] = *(const u32x4_t*)(pool + s_src[j0 + e] * kv.d);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j0 + e <= a && s_src[j0 + e] >= 0) *(u32x4_t*)(pool + s_dst[j0 + e] * kv.d) = t[e];
            }
        } else {
            uint8_t* pool = (c == 2 * cols ? kv.k_exp : kv.v_exp) + base;
            for (int j0 = 1; j0 <= a; j0 += 8) {
                uint8_t t[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j0 + e <= a && s_src[j0 + e] >= 0) t[e] = pool[s_src[j0 + e]];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j0 + e <= a && s_src[j0 + e] >= 0) pool[s_dst[j0 + e]] = t[e];
            }
        }
    }
}

__global__ void kv8_advance_k(int B, int32_t* __restrict__ seq_len, const int32_t* __restrict__ accept_len, int stride) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B) seq_len[b] += accepted(accept_len, b, stride) + 1;
}

hipError_t kv8_commit(hipStream_t s, int n_layers, int B, const KV8Layer& kv, int32_t* seq_len, const int32_t* accept_len, const int32_t* path_idx, int stride) {
    const int64_t units = (int64_t)n_layers * kv.n_kv * (2 * (kv.d / 16) + 2);
    // One launch while a thread has two columns at most: a second launch costs its caller 2.8 us (3 with cold caches on the GPU, 2 with warm ones), a third turn more. One / two, us,
    // 8 and 32 sequences, 4 accepted, heads of 128: captured behind a fill kernel, eager behind one (the caller's time), alone on cold caches.
    //   864 columns (12 layers of 4 heads)   8.6 / 9.6, 8.9 / 9.7       11.3 / 14.1, 11.2 / 14.1   13.8 / 14.6, 14.0 / 14.7
    //   1152                                 10.2 / 9.7, 10.3 / 9.8     11.3 / 14.1, 11.3 / 14.0   17.6 / 14.7, 18.0 / 15.9
    //   2016 (28 of 4)                       11.1 / 9.7, 11.8 / 10.0    11.2 / 14.0, 11.2 / 13.9   18.4 / 14.9, 19.5 / 16.0
    //   2304                                 12.8 / 9.8, 13.4 / 10.2    11.6 / 14.0, 11.7 / 14.0   21.9 / 15.1, 23.7 / 15.9
    //   4032 (28 of 8)                       15.9 / 9.9, 17.1 / 10.7    14.2 / 13.7, 14.8 / 14.0   27.6 / 15.1, 29.5 / 17.5
    // (Between 1024 and 2048 columns the caller's gain stands against the GPU's loss: one launch for callers that enqueue step by step, who pay for it in every step.)
    if (units <= 2048) {
        const int threads = (int)std::min<int64_t>(1024, (units + 63) / 64 * 64);
        hipLaunchKernelGGL(kv8_commit_k<true>, dim3(1, B), dim3(threads), 0, s, n_layers, kv, seq_len, accept_len, path_idx, stride);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(kv8_commit_k<false>, dim3((unsigned)((units + 255) / 256), B), dim3(256), 0, s, n_layers, kv, seq_len, accept_len, path_idx, stride);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kv8_advance_k, dim3((B + 63) / 64), dim3(64), 0, s, B, seq_len, accept_len, stride);
    return hipGetLastError();
}

// ---- attention, a workgroup per (row, query head): any dtype and shape
// Four waves, each taking every fourth tile of 64 keys: lanes own keys for the scores and 16-code pieces of value rows for the sums; the running maximum
// and sum of a wave's tiles, the waves merged at the end.  A simple kernel for small decoders and tests, bound by latency (two sequences of 128 keys with 5 nodes, 7 us);
// it reads the keys of a kv head once per row and query head.
constexpr int kRowWaves = 4;
template <typename T>
__global__ __launch_bounds__(64 * kRowWaves) void kv8_attn_row_k(KV8Rows rows, KV8Layer kv, const T* __restrict__ q, int64_t q_stride, T* __restrict__ out,
                                                                 int n_q_heads, float scale) {
    __shared__ __align__(16) float q_s[256], o_s[kRowWaves][1024];   // (groups * head_dim is 1024 at most)
    __shared__ float m_s[kRowWaves], l_s[kRowWaves], p_s[kRowWaves][64];
    __shared__ int64_t at_s[kRowWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tid = threadIdx.x;
    const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, r = b * rows.n + i, d = kv.d;
    const int kh = hq / (n_q_heads / kv.n_kv);
    const int ctx = min(max(kv.seq_len[b], 0), kv.seq_len_bound), total = ctx + rows.n;
    const uint64_t mask = rows.mask ? rows.mask[r] : (2ull << i) - 1ull;   // (none: the rows up to this one)
    if (tid < d) q_s[tid] = to_float(q[(int64_t)r * q_stride + hq * d + tid]) * scale;
    __syncthreads();
    const int lpk = d / 16, groups = 64 / lpk, grp = lane / lpk, piece = (lane - grp * lpk) * 16;
    float m = -INFINITY, l = 0.f, acc[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    for (int t0 = 64 * wave; t0 < total; t0 += 64 * kRowWaves) {
        const int key = t0 + lane, jj = key - ctx;
        const int64_t at0 = key < total ? row_of(kv, b, key) : -1;
        const bool vis = key < total && (jj < 0 || ((mask >> (jj & 63)) & 1ull));
        // (a visible key without a page counts as a key and a value of zero)
        const int64_t at = at0 < 0 ? -1 : at0 + (int64_t)kh * kv.page_size;
        float s = 0.f;
        if (vis && at >= 0) {
            const uint32_t ke = kv.k_exp[at];
            for (int c0 = 0; c0 < d; c0 += 64) {
                u32x4_t w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    w[c] = *(const u32x4_t*)(kv.k + at * d + c0 + 16 * c);
                    if (ke >= kTopExp) w[c] = finite16(w[c]);
                }
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    float f[4];
                    decode4(w[c >> 2][c & 3], 1.f, f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s = fmaf(q_s[c0 + 4 * c + e], f[e], s);
                }
            }
            s *= scale_of(ke);
        }
        if (!vis) s = -INFINITY;
        const float m_new = fmaxf(m, wave_max(s));   // (a NaN does not count here; it comes through the weights)
        const float ref = m_new == -INFINITY ? 0.f : m_new;
        const float corr = expf(m - ref), p = vis ? expf(s - ref) : 0.f;
        l = l * corr + wave_sum(p);
        m = m_new;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] *= corr;
        p_s[wave][lane] = at >= 0 ? p : 0.f;
        at_s[wave][lane] = vis ? at : -1;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // (read back by the same wave only)
        __builtin_amdgcn_wave_barrier();
        if (grp < groups)
            for (int k = grp; k < 64; k += groups) {
                const int64_t kat = at_s[wave][k];
                if (kat < 0) continue;
                const uint32_t ve = kv.v_exp[kat];
                const float w = p_s[wave][k] * scale_of(ve);
                u32x4_t v = *(const u32x4_t*)(kv.v + kat * d + piece);
                if (ve >= kTopExp) v = finite16(v);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float f[4];
                    decode4(v[c], 1.f, f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[4 * c + e] = fmaf(w, f[e], acc[4 * c + e]);
                }
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    if (grp < groups)
#pragma unroll
        for (int e = 0; e < 16; ++e) o_s[wave][grp * d + piece + e] = acc[e];
    if (lane == 0) m_s[wave] = m, l_s[wave] = l;
    __syncthreads();
    if (tid >= d) return;
    float mm = m_s[0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) mm = fmaxf(mm, m_s[w]);
    float ll = 0.f, a = 0.f;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) {
        const float f = m_s[w] == -INFINITY ? (l_s[w] == 0.f ? 0.f : 1.f) : expf(m_s[w] - mm);   // (keys of NaN only: their sum is NaN)
        float o_w = 0.f;
        for (int g = 0; g < groups; ++g) o_w += o_s[w][g * d + tid];
        ll += f * l_s[w];
        a += f * o_w;
    }
    const bool sees = ctx > 0 || (mask & (~0ull >> (64 - rows.n))) != 0;   // (a row that sees something and has a sum of zero has scores of -infinity only: 0 / 0)
    out[((int64_t)r * n_q_heads + hq) * d + tid] = from_float<T>(ll == 0.f && !sees ? 0.f : a / ll);
}

// ---- attention by matrix instructions: bf16, head_dim 128, pages of 16
// The rows of a kv head are its G query heads times the n nodes, r = i * G + g, in tiles of 16.  Both products run on v_mfma_f32_16x16x32_bf16 in the
// transposed orientation, S^T[key][row] = K Q^T and O^T[d][row] = V^T P^T: a lane's scores are four consecutive keys of its own row, which is what the
// second product's B operand wants, and its accumulators all belong to that row.  Codes become bf16 exactly, exponent included, in one conversion per
// two elements.  (The 8-bit matrix instructions would take the codes as they are, with the queries in two parts; but they add products up with
// 12 bits below the largest one, measured: a score whose products cancel would be off by their size / 4096.)
//
// A work item is (sequence, range of tiles of 64 keys); every item is run by n_kv workgroups (times the groups of row tiles), which leave
// unnormalised outputs with their maximum and sum in fp32, and a second kernel joins the items of a sequence.  The ranges follow from the lengths on the
// device: every wave works them out for itself (up to 256 sequences), which costs less than a kernel in front.
constexpr int kD = 128, kKT = 64;
constexpr float kNegBig = -1e30f;
constexpr int kPlanned = 256;   // most sequences whose ranges are balanced

template <typename F>
__device__ __forceinline__ int wave_all(int v, F op) {
    const auto a = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    v = op((int)a[0], (int)a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = op((int)b[0], (int)b[1]);
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, false));
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, false));
    v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false));
    return op(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false));
}
__device__ __forceinline__ int wave_sum_i(int v) {
    return wave_all(v, [](int x, int y) { return x + y; });
}
// the maximum over lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float group_max4(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float m = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

struct KV8Item {
    int b, ctx;        // sequence, its committed length (no more than the bound that the grid was made for)
    int lo, hi;        // tiles
    int slot, first;   // partial result of this range, of the sequence's first range
    int k;             // ranges of the sequence
};
struct KV8Split {
    int slots;         // items that run at once
    int t_max;         // longest range, in tiles
    int whole;         // sequences of that many tiles are not cut to fill the chip
    bool planned;      // ranges are balanced, else all are of t_max
    int max_items;     // upper bound of the item count, from the host's bound on the lengths
};

// Shortest range where the longest sequence has that many tiles: a range's time grows with its length, the joining with the number of ranges, so their
// best balance grows with the root of the tiles.  (One sequence, 28 and 4 heads, ranges of 2, 4, 8 and 16: one token at 2048 keys 8.6, 9.8, 10.5, 11.6 us, at 8192
// 11.8, 9.7, 11.1, 14.0, at 30000 16.3, 15.5, 13.2, 17.0; 8 nodes at 2048 11.8, 14.1, 15.8, 19.3, at 30000 21.9, 21.8, 20.9, 26.1.)  Up to `whole` tiles cost less
// than a joining (32 sequences of 200 keys with 16 nodes, four tiles: 13 us, cut in two 22).
__host__ __device__ __forceinline__ int shortest_range(int tiles, int whole) {
    const int t = tiles <= whole ? tiles : (int)sqrtf((float)tiles * (1.f / 7.f));
    return t < 2 ? 2 : (t > 32 ? 32 : t);
}

// Item number `item`: false where there is none.  Planned: of the range lengths from the shortest to t_max the smallest whose items fit the
// fewest rounds of `slots` that t_max allows; items are numbered sequence by sequence.  Not planned: ranges of t_max, item = range * B + sequence.
__device__ __forceinline__ bool kv8_item(const int32_t* __restrict__ seq_len, int B, int n, int len_bound, const KV8Split& sp, int item, KV8Item& out) {
    const int lane = threadIdx.x & 63;
    auto len_of = [&](int b) { return min(max(seq_len[b], 0), len_bound); };
    auto ceil_div = [](int x, int T) { return (int)__umulhi((uint32_t)(x + T - 1), 0xffffffffu / (uint32_t)T + 1u); };   // (exact: x < 2^26, 2 <= T <= 64)
    // (everything about an item is uniform, and said to be)
    auto give = [&](int b, int len, int tiles, int slot, int first, int k) {
        const int c = __builtin_amdgcn_readfirstlane(sp.planned ? slot - first : slot / B), per = tiles / k, more = tiles - per * k;   // the first `more` ranges are one tile longer
        out.b = __builtin_amdgcn_readfirstlane(b);
        out.ctx = __builtin_amdgcn_readfirstlane(len);
        out.lo = __builtin_amdgcn_readfirstlane(c * per + min(c, more));
        out.hi = __builtin_amdgcn_readfirstlane(out.lo + per + (c < more ? 1 : 0));
        out.slot = __builtin_amdgcn_readfirstlane(slot);
        out.first = __builtin_amdgcn_readfirstlane(first);
        out.k = __builtin_amdgcn_readfirstlane(k);
        return true;
    };
    if (!sp.planned) {
        const int b = item % B, len = len_of(b), tiles = (len + n + kKT - 1) / kKT, k = (tiles + sp.t_max - 1) / sp.t_max;
        return item / B < k && give(b, len, tiles, item, b, k);
    }
    int len[kPlanned / 64], tiles[kPlanned / 64];
#pragma unroll
    for (int j = 0; j < kPlanned / 64; ++j) {
        const int b = 64 * j + lane;
        len[j] = b < B ? len_of(b) : 0;
        tiles[j] = b < B ? (len[j] + n + kKT - 1) / kKT : 0;
    }
    auto items = [&](int T) {
        int s = 0;
#pragma unroll
        for (int j = 0; j < kPlanned / 64; ++j)
            if (64 * j < B) s += ceil_div(tiles[j], T);
        return wave_sum_i(s);
    };
    int longest = 0;
#pragma unroll
    for (int j = 0; j < kPlanned / 64; ++j) longest = max(longest, tiles[j]);
    int T = shortest_range(__builtin_amdgcn_readfirstlane(wave_all(longest, [](int x, int y) { return max(x, y); })), sp.whole);
    if (items(T) > sp.slots) {
        const int most = (items(sp.t_max) + sp.slots - 1) / sp.slots * sp.slots;
        int sum = 0;
#pragma unroll
        for (int j = 0; j < kPlanned / 64; ++j) sum += tiles[j];
        sum = wave_sum_i(sum);
        // items(T) is at least sum / T and at most sum / T + B, and longer ranges never make more items
        T = min(max(T, (sum + most - 1) / most), sp.t_max);
        int up = most > B ? min(max((sum + most - B - 1) / (most - B), T), sp.t_max) : sp.t_max;
        while (T < up) {
            const int mid = (T + up) >> 1;
            if (items(mid) <= most) up = mid; else T = mid + 1;
        }
    }
    T = __builtin_amdgcn_readfirstlane(T);
    int base = 0;
#pragma unroll
    for (int j = 0; j < kPlanned / 64; ++j) {
        if (64 * j >= B) break;
        const int k = ceil_div(tiles[j], T);
        int end = k;
        for (int o = 1; o < min(B - 64 * j, 64); o <<= 1) {
            const int x = __shfl_up(end, o, 64);
            if (lane >= o) end += x;
        }
        const uint64_t hit = __builtin_amdgcn_ballot_w64(item >= base + end - k && item < base + end);
        if (hit) {
            const int l = __ffsll((unsigned long long)hit) - 1;
            const int kk = __builtin_amdgcn_readlane(k, l), tt = __builtin_amdgcn_readlane(tiles[j], l);
            return give(64 * j + l, __builtin_amdgcn_readlane(len[j], l), tt, item, base + __builtin_amdgcn_readlane(end, l) - kk, kk);
        }
        base += __builtin_amdgcn_readlane(end, min(B - 64 * j, 64) - 1);
    }
    return false;
}

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

// codes 2w, 2w + 1 of a dword times 2^(e - 127), as bf16 (scale: a float of that exponent; E = 255 makes it infinite, which gives NaN)
template <bool HI>
__device__ __forceinline__ uint32_t cvt2(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}
__device__ __forceinline__ u32x4_t cvt8(uint32_t c0, uint32_t c1, float scale) {
    return u32x4_t{cvt2<false>(c0, scale), cvt2<true>(c0, scale), cvt2<false>(c1, scale), cvt2<true>(c1, scale)};
}
typedef __amdgpu_buffer_rsrc_t buffer_t;
__device__ __forceinline__ buffer_t buffer_of(const void* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00020000); }

// Which of the keys first .. first + 63 a row sees, `first` counted from the end of the context, by its mask over the new rows.
__device__ __forceinline__ uint64_t seen_from(int first, uint64_t mask) {
    const uint64_t up = first < 64 ? mask >> (first & 63) : 0ull, down = first > -64 ? ~(~mask << (-first & 63)) : ~0ull;
    return first >= 0 ? up : down;
}

struct KV8Seg {   // per sequence, for the joining kernel
    int first, k;
};

// What a wave holds of NT tiles of rows: queries in the order of the keys' pieces, unnormalised sums, the weights' sums, the reference of the
// exponentials.  Lane (l16, g4) has row l16 of a tile.
template <int NT>
struct KV8Tiles {
    u32x4_t q[NT][4];
    f32x4_t acc[NT][8], l[NT];
    float m[NT];
};
// Visibility of row r over the new rows
__device__ __forceinline__ uint64_t kv8_mask(const KV8Rows& rows, int b, int G, int r) {
    const int n = rows.n, i = r / G;
    return r >= n * G ? 0ull : (rows.mask ? rows.mask[b * n + i] : (2ull << i) - 1ull) & (~0ull >> (64 - n));
}
template <int NT, typename F>   // row_of_tile(t): first row of tile t
__device__ __forceinline__ void kv8_tiles(KV8Tiles<NT>& x, const KV8Rows& rows, int b, int kh, int G, const uint16_t* __restrict__ q, int64_t q_stride, F row_of_tile) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, g4 = lane >> 4, n = rows.n;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = row_of_tile(t) + l16, i = r / G, g = r - i * G;
        const bool on = r < n * G;
        const uint16_t* p = q + (int64_t)(b * n + (on ? i : 0)) * q_stride + (kh * G + (on ? g : 0)) * kD + 16 * g4;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const u32x4_t z = {0u, 0u, 0u, 0u};
            x.q[t][ks] = on ? *(const u32x4_t*)(p + (ks >> 1) * 64 + (ks & 1) * 8) : z;
        }
        x.m[t] = kNegBig;
        x.l[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) x.acc[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
}
// S^T of 16 keys, whose codes lane (l16, g4) has of key l16, pieces g4 and 4 + g4.  Values that are not finite: their codes are zero, the NaN comes through the
// score, which only rows that see the key keep.
template <int NT>
__device__ __forceinline__ void kv8_scores(const KV8Tiles<NT>& x, u32x4_t c0, u32x4_t c1, uint32_t k_exp, uint32_t v_exp, f32x4_t* const (&sc)[NT]) {
    const float scale = __uint_as_float((v_exp == 255u ? 255u : k_exp) << 23);
    bf16x8_t kf[4];
    kf[0] = __builtin_bit_cast(bf16x8_t, cvt8(c0[0], c0[1], scale));
    kf[1] = __builtin_bit_cast(bf16x8_t, cvt8(c0[2], c0[3], scale));
    kf[2] = __builtin_bit_cast(bf16x8_t, cvt8(c1[0], c1[1], scale));
    kf[3] = __builtin_bit_cast(bf16x8_t, cvt8(c1[2], c1[3], scale));
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        *sc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) *sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks], __builtin_bit_cast(bf16x8_t, x.q[t][ks]), *sc[t], 0, 0, 0);
    }
}
// Scores sc[t][s][v] of keys t0 + 16 * s + 4 * g4 + v to weights, packed for the second product: k slot 4 * (s & 1) + v of half s / 2.  behind: t0 less the
// context's length; edge: some keys are new rows or lie behind the last; mask_of(t, lane): visibility of the lane's row of tile t.
template <int NT, typename F>
__device__ __forceinline__ void kv8_weights(KV8Tiles<NT>& x, f32x4_t (&sc)[NT][4], u32x4_t (&pb)[NT][2], bool edge, int behind, F mask_of, float scale_log2, float lazy) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (edge) {
            int ln = threadIdx.x & 63;
            asm volatile("" : "+v"(ln));   // (worked out anew where it is wanted: kept through the loop, such values cost registers that the products need)
            const uint64_t seen = seen_from(behind + 4 * (ln >> 4), mask_of(t, ln));
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int v = 0; v < 4; ++v) sc[t][s][v] = seen >> (16 * s + v) & 1ull ? sc[t][s][v] : kNegBig;
        }
        float tmax = kNegBig;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int v = 0; v < 4; ++v) tmax = fmaxf(tmax, sc[t][s][v]);
        // the reference of the exponentials only has to keep them in range: it follows the maximum when some score exceeds it by 2^8
        if (__builtin_amdgcn_ballot_w64(tmax > x.m[t] + lazy) != 0) {
            const float m_new = fmaxf(x.m[t], group_max4(tmax));
            const float alpha = __builtin_amdgcn_exp2f((x.m[t] - m_new) * scale_log2);
            x.m[t] = m_new;
            x.l[t] *= alpha;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) x.acc[t][dt] *= alpha;
        }
        const float mc = fmaxf(x.m[t], -1e29f) * scale_log2;   // (rows that have seen nothing yet: exp2(-1e30 * c + 1e29 * c) = 0)
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            float e[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) e[v] = __builtin_amdgcn_exp2f(fmaf(sc[t][s][v], scale_log2, -mc));
            // Weights are rounded to bf16, what the second product takes beside values in bf16: each by 2^-8 of itself at most, which moves the mean by 2^-8 (mean |v| + |o|) at
            // most, as much as the rounding of the output to bf16 for values of one size; their sum is that of the rounded ones, so that a common factor cancels.  (Two
            // products, of a weight's upper and lower half, would double the second product, half of the matrix work.)
            pb[t][s >> 1][2 * (s & 1)] = pack_bf16x2(e[0], e[1]);
            pb[t][s >> 1][2 * (s & 1) + 1] = pack_bf16x2(e[2], e[3]);
        }
    }
}
// O^T += V^T P^T over 32 keys: vc[sub][v] has 8 codes, d = 8 * l16 .., of key 16 * sub + 4 * g4 + v, byte v of ve[sub] its exponent.  Pairs of d are converted,
// pairs of keys made by byte permutations; instruction dt has d = 8 * l16 + dt.
template <int NT>
__device__ __forceinline__ void kv8_sums(KV8Tiles<NT>& x, const u32x2_t (&vc)[2][4], uint32_t ve0, uint32_t ve1, const u32x4_t* const (&pb)[NT]) {
    float scale[8];
#pragma unroll
    for (int a = 0; a < 8; ++a) {
        const uint32_t e8 = ((a < 4 ? ve0 : ve1) >> (8 * (a & 3))) & 255u;
        scale[a] = __uint_as_float((e8 == 255u ? 127u : e8) << 23);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint32_t y[8];
#pragma unroll
        for (int a = 0; a < 8; ++a) {
            const uint32_t w = vc[a >> 2][a & 3][c >> 1];
            y[a] = c & 1 ? cvt2<true>(w, scale[a]) : cvt2<false>(w, scale[a]);
        }
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            u32x4_t a;
#pragma unroll
            for (int p = 0; p < 4; ++p) a[p] = __builtin_amdgcn_perm(y[2 * p + 1], y[2 * p], o ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int t = 0; t < NT; ++t)
                x.acc[t][2 * c + o] =
                    __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, *pb[t]), x.acc[t][2 * c + o], 0, 0, 0);
        }
    }
    const u32x4_t ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
    for (int t = 0; t < NT; ++t)
        x.l[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ones), __builtin_bit_cast(bf16x8_t, *pb[t]), x.l[t], 0, 0, 0);
}
// Where a row's result goes: the output, or the partial results of its range.  sees: the row sees anything.  Its largest weight is 1 or more, so a sum of zero means
// that all its scores are -infinity: 0 / 0.  (A sequence of two ranges or more has a context, so that every row does: where ranges are joined, nobody asks.)
struct KV8Out {
    uint16_t* out;
    float *part_o, *part_ml;
    int n, n_q_heads, n_kv, r_pad;
    __device__ __forceinline__ void put4(const KV8Item& it, int kh, int G, int r, int c, f32x4_t o, float M, float L, bool sees) const {
        if (it.k == 1) {
            const float inv = L == 0.f && !sees ? 0.f : 1.0f / L;
            const int i = r / G, g = r - i * G;
            *(u32x2_t*)(out + ((int64_t)(it.b * n + i) * n_q_heads + kh * G + g) * kD + c) = u32x2_t{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
        } else {
            const int64_t at = ((int64_t)it.slot * n_kv + kh) * r_pad + r;
            *(f32x4_t*)(part_o + at * kD + c) = o;
            if (c == 0) part_ml[at * 2] = M, part_ml[at * 2 + 1] = L;
        }
    }
    // 8 sums of row r from column c on, their weights' sum L and reference M
    __device__ __forceinline__ void put8(const KV8Item& it, int kh, int G, int r, int c, const float* o, float M, float L, bool sees) const {
        if (it.k == 1) {
            const float inv = L == 0.f && !sees ? 0.f : 1.0f / L;
            const int i = r / G, g = r - i * G;
            uint16_t* p = out + ((int64_t)(it.b * n + i) * n_q_heads + kh * G + g) * kD + c;
            *(u32x4_t*)p = u32x4_t{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv), pack_bf16x2(o[4] * inv, o[5] * inv),
                                   pack_bf16x2(o[6] * inv, o[7] * inv)};
        } else {
            const int64_t at = ((int64_t)it.slot * n_kv + kh) * r_pad + r;
#pragma unroll
            for (int e = 0; e < 8; e += 4) *(f32x4_t*)(part_o + at * kD + c + e) = f32x4_t{o[e], o[e + 1], o[e + 2], o[e + 3]};
            if (c == 0) part_ml[at * 2] = M, part_ml[at * 2 + 1] = L;
        }
    }
};

// Few rows (NT tiles of 16): bound by memory.  A wave of the workgroup's four owns every fourth tile of the item's range with all rows, takes codes from
// memory straight into the registers that the products want (no LDS, no barrier until the end) and keeps the next tile's in flight: keys once the
// scores are done, values once the sums are.  The waves are joined through LDS.  64 sequences of ~8192 keys, 40 and 8 heads, one token: 1.08 GB in 177 us (6.1
// TB/s); 16 of 8192, 28 and 4 heads: 135 MB in 28.6 us (4.7 TB/s, most of a fixed 5 us being planning and the first tile's way from memory); one: 6.9 us.
// Two waves per SIMD: three have no registers for the next tile (the same 64 sequences 205 us).
template <int NT>
__global__ __launch_bounds__(256, 2) void kv8_attn_few_k(KV8Split sp, int64_t q_stride, const uint16_t* __restrict__ q, KV8Rows rows, KV8Layer kv, KV8Out to,
                                                                      KV8Seg* __restrict__ seg, float scale_log2, float lazy) {
    constexpr int kPad = kD + 4;
    __shared__ __align__(16) float o_s[4][16][kPad];
    __shared__ float m_s[4][16], l_s[4][16];
    const int n_kv = kv.n_kv, kh = blockIdx.x % n_kv;
    KV8Item it;
    if (!kv8_item(kv.seq_len, rows.B, rows.n, kv.seq_len_bound, sp, blockIdx.x / n_kv, it)) return;   // uniform
    const int b = it.b, ctx = it.ctx, total = ctx + rows.n;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int G = to.n_q_heads / n_kv, R = rows.n * G;
    if (kh == 0 && it.slot == it.first && tid == 0) seg[b] = KV8Seg{it.first, it.k};
    // pages of this wave's tiles (ranges are 64 tiles at most, so 16 of them), lane 4 * i + s: page s of the i-th; -1: none
    const int my_tiles = (it.hi - it.lo - wave + 3) >> 2;   // (0 or less: none)
    int pages;
    {
        const int lp = (it.lo + wave + 4 * (lane >> 2)) * 4 + (lane & 3);
        pages = (lane >> 2) < my_tiles && lp < kv.max_pages && lp * 16 < total ? kv.block_table[(int64_t)b * kv.max_pages + lp] : -1;
        pages = pages < kv.n_pages ? pages : -1;
    }
    // codes and exponents of tile i; a page that is not there reads as zeros
    u32x4_t kc[4][2];
    u32x2_t vc[2][2][4];
    uint32_t ke[4], kve[4], ve[4];   // (kve: the exponents of the values of the lane's key)
    const int k_off = l16 * kD + 16 * g4, v_off = g4 * (4 * kD) + 8 * l16;
    auto page_row = [&](int pg) { return ((int64_t)max(pg, 0) * n_kv + kh) * 16; };
    auto load_k = [&](int i) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int pg = __builtin_amdgcn_readlane(pages, i * 4 + s);
            const int64_t row = page_row(pg);
            const buffer_t r = buffer_of(kv.k + row * kD, pg < 0 ? 0 : 16 * kD), re = buffer_of(kv.k_exp + row, pg < 0 ? 0 : 16);
            const buffer_t rv = buffer_of(kv.v_exp + row, pg < 0 ? 0 : 16);
            ke[s] = __builtin_amdgcn_raw_buffer_load_b8(re, l16, 0, 0);
            kve[s] = __builtin_amdgcn_raw_buffer_load_b8(rv, l16, 0, 0);
#pragma unroll
            for (int h = 0; h < 2; ++h) kc[s][h] = __builtin_amdgcn_raw_buffer_load_b128(r, k_off, 64 * h, 2);   // (2: read once)
        }
    };
    auto load_v = [&](int i) {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int pg = __builtin_amdgcn_readlane(pages, i * 4 + s);
            const int64_t row = page_row(pg);
            const buffer_t r = buffer_of(kv.v + row * kD, pg < 0 ? 0 : 16 * kD), re = buffer_of(kv.v_exp + row, pg < 0 ? 0 : 16);
            ve[s] = __builtin_amdgcn_raw_buffer_load_b32(re, 4 * g4, 0, 0);
#pragma unroll
            for (int v = 0; v < 4; ++v) vc[s >> 1][s & 1][v] = __builtin_amdgcn_raw_buffer_load_b64(r, v_off, v * kD, 2);
        }
    };
    if (my_tiles > 0) load_k(0), load_v(0);
    KV8Tiles<NT> x;
    kv8_tiles(x, rows, b, kh, G, q, q_stride, [](int t) { return 16 * t; });
    uint64_t mask[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) mask[t] = kv8_mask(rows, b, G, 16 * t + l16);
    for (int i = 0; i < my_tiles; ++i) {
        const int t0 = (it.lo + wave + 4 * i) * kKT;
        const bool edge = t0 + kKT > ctx;
        f32x4_t sc[NT][4];
        u32x4_t pb[NT][2];
        // (rows near the type's largest value, and those that are not finite; the lanes have the exponents of all 64 keys and values)
        const uint32_t top_exp = max(max(max(ke[0], ke[1]), max(ke[2], ke[3])), max(max(kve[0], kve[1]), max(kve[2], kve[3])));
        for (int rep = __builtin_amdgcn_ballot_w64(top_exp >= kTopExp) != 0 ? 0 : 1; rep < 1; ++rep) {   // (a loop, which stays a branch)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
#pragma unroll
                for (int h = 0; h < 2; ++h) kc[s][h] = ke[s] >= kTopExp ? finite16(kc[s][h]) : kc[s][h];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    u32x2_t& c = vc[s >> 1][s & 1][v];
                    c = (ve[s] >> (8 * v) & 255u) >= kTopExp ? u32x2_t{finite4(c[0]), finite4(c[1])} : c;
                }
            }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            f32x4_t* to_sc[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) to_sc[t] = &sc[t][s];
            kv8_scores(x, kc[s][0], kc[s][1], ke[s], kve[s], to_sc);
        }
        if (i + 1 < my_tiles) load_k(i + 1);
        kv8_weights(x, sc, pb, edge, t0 - ctx, [&](int t, int) { return mask[t]; }, scale_log2, lazy);
        if (edge) {   // (keys behind the last are weighted with zero, and slots that nobody has written may hold anything)
            int ln = lane;
            asm volatile("" : "+v"(ln));
            const int left = total - t0 - 4 * (ln >> 4);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int v = 0; v < 4; ++v) vc[s >> 1][s & 1][v] = 16 * s + v < left ? vc[s >> 1][s & 1][v] : u32x2_t{0u, 0u};
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const u32x4_t* w[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) w[t] = &pb[t][half];
            kv8_sums(x, vc[half], ve[2 * half], ve[2 * half + 1], w);
        }
        if (i + 1 < my_tiles) load_v(i + 1);
    }
    // ---- the waves joined, a tile of rows at a time: lane (l16, g4) holds d = 32 * g4 + 8 * v + dt of row l16
    int le = lane;
    asm volatile("" : "+v"(le));
    const int row_e = le & 15, grp_e = le >> 4;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t > 0) __syncthreads();
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            *(f32x4_t*)&o_s[wave][row_e][32 * grp_e + 8 * v] = f32x4_t{x.acc[t][0][v], x.acc[t][1][v], x.acc[t][2][v], x.acc[t][3][v]};
            *(f32x4_t*)&o_s[wave][row_e][32 * grp_e + 8 * v + 4] = f32x4_t{x.acc[t][4][v], x.acc[t][5][v], x.acc[t][6][v], x.acc[t][7][v]};
        }
        if (grp_e == 0) m_s[wave][row_e] = x.m[t], l_s[wave][row_e] = x.l[t][0];
        __syncthreads();
        const int rl = tid >> 4, c = (tid & 15) * 8;
        if (16 * t + rl >= R) continue;
        float M = kNegBig, L = 0.f, w[4], o[8];
#pragma unroll
        for (int y = 0; y < 4; ++y) M = fmaxf(M, m_s[y][rl]);
#pragma unroll
        for (int y = 0; y < 4; ++y) w[y] = __builtin_amdgcn_exp2f((m_s[y][rl] - M) * scale_log2), L += w[y] * l_s[y][rl];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(w[y], o_s[y][rl][c + e], o[e]);
        to.put8(it, kh, G, 16 * t + rl, c, o, M, L, ctx > 0 || kv8_mask(rows, b, G, 16 * t + rl) != 0);
    }
}

// From memory straight into LDS, lane i's 16 (4) bytes at base + offset to lds_bytes + 16 (4) * i.  The compiler does not count these loads: they are
// waited for by number.
__device__ __forceinline__ void dma_16(const uint8_t* base, uint32_t offset, uint32_t lds_bytes) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" : : "v"(offset), "s"(base), "s"(lds_bytes) : "memory", "m0");
}
__device__ __forceinline__ void dma_4(const uint8_t* base, uint32_t offset, uint32_t lds_bytes) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(offset), "s"(base), "s"(lds_bytes) : "memory", "m0");
}
template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_at(uint32_t offset) { return (__attribute__((address_space(3))) T*)(uintptr_t)offset; }

// More rows: bound by the matrix pipe and, side by side with it, the exponentials (32 sequences of ~4096 keys, 28 and 4 heads, 48 nodes, 91 GFLOP: 119 us, 64 % of
// the rate of a large product; the matrix pipes are busy 43 % of it).  One workgroup of eight waves, two per SIMD, streams the item's range once for up to 24
// tiles of rows, dealt round-robin to the waves (NT each).  A tile of 64 keys passes through LDS twice: its codes come from memory by direct loads, kRaw tiles ahead,
// a wave's eight keys (1 KB each of K and V) to a place that only this wave reads; the wave converts them to bf16 and stores them for all, K rows swizzled by
// the key (the 16-byte fragments of 16 keys hit 16 distinct places), V rows by twice the key (a transposing read takes two neighbouring places of each of 8
// keys; the stores of two neighbouring keys, though, meet in the 8 even places and then in the odd ones).  The two waves of a SIMD run half a period apart, so that one's softmax runs under the other's products: per tile a wave does [P V of the tile
// before, Q K^T] and then [softmax, conversion of the next tile], and the early waves 0 .. 3 meet the tile's barrier in front of the first half, the
// late ones 4 .. 7 between the two.  Between barriers `it` and `it + 1` all read K of tile it and V of it - 1, and write both of tile it + 1: two
// stages of K and three of V.
constexpr int kRaw = 3, kRawBytes = 2 * kKT * kD + 2 * kKT, kStage = kKT * kD * 2;   // (raw: K codes, V codes, exponents of K and V)
constexpr int kManyLds = 5 * kStage + kRaw * kRawBytes + 64 * 8;

template <int NT>
__device__ __forceinline__ void kv8_many_body(const KV8Item& it, int kh, int rg, int64_t q_stride, const uint16_t* __restrict__ q, const KV8Rows& rows, const KV8Layer& kv,
                                              const KV8Out& to, int per_group, float scale_log2, float lazy, uint8_t* lds) {
    constexpr int TPW = NT > 0 ? NT : 1;
    typedef __attribute__((ext_vector_type(4))) short s16x4_t;
    typedef __attribute__((ext_vector_type(8))) short s16x8_t;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int b = it.b, ctx = it.ctx, n = rows.n, total = ctx + n, n_kv = kv.n_kv, G = to.n_q_heads / n_kv, R = n * G;
    const int n_tiles = it.hi - it.lo, k0 = it.lo * kKT;
    uint8_t* raw = lds + 5 * kStage;   // (the stages first: their places are worked out with exclusive ors below 256)
    uint64_t* mask_lds = (uint64_t*)(raw + kRaw * kRawBytes);
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;

    // ---- codes and exponents from memory: this wave's keys 8 * wave .. + 7 of a tile lie in one page, lane t of `pages` has that of tile t (a range is 64 tiles at
    // most); -1: none
    int pages;
    {
        const int lp = (it.lo + lane) * 4 + (wave >> 1);
        pages = lane < n_tiles && lp < kv.max_pages && lp * 16 < total ? kv.block_table[(int64_t)b * kv.max_pages + lp] : -1;
        pages = pages < kv.n_pages ? pages : -1;
    }
    constexpr int kOps = 4;   // loads of a fetch
    auto fetch = [&](int t) {   // (of a page that is not there, page 0 instead: the conversion does not look)
        const int64_t row = ((int64_t)max(__builtin_amdgcn_readlane(pages, t), 0) * n_kv + kh) * 16 + (wave & 1) * 8;
        const uint32_t at = __builtin_amdgcn_readfirstlane(base + 5 * kStage + (t % kRaw) * kRawBytes);
        dma_16(kv.k + row * kD, lane * 16, at + wave * 1024);
        dma_16(kv.v + row * kD, lane * 16, at + kKT * kD + wave * 1024);
        if (lane < 2) dma_4(kv.k_exp + row, lane * 4, at + 2 * kKT * kD + wave * 8);
        if (lane < 2) dma_4(kv.v_exp + row, lane * 4, at + 2 * kKT * kD + kKT + wave * 8);
    };
#pragma unroll
    for (int t = 0; t < kRaw; ++t)
        if (t < n_tiles) fetch(t);
    if (tid < n) mask_lds[tid] = kv8_mask(rows, b, G, tid * G);
    KV8Tiles<TPW> x;
    if constexpr (NT > 0) kv8_tiles(x, rows, b, kh, G, q, q_stride, [&](int t) { return (rg * per_group + wave + 8 * t) * 16; });
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");

    // (with three tiles of rows, places in LDS are worked out anew for every tile: kept, they would cost registers that the products need)
    auto place = [](int ln) {
        if constexpr (NT >= 3) asm volatile("" : "+v"(ln));
        return ln;
    };
    // this wave's keys of a tile in registers: 16 codes of key lane / 8 of K and V, and the key's exponents
    struct Raw {
        u32x4_t k, v;
        uint32_t ke, ve;
    };
    auto read_raw = [&](int t, Raw& r) {   // tile t has landed when all but the fetches behind it have
        if (t + kRaw <= n_tiles) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kOps * (kRaw - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const int ln = place(lane);
        const uint8_t* p = raw + (t % kRaw) * kRawBytes;
        r.k = *(const u32x4_t*)(p + wave * 1024 + ln * 16), r.v = *(const u32x4_t*)(p + kKT * kD + wave * 1024 + ln * 16);
        r.ke = p[2 * kKT * kD + wave * 8 + (ln >> 3)], r.ve = p[2 * kKT * kD + kKT + wave * 8 + (ln >> 3)];
    };
    auto convert = [&](int t, Raw& r) {
        const int ln = place(lane), key = 8 * wave + (ln >> 3), p = ln & 7;
        const bool there = __builtin_amdgcn_readlane(pages, t) >= 0;
        const int left = there ? total - k0 - t * kKT : 0;   // (slots that nobody has written may hold anything)
        const bool top = __builtin_amdgcn_ballot_w64(max(r.ke, r.ve) >= kTopExp) != 0;
        for (int rep = left < kKT || top ? 0 : 1; rep < 1; ++rep) {   // (a loop, which stays a branch)
            const bool in = key < left;
#pragma unroll
            for (int y = 0; y < 4; ++y) r.v[y] = in ? r.v[y] : 0u, r.k[y] = there ? r.k[y] : 0u;
            r.ke = there ? r.ke : 127u, r.ve = there ? r.ve : 127u;
            r.k = r.ke >= kTopExp ? finite16(r.k) : r.k;
            r.v = r.ve >= kTopExp ? finite16(r.v) : r.v;
        }
        // (values that are not finite: their codes are zero, the NaN comes through the key, whose score only rows that see it keep)
        const float sk = __uint_as_float((r.ve == 255u ? 255u : r.ke) << 23), sv = __uint_as_float((r.ve == 255u ? 127u : r.ve) << 23);
        uint8_t* ko = lds + (t & 1) * kStage + key * (2 * kD);
        uint8_t* vo = lds + (2 + t % 3) * kStage + key * (2 * kD);
        *(u32x4_t*)(ko + ((2 * p) ^ (key & 15)) * 16) = cvt8(r.k[0], r.k[1], sk);
        *(u32x4_t*)(ko + ((2 * p + 1) ^ (key & 15)) * 16) = cvt8(r.k[2], r.k[3], sk);
        *(u32x4_t*)(vo + ((2 * p) ^ ((2 * key) & 15)) * 16) = cvt8(r.v[0], r.v[1], sv);
        *(u32x4_t*)(vo + ((2 * p + 1) ^ ((2 * key) & 15)) * 16) = cvt8(r.v[2], r.v[3], sv);
        if (t + kRaw < n_tiles) fetch(t + kRaw);   // (the codes have been read: they are converted)
    };
    auto meet = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    u32x4_t pb[TPW][2];   // weights of the tile whose second product is still owed
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) pb[t][h] = u32x4_t{0u, 0u, 0u, 0u};
    // ---- O^T += V^T P^T: a transposing read hands lane (l16, g4) keys 4 * g4 .. + 3 of 16 for d = 16 * dt + l16; two of them are 8 k slots.  Batches of
    // half of d (and half of the keys), each read under the products of the one before.
    auto second = [&](int stage) {
        if constexpr (NT == 0) return;
        s16x4_t vv[2][4][2];
        const int ln = place(lane);
        // key 4 * g4 + l16 / 4 of the 16, its piece 2 * dt + (l16 & 3) / 2 swizzled by twice the key (16 keys further on: by the same)
        const int kr = 4 * (ln >> 4) + ((ln & 15) >> 2);
        const uint32_t at = base + (2 + stage) * kStage + kr * (2 * kD) + ((((ln & 3) >> 1) ^ ((2 * kr) & 15)) * 16) + (ln & 1) * 8;
        auto read_v = [&](int half, int dq, s16x4_t (*v)[2]) {
#pragma unroll
            for (int d4 = 0; d4 < 4; ++d4)
#pragma unroll
                for (int sub = 0; sub < 2; ++sub) {
                    const uint32_t vp = (at ^ (uint32_t)((dq * 4 + d4) * 32)) + (half * 32 + sub * 16) * (2 * kD);
                    v[d4][sub] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4_t>(vp));
                }
        };
        auto mul_v = [&](int half, int dq, s16x4_t (*v)[2]) {
            if (dq == 0) {   // the weights' sum: the same product against ones
                const u32x4_t ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    x.l[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ones), __builtin_bit_cast(bf16x8_t, pb[t][half]), x.l[t], 0, 0, 0);
            }
#pragma unroll
            for (int d4 = 0; d4 < 4; ++d4) {
                const s16x8_t a = {v[d4][0][0], v[d4][0][1], v[d4][0][2], v[d4][0][3], v[d4][1][0], v[d4][1][1], v[d4][1][2], v[d4][1][3]};
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    x.acc[t][dq * 4 + d4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, pb[t][half]),
                                                                                    x.acc[t][dq * 4 + d4], 0, 0, 0);
            }
        };
        read_v(0, 0, vv[0]);
        read_v(0, 1, vv[1]);
        mul_v(0, 0, vv[0]);
        read_v(1, 0, vv[0]);
        mul_v(0, 1, vv[1]);
        read_v(1, 1, vv[1]);
        mul_v(1, 0, vv[0]);
        mul_v(1, 1, vv[1]);
        __builtin_amdgcn_sched_group_barrier(0x100, 16, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 5 * NT, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 4 * NT, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 9 * NT, 0);
    };
    const bool late = wave >= 4;
    {
        Raw r;
        read_raw(0, r);
        convert(0, r);
        if (late) {
            meet();
            if (n_tiles > 1) {
                read_raw(1, r);
                convert(1, r);
            }
        }
    }
    for (int i = 0; i < n_tiles; ++i) {
        if (!late) meet();
        __builtin_amdgcn_s_setprio(2);
        if (i > 0) second((i - 1) % 3);
        // ---- S^T = K Q^T, the next 16 keys' fragments read under the products of those before
        f32x4_t sc[TPW][4];
        if constexpr (NT > 0) {
            const int ln = place(lane);
            // key l16 of 16, pieces of 8 elements 2 * g4, 2 * g4 + 1 and 8 further on, swizzled by the key
            const uint32_t k_at = base + (i & 1) * kStage + (ln & 15) * (2 * kD) + (((2 * (ln >> 4)) ^ (ln & 15)) * 16);
            bf16x8_t kf[2][4];
            auto read_k = [&](int s, bf16x8_t* f) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    f[ks] = __builtin_bit_cast(bf16x8_t, *lds_at<u32x4_t>((k_at ^ (uint32_t)((ks >> 1) * 128 + (ks & 1) * 16)) + s * 16 * (2 * kD)));
            };
            auto mul_k = [&](int s, const bf16x8_t* f) {
#pragma unroll
                for (int t = 0; t < NT; ++t) sc[t][s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        sc[t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[ks], __builtin_bit_cast(bf16x8_t, x.q[t][ks]), sc[t][s], 0, 0, 0);
            };
            read_k(0, kf[0]);
            read_k(1, kf[1]);
            mul_k(0, kf[0]);
            read_k(2, kf[0]);
            mul_k(1, kf[1]);
            read_k(3, kf[1]);
            mul_k(2, kf[0]);
            mul_k(3, kf[1]);
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 4 * NT, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 4 * NT, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 8 * NT, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (late && i + 1 < n_tiles) meet();
        // ---- softmax, with the next tile's codes on their way
        const int next = i + (late ? 2 : 1);
        Raw r;
        if (next < n_tiles) read_raw(next, r);
        if constexpr (NT > 0)
            kv8_weights(x, sc, pb, k0 + i * kKT + kKT > ctx, k0 + i * kKT - ctx,
                            [&](int t, int ln) {
                                const int row = (rg * per_group + wave + 8 * t) * 16 + (ln & 15);
                                return row < R ? mask_lds[row / G] : 0ull;
                            },
                            scale_log2, lazy);
        __builtin_amdgcn_sched_barrier(0);   // (registers again: neither half of the period may reach into the conversion)
        if (next < n_tiles) convert(next, r);
        __builtin_amdgcn_sched_barrier(0);
    }
    second((n_tiles - 1) % 3);
    // ---- lane (l16, g4) holds d = 16 * dt + 4 * g4 + v of row l16
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = (rg * per_group + wave + 8 * t) * 16 + l16;
        if (row >= R) continue;
        const bool sees = ctx > 0 || mask_lds[row / G] != 0;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) to.put4(it, kh, G, row, 16 * dt + 4 * g4, x.acc[t][dt], x.m[t], x.l[t][0], sees);
    }
}

// Workgroup id -> (item, kv head, group of row tiles).  Ids are dealt round-robin over the 8 XCDs, and the groups of one (item, kv head) read the same keys and
// values: they get ids 8 apart, so that they run on one XCD at the same time.
template <int TPW>
__global__ __launch_bounds__(512) void kv8_attn_many_k(KV8Split sp, int64_t q_stride, const uint16_t* __restrict__ q, KV8Rows rows, KV8Layer kv, KV8Out to,
                                                       KV8Seg* __restrict__ seg, int row_tiles, int groups, int per_group, float scale_log2, float lazy) {
    __shared__ __align__(256) uint8_t lds[kManyLds];
    const int id = blockIdx.x, g = id / (8 * groups), within = id - g * 8 * groups, rg = within >> 3, pair = g * 8 + (within & 7);
    const int item = pair / kv.n_kv, kh = pair - item * kv.n_kv;
    KV8Item it;
    if (!kv8_item(kv.seq_len, rows.B, rows.n, kv.seq_len_bound, sp, item, it)) return;   // uniform
    if (kh == 0 && rg == 0 && it.slot == it.first && threadIdx.x == 0) seg[it.b] = KV8Seg{it.first, it.k};
    // row tiles of this wave (a wave runs the program for as many as it has; all pass the same barriers)
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int mine = min(per_group, row_tiles - rg * per_group), n_on = mine > wave ? (mine - wave + 7) / 8 : 0;
#define TLT_BODY(N) kv8_many_body<N>(it, kh, rg, q_stride, q, rows, kv, to, per_group, scale_log2, lazy, lds)
    if (n_on >= TPW) TLT_BODY(TPW);
    else if (TPW >= 2 && n_on == TPW - 1) TLT_BODY((TPW >= 2 ? TPW - 1 : 0));
    else if (TPW >= 3 && n_on == TPW - 2) TLT_BODY((TPW >= 3 ? TPW - 2 : 0));
    else TLT_BODY(0);
#undef TLT_BODY
}

// Up to 8 tiles of rows: workgroups of four waves, two of them on a CU, so that one's softmax runs under the other's products and one's end and the next one's
// start under the other's work.  They stream the item's range for all tiles of rows, dealt round-robin to the waves (NT each).  A tile of 64 keys passes
// through LDS twice: its codes come from memory by direct loads, two tiles ahead, a wave's page (2 KB each of K and V) to a place that only this wave reads;
// the wave converts them to bf16 and stores them for all, K rows swizzled by the key (the 16-byte fragments of 16 keys hit 16 distinct places), V rows by
// twice the key (a transposing read takes two neighbouring places of each of 8 keys; stores of two neighbouring keys meet).  There is one stage of either: V of a tile is converted
// under Q K^T, K of the next one under P V.  16 sequences of 8192 keys, 28 and 4 heads, 16 nodes (7 tiles of rows, 30 GFLOP): 56 us; the matrix pipes are busy 29 % of
// it, the chain of barrier, reads, products and exponentials is what takes the time (two workgroups per CU hide one another's only in part).
constexpr int kMidRaw = 2, kMidLds = 2 * kStage + kMidRaw * kRawBytes + 64 * 8;

template <int NT>
__device__ __forceinline__ void kv8_mid_body(const KV8Item& it, int kh, int64_t q_stride, const uint16_t* __restrict__ q, const KV8Rows& rows, const KV8Layer& kv,
                                              const KV8Out& to, float scale_log2, float lazy, uint8_t* lds) {
    constexpr int TPW = NT > 0 ? NT : 1;
    typedef __attribute__((ext_vector_type(4))) short s16x4_t;
    typedef __attribute__((ext_vector_type(8))) short s16x8_t;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int b = it.b, ctx = it.ctx, n = rows.n, total = ctx + n, n_kv = kv.n_kv, G = to.n_q_heads / n_kv, R = n * G;
    const int n_tiles = it.hi - it.lo, k0 = it.lo * kKT;
    uint8_t* raw = lds + 2 * kStage;   // (the stages first: their places are worked out with exclusive ors below 256)
    uint64_t* mask_lds = (uint64_t*)(raw + kMidRaw * kRawBytes);
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;

    int pages;   // lane t: this wave's page of tile t (a range is 64 tiles at most); -1: none
    {
        const int lp = (it.lo + lane) * 4 + wave;
        pages = lane < n_tiles && lp < kv.max_pages && lp * 16 < total ? kv.block_table[(int64_t)b * kv.max_pages + lp] : -1;
        pages = pages < kv.n_pages ? pages : -1;
    }
    constexpr int kOps = 6;   // loads of a fetch
    auto fetch = [&](int t) {   // (of a page that is not there, page 0 instead: the conversion does not look)
        const int64_t row = ((int64_t)max(__builtin_amdgcn_readlane(pages, t), 0) * n_kv + kh) * 16;
        const uint32_t at = __builtin_amdgcn_readfirstlane(base + 2 * kStage + (t & 1) * kRawBytes);
        dma_16(kv.k + row * kD, lane * 16, at + wave * 2048);
        dma_16(kv.k + row * kD + 1024, lane * 16, at + wave * 2048 + 1024);
        dma_16(kv.v + row * kD, lane * 16, at + kKT * kD + wave * 2048);
        dma_16(kv.v + row * kD + 1024, lane * 16, at + kKT * kD + wave * 2048 + 1024);
        if (lane < 4) dma_4(kv.k_exp + row, lane * 4, at + 2 * kKT * kD + wave * 16);
        if (lane < 4) dma_4(kv.v_exp + row, lane * 4, at + 2 * kKT * kD + kKT + wave * 16);
    };
    fetch(0);
    if (n_tiles > 1) fetch(1);
    if (tid < n) mask_lds[tid] = kv8_mask(rows, b, G, tid * G);
    KV8Tiles<TPW> x;
    if constexpr (NT > 0) kv8_tiles(x, rows, b, kh, G, q, q_stride, [&](int t) { return (wave + 4 * t) * 16; });
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

    // this wave's page of a tile in registers, of K or V: 16 codes of rows lane / 8 and 8 + lane / 8, and the rows' exponents (of K: of V too)
    struct Raw {
        u32x4_t c[2];
        uint32_t e[2], ev[2];
    };
    auto read_raw = [&](int t, bool v, Raw& r) {
        const int ln = lane;
        const uint8_t* p = raw + (t & 1) * kRawBytes;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            r.c[j] = *(const u32x4_t*)(p + (v ? kKT * kD : 0) + wave * 2048 + j * 1024 + ln * 16);
            r.ev[j] = p[2 * kKT * kD + kKT + wave * 16 + 8 * j + (ln >> 3)];
            if (!v) r.e[j] = p[2 * kKT * kD + wave * 16 + 8 * j + (ln >> 3)];
        }
    };
    auto backed = [&](int t) { return __builtin_amdgcn_readlane(pages, t) >= 0; };
    bool top = false;   // some key or value of the page of the tile whose K was written last has the largest exponent, or is not finite
    auto write_k = [&](Raw& r, bool there) {
        const int ln = lane;
        top = __builtin_amdgcn_ballot_w64(max(max(r.e[0], r.e[1]), max(r.ev[0], r.ev[1])) >= kTopExp) != 0;
        for (int rep = there && !top ? 1 : 0; rep < 1; ++rep)   // (a loop, which stays a branch)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                r.c[j] = there ? (r.e[j] >= kTopExp ? finite16(r.c[j]) : r.c[j]) : u32x4_t{0u, 0u, 0u, 0u};
                r.e[j] = there ? r.e[j] : 127u, r.ev[j] = there ? r.ev[j] : 127u;
            }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = 16 * wave + 8 * j + (ln >> 3), p = ln & 7;
            // (values that are not finite: their codes are zero, the NaN comes through the key, whose score only rows that see it keep)
            const float s = __uint_as_float((r.ev[j] == 255u ? 255u : r.e[j]) << 23);
            uint8_t* o = lds + key * (2 * kD);
            *(u32x4_t*)(o + ((2 * p) ^ (key & 15)) * 16) = cvt8(r.c[j][0], r.c[j][1], s);
            *(u32x4_t*)(o + ((2 * p + 1) ^ (key & 15)) * 16) = cvt8(r.c[j][2], r.c[j][3], s);
        }
    };
    auto write_v = [&](Raw& r, int t, bool there) {
        const int ln = lane;
        const int left = there ? total - k0 - t * kKT : 0;   // (slots that nobody has written may hold anything)
        for (int rep = left < kKT || top ? 0 : 1; rep < 1; ++rep)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int y = 0; y < 4; ++y) r.c[j][y] = 16 * wave + 8 * j + (ln >> 3) < left ? r.c[j][y] : 0u;
                r.c[j] = r.ev[j] >= kTopExp ? finite16(r.c[j]) : r.c[j];
            }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = 16 * wave + 8 * j + (ln >> 3), p = ln & 7;
            const float s = __uint_as_float((r.ev[j] == 255u ? 127u : r.ev[j]) << 23);
            uint8_t* o = lds + kStage + key * (2 * kD);
            *(u32x4_t*)(o + ((2 * p) ^ ((2 * key) & 15)) * 16) = cvt8(r.c[j][0], r.c[j][1], s);
            *(u32x4_t*)(o + ((2 * p + 1) ^ ((2 * key) & 15)) * 16) = cvt8(r.c[j][2], r.c[j][3], s);
        }
    };
    auto meet = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    bool there = backed(0);
    {
        Raw r;
        read_raw(0, false, r);
        write_k(r, there);
    }
    for (int i = 0; i < n_tiles; ++i) {
        meet();   // K of tile i stands in its stage, and V's is free
        Raw rv, rk;
        read_raw(i, true, rv);
        f32x4_t sc[TPW][4];
        u32x4_t pb[TPW][2];
        if constexpr (NT > 0) {
            const int ln = lane;
            // key l16 of 16, pieces of 8 elements 2 * g4, 2 * g4 + 1 and 8 further on, swizzled by the key
            const uint32_t k_at = base + (ln & 15) * (2 * kD) + (((2 * (ln >> 4)) ^ (ln & 15)) * 16);
            bf16x8_t kf[2][4];
            auto read_k = [&](int s, bf16x8_t* f) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    f[ks] = __builtin_bit_cast(bf16x8_t, *lds_at<u32x4_t>((k_at ^ (uint32_t)((ks >> 1) * 128 + (ks & 1) * 16)) + s * 16 * (2 * kD)));
            };
            auto mul_k = [&](int s, const bf16x8_t* f) {
#pragma unroll
                for (int t = 0; t < NT; ++t) sc[t][s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        sc[t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[ks], __builtin_bit_cast(bf16x8_t, x.q[t][ks]), sc[t][s], 0, 0, 0);
            };
            read_k(0, kf[0]);
            read_k(1, kf[1]);
            mul_k(0, kf[0]);
            read_k(2, kf[0]);
            mul_k(1, kf[1]);
            read_k(3, kf[1]);
            mul_k(2, kf[0]);
            mul_k(3, kf[1]);
        }
        write_v(rv, i, there);
        meet();   // V of tile i stands, and K's stage is free; this wave has read tile i's codes
        if (i + 2 < n_tiles) fetch(i + 2);
        const bool more = i + 1 < n_tiles;
        if (more) {
            if (i + 2 < n_tiles) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kOps) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            there = backed(i + 1);
            read_raw(i + 1, false, rk);
        }
        if constexpr (NT > 0)
            kv8_weights(x, sc, pb, k0 + i * kKT + kKT > ctx, k0 + i * kKT - ctx,
                            [&](int t, int ln) {
                                const int row = (wave + 4 * t) * 16 + (ln & 15);
                                return row < R ? mask_lds[row / G] : 0ull;
                            },
                            scale_log2, lazy);
        if (more) write_k(rk, there);
        if constexpr (NT > 0) {
            // O^T += V^T P^T: a transposing read hands lane (l16, g4) keys 4 * g4 .. + 3 of 16 for d = 16 * dt + l16; two of them are 8 k slots
            s16x4_t vv[2][4][2];
            const int ln = lane;
            // key 4 * g4 + l16 / 4 of the 16, its piece 2 * dt + (l16 & 3) / 2 swizzled by twice the key (16 keys further on: by the same)
            const int kr = 4 * (ln >> 4) + ((ln & 15) >> 2);
            const uint32_t at = base + kStage + kr * (2 * kD) + ((((ln & 3) >> 1) ^ ((2 * kr) & 15)) * 16) + (ln & 1) * 8;
            auto read_v = [&](int half, int dq, s16x4_t (*v)[2]) {
#pragma unroll
                for (int d4 = 0; d4 < 4; ++d4)
#pragma unroll
                    for (int sub = 0; sub < 2; ++sub) {
                        const uint32_t vp = (at ^ (uint32_t)((dq * 4 + d4) * 32)) + (half * 32 + sub * 16) * (2 * kD);
                        v[d4][sub] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s16x4_t>(vp));
                    }
            };
            auto mul_v = [&](int half, int dq, s16x4_t (*v)[2]) {
                if (dq == 0) {   // the weights' sum: the same product against ones
                    const u32x4_t ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        x.l[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ones), __builtin_bit_cast(bf16x8_t, pb[t][half]), x.l[t], 0, 0, 0);
                }
#pragma unroll
                for (int d4 = 0; d4 < 4; ++d4) {
                    const s16x8_t a = {v[d4][0][0], v[d4][0][1], v[d4][0][2], v[d4][0][3], v[d4][1][0], v[d4][1][1], v[d4][1][2], v[d4][1][3]};
#pragma unroll
                    for (int t = 0; t < NT; ++t)
                        x.acc[t][dq * 4 + d4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, pb[t][half]),
                                                                                        x.acc[t][dq * 4 + d4], 0, 0, 0);
                }
            };
            read_v(0, 0, vv[0]);
            read_v(0, 1, vv[1]);
            mul_v(0, 0, vv[0]);
            read_v(1, 0, vv[0]);
            mul_v(0, 1, vv[1]);
            read_v(1, 1, vv[1]);
            mul_v(1, 0, vv[0]);
            mul_v(1, 1, vv[1]);
        }
    }
    // ---- lane (l16, g4) holds d = 16 * dt + 4 * g4 + v of row l16
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = (wave + 4 * t) * 16 + l16;
        if (row >= R) continue;
        const bool sees = ctx > 0 || mask_lds[row / G] != 0;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) to.put4(it, kh, G, row, 16 * dt + 4 * g4, x.acc[t][dt], x.m[t], x.l[t][0], sees);
    }
}

template <int TPW>
__global__ __launch_bounds__(256, 2) void kv8_attn_mid_k(KV8Split sp, int64_t q_stride, const uint16_t* __restrict__ q, KV8Rows rows, KV8Layer kv, KV8Out to,
                                                         KV8Seg* __restrict__ seg, int row_tiles, float scale_log2, float lazy) {
    __shared__ __align__(256) uint8_t lds[kMidLds];
    const int item = blockIdx.x / kv.n_kv, kh = blockIdx.x - item * kv.n_kv;
    KV8Item it;
    if (!kv8_item(kv.seq_len, rows.B, rows.n, kv.seq_len_bound, sp, item, it)) return;   // uniform
    if (kh == 0 && it.slot == it.first && threadIdx.x == 0) seg[it.b] = KV8Seg{it.first, it.k};
    // (a wave runs the program for as many row tiles as it has; all pass the same barriers)
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n_on = row_tiles > wave ? (row_tiles - wave + 3) / 4 : 0;
    if (n_on >= TPW) kv8_mid_body<TPW>(it, kh, q_stride, q, rows, kv, to, scale_log2, lazy, lds);
    else if (n_on == TPW - 1) kv8_mid_body<TPW - 1>(it, kh, q_stride, q, rows, kv, to, scale_log2, lazy, lds);
    else kv8_mid_body<0>(it, kh, q_stride, q, rows, kv, to, scale_log2, lazy, lds);
}

// The ranges of a sequence joined, in a fixed order.  Few rows: four waves per row, 16 ranges of each requested together; the lanes read a range's maximum and sum
// each.  Bound by latency.
__global__ __launch_bounds__(256) void kv8_join_few_k(const KV8Seg* __restrict__ seg, const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                      uint16_t* __restrict__ out, int n, int n_q_heads, int n_kv, int r_pad, int slot_step, float scale_log2) {
    constexpr int U = 16, W = 4;
    __shared__ float2 s_a[W - 1][64];
    __shared__ float s_l[W];
    const int part = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = blockIdx.x, kh = blockIdx.y, b = blockIdx.z;
    const int G = n_q_heads / n_kv;
    const KV8Seg sg = seg[b];
    if (sg.k <= 1) return;   // (one range: its workgroup has written the row; uniform)
    const int64_t base = ((int64_t)sg.first * n_kv + kh) * r_pad + r, step = (int64_t)slot_step * n_kv * r_pad;
    float2 ml = make_float2(kNegBig, 0.f), v[U];
    auto fetch = [&](int c) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            v[u] = c + u < sg.k ? *(const float2*)(part_o + (base + (c + u) * step) * kD + lane * 2) : make_float2(0.f, 0.f);
    };
    if (lane < sg.k) ml = *(const float2*)(part_ml + (base + lane * step) * 2);
    fetch(U * part);
    float M = ml.x;
    for (int c = lane + 64; c < sg.k; c += 64) M = fmaxf(M, part_ml[(base + c * step) * 2]);
    M = wave_max(M);
    float w = exp2f((ml.x - M) * scale_log2), wl = ml.y * w, a0 = 0.f, a1 = 0.f, L = 0.f;
    for (int c0 = U * part; c0 < sg.k; c0 += U * W) {   // (a round is 64 ranges; uniform for the wave)
        if (c0 > U * part) {
            fetch(c0);
            const int c = (c0 & ~63) + lane;
            ml = c < sg.k ? *(const float2*)(part_ml + (base + c * step) * 2) : make_float2(kNegBig, 0.f);
            w = exp2f((ml.x - M) * scale_log2), wl = ml.y * w;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u >= sg.k) break;
            const float wu = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), (c0 + u) & 63));
            L += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wl), (c0 + u) & 63));
            a0 = fmaf(wu, v[u].x, a0), a1 = fmaf(wu, v[u].y, a1);
        }
    }
    if (part > 0) s_a[part - 1][lane] = make_float2(a0, a1);
    if (lane == 0) s_l[part] = L;
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int p = 1; p < W; ++p) a0 += s_a[p - 1][lane].x, a1 += s_a[p - 1][lane].y, L += s_l[p];
    const float inv = 1.0f / L;
    const int i = r / G, g = r - i * G;
    ((uint32_t*)(out + ((int64_t)(b * n + i) * n_q_heads + kh * G + g) * kD))[lane] = pack_bf16x2(a0 * inv, a1 * inv);
}
// Many rows: half a wave per row, four columns a lane.  Bound by the partial results that it reads: 32 sequences with 336 rows per kv head, 40 MB in 9.5 us (a wave
// per row 12.8).
__global__ __launch_bounds__(256) void kv8_join_many_k(const KV8Seg* __restrict__ seg, const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                       uint16_t* __restrict__ out, int n, int n_q_heads, int n_kv, int r_pad, int slot_step, float scale_log2) {
    constexpr int U = 8;
    const int lane = threadIdx.x & 31, r = blockIdx.x * 8 + (threadIdx.x >> 5), kh = blockIdx.y, b = blockIdx.z, G = n_q_heads / n_kv;
    const KV8Seg sg = seg[b];
    if (r >= n * G || sg.k <= 1) return;   // (halves of a wave leave as wholes)
    const int64_t base = ((int64_t)sg.first * n_kv + kh) * r_pad + r, step = (int64_t)slot_step * n_kv * r_pad;
    f32x4_t v[U], a = {0.f, 0.f, 0.f, 0.f};
    float2 ml;
    float L = 0.f;
    auto fetch = [&](int c0) {
        const int c = c0 + (lane & (U - 1));
        ml = c < sg.k ? *(const float2*)(part_ml + (base + c * step) * 2) : make_float2(kNegBig, 0.f);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c0 + u < sg.k) v[u] = *(const f32x4_t*)(part_o + (base + (c0 + u) * step) * kD + lane * 4);
    };
    fetch(0);
    float M = ml.x;
    for (int c = U + lane; c < sg.k; c += 32) M = fmaxf(M, part_ml[(base + c * step) * 2]);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) M = fmaxf(M, __shfl_xor(M, o, 32));
    for (int c0 = 0; c0 < sg.k; c0 += U) {
        if (c0 > 0) fetch(c0);
        const float w = exp2f((ml.x - M) * scale_log2), wl = ml.y * w;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u >= sg.k) break;
            L += __shfl(wl, u, 32);
            a += __shfl(w, u, 32) * v[u];
        }
    }
    const float inv = 1.0f / L;
    const int i = r / G, g = r - i * G;
    *(u32x2_t*)(out + ((int64_t)(b * n + i) * n_q_heads + kh * G + g) * kD + lane * 4) = u32x2_t{pack_bf16x2(a[0] * inv, a[1] * inv), pack_bf16x2(a[2] * inv, a[3] * inv)};
}

struct KV8Plan {
    KV8Split sp;
    bool few, mid;   // the kernels of few rows and of up to 8 tiles of rows
    bool one_each;   // no sequence has a second range
    bool runs;       // the launch fits a grid
    int row_tiles, groups, per_group;
    size_t seg, part_o, part_ml, total;   // byte offsets into the workspace
};
static KV8Plan plan_kv8(int B, int n, int n_q_heads, int n_kv, int bound_total) {
    KV8Plan p;
    const int R = n * (n_q_heads / n_kv), tiles = (bound_total + kKT - 1) / kKT;
    p.row_tiles = (R + 15) / 16;
    // Which kernel, 28 and 4 heads unless said otherwise.  Two tiles of rows: few / mid 38.4 / 42.0 us for 16 sequences of 8192 with 4 nodes, 39.4 / 49.1 for 32 of ~4096
    // (32 and 8 heads, 16 of 8192: 58.3 / 56.1); a third tile has no registers there.  Mid / many: 4 tiles of rows, 256 of ~4000, 363 / 466; 5 tiles (40 and
    // 8 heads), 256 of ~4000, 763 / 897; 7 tiles, 16 of 8192, 62.0 / 61.8; 21 tiles, 32 of ~4096, 141 (three a wave, in two groups) / 122.
    p.few = p.row_tiles <= 2;
    p.mid = !p.few && p.row_tiles <= 8;
    p.groups = p.few ? 1 : (p.row_tiles + 23) / 24;
    p.per_group = (p.row_tiles + p.groups - 1) / p.groups;
    p.sp.slots = std::max(1, (p.few || p.mid ? 512 : 256) / (n_kv * p.groups));   // (workgroups that the chip holds)
    p.sp.t_max = 64;   // (as many as a wave has lanes for their pages; 24, 32, 48: 64 sequences of ~8192, 40 and 8 heads, 260, 240, 223 us against 217)
    p.sp.whole = p.few ? 8 : 4;
    // Planning costs every workgroup some 2 us (7 at 256 sequences) and is worth it where sequences are cut to fill the chip or whole rounds of it: long ones while the
    // rounds are few, short ones while there are fewer sequences than places.  Planned / ranges of t_max: 28 and 4 heads, ~4000 keys: 96 with 8 nodes (128 places) 139 / 180 us, 192
    // 274 / 302, 128 with 24 nodes (64 places) 344 / 388; 256 with 16 nodes and 8 kv heads (64) 760 / 771, (32) 964 / 899.  Short ones, eight shapes (32 to 128 places) with
    // lengths of ~400 and ~2000 that differ and of 1000 that do not, unplanned over planned by the share of places taken: 5/8 1.20 and 0.89 (differing, equal), 6/8 1.22 and 0.88, 7/8
    // 1.10 and 0.87, 15/16 1.01 and 0.87; in the second round 0 0.91 and 0.88, 1/8 1.05 and 0.88, 1/4 1.02 and 0.88, 1/2 1.02 and 0.87, 3/4 0.99 and 0.87; in the third 0.90 to 0.97 and 0.87.
    p.sp.planned = B <= kPlanned && (tiles > p.sp.t_max ? B <= 4 * p.sp.slots : B < p.sp.slots);
    p.one_each = tiles <= (p.sp.planned ? p.sp.whole : p.sp.t_max);
    // (planned: items that fit `slots`, or those of ranges of t_max rounded up to whole rounds)
    const int64_t longest = (int64_t)B * ((tiles + p.sp.t_max - 1) / p.sp.t_max);
    const int64_t rounds = (std::min(longest, (int64_t)B * tiles / p.sp.t_max + B) + p.sp.slots - 1) / p.sp.slots;
    p.sp.max_items = (int)(p.one_each ? B : (p.sp.planned ? rounds * p.sp.slots : longest));
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    p.runs = (rounds * p.sp.slots + longest) * n_kv * p.groups < (1 << 23);   // (a grid holds fewer than 2^32 threads, the kernel of many rows 512 in a workgroup)
    const size_t rows = (size_t)p.sp.max_items * n_kv * p.row_tiles * 16;
    p.seg = 0;
    p.part_ml = up((size_t)B * sizeof(KV8Seg));
    p.part_o = p.part_ml + up(rows * 8);
    p.total = p.part_o + up(rows * kD * 4);
    return p;
}

size_t kv8_attention_workspace_bytes(int B, int n, int n_q_heads, int n_kv_heads, int d, int max_ctx) {
    size_t need = 256;
    if (d == kD)
        for (int m = 1; m <= n; ++m) {   // (any number of rows up to n may be asked for later)
            const KV8Plan p = plan_kv8(B, m, n_q_heads, n_kv_heads, max_ctx);
            if (!p.runs) return 0;
            need = std::max(need, p.total);
        }
    return need;
}

hipError_t kv8_attention(hipStream_t s, int dtype, const KV8Rows& rows, const KV8Layer& kv, const void* q, int64_t q_stride, void* out, int n_q_heads, void* ws,
                         size_t ws_bytes, int impl) {
    const int R = rows.n * (n_q_heads / kv.n_kv);
    const bool fits = dtype == BF16 && kv.d == kD && kv.page_size == 16 && (((uintptr_t)kv.k_exp | (uintptr_t)kv.v_exp) & 3) == 0;
    if (fits && impl != 0) {
        const KV8Plan p = plan_kv8(rows.B, rows.n, n_q_heads, kv.n_kv, kv.seq_len_bound + rows.n);
        if (!p.runs || p.total > ws_bytes) return hipErrorInvalidValue;
        KV8Seg* seg = (KV8Seg*)((char*)ws + p.seg);
        const KV8Out to{(uint16_t*)out, (float*)((char*)ws + p.part_o), (float*)((char*)ws + p.part_ml), rows.n, n_q_heads, kv.n_kv, p.row_tiles * 16};
        const float scale_log2 = 1.4426950408889634f / sqrtf((float)kD), lazy = 8.0f / scale_log2;
        const unsigned pairs = (unsigned)(p.sp.max_items * kv.n_kv);
        auto few = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(pairs), dim3(256), 0, s, p.sp, q_stride, (const uint16_t*)q, rows, kv, to, seg, scale_log2, lazy); };
        auto mid = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(pairs), dim3(256), 0, s, p.sp, q_stride, (const uint16_t*)q, rows, kv, to, seg, p.row_tiles, scale_log2, lazy); };
        auto many = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((pairs + 7) / 8 * 8 * p.groups), dim3(512), 0, s, p.sp, q_stride, (const uint16_t*)q, rows, kv, to, seg, p.row_tiles, p.groups,
                               p.per_group, scale_log2, lazy);
        };
        if (p.row_tiles == 1) few(kv8_attn_few_k<1>);
        else if (p.few) few(kv8_attn_few_k<2>);
        else if (p.row_tiles <= 4) mid(kv8_attn_mid_k<1>);
        else if (p.mid) mid(kv8_attn_mid_k<2>);
        else if (p.per_group <= 16) many(kv8_attn_many_k<2>);
        else many(kv8_attn_many_k<3>);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.one_each) return e;
        auto join = [&](auto kernel, int blocks) {
            hipLaunchKernelGGL(kernel, dim3(blocks, kv.n_kv, rows.B), dim3(256), 0, s, seg, to.part_o, to.part_ml, (uint16_t*)out, rows.n, n_q_heads, kv.n_kv,
                               p.row_tiles * 16, p.sp.planned ? 1 : rows.B, scale_log2);
        };
        // the most ranges that a sequence can have
        const int tiles = (kv.seq_len_bound + rows.n + kKT - 1) / kKT, shortest = shortest_range(tiles, p.sp.whole);
        const int ranges = std::max(std::min(p.sp.slots, (tiles + shortest - 1) / shortest), (tiles + p.sp.t_max - 1) / p.sp.t_max);
        // Four waves per row / half a one, 28 and 4 heads, us with the kernel in front: one sequence, one token, of 2048 8.6 / 10.3, of 8192 9.7 / 13.0, of 30000 12.9 / 19.7;
        // 8 nodes at 30000 22.1 / 29.4; 4 sequences of 8192, 8 nodes, 25.7 / 27.6; 64 nodes 54.1 / 51.0; 64 of 2048, one token (few ranges each), 32.8 / 31.5
        if (ranges > 16 && (int64_t)R * kv.n_kv * rows.B <= 2048) join(kv8_join_few_k, R);
        else join(kv8_join_many_k, (R + 7) / 8);
        return hipGetLastError();
    }
    const float scale = 1.0f / sqrtf((float)kv.d);
    const dim3 grid(rows.n, n_q_heads, rows.B), block(64 * kRowWaves);
    if (dtype == F32)
        hipLaunchKernelGGL(kv8_attn_row_k<float>, grid, block, 0, s, rows, kv, (const float*)q, q_stride, (float*)out, n_q_heads, scale);
    else
        hipLaunchKernelGGL(kv8_attn_row_k<bf16>, grid, block, 0, s, rows, kv, (const bf16*)q, q_stride, (bf16*)out, n_q_heads, scale);
    return hipGetLastError();
}

}  // namespace tlt
