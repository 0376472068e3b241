// The 8-bit paged KV cache: writing rows, attention over them, keeping the accepted path, reading rows back.
//
// A row (one token of one kv head, d elements) is d codes in e4m3 (OCP: 4 exponent bits, bias 7, largest value 448, no infinities) and one
// exponent byte E; its values are code * 2^(E - 127).  E - 127 is the smallest e >= -126 with max|x| <= 448 * 2^e, so scaling by it is exact, the one
// rounding is that to e4m3, nothing saturates, and a value has four significant bits: it is exact in bf16 too.  A row with an element that is not
// finite keeps E = 255 and codes of zero, and all of it reads as NaN.
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

// row number of a slot in the pools' rows of kv head 0 (kv head kh: + kh * page_size), -1: the block table does not back it
__device__ __forceinline__ int64_t row_of(const KV8Layer& kv, int b, int slot) {
    PageRef pr;
    if (!locate(kv.block_table, kv.max_pages, kv.n_pages, kv.page_size, b, slot, pr)) return -1;
    return pr.page * kv.n_kv * kv.page_size + pr.row;
}

// ---- write
// One workgroup per row (b, i).  A head (of q, k or v) belongs to a group of `lanes` lanes (a power of two); a lane holds VEC pairs (j, j + d/2) of it, one
// 16-byte piece of either half.  The largest magnitude of a k or v head is taken over its group.  Angles are formed in double (positions reach
// 32K, where an fp32 product position * frequency is 1e-3 rad off), once per row, and shared by the heads.
template <typename T>
__global__ __launch_bounds__(512) void kv8_write_k(const T* __restrict__ qkv, const T* __restrict__ bias, T* __restrict__ q_out, int64_t q_stride,
                                                   const int32_t* __restrict__ depth, int n, int n_q_heads, int lanes, double log2_theta, KV8Layer kv) {
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float cs[128], sn[128];
    const int r = blockIdx.x, b = r / n, i = r - b * n, d = kv.d, half = d >> 1, n_kv = kv.n_kv;
    const int heads = n_q_heads + 2 * n_kv;
    const T* row = qkv + (int64_t)r * heads * d;
    const int ctx = max(kv.seq_len[b], 0);
    if ((int)threadIdx.x < half) {
        const int pos = ctx + (depth ? depth[r] : i);
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
// One wave per (layer, sequence, 16 rows, kv head): a row's d / 16 pieces of 16 codes go to d / 16 lanes.
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
// of an earlier j (path[j] >= j), which the same thread has read by then.
constexpr int kCommitThreads = 256;
__global__ __launch_bounds__(kCommitThreads) void kv8_commit_k(int n_layers, KV8Layer kv, const int32_t* __restrict__ accept_len,
                                                               const int32_t* __restrict__ path_idx, int stride) {
    __shared__ int64_t s_src[64], s_dst[64];
    const int b = blockIdx.y, tid = threadIdx.x;
    const int a = min(accept_len[b], min(stride - 1, 63));
    if (a <= 0) return;
    if (tid < 64) {
        int64_t src = -1, dst = -1;
        if (tid >= 1 && tid <= a) {
            const int ctx = kv.seq_len[b], p = path_idx[(int64_t)b * stride + tid];
            if (p > tid && p < 64 && ctx >= 0) src = row_of(kv, b, ctx + p), dst = row_of(kv, b, ctx + tid);
        }
        s_src[tid] = dst < 0 ? -1 : src, s_dst[tid] = dst;
    }
    __syncthreads();
    const int cols = kv.d / 16, per_head = 2 * cols + 2;
    const int64_t rows_per_layer = kv.n_pages * kv.n_kv * kv.page_size;
    const int u = blockIdx.x * kCommitThreads + tid;
    if (u >= n_layers * kv.n_kv * per_head) return;
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

__global__ void kv8_advance_k(int B, int32_t* __restrict__ seq_len, const int32_t* __restrict__ accept_len, int stride) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B) seq_len[b] += max(min(accept_len[b], min(stride - 1, 63)), 0) + 1;
}

hipError_t kv8_commit(hipStream_t s, int n_layers, int B, const KV8Layer& kv, int32_t* seq_len, const int32_t* accept_len, const int32_t* path_idx, int stride) {
    const int64_t units = (int64_t)n_layers * kv.n_kv * (2 * (kv.d / 16) + 2);
    hipLaunchKernelGGL(kv8_commit_k, dim3((unsigned)((units + kCommitThreads - 1) / kCommitThreads), B), dim3(kCommitThreads), 0, s, n_layers, kv, accept_len, path_idx, stride);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kv8_advance_k, dim3((B + 63) / 64), dim3(64), 0, s, B, seq_len, accept_len, stride);
    return hipGetLastError();
}

// ---- attention, a workgroup per (row, query head): any dtype and shape
// Four waves, each taking every fourth tile of 64 keys: lanes own keys for the scores and 16-code pieces of value rows for the sums; the running maximum
// and sum of a wave's tiles, the waves merged at the end.
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
    const int ctx = max(kv.seq_len[b], 0), total = ctx + rows.n;
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
            for (int c0 = 0; c0 < d; c0 += 64) {
                u32x4_t w[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) w[c] = *(const u32x4_t*)(kv.k + at * d + c0 + 16 * c);
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    float f[4];
                    decode4(w[c >> 2][c & 3], 1.f, f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s = fmaf(q_s[c0 + 4 * c + e], f[e], s);
                }
            }
            s *= scale_of(kv.k_exp[at]);
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
                const float w = p_s[wave][k] * scale_of(kv.v_exp[kat]);
                const u32x4_t v = *(const u32x4_t*)(kv.v + kat * d + piece);
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
    out[((int64_t)r * n_q_heads + hq) * d + tid] = from_float<T>(ll == 0.f ? 0.f : a / ll);
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
constexpr int kPlanned = 256;   // sequences whose ranges are balanced

__device__ __forceinline__ int wave_sum_i(int v) {
    const auto a = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    v = (int)(a[0] + a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = (int)(b[0] + b[1]);
    v += __builtin_amdgcn_update_dpp(0, v, 0x128, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x124, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false);
    return v;
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
    int t_min, t_max;  // shortest and longest range, in tiles
    int max_items;     // upper bound of the item count, from the host's bound on the lengths
};

// Item number `item`: false where there is none.  Up to kPlanned sequences: of the range lengths t_min .. t_max the smallest whose items fit the
// fewest rounds of `slots` that t_max allows; items are numbered sequence by sequence.  Beyond: ranges of t_max, item = range * B + sequence.
__device__ __forceinline__ bool kv8_item(const int32_t* __restrict__ seq_len, int B, int n, int len_bound, const KV8Split& sp, int item, KV8Item& out) {
    const int lane = threadIdx.x & 63;
    auto len_of = [&](int b) { return min(max(seq_len[b], 0), len_bound); };
    auto ceil_div = [](int x, int T) { return (int)__umulhi((uint32_t)(x + T - 1), 0xffffffffu / (uint32_t)T + 1u); };   // (exact: x < 2^26, 2 <= T <= 64)
    auto cut = [&](int tiles, int k, int c) { return (int)((int64_t)tiles * c / k); };
    if (B > kPlanned) {
        const int b = item % B, c = item / B, len = len_of(b), tiles = (len + n + kKT - 1) / kKT, k = (tiles + sp.t_max - 1) / sp.t_max;
        if (c >= k) return false;
        out = KV8Item{b, len, cut(tiles, k, c), cut(tiles, k, c + 1), item, b, k};
        return true;
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
    const int most = (items(sp.t_max) + sp.slots - 1) / sp.slots * sp.slots;
    int T = sp.t_min, up = sp.t_max;
    while (T < up) {   // (longer ranges never make more items)
        const int mid = (T + up) >> 1;
        if (items(mid) <= most) up = mid; else T = mid + 1;
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
            const int first = base + __builtin_amdgcn_readlane(end, l) - kk, c = item - first;
            out = KV8Item{64 * j + l, __builtin_amdgcn_readlane(len[j], l), cut(tt, kk, c), cut(tt, kk, c + 1), item, first, kk};
            return true;
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

// Few rows (NT tiles of 16): bound by memory.  A wave owns every fourth tile of the item's range with all rows, takes codes from memory straight into
// the registers that the products want (no LDS, no barrier until the end) and keeps the next tile's in flight: keys once the scores are done,
// values once the sums are.  d is permuted alike on both sides of the first product (a key's row in two pieces of 16 bytes per lane); for the second one a lane
// loads 8 bytes of each of its 8 keys, so that d = 8 * (lane % 16) + instruction, converts pairs of d, and pairs up keys by byte permutations.
// The four waves are joined through LDS.
template <int NT>
__global__ __launch_bounds__(256) void kv8_attn_few_k(KV8Split sp, int n_q_heads, int64_t q_stride, const uint16_t* __restrict__ q, KV8Rows rows, KV8Layer kv,
                                                      uint16_t* __restrict__ out, KV8Seg* __restrict__ seg, float* __restrict__ part_o,
                                                      float* __restrict__ part_ml, float scale_log2) {
    constexpr int kPad = kD + 4;
    __shared__ __align__(16) float o_s[4][16][kPad];
    __shared__ float m_s[4][16 * NT], l_s[4][16 * NT];
    const int n_kv = kv.n_kv, kh = blockIdx.x % n_kv;
    KV8Item it;
    if (!kv8_item(kv.seq_len, rows.B, rows.n, kv.seq_len_bound, sp, blockIdx.x / n_kv, it)) return;   // uniform
    const int b = it.b, ctx = it.ctx, n = rows.n, total = ctx + n;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int G = n_q_heads / n_kv, R = n * G;
    if (kh == 0 && it.slot == it.first && tid == 0) seg[b] = KV8Seg{it.first, it.k};
    // pages of this wave's tiles (at most 16 of them: ranges are 64 tiles at most), lane 4 * i + s: page s of its i-th tile; -1: none
    const int my_tiles = (it.hi - it.lo - wave + 3) >> 2;   // (0 or less: none)
    int pages;
    {
        const int lp = (it.lo + wave + 4 * (lane >> 2)) * 4 + (lane & 3);
        pages = lp < kv.max_pages && lp * 16 < total && (lane >> 2) < my_tiles ? kv.block_table[(int64_t)b * kv.max_pages + lp] : -1;
        pages = pages < kv.n_pages ? pages : -1;
    }
    // codes and exponents of tile i; a page that is not there reads as zeros
    u32x4_t kc[4][2];
    u32x2_t vc[4][4];
    uint32_t ke[4], kve[4], ve[4];   // (kve: the exponents of the values of the lane's key)
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
            for (int h = 0; h < 2; ++h) kc[s][h] = __builtin_amdgcn_raw_buffer_load_b128(r, l16 * kD + 64 * h + 16 * g4, 0, 2);   // (2: read once)
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
            for (int v = 0; v < 4; ++v) vc[s][v] = __builtin_amdgcn_raw_buffer_load_b64(r, (4 * g4 + v) * kD + 8 * l16, 0, 2);
        }
    };
    if (my_tiles > 0) load_k(0), load_v(0);
    // queries of this lane's row, in the order of the keys' pieces; visibility of the new rows
    u32x4_t qf[NT][4];
    uint64_t mask[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = 16 * t + l16, i = r / G, g = r - i * G;
        const bool on = r < R;
        const uint16_t* p = q + (int64_t)(b * n + (on ? i : 0)) * q_stride + (kh * G + (on ? g : 0)) * kD + 16 * g4;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const u32x4_t z = {0u, 0u, 0u, 0u};
            qf[t][ks] = on ? *(const u32x4_t*)(p + (ks >> 1) * 64 + (ks & 1) * 8) : z;
        }
        mask[t] = !on ? 0ull : (rows.mask ? rows.mask[b * n + i] : (2ull << i) - 1ull) & (~0ull >> (64 - n));
    }
    f32x4_t acc[NT][8], acc_l[NT];
    float m_run[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m_run[t] = kNegBig;
        acc_l[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const float lazy = 8.0f / scale_log2;
    for (int i = 0; i < my_tiles; ++i) {
        const int t0 = (it.lo + wave + 4 * i) * kKT;
        const bool edge = t0 + kKT > ctx;   // new rows, or keys behind the last
        // ---- S^T = K Q^T
        f32x4_t sc[NT][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            // (values that are not finite: their codes are zero, the NaN comes through the score, which only rows that see the key keep)
            const float scale = __uint_as_float((kve[s] == 255u ? 255u : ke[s]) << 23);
            bf16x8_t kf[4];
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) kf[ks] = __builtin_bit_cast(bf16x8_t, cvt8(kc[s][ks >> 1][2 * (ks & 1)], kc[s][ks >> 1][2 * (ks & 1) + 1], scale));
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                sc[t][s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    sc[t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks], __builtin_bit_cast(bf16x8_t, qf[t][ks]), sc[t][s], 0, 0, 0);
            }
        }
        if (i + 1 < my_tiles) load_k(i + 1);
        // ---- running maximum and weights
        u32x4_t pb[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (edge) {
                const uint64_t seen = seen_from(t0 + 4 * g4 - ctx, mask[t]);
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
            if (__builtin_amdgcn_ballot_w64(tmax > m_run[t] + lazy) != 0) {
                const float m_new = fmaxf(m_run[t], group_max4(tmax));
                const float alpha = __builtin_amdgcn_exp2f((m_run[t] - m_new) * scale_log2);
                m_run[t] = m_new;
                acc_l[t] *= alpha;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) acc[t][dt] *= alpha;
            }
            const float mc = fmaxf(m_run[t], -1e29f) * scale_log2;   // (rows that have seen nothing yet: exp2(-1e30 * c + 1e29 * c) = 0)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                float e[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) e[v] = __builtin_amdgcn_exp2f(fmaf(sc[t][s][v], scale_log2, -mc));
                pb[t][s >> 1][2 * (s & 1)] = pack_bf16x2(e[0], e[1]);       // weights are rounded to bf16 for the second product, their sum is that of the rounded ones
                pb[t][s >> 1][2 * (s & 1) + 1] = pack_bf16x2(e[2], e[3]);
            }
        }
        // ---- O^T += V^T P^T: k slot 4 * sub + v of lane group g4 is key 16 * (2 * half + sub) + 4 * g4 + v
        const int left = total - t0;   // (keys from there on are weighted with zero; slots that nobody has written may hold anything)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t vv[8][4];
#pragma unroll
            for (int a = 0; a < 8; ++a) {
                const int s = 2 * half + (a >> 2), v = a & 3;
                uint32_t e8 = (ve[s] >> (8 * v)) & 255u;
                e8 = e8 == 255u ? 127u : e8;
                const float scale = __uint_as_float(e8 << 23);
                u32x4_t x = cvt8(vc[s][v][0], vc[s][v][1], scale);
                if (edge) {
                    const bool in = 16 * s + 4 * g4 + v < left;
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[c] = in ? x[c] : 0u;
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) vv[a][c] = x[c];
            }
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                u32x4_t a;
#pragma unroll
                for (int p = 0; p < 4; ++p)
                    a[p] = __builtin_amdgcn_perm(vv[2 * p + 1][dt >> 1], vv[2 * p][dt >> 1], dt & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    acc[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, pb[t][half]), acc[t][dt], 0, 0, 0);
            }
            const u32x4_t ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
            for (int t = 0; t < NT; ++t)
                acc_l[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ones), __builtin_bit_cast(bf16x8_t, pb[t][half]), acc_l[t], 0, 0, 0);
        }
        if (i + 1 < my_tiles) load_v(i + 1);
    }
    // ---- the four waves joined, a tile of rows at a time: lane (l16, g4) holds d = 32 * g4 + 8 * v + dt of row l16
    const int64_t pbase = ((int64_t)it.slot * n_kv + kh) * (16 * NT);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t > 0) __syncthreads();
        if (16 * t >= R) break;   // uniform
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            *(f32x4_t*)&o_s[wave][l16][32 * g4 + 8 * v] = f32x4_t{acc[t][0][v], acc[t][1][v], acc[t][2][v], acc[t][3][v]};
            *(f32x4_t*)&o_s[wave][l16][32 * g4 + 8 * v + 4] = f32x4_t{acc[t][4][v], acc[t][5][v], acc[t][6][v], acc[t][7][v]};
        }
        if (g4 == 0) m_s[wave][16 * t + l16] = m_run[t], l_s[wave][16 * t + l16] = acc_l[t][0];
        __syncthreads();
        const int rl = tid >> 4, r = 16 * t + rl, c = (tid & 15) * 8;
        if (r >= R) continue;
        float M = kNegBig, L = 0.f, w[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) M = fmaxf(M, m_s[x][r]);
#pragma unroll
        for (int x = 0; x < 4; ++x) w[x] = __builtin_amdgcn_exp2f((m_s[x][r] - M) * scale_log2), L += w[x] * l_s[x][r];
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(w[x], o_s[x][rl][c + e], o[e]);
        if (it.k == 1) {
            const float inv = L == 0.f ? 0.f : 1.0f / L;
            const int i = r / G, g = r - i * G;
            *(u32x4_t*)(out + ((int64_t)(b * n + i) * n_q_heads + kh * G + g) * kD + c) =
                u32x4_t{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv), pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv)};
        } else {
            float* po = part_o + (pbase + r) * kD + c;
            *(f32x4_t*)po = f32x4_t{o[0], o[1], o[2], o[3]};
            *(f32x4_t*)(po + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
            if (c == 0) part_ml[(pbase + r) * 2] = M, part_ml[(pbase + r) * 2 + 1] = L;
        }
    }
}

// Many rows: bound by the matrix pipe and, side by side with it, the exponentials.  One workgroup of eight waves, two per SIMD, streams the item's range once
// for up to 24 tiles of rows, dealt round-robin to the waves, which keep their queries and accumulators in registers (NT tiles each).  A tile of
// 64 keys passes through LDS twice: its codes come from memory by direct loads, kRaw tiles ahead, a wave's eight keys (1 KB each of K and V) to a
// place that only this wave reads; the wave converts them to bf16 and stores them for all, K rows swizzled by the key (the 16-byte fragments of 16
// keys hit 16 distinct places), V rows by twice the key (a transposing read takes two neighbouring places of each of 8 keys).
// The two waves of a SIMD run half a period apart, so that one's softmax runs under the other's products: per tile a wave does [P V of the tile
// before, Q K^T] and then [softmax, conversion of the next tile], and the early waves 0 .. 3 meet the tile's barrier in front of the first half, the
// late ones 4 .. 7 between the two.  Between barriers `it` and `it + 1` all read K of tile it and V of it - 1, and write both of tile it + 1: two
// stages of K and three of V.
constexpr int kRaw = 3;
constexpr int kRawBytes = 2 * kKT * kD + 128, kStageK = kKT * kD * 2;   // (raw: K codes, V codes, 16 exponent bytes per wave)
constexpr int kManyPages = 64 * 4;
constexpr int kManyLds = kRaw * kRawBytes + 5 * kStageK + kManyPages * 4 + 64 * 8;

__device__ __forceinline__ void dma_16(u32x4_t rsrc, uint32_t voff, uint32_t lds_bytes) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen nt lds" : : "v"(voff), "s"(rsrc), "s"(lds_bytes) : "memory", "m0");
}
__device__ __forceinline__ void dma_4(u32x4_t rsrc, uint32_t voff, uint32_t lds_bytes) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" : : "v"(voff), "s"(rsrc), "s"(lds_bytes) : "memory", "m0");
}

template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_at(uint32_t offset) { return (__attribute__((address_space(3))) T*)(uintptr_t)offset; }

template <int NT>
__device__ __forceinline__ void kv8_many_body(const KV8Item& it, int kh, int rg, int n_q_heads, int64_t q_stride, const uint16_t* __restrict__ q, const KV8Rows& rows,
                                              const KV8Layer& kv, uint16_t* __restrict__ out, float* __restrict__ part_o, float* __restrict__ part_ml,
                                              int row_tiles, int per_group, float scale_log2, uint8_t* lds) {
    constexpr int TPW = NT > 0 ? NT : 1;
    typedef __attribute__((ext_vector_type(4))) short s16x4_t;
    typedef __attribute__((ext_vector_type(8))) short s16x8_t;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int b = it.b, ctx = it.ctx, n = rows.n, total = ctx + n, n_kv = kv.n_kv, G = n_q_heads / n_kv, R = n * G;
    const int n_tiles = it.hi - it.lo, k0 = it.lo * kKT;
    uint16_t* st_k = (uint16_t*)lds;   // (the stages first: their places are worked out with exclusive ors below 256)
    uint16_t* st_v = st_k + 2 * (kStageK / 2);
    uint8_t* raw = lds + 5 * kStageK;
    int32_t* page_ids = (int32_t*)(raw + kRaw * kRawBytes);
    uint64_t* mask_lds = (uint64_t*)(page_ids + kManyPages);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds, raw_base = lds_base + 5 * kStageK;

    // ---- this wave's row tiles
    u32x4_t qf[TPW][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = (rg * per_group + wave + 8 * t) * 16 + l16, i = r / G, g = r - i * G;
        const bool on = r < R;
        const uint16_t* p = q + (int64_t)(b * n + (on ? i : 0)) * q_stride + (kh * G + (on ? g : 0)) * kD + g4 * 8;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const u32x4_t z = {0u, 0u, 0u, 0u};
            qf[t][ks] = on ? *(const u32x4_t*)(p + ks * 32) : z;
        }
    }
    // ---- codes and exponents from memory: this wave's keys 8 * wave .. + 7 of a tile lie in one page
    auto rsrc = [&](const uint8_t* p, uint32_t bytes) {
        const uint64_t a = (uint64_t)(uintptr_t)p;
        u32x4_t d;
        d[0] = __builtin_amdgcn_readfirstlane((uint32_t)a);
        d[1] = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xffffu);
        d[2] = __builtin_amdgcn_readfirstlane(bytes);
        d[3] = 0x00020000u;
        return d;
    };
    auto fetch = [&](int slot, int pg) {   // pg < 0: nothing is fetched (the conversion does not look)
        const int64_t row = ((int64_t)max(pg, 0) * n_kv + kh) * 16 + (wave & 1) * 8;
        const uint32_t some = pg < 0 ? 0u : 1u, at = raw_base + slot * kRawBytes + wave * 1024;
        dma_16(rsrc(kv.k + row * kD, some * 1024u), lane * 16, __builtin_amdgcn_readfirstlane(at));
        dma_16(rsrc(kv.v + row * kD, some * 1024u), lane * 16, __builtin_amdgcn_readfirstlane(at + kKT * kD));
        const uint32_t ex = raw_base + slot * kRawBytes + 2 * kKT * kD + wave * 16;
        if (lane < 2) dma_4(rsrc(kv.k_exp + row, some * 8u), lane * 4, __builtin_amdgcn_readfirstlane(ex));
        if (lane < 2) dma_4(rsrc(kv.v_exp + row, some * 8u), lane * 4, __builtin_amdgcn_readfirstlane(ex + 8));
    };
    constexpr int kOps = 4;   // loads of a fetch
    auto page_at = [&](int lp) {
        const int pg = lp < kv.max_pages && lp * 16 < total ? kv.block_table[(int64_t)b * kv.max_pages + lp] : -1;
        return pg < kv.n_pages ? pg : -1;
    };
    {
        int pg[kRaw];
#pragma unroll
        for (int t = 0; t < kRaw; ++t) pg[t] = t < n_tiles ? page_at((it.lo + t) * 4 + (wave >> 1)) : -1;
#pragma unroll
        for (int t = 0; t < kRaw; ++t)
            if (t < n_tiles) fetch(t, __builtin_amdgcn_readfirstlane(pg[t]));
    }
    for (int i = tid; i < 4 * n_tiles; i += 512) page_ids[i] = page_at(it.lo * 4 + i);
    for (int i = tid; i < n; i += 512) mask_lds[i] = (rows.mask ? rows.mask[b * n + i] : (2ull << i) - 1ull) & (~0ull >> (64 - n));
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

    // tile t, which has landed, to bf16; then the fetch of tile t + kRaw into its place
    auto convert = [&](int t) {
        if (t >= n_tiles) return;   // uniform
        if (t + kRaw <= n_tiles) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kOps * (kRaw - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        int ln = lane;
        asm volatile("" : "+v"(ln));   // (places are worked out anew for every tile: kept, they would cost registers that the products need)
        const int slot = t % kRaw, key = 8 * wave + (ln >> 3), p = ln & 7;
        const uint8_t* rp = raw + slot * kRawBytes;
        u32x4_t kc = *(const u32x4_t*)(rp + wave * 1024 + ln * 16), vc = *(const u32x4_t*)(rp + kKT * kD + wave * 1024 + ln * 16);
        uint32_t ke = rp[2 * kKT * kD + wave * 16 + (ln >> 3)], ve = rp[2 * kKT * kD + wave * 16 + 8 + (ln >> 3)];
        const bool backed = __builtin_amdgcn_readfirstlane(page_ids[4 * t + (wave >> 1)]) >= 0;
        const int next = t + kRaw < n_tiles ? __builtin_amdgcn_readfirstlane(page_ids[4 * (t + kRaw) + (wave >> 1)]) : -1;
        const bool in = backed && k0 + t * kKT + key < total;   // (slots that nobody has written may hold anything)
        // (values that are not finite: their codes are zero, the NaN comes through the key, whose score only rows that see it keep)
        ke = !backed ? 127u : (in && ve == 255u ? 255u : ke);
        ve = ve == 255u ? 127u : ve;
#pragma unroll
        for (int c = 0; c < 4; ++c) kc[c] = backed ? kc[c] : 0u, vc[c] = in ? vc[c] : 0u;
        const float sk = __uint_as_float(ke << 23), sv = __uint_as_float(ve << 23);
        uint16_t* ko = st_k + (t & 1) * (kStageK / 2) + key * kD;
        uint16_t* vo = st_v + (t % 3) * (kStageK / 2) + key * kD;
        *(u32x4_t*)(ko + ((2 * p) ^ (key & 15)) * 8) = cvt8(kc[0], kc[1], sk);
        *(u32x4_t*)(ko + ((2 * p + 1) ^ (key & 15)) * 8) = cvt8(kc[2], kc[3], sk);
        // (rows of odd keys start with their other half: even pieces of one row and odd ones of its neighbour share no bank)
        const u32x4_t v0 = cvt8(vc[0], vc[1], sv), v1 = cvt8(vc[2], vc[3], sv);
        const int odd = key & 1;
        *(u32x4_t*)(vo + ((2 * p + odd) ^ ((2 * key) & 15)) * 8) = odd ? v1 : v0;
        *(u32x4_t*)(vo + ((2 * p + 1 - odd) ^ ((2 * key) & 15)) * 8) = odd ? v0 : v1;
        if (t + kRaw < n_tiles) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (the codes have been read)
            fetch(slot, next);
        }
    };
    auto meet = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    f32x4_t acc[TPW][8], acc_l[TPW];
    float m_run[TPW];
    u32x4_t pb[TPW][2];   // weights of the tile whose second product is still owed
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m_run[t] = kNegBig;
        acc_l[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        pb[t][0] = pb[t][1] = u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    // ---- O^T += V^T P^T: a transposing read hands lane (l16, g4) keys 4 * g4 .. + 3 of 16 for d = 16 * dt + l16; two of them are 8 k slots.  Four batches
    // (half of the keys, half of d), each read under the products of the one before.
    auto second = [&](int stage) {
        if constexpr (NT == 0) return;
        s16x4_t vv[2][4][2];
        int ln = lane;
        asm volatile("" : "+v"(ln));   // (as in the conversion)
        // key 4 * g4 + l16 / 4 of the 16, its piece 2 * dt + (l16 & 3) / 2 swizzled by twice the key (16 keys further on: by the same)
        const int kr = 4 * (ln >> 4) + ((ln & 15) >> 2);
        const uint32_t at = lds_base + 2 * kStageK + stage * kStageK + kr * (2 * kD) + ((((ln & 3) >> 1) ^ ((2 * kr) & 15)) * 16) + (ln & 1) * 8;
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
                    acc_l[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ones), __builtin_bit_cast(bf16x8_t, pb[t][half]), acc_l[t], 0, 0, 0);
            }
#pragma unroll
            for (int d4 = 0; d4 < 4; ++d4) {
                const s16x8_t a = {v[d4][0][0], v[d4][0][1], v[d4][0][2], v[d4][0][3], v[d4][1][0], v[d4][1][1], v[d4][1][2], v[d4][1][3]};
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    acc[t][dq * 4 + d4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, pb[t][half]),
                                                                                  acc[t][dq * 4 + d4], 0, 0, 0);
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
    const float lazy = 8.0f / scale_log2;
    const bool late = wave >= 4;
    convert(0);
    if (late) {
        meet();
        convert(1);
    }
    for (int i = 0; i < n_tiles; ++i) {
        if (!late) meet();
        __builtin_amdgcn_s_setprio(2);
        if (i > 0) second((i - 1) % 3);
        const int t0 = k0 + i * kKT;
        int lk = lane;
        asm volatile("" : "+v"(lk));
        const uint32_t k_at = lds_base + (i & 1) * kStageK + (lk & 15) * (2 * kD) + (((lk >> 4) ^ (lk & 15)) * 16);
        // ---- S^T = K Q^T, the next 16 keys' fragments read under the products of those before
        f32x4_t sc[TPW][4];
        bf16x8_t kf[2][4];
        auto read_k = [&](int s, bf16x8_t* f) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                f[ks] = __builtin_bit_cast(bf16x8_t, *lds_at<u32x4_t>((k_at ^ (uint32_t)(ks * 64)) + s * 16 * (2 * kD)));
        };
        auto mul_k = [&](int s, const bf16x8_t* f) {
#pragma unroll
            for (int t = 0; t < NT; ++t) sc[t][s] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    sc[t][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[ks], __builtin_bit_cast(bf16x8_t, qf[t][ks]), sc[t][s], 0, 0, 0);
        };
        if constexpr (NT > 0) {
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
        // ---- running maximum and weights
        const int edge = t0 + kKT > ctx ? 1 : 0;   // new rows, or keys behind the last (a trip count: an `if` around so many selects would run on every tile)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            for (int rep = 0; rep < edge; ++rep) {
                int ln = lane;
                asm volatile("" : "+v"(ln));
                const int r = (rg * per_group + wave + 8 * t) * 16 + (ln & 15);
                const uint64_t seen = seen_from(t0 + 4 * (ln >> 4) - ctx, r < R ? mask_lds[r / G] : 0ull);
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
            if (__builtin_amdgcn_ballot_w64(tmax > m_run[t] + lazy) != 0) {   // (as in the kernel of few rows)
                const float m_new = fmaxf(m_run[t], group_max4(tmax));
                const float alpha = __builtin_amdgcn_exp2f((m_run[t] - m_new) * scale_log2);
                m_run[t] = m_new;
                acc_l[t] *= alpha;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) acc[t][dt] *= alpha;
            }
            const float mc = fmaxf(m_run[t], -1e29f) * scale_log2;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                float e[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) e[v] = __builtin_amdgcn_exp2f(fmaf(sc[t][s][v], scale_log2, -mc));
                pb[t][s >> 1][2 * (s & 1)] = pack_bf16x2(e[0], e[1]);
                pb[t][s >> 1][2 * (s & 1) + 1] = pack_bf16x2(e[2], e[3]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);   // (registers again: neither half of the period may reach into the conversion)
        convert(i + (late ? 2 : 1));
        __builtin_amdgcn_sched_barrier(0);
    }
    second((n_tiles - 1) % 3);
    // ---- lane (l16, g4) holds d = 16 * dt + 4 * g4 + v of row l16
    const int r_pad = row_tiles * 16;
    const int64_t pbase = ((int64_t)it.slot * n_kv + kh) * r_pad;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = (rg * per_group + wave + 8 * t) * 16 + l16;
        if (r >= R) continue;
        const float l = acc_l[t][0];
        if (it.k == 1) {
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            const int i = r / G, g = r - i * G;
            uint16_t* o = out + ((int64_t)(b * n + i) * n_q_heads + kh * G + g) * kD + 4 * g4;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
                *(u32x2_t*)(o + 16 * dt) = u32x2_t{pack_bf16x2(acc[t][dt][0] * inv, acc[t][dt][1] * inv), pack_bf16x2(acc[t][dt][2] * inv, acc[t][dt][3] * inv)};
        } else {
            float* po = part_o + (pbase + r) * kD + 4 * g4;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) *(f32x4_t*)(po + 16 * dt) = acc[t][dt];
            if (g4 == 0) part_ml[(pbase + r) * 2] = m_run[t], part_ml[(pbase + r) * 2 + 1] = l;
        }
    }
}

// Workgroup id -> (item, kv head, group of row tiles).  Ids are dealt round-robin over the 8 XCDs, and the groups of one (item, kv head) read the same keys and
// values: they get ids 8 apart, so that they run on one XCD at the same time.
template <int TPW>
__global__ __launch_bounds__(512) void kv8_attn_many_k(KV8Split sp, int n_q_heads, int64_t q_stride, const uint16_t* __restrict__ q, KV8Rows rows, KV8Layer kv,
                                                       uint16_t* __restrict__ out, KV8Seg* __restrict__ seg, float* __restrict__ part_o,
                                                       float* __restrict__ part_ml, int row_tiles, int groups, int per_group, float scale_log2) {
    __shared__ __align__(256) uint8_t lds[kManyLds];
    const int id = blockIdx.x, g = id / (8 * groups), within = id - g * 8 * groups, rg = within >> 3, pair = g * 8 + (within & 7);
    const int item = pair / kv.n_kv, kh = pair - item * kv.n_kv;
    KV8Item it;
    if (!kv8_item(kv.seq_len, rows.B, rows.n, kv.seq_len_bound, sp, item, it)) return;   // uniform
    if (kh == 0 && rg == 0 && it.slot == it.first && threadIdx.x == 0) seg[it.b] = KV8Seg{it.first, it.k};
    // row tiles of this wave (a wave runs the program for as many as it has; all pass the same barriers)
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int mine = min(per_group, row_tiles - rg * per_group), n_on = mine > wave ? (mine - wave + 7) / 8 : 0;
#define TLT_BODY(N) kv8_many_body<N>(it, kh, rg, n_q_heads, q_stride, q, rows, kv, out, part_o, part_ml, row_tiles, per_group, scale_log2, lds)
    if (n_on >= TPW) TLT_BODY(TPW);
    else if (TPW >= 2 && n_on == TPW - 1) TLT_BODY((TPW >= 2 ? TPW - 1 : 0));
    else if (TPW >= 3 && n_on == TPW - 2) TLT_BODY((TPW >= 3 ? TPW - 2 : 0));
    else TLT_BODY(0);
#undef TLT_BODY
}

// The ranges of a sequence joined: a wave per row, in the order of the ranges; the lanes read a range's maximum and sum each, and the outputs of
// 16 ranges are requested together.
__global__ __launch_bounds__(256) void kv8_join_k(const KV8Seg* __restrict__ seg, const float* __restrict__ part_o, const float* __restrict__ part_ml,
                                                  uint16_t* __restrict__ out, int n, int n_q_heads, int n_kv, int r_pad, int slot_step, float scale_log2) {
    constexpr int U = 16;
    const int r = blockIdx.x * 4 + (threadIdx.x >> 6), kh = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63;
    const int G = n_q_heads / n_kv;
    const KV8Seg sg = seg[b];
    if (r >= n * G || sg.k <= 1) return;   // (one range: its workgroup has written the row)
    const int64_t base = ((int64_t)sg.first * n_kv + kh) * r_pad + r, step = (int64_t)slot_step * n_kv * r_pad;
    float2 ml = make_float2(kNegBig, 0.f), v[U];
    auto fetch = [&](int c) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            v[u] = c + u < sg.k ? *(const float2*)(part_o + (base + (c + u) * step) * kD + lane * 2) : make_float2(0.f, 0.f);
    };
    if (lane < sg.k) ml = *(const float2*)(part_ml + (base + lane * step) * 2);
    fetch(0);
    float M = ml.x;
    for (int c = lane + 64; c < sg.k; c += 64) M = fmaxf(M, part_ml[(base + c * step) * 2]);
    M = wave_max(M);
    float w = exp2f((ml.x - M) * scale_log2), wl = ml.y * w, a0 = 0.f, a1 = 0.f, L = 0.f;
    for (int c0 = 0; c0 < sg.k; c0 += U) {   // (uniform)
        if (c0 > 0) {
            fetch(c0);
            if ((c0 & 63) == 0) {
                ml = c0 + lane < sg.k ? *(const float2*)(part_ml + (base + (c0 + lane) * step) * 2) : make_float2(kNegBig, 0.f);
                w = exp2f((ml.x - M) * scale_log2), wl = ml.y * w;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (c0 + u >= sg.k) break;
            const float wu = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), (c0 + u) & 63));
            L += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wl), (c0 + u) & 63));
            a0 = fmaf(wu, v[u].x, a0), a1 = fmaf(wu, v[u].y, a1);
        }
    }
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    const int i = r / G, g = r - i * G;
    ((uint32_t*)(out + ((int64_t)(b * n + i) * n_q_heads + kh * G + g) * kD))[lane] = pack_bf16x2(a0 * inv, a1 * inv);
}

constexpr int kFewRows = 16;
struct KV8Plan {
    KV8Split sp;
    bool few;        // the kernel of few rows
    bool one_each;   // no sequence has a second range
    int row_tiles, groups, per_group, tpw;
    size_t seg, part_o, part_ml, total;   // byte offsets into the workspace
};
static KV8Plan plan_kv8(int B, int n, int n_q_heads, int n_kv, int bound_total) {
    KV8Plan p;
    const int R = n * (n_q_heads / n_kv), tiles = (bound_total + kKT - 1) / kKT;
    p.few = R <= kFewRows;
    p.row_tiles = (R + 15) / 16;
    p.groups = p.few ? 1 : (p.row_tiles + 23) / 24;
    p.per_group = (p.row_tiles + p.groups - 1) / p.groups;
    p.tpw = (p.per_group + 7) / 8;
    p.sp.slots = std::max(1, (p.few ? 768 : 256) / (n_kv * p.groups));
    p.sp.t_min = 4;
    p.sp.t_max = 64;
    p.one_each = tiles <= p.sp.t_min || (B > kPlanned && tiles <= p.sp.t_max);
    p.sp.max_items = p.one_each ? B : (int)(B > kPlanned ? (int64_t)B * ((tiles + p.sp.t_max - 1) / p.sp.t_max) : (int64_t)B * tiles / p.sp.t_max + B + p.sp.slots);
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
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
        for (int m = 1; m <= n; ++m)   // (any number of rows up to n may be asked for later)
            need = std::max(need, plan_kv8(B, m, n_q_heads, n_kv_heads, max_ctx).total);
    return need;
}

hipError_t kv8_attention(hipStream_t s, int dtype, const KV8Rows& rows, const KV8Layer& kv, const void* q, int64_t q_stride, void* out, int n_q_heads, void* ws,
                         size_t ws_bytes, int impl) {
    const int R = rows.n * (n_q_heads / kv.n_kv);
    const bool fits = dtype == BF16 && kv.d == kD && kv.page_size == 16 && (((uintptr_t)kv.k_exp | (uintptr_t)kv.v_exp) & 3) == 0;
    if (fits && impl != 0) {
        const KV8Plan p = plan_kv8(rows.B, rows.n, n_q_heads, kv.n_kv, kv.seq_len_bound + rows.n);
        if (p.total > ws_bytes) return hipErrorInvalidValue;
        KV8Seg* seg = (KV8Seg*)((char*)ws + p.seg);
        float *part_o = (float*)((char*)ws + p.part_o), *part_ml = (float*)((char*)ws + p.part_ml);
        const float scale_log2 = 1.4426950408889634f / sqrtf((float)kD);
        const unsigned pairs = (unsigned)(p.sp.max_items * kv.n_kv);
        if (p.few) {
            hipLaunchKernelGGL(kv8_attn_few_k<1>, dim3(pairs), dim3(256), 0, s, p.sp, n_q_heads, q_stride, (const uint16_t*)q, rows, kv, (uint16_t*)out, seg, part_o,
                               part_ml, scale_log2);
        } else {
            auto many = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3((pairs + 7) / 8 * 8 * p.groups), dim3(512), 0, s, p.sp, n_q_heads, q_stride, (const uint16_t*)q, rows, kv,
                                   (uint16_t*)out, seg, part_o, part_ml, p.row_tiles, p.groups, p.per_group, scale_log2);
            };
            if (p.tpw == 1) many(kv8_attn_many_k<1>);
            else if (p.tpw == 2) many(kv8_attn_many_k<2>);
            else many(kv8_attn_many_k<3>);
        }
        hipError_t e = hipGetLastError();
        if (e != hipSuccess || p.one_each) return e;
        hipLaunchKernelGGL(kv8_join_k, dim3((R + 3) / 4, kv.n_kv, rows.B), dim3(256), 0, s, seg, part_o, part_ml, (uint16_t*)out, rows.n, n_q_heads, kv.n_kv,
                           p.row_tiles * 16, rows.B > kPlanned ? rows.B : 1, scale_log2);
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
