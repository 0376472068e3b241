// The 8-bit paged KV cache: writing rows, attention over them, keeping the accepted path, reading rows back.
//
// A row (one token of one kv head, d elements) is d codes in e4m3 (OCP: 4 exponent bits, bias 7, largest value 448, no infinities) and one
// exponent byte E; its values are code * 2^(E - 127).  E - 127 is the smallest e >= -126 with max|x| <= 448 * 2^e, so scaling by it is exact, the one
// rounding is that to e4m3, nothing saturates, and a value has four significant bits: it is exact in bf16 too.  A row with an element that is not
// finite keeps E = 255 and codes of zero, and all of it reads as NaN.
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

size_t kv8_attention_workspace_bytes(int B, int n, int n_q_heads, int n_kv_heads, int d, int max_ctx) { return 256; }

hipError_t kv8_attention(hipStream_t s, int dtype, const KV8Rows& rows, const KV8Layer& kv, const void* q, int64_t q_stride, void* out, int n_q_heads, void* ws,
                         size_t ws_bytes, int impl) {
    const float scale = 1.0f / sqrtf((float)kv.d);
    const dim3 grid(rows.n, n_q_heads, rows.B), block(64 * kRowWaves);
    if (dtype == F32)
        hipLaunchKernelGGL(kv8_attn_row_k<float>, grid, block, 0, s, rows, kv, (const float*)q, q_stride, (float*)out, n_q_heads, scale);
    else
        hipLaunchKernelGGL(kv8_attn_row_k<bf16>, grid, block, 0, s, rows, kv, (const bf16*)q, q_stride, (bf16*)out, n_q_heads, scale);
    return hipGetLastError();
}

}  // namespace tlt
