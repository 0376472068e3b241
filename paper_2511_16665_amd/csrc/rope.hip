// Rotary positions for new rows, written to rows, to the slots of a paged cache, or to those of an 8-bit one.
#include <algorithm>

#include "dev_common.h"
#include "kernels.h"
#include "kv8_format.h"

namespace tlt {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

__device__ __forceinline__ void unpack(u32x4_t w, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(w[e]);
}
__device__ __forceinline__ void unpack(u32x4_t w, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(w[e] << 16), x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
}
template <typename T, int VEC>
__device__ __forceinline__ u32x4_t packed(const float (&x)[VEC]) {
    u32x4_t w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (VEC == 4) w[e] = __float_as_uint(x[e]);
        else w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
    }
    return w;
}

// amplitude times cos and sin of position * freq.  The product in double, in turns, of which the fraction is exact; an eighth of a turn at most from a quarter turn, where Taylor's series to the 12th and 11th
// power are 2^-37 off: so both are right to half a unit of fp32's last place but for one in a thousand.  (sincospif of the fraction in fp32 is up to 2^-23 off: rows of an 8-bit cache then differed from angles in
// double by 1.7e-5, root mean square, as some values round the other way, now by 6.5e-7; it takes as long.)
__device__ __forceinline__ void turn(int position, double freq, float amplitude, float& c, float& s) {
    const double t = (double)position * (freq * 0.15915494309189533577);   // 1 / 2 pi
    const double f = t - rint(t), q = rint(4.0 * f), x = (f - 0.25 * q) * 6.2831853071795864769, z = x * x;
    double u = fma(z, -1.0 / 39916800, 1.0 / 362880);
    u = fma(z, u, -1.0 / 5040);
    u = fma(z, u, 1.0 / 120);
    u = fma(z, u, -1.0 / 6);
    u = fma(z * x, u, x);
    double v = fma(z, 1.0 / 479001600, -1.0 / 3628800);
    v = fma(z, v, 1.0 / 40320);
    v = fma(z, v, -1.0 / 720);
    v = fma(z, v, 1.0 / 24);
    v = fma(z, v, -0.5);
    v = fma(z, v, 1.0);
    const int quarter = (int)q;   // -2 .. 2
    const double a = (double)amplitude, cs = quarter & 1 ? u : v, sn = quarter & 1 ? v : u;
    c = (float)(a * ((quarter + 1) & 2 ? -cs : cs)), s = (float)(a * (quarter & 2 ? -sn : sn));
}

// One wave per row and head, lane l holding elements of pairs l and l + 64: any layout, any even head_dim up to 256, any alignment.
template <typename T>
__global__ __launch_bounds__(256) void rope_any_k(int rows, int n_q_heads, RopeIn in, RopeOut out) {
    const int heads = n_q_heads + 2 * out.n_kv, d = out.d, half = in.rot_dim >> 1;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= (int64_t)rows * heads) return;
    const int r = (int)(unit / heads), h = (int)(unit - (int64_t)r * heads), lane = threadIdx.x & 63;
    const bool is_q = h < n_q_heads, turned = h < n_q_heads + out.n_kv;
    const T* x = (const T*)in.qkv + (int64_t)r * in.stride + h * d;
    const T* bias = in.bias ? (const T*)in.bias + h * d : nullptr;
    const int position = in.position[r];
    float a[2], b[2];
    int ia[2], ib[2];
    uint32_t amax = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int p = lane + 64 * k;
        ia[k] = -1;
        if (2 * p >= d) continue;
        const bool pair = p < half;
        ia[k] = !pair || in.interleaved ? 2 * p : p;
        ib[k] = !pair || in.interleaved ? 2 * p + 1 : p + half;
        a[k] = to_float(x[ia[k]]), b[k] = to_float(x[ib[k]]);
        if (bias) a[k] += to_float(bias[ia[k]]), b[k] += to_float(bias[ib[k]]);
        if (turned && pair) {
            float c, s;
            turn(position, in.freq[p], in.amplitude, c, s);
            const float u = a[k], v = b[k];
            a[k] = u * c - v * s, b[k] = v * c + u * s;
        }
        amax = max(amax, max(__float_as_uint(a[k]) & 0x7fffffffu, __float_as_uint(b[k]) & 0x7fffffffu));
    }
    if (is_q) {
        if (!out.q) return;
        T* o = (T*)out.q + (int64_t)r * out.q_stride + h * d;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (ia[k] >= 0) o[ia[k]] = from_float<T>(a[k]), o[ib[k]] = from_float<T>(b[k]);
        return;
    }
    const int kh = h - n_q_heads;   // keys, then values
    if (out.rows) {
        T* o = (T*)out.rows + (int64_t)r * out.rows_stride + kh * d;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (ia[k] >= 0) o[ia[k]] = from_float<T>(a[k]), o[ib[k]] = from_float<T>(b[k]);
    }
    if (!out.k) return;
    const int64_t slot = in.slot[r];
    if (slot < 0 || slot >= out.n_slots) return;
    const int64_t page = slot / out.page_size;
    const int64_t to = (page * out.n_kv + (turned ? kh : kh - out.n_kv)) * out.page_size + (slot - page * out.page_size);
    if (!out.k_exp) {
        T* o = (T*)(turned ? out.k : out.v) + to * d;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (ia[k] >= 0) o[ia[k]] = from_float<T>(a[k]), o[ib[k]] = from_float<T>(b[k]);
        return;
    }
    for (int o = 1; o < 64; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, 64));
    const uint32_t e = exponent_of(amax);
    const float inv = inverse_scale_of(e);
    uint8_t* o = (uint8_t*)(turned ? out.k : out.v) + to * d;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (ia[k] >= 0) {
            const uint32_t w = encode4(a[k], b[k], 0.f, 0.f, inv);
            o[ia[k]] = (uint8_t)w, o[ib[k]] = (uint8_t)(w >> 8);
        }
    if (lane == 0) (turned ? out.k_exp : out.v_exp)[to] = (uint8_t)e;
}

// A workgroup per row and 2 x 16 bytes of a head per thread, the two pieces holding whole pairs: with pairs (j, j + rot_dim / 2) a piece of either half of the turned part (or two
// pieces behind it), with pairs (2j, 2j + 1) two pieces side by side.  The row's angles are formed once and shared through LDS; its elements are asked for before that.
// Bound by memory for many rows: 8190 rows of 64 + 8 + 8 heads of 128 (336 MB) in 62 us, 5.4 TB/s; rope_any_k, which forms a head's angles for itself, 208.  Few rows are a chain, position, angle, LDS, store: one row
// 2.6 us, 1536 rows of 28 + 4 + 4 heads into 8 bits 9.5 (a wave per head 24).
template <typename T, bool INTERLEAVED, bool E8>
__global__ __launch_bounds__(1024) void rope_row_k(int n_q_heads, int lanes_log2, RopeIn in, RopeOut out) {
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float cs[128], sn[128];
    const int r = blockIdx.x, tid = threadIdx.x, d = out.d, n_kv = out.n_kv, heads = n_q_heads + 2 * n_kv, half = in.rot_dim >> 1;
    const int units = d / (2 * VEC), total = heads * units, turned_units = half / VEC;   // (of pairs that lie half a turned part from each other)
    const T* row = (const T*)in.qkv + (int64_t)r * in.stride;
    const int64_t slot = out.k ? in.slot[r] : -1;
    const int position = tid < half ? in.position[r] : 0;
    const double freq = tid < half ? in.freq[tid] : 0.0;
    auto place = [&](int u, int& h, int& p, int& lo, int& hi) {
        h = lanes_log2 >= 0 ? u >> lanes_log2 : u / units;
        p = u - h * units;
        if (INTERLEAVED) lo = p * 2 * VEC, hi = lo + VEC;
        else if (p < turned_units) lo = p * VEC, hi = half + lo;
        else lo = in.rot_dim + (p - turned_units) * 2 * VEC, hi = lo + VEC;
    };
    int h, p, lo, hi;
    u32x4_t wa = {}, wb = {};
    if (tid < total) {
        place(tid, h, p, lo, hi);
        wa = *(const u32x4_t*)(row + h * d + lo), wb = *(const u32x4_t*)(row + h * d + hi);
    }
    if (tid < half) {
        float c, s;
        turn(position, freq, in.amplitude, c, s);
        cs[tid] = c, sn[tid] = s;
    }
    const bool cached = slot >= 0 && slot < out.n_slots;
    int64_t to_row = 0;   // of kv head 0
    if (cached) {
        const int64_t page = slot / out.page_size;
        to_row = page * n_kv * out.page_size + (slot - page * out.page_size);
    }
    __syncthreads();
    for (int u = tid; u - (tid & 63) < total; u += blockDim.x) {   // (whole waves: a head's lanes meet below)
        const bool on = u < total;
        if (u != tid && on) {
            place(u, h, p, lo, hi);
            wa = *(const u32x4_t*)(row + h * d + lo), wb = *(const u32x4_t*)(row + h * d + hi);
        }
        float a[VEC], b[VEC];
        unpack(wa, a), unpack(wb, b);
        const bool is_q = on && h < n_q_heads, turned = on && h < n_q_heads + n_kv;
        if (on && in.bias) {
            float x[VEC], y[VEC];
            unpack(*(const u32x4_t*)((const T*)in.bias + h * d + lo), x), unpack(*(const u32x4_t*)((const T*)in.bias + h * d + hi), y);
#pragma unroll
            for (int e = 0; e < VEC; ++e) a[e] += x[e], b[e] += y[e];
        }
        if (turned) {
            if (INTERLEAVED) {
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    const int i = p * VEC + e / 2, k = i + VEC / 2;   // the pairs
                    const float x = a[e], y = a[e + 1], z = b[e], w = b[e + 1];
                    if (i < half) a[e] = x * cs[i] - y * sn[i], a[e + 1] = y * cs[i] + x * sn[i];
                    if (k < half) b[e] = z * cs[k] - w * sn[k], b[e + 1] = w * cs[k] + z * sn[k];
                }
            } else if (p < turned_units) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float x = a[e], y = b[e], c = cs[lo + e], s = sn[lo + e];
                    a[e] = x * c - y * s, b[e] = y * c + x * s;
                }
            }
        }
        uint32_t amax = 0;
        if (E8) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) amax = max(amax, max(__float_as_uint(a[e]) & 0x7fffffffu, __float_as_uint(b[e]) & 0x7fffffffu));
            for (int o = 1; o < units; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, 64));   // (units is a power of two here)
        }
        if (!on) continue;
        wa = packed<T>(a), wb = packed<T>(b);
        if (is_q) {
            if (out.q) {
                T* o = (T*)out.q + (int64_t)r * out.q_stride + h * d;
                *(u32x4_t*)(o + lo) = wa, *(u32x4_t*)(o + hi) = wb;
            }
            continue;
        }
        const int kh = h - n_q_heads;   // keys, then values
        if (out.rows) {
            T* o = (T*)out.rows + (int64_t)r * out.rows_stride + kh * d;
            *(u32x4_t*)(o + lo) = wa, *(u32x4_t*)(o + hi) = wb;
        }
        if (!cached) continue;
        const int64_t to = to_row + (int64_t)(turned ? kh : kh - n_kv) * out.page_size;
        if (!E8) {
            T* o = (T*)(turned ? out.k : out.v) + to * d;
            *(u32x4_t*)(o + lo) = wa, *(u32x4_t*)(o + hi) = wb;
        } else {
            const uint32_t e8 = exponent_of(amax);
            const float inv = inverse_scale_of(e8);
            uint8_t* o = (uint8_t*)(turned ? out.k : out.v) + to * d;
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
                *(uint32_t*)(o + lo + e) = encode4(a[e], a[e + 1], a[e + 2], a[e + 3], inv);
                *(uint32_t*)(o + hi + e) = encode4(b[e], b[e + 1], b[e + 2], b[e + 3], inv);
            }
            if (p == 0) (turned ? out.k_exp : out.v_exp)[to] = (uint8_t)e8;
        }
    }
}

template <typename T>
static bool by_rows(const RopeIn& in, const RopeOut& out) {
    constexpr int VEC = 16 / sizeof(T);
    auto aligned = [](const void* p, int64_t stride) { return ((uintptr_t)p & 15) == 0 && stride % VEC == 0; };
    if (out.d % (2 * VEC) || !aligned(in.qkv, in.stride) || !aligned(in.bias, 0) || !aligned(out.q, out.q ? out.q_stride : 0) || !aligned(out.rows, out.rows ? out.rows_stride : 0)) return false;
    if (!in.interleaved && in.rot_dim % (2 * VEC)) return false;
    if (out.k_exp) return ((out.d / (2 * VEC)) & (out.d / (2 * VEC) - 1)) == 0;
    return aligned(out.k, 0) && aligned(out.v, 0);
}

template <typename T>
static void rope_launch(hipStream_t s, int rows, int n_q_heads, const RopeIn& in, const RopeOut& out) {
    constexpr int VEC = 16 / sizeof(T);
    const int heads = n_q_heads + 2 * out.n_kv;
    if (!by_rows<T>(in, out)) {
        const int64_t units = (int64_t)rows * heads;
        hipLaunchKernelGGL(rope_any_k<T>, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, rows, n_q_heads, in, out);
        return;
    }
    const int units = out.d / (2 * VEC), total = heads * units, log2 = (units & (units - 1)) == 0 ? __builtin_ctz(units) : -1;
    // as many threads as pieces, in rounds of equal size; enough for the angles
    const int rounds = (total + 1023) / 1024, threads = std::max(128, ((total + rounds - 1) / rounds + 63) / 64 * 64);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(rows), dim3(threads), 0, s, n_q_heads, log2, in, out); };
    if (out.k_exp) in.interleaved ? launch(rope_row_k<T, true, true>) : launch(rope_row_k<T, false, true>);
    else in.interleaved ? launch(rope_row_k<T, true, false>) : launch(rope_row_k<T, false, false>);
}

hipError_t rope_write(hipStream_t s, int dtype, int rows, int n_q_heads, const RopeIn& in, const RopeOut& out) {
    if (dtype == F32) rope_launch<float>(s, rows, n_q_heads, in, out);
    else rope_launch<bf16>(s, rows, n_q_heads, in, out);
    return hipGetLastError();
}

}  // namespace tlt
