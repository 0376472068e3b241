// Rotary positions for new rows, written to rows, to the slots of a paged cache, or to those of an 8-bit one.
#include <algorithm>

#include "dev_common.h"
#include "kernels.h"
#include "kv8_format.h"

namespace tlt {

// cos and sin of position * freq: the product in double, in turns, of which the fraction is exact, so the angle is good to fp32 at any position
__device__ __forceinline__ void turn(int position, double freq, float amplitude, float& c, float& s) {
    const double t = (double)position * (freq * 0.15915494309189533577);   // 1 / 2 pi
    sincospif((float)(2.0 * (t - rint(t))), &s, &c);
    c *= amplitude, s *= amplitude;
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

hipError_t rope_write(hipStream_t s, int dtype, int rows, int n_q_heads, const RopeIn& in, const RopeOut& out) {
    const int64_t units = (int64_t)rows * (n_q_heads + 2 * out.n_kv);
    const dim3 grid((unsigned)((units + 3) / 4)), block(256);
    if (dtype == F32)
        hipLaunchKernelGGL(rope_any_k<float>, grid, block, 0, s, rows, n_q_heads, in, out);
    else
        hipLaunchKernelGGL(rope_any_k<bf16>, grid, block, 0, s, rows, n_q_heads, in, out);
    return hipGetLastError();
}

}  // namespace tlt
