// Frequencies of rotary positions, scaled for contexts longer than the ones a model was trained on (host only).
#include <algorithm>
#include <cmath>

#include "../../include/tlt.h"

int tlt_rope_freqs(int kind, int rot_dim, double theta, double factor, double original_len, double low, double high, double* freq, float* amplitude) {
    if (kind < TLT_ROPE_PLAIN || kind > TLT_ROPE_BANDS || rot_dim < 2 || rot_dim % 2 || rot_dim > 65536 || !(theta > 1.0) || !std::isfinite(theta) || !freq) return TLT_EINVAL;
    if (kind != TLT_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return TLT_EINVAL;
    if (kind == TLT_ROPE_BASE && rot_dim < 4) return TLT_EINVAL;
    const bool parts = kind == TLT_ROPE_RAMP || kind == TLT_ROPE_BANDS;
    if (parts && (!(original_len > 0.0) || !std::isfinite(original_len) || !(low > 0.0) || !(high > low) || !std::isfinite(high))) return TLT_EINVAL;
    if (kind == TLT_ROPE_PLAIN) factor = 1.0;
    const double two_pi = 6.283185307179586476925;
    const double base = kind == TLT_ROPE_BASE ? theta * std::pow(factor, (double)rot_dim / (rot_dim - 2)) : theta;
    // the pair that turns n times over original_len: theta^(-2j / rot_dim) * original_len = 2 pi n
    auto pair_of = [&](double n) { return rot_dim * std::log(original_len / (two_pi * n)) / (2.0 * std::log(theta)); };
    const double from = parts ? std::max(std::floor(pair_of(high)), 0.0) : 0.0, to = parts ? std::min(std::ceil(pair_of(low)), rot_dim - 1.0) : 0.0;
    for (int j = 0; j < rot_dim / 2; ++j) {
        const double f = std::pow(base, -2.0 * j / rot_dim);
        double slow = 0.0;   // share of the scaled frequency
        if (kind == TLT_ROPE_LINEAR) slow = 1.0;
        if (kind == TLT_ROPE_RAMP) slow = (j - from) / std::max(to - from, 1e-3);   // (a ramp without width is a step)
        if (kind == TLT_ROPE_BANDS) slow = 1.0 - (original_len * f / two_pi - low) / (high - low);
        slow = std::min(std::max(slow, 0.0), 1.0);
        freq[j] = kind == TLT_ROPE_LINEAR ? f / factor : f * (1.0 - slow) + f / factor * slow;
    }
    if (amplitude) *amplitude = kind == TLT_ROPE_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return TLT_OK;
}
