// Rotary positions, host side: the frequencies of a head's pairs, scaled for contexts longer than a model was trained for, and the
// form in which the kernels of deft_heads.hip take them.  No device calls.
#include <algorithm>
#include <cmath>

#include "deft.h"

namespace {
constexpr int kMaxRot = 128;
constexpr double kMaxFrequency = 1e6;  // radians a position
bool rot_ok(int32_t rot) { return rot >= 16 && rot <= kMaxRot && rot % 16 == 0; }
constexpr long double kTurn = 6.283185307179586476925286766559005768L;
}  // namespace

extern "C" int deft_rope_frequencies(int32_t rot, double base, int32_t scaling, double scale, double original, double low, double high,
                                     double *frequency, double *factor) {
    if (!rot_ok(rot) || !frequency || !factor || !std::isfinite(base) || base <= 1) return DEFT_EINVAL;
    if (scaling < DEFT_ROPE_PLAIN || scaling > DEFT_ROPE_WAVELENGTH) return DEFT_EINVAL;
    if (scaling != DEFT_ROPE_PLAIN && !(std::isfinite(scale) && scale > 0)) return DEFT_EINVAL;
    const bool ramp = scaling == DEFT_ROPE_DIMENSION || scaling == DEFT_ROPE_WAVELENGTH;
    if (ramp) {
        if (!(low > 0)) low = 1;
        if (!(high > 0)) high = scaling == DEFT_ROPE_DIMENSION ? 32 : 4;
        if (!std::isfinite(original) || original <= 0 || !std::isfinite(high) || low >= high) return DEFT_EINVAL;
    }
    if (scaling == DEFT_ROPE_BASE) base *= std::pow(scale, rot / (rot - 2.0));
    if (!std::isfinite(base) || base <= 1) return DEFT_EINVAL;
    // the dimension that makes `turns` turns within the original length, as a real number
    auto dimension = [&](double turns) { return rot * std::log(original / (turns * (double)kTurn)) / (2 * std::log(base)); };
    double first = 0, width = 1;
    if (scaling == DEFT_ROPE_DIMENSION) {
        first = std::max(std::floor(dimension(high)), 0.0);
        width = std::max(std::min(std::ceil(dimension(low)), rot - 1.0) - first, 0.001);
    }
    double out[kMaxRot / 2];
    for (int32_t i = 0; i < rot / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot);
        double keep = 1;  // share of f that stays f; the rest becomes f / scale
        if (scaling == DEFT_ROPE_LINEAR) keep = 0;
        if (scaling == DEFT_ROPE_DIMENSION) keep = 1 - std::clamp((i - first) / width, 0.0, 1.0);
        if (scaling == DEFT_ROPE_WAVELENGTH) keep = std::clamp((original * f / (double)kTurn - low) / (high - low), 0.0, 1.0);
        out[i] = f * keep + (keep < 1 ? f / scale * (1 - keep) : 0);
        if (!(out[i] <= kMaxFrequency)) return DEFT_EINVAL;
    }
    std::copy(out, out + rot / 2, frequency);
    *factor = scaling == DEFT_ROPE_DIMENSION && scale > 1 ? 0.1 * std::log(scale) + 1 : 1;
    return DEFT_OK;
}

// A position is a whole number, so whole turns of a frequency say nothing and its fraction of a turn is held in 64 bits behind the
// point: position x fraction modulo one turn is then a product of whole numbers, and a far position's angle is as exact as a near one's
// (2^-64 of a turn a position: 2^-33 at the farthest, where an fp32 product is off by whole radians).
extern "C" int deft_rope(const double *frequency, int32_t rot, int32_t layout, double factor, deft_rope_t *out) {
    if (!frequency || !out || !rot_ok(rot) || (layout != DEFT_ROPE_HALF && layout != DEFT_ROPE_INTERLEAVED)) return DEFT_EINVAL;
    if (!std::isfinite(factor) || !std::isfinite((float)factor)) return DEFT_EINVAL;
    deft_rope_t rope = {};
    rope.rot = rot;
    rope.layout = layout;
    rope.factor = (float)factor;
    for (int32_t i = 0; i < rot / 2; ++i) {
        if (!std::isfinite(frequency[i]) || std::fabs(frequency[i]) > kMaxFrequency) return DEFT_EINVAL;
        const long double turns = std::fabs((long double)frequency[i]) / kTurn, part = std::ldexp(turns - std::floor(turns), 64);
        const long double bits = std::round(part);  // 0 .. 2^64
        rope.turns[i] = bits >= std::ldexp(1.0L, 64) ? 0 : (uint64_t)bits;
        if (frequency[i] < 0) rope.turns[i] = 0 - rope.turns[i];
    }
    *out = rope;
    return DEFT_OK;
}
