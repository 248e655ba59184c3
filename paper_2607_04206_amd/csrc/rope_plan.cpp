// Host-side plan of rotary positions: validates the descriptor and computes
// the turns per position of every pair in 64 bits. No HIP call is made here.
#include <cmath>
#include <cstring>
#include <string>

#include "../../include/sangam_rope.h"
#include "entry.h"
#include "rope_format.h"

namespace sangam {
void set_error(const std::string& msg);
void clear_error();

const RopePlanHeader* check_rope_plan(const void* plan) {
    if (!plan) return nullptr;
    const RopePlanHeader* h = static_cast<const RopePlanHeader*>(plan);
    if (h->magic != kRopePlanMagic || h->version != kRopePlanVersion) return nullptr;
    return h;
}
}  // namespace sangam

using namespace sangam;

namespace {

sangam_status rope_fail(sangam_status code, const char* msg) {
    set_error(msg);
    return code;
}

sangam_status rope_plan(const sangam_rope_desc* d, void* plan_buf, size_t cap, size_t* used) {
    clear_error();
    if (!d || !used) return rope_fail(SANGAM_ERR_INVALID_ARG, "desc and used must not be NULL");
    *used = 0;
    const int R = d->rot_dim;
    if (R < 2 || R > kRopeMaxDim || R % 2) return rope_fail(SANGAM_ERR_INVALID_ARG, "rot_dim must be even, 2 to 512");
    if (d->interleaved != 0 && d->interleaved != 1) return rope_fail(SANGAM_ERR_INVALID_ARG, "interleaved must be 0 or 1");
    if (d->scaling < SANGAM_ROPE_NONE || d->scaling > SANGAM_ROPE_YARN_INDEX)
        return rope_fail(SANGAM_ERR_INVALID_ARG, "scaling must be one of SANGAM_ROPE_NONE, _LINEAR, _NTK, _YARN and _YARN_INDEX");
    // (comparisons that a NaN fails)
    if (!(d->base > 1.0 && d->base <= 1e30)) return rope_fail(SANGAM_ERR_INVALID_ARG, "base must be above 1 and at most 1e30");
    const bool scaled = d->scaling != SANGAM_ROPE_NONE;
    const double s = scaled ? d->factor : 1.0;
    if (!(s >= 1.0 && s <= 1e6)) return rope_fail(SANGAM_ERR_INVALID_ARG, "factor must be 1 to 1e6");
    if (d->scaling == SANGAM_ROPE_NTK && R < 4) return rope_fail(SANGAM_ERR_INVALID_ARG, "rot_dim must be at least 4 for NTK scaling");
    const bool yarn = d->scaling == SANGAM_ROPE_YARN || d->scaling == SANGAM_ROPE_YARN_INDEX;
    if (yarn &&
        !(d->original_len > 0.0 && d->original_len <= 1e12 && d->beta_slow >= 0.0 && d->beta_fast > d->beta_slow && d->beta_fast <= 1e12))
        return rope_fail(SANGAM_ERR_INVALID_ARG, "YaRN scaling needs original_len > 0 and 0 <= beta_slow < beta_fast");
    if (!(d->magnitude >= 0.0 && d->magnitude <= 1e6)) return rope_fail(SANGAM_ERR_INVALID_ARG, "magnitude must be 0 to 1e6");

    const double two_pi = 6.283185307179586476925286766559;
    // ends of the ramp in the pair's index (beta_slow 0: at infinity)
    double lo = 0.0, hi = 0.0;
    if (d->scaling == SANGAM_ROPE_YARN_INDEX) {
        auto index = [&](double turns) { return R * std::log(d->original_len / (two_pi * turns)) / (2.0 * std::log(d->base)); };
        lo = std::fmin(double(R - 1), std::fmax(0.0, std::floor(index(d->beta_fast))));
        hi = std::fmin(double(R - 1), std::ceil(index(d->beta_slow)));
        if (!(hi >= lo)) return rope_fail(SANGAM_ERR_INVALID_ARG, "original_len is too short for YaRN scaling by index");
    }

    const uint64_t off_turns = (sizeof(RopePlanHeader) + 255u) & ~uint64_t(255);
    const uint64_t total = off_turns + uint64_t(R / 2) * sizeof(double);
    *used = size_t(total);
    if (!plan_buf || cap < total) return rope_fail(SANGAM_ERR_BUFFER, "plan buffer is too small");
    uint8_t* base = static_cast<uint8_t*>(plan_buf);
    std::memset(base, 0, size_t(total));
    RopePlanHeader* h = reinterpret_cast<RopePlanHeader*>(base);
    h->magic = kRopePlanMagic;
    h->version = kRopePlanVersion;
    h->total_bytes = total;
    h->rot_dim = R;
    h->interleaved = d->interleaved;
    h->magnitude = float(d->magnitude > 0.0 ? d->magnitude : yarn ? 0.1 * std::log(s) + 1.0 : 1.0);
    h->off_turns = off_turns;
    double* turns = reinterpret_cast<double*>(base + off_turns);
    const double b = d->scaling == SANGAM_ROPE_NTK ? d->base * std::pow(s, double(R) / (R - 2)) : d->base;
    for (int j = 0; j < R / 2; ++j) {
        double f = std::pow(b, -2.0 * j / R);
        if (d->scaling == SANGAM_ROPE_LINEAR) f /= s;
        if (yarn) {
            const double g = d->scaling == SANGAM_ROPE_YARN_INDEX ? (hi > lo ? (hi - j) / (hi - lo) : j <= lo ? 1.0 : 0.0)
                                                                  : (d->original_len * f / two_pi - d->beta_slow) / (d->beta_fast - d->beta_slow);
            const double kept = std::fmin(1.0, std::fmax(0.0, g));
            f = kept * f + (1.0 - kept) * f / s;
        }
        turns[j] = f / two_pi;
    }
    return SANGAM_OK;
}

}  // namespace

extern "C" sangam_status sangam_rope_plan(const sangam_rope_desc* d, void* plan_buf, size_t cap, size_t* used) {
    return entry([&] { return rope_plan(d, plan_buf, cap, used); });
}
