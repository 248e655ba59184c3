// Drives the host planner of rotary positions over random and malformed
// descriptors, each plan into a buffer of exactly its size.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <random>
#include <string>
#include <vector>

#include "../../include/sangam_rope.h"

namespace sangam {
static std::string g_error;
void set_error(const std::string& msg) { g_error = msg; }
void clear_error() { g_error.clear(); }
}  // namespace sangam

int main(int argc, char** argv) {
    std::mt19937_64 rng(argc > 1 ? std::strtoull(argv[1], nullptr, 10) : 1);
    const double odd[] = {0.0, -1.0, 1.0, 0.5, 1e300, std::numeric_limits<double>::infinity(), std::numeric_limits<double>::quiet_NaN()};
    int accepted = 0, refused = 0, failed = 0;
    auto pick = [&](double usual) { return rng() % 6 == 0 ? odd[rng() % 7] : usual; };
    for (int k = 0; k < 20000; ++k) {
        sangam_rope_desc d{};
        d.rot_dim = int32_t(rng() % 8 == 0 ? rng() : rng() % 600);
        d.interleaved = int32_t(rng() % 8 == 0 ? rng() : rng() % 2);
        d.scaling = int32_t(rng() % 8 == 0 ? rng() : rng() % 4);
        d.base = pick(10000.0);
        d.factor = pick(8.0);
        d.original_len = pick(4096.0);
        d.beta_fast = pick(32.0);
        d.beta_slow = pick(1.0);
        d.magnitude = pick(0.0);
        size_t used = 7;
        const sangam_status want = sangam_rope_plan(&d, nullptr, 0, &used);
        if (want == SANGAM_ERR_INVALID_ARG) {
            failed += used != 0 || sangam::g_error.empty();
            ++refused;
            continue;
        }
        failed += want != SANGAM_ERR_BUFFER;
        std::vector<unsigned char> buf(used);
        size_t again = 0;
        failed += sangam_rope_plan(&d, buf.data(), used - 1, &again) != SANGAM_ERR_BUFFER || again != used;
        failed += sangam_rope_plan(&d, buf.data(), used, &again) != SANGAM_OK || again != used || !sangam::g_error.empty();
        for (int j = 0; j < d.rot_dim / 2; ++j) {
            double t;
            std::memcpy(&t, buf.data() + 256 + 8 * j, 8);
            failed += !(t > 0.0 && t <= 0.16);  // at most a radian a position
        }
        ++accepted;
    }
    std::printf("%d accepted, %d refused, %d failed checks\n", accepted, refused, failed);
    return failed != 0;
}
