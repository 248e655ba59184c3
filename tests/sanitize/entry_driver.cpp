// The body of a C entry (entry.h) that throws, also while the message is set.
#include <cstdio>
#include <new>
#include <stdexcept>
#include <string>

#include "../../paper_2607_04206_amd/csrc/entry.h"

namespace sangam {
static std::string g_error;
static bool g_full = false;
void set_error(const std::string& msg) {
    if (g_full) throw std::bad_alloc();
    g_error = msg;
}
}  // namespace sangam

int main() {
    using namespace sangam;
    int failed = 0;
    failed += entry([]() -> sangam_status { return SANGAM_ERR_ALIGN; }) != SANGAM_ERR_ALIGN || !g_error.empty();
    failed += entry([]() -> sangam_status { throw std::bad_alloc(); }) != -9 || g_error.empty();
    g_error.clear();
    failed += entry([]() -> sangam_status { throw std::length_error("x"); }) != -9 || g_error.empty();
    g_full = true;
    failed += entry([]() -> sangam_status { throw std::bad_alloc(); }) != -9;
    std::printf("%d failed checks\n", failed);
    return failed;
}
