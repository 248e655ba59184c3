// Sums that do not hang on the order of what is added. Host and device code.
#pragma once

#include <stdint.h>

#include "mixed_order.h"

namespace sangam {

// Up to 2^18 numbers from 0 to 64 (not 64 itself), as whole numbers of 2^-38 and, of what is left of
// each, of 2^-83: both sums fit 64 bits. A number is added with an error of 2^-84, and nothing else is rounded.
struct ExactSum {
    uint64_t high, low;
    SANGAM_HD void add(double x) {
        constexpr double kWhole = 0x1p52, kSigned = 0x1.8p52;  // a sum with them ends in a whole number
        const double units = x * 0x1p38, whole = units + kWhole, rest = (units - (whole - kWhole)) * 0x1p45 + kSigned;
        high += bits(whole) - bits(kWhole);
        low += bits(rest) - bits(kSigned);  // (of either sign, modulo 2^64)
    }
    SANGAM_HD double value() const { return double(high) * 0x1p-38 + double(int64_t(low)) * 0x1p-83; }

  private:
    SANGAM_HD static uint64_t bits(double x) { return __builtin_bit_cast(uint64_t, x); }
};

}  // namespace sangam
