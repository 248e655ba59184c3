// Sums, for tests/test_sample.py, lines of numbers with ExactSum: reads "n x1 ... xn"
// (as hexadecimal floating point), prints both whole numbers and the value.
#include <cstdio>

#include "../../paper_2607_04206_amd/csrc/exact_sum.h"

int main() {
    int n;
    while (std::scanf("%d", &n) == 1) {
        sangam::ExactSum s{};
        for (int k = 0; k < n; ++k) {
            double x;
            if (std::scanf("%la", &x) != 1) return 1;
            s.add(x);
        }
        std::printf("%llu %llu %a\n", (unsigned long long)s.high, (unsigned long long)s.low, s.value());
    }
    return 0;
}
