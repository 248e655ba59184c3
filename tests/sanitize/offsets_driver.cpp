// Looks up, for tests/test_tables.py, places among n + 1 offsets that are 0 up to
// the last, which is 5: reads "n x" lines, prints last_offset of each. The offsets
// lie in memory that is not there before it is touched.
#include <sys/mman.h>

#include <cstdio>

#include "../../paper_2607_04206_amd/csrc/offsets.h"

int main() {
    int n;
    long long x;
    while (std::scanf("%d %lld", &n, &x) == 2) {
        const size_t bytes = (size_t(n) + 1) * sizeof(int32_t);
        void* p = mmap(nullptr, bytes, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
        if (p == MAP_FAILED) return 1;
        int32_t* const offsets = static_cast<int32_t*>(p);
        offsets[n] = 5;
        std::printf("%d\n", sangam::last_offset(offsets, n, x));
        std::fflush(stdout);
        munmap(p, bytes);
    }
    return 0;
}
