// Workgroups of the norm's backward (norm_parts of csrc/fsa_block.h): one round of the chip at 16 waves a CU, whatever a row takes.
#include "../../paper_2511_13645_amd/csrc/fsa_block.h"

#include <cstdio>
#include <initializer_list>

using namespace fsa;

int main() {
    for (int elem : {2, 4})
        for (int64_t D = 1; D <= kNormDmax; D += D < 5000 ? 1 : 61)
            for (int64_t T : {0, 1, 5, 1000, 4099, 65536, 1 << 30}) {
                const int64_t parts = norm_parts(T, D, elem), waves = parts * norm_plan(D, elem).threads / 64;
                if (parts >= 1 && waves <= 16 * kChip && parts * norm_plan(D, elem).rows < T + norm_plan(D, elem).rows + 1) continue;
                std::printf("%lld x %lld, elements of %d bytes: %lld parts\n", (long long)T, (long long)D, elem, (long long)parts);
                return 1;
            }
    std::puts("ok");
}
