// When a launch's last workgroup ends, as the plans of the block's products estimate it (makespan of csrc/fsa_block.h): never before the
// chip could have done all of them, whichever job has how many workgroups, and near what dealing them out one by one gives; and the
// tiles that follow from it for products of many tiles.
#include "../../paper_2511_13645_amd/csrc/fsa_block.h"

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <queue>
#include <random>
#include <vector>

using namespace fsa;

static void fail(const char* what, int count, const int64_t* groups, const double* length, double got, double want) {
    std::printf("%s: %g, wanted %g of", what, got, want);
    for (int j = 0; j < count; ++j) std::printf(" %lld x %g", (long long)groups[j], length[j]);
    std::printf("\n");
    std::exit(1);
}

// The longest first, each to the CU that is free first.
static double dealt(int count, const int64_t* groups, const double* length) {
    std::priority_queue<double, std::vector<double>, std::greater<double>> cus;
    for (int i = 0; i < kChip; ++i) cus.push(0.0);
    std::vector<int> order(count);
    for (int j = 0; j < count; ++j) order[j] = j;
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return length[a] > length[b]; });
    double last = 0.0;
    for (int j : order)
        for (int64_t i = 0; i < groups[j]; ++i) {
            const double at = cus.top() + length[j];
            cus.pop();
            cus.push(at);
            last = std::max(last, at);
        }
    return last;
}

static int tile_of_backward(int64_t T, int64_t D, int64_t H, int64_t O, int kind) { return gated_plan({T, D, H, O, kind}, true, true, 0).products.choice; }

int main() {
    std::mt19937_64 rng(1);
    for (int round = 0; round < 3000; ++round) {
        const int count = 1 + (int)(rng() % kMostJobs);
        int64_t groups[kMostJobs];
        double length[kMostJobs], work = 0.0, longest = 0.0;
        for (int j = 0; j < count; ++j) {
            groups[j] = (int64_t)std::exp2((double)(rng() % 1700) / 100.0);             // up to 131000, on either side of 64 a CU
            length[j] = 1.0 + (double)(rng() % 1000) / 10.0;
            work += (double)groups[j] * length[j];
            longest = std::max(longest, length[j]);
        }
        const double got = makespan(count, groups, length);
        if (got < work / kChip * (1.0 - 1e-9)) fail("sooner than all CUs together", count, groups, length, got, work / kChip);
        if (round % 10) continue;
        const double want = dealt(count, groups, length);
        // (a job of more than 64 a CU is taken to end with one more of its workgroups)
        if (got < want - longest - 1e-6 || got > want + count * longest + 1e-6) fail("far from what dealing out gives", count, groups, length, got, want);
    }
    // Gradients of so many tiles that the smallest fill the chip a hundred times: the largest have twice their rate.
    for (int kind = 0; kind < 3; ++kind) {
        if (tile_of_backward(65536, 4096, 16384, 4096, kind) != 2) { std::printf("65536 x 4096 -> 16384, kind %d\n", kind); return 1; }
        if (tile_of_backward(32768, 8192, 32768, 8192, kind) != 2) { std::printf("32768 x 8192 -> 32768, kind %d\n", kind); return 1; }
    }
    for (int64_t T : {2048, 4096})
        if (tile_of_backward(T, 8192, 28672, 8192, 0) != 2) { std::printf("%lld x 8192 -> 28672\n", (long long)T); return 1; }
    std::puts("ok");
}
