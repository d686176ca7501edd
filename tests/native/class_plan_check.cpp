// The plan of the class losses (csrc/fsa_class.h), for many shapes: every streamed tile belongs to one part, every held
// block to one workgroup, a launch's pieces fit what the kernels keep of them, and the workspace's areas follow each other.
#include "../../paper_2511_13645_amd/csrc/fsa_class.h"

#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#define CHECK(x) do { if (!(x)) { std::printf("%s: T %lld V %lld D %lld kind %d K %d\n", #x, (long long)s.T, (long long)s.V, (long long)s.D, s.kind, s.K); std::exit(1); } } while (0)

static void check_cut(const fsa::ClassShape& s, const fsa::ClassCut& c, int64_t held, int64_t streamed) {
    const int depth = fsa::class_depth(s.D);
    const int64_t rows = fsa::narrow_depth(depth) ? fsa::blocks_per_tile(c.wy, depth, s.kind) * fsa::kBlock : fsa::kBlock;
    CHECK(c.groups * c.wx * fsa::kBlock >= held && (held == 0 || (c.groups - 1) * c.wx * fsa::kBlock < held));
    CHECK(c.tiles * rows >= streamed && (c.tiles == 0 || (c.tiles - 1) * rows < streamed));
    CHECK(c.parts >= 1 && (c.parts <= c.tiles || c.parts == 1) && c.groups * c.parts < (int64_t)1 << 24);
    if (held == 0) return;
    int64_t next = 0;
    for (int64_t p = 0; p < c.parts; ++p) {
        const auto at = c.place((unsigned)((c.groups - 1) * c.parts + p));
        CHECK(at.part == p && at.group == c.groups - 1 && at.first == next && at.last >= at.first);
        next = at.last;
    }
    CHECK(next == c.tiles);
}

int main() {
    const int64_t sizes[] = {0, 1, 2, 31, 32, 33, 64, 65, 96, 127, 128, 129, 257, 1000, 4096, 5000, 65536, 169343, 1 << 20, 2500000, 1 << 23};
    const int64_t classes[] = {1, 2, 47, 128, 129, 10000, 169343, 2500000, 1 << 27};
    const int64_t depths[] = {1, 64, 65, 128, 129, 256, 257, 384, 602, 640, 641, 1024};
    for (int64_t T : sizes) for (int64_t V : classes) for (int64_t D : depths) for (int kind = 0; kind < 3; ++kind) for (int K : std::initializer_list<int>{1, 7, 64}) {
        const fsa::ClassShape s{T, V, D, kind, K};
        const fsa::ClassCut f = fsa::forward_cut(s), g = fsa::gradient_cut(s);
        check_cut(s, f, T, V);
        check_cut(s, g, V, T);
        CHECK(f.slices() <= 4096);                                            // class_finish_kernel's weights
        CHECK(fsa::forward_packs(s, true) == false);
        CHECK(f.wy == 1 || !fsa::forward_packs(s, false));                    // planes are only streamed by wy == 1
        const fsa::ClassBuckets b = fsa::buckets_of(V, K);
        CHECK(b.count <= fsa::kMostBuckets && b.count * b.per >= fsa::ceil_div(V, fsa::kBlock) && (b.count - 1) * b.per < fsa::ceil_div(V, fsa::kBlock));
        for (int what = 0; what < 16; ++what) {
            const fsa::ClassPlan p = fsa::plan_of(s, what & 1, what & 2, what & 4, what & 8), q = fsa::plan_of(s, false, what & 2, what & 4, what & 8);
            CHECK(p.bytes <= q.bytes);                                        // the size that callers are told covers both
        }
    }
    std::printf("ok\n");
    return 0;
}
