// What a workgroup streams: "T V D kind K" on a line in, "forward waves over streamed blocks, tiles a workgroup; the same of the
// gradient; whether the forward lays the table out" on a line out.  kind + 4: the table is in 16 bits at a whole depth.
#include "../../paper_2511_13645_amd/csrc/fsa_class.h"

#include <cstdio>

int main() {
    long long T, V, D;
    int kind, K;
    while (std::scanf("%lld %lld %lld %d %d", &T, &V, &D, &kind, &K) == 5) {
        const fsa::ClassShape s{T, V, D, kind & 3, K};
        const fsa::ClassCut f = fsa::forward_cut(s), g = fsa::gradient_cut(s);
        const fsa::ClassPlan p = fsa::plan_of(s, kind & 4, true, true, false);
        std::printf("%d %lld %d %lld %d\n", f.wy, (long long)(f.tiles / f.parts), g.wy, (long long)(g.tiles / g.parts), (int)p.packed);
    }
}
