// Which tiles the plans of the block's products choose (csrc/fsa_block.h).  A line of numbers in, a line of names out:
//   gated KIND FINE T D H O   the pass, its tile and the planes between products, of each pass of which more than one tile's rows and columns there are
//   ortho B M N               the same of an orthogonalised matrix' products
#include "../../paper_2511_13645_amd/csrc/fsa_block.h"

#include <cstdio>
#include <cstring>

using namespace fsa;

static void name(bool wide, const char* pass, const TileChoice& t) { if (wide) std::printf(" %s:%dx%d", pass, t.m, t.n); }

int main() {
    char what[16];
    while (std::scanf("%15s", what) == 1) {
        if (!std::strcmp(what, "gated")) {
            long long kind, fine, T, D, H, O;
            if (std::scanf("%lld %lld %lld %lld %lld %lld", &kind, &fine, &T, &D, &H, &O) != 6) return 1;
            const GatedShape s{T, D, H, O, (int)kind, fine != 0};
            const GatedPlan f = gated_plan(s, false, false, 15), b = gated_plan(s, true, false, 31), k = gated_plan(s, true, true, 31);
            std::printf("planes:%d", f.planes);
            const TileChoice &hidden = pair_tile(s.kind, f.pairs, false), &answer = product_tile(s.kind, f.products.choice);
            if (!gated_few(s)) {
                name(T > hidden.m && H > hidden.n, "hidden", hidden);
                name(T > answer.m && O > answer.n, f.products.job[0].splits > 1 ? "shares" : "answer", answer);
            }
            const TileChoice &slopes = pair_tile(s.kind, b.slopes, true), &kept = product_tile(s.kind, k.slopes), &grads = product_tile(s.kind, b.products.choice);
            name(T > slopes.m && H > slopes.n, "slopes", slopes);
            name(T > kept.m && H > kept.n, "kept", kept);
            name(T > grads.m && H > grads.m && H > grads.n && O > grads.m && D > grads.n, "grads", grads);
        } else {
            long long B, M, N;
            if (std::scanf("%lld %lld %lld", &B, &M, &N) != 3) return 1;
            const OrthoPlan p = ortho_plan({B, M, N, 0});
            const TileChoice &gram = kTilesTwo[p.gram], &poly = kTilesTwo[p.poly], &update = kTilesTwo[p.update];
            std::printf("%s", M > N ? "tall" : "wide");
            name(p.m > gram.m, p.splits > 1 ? "parts" : "gram", gram);
            name(p.m > poly.m, "poly", poly);
            name(p.m > update.m && p.n > update.n, "update", update);
        }
        std::puts("");
    }
}
