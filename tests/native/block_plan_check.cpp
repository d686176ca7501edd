// The plans of the block's operators (csrc/fsa_block.h), for many shapes: a workspace of the size that a caller is told holds what any
// call of those sizes puts there, areas follow each other, shares of a split depth have work, launches are of a size that there is,
// what is kept has a place of its own for every element, and a row of the norm fits its lanes.
#include "../../paper_2511_13645_amd/csrc/fsa_block.h"

#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <vector>

#define CHECK(x) do { if (!(x)) { std::printf("%s: %lld %lld %lld %lld kind %d\n", #x, (long long)w[0], (long long)w[1], (long long)w[2], (long long)w[3], kind); std::exit(1); } } while (0)

using namespace fsa;

constexpr int64_t kMemory = (int64_t)288 << 30;
constexpr int64_t kMostThreads = (int64_t)1 << 32;      // of a launch in one direction

// Whether a call's operands, gradients and workspace are all there at a time.
static bool fits(const int64_t (&w)[4], int kind, size_t workspace) {
    return (w[0] * (2 * w[1] + w[3]) + w[2] * (2 * w[1] + w[3])) * (kind == 0 ? 4 : 2) + (int64_t)workspace <= kMemory;
}
static void check_products(const int64_t (&w)[4], int kind, const GatedPlan& p) {
    const TileChoice& tile = product_tile(kind, p.products.choice);
    int64_t groups = 0, joined = 0;
    for (int j = 0; j < p.products.count; ++j) {
        const ProductJob& job = p.products.job[j];
        const int64_t steps = cut_into(job.K, 32);
        CHECK(job.splits >= 1 && job.splits <= 64 && (job.splits == 1 || job.splits <= steps));
        groups += cut_into(job.M, tile.m) * cut_into(job.N, tile.n) * job.copies * job.splits;
        joined += job.joined();
    }
    CHECK(joined / 4 + 256 * p.products.count < kMostThreads);
    if (fits(w, kind, p.bytes)) CHECK(groups * (tile.m * tile.n > 8192 ? 512 : 256) < kMostThreads);
}

static void check_gated(int64_t T, int64_t D, int64_t H, int64_t O, int kind) {
    const int64_t w[4] = {T, D, H, O};
    const GatedShape s{T, D, H, O, kind};
    const size_t forward = gated_plan(s, false, false, 31).bytes, backward = gated_plan(s, true, false, 31).bytes;
    for (int packs : {0, 1, 6, 8, 9, 15, 16, 31}) {
        if (kind == 0 && (packs & 15) != 15) continue;  // (fp32 is laid out whole)
        const GatedPlan f = gated_plan(s, false, false, packs & 15);
        const TileChoice& pair = pair_tile(kind, f.pairs, false);
        if (fits(w, kind, f.bytes)) CHECK(cut_into(T, pair.m) * cut_into(H, pair.n) * 512 < kMostThreads);
        CHECK(f.bytes <= forward && f.h < f.bytes && f.parts <= f.bytes);
        CHECK(!gated_few(s) || (size_t)(T * H * 4) <= (f.parts > f.h ? f.parts : f.bytes) - f.h);
        check_products(w, kind, f);
        size_t least = 0;
        for (bool kept : {false, true}) {
            const GatedPlan b = gated_plan(s, true, kept, packs);
            CHECK(b.bytes <= backward && b.h <= b.dg && b.dg < b.du && b.du < b.peaks && b.peaks % 256 == 0 && b.parts <= b.bytes);
            CHECK(b.dg + (size_t)(T * b.H8 * 2 * b.planes) <= b.du);
            size_t at = b.parts;
            for (int j = 0; j < b.products.count; ++j) at += (size_t)up_to(b.products.job[j].parts_bytes(), 256);
            CHECK(at <= b.bytes);
            check_products(w, kind, b);
            const TileChoice& slopes = kept ? product_tile(kind, b.slopes) : pair_tile(kind, b.slopes, true);
            if (fits(w, kind, b.bytes)) CHECK(cut_into(T, slopes.m) * cut_into(H, slopes.n) * 512 < kMostThreads);
            if (!kept) least = b.bytes;
            CHECK(b.bytes == least);
        }
    }
    const KeptPlan k = kept_plan(s);
    const size_t area = (size_t)(up_to(T, kKeptRows) * up_to(H, kKeptCols));
    CHECK(k.g + area * (kind == 0 ? 4 : 2) <= k.u && k.u < k.h && k.h % 256 == 0 && k.h < k.bytes);
    CHECK(kept_at(T - 1, up_to(H, 8) - 1, cut_into(H, kKeptCols)) < (int64_t)area);
    CHECK(gated_keep_pays(s) == (D >= (kind == 0 ? 128 : 384)));
}

int main() {
    for (int kind = 0; kind < 3; ++kind) {
        for (int64_t T : {1, 2, 15, 16, 17, 33, 100, 1000, 4099, 8192, 65536, 1100000, 1 << 26})
            for (int64_t D : {1, 7, 64, 100, 128, 602, 1024, 4096, 65536})
                for (int64_t H : {1, 8, 31, 333, 512, 2048, 65536})
                    for (int64_t O : {int64_t(1), int64_t(47), D})
                        check_gated(T, D, H, O, kind);
        for (int64_t M : {1, 2, 16, 63, 64, 65, 128, 300, 602, 1024, 2047, 4096, 65536})
            for (int64_t N : {1, 3, 64, 127, 512, 1400, 4096, 65536})
                for (int64_t B : {1, 3, 70, 2200, 65535}) {
                    const int64_t w[4] = {B, M, N, 0};
                    const OrthoPlan p = ortho_plan({B, M, N, kind});
                    CHECK(p.m <= p.n && p.splits >= 1 && p.splits <= 16 && (p.splits == 1 || p.n / p.splits >= 128));
                    CHECK(p.squares + (size_t)(B * kOrthoPeaks * 8) <= p.x[0] && p.x[0] + (size_t)(B * p.m * p.n8 * 4) <= p.x[1]);
                    CHECK(p.x[1] + (size_t)(B * p.m * p.n8 * 4) <= p.a && p.a + (size_t)(B * p.m * p.m8 * 4) <= p.p);
                    CHECK(p.p + (size_t)(B * p.m * p.m8 * 4) <= p.parts && p.parts <= p.bytes);
                    const TileChoice& g = kTilesTwo[p.gram];
                    CHECK(p.splits == 1 || p.parts + (size_t)(B * upper_tiles(p.m, g.m) * p.splits * g.m * g.n * 4) <= p.bytes);
                    const TileChoice& u = kTilesTwo[p.update];
                    CHECK(cut_into(p.m, u.m) * cut_into(p.n, u.n) * 512 < kMostThreads && B < 1 << 16);
                }
        for (int64_t D = 1; D <= kNormDmax; D += D < 1100 ? 1 : 37) {
            const int64_t w[4] = {D, 0, 0, 0};
            const int elem = kind == 0 ? 4 : 2, per = 16 / elem;
            const NormPlan p = norm_plan(D, elem);
            CHECK(p.lanes > 0 && (int64_t)p.lanes * p.pieces * per >= D && p.rows * p.lanes == p.threads);
            CHECK(p.pieces == 1 || p.pieces == 2 || (p.pieces == 4 && kind == 0));
            for (int64_t T : {1, 2, 1000, 1 << 30}) CHECK(norm_parts(T, D, elem) >= 1 && norm_parts(T, D, elem) <= kNormParts);
        }
    }
    // every element that is kept has a place of its own
    for (int64_t H : {1, 31, 32, 33, 100}) {
        const int64_t T = 37, w[4] = {T, H, 0, 0};
        const int kind = 0;
        std::vector<char> seen((size_t)(up_to(T, kKeptRows) * up_to(H, kKeptCols)));
        for (int64_t m = 0; m < T; ++m) for (int64_t n = 0; n < up_to(H, 8); ++n) {
            const int64_t at = kept_at(m, n, cut_into(H, kKeptCols));
            CHECK(at >= 0 && at < (int64_t)seen.size() && !seen[(size_t)at]);
            CHECK(n % 8 == 0 || at == kept_at(m, n - 1, cut_into(H, kKeptCols)) + 1);
            seen[(size_t)at] = 1;
        }
    }
    std::puts("ok");
}
