// The block between a mean and its loss (residual norm, gated feed-forward) and the orthogonalised update of its matrices: the
// launch interface between the C ABI (fsa_block_api.hip) and the kernel files, and the arithmetic of the plans that both
// follow.  Plain C++.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace fsa {

constexpr int64_t up_to(int64_t n, int64_t grid) { return (n + grid - 1) / grid * grid; }
constexpr int64_t cut_into(int64_t n, int64_t piece) { return (n + piece - 1) / piece; }
constexpr int64_t kChip = 256;                          // CUs

// ---------------------------------------------------------------------------------------------------------------
// norm
// ---------------------------------------------------------------------------------------------------------------
// A row is held by `lanes` lanes, at most 16 elements to each, in one of two or three lengths.
constexpr int kNormLanes[] = {4, 16, 64, 256, 1024};
constexpr int64_t kNormDmax = 16384;
constexpr int kNormParts = 1024;                        // most workgroups of the backward, one part of grad_weight each

struct NormPlan {
    int lanes, pieces;                                  // 16-byte pieces a lane
    int threads, rows;                                  // of a workgroup, and how many rows it has at a time
};
inline NormPlan norm_plan(int64_t D, int elem) {
    NormPlan p{};
    const int per = 16 / elem;
    for (int l : kNormLanes)
        if (D <= (int64_t)l * 16) { p.lanes = l; break; }
    p.pieces = (int)cut_into(cut_into(D, per), p.lanes);
    if (p.pieces == 3) p.pieces = 4;
    p.threads = p.lanes > 256 ? p.lanes : 256;
    p.rows = p.threads / p.lanes;
    return p;
}
// Workgroups of the backward: about four turns of rows each, so that a part of grad_weight is worth its writing, and no more than the
// chip holds at a time, 16 waves a CU: 1024 of 256 lanes, or 256 of 1024, to rows of more than 4096 elements (1024 of those are four rounds
// and four times the parts: 4096 x 16384 bfloat16 168 us rather than 124, 16384 x 5000 fp16 197 and 181).
inline int64_t norm_parts(int64_t T, int64_t D, int elem) {
    const int64_t turns = cut_into(T, norm_plan(D, elem).rows);
    const int64_t want = cut_into(turns, 4);
    const int64_t most = (int64_t)kNormParts * 256 / norm_plan(D, elem).threads;
    return want < 1 ? 1 : want < most ? want : most;
}

struct NormArgs {
    const void *x, *residual, *weight;                  // backward: x is the sum
    const void *grad_y, *grad_s;
    void *y, *s;                                        // backward: y is grad_x
    void* grad_weight;
    float* parts;
    int64_t x_stride, residual_stride, T, D;
    int kind, weight_kind;
    float eps;
};

// ---------------------------------------------------------------------------------------------------------------
// gated feed-forward
// ---------------------------------------------------------------------------------------------------------------
//   hidden     g, u = x [Wg; Wu]^T side by side, h = act(g) u
//   answer     y = h Wd^T
//   slopes     dh = gy Wd, g and u once more: h, dg, du
//   gradients  dx = dg Wg + du Wu,  dWd = gy^T h,  dWg = dg^T x, dWu = du^T x
// Operands are read in place where they lie on the 16-byte grid in rows of a multiple of 8 16-bit elements; others, and all of
// fp32, are laid out as planes first.
struct GatedShape {
    int64_t T, D, H, O;
    int kind;                                           // 0 fp32, 1 bfloat16, 2 fp16
    bool fine = false;                                  // two planes between the products whatever the sizes
};
constexpr int planes_of_kind(int kind) { return kind == 0 ? 3 : 1; }
// fp16 holds h, dg and du beside powers of two that bring what they may be at most near the end of its range: a product of the largest
// lengths of rows (x, both tables, grad_y) and columns (w_down), for which so many workgroups look.
constexpr int kGatedPeaks = 256;
enum { kPeakX, kPeakGate, kPeakUp, kPeakGradY, kPeakDown, kPeakKinds };

// Tiles that a product may be cut into, with the rate that each reached (TFLOP/s of 16-bit products, 8192 x 4096 x 4096).  `alone`: ns
// that 1 of the depth takes a workgroup that no other keeps company, by its chain of requests, reads and products.  What is made
// of them by estimate: the plan that cut_products, cut_pairs or ortho_plan thinks the quickest, all sizes alike.
struct TileChoice { int m, n; double rate, alone; };
constexpr int kTileKinds = 3;
constexpr TileChoice kTilesOne[kTileKinds] = {{64, 64, 700, 8}, {128, 128, 980, 10}, {256, 256, 1300, 26}};
constexpr TileChoice kTilesThree[kTileKinds] = {{64, 64, 950, 16}, {128, 64, 1150, 22}, {256, 128, 1390, 72}};
constexpr const TileChoice& product_tile(int kind, int choice) { return kind == 0 ? kTilesThree[choice] : kTilesOne[choice]; }
// The same of the pairs of products of the hidden rows: columns of each.
constexpr TileChoice kPairsOne[kTileKinds] = {{64, 64, 700, 10}, {128, 64, 900, 10}, {256, 128, 1250, 26}};
constexpr TileChoice kPairsThree[kTileKinds] = {{64, 64, 900, 25}, {128, 64, 1100, 45}, {256, 64, 1300, 72}};
constexpr TileChoice kSlopesOne[kTileKinds] = {{64, 64, 700, 10}, {128, 64, 900, 10}, {128, 128, 1000, 16}};
constexpr const TileChoice& pair_tile(int kind, int choice, bool slopes) {
    return kind == 0 ? kPairsThree[choice] : slopes ? kSlopesOne[choice] : kPairsOne[choice];
}
constexpr int64_t kMostGroups = (1 << 23) - 1;          // workgroups of up to 512: a launch has less than 2^32 threads
constexpr double kTurn = 2.0;                           // us that a workgroup takes besides its products: first reads, writing out
constexpr double kJoin = 4.0;                           // and a second launch

// Products that one launch makes: `copies` of M x N over a depth K, in `splits` shares of the depth.
constexpr int kMostJobs = 3;
struct ProductJob {
    int64_t M, N, K, copies, splits;
    int64_t joined() const { return splits > 1 ? copies * M * up_to(N, 8) : 0; }        // elements that a second launch joins
    int64_t parts_bytes() const { return joined() * splits * 4; }
};
struct ProductCut {
    int choice, count;
    ProductJob job[kMostJobs];
};
// When the last of the chip's CUs is done with `count` jobs' workgroups, `groups[j]` of length `length[j]`, the longest first, each
// given to the CU that is free first.
struct Load { int64_t cus; double at; };
inline double makespan(int count, const int64_t* groups, const double* length) {
    constexpr int kMost = 16;
    Load load[kMost] = {{kChip, 0.0}};
    int n = 1;                                          // loads in order, the least first
    bool done[kMostJobs] = {};
    for (int k = 0; k < count; ++k) {
        int j = -1;
        for (int i = 0; i < count; ++i) if (!done[i] && (j < 0 || length[i] > length[j])) j = i;
        done[j] = true;
        int64_t left = groups[j];
        if (left > 64 * kChip) {                        // many: they even out what was before them
            load[0] = {kChip, load[n - 1].at + ((double)left / kChip + 1.0) * length[j]};
            n = 1;
            continue;
        }
        while (left > 0) {
            Load take = load[0];
            if (left < take.cus) { load[0].cus -= left; take.cus = left; }
            else { --n; for (int i = 0; i < n; ++i) load[i] = load[i + 1]; }
            left -= take.cus;
            take.at += length[j];
            int i = n;
            for (; i > 0 && load[i - 1].at > take.at; --i) ;
            if (i > 0 && load[i - 1].at == take.at) load[i - 1].cus += take.cus;
            else if (n == kMost) return 1e30;           // (never: a job leaves at most two loads more than it found)
            else { for (int q = n; q > i; --q) load[q] = load[q - 1]; load[i] = take; ++n; }
        }
    }
    return load[n - 1].at;
}
// The tile and the shares that are estimated to take the least time: depths cut into shares of about one length, or one job's
// alone in two; parts of a split product are written and read once more.
inline ProductCut cut_products(int kind, ProductCut want) {
    ProductCut best = want;
    double least = 1e30;
    const double each = kind == 0 ? 6.0 : 1.0;
    for (int choice = 0; choice < kTileKinds; ++choice) {
        const TileChoice& tile = product_tile(kind, choice);
        const double depth_us = 2.0 * tile.m * tile.n * each / (tile.rate / kChip) * 1e-6;          // a workgroup's step of one
        int64_t tiles[kMostJobs];
        double work = 0.0;
        for (int j = 0; j < want.count; ++j) {
            tiles[j] = cut_into(want.job[j].M, tile.m) * cut_into(want.job[j].N, tile.n) * want.job[j].copies;
            work += (double)tiles[j] * (double)want.job[j].K;
        }
        for (int way = 0; way < 5 + want.count; ++way) { // whole, shares of 1, 1/2, 1/3, 1/4 of a CU's work, one job's halves
            ProductCut c = want;
            c.choice = choice;
            double share = way >= 1 && way < 5 ? work / (double)(kChip * way) : 1e30, bytes = 0.0, us[kMostJobs], longest = 0.0;
            if (share < 128.0) share = 128.0;
            int64_t groups[kMostJobs], all = 0, joined = 0;
            for (int j = 0; j < c.count; ++j) {
                ProductJob& job = c.job[j];
                const double n = (double)job.K / share + 0.5;
                job.splits = way - 5 == j ? 2 : n > 64.0 ? 64 : n < 1.0 ? 1 : (int64_t)n;
                groups[j] = tiles[j] * job.splits;
                all += groups[j];
                us[j] = (double)job.K / (double)job.splits * depth_us + kTurn;
                const double alone = (double)job.K / (double)job.splits * tile.alone * 1e-3 + kTurn;
                longest = alone > longest ? alone : longest;
                joined += job.joined();
                bytes += (double)job.parts_bytes();
            }
            if ((all > kMostGroups || joined / 4 > kMostGroups * 256) && (way > 0 || choice + 1 < kTileKinds)) continue;
            const double span = makespan(c.count, groups, us);
            const double total = (span > longest ? span : longest) + (bytes > 0.0 ? kJoin + bytes * 2.0 / 4e6 : 0.0);
            if (total < least) { least = total; best = c; }
        }
    }
    return best;
}
enum { kHiddenPass, kSlopesPass, kKeptPass };
inline int cut_pairs(int kind, int64_t T, int64_t H, int64_t depth, int pass) {
    int best = 0;
    double least = 1e30;
    for (int choice = 0; choice < kTileKinds; ++choice) {
        const TileChoice& tile = pass == kKeptPass ? product_tile(kind, choice) : pair_tile(kind, choice, pass == kSlopesPass);
        const double one = 2.0 * tile.m * tile.n * (double)depth * (kind == 0 ? 6.0 : 1.0) / (tile.rate / kChip) * 1e-6 + kTurn;
        double us = (double)cut_into(cut_into(T, tile.m) * cut_into(H, tile.n), kChip) * one;
        if (const double alone = (double)depth * tile.alone * 1e-3 + kTurn; alone > us) us = alone;
        if (cut_into(T, tile.m) * cut_into(H, tile.n) > kMostGroups && choice + 1 < kTileKinds) continue;
        if (us < least) { least = us; best = choice; }
    }
    return best;
}

// Whether h, dg and du are held with what their rounding to 16 bits leaves, as a second plane: results are off by their own rounding
// alone, and their products take twice as long, which is less than the launches of a pass up to about this many operations
// (1024 x 128 -> 512 -> 128, bfloat16: 4 us of 90).  Few rows are bound by the tables, and have h in two planes where nothing is kept:
// an answer is as exact whether its gradient is wanted or not.  In larger calls it is the caller's choice.
inline bool gated_few(const GatedShape& s);
inline bool gated_fine(const GatedShape& s) {
    return s.kind != 0 && (s.fine || gated_few(s) || 6.0 * (double)s.T * (double)s.H * (double)(2 * s.D + s.O) < 4e9);
}
inline int gated_planes(const GatedShape& s) { return s.kind == 0 ? 3 : gated_fine(s) ? 2 : 1; }

// A forward of few rows is bound by its reading of the tables: waves read them straight into registers, h is fp32.
inline bool gated_few(const GatedShape& s) { return s.T <= (s.kind == 0 ? 32 : 16); }

// Whether a forward whose backward follows keeps g, u and h rather than that they are made again: some 10 bytes of traffic an
// element (16 in fp32) against 4 D operations (of six products each in fp32), in a kernel of its own tiles.  Forward and backward
// of T x D -> 4 D -> D, made again and kept, us: bfloat16, T 32768: D 256 323 and 331, 384 605 and 598, 768 2000 and 1724; fp32:
// D 64 178 and 185, 128 444 and 415, 512 4329 and 3696.
inline bool gated_keep_pays(const GatedShape& s) { return s.D >= (s.kind == 0 ? 128 : 384); }

// What it keeps, as byte offsets.  h lies in rows of H8 elements, g and u in blocks of 16 x 32 (see kept_at), which is what a wave
// writes or reads at a time.  g and u are fp32, or the upper 24 bits of it, rounded, beside 16-bit tables: the upper 16 in one
// array, the next 8 in another.  Those are 2^-17 of an element, where what is made of it is rounded to 2^-9 or 2^-12.
struct KeptPlan { size_t g, u, g_low, u_low, h, bytes; };
constexpr int64_t kKeptRows = 16, kKeptCols = 32;
constexpr int64_t kept_at(int64_t m, int64_t n, int64_t across) {           // element (m, n), `across` blocks side by side
    return (m / kKeptRows * across + n / kKeptCols) * kKeptRows * kKeptCols + m % kKeptRows * kKeptCols + n % kKeptCols;
}
inline KeptPlan kept_plan(const GatedShape& s) {
    KeptPlan k{};
    size_t at = 0;
    const int64_t n = up_to(s.T, kKeptRows) * up_to(s.H, kKeptCols);
    auto room = [&at](int64_t bytes) { const size_t a = at; at += (size_t)up_to(bytes, 256); return a; };
    k.g = room(n * (s.kind == 0 ? 4 : 2));
    k.u = room(n * (s.kind == 0 ? 4 : 2));
    if (s.kind != 0) { k.g_low = room(n); k.u_low = room(n); }
    k.h = room(s.T * up_to(s.H, 8) * 2 * gated_planes(s));
    k.bytes = at;
    return k;
}

// Byte offsets into the caller's workspace.
struct GatedPlan {
    size_t x, gate, up, down, grad_y;                   // laid out operands
    size_t h, dg, du, peaks, parts, bytes;
    int64_t D8, H8, O8;
    int planes;                                         // of h, dg and du
    int pairs, slopes;                                  // choices of tiles
    ProductCut products;
};
// `packs`: bits x, gate, up, down, grad_y of operands that are laid out.  `kept`: the backward is given g and u.  Products of the
// backward are cut as if all were wanted, so that room for them does not depend on which are.
enum { kJobGates, kJobDown, kJobX };
inline GatedPlan gated_plan(const GatedShape& s, bool backward, bool kept, int packs) {
    GatedPlan p{};
    size_t at = 0;
    auto room = [&at](int64_t n) { const size_t a = at; at += (size_t)up_to(n, 256); return a; };
    p.D8 = up_to(s.D, 8); p.H8 = up_to(s.H, 8); p.O8 = up_to(s.O, 8);
    p.planes = gated_planes(s);
    const int64_t planes = 2 * planes_of_kind(s.kind), own = s.T * p.H8 * 2 * p.planes;             // bytes
    if (packs & 1) p.x = room(s.T * p.D8 * planes);
    if (packs & 2) p.gate = room(s.H * p.D8 * planes);
    if (packs & 4) p.up = room(s.H * p.D8 * planes);
    if (packs & 8) p.down = room(s.O * p.H8 * planes);
    p.h = room(!backward && gated_few(s) && own < s.T * s.H * 4 ? s.T * s.H * 4 : own);
    const int64_t few = gated_few(s) ? cut_into(s.H, 16) : 0;          // of few rows the largest |h| of each workgroup's
    if (s.kind == 2 && !backward) p.peaks = room((few > kPeakKinds * kGatedPeaks ? few : kPeakKinds * kGatedPeaks) * 4);
    const int64_t sums = s.kind != 0 ? p.planes : 1;    // products that make one, of h's, dg's or du's planes
    ProductCut want{};
    if (!backward) {
        p.pairs = cut_pairs(s.kind, s.T, s.H, 2 * s.D, kHiddenPass);
        want.job[want.count++] = {s.T, s.O, sums * s.H, 1, 1};
    } else {
        if (packs & 16) p.grad_y = room(s.T * p.O8 * planes);
        p.dg = room(own);
        p.du = room(own);
        p.peaks = room(kPeakKinds * kGatedPeaks * 4);
        p.slopes = cut_pairs(s.kind, s.T, s.H, (kept ? 0 : 2 * s.D) + s.O, kept ? kKeptPass : kSlopesPass);
        want.count = 3;
        want.job[kJobGates] = {s.H, s.D, sums * s.T, 2, 1};
        want.job[kJobDown] = {s.O, s.H, sums * s.T, 1, 1};
        want.job[kJobX] = {s.T, s.D, 2 * sums * s.H, 1, 1};
    }
    p.products = cut_products(s.kind, want);
    int64_t parts = 0;
    for (int j = 0; j < p.products.count; ++j) parts += up_to(p.products.job[j].parts_bytes(), 256);
    p.parts = room(parts);
    p.bytes = at;
    return p;
}

struct Matrix {                                         // as a caller has it
    const void* p;
    int64_t stride, rows, cols;
};
struct GatedArgs {
    GatedShape s;
    int activation;
    Matrix x, gate, up, down, grad_y;
    void *y, *grad_x, *grad_gate, *grad_up, *grad_down; // contiguous
    char* kept;                                         // forward: written if not null; backward: read
    GatedPlan plan;
    int packs;
    char* ws;
};

// ---------------------------------------------------------------------------------------------------------------
// orthogonalised updates
// ---------------------------------------------------------------------------------------------------------------
// X [m,n] with m <= n (the transpose of a tall matrix): two fp16 planes of X 2^13, likewise A = X X^T and P = b A + c A^2 of
// which planes hold A 2^13 and P 2^10; a step whose singular values may grow so far that one of them would not fit has it at a lower power.
constexpr int kMostSteps = 32;
constexpr int kOrthoPeaks = 256;                        // workgroups a matrix that sum its squares
constexpr int kUnitX = 13, kUnitA = 13, kUnitP = 10, kLeastUnit = -110;
constexpr double kMostHeld = 65504.0 / 1.02;            // of a plane, with room for what the sums are off by

// No singular value of the first X is above one, and a step takes s to p(s) = a s + b s^3 + c s^5: what X, A = X X^T and P may have at
// most follows from the coefficients alone, as the largest |b t + c t^2| and |p| over t = s^2 from 0 to the square of the largest s, at
// an end or where their derivative is zero.  No element of a matrix is larger than its largest singular value.
struct OrthoReach {
    double poly, next;                                  // the largest |P| of a step, and the largest singular value after it
};
inline OrthoReach ortho_reach(const float* abc, double reach) {
    const double a = abc[0], b = abc[1], c = abc[2], end = reach * reach;
    OrthoReach r{0.0, 0.0};
    auto at = [&](double t) {
        if (!(t >= 0.0 && t <= end)) return;
        const double poly = b * t + c * t * t, next = __builtin_sqrt(t) * (a + poly);
        if (!(poly <= r.poly && -poly <= r.poly)) r.poly = poly < 0.0 ? -poly : poly;
        if (!(next <= r.next && -next <= r.next)) r.next = next < 0.0 ? -next : next;
    };
    at(end);
    if (c != 0.0) at(-b / (2.0 * c));
    if (const double root = 9.0 * b * b - 20.0 * a * c; root >= 0.0) {      // a + 3 b t + 5 c t^2 = 0
        const double q = -0.5 * (3.0 * b + (b < 0.0 ? -1.0 : 1.0) * __builtin_sqrt(root));
        if (c != 0.0) at(q / (5.0 * c));
        if (q != 0.0) at(a / q);
    }
    return r;
}
// The power of two at which planes hold what is `reach` at most.
inline int ortho_unit(double reach, int most) {
    int unit = most;
    double held = reach;
    for (int i = 0; i < most; ++i) held *= 2.0;
    while (unit > kLeastUnit && !(held <= kMostHeld)) { held *= 0.5; --unit; }
    return unit;
}
struct OrthoUnits { int x, a, p; };                     // of a step: of the X that it takes, and of its A and P
// Coefficients above `plain` are taken where singular values stay below 8 after every step.
inline bool ortho_units(const float* coefficients, int steps, double plain, OrthoUnits* units) {
    double reach = 1.0;
    bool small = true, near = true;
    for (int i = 0; i < steps; ++i) {
        const float* abc = coefficients + 3 * i;
        for (int j = 0; j < 3; ++j) {
            if (!(abc[j] <= 1024.0f && abc[j] >= -1024.0f)) return false;
            small = small && abc[j] <= plain && abc[j] >= -plain;
        }
        const OrthoReach r = ortho_reach(abc, reach);
        units[i] = {ortho_unit(reach, kUnitX), ortho_unit(reach * reach, kUnitA), ortho_unit(r.poly, kUnitP)};
        reach = r.next;
        near = near && reach <= 8.0;
    }
    return small || near;
}

struct OrthoShape {
    int64_t B, M, N;
    int kind;
};
constexpr TileChoice kTilesTwo[kTileKinds] = {{64, 64, 860, 10}, {128, 128, 1150, 22}, {256, 256, 1400, 72}};
struct OrthoPlan {
    size_t squares, x[2], a, p, parts, bytes;
    int64_t m, n, m8, n8;
    int gram, poly, update;                             // choices of tiles
    int64_t splits;                                     // of the gram matrix' depth: then half of its tiles are made, and joined
};
constexpr int64_t upper_tiles(int64_t m, int tile) { return cut_into(m, tile) * (cut_into(m, tile) + 1) / 2; }
inline double ortho_us(int choice, int64_t tiles, int64_t depth) {
    const TileChoice& t = kTilesTwo[choice];
    const double alone = (double)depth * t.alone * 1e-3 + kTurn;
    const double us = (double)cut_into(tiles, kChip) * (2.0 * t.m * t.n * 3.0 * (double)depth / (t.rate / kChip) * 1e-6 + kTurn);
    return us > alone ? us : alone;
}
inline OrthoPlan ortho_plan(const OrthoShape& s) {
    OrthoPlan p{};
    size_t at = 0;
    auto room = [&at](int64_t n) { const size_t a = at; at += (size_t)up_to(n, 256); return a; };
    p.m = s.M < s.N ? s.M : s.N;
    p.n = s.M < s.N ? s.N : s.M;
    p.m8 = up_to(p.m, 8); p.n8 = up_to(p.n, 8);
    double gram = 1e30, poly = 1e30, update = 1e30;
    for (int c = 0; c < kTileKinds; ++c) {
        const int64_t mt = cut_into(p.m, kTilesTwo[c].m), nt = cut_into(p.n, kTilesTwo[c].n);
        double us = ortho_us(c, s.B * mt * mt, p.m);
        if (us < poly) { poly = us; p.poly = c; }
        us = ortho_us(c, s.B * mt * nt, p.m);
        if (us < update) { update = us; p.update = c; }
        us = ortho_us(c, s.B * mt * mt, p.n);
        if (us < gram) { gram = us; p.gram = c; p.splits = 1; }
        const int64_t upper = s.B * upper_tiles(p.m, kTilesTwo[c].m);
        for (int64_t splits = 2; splits <= 16 && p.n / splits >= 128; ++splits) {
            const double bytes = (double)(upper * splits) * kTilesTwo[c].m * kTilesTwo[c].n * 4.0;
            us = ortho_us(c, upper * splits, p.n / splits) + kJoin + bytes * 2.0 / 4e6;
            if (us < gram) { gram = us; p.gram = c; p.splits = splits; }
        }
    }
    p.squares = room(s.B * kOrthoPeaks * 8);
    for (size_t& x : p.x) x = room(s.B * p.m * p.n8 * 4);
    p.a = room(s.B * p.m * p.m8 * 4);
    p.p = room(s.B * p.m * p.m8 * 4);
    const TileChoice& t = kTilesTwo[p.gram];
    p.parts = room(p.splits > 1 ? s.B * upper_tiles(p.m, t.m) * p.splits * t.m * t.n * 4 : 0);
    p.bytes = at;
    return p;
}
struct OrthoArgs {
    OrthoShape s;
    const void* g;
    int64_t batch_stride, stride;
    void* out;                                          // contiguous
    float coefficients[3 * kMostSteps];
    OrthoUnits units[kMostSteps];
    int steps;
    float eps, scale;
    OrthoPlan plan;
    char* ws;
};

}  // namespace fsa
