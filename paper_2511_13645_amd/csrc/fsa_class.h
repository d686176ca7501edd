// Losses over many classes (softmax cross entropy, distillation): the launch interface between the C ABI
// (fsa_class_api.hip) and the kernel files, and the arithmetic of the plan that both follow.  Plain C++.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace fsa {

// z[t,v] = scale * h[t] . w[v] is never kept: a launch streams one side past the other, 32 x 32 scores at a time.
//   forward    waves hold rows of h, the table streams by: running maximum and sum of every row, and where wanted the
//              running mean of the table's rows under the softmax
//   gradient   waves hold classes, the rows stream by: the scores again, their gradients, a class's gradient row
// Each splits the streamed side over `parts` of the grid, joined in part order by a second launch.
//
// Rows of up to 256 elements are held by one wave each ("narrow"); longer ones by the four waves of a workgroup, a quarter
// of the elements each ("wide"), whose partial scores meet in LDS.
constexpr int kBlock = 32;                              // rows and classes come in blocks of one matrix instruction
constexpr int kClassThreads = 256;
constexpr int kClassWaves = kClassThreads / 64;

struct ClassShape {
    int64_t T, V, D;
    int kind;                                           // 0 fp32, 1 bfloat16, 2 fp16
    int K;                                              // slots a row
};

constexpr int class_planes(int kind) { return kind == 0 ? 2 : 1; }       // 16-bit planes that hold an element
constexpr bool narrow_depth(int depth) { return depth <= 256; }
inline int class_depth(int64_t D) {                     // what rows are padded to; 0: too long
    constexpr int depths[] = {64, 128, 256, 384, 640, 1024};
    for (int d : depths) if (D <= d) return d;
    return 0;
}
constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t padded_rows(int64_t T) { return ceil_div(T, 4 * kBlock) * 4 * kBlock; }

// How one launch is cut: wx waves of a workgroup side by side over held blocks, wy over streamed ones (narrow).
struct ClassCut {
    int wx, wy;
    int64_t groups;                                     // workgroups over held blocks
    int64_t tiles;                                      // streamed tiles
    int64_t parts;                                      // shares of the streamed tiles in the grid
    constexpr int64_t slices() const { return parts * wy; }   // partial results of every held row
    // A workgroup's place in the launch and its tiles [first, last).
    struct Place { int part, group; int first, last; };
    constexpr Place place(unsigned workgroup) const {
        const unsigned p = (unsigned)parts, part = workgroup % p, each = (unsigned)tiles / p, more = (unsigned)tiles % p;
        const unsigned first = part * each + (part < more ? part : more);
        return {(int)part, (int)(workgroup / p), (int)first, (int)(first + each + (part < more ? 1 : 0))};
    }
};

// Streamed blocks of a tile: two tiles and what else a workgroup keeps fit into LDS.
constexpr int blocks_per_tile(int wy, int depth, int kind) { return depth * class_planes(kind) > 256 ? wy : wy == 4 ? 4 : 2; }

// Workgroups that the chip's 256 CUs hold at a time: two to a CU where registers and LDS allow it.
constexpr int64_t resident_workgroups(int depth, int kind) {
    return depth * class_planes(kind) <= 128 || (!narrow_depth(depth) && depth * class_planes(kind) <= 768) ? 512 : 256;
}
// As many shares of the streamed side as make one round of workgroups; where that costs little a multiple of 8, so that the
// workgroups of one share, dealt out to the 8 XCDs in turn, meet on one XCD's L2.
inline int64_t parts_for(int64_t groups, int64_t tiles, int64_t workgroups, int64_t most) {
    int64_t want = groups > 0 ? workgroups / groups : 1;           // no rows: no workgroups either
    if (want >= 8 && want / 8 * 8 * 8 >= want * 7) want = want / 8 * 8;
    if (want > most) want = most;
    if (want > tiles) want = tiles;
    return want < 1 ? 1 : want;
}
inline ClassCut cut_of(int64_t held, int64_t streamed, int depth, int kind, int64_t most_parts) {
    ClassCut c;
    const int64_t blocks = ceil_div(held, kBlock);
    if (!narrow_depth(depth)) {
        c.wx = 1; c.wy = 1;
        c.groups = blocks;
        c.tiles = ceil_div(streamed, kBlock);
        c.parts = parts_for(c.groups, c.tiles, resident_workgroups(depth, kind), most_parts);
        return c;
    }
    c.wy = blocks >= 4 ? 1 : blocks >= 2 ? 2 : 4;
    if (c.wy == 4 && depth * class_planes(kind) > 256) c.wy = 2;
    c.wx = kClassWaves / c.wy;
    c.groups = ceil_div(blocks, c.wx);
    c.tiles = ceil_div(streamed, (int64_t)blocks_per_tile(c.wy, depth, kind) * kBlock);
    c.parts = parts_for(c.groups, c.tiles, resident_workgroups(depth, kind), most_parts);
    return c;
}
inline ClassCut forward_cut(const ClassShape& s) { return cut_of(s.T, s.V, class_depth(s.D), s.kind, 1024); }
inline ClassCut gradient_cut(const ClassShape& s) {
    ClassCut c = cut_of(s.V, s.T, class_depth(s.D), s.kind, 64);
    return c;
}

// Slots of 32 rows are sorted by the classes that they name, for the gradient: `per` blocks of classes to a bucket, 16 buckets
// to a slot while they last, so that a wave mostly learns from one word that no slot of these rows names one of its classes.
struct ClassBuckets { int64_t per, count; };
constexpr int kMostBuckets = 2 * kBlock * 64;
constexpr ClassBuckets buckets_of(int64_t V, int K) {
    const int64_t blocks = ceil_div(V, kBlock), most = 16 * kBlock * K, per = ceil_div(blocks, most < kMostBuckets ? most : kMostBuckets);
    return {per, ceil_div(blocks, per)};
}

constexpr int kWaveSlots = 2;                           // slots a row that a wave of the forward sorts itself: two to a lane pair
// Whether 64 classes have more than 8 slots of 32 rows, on an average: for the forward with row gradients, which then reads the
// (small) table as it is.
constexpr bool crowded_tiles(const ClassShape& s) { return s.K > kWaveSlots && (int64_t)s.K * kBlock * 64 > 8 * s.V; }
// Whether workgroups of that forward look all their rows' slots through for every tile, or read them from a list that a launch
// ahead sorts.  2 to 6 us a tile against 10 to 21 of the launch: 51 rows x 9896 x 144 bfloat16, 62 slots, 22.4 us against 16.1 and
// 17.8; 1024 x 47 x 100 fp32, 10 slots, 18.9 against 19.4 and 9.5.
inline bool looks_through(const ClassShape& s) {
    const ClassCut c = forward_cut(s);
    return (!narrow_depth(class_depth(s.D)) || crowded_tiles(s)) && c.tiles <= 4 * c.parts;
}

// Whether the gradient scores the slots of a row in a launch of its own, a workgroup a row, or where it sorts them, a wave to two
// rows.  One slot: sorting takes 4 us longer for it (1024 rows x 128: 7.5 to 11.2), as much as a launch.  1024 rows x 47 x 100 fp32,
// 10 slots: 23.6 us together, 12.0 and 8.9 apart; 257 rows x 602, 50 slots: 250 us together.
constexpr bool slots_apart(const ClassShape& s) { return s.K > 1; }

// Whether the forward first lays the table out as planes of padded rows: one more pass over the table, against rows that
// the kernel has to read off the 16-byte grid, to pad, or to split into planes, once for every workgroup beside it (measured
// on 2 to 9 of them: it pays from 3 on, and from 5 on for wide 16-bit rows of which two workgroups fit a CU and hide that work).
// Tables of a quarter of a million elements and less are not worth the launch.
inline bool forward_packs(const ClassShape& s, bool straight) {
    const int depth = class_depth(s.D);
    if (!straight && !narrow_depth(depth) && s.kind == 0) return true;          // (no wave has a row whole, to make its unit of)
    const int64_t few = !narrow_depth(depth) && resident_workgroups(depth, s.kind) == 512 ? 4 : 2;
    return !straight && forward_cut(s).groups > few && s.V * s.D > (1 << 18);
}

// Byte offsets into the caller's workspace.
struct ClassPlan {
    size_t peaks, rows, table, top, sum, mean_parts, norm, back, pulls, table_scales, scales, named, named_starts, loss, start, signs, buckets, slots, row_slots, row_grad, grad_parts, bytes;
    bool packed;                                        // the forward reads the table from planes made for the call,
    bool straight;                                      // or as it is: 16-bit rows of a depth, on the 16-byte grid
};
constexpr int kPeaks = 64;                              // workgroups that look for the gradients' largest

inline ClassPlan plan_of(const ClassShape& s, bool straight, bool forward, bool want_rows, bool want_grad_w) {
    ClassPlan p{};
    size_t at = 0;
    auto room = [&at](size_t n) { const size_t a = at; at += (n + 255) / 256 * 256; return a; };
    const size_t depth = class_depth(s.D), T = padded_rows(s.T);
    p.peaks = room(kPeaks * 4);
    if (forward) {
        const bool narrow = narrow_depth((int)depth);
        const size_t slices = forward_cut(s).slices(), stats = narrow ? slices : slices * kClassWaves;
        p.straight = straight;
        p.packed = forward_packs(s, straight) && !(want_rows && narrow && crowded_tiles(s));
        if (p.packed) p.table = room(padded_rows(s.V) * depth * 2 * class_planes(s.kind));
        if (p.packed && s.kind == 0) p.table_scales = room(padded_rows(s.V) * 4);
        p.top = room(stats * T * 4);
        p.sum = room(stats * T * 4);
        if (want_rows) p.mean_parts = room(slices * T * depth * 4);
        if (want_rows && !narrow) p.norm = room(T * 4);
        if (want_rows && !narrow) p.back = room(T * 4);
        if (want_rows && !narrow) p.pulls = room(T * s.K * 4);
        if (want_rows && s.K > kWaveSlots && !looks_through(s)) {
            p.named = room(T * s.K * 4);
            p.named_starts = room(T / kBlock * (forward_cut(s).parts + 1) * 4);
        }
    }
    if (forward && want_rows) {                         // a backward that computes the rows' gradients again keeps them here
        p.row_grad = room((size_t)s.T * s.D * 4);
        p.loss = room(2 * T * 4);
    }
    if (want_grad_w) {
        const ClassCut c = gradient_cut(s);
        p.rows = room(T * depth * 2 * class_planes(s.kind));
        p.start = room(T * 4);
        if (s.kind == 0) p.scales = room(T * 4);
        p.signs = room(T / kBlock * 4);
        p.buckets = room(T / kBlock * buckets_of(s.V, s.K).count * 4);
        p.slots = room(T * s.K * 8);
        if (slots_apart(s)) p.row_slots = room(T * s.K * 8);
        if (c.slices() > 1) p.grad_parts = room((size_t)c.slices() * ceil_div(s.V, kBlock) * kBlock * depth * 4);
    }
    p.bytes = at;
    return p;
}

}  // namespace fsa
