// The block between a mean and its loss (residual norm, gated feed-forward) and the orthogonalised update of its matrices: the
// launch interface between the C ABI (fsa_block_api.hip) and the kernel files, and the arithmetic of the plans that both
// follow.  Plain C++.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace fsa {

constexpr int64_t up_to(int64_t n, int64_t grid) { return (n + grid - 1) / grid * grid; }
constexpr int64_t cut_into(int64_t n, int64_t piece) { return (n + piece - 1) / piece; }

// ---------------------------------------------------------------------------------------------------------------
// norm
// ---------------------------------------------------------------------------------------------------------------
// A row is held by `lanes` lanes, at most 16 elements to each, in one of two or three lengths.
constexpr int kNormLanes[] = {4, 16, 64, 256, 1024};
constexpr int64_t kNormDmax = 16384;
constexpr int kNormParts = 512;                         // workgroups of the backward, one part of grad_weight each

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
// Workgroups of the backward: at least two turns of rows each, so that a part of grad_weight is worth its writing.
inline int64_t norm_parts(int64_t T, int64_t D, int elem) {
    const int64_t turns = cut_into(T, norm_plan(D, elem).rows);
    const int64_t want = cut_into(turns, 2);
    return want < 1 ? 1 : want < kNormParts ? want : kNormParts;
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
};
constexpr int planes_of_kind(int kind) { return kind == 0 ? 3 : 1; }
constexpr int kGatedPeaks = 64;                         // workgroups that look for the gradients' largest

// One product's cut: tiles of `tile` x `tile`, the depth in `splits` shares.
struct ProductCut {
    int tile;
    int64_t mt, nt, splits;
};
constexpr int64_t kChip = 256;                          // CUs
inline ProductCut product_cut(int64_t M, int64_t N, int64_t K, int64_t products) {
    ProductCut c{};
    const int64_t wide = cut_into(M, 128) * cut_into(N, 128) * products;
    c.tile = wide >= kChip ? 128 : 64;
    c.mt = cut_into(M, c.tile);
    c.nt = cut_into(N, c.tile);
    const int64_t tiles = c.mt * c.nt * products > 0 ? c.mt * c.nt * products : 1, steps = cut_into(K, 64);    // (no rows: no tiles)
    c.splits = 2 * kChip / tiles;
    if (c.splits > steps / 4) c.splits = steps / 4;
    if (c.splits < 1) c.splits = 1;
    return c;
}
inline int pair_tile(int64_t T, int64_t H) { return cut_into(T, 128) * cut_into(H, 64) >= kChip ? 128 : 64; }

// Byte offsets into the caller's workspace.
struct GatedPlan {
    size_t x, gate, up, down, grad_y;                   // laid out operands
    size_t h, dg, du, peaks, parts, bytes;
    int64_t D8, H8, O8;
    ProductCut answer, dx, down_grad, gate_grad;
};
// `packs`: bits x, gate, up, down, grad_y of operands that are laid out.
inline GatedPlan gated_plan(const GatedShape& s, bool backward, bool want_x, bool want_w, int packs) {
    GatedPlan p{};
    size_t at = 0;
    auto room = [&at](int64_t n) { const size_t a = at; at += (size_t)up_to(n, 256); return a; };
    p.D8 = up_to(s.D, 8); p.H8 = up_to(s.H, 8); p.O8 = up_to(s.O, 8);
    const int64_t planes = 2 * planes_of_kind(s.kind);  // bytes of an element's planes
    if (packs & 1) p.x = room(s.T * p.D8 * planes);
    if (packs & 2) p.gate = room(s.H * p.D8 * planes);
    if (packs & 4) p.up = room(s.H * p.D8 * planes);
    if (packs & 8) p.down = room(s.O * p.H8 * planes);
    p.h = room(s.T * p.H8 * planes);
    int64_t parts = 0;
    auto product = [&](int64_t M, int64_t N, int64_t K, int64_t products) {
        const ProductCut c = product_cut(M, N, K, products);
        if (c.splits > 1) { const int64_t b = products * c.splits * M * up_to(N, 8) * 4; parts = parts > b ? parts : b; }
        return c;
    };
    if (!backward) p.answer = product(s.T, s.O, s.H, 1);
    else {
        if (packs & 16) p.grad_y = room(s.T * p.O8 * planes);
        p.dg = room(s.T * p.H8 * planes);
        p.du = room(s.T * p.H8 * planes);
        p.peaks = room(kGatedPeaks * 4);
        if (want_x) p.dx = product(s.T, s.D, 2 * s.H, 1);
        if (want_w) {
            p.down_grad = product(s.O, s.H, s.T, 1);
            p.gate_grad = product(s.H, s.D, s.T, 2);
        }
    }
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
    GatedPlan plan;
    int packs;
    char* ws;
};

// ---------------------------------------------------------------------------------------------------------------
// orthogonalised updates
// ---------------------------------------------------------------------------------------------------------------
// X [m,n] with m <= n (the transpose of a tall matrix): two fp16 planes of X 2^13, likewise A = X X^T and P = b A + c A^2 of
// which planes hold A 2^13 and P 2^10.
constexpr int kMostSteps = 32;
constexpr int kOrthoPeaks = 64;                         // workgroups a matrix that sum its squares
constexpr int kUnitX = 13, kUnitA = 13, kUnitP = 10;

struct OrthoShape {
    int64_t B, M, N;
    int kind;
};
struct OrthoPlan {
    size_t squares, x[2], a, p, bytes;
    int64_t m, n, m8, n8;
    int tile_square, tile_wide;                         // of m x m and m x n results
};
inline OrthoPlan ortho_plan(const OrthoShape& s) {
    OrthoPlan p{};
    size_t at = 0;
    auto room = [&at](int64_t n) { const size_t a = at; at += (size_t)up_to(n, 256); return a; };
    p.m = s.M < s.N ? s.M : s.N;
    p.n = s.M < s.N ? s.N : s.M;
    p.m8 = up_to(p.m, 8); p.n8 = up_to(p.n, 8);
    p.tile_square = s.B * cut_into(p.m, 128) * cut_into(p.m, 128) >= kChip ? 128 : 64;
    p.tile_wide = s.B * cut_into(p.m, 128) * cut_into(p.n, 128) >= kChip ? 128 : 64;
    p.squares = room(s.B * kOrthoPeaks * 8);
    for (size_t& x : p.x) x = room(s.B * p.m * p.n8 * 4);
    p.a = room(s.B * p.m * p.m8 * 4);
    p.p = room(s.B * p.m * p.m8 * 4);
    p.bytes = at;
    return p;
}
struct OrthoArgs {
    OrthoShape s;
    const void* g;
    int64_t batch_stride, stride;
    void* out;                                          // contiguous
    float coefficients[3 * kMostSteps];
    int steps;
    float eps, scale;
    OrthoPlan plan;
    char* ws;
};

}  // namespace fsa
