// The gated feed-forward block, one element type a translation unit (fsa_gated_{f32,bf16,f16}.hip).
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T;   dh = gy Wd, dg = dh u act'(g), du = dh act(g)
//   dx = dg Wg + du Wu,  dWd = gy^T h,  dWg = dg^T x,  dWu = du^T x
//
// g and u are made side by side (one x, two tables), so that a lane has both of an element and h is all that has to be written.  The
// backward makes them again beside dh, in a kernel of three sums, or reads them where the forward kept them: in 16 bits they would be
// rounded once more on the way to every gradient, so they are kept in 24 bits beside 16-bit tables.  16384 x 1024 -> 4096 bfloat16: the
// hidden pass takes some 290 us instead of 253 and the slopes 240 instead of 623, since three sums only leave room for tiles of
// 128 x 128, of which the reads are as much as L2 gives.  What bounds them kept is the matrix cores (212 and 106 us of it at the rate of
// the largest tile) and then what they write and read (0.54 and 0.67 GB), the one after the other: all workgroups are at the same
// part of their tile, and one told to begin later gains as little as it loses.  The products of the backward, 5/9 of the work, reach 1160
// TFLOP/s with their join (687 GFLOP in 563 and 30 us).
// h, dg and du are rounded to the type once: each gradient is then off by its own rounding and one of a factor, as in any product of
// tensors of that type (0.0023 for 0.0017).  Two planes of them leave its own alone and take 1990 us of such a pass where one takes 1240: in
// small calls, and where the caller asks for them.  fp32 has three planes and loses nothing.
// fp16: h, dg and du are kept times powers of two, which the products take back, so that none is beyond fp16's largest number and the smallest
// are not rounded among its subnormal ones.  A product of two rows is no larger than that of their lengths:  |h| <= |g| |u| <= |x|^2 |wg| |wu|
// and |dg|, |du| <= 1.13 |gy| |wd| |x| max(|wu|, |wg|), of the longest rows (columns of wd), are brought to [2^14, 2^15).  Such bounds
// lie some 2^4 to 2^8 above the largest element that random numbers have; numbers of up to 2^-28 of a bound are normal ones.  Looking for the
// longest rows is a launch: 4 us of 64 x 256 -> 1024, 13 us (3.8 TB/s) of 16384 x 1024 -> 4096's forward of 380 and 21 of its backward of 900.
#pragma once

#include "fsa_block_kernels.h"
#include "fsa_product.hip.h"
#include "../../include/fsa.h"

#include <type_traits>

#ifdef FSA_GATED_KIND
namespace fsa {
namespace {

using namespace product;

constexpr int kKind = FSA_GATED_KIND;
constexpr int NP = planes_of_kind(kKind);
constexpr bool kHalf = kKind == 2;
constexpr int BK = NP == 3 ? 32 : 64;
using Elem = typename std::conditional<kKind == 0, float, uint16_t>::type;

// The tiles that fsa_block.h chooses from, in its order.  fp32's small ones have 8 waves and steps of 64 of the depth where two of them
// fit, since they mostly have a CU to themselves: 64 rows of 1024 -> 4096 in tiles of 64 x 64 x 2 take 25 us, with 4 waves
// 28 and with steps of 32 as well 33; 256 x 4096 -> 1024 in tiles of 128 x 64 18.6 rather than 24.4.  16-bit tiles of 64 x 64 are as quick with 4 waves.
template <int CHOICE> struct Tiles;
template <> struct Tiles<0> {
    using Product = Tile<NP, kHalf, 64, 64, 64, NP == 3 ? 4 : 2, 2>;
    using Hidden = Product;
    using Slopes = Product;
};
template <> struct Tiles<1> {
    using Product = Tile<NP, kHalf, 128, NP == 1 ? 128 : 64, 64, 4, 2>;
    using Hidden = Tile<NP, kHalf, 128, 64, BK, 2, 2>;
    using Slopes = Hidden;
};
template <> struct Tiles<2> {
    using Product = Tile<NP, kHalf, 256, NP == 1 ? 256 : 128, BK, NP == 1 ? 2 : 4, NP == 1 ? 4 : 2>;
    using Hidden = Tile<NP, kHalf, 256, NP == 1 ? 128 : 64, BK, NP == 1 ? 2 : 4, NP == 1 ? 4 : 2>;
    using Slopes = Tile<NP, kHalf, NP == 1 ? 128 : 256, NP == 1 ? 128 : 64, BK, 4, 2>;
};
template <int CHOICE> constexpr bool same_tiles() {
    using C = Tiles<CHOICE>;
    constexpr TileChoice p = product_tile(kKind, CHOICE), h = pair_tile(kKind, CHOICE, false), s = pair_tile(kKind, CHOICE, true);
    return C::Product::BM == p.m && C::Product::BN == p.n && C::Hidden::BM == h.m && C::Hidden::BN == h.n && C::Slopes::BM == s.m &&
           C::Slopes::BN == s.n;
}
static_assert(same_tiles<0>() && same_tiles<1>() && same_tiles<2>(), "as the plan has them");

// ---------------------------------------------------------------------------------------------------------------
// operands laid out as planes: rows of a multiple of 8 elements, zeros behind their end
// ---------------------------------------------------------------------------------------------------------------
struct PackList {
    Matrix from[5];
    uint16_t* to[5];
    int64_t first[6];                                   // pieces of 8 elements before each
    int count;
    unsigned packers;                                   // workgroups that lay out; behind them kGatedPeaks a kind look for the longest rows
    Matrix measured[kPeakKinds];
    float* peaks;                                       // [kinds][kGatedPeaks], squares
};
__device__ __forceinline__ void load_piece(const Matrix& from, int64_t row, int64_t col, Elem (&e)[8]) {
    const Elem* p = static_cast<const Elem*>(from.p) + row * from.stride + col;
    if (col + 8 <= from.cols) __builtin_memcpy(e, p, sizeof(e));
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = col + j < from.cols ? p[j] : Elem(0);
    }
}
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return a <= 0x7fffffff ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// fp16: the square of the longest row of a workgroup's share, among those that are finite; of this wave's rows.  A lane asks for kAhead pieces
// before it adds them up, with no branch but whether they are there.
constexpr int kAhead = 8;
__device__ __forceinline__ float half_of(u32x4 raw, int j) { return as_float<true>(j % 2 ? raw[j / 2] >> 16 : raw[j / 2] & 0xffff); }
__device__ __forceinline__ float longest_row(const Matrix& m, unsigned share) {
    const int64_t whole = m.cols / 8;
    int bits = 0;                                       // lanes to a row
    while (bits < 6 && kAhead << bits < whole) ++bits;
    const int lane = threadIdx.x & 63, rows = 64 >> bits, lanes = 1 << bits, own = lane & (lanes - 1);
    float top = 0.0f;
    for (int64_t r = ((int64_t)share * 4 + (threadIdx.x >> 6)) * rows; r < m.rows; r += (int64_t)kGatedPeaks * 4 * rows) {
        const int64_t row = r + (lane >> bits);
        float sum = 0.0f;
        if (row < m.rows) {
            const Elem* p = static_cast<const Elem*>(m.p) + row * m.stride;
            for (int64_t at = own; at < whole; at += kAhead * lanes) {
                u32x4 raw[kAhead] = {};
#pragma unroll
                for (int i = 0; i < kAhead; ++i) if (at + i * lanes < whole) __builtin_memcpy(&raw[i], p + (at + i * lanes) * 8, 16);
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum = fmaf(half_of(raw[i], j), half_of(raw[i], j), sum);
            }
            if (own == 0)
                for (int64_t c = whole * 8; c < m.cols; ++c) {
                    const float x = as_float<true>((uint32_t)p[c]);
                    sum = fmaf(x, x, sum);
                }
        }
        for (int d = 1; d < lanes; d *= 2) sum += __shfl_xor(sum, d, 64);
        if (sum < __builtin_inff()) top = fmaxf(top, sum);
    }
    return top;
}
// The same of columns, 32 a workgroup at a time: four lanes to a row's, 64 rows side by side; all of the workgroup calls.
__device__ __forceinline__ float longest_column(const Matrix& m, unsigned share) {
    __shared__ float lds[4][32];
    const int lane = threadIdx.x & 63, line = threadIdx.x >> 2;
    float top = 0.0f;
    for (int64_t c0 = (int64_t)share * 32; c0 < m.cols; c0 += (int64_t)kGatedPeaks * 32) {
        const int64_t col = c0 + 8 * (lane & 3);
        const Elem* p = static_cast<const Elem*>(m.p) + col;
        float sum[8] = {};
        if (col + 8 <= m.cols) {
            for (int64_t row = line; row < m.rows; row += kAhead * 64) {
                u32x4 raw[kAhead] = {};
#pragma unroll
                for (int i = 0; i < kAhead; ++i) if (row + i * 64 < m.rows) __builtin_memcpy(&raw[i], p + (row + i * 64) * m.stride, 16);
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] = fmaf(half_of(raw[i], j), half_of(raw[i], j), sum[j]);
            }
        } else if (col < m.cols) {
            for (int64_t row = line; row < m.rows; row += 64)
#pragma unroll
                for (int j = 0; j < 7; ++j) {
                    const float x = col + j < m.cols ? as_float<true>((uint32_t)p[row * m.stride + j]) : 0.0f;
                    sum[j] = fmaf(x, x, sum[j]);
                }
        }
#pragma unroll
        for (int d = 4; d < 64; d *= 2)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += __shfl_xor(sum[j], d, 64);
        if (lane < 4)
#pragma unroll
            for (int j = 0; j < 8; ++j) lds[threadIdx.x >> 6][8 * lane + j] = sum[j];
        __syncthreads();
        if (threadIdx.x < 32) {
            const float all = (lds[0][threadIdx.x] + lds[1][threadIdx.x]) + (lds[2][threadIdx.x] + lds[3][threadIdx.x]);
            if (all < __builtin_inff()) top = fmaxf(top, all);
        }
        __syncthreads();
    }
    return top;
}
__device__ __forceinline__ void find_peak(const PackList& l) {
    __shared__ float lds[4];
    const unsigned kind = (blockIdx.x - l.packers) / kGatedPeaks, share = (blockIdx.x - l.packers) % kGatedPeaks;
    float top = kind == kPeakDown ? longest_column(l.measured[kind], share) : longest_row(l.measured[kind], share);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) l.peaks[kind * kGatedPeaks + share] = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}
__global__ __launch_bounds__(256) void pack_kernel(PackList l) {
    if constexpr (kHalf)
        if (blockIdx.x >= l.packers) return find_peak(l);
    const int64_t all = l.first[l.count];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)l.packers * 256) {
        int m = 0;
#pragma unroll
        for (int j = 1; j < 5; ++j) if (j < l.count && i >= l.first[j]) m = j;
        const Matrix from = l.from[m];
        const int64_t pieces = cut_into(from.cols, 8), at = i - l.first[m], row = quotient(at, pieces), col = (at - row * pieces) * 8;
        Elem e[8];
        load_piece(from, row, col, e);
        const int64_t plane = from.rows * pieces * 8;
        uint16_t* to = l.to[m] + (row * pieces * 8 + col);
        if constexpr (kKind == 0) {
            uint32_t w[4][NP];
#pragma unroll
            for (int j = 0; j < 4; ++j) split2<NP, kHalf>(e[2 * j], e[2 * j + 1], w[j]);
#pragma unroll
            for (int q = 0; q < NP; ++q) *reinterpret_cast<u32x4*>(to + q * plane) = u32x4{w[0][q], w[1][q], w[2][q], w[3][q]};
        } else {
            u32x4 w;
            __builtin_memcpy(&w, e, 16);
            *reinterpret_cast<u32x4*>(to) = w;
        }
    }
}

// e with bound * 2^e in [2^14, 2^15).
__device__ __forceinline__ int lift_to_end(float bound) {
    if (!(bound > 0.0f)) return 0;
    const int e = 14 + 127 - (int)(__builtin_bit_cast(uint32_t, bound) >> 23);
    return e < -110 ? -110 : e > 110 ? 110 : e;
}
enum { kNoLift, kLiftH, kLiftD };
// The power of two beside which h, or dg and du are kept (see above); 1.02 for what the sums are off by.
template <int OF> __device__ __forceinline__ int lift_of(const float* peaks) {
    constexpr int KINDS = OF == kLiftH ? kPeakGradY : kPeakKinds;
    static_assert(kGatedPeaks == 256, "four a lane");
    float top[KINDS];
#pragma unroll
    for (int k = 0; k < KINDS; ++k) {
        const f32x4 four = reinterpret_cast<const f32x4*>(peaks + k * kGatedPeaks)[threadIdx.x & 63];
        top[k] = fmaxf(fmaxf(four[0], four[1]), fmaxf(four[2], four[3]));
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < KINDS; ++k) top[k] = fmaxf(top[k], __shfl_xor(top[k], d, 64));
#pragma unroll
    for (int k = 0; k < KINDS; ++k) top[k] = sqrtf(top[k]);
    if constexpr (OF == kLiftH) return lift_to_end(1.02f * (top[kPeakX] * top[kPeakGate]) * (top[kPeakX] * top[kPeakUp]));
    else return lift_to_end(1.02f * 1.13f * (top[kPeakGradY] * top[kPeakDown]) * (top[kPeakX] * fmaxf(top[kPeakGate], top[kPeakUp])));
}
__device__ __forceinline__ int lift_of(const float* peaks, int of) { return of == kLiftH ? lift_of<kLiftH>(peaks) : of == kLiftD ? lift_of<kLiftD>(peaks) : 0; }
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// ---------------------------------------------------------------------------------------------------------------
// activations: value and derivative
// ---------------------------------------------------------------------------------------------------------------
struct Gate { float value, slope; };
__device__ __forceinline__ float inverse(float x) { return kKind == 0 ? 1.0f / x : __builtin_amdgcn_rcpf(x); }
// The normal distribution beside 16-bit types, from its density: what lies beyond |g| is the density times Mills' ratio, which a polynomial of
// 1 / (1 + 0.35 |g|) meets within 2^-20 of itself (fitted for the least largest error up to 14, where the density is 1e-43).  1 + erf
// leaves nothing of gates below -5 (of gelu(-5) it is 4 % off).  Forward of 16384 x 1024 -> 4096 bfloat16: 379 us, with the library's erfc
// 423, with 1 + erf 404.
__device__ __forceinline__ float distribution(float g, float density) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, fabsf(g), 1.0f));
    float ratio = 0.122679926f;
    ratio = fmaf(ratio, t, -0.506635785f);
    ratio = fmaf(ratio, t, 0.603193879f);
    ratio = fmaf(ratio, t, -0.0426689051f);
    ratio = fmaf(ratio, t, 0.390936345f);
    ratio = fmaf(ratio, t, 0.334271938f);
    ratio = fmaf(ratio, t, 0.351605564f);
    ratio = fmaf(ratio, t, -6.84674669e-05f);
    const float beyond = density * ratio;
    return g < 0.0f ? beyond : 1.0f - beyond;
}
template <int ACT> __device__ __forceinline__ Gate gate_of(float g) {
    if constexpr (ACT == FSA_ACT_SILU) {
        const float p = inverse(1.0f + (kKind == 0 ? expf(-g) : __expf(-g)));
        return {g * p, p * fmaf(g, 1.0f - p, 1.0f)};
    } else if constexpr (ACT == FSA_ACT_GELU) {
        const float bell = 0.39894228040143267794f * (kKind == 0 ? expf(-0.5f * g * g) : __expf(-0.5f * g * g));
        const float p = kKind == 0 ? 0.5f * erfcf(-0.70710678118654752440f * g) : distribution(g, bell);
        return {g * p, fmaf(g, bell, p)};
    } else {
        return {g > 0.0f ? g : (g != g ? g : 0.0f), g > 0.0f ? 1.0f : 0.0f};
    }
}

__device__ __forceinline__ int at_most(int most, int64_t n) { return n < most ? (int)n : most; }
struct HiddenArgs {
    Side x, gate, up, down, grad_y;
    uint16_t *h, *dg, *du;                              // [T, H8] planes
    char* kept;                                         // or null
    KeptPlan at;                                        // of it
    int64_t T, D, H, O, H8;
    const float* peaks;
    unsigned mt, nt;
};

// W elements of g or u as they are kept (see KeptPlan), at element `at`; `left` of the row's H8 are there from it on.  Nothing reads
// them before the backward, and a wave, 8 to a lane, writes whole lines: past the caches, which the next product's h has to itself.
// 16384 x 1024 -> 4096 bfloat16: the answer takes 109 us rather than 136; in rows of H8 elements, 64 bytes of each of 16, the hidden pass
// took 313 us and 425 past the caches, where blocks take 292 either way.
template <int W> __device__ __forceinline__ void store_kept(char* p, char* low, int64_t at, int left, const float (&x)[W]) {
#pragma unroll
    for (int i = 0; i < W; i += 8) {
        if (i >= left) return;
        if constexpr (kKind == 0) {
#pragma unroll
            for (int j = 0; j < 8; j += 4)
                __builtin_nontemporal_store(f32x4{x[i + j], x[i + j + 1], x[i + j + 2], x[i + j + 3]}, reinterpret_cast<f32x4*>(p + (at + i + j) * 4));
        } else {
            uint32_t word[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)                 // to nearest 24 bits, which leaves infinities as they are
                word[j] = x[i + j] != x[i + j] ? 0x7fc00000u : __builtin_bit_cast(uint32_t, x[i + j]) + 0x80u;
            u32x4 high;
#pragma unroll
            for (int j = 0; j < 4; ++j) high[j] = __builtin_amdgcn_perm(word[2 * j + 1], word[2 * j], 0x07060302u);
            u32x2 rest;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                rest[j] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(word[4 * j + 3], word[4 * j + 2], 0x0c0c0501u),
                                                __builtin_amdgcn_perm(word[4 * j + 1], word[4 * j], 0x0c0c0501u), 0x05040100u);
            __builtin_nontemporal_store(high, reinterpret_cast<u32x4*>(p + (at + i) * 2));
            __builtin_nontemporal_store(rest, reinterpret_cast<u32x2*>(low + at + i));
        }
    }
}
// The same elements on their way back.
template <int W> struct KeptRow {
    static constexpr int PER = kKind == 0 ? 4 : 8;
    u32x4 high[W / PER];
    u32x2 rest[kKind == 0 ? 1 : W / 8];
    __device__ __forceinline__ void ask(const char* p, const char* low, int64_t at, int left) {
#pragma unroll
        for (int i = 0; i < W; i += PER) {
            high[i / PER] = u32x4{};
            if constexpr (kKind != 0) rest[i / 8] = u32x2{};
            if (i >= left) continue;
            high[i / PER] = *reinterpret_cast<const u32x4*>(p + (at + i) * (16 / PER));
            if constexpr (kKind != 0) rest[i / 8] = *reinterpret_cast<const u32x2*>(low + at + i);
        }
    }
    __device__ __forceinline__ void get(float (&x)[W]) const {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const uint32_t word = high[i / PER][i % PER * 4 / PER];     // (a vector's element itself is not what a bit cast takes)
            if constexpr (kKind == 0) x[i] = __builtin_bit_cast(float, word);
            else {
                const uint32_t up = i % 2 ? word & 0xffff0000u : word << 16;
                x[i] = __builtin_bit_cast(float, up | (rest[i / 8][i % 8 / 4] >> (i % 4 * 8) & 0xff) << 8);
            }
        }
    }
};

// PLANES of h, dg and du: one more than an operand has where the rounding's rest is kept.
template <class T, int ACT, int PLANES> __global__ __launch_bounds__(T::THREADS, T::waves(2)) void hidden_kernel(HiddenArgs a) {
    __shared__ __attribute__((aligned(256))) char lds[T::lds_bytes(2)];
    unsigned mi, ni;
    tile_of(blockIdx.x, a.mt, a.nt, mi, ni);
    const int64_t m0 = (int64_t)mi * T::BM, n0 = (int64_t)ni * T::BN;
    using Stream = OneStream<T, true, true, 2>;
    Stream stream;
    const Side tables[2] = {a.gate, a.up};
    stream.flow.start(a.x, tables, m0, a.T, n0, a.H, 0, a.D);
    Ring<T, T::stage_bytes(2), Stream> ring{lds, stream};
    ring.fill();
    const float lift = kHalf ? power_of_two(lift_of<kLiftH>(a.peaks)) : 1.0f;       // (beside the first requests)
    Sums<T, 2> acc = {};
    accumulate<T, true, true, 2>(acc, ring, cut_into(a.D, T::BK));
    ring.end();
    each_stretch<T>(m0, n0, [&](int i, int64_t m, int64_t n) {
        if (m >= a.T) return;
        constexpr int W = 4 * T::NJ;
        float g[W], u[W];
#pragma unroll
        for (int j = 0; j < W; ++j) { g[j] = acc[0][i][j / 4][j % 4]; u[j] = acc[1][i][j / 4][j % 4]; }
        if (a.kept) {
            const int left = at_most(W, a.H8 - n);
            const int64_t at = kept_at(m, n, cut_into(a.H, kKeptCols));
            store_kept(a.kept + a.at.g, a.kept + a.at.g_low, at, left, g);
            store_kept(a.kept + a.at.u, a.kept + a.at.u_low, at, left, u);
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
            g[j] = gate_of<ACT>(g[j]).value * u[j];
            if constexpr (kHalf) g[j] *= lift;
        }
        store_planes<PLANES, T::HALF>(a.h, a.T * a.H8, m * a.H8 + n, n, a.H, g);
    });
}

// What slopes without kept gates ask for: grad_y and w_down, then x and both tables.
template <class T> struct SlopesStream {
    using F = Flow<T, true, false, 1>;
    using G = Flow<T, true, true, 2>;
    static constexpr int ASKS = G::ASKS, SURE = F::SURE < G::SURE ? F::SURE : G::SURE;
    static_assert(F::ASKS <= G::ASKS, "");
    F down;
    G gates;
    bool at_gates = false;
    __device__ __forceinline__ SlopesStream(const HiddenArgs& a, int64_t m0, int64_t n0) {
        const Side table[1] = {a.down}, tables[2] = {a.gate, a.up};
        down.start(a.grad_y, table, m0, a.T, n0, a.H8, 0, a.O);
        gates.start(a.x, tables, m0, a.T, n0, a.H, 0, a.D);
    }
    __device__ __forceinline__ void ask(uint32_t stage, int piece) const {
        if (at_gates) gates.ask(stage, piece);
        else if (piece < F::ASKS) down.ask(stage, piece);
    }
    __device__ __forceinline__ void next() {
        if (at_gates) gates.next();
        else { down.next(); at_gates = down.left == 0; }
    }
};

template <class T, int ACT, int PLANES, bool KEPT> __global__ __launch_bounds__(T::THREADS, T::waves(KEPT ? 1 : 2)) void slopes_kernel(HiddenArgs a) {
    constexpr int PARTS = KEPT ? 1 : 2;
    __shared__ __attribute__((aligned(256))) char lds[T::lds_bytes(PARTS)];
    unsigned mi, ni;
    tile_of(blockIdx.x, a.mt, a.nt, mi, ni);
    const int64_t m0 = (int64_t)mi * T::BM, n0 = (int64_t)ni * T::BN;
    Sums<T, PARTS> acc = {};
    Sums<T, 1> dh = {};
    float lift = 1.0f, lift_h = 1.0f;                   // found beside the first requests
    if constexpr (KEPT) {
        using Stream = OneStream<T, true, false, 1>;
        Stream stream;
        const Side table[1] = {a.down};
        stream.flow.start(a.grad_y, table, m0, a.T, n0, a.H8, 0, a.O);
        Ring<T, T::stage_bytes(1), Stream> ring{lds, stream};
        ring.fill();
        if constexpr (kHalf) lift = power_of_two(lift_of<kLiftD>(a.peaks));
        accumulate<T, true, false, 1>(dh, ring, cut_into(a.O, T::BK));
        ring.end();
    } else {
        SlopesStream<T> stream(a, m0, n0);
        Ring<T, T::stage_bytes(2), SlopesStream<T>> ring{lds, stream};
        ring.fill();
        if constexpr (kHalf) { lift = power_of_two(lift_of<kLiftD>(a.peaks)); lift_h = power_of_two(lift_of<kLiftH>(a.peaks)); }
        accumulate<T, true, false, 1>(dh, ring, cut_into(a.O, T::BK));
        accumulate<T, true, true, 2>(acc, ring, cut_into(a.D, T::BK));
        ring.end();
    }
    settle<T, 1>(dh);
    constexpr int W = 4 * T::NJ;
    KeptRow<W> kept_g, kept_u;                          // asked for a row ahead, before the one before is written
    auto ask_kept = [&](int64_t m, int64_t n) {
        const int left = m < a.T ? at_most(W, a.H8 - n) : 0;
        const int64_t at = kept_at(m, n, cut_into(a.H, kKeptCols));
        kept_g.ask(a.kept + a.at.g, a.kept + a.at.g_low, at, left);
        kept_u.ask(a.kept + a.at.u, a.kept + a.at.u_low, at, left);
    };
    if constexpr (KEPT) each_stretch<T>(m0, n0, [&](int i, int64_t m, int64_t n) { if (i == 0) ask_kept(m, n); });
    each_stretch<T>(m0, n0, [&](int i, int64_t m, int64_t n) {
        float g[W], u[W], dg[W], du[W];
        if constexpr (KEPT) {
            kept_g.get(g);
            kept_u.get(u);
            if (i + 1 < T::MI) ask_kept(m + 16, n);
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j) { g[j] = acc[0][i][j / 4][j % 4]; u[j] = acc[1][i][j / 4][j % 4]; }
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const Gate at = gate_of<ACT>(g[j]);
            const float d = kHalf ? dh[0][i][j / 4][j % 4] * lift : dh[0][i][j / 4][j % 4];
            g[j] = kHalf ? at.value * u[j] * lift_h : at.value * u[j];
            dg[j] = d * u[j] * at.slope;
            du[j] = d * at.value;
        }
        if (m >= a.T) return;
        if constexpr (!KEPT) store_planes<PLANES, T::HALF>(a.h, a.T * a.H8, m * a.H8 + n, n, a.H, g);
        store_planes<PLANES, T::HALF>(a.dg, a.T * a.H8, m * a.H8 + n, n, a.H, dg);
        store_planes<PLANES, T::HALF>(a.du, a.T * a.H8, m * a.H8 + n, n, a.H, du);
    });
}

// ---------------------------------------------------------------------------------------------------------------
// products that leave in the caller's type
// ---------------------------------------------------------------------------------------------------------------
// Up to three at a time, so that one's last workgroups run beside the next one's first, and small ones side by side.
struct Job {
    Side a[2][4], b[2][4];                              // of up to two results, the pairs of operands whose products make one
    void* out[2];
    int64_t M, N, K, out_ld;                            // K: depth of one pair
    int64_t M8, N8;                                     // ends of flat operands
    float* parts;                                       // [results][splits][M][N8], where there are splits
    int pairs, results, planned;                        // planned: which of the plan's
    int lift;                                           // beside which of them one operand is kept
    bool adeep, grid;
    unsigned mt, nt, splits, first, first_join;         // workgroups before this job's
};
struct Jobs {
    Job job[kMostJobs];
    int count;
    const float* peaks;
};

// A workgroup's place in a launch: its job, result, share of the depth and tile.
struct Place {
    const Job* job;
    unsigned which, split;
    unsigned mi, ni;
};
__device__ __forceinline__ Place place_of(const Jobs& l, unsigned id) {
    int j = 0;
#pragma unroll
    for (int i = 1; i < kMostJobs; ++i) if (i < l.count && id >= l.job[i].first) j = i;
    const Job& a = l.job[j];
    const unsigned tiles = a.mt * a.nt, at = id - a.first;
    Place p{&a, at / tiles / a.splits, at / tiles % a.splits, 0, 0};
    tile_of(at % tiles, a.mt, a.nt, p.mi, p.ni);
    return p;
}
// What the products of a place ask for: its share of all its pairs' steps, one pair after the other.  Pairs lie alike, so that to
// whoever multiplies they are one product.
template <class T, bool ADEEP, bool BDEEP> struct ProductStream {
    using F = Flow<T, ADEEP, BDEEP, 1>;
    static constexpr int ASKS = F::ASKS, SURE = F::SURE;
    const Job& a;
    int64_t m0, n0, steps, last;                            // steps: in all; last: of the share, from the present pair's first
    unsigned which;
    int pair;
    F flow;
    __device__ __forceinline__ explicit ProductStream(const Place& p) : a(*p.job), m0((int64_t)p.mi * T::BM), n0((int64_t)p.ni * T::BN), which(p.which) {
        const int64_t each = cut_into(a.K, T::BK), all = a.pairs * each, first = all * p.split / a.splits;
        pair = (int)(first / each);
        last = all * (p.split + 1) / a.splits;
        steps = last - first;
        last -= pair * each;
        const Side b[1] = {a.b[which][pair]};
        flow.start(a.a[which][pair], b, m0, ADEEP ? a.M : a.M8, n0, BDEEP ? a.N : a.N8, (first - pair * each) * T::BK, end());
    }
    __device__ __forceinline__ int64_t end() const { return last * T::BK < a.K ? last * T::BK : a.K; }
    __device__ __forceinline__ void ask(uint32_t stage, int piece) const { flow.ask(stage, piece); }
    __device__ __forceinline__ void next() {
        flow.next();
        if (flow.left > 0) return;
        last -= cut_into(a.K, T::BK);
        if (last <= 0) return;
        ++pair;
        flow.a.move(a.a[which][pair], m0, 0);
        flow.b[0].move(a.b[which][pair], n0, 0);
        flow.left = end();
    }
};

// `back`: what takes the operand's power of two from the result, found beside the first requests.
template <class T, bool ADEEP, bool BDEEP> __device__ __forceinline__ void make_products(Sums<T, 1>& acc, char* lds, const Place& p, const float* peaks, float& back) {
    using Stream = ProductStream<T, ADEEP, BDEEP>;
    Stream stream(p);
    Ring<T, T::stage_bytes(1), Stream> ring{lds, stream};
    ring.fill();
    if (kHalf && p.job->splits == 1) back = power_of_two(-lift_of(peaks, p.job->lift));
    accumulate<T, ADEEP, BDEEP, 1>(acc, ring, stream.steps);
    ring.end();
    if constexpr (!BDEEP) settle<T, 1>(acc);
}

template <class T, bool FORWARD> __global__ __launch_bounds__(T::THREADS, T::waves(1)) void product_kernel(Jobs l) {
    __shared__ __attribute__((aligned(256))) char lds[T::lds_bytes(1)];
    const Place p = place_of(l, blockIdx.x);
    const Job& a = *p.job;
    Sums<T, 1> acc = {};
    float back = 1.0f;
    if constexpr (FORWARD) make_products<T, true, true>(acc, lds, p, l.peaks, back);
    else if (a.adeep) make_products<T, true, false>(acc, lds, p, l.peaks, back);
    else make_products<T, false, false>(acc, lds, p, l.peaks, back);
    each_stretch<T>((int64_t)p.mi * T::BM, (int64_t)p.ni * T::BN, [&](int i, int64_t m, int64_t n) {
        float x[4 * T::NJ];
#pragma unroll
        for (int j = 0; j < 4 * T::NJ; ++j) x[j] = kHalf ? acc[0][i][j / 4][j % 4] * back : acc[0][i][j / 4][j % 4];
        if (a.splits > 1) store_numbers(a.parts + ((p.which * a.splits + p.split) * a.M + m) * a.N8, m < a.M, n, a.N8, true, x);
        else if constexpr (kKind == 0) store_numbers(static_cast<float*>(a.out[p.which]) + m * a.out_ld, m < a.M, n, a.N, a.grid, x);
        else if (m < a.M) store_row<kKind>(a.out[p.which], m * a.out_ld, n, a.N, a.grid, x);
    });
}

// Splits' parts joined in their order, 4 elements a lane.
__global__ __launch_bounds__(256) void join_kernel(Jobs l) {
    int which_job = 0;
#pragma unroll
    for (int j = 1; j < kMostJobs; ++j) if (j < l.count && blockIdx.x >= l.job[j].first_join) which_job = j;
    const Job& a = l.job[which_job];
    const float back = kHalf ? power_of_two(-lift_of(l.peaks, a.lift)) : 1.0f;
    const int64_t pieces = a.N8 / 4, all = a.M * pieces, at = (int64_t)(blockIdx.x - a.first_join) * 256 + threadIdx.x;
    if (at >= all * a.results) return;
    const int64_t which = at >= all ? 1 : 0, i = at - which * all, row = quotient(i, pieces);
    const float* parts = a.parts + which * a.splits * a.M * a.N8 + i * 4;
    f32x4 sum = {};
#pragma unroll 4
    for (unsigned s = 0; s < a.splits; ++s) sum += *reinterpret_cast<const f32x4*>(parts + s * a.M * a.N8);
    const float x[4] = {sum[0] * back, sum[1] * back, sum[2] * back, sum[3] * back};
    store_row<kKind>(a.out[which], row * a.out_ld, (i - row * pieces) * 4, a.N, a.grid, x);
}

// Gradients of weights over no rows at all.
__global__ __launch_bounds__(256) void zero_kernel(Elem* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = Elem(0);
}

// ---------------------------------------------------------------------------------------------------------------
// few rows
// ---------------------------------------------------------------------------------------------------------------
// Up to 16 rows, 32 in fp32, against tables that are read once: 16 rows of a table a workgroup, its waves a
// share of the depth each, from memory to registers at whatever alignment they have; the shares meet in LDS.  h stays fp32.
// 1 x 1024 -> 4096 -> 1024 bfloat16: 5.2 + 8.1 us, tables read at 3.2 and 1.0 TB/s; chains of a cold read, a meeting and, for the
// second, h from other XCDs bound it (8 or 4 rows a workgroup, for more of them, change nothing).  17 rows and more are as quick with the
// tiles above (18.5 and 18.9 us); 32 rows of fp32 take 47 us and in tiles 60.
struct FewArgs {
    Matrix x, gate, up, down;
    float* h;                                           // [T,H]
    float* peaks;                                       // fp16: the largest |h| of each workgroup
    void* y;
    int64_t T, D, H, O;
    int activation;
};
constexpr int kFewWaves = 4, kFewAnswerWaves = 16;
constexpr int kHeld = NP == 1 ? 2 : 3;                  // planes of h

// Eight elements of a row as planes, zeros behind its end and of rows that there are not.
template <int PLANES> __device__ __forceinline__ void few_planes(const float (&e)[8], u32x4 (&out)[PLANES]) {
    uint32_t w[4][PLANES];
#pragma unroll
    for (int j = 0; j < 4; ++j) split2<PLANES, kHalf>(e[2 * j], e[2 * j + 1], w[j]);
#pragma unroll
    for (int q = 0; q < PLANES; ++q) out[q] = u32x4{w[0][q], w[1][q], w[2][q], w[3][q]};
}
// WHOLE: all of the 32 columns that a wave reads are there, and no branch keeps loads from being on their way together.
template <bool WHOLE, class E> __device__ __forceinline__ void few_elements(const E* p, int64_t col, int64_t cols, E (&e)[8]) {
    if constexpr (WHOLE) __builtin_memcpy(e, p + col, sizeof(e));
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = col + j < cols ? p[col + j] : E(0);
    }
}
template <class E> __device__ __forceinline__ void few_operand(const E (&e)[8], u32x4 (&out)[NP]) {
    if constexpr (sizeof(E) == 4) few_planes<NP>(e, out);
    else __builtin_memcpy(&out[0], e, 16);
}
// A row of a matrix; behind its end its last one, of which no result is kept.
__device__ __forceinline__ const Elem* few_row(const Matrix& m, int64_t row) {
    return static_cast<const Elem*>(m.p) + (row < m.rows ? row : m.rows - 1) * m.stride;
}
// Calls f(whole, how many steps, first column) for a wave's share of the steps of 32 columns: four at a time, whose loads are
// all asked for before the first product (few rows leave room for few waves), then one by one.
template <class F> __device__ __forceinline__ void few_steps(int64_t cols, int wave, int waves, F f) {
    using One = std::integral_constant<int, 1>;
    const int64_t steps = cut_into(cols, 32), last = steps * (wave + 1) / waves, full = last * 32 <= cols ? last : last - 1;
    int64_t s = steps * wave / waves;
#pragma unroll 1
    for (; s + 4 <= full; s += 4) f(std::true_type{}, std::integral_constant<int, 4>{}, s * 32);
#pragma unroll 1
    for (; s < full; ++s) f(std::true_type{}, One{}, s * 32);
    if (s < last) f(std::false_type{}, One{}, s * 32);
}

// Products of a wave's fragments: rows of a table are the result's rows, 4 * (lane / 16) ..., its columns the rows of x.
template <int PA, int PB> __device__ __forceinline__ f32x4 few_product(const u32x4 (&table)[PA], const u32x4 (&rows)[PB], f32x4 acc) {
#pragma unroll
    for (int rank = (PA > PB ? PA : PB) - 1; rank >= 0; --rank)
#pragma unroll
        for (int p = 0; p < PA; ++p)
            if (rank - p >= 0 && rank - p < PB) acc = mfma<kHalf>(table[p], rows[rank - p], acc);
    return acc;
}

__device__ __forceinline__ float gate_value(int activation, float g) {
    return activation == FSA_ACT_SILU ? gate_of<FSA_ACT_SILU>(g).value
         : activation == FSA_ACT_GELU ? gate_of<FSA_ACT_GELU>(g).value : gate_of<FSA_ACT_RELU>(g).value;
}

template <int MT> __global__ __launch_bounds__(64 * kFewWaves) void few_hidden_kernel(FewArgs a) {
    __shared__ f32x4 lds[2 * MT * (kFewWaves - 1) * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, q = lane >> 4;
    const int64_t row = (int64_t)blockIdx.x * 16 + r16;
    const Elem *gates = few_row(a.gate, row), *ups = few_row(a.up, row), *xs[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xs[t] = few_row(a.x, 16 * t + r16);
    f32x4 g[MT] = {}, u[MT] = {};
    few_steps(a.D, wave, kFewWaves, [&](auto whole, auto count, int64_t first) {
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr int N = decltype(count)::value;
        Elem ge[N][8], ue[N][8], xe[N][MT][8];
#pragma unroll
        for (int s = 0; s < N; ++s) {
            const int64_t col = first + 32 * s + 8 * q;
            few_elements<WHOLE>(gates, col, a.D, ge[s]);
            few_elements<WHOLE>(ups, col, a.D, ue[s]);
#pragma unroll
            for (int t = 0; t < MT; ++t) few_elements<WHOLE>(xs[t], col, a.D, xe[s][t]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < N; ++s) {
            u32x4 gate[NP], up[NP], x[NP];
            few_operand(ge[s], gate);
            few_operand(ue[s], up);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                few_operand(xe[s][t], x);
                g[t] = few_product(gate, x, g[t]);
                u[t] = few_product(up, x, u[t]);
            }
        }
    });
#pragma unroll
    for (int t = 0; t < MT; ++t)
        if (wave > 0) { lds[((wave - 1) * MT + t) * 128 + lane] = g[t]; lds[((wave - 1) * MT + t) * 128 + 64 + lane] = u[t]; }
    __syncthreads();
    if (wave > 0) return;
    float top = 0.0f;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int w = 0; w < kFewWaves - 1; ++w) { g[t] += lds[(w * MT + t) * 128 + lane]; u[t] += lds[(w * MT + t) * 128 + 64 + lane]; }
        const int64_t m = 16 * t + r16;
        if (m >= a.T) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = (int64_t)blockIdx.x * 16 + 4 * q + j;
            if (n >= a.H) continue;
            const float h = gate_value(a.activation, g[t][j]) * u[t][j];
            a.h[m * a.H + n] = h;
            if (kHalf && fabsf(h) < __builtin_inff()) top = fmaxf(top, fabsf(h));
        }
    }
    if constexpr (kHalf) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
        if (lane == 0) a.peaks[blockIdx.x] = top;
    }
}
// The power of two beside which few rows' h is split into planes, from the largest of all workgroups: asked for first, and found once the first
// tables' elements are on their way.
struct NoLift {
    static constexpr int lift = 0;
    __device__ __forceinline__ explicit NoLift(const FewArgs&) {}
    __device__ __forceinline__ void find() {}
};
struct FewLift {
    static constexpr int N = 4;
    float top[N];
    int lift = 1000;
    __device__ __forceinline__ explicit FewLift(const FewArgs& a) {
        const int64_t count = cut_into(a.H, 16);
#pragma unroll
        for (int i = 0; i < N; ++i) top[i] = (int)(threadIdx.x & 63) + 64 * i < count ? a.peaks[(threadIdx.x & 63) + 64 * i] : 0.0f;
        for (int64_t i = (threadIdx.x & 63) + 64 * N; i < count; i += 64) top[0] = fmaxf(top[0], a.peaks[i]);
    }
    __device__ __forceinline__ void find() {
        if (lift != 1000) return;
        float all = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
#pragma unroll
        for (int d = 1; d < 64; d *= 2) all = fmaxf(all, __shfl_xor(all, d, 64));
        lift = __builtin_amdgcn_readfirstlane(lift_to_end(all));
    }
};

template <int MT> __global__ __launch_bounds__(64 * kFewAnswerWaves) void few_answer_kernel(FewArgs a) {
    __shared__ f32x4 lds[MT * kFewAnswerWaves * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, q = lane >> 4;
    const Elem* downs = few_row(a.down, (int64_t)blockIdx.x * 16 + r16);
    const float* hs[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) hs[t] = a.h + (16 * t + r16 < a.T ? 16 * t + r16 : a.T - 1) * a.H;
    f32x4 acc[MT] = {};
    typename std::conditional<kHalf, FewLift, NoLift>::type lift(a);
    few_steps(a.H, wave, kFewAnswerWaves, [&](auto whole, auto count, int64_t first) {
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr int N = decltype(count)::value;
        Elem de[N][8];
        float he[N][MT][8];
#pragma unroll
        for (int s = 0; s < N; ++s) {
            const int64_t col = first + 32 * s + 8 * q;
            few_elements<WHOLE>(downs, col, a.H, de[s]);
#pragma unroll
            for (int t = 0; t < MT; ++t) few_elements<WHOLE>(hs[t], col, a.H, he[s][t]);
        }
        __builtin_amdgcn_sched_barrier(0);
        lift.find();
        const float up = power_of_two(lift.lift);
#pragma unroll
        for (int s = 0; s < N; ++s) {
            u32x4 down[NP], h[kHeld];
            few_operand(de[s], down);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (kHalf) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) he[s][t][j] *= up;
                }
                few_planes<kHeld>(he[s][t], h);
                acc[t] = few_product(down, h, acc[t]);
            }
        }
    });
#pragma unroll
    for (int t = 0; t < MT; ++t) lds[(wave * MT + t) * 64 + lane] = acc[t];
    __syncthreads();
    lift.find();                                        // (a wave without a share has not)
    const float back = power_of_two(-lift.lift);
    // a sum a thread: 256 of each 16 rows
    for (int i = threadIdx.x; i < MT * 256; i += 64 * kFewAnswerWaves) {
        const int t = i >> 8, at = i >> 2 & 63, j = i & 3;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewAnswerWaves; ++w) sum += lds[(w * MT + t) * 64 + at][j];
        const int64_t m = 16 * t + (at & 15), n = (int64_t)blockIdx.x * 16 + 4 * (at >> 4) + j;
        if (m >= a.T || n >= a.O) continue;
        const float one[4] = {kHalf ? sum * back : sum, 0.0f, 0.0f, 0.0f};
        store_row<kKind>(a.y, m * a.O, n, n + 1, false, one);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------------------------
bool on_grid(const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (int64_t)sizeof(Elem) % 16 == 0; }

template <class T, bool FORWARD> hipError_t launch_products(Jobs& l, hipStream_t st) {
    unsigned groups = 0, joins = 0;
    for (int j = 0; j < l.count; ++j) {
        Job& a = l.job[j];
        a.mt = (unsigned)cut_into(a.M, T::BM);
        a.nt = (unsigned)cut_into(a.N, T::BN);
        a.first = groups;
        a.first_join = joins;
        groups += a.mt * a.nt * a.splits * a.results;
        if (a.splits > 1) joins += (unsigned)cut_into(a.M * (a.N8 / 4) * a.results, 256);
    }
    product_kernel<T, FORWARD><<<dim3(groups), dim3(T::THREADS), 0, st>>>(l);
    if (hipError_t e = hipGetLastError()) return e;
    if (joins) {
        // (jobs without splits have no workgroup: the next job's start is theirs)
        Jobs k = l;
        k.count = 0;
        for (int j = 0; j < l.count; ++j) if (l.job[j].splits > 1) k.job[k.count++] = l.job[j];
        join_kernel<<<dim3(joins), dim3(256), 0, st>>>(k);
    }
    return hipGetLastError();
}
// `l` has everything but cuts and places.
template <bool FORWARD> hipError_t run_products(const GatedArgs& g, Jobs& l, hipStream_t st) {
    float* parts = reinterpret_cast<float*>(g.ws + g.plan.parts);
    for (int j = 0; j < l.count; ++j) {
        Job& a = l.job[j];
        const ProductJob& plan = g.plan.products.job[a.planned];
        a.splits = (unsigned)plan.splits;
        a.M8 = up_to(a.M, 8); a.N8 = up_to(a.N, 8);
        a.grid = on_grid(a.out[0], a.out_ld) && (a.results == 1 || on_grid(a.out[1], a.out_ld));
        a.parts = parts;
        parts += up_to(plan.parts_bytes(), 256) / 4;
    }
    const int choice = g.plan.products.choice;
    return choice == 2 ? launch_products<Tiles<2>::Product, FORWARD>(l, st)
         : choice == 1 ? launch_products<Tiles<1>::Product, FORWARD>(l, st) : launch_products<Tiles<0>::Product, FORWARD>(l, st);
}

template <int CHOICE, int ACT, int PLANES> hipError_t launch_pair(HiddenArgs a, bool forward, hipStream_t st) {
    using Hidden = typename Tiles<CHOICE>::Hidden;
    using Slopes = typename Tiles<CHOICE>::Slopes;
    using Kept = typename Tiles<CHOICE>::Product;
    const int bm = forward ? Hidden::BM : a.kept ? Kept::BM : Slopes::BM, bn = forward ? Hidden::BN : a.kept ? Kept::BN : Slopes::BN;
    a.mt = (unsigned)cut_into(a.T, bm);
    a.nt = (unsigned)cut_into(a.H, bn);
    const dim3 grid(a.mt * a.nt);
    if (forward) hidden_kernel<Hidden, ACT, PLANES><<<grid, dim3(Hidden::THREADS), 0, st>>>(a);
    else if (a.kept) slopes_kernel<Kept, ACT, PLANES, true><<<grid, dim3(Kept::THREADS), 0, st>>>(a);
    else slopes_kernel<Slopes, ACT, PLANES, false><<<grid, dim3(Slopes::THREADS), 0, st>>>(a);
    return hipGetLastError();
}
template <int CHOICE, int ACT> hipError_t by_planes(const HiddenArgs& a, int planes, bool forward, hipStream_t st) {
    if constexpr (NP == 1) if (planes == 2) return launch_pair<CHOICE, ACT, 2>(a, forward, st);
    return launch_pair<CHOICE, ACT, NP>(a, forward, st);
}
template <int ACT> hipError_t by_choice(const GatedPlan& p, const HiddenArgs& a, bool forward, hipStream_t st) {
    const int choice = forward ? p.pairs : p.slopes;
    return choice == 2 ? by_planes<2, ACT>(a, p.planes, forward, st)
         : choice == 1 ? by_planes<1, ACT>(a, p.planes, forward, st) : by_planes<0, ACT>(a, p.planes, forward, st);
}
hipError_t run_pair(const GatedArgs& g, const HiddenArgs& a, bool forward, hipStream_t st) {
    return g.activation == FSA_ACT_SILU ? by_choice<FSA_ACT_SILU>(g.plan, a, forward, st)
         : g.activation == FSA_ACT_GELU ? by_choice<FSA_ACT_GELU>(g.plan, a, forward, st) : by_choice<FSA_ACT_RELU>(g.plan, a, forward, st);
}

struct Operands { Side x, gate, up, down, grad_y; };

// Lays out what products cannot read in place, and looks for the first `kinds` of the longest rows.
hipError_t lay_out(const GatedArgs& a, Operands& o, int kinds, hipStream_t st) {
    const Matrix* from[5] = {&a.x, &a.gate, &a.up, &a.down, &a.grad_y};
    Side* to[5] = {&o.x, &o.gate, &o.up, &o.down, &o.grad_y};
    const size_t at[5] = {a.plan.x, a.plan.gate, a.plan.up, a.plan.down, a.plan.grad_y};
    PackList l{};
    for (int i = 0; i < 5; ++i) {
        if (!(a.packs >> i & 1)) {
            *to[i] = {static_cast<const uint16_t*>(from[i]->p), from[i]->stride, 0};
            continue;
        }
        const int64_t ld = up_to(from[i]->cols, 8);
        uint16_t* p = reinterpret_cast<uint16_t*>(a.ws + at[i]);
        *to[i] = {p, ld, from[i]->rows * ld};
        l.from[l.count] = *from[i];
        l.to[l.count] = p;
        l.first[l.count + 1] = l.first[l.count] + from[i]->rows * (ld / 8);
        ++l.count;
    }
    const int64_t blocks = cut_into(l.first[l.count], 256);
    l.packers = (unsigned)(blocks < 8192 ? blocks : 8192);
    const Matrix* measured[kPeakKinds] = {&a.x, &a.gate, &a.up, &a.grad_y, &a.down};
    for (int k = 0; k < kinds; ++k) l.measured[k] = *measured[k];
    l.peaks = reinterpret_cast<float*>(a.ws + a.plan.peaks);
    const unsigned groups = l.packers + kinds * kGatedPeaks;
    if (groups == 0) return hipSuccess;
    pack_kernel<<<dim3(groups), dim3(256), 0, st>>>(l);
    return hipGetLastError();
}

HiddenArgs hidden_args(const GatedArgs& a, const Operands& o) {
    HiddenArgs h{};
    h.x = o.x; h.gate = o.gate; h.up = o.up; h.down = o.down; h.grad_y = o.grad_y;
    h.at = kept_plan(a.s);
    h.h = reinterpret_cast<uint16_t*>(a.kept ? a.kept + h.at.h : a.ws + a.plan.h);
    h.dg = reinterpret_cast<uint16_t*>(a.ws + a.plan.dg);
    h.du = reinterpret_cast<uint16_t*>(a.ws + a.plan.du);
    h.kept = a.kept;
    h.T = a.s.T; h.D = a.s.D; h.H = a.s.H; h.O = a.s.O; h.H8 = a.plan.H8;
    h.peaks = reinterpret_cast<const float*>(a.ws + a.plan.peaks);
    return h;
}

// Pairs whose products' sum is that of all planes of `held` (h, dg or du) with `other`; fp32's planes belong to one pair.
void add_pairs(Job& j, int result, int& pairs, const GatedPlan& p, Side held, const Side& other, bool held_first) {
    for (int q = 0; q < (NP == 1 ? p.planes : 1); ++q) {
        j.a[result][pairs] = held_first ? held : other;
        j.b[result][pairs] = held_first ? other : held;
        held.p += held.plane;
        ++pairs;
    }
}

template <int MT> hipError_t launch_few(const FewArgs& f, hipStream_t st) {
    few_hidden_kernel<MT><<<dim3((unsigned)cut_into(f.H, 16)), dim3(64 * kFewWaves), 0, st>>>(f);
    if (hipError_t e = hipGetLastError()) return e;
    few_answer_kernel<MT><<<dim3((unsigned)cut_into(f.O, 16)), dim3(64 * kFewAnswerWaves), 0, st>>>(f);
    return hipGetLastError();
}

hipError_t forward(const GatedArgs& a, hipStream_t st) {
    if (gated_few(a.s) && !a.kept) {
        const FewArgs f{a.x, a.gate, a.up, a.down, reinterpret_cast<float*>(a.ws + a.plan.h), reinterpret_cast<float*>(a.ws + a.plan.peaks), a.y, a.s.T, a.s.D, a.s.H, a.s.O, a.activation};
        if constexpr (kKind == 0) if (a.s.T > 16) return launch_few<2>(f, st);
        return launch_few<1>(f, st);
    }
    Operands o{};
    if (hipError_t e = lay_out(a, o, kHalf ? kPeakGradY : 0, st)) return e;
    const HiddenArgs h = hidden_args(a, o);
    if (hipError_t e = run_pair(a, h, true, st)) return e;
    Jobs l{};
    l.count = 1;
    l.peaks = h.peaks;
    Job& j = l.job[0];
    add_pairs(j, 0, j.pairs, a.plan, {h.h, h.H8, a.s.T * h.H8}, o.down, true);
    j.results = 1;
    j.out[0] = a.y;
    j.M = a.s.T; j.N = a.s.O; j.K = a.s.H; j.out_ld = a.s.O;
    j.adeep = true;
    j.lift = kLiftH;
    return run_products<true>(a, l, st);
}

hipError_t backward(const GatedArgs& a, hipStream_t st) {
    void* const outs[4] = {a.grad_gate, a.grad_up, a.grad_down, a.grad_x};
    if (a.s.T == 0) {
        const int64_t sizes[3] = {a.s.H * a.s.D, a.s.H * a.s.D, a.s.O * a.s.H};
        for (int i = 0; i < 3; ++i)
            if (outs[i]) {
                const int64_t blocks = cut_into(sizes[i], 256);
                zero_kernel<<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st>>>(static_cast<Elem*>(outs[i]), sizes[i]);
                if (hipError_t e = hipGetLastError()) return e;
            }
        return hipSuccess;
    }
    if (!outs[0] && !outs[1] && !outs[2] && !outs[3]) return hipSuccess;
    Operands o{};
    if (hipError_t e = lay_out(a, o, kHalf ? kPeakKinds : 0, st)) return e;
    const HiddenArgs h = hidden_args(a, o);
    if (hipError_t e = run_pair(a, h, false, st)) return e;
    const int64_t plane = a.s.T * h.H8;
    const Side hs = {h.h, h.H8, plane}, dg = {h.dg, h.H8, plane}, du = {h.du, h.H8, plane};
    Jobs l{};
    l.peaks = h.peaks;
    if (a.grad_gate || a.grad_up) {
        Job& j = l.job[l.count++];
        for (int i = 0; i < 2; ++i)
            if (outs[i]) {
                j.pairs = 0;
                add_pairs(j, j.results, j.pairs, a.plan, i == 0 ? dg : du, o.x, true);
                j.out[j.results++] = outs[i];
            }
        j.M = a.s.H; j.N = a.s.D; j.K = a.s.T; j.out_ld = a.s.D;
        j.lift = kLiftD;
        j.planned = kJobGates;
    }
    if (a.grad_down) {
        Job& j = l.job[l.count++];
        j.planned = kJobDown;
        j.lift = kLiftH;
        add_pairs(j, 0, j.pairs, a.plan, hs, o.grad_y, false);
        j.results = 1;
        j.out[0] = a.grad_down;
        j.M = a.s.O; j.N = a.s.H; j.K = a.s.T; j.out_ld = a.s.H;
    }
    if (a.grad_x) {
        Job& j = l.job[l.count++];
        add_pairs(j, 0, j.pairs, a.plan, dg, o.gate, true);
        add_pairs(j, 0, j.pairs, a.plan, du, o.up, true);
        j.results = 1;
        j.out[0] = a.grad_x;
        j.M = a.s.T; j.N = a.s.D; j.K = a.s.H; j.out_ld = a.s.D;
        j.adeep = true;
        j.lift = kLiftD;
        j.planned = kJobX;
    }
    return run_products<false>(a, l, st);
}

}  // namespace
}  // namespace fsa
#endif
