// Matrix products of 16-bit planes on the matrix cores: the tile that the gated feed-forward block and the orthogonalised
// update are made of.  Device code only; what a tile is written out as is its kernel's own.
//
//   C[m,n] = sum_k A[m,k] B[n,k]
//
// An operand is one plane of bfloat16 or fp16, or several whose sum it is: three bfloat16 planes hold the 24 bits of an fp32
// element (in its whole range), two fp16 planes 23 bits of a bounded one.  Of the products of planes those that matter to
// fp32 are made, smallest first: 6 of 9, 3 of 4.
//
// A workgroup makes BM x BN of C (of `PARTS` products with one A, side by side).  Planes go to LDS without passing registers
// (16 bytes a lane), two steps of BK deep; a wave reads fragments of its WM x WN share and keeps the sums in registers.  An
// operand lies in memory with its depth k contiguous ("deep") or with its rows contiguous ("flat"): a flat one is transposed
// as it is read from LDS.
#pragma once

#include "fsa_device.hip.h"

namespace fsa {
namespace product {

using f32x4 = __attribute__((ext_vector_type(4))) float;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using s16x4 = __attribute__((ext_vector_type(4))) short;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using lds_void = __attribute__((address_space(3))) void;

constexpr uint32_t kNowhere = 0x80000000u;              // an offset that a buffer read answers with zeros
constexpr int kMostBytes = 0x7fffffff;

// An operand as a launch takes it: element (r, k) of plane p at p + p * plane + r * ld + k (deep) or k * ld + r (flat).  Every
// stretch of contiguous elements starts on the 16-byte grid, and what follows its end up to a multiple of 8 elements is zero.
struct Side {
    const uint16_t* p;
    int64_t ld, plane;
};

// BN of each part; WGM x WGN waves.
template <int NP_, bool HALF_, int BM_, int BN_, int BK_, int WGM_, int WGN_> struct Tile {
    static constexpr int NP = NP_, BM = BM_, BN = BN_, BK = BK_, WGM = WGM_, WGN = WGN_;
    static constexpr bool HALF = HALF_;
    static constexpr int THREADS = 64 * WGM * WGN, MI = BM / WGM / 16, NJ = BN / WGN / 16;
    static_assert(BM % (16 * WGM) == 0 && BN % (16 * WGN) == 0 && (BK == 32 || BK == 64), "whole fragments");
    static constexpr int stage_bytes(int parts) { return (BM + parts * BN) * BK * 2 * NP; }
    static constexpr int lds_bytes(int parts) { return 2 * stage_bytes(parts); }
};

// Chunk (8 elements, 16 bytes) c of a row lies at chunk c ^ turn of that row, so that what a wave reads at a time lies on
// different banks (64 of 4 bytes).  Deep: 16 rows of one chunk; `r16` is the row's place in its fragment.
template <int BK> __device__ __forceinline__ int turn_deep(int r16) { return BK == 64 ? (r16 >> 1) & 7 : (r16 >> 2) & 3; }
// Flat: rows are steps of k, R elements long; a read takes four of them, and four pieces of 4 elements, 4 * NJ apart (NJ 1: side by
// side, and eight rows).
template <int R, int NJ> __device__ __forceinline__ int turn_flat(int k) {
    if constexpr (NJ == 1) return R >= 128 ? 2 * ((k & 3) | (k >> 1 & 4)) : 2 * ((k >> 1 & 1) | (k >> 2 & 2));
    else if constexpr (NJ == 2) return R >= 128 ? 4 * (k & 3) : 4 * (k >> 1 & 1);
    else return R >= 128 ? (k & 1) + 8 * (k >> 1 & 1) : k >> 1 & 1;
}

template <bool HALF> __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (HALF)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Brings R rows of an operand, BK deep, to LDS, step by step.  NJ: how a fragment's rows lie (1: 16 side by side, else four
// fours 4 * NJ apart, see Reader).
template <class T, int R, bool DEEP, int NJ> struct Feed {
    static constexpr int N = R * T::BK / 8 / T::THREADS;    // 16-byte pieces a thread and plane
    static_assert(N >= 1 && N * 8 * T::THREADS == R * T::BK, "whole pieces");
    static constexpr int PLANE = R * T::BK * 2, BYTES = PLANE * T::NP;
    static constexpr int ROW = DEEP ? T::BK / 8 : R / 8;    // chunks of a row in LDS
    const char* at;
    int64_t plane, step;
    uint32_t off[N];
    int depth[N];                                           // of the piece within a step
    int wave;

    // Rows from r0 on, `rows` of them in all (up to a multiple of 8 where flat), from depth k0 on.
    __device__ __forceinline__ Feed(const Side& s, int64_t r0, int64_t rows, int64_t k0) {
        const int tid = threadIdx.x;
        wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        at = reinterpret_cast<const char*>(s.p + (DEEP ? r0 * s.ld + k0 : k0 * s.ld + r0));
        plane = s.plane * 2;
        step = DEEP ? T::BK * 2 : s.ld * T::BK * 2;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int slot = i * T::THREADS + tid, row = slot / ROW, c = slot % ROW;
            if constexpr (DEEP) {
                const int r16 = (row & 3) | (row / (4 * NJ) & 3) << 2;
                depth[i] = 8 * (c ^ turn_deep<T::BK>(r16));
                off[i] = r0 + row < rows ? (uint32_t)(row * s.ld * 2 + depth[i] * 2) : kNowhere;
            } else {
                depth[i] = row;
                const int r = 8 * (c ^ turn_flat<R, NJ>(row));
                off[i] = r0 + r < rows ? (uint32_t)(row * s.ld * 2 + r * 2) : kNowhere;
            }
        }
    }
    // Asks for one step of which `left` (at least 1) of the depth is there, and moves on to the next.
    __device__ __forceinline__ void ask(char* lds, int64_t left) {
#pragma unroll
        for (int p = 0; p < T::NP; ++p) {
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at + p * plane), 0, kMostBytes, 0x00020000);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint32_t o = off[i];
                if (left < T::BK && depth[i] >= left) o = kNowhere;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(lds + p * PLANE + (i * T::THREADS + wave * 64) * 16), 16,
                                                         (int)o, 0, 0, 0);
            }
        }
        at += step;
    }
};

// Reads fragments of 16 rows x 32 of depth: lane l has depth 8 * (l / 16) ... + 7 of the fragment's row l % 16.
//   NJ 1    fragment f holds rows first + 16 f ... + 15
//   NJ > 1  its row 4 q + i is row first + 4 NJ q + 4 f + i of the tile: of a result whose rows these are, a lane then has
//           4 NJ side by side
template <class T, int R, bool DEEP, int NJ, int FRAGS> struct Reader {
    int lane_at[DEEP ? T::BK / 32 : NJ == 1 ? FRAGS : (FRAGS + 1) / 2];
    __device__ __forceinline__ explicit Reader(int first) {
        const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4;
        if constexpr (DEEP) {
            const int row = first + (NJ == 1 ? r16 : (r16 >> 2) * 4 * NJ + (r16 & 3));
#pragma unroll
            for (int kk = 0; kk < T::BK / 32; ++kk) lane_at[kk] = row * T::BK * 2 + ((4 * kk + q) ^ turn_deep<T::BK>(r16)) * 16;
        } else {
            const int k = 8 * q + (r16 >> 2), piece = r16 & 3;
#pragma unroll
            for (int f = 0; f < (int)(sizeof(lane_at) / sizeof(int)); ++f) {
                const int r = first + (NJ == 1 ? 16 * f + 4 * piece : 4 * NJ * piece + 8 * f);
                lane_at[f] = k * R * 2 + ((r >> 3) ^ turn_flat<R, NJ>(k)) * 16 + (r & 4) * 2;
            }
        }
    }
    __device__ __forceinline__ u32x4 get(const char* plane, int kk, int f) const {
        if constexpr (DEEP) {
            return *reinterpret_cast<const u32x4*>(plane + lane_at[kk] + f * (NJ == 1 ? 16 : 4) * T::BK * 2);
        } else {
            using lds_s16x4 = __attribute__((address_space(3))) s16x4;
            const char* p = plane + (NJ == 1 ? lane_at[f] : lane_at[f / 2] + 8 * (f & 1)) + kk * 32 * R * 2;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * R * 2)));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

// What a workgroup brought so far is whole in LDS, and every wave is done with the step before.
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Sums of a wave: acc[part][mi][nj][i] belongs to row 16 mi + lane % 16 of the wave's rows and to column
// 4 NJ (lane / 16) + 4 nj + i of its columns.
template <class T, int PARTS> using Sums = f32x4[PARTS][T::MI][T::NJ];

// Adds the product of rows m0 ... of A and rows n0 ... of every part of B, over the depth [k0, k1).
template <class T, bool ADEEP, bool BDEEP, int PARTS>
__device__ __forceinline__ void accumulate(Sums<T, PARTS>& acc, char* lds, const Side& a, const Side (&b)[PARTS], int64_t m0, int64_t M,
                                           int64_t n0, int64_t N, int64_t k0, int64_t k1) {
    using FeedA = Feed<T, T::BM, ADEEP, 1>;
    using FeedB = Feed<T, T::BN, BDEEP, T::NJ>;
    constexpr int STAGE = T::stage_bytes(PARTS);
    static_assert(STAGE == FeedA::BYTES + PARTS * FeedB::BYTES, "");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / T::WGN, wn = wave % T::WGN;
    if (k0 >= k1) return;
    FeedA fa(a, m0, M, k0);
    FeedB fb0(b[0], n0, N, k0), fb1(b[PARTS - 1], n0, N, k0);
    const Reader<T, T::BM, ADEEP, 1, T::MI> ra(wm * 16 * T::MI);
    const Reader<T, T::BN, BDEEP, T::NJ, T::NJ> rb(wn * 16 * T::NJ);
    auto ask = [&](int stage, int64_t left) {
        char* at = lds + stage * STAGE;
        fa.ask(at, left);
        fb0.ask(at + FeedA::BYTES, left);
        if constexpr (PARTS == 2) fb1.ask(at + FeedA::BYTES + FeedB::BYTES, left);
    };
    ask(0, k1 - k0);
    int stage = 0;
#pragma unroll 1
    for (int64_t k = k0; k < k1; k += T::BK) {
        meet();
        if (k + T::BK < k1) ask(stage ^ 1, k1 - k - T::BK);
        const char* at = lds + stage * STAGE;
#pragma unroll
        for (int kk = 0; kk < T::BK / 32; ++kk) {
            u32x4 fragA[T::NP][T::MI], fragB[T::NP][PARTS][T::NJ];
#pragma unroll
            for (int p = 0; p < T::NP; ++p) {
#pragma unroll
                for (int y = 0; y < PARTS; ++y)
#pragma unroll
                    for (int j = 0; j < T::NJ; ++j)
                        fragB[p][y][j] = rb.get(at + FeedA::BYTES + y * FeedB::BYTES + p * FeedB::PLANE, kk, j);
#pragma unroll
                for (int i = 0; i < T::MI; ++i) fragA[p][i] = ra.get(at + p * FeedA::PLANE, kk, i);
            }
#pragma unroll
            for (int rank = T::NP - 1; rank >= 0; --rank)       // planes' products of one magnitude, the smallest first
#pragma unroll
                for (int p = 0; p <= rank; ++p)
#pragma unroll
                    for (int y = 0; y < PARTS; ++y)
#pragma unroll
                        for (int i = 0; i < T::MI; ++i)
#pragma unroll
                            for (int j = 0; j < T::NJ; ++j)
                                acc[y][i][j] = mfma<T::HALF>(fragB[rank - p][y][j], fragA[p][i], acc[y][i][j]);
        }
        stage ^= 1;
    }
    meet();                                                 // the next product may ask for its first step
}

// Calls f(part-independent m, n, columns) for every stretch of 4 NJ columns that this lane has: m the row, n the first column.
template <class T, class F> __device__ __forceinline__ void each_stretch(int64_t m0, int64_t n0, F f) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / T::WGN, wn = wave % T::WGN, lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < T::MI; ++i)
        f(i, m0 + wm * 16 * T::MI + 16 * i + (lane & 15), n0 + wn * 16 * T::NJ + 4 * T::NJ * (lane >> 4));
}

// ---------------------------------------------------------------------------------------------------------------
// elements and planes
// ---------------------------------------------------------------------------------------------------------------
template <bool HALF> __device__ __forceinline__ uint32_t pack2(float a, float b) {     // nearest even
    if constexpr (HALF) {
        using v2 = __attribute__((ext_vector_type(2))) _Float16;
        return __builtin_bit_cast(uint32_t, v2{(_Float16)a, (_Float16)b});
    } else {
        using v2 = __attribute__((ext_vector_type(2))) __bf16;
        return __builtin_bit_cast(uint32_t, v2{(__bf16)a, (__bf16)b});
    }
}
template <bool HALF> __device__ __forceinline__ float as_float(uint32_t bits) {        // of the low half
    if constexpr (HALF) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    else return __builtin_bit_cast(float, bits << 16);
}

// Planes of two elements, one word each.  Three bfloat16 planes: the first is cut off rather than rounded, so that the largest
// fp32 numbers stay finite; an infinity has no rest, a NaN stays one.  Two fp16 planes: nearest, of elements in range.
template <int NP, bool HALF> __device__ __forceinline__ void split2(float a, float b, uint32_t (&out)[NP]) {
    if constexpr (NP == 1) out[0] = pack2<HALF>(a, b);
    else if constexpr (NP == 2) {
        out[0] = pack2<HALF>(a, b);
        out[1] = pack2<HALF>(a - as_float<HALF>(out[0] & 0xffff), b - as_float<HALF>(out[0] >> 16));
    } else {
        static_assert(!HALF, "");
        uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
        float ra = a - __builtin_bit_cast(float, x & 0xffff0000u), rb = b - __builtin_bit_cast(float, y & 0xffff0000u);
        if (!(fabsf(a) < __builtin_inff())) { ra = 0.0f; x |= a != a ? 0x00400000u : 0u; }
        if (!(fabsf(b) < __builtin_inff())) { rb = 0.0f; y |= b != b ? 0x00400000u : 0u; }
        out[0] = x >> 16 | (y & 0xffff0000u);
        out[1] = pack2<false>(ra, rb);
        out[2] = pack2<false>(ra - as_float<false>(out[1] & 0xffff), rb - as_float<false>(out[1] >> 16));
    }
}

// Writes W (a multiple of 4) elements as planes at column n of row m: those at `N` and behind are written as zero up to the next
// multiple of 8, which is as far as a reader of the planes looks.
template <int NP, bool HALF, int W>
__device__ __forceinline__ void store_planes(uint16_t* p, int64_t plane, int64_t at, int64_t n, int64_t N, const float (&x)[W]) {
    const int64_t end = (N + 7) / 8 * 8;
    if (n >= end) return;
    uint32_t w[W / 2][NP];
#pragma unroll
    for (int i = 0; i < W / 2; ++i)
        split2<NP, HALF>(n + 2 * i < N ? x[2 * i] : 0.0f, n + 2 * i + 1 < N ? x[2 * i + 1] : 0.0f, w[i]);
#pragma unroll
    for (int q = 0; q < NP; ++q)
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            if (n + 4 * i >= end) break;
            *reinterpret_cast<u32x2*>(p + q * plane + at + 4 * i) = u32x2{w[2 * i][q], w[2 * i + 1][q]};
        }
}

// Writes W elements of row `row` (its first element at p) from column n on, those before N, in the caller's type.
template <int KIND, int W> __device__ __forceinline__ void store_row(void* p, int64_t row_at, int64_t n, int64_t N, bool grid, const float (&x)[W]) {
    if constexpr (KIND == 0) {
        float* o = static_cast<float*>(p) + row_at + n;
        if (grid && n + W <= N) {
#pragma unroll
            for (int i = 0; i < W; i += 4) *reinterpret_cast<f32x4*>(o + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) if (n + i < N) o[i] = x[i];
        }
    } else {
        uint16_t* o = static_cast<uint16_t*>(p) + row_at + n;
        uint32_t w[W / 2];
#pragma unroll
        for (int i = 0; i < W / 2; ++i) w[i] = pack2<KIND == 2>(x[2 * i], x[2 * i + 1]);
        if (grid && n + W <= N) {
            if constexpr (W % 8 == 0) {
#pragma unroll
                for (int i = 0; i < W / 2; i += 4) *reinterpret_cast<u32x4*>(o + 2 * i) = u32x4{w[i], w[i + 1], w[i + 2], w[i + 3]};
            } else {
#pragma unroll
                for (int i = 0; i < W / 2; i += 2) *reinterpret_cast<u32x2*>(o + 2 * i) = u32x2{w[i], w[i + 1]};
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) if (n + i < N) o[i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
        }
    }
}

// The workgroup's place among mt x nt tiles.  Workgroups are dealt out to the 8 XCDs in turn: those of one XCD take
// neighbouring tiles, column by column of bands of 8 rows of tiles, so that what they read meets in its L2.
__device__ __forceinline__ void tile_of(unsigned id, unsigned mt, unsigned nt, unsigned& m, unsigned& n) {
    const unsigned total = mt * nt, per = total / 8, more = total % 8, xcd = id % 8, at = id / 8;
    const unsigned t = xcd * per + (xcd < more ? xcd : more) + at;
    const unsigned band = t / (8 * nt), first = band * 8, high = mt - first < 8 ? mt - first : 8, in = t - first * nt;
    m = first + in % high;
    n = in / high;
}

}  // namespace product
}  // namespace fsa
