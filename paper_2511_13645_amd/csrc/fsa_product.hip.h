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
// (16 bytes a lane), two steps of BK deep; a wave reads fragments of its share and keeps the sums in registers.  An operand lies
// in memory with its depth k contiguous ("deep") or with its rows contiguous ("flat"): a flat one is transposed as it is read
// from LDS.  What a workgroup asks memory for is one stream of steps over all products that make its tile, so that one's first
// steps are on their way while the one before is multiplied.
//
// Measured, 8192 x 4096 x 4096 bfloat16 on a warm card, deep and deep, deep and flat, flat and flat: 256 x 256 tiles 1395, 1380, 1303
// TFLOP/s (a library product of 8192^3: 1293), 128 x 128 1045, 1010, 1015; all requests at once behind the meeting 910 to 1150
// (every wave's first product waits for all waves' requests), and with requests that the compiler knows of 960 to 1030 where an
// operand is flat (it waits for all of them before any transposing read).
#pragma once

#include "fsa_device.hip.h"

#include <type_traits>

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
    // One half of a step after the other, fragments read half a step ahead; several planes: one step after the other.
    static constexpr bool HALVES = NP == 1 && BK == 64;
    // Waves of a SIMD that LDS has room for, which registers are to leave room for as well.
    static constexpr int waves(int parts) {
        const int w = 160 * 1024 / lds_bytes(parts) * THREADS / 256;
        return w < 4 ? w : 4;
    }
};

// Chunk (8 elements, 16 bytes) c of a row lies at chunk c ^ turn of that row, so that what a wave reads at a time, 256 bytes, lies
// on different banks.  Deep: LDS serves 16 lanes of a 16-byte read together, rows 0-3 and 12-15 of one chunk with rows 4-11 of
// the next; `r16` is the row's place in its fragment.
template <int BK> __device__ __forceinline__ int turn_deep(int r16) {
    return BK == 64 ? (r16 >> 1) & 7 : (r16 >> 3) | (r16 >> 1 & 2) ^ (r16 >> 2 & 2);
}
// Flat: rows are steps of k, R elements long; a read takes rows k ... k + 3 and k + 8 ... k + 11 of them, and of each four pieces of
// 4 elements (8 bytes): side by side (NJ 1), or 4 * NJ elements apart, every other piece from the other half of its chunk.
template <int R, int NJ> __device__ __forceinline__ int turn_flat(int k) {
    if constexpr (NJ == 1) return R >= 128 ? 2 * ((k & 3) | (k >> 1 & 4)) : 2 * ((k >> 1 & 1) | (k >> 2 & 2));
    else if constexpr (NJ == 2) return (R >= 128 ? 4 * (k & 3) : 4 * (k >> 1 & 1)) + (k >> 3 & 1);
    else return (R >= 128 ? (k & 1) + 8 * (k >> 1 & 1) : k >> 1 & 1) + 2 * (k >> 3 & 1);
}

template <bool HALF> __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (HALF)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t first_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

// Asks for 16 bytes a lane, from o + more on in a buffer, to be put side by side to LDS from `to` on.  As assembly because the
// compiler, where it knows of such a request, has every transposing read of LDS wait for all of them; what has to wait does so in
// meet().  It writes no register; one idle cycle lies between M0's writing and its reading.
__device__ __forceinline__ void ask_lds(u32x4 buffer, uint32_t o, uint32_t more, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(to), "v"(o), "s"(buffer), "s"(more) : "memory", "m0");
}

// Brings R rows of an operand, BK deep, to LDS, step by step.  NJ: how a fragment's rows lie (1: 16 side by side, else four
// fours 4 * NJ apart, see Reader).
template <class T, int R, bool DEEP, int NJ> struct Feed {
    static constexpr int PIECES = R * T::BK / 8;            // of 16 bytes, of a plane
    static constexpr int N = (PIECES + T::THREADS - 1) / T::THREADS;
    static constexpr int PLANE = R * T::BK * 2, BYTES = PLANE * T::NP;
    static constexpr int ROW = DEEP ? T::BK / 8 : R / 8;    // chunks of a row in LDS
    static constexpr int LINES = T::THREADS / ROW;          // rows (of LDS) from one of a thread's pieces to the next
    static_assert(PIECES % 64 == 0 && LINES % (DEEP ? 16 * NJ : 16) == 0, "whole waves, and every piece of a thread turned alike");
    const char* at;
    int64_t plane, step;
    uint32_t off, between;
    int line, depth, lines;                                 // deep: rows of the operand from this tile's first on

    // Rows from r0 on, `rows` of them in all (up to a multiple of 8 where flat), from depth k0 on.
    __device__ __forceinline__ void start(const Side& s, int64_t r0, int64_t rows, int64_t k0) {
        const int tid = threadIdx.x, c = tid % ROW;
        line = tid / ROW;
        move(s, r0, k0);
        plane = s.plane * 2;
        step = DEEP ? T::BK * 2 : s.ld * T::BK * 2;
        between = (uint32_t)(LINES * s.ld * 2);
        if constexpr (DEEP) {
            depth = 8 * (c ^ turn_deep<T::BK>((line & 3) | (line / (4 * NJ) & 3) << 2));
            off = (uint32_t)(line * s.ld * 2 + depth * 2);
            lines = rows - r0 < R ? (int)(rows - r0) : R;
        } else {
            depth = line;
            const int r = 8 * (c ^ turn_flat<R, NJ>(line));
            off = r0 + r < rows ? (uint32_t)(line * s.ld * 2 + r * 2) : kNowhere;
        }
    }
    // Another operand that lies like this one.
    __device__ __forceinline__ void move(const Side& s, int64_t r0, int64_t k0) {
        at = reinterpret_cast<const char*>(s.p + (DEEP ? r0 * s.ld + k0 : k0 * s.ld + r0));
    }
    // Asks for piece i of plane p of the step that it is at, of which `left` of the depth is there.
    __device__ __forceinline__ void ask(uint32_t lds, int left, int p, int i) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (PIECES % T::THREADS != 0 && i * T::THREADS + wave * 64 >= PIECES) return;
        const uint64_t base = reinterpret_cast<uint64_t>(at + p * plane);
        uint32_t o = off;
        if constexpr (DEEP) {
            if (line + i * LINES >= lines || depth >= left) o = kNowhere;
        } else if (depth + i * LINES >= left) o = kNowhere;
        ask_lds(u32x4{first_lane((uint32_t)base), first_lane((uint32_t)(base >> 32) & 0xffff), kMostBytes, 0x00020000}, o,
                first_lane(i * between), first_lane(lds + (uint32_t)(p * PLANE + (i * T::THREADS + wave * 64) * 16)));
    }
    __device__ __forceinline__ void next() { at += step; }
};

// Reads fragments of 16 rows x 32 of depth: lane l has depth 8 * (l / 16) ... + 7 of the fragment's row l % 16.
//   NJ 1    fragment f holds rows first + 16 f ... + 15
//   NJ > 1  its row 4 q + i is row first + 4 NJ q + 4 f + i of the tile, of a flat one 4 NJ q + 4 (f ^ q & 1) + i: of a result
//           whose rows these are, a lane then has 4 NJ side by side
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
                const int r = first + (NJ == 1 ? 16 * f + 4 * piece : 4 * NJ * piece + 8 * f + 4 * (piece & 1));
                lane_at[f] = k * R * 2 + ((r >> 3) ^ turn_flat<R, NJ>(k)) * 16 + (r & 4) * 2;
            }
        }
    }
    __device__ __forceinline__ u32x4 get(const char* plane, int kk, int f) const {
        if constexpr (DEEP) {
            return *reinterpret_cast<const u32x4*>(plane + lane_at[kk] + f * (NJ == 1 ? 16 : 4) * T::BK * 2);
        } else {
            using lds_s16x4 = __attribute__((address_space(3))) s16x4;
            const char* p = plane + (NJ == 1 ? lane_at[f] : lane_at[f / 2] ^ 8 * (f & 1)) + kk * 32 * R * 2;
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * R * 2)));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

// Waits until all but `later` of this wave's requests are there and its reads of LDS are done, and for the other waves.
template <int LATER> __device__ __forceinline__ void meet() {
    static_assert(LATER < 64, "");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(LATER) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Both operands of a product, or A and both parts of B.
template <class T, bool ADEEP, bool BDEEP, int PARTS> struct Flow {
    using FeedA = Feed<T, T::BM, ADEEP, 1>;
    using FeedB = Feed<T, T::BN, BDEEP, T::NJ>;
    static constexpr int PA = T::NP * FeedA::N, PB = T::NP * FeedB::N, ASKS = PA + PARTS * PB;
    // requests that every wave makes for a step
    static constexpr int SURE = (FeedA::PIECES % T::THREADS ? 0 : PA) + (FeedB::PIECES % T::THREADS ? 0 : PARTS * PB);
    static_assert(T::stage_bytes(PARTS) == FeedA::BYTES + PARTS * FeedB::BYTES, "");
    FeedA a;
    FeedB b[PARTS];
    int64_t left;                                           // of the depth, from the step on that it is at

    __device__ __forceinline__ void start(const Side& sa, const Side (&sb)[PARTS], int64_t m0, int64_t M, int64_t n0, int64_t N,
                                          int64_t k0, int64_t k1) {
        a.start(sa, m0, M, k0);
#pragma unroll
        for (int y = 0; y < PARTS; ++y) b[y].start(sb[y], n0, N, k0);
        left = k1 - k0;
    }
    __device__ __forceinline__ void ask(uint32_t stage, int piece) const {
        const int here = left < T::BK ? (int)left : T::BK;
        if (piece < PA) a.ask(stage, here, piece / FeedA::N, piece % FeedA::N);
        else {
            const int y = (piece - PA) / PB, at = (piece - PA) % PB;
            b[y].ask(stage + FeedA::BYTES + y * FeedB::BYTES, here, at / FeedB::N, at % FeedB::N);
        }
    }
    __device__ __forceinline__ void next() {
        a.next();
#pragma unroll
        for (int y = 0; y < PARTS; ++y) b[y].next();
        left = left > T::BK ? left - T::BK : 0;
    }
};

// Sums of a wave: acc[part][mi][nj][i] belongs to row 16 mi + lane % 16 of the wave's rows and to column
// 4 NJ (lane / 16) + 4 nj + i of its columns.
template <class T, int PARTS> using Sums = f32x4[PARTS][T::MI][T::NJ];

// What all products of a workgroup ask for is one stream: `Stream` has ask(stage, piece) for a step's pieces 0 ... ASKS - 1, next(),
// and SURE, the requests that every wave makes for any of its steps.  Behind its last step it asks for nothing, which takes no
// memory traffic and lets the loops go without a branch: the requests are made, all of them out of range.
template <class T, int STAGE, class Stream> struct Ring {
    char* lds;
    Stream& stream;
    int at = 0;                                             // stage that holds the step to be multiplied next

    __device__ __forceinline__ const char* stage(int ahead) const { return lds + (at ^ ahead) * STAGE; }
    __device__ __forceinline__ void ask(int ahead, int piece) { stream.ask((uint32_t)(uintptr_t)(lds_void*)lds + (at ^ ahead) * STAGE, piece); }
    __device__ __forceinline__ void fill() {                // before the first product
#pragma unroll 1
        for (int s = 0; s < (T::HALVES ? 2 : 1); ++s) {
#pragma unroll
            for (int i = 0; i < Stream::ASKS; ++i) ask(s, i);
            stream.next();
        }
    }
    // Waits for all steps asked for but the last `STEPS`.
    template <int STEPS> __device__ __forceinline__ void wait() const { meet<STEPS * Stream::SURE>(); }
    __device__ __forceinline__ void move() { at ^= 1; }
    // After the last product: LDS is no wave's any more once a workgroup has ended, and requests would still write to it.
    __device__ __forceinline__ void end() const { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
};

// Adds the product of a tile of A with every part of B over `steps` steps of the ring.  With a flat B, sums are for settle() to
// put in order.
template <class T, bool ADEEP, bool BDEEP, int PARTS, int STAGE, class Stream>
__device__ __forceinline__ void accumulate(Sums<T, PARTS>& acc, Ring<T, STAGE, Stream>& ring, int64_t steps) {
    using F = Flow<T, ADEEP, BDEEP, PARTS>;
    static_assert(T::stage_bytes(PARTS) <= STAGE, "");
    if (steps <= 0) return;
    constexpr int ASKS = Stream::ASKS, COLS = PARTS * T::NJ;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / T::WGN, wn = wave % T::WGN;
    const Reader<T, T::BM, ADEEP, 1, T::MI> ra(wm * 16 * T::MI);
    const Reader<T, T::BN, BDEEP, T::NJ, T::NJ> rb(wn * 16 * T::NJ);
    auto fragA = [&](const char* stage, int p, int kk, int i) { return ra.get(stage + p * F::FeedA::PLANE, kk, i); };
    auto fragB = [&](const char* stage, int p, int c, int kk) {
        return rb.get(stage + F::FeedA::BYTES + c / T::NJ * F::FeedB::BYTES + p * F::FeedB::PLANE, kk, c % T::NJ);
    };
    if constexpr (T::HALVES) {
        // A wave's matrix instructions of half a step go row of fragments by row; once a row's are issued, the row's fragment of the
        // next half takes its place, and the fragments of B have two places.  What a step asks for is spread over its second half,
        // once all waves have read its stage: no wave's first product waits for all waves' requests.
        // The last step is like any other: what it reads and asks for is the next product's, or no one's.
        u32x4 rowsA[T::MI], colsB[2][COLS];
        auto half = [&](auto which, const char* from, int kk) {
            constexpr int WHICH = decltype(which)::value;
#pragma unroll
            for (int i = 0; i < T::MI; ++i) {
#pragma unroll
                for (int c = 0; c < COLS; ++c)
                    acc[c / T::NJ][i][c % T::NJ] = mfma<T::HALF>(colsB[WHICH][c], rowsA[i], acc[c / T::NJ][i][c % T::NJ]);
                __builtin_amdgcn_sched_barrier(0);
                rowsA[i] = fragA(from, 0, kk, i);
#pragma unroll
                for (int c = i * COLS / T::MI; c < (i + 1) * COLS / T::MI; ++c) colsB[WHICH ^ 1][c] = fragB(from, 0, c, kk);
                if constexpr (WHICH == 1) {
#pragma unroll
                    for (int a = i * ASKS / T::MI; a < (i + 1) * ASKS / T::MI; ++a) ring.ask(0, a);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        ring.template wait<1>();
#pragma unroll
        for (int i = 0; i < T::MI; ++i) rowsA[i] = fragA(ring.stage(0), 0, 0, i);
#pragma unroll
        for (int c = 0; c < COLS; ++c) colsB[0][c] = fragB(ring.stage(0), 0, c, 0);
#pragma unroll 1
        for (; steps > 0; --steps) {
            half(std::integral_constant<int, 0>{}, ring.stage(0), 1);
            ring.template wait<0>();
            half(std::integral_constant<int, 1>{}, ring.stage(1), 0);
            ring.stream.next();
            ring.move();
        }
    } else {
        constexpr int KK = T::BK / 32, RANKS = T::NP * (T::NP + 1) / 2, TURNS = KK * RANKS * T::MI;
#pragma unroll 1
        for (; steps > 0; --steps) {
            ring.template wait<0>();
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                u32x4 a[T::NP][T::MI], b[T::NP][COLS];
#pragma unroll
                for (int r = 0; r < T::NP; ++r) {           // in the order that products want them
                    const int p = r % 2 ? r / 2 : T::NP - 1 - r / 2;
#pragma unroll
                    for (int i = 0; i < T::MI; ++i) a[p][i] = fragA(ring.stage(0), p, kk, i);
#pragma unroll
                    for (int c = 0; c < COLS; ++c) b[T::NP - 1 - p][c] = fragB(ring.stage(0), T::NP - 1 - p, c, kk);
                }
#pragma unroll
                for (int rank = T::NP - 1; rank >= 0; --rank)   // planes' products of one magnitude, the smallest first
#pragma unroll
                    for (int q = 0; q <= rank; ++q) {
                        const int p = q % 2 ? q / 2 : rank - q / 2, done = RANKS - (rank + 1) * (rank + 2) / 2 + q;
#pragma unroll
                        for (int i = 0; i < T::MI; ++i) {
#pragma unroll
                            for (int c = 0; c < COLS; ++c)
                                acc[c / T::NJ][i][c % T::NJ] = mfma<T::HALF>(b[rank - p][c], a[p][i], acc[c / T::NJ][i][c % T::NJ]);
                            const int turn = (kk * RANKS + done) * T::MI + i;
                            if ((turn + 1) * ASKS / TURNS > turn * ASKS / TURNS) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                            for (int c = turn * ASKS / TURNS; c < (turn + 1) * ASKS / TURNS; ++c) ring.ask(1, c);
                            if ((turn + 1) * ASKS / TURNS > turn * ASKS / TURNS) __builtin_amdgcn_sched_barrier(0);
                        }
                    }
            }
            ring.stream.next();
            ring.move();
        }
    }
}

// The stream of one product.
template <class T, bool ADEEP, bool BDEEP, int PARTS> struct OneStream {
    using F = Flow<T, ADEEP, BDEEP, PARTS>;
    static constexpr int ASKS = F::ASKS, SURE = F::SURE;
    F flow;
    __device__ __forceinline__ void ask(uint32_t stage, int piece) const { flow.ask(stage, piece); }
    __device__ __forceinline__ void next() { flow.next(); }
};

// After the last product with a flat B: a lane's odd and even fours of columns to their places (see Reader).
template <class T, int PARTS> __device__ __forceinline__ void settle(Sums<T, PARTS>& acc) {
    if constexpr (T::NJ > 1) {
        const bool odd = threadIdx.x >> 4 & 1;
#pragma unroll
        for (int y = 0; y < PARTS; ++y)
#pragma unroll
            for (int i = 0; i < T::MI; ++i)
#pragma unroll
                for (int j = 0; j < T::NJ; j += 2) {
                    const f32x4 p = acc[y][i][j], q = acc[y][i][j + 1];
#pragma unroll
                    for (int e = 0; e < 4; ++e) { acc[y][i][j][e] = odd ? q[e] : p[e]; acc[y][i][j + 1][e] = odd ? p[e] : q[e]; }
                }
    }
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
// fp32 numbers stay finite.  Two planes: nearest.  What is not finite has no rest.  The rest is that of the number that was rounded:
// a product that the compiler rounds to fp16 at once in one place and by way of fp32 in another may differ by a step near a tie,
// so planes are made of fp32 numbers that are there as such.
template <int NP, bool HALF> __device__ __forceinline__ void split2(float a, float b, uint32_t (&out)[NP]) {
    if constexpr (NP > 1) asm("" : "+v"(a), "+v"(b));
    if constexpr (NP == 1) out[0] = pack2<HALF>(a, b);
    else if constexpr (NP == 2) {
        out[0] = pack2<HALF>(a, b);
        const float ra = a - as_float<HALF>(out[0] & 0xffff), rb = b - as_float<HALF>(out[0] >> 16);
        out[1] = pack2<HALF>(fabsf(ra) < __builtin_inff() ? ra : 0.0f, fabsf(rb) < __builtin_inff() ? rb : 0.0f);
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

// Writes W (a multiple of 8) elements as planes at column n of row m: those at `N` and behind are written as zero up to the next
// multiple of 8, which is as far as a reader of the planes looks (they need not be zero in x: infinity times a zero is not).
template <int NP, bool HALF, int W>
__device__ __forceinline__ void store_planes(uint16_t* p, int64_t plane, int64_t at, int64_t n, int64_t N, const float (&x)[W]) {
    static_assert(W % 8 == 0, "whole chunks");
    const int left = N - n < W ? (int)(N - n) : W;
    if (left <= 0) return;                              // (n is a multiple of 8)
#pragma unroll
    for (int i = 0; i < W; i += 8) {
        if (i >= left) break;
        uint32_t w[4][NP];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = i + 2 * j;
            split2<NP, HALF>(x[k], x[k + 1], w[j]);
            const uint32_t there = k + 1 < left ? 0xffffffffu : k < left ? 0xffffu : 0u;
#pragma unroll
            for (int q = 0; q < NP; ++q) w[j][q] &= there;
        }
#pragma unroll
        for (int q = 0; q < NP; ++q) *reinterpret_cast<u32x4*>(p + q * plane + at + i) = u32x4{w[0][q], w[1][q], w[2][q], w[3][q]};
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

// Writes the W numbers that every lane has of a row, from its column n on, those before N: lane by lane of four they lie side by side.  They are
// exchanged first, four at a time, so that what four lanes write at a time is 64 bytes side by side and not four times 16.
// All lanes call it; a row that is not there is written by none.  Three gradients of 4096 x 1024 fp32 over a few rows: 38 us rather
// than 47.
template <int W> __device__ __forceinline__ void store_numbers(float* row, bool there, int64_t n, int64_t N, bool grid, const float (&x)[W]) {
    constexpr int C = W / 4;
    static_assert(C == 2 || C == 4, "");
    uint32_t w[C][4];
#pragma unroll
    for (int j = 0; j < W; ++j) w[j / 4][j % 4] = __builtin_bit_cast(uint32_t, x[j]);
    // odd rows of 16 lanes of one against even rows of the other, then upper halves against lower ones: lane q of four then has fours
    // q, 4 + q, ... of the W
    auto swap = [&](int i, int j, auto swapped) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto r = swapped(w[i][e], w[j][e]);
            w[i][e] = r[0];
            w[j][e] = r[1];
        }
    };
    const auto rows = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane16_swap(a, b, false, false); };
    const auto halves = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane32_swap(a, b, false, false); };
#pragma unroll
    for (int i = 0; i < C; i += 2) swap(i, i + 1, rows);
#pragma unroll
    for (int i = 0; i < C / 2; ++i) swap(i, i + C / 2, halves);
    if (!there) return;
    const int q = threadIdx.x >> 4 & 3;
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const int64_t col = n - W * q + 16 * k + 4 * q;
        float* o = row + col;
        if (grid && col + 4 <= N) *reinterpret_cast<u32x4*>(o) = u32x4{w[k][0], w[k][1], w[k][2], w[k][3]};
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e) if (col + e < N) o[e] = __builtin_bit_cast(float, w[k][e]);
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
