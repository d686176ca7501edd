// Orthogonalised updates: X = G / (|G| + eps), then steps of X = a X + P X with A = X X^T, P = b A + c A^2.
//
// Singular values of X stay as they are paired with their vectors and are moved towards one by the steps' polynomial.  What bounds
// it is the matrix cores: 2 m^2 n + m^3 multiplications a step.  X, A and P are two fp16 planes each, whose three products carry 23
// bits: small singular values grow by up to a^steps, and with them what was rounded beside large ones, so that 16 bits of X
// would leave nothing of directions a hundredth as strong as the strongest.
#include "fsa_block_kernels.h"
#include "fsa_product.hip.h"

#include <cmath>
#include <type_traits>

namespace fsa {
namespace {

using namespace product;

// The tiles that fsa_block.h chooses from, in its order.  Steps of 64 of the depth where two stages of them fit: one 1024 x 1024 -> 4096
// update takes 30 us rather than 37 with steps of 32, eight 600 x 2400 matrices 678 us rather than 745, though a CU then
// holds one workgroup of 128 x 128 instead of two.  Tiles of 64 x 64 wait for all of a step's requests at its head.  With four stages A A of
// 1024 x 1024 takes 12.8 us rather than 15.5, one workgroup a CU, but P X of 602 x 2047, of more, 20.2 rather than 14.2, since LDS then has room
// for one alone; two sets of fragments (15.5 and 14.8) and 8 waves (15.8 and 14.2) are no gain.
template <int CHOICE> using OrthoTile = Tile<2, true, kTilesTwo[CHOICE].m, kTilesTwo[CHOICE].n, CHOICE <= 1 ? 64 : 32, 2, CHOICE == 0 ? 2 : 4>;
template <int KIND> using ElemOf = typename std::conditional<KIND == 0, float, uint16_t>::type;
template <int E> constexpr float kTwoTo = E > 0 ? (float)(1ull << (E > 0 ? E : 0)) : 1.0f / (float)(1ull << (E < 0 ? -E : 0));

template <int KIND> __device__ __forceinline__ float number(ElemOf<KIND> e) {
    if constexpr (KIND == 0) return e;
    else return as_float<KIND == 2>(e);
}

// Elements c ... c + 3 of row r of a matrix, those that there are.
template <int KIND> __device__ __forceinline__ void load_four(const ElemOf<KIND>* g, int64_t r, int64_t c, const OrthoArgs& a, ElemOf<KIND> (&e)[4]) {
    if (r >= a.s.M) return;
    const ElemOf<KIND>* p = g + r * a.stride + c;
    if (c + 4 <= a.s.N) __builtin_memcpy(e, p, sizeof(e));
    else {
#pragma unroll
        for (int j = 0; j < 3; ++j) if (c + j < a.s.N) e[j] = p[j];
    }
}

// Squares of a matrix, summed in 64 bits: gradients of 1e-30 have norms too.
template <int KIND> __global__ __launch_bounds__(256) void squares_kernel(OrthoArgs a) {
    __shared__ double lds[4];
    const ElemOf<KIND>* g = static_cast<const ElemOf<KIND>*>(a.g) + blockIdx.y * a.batch_stride;
    double sum = 0.0;
    // a wave's 64 pieces of 4 elements, row by row: few rows take several waves to one
    const int64_t pieces = cut_into(a.s.N, 256), all = a.s.M * pieces, waves = (int64_t)gridDim.x * 4;
    const int lane = threadIdx.x & 63;
    for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < all; i += waves) {
        const int64_t row = all <= 0x7fffffff ? (uint32_t)i / (uint32_t)pieces : i / pieces;
        ElemOf<KIND> e[4] = {};
        load_four<KIND>(g, row, (i - row * pieces) * 256 + lane * 4, a, e);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const double x = number<KIND>(e[j]);
            sum = fma(x, x, sum);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        reinterpret_cast<double*>(a.ws + a.plan.squares)[blockIdx.y * kOrthoPeaks + blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}
// What brings a matrix to the planes of the first X, in 64 bits as well: 2^13 over a norm of 1e-36, or of 1e39, is no number of 32.
__device__ __forceinline__ double first_unit(const OrthoArgs& a, unsigned batch) {
    const double* parts = reinterpret_cast<const double*>(a.ws + a.plan.squares) + batch * kOrthoPeaks + 4 * (threadIdx.x & 63);
    static_assert(kOrthoPeaks == 256, "four a lane");
    double sum = (parts[0] + parts[1]) + (parts[2] + parts[3]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
    const double norm = sqrt(sum) + (double)a.eps;
    return norm > 0.0 ? (double)kTwoTo<kUnitX> / norm : norm == 0.0 ? 0.0 : __builtin_nan("");
}

// Planes of the first X, 64 x 64 of it a workgroup; of a tall matrix its transpose.
template <int KIND> __global__ __launch_bounds__(256) void first_kernel(OrthoArgs a) {
    __shared__ float tile[64][65];
    const unsigned batch = blockIdx.z;
    const bool tall = a.s.M > a.s.N;
    const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)blockIdx.y * 64;      // of the matrix as it is given
    const ElemOf<KIND>* g = static_cast<const ElemOf<KIND>*>(a.g) + batch * a.batch_stride;
    ElemOf<KIND> e[4][4] = {};                          // 4 elements of each fourth of the rows, asked for before the norm is there
#pragma unroll
    for (int i = 0; i < 4; ++i) load_four<KIND>(g, r0 + i * 16 + threadIdx.x / 16, c0 + threadIdx.x % 16 * 4, a, e[i]);
    const double unit = first_unit(a, batch);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) tile[i * 16 + threadIdx.x / 16][threadIdx.x % 16 * 4 + j] = (float)((double)number<KIND>(e[i][j]) * unit);
    __syncthreads();
    const int64_t m = a.plan.m, n = a.plan.n, n8 = a.plan.n8, plane = m * n8;
    uint16_t* x = reinterpret_cast<uint16_t*>(a.ws + a.plan.x[0]) + batch * 2 * plane;
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int row = i / 8, col = i % 8 * 8;
        const int64_t xm = (tall ? c0 : r0) + row, xn = (tall ? r0 : c0) + col;
        if (xm >= m) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = tall ? tile[col + j][row] : tile[row][col + j];
        store_planes<2, true>(x, plane, xm * n8 + xn, xn, n, v);
    }
}

struct StepArgs {
    const uint16_t *x, *sq, *poly;                      // planes of X, A, P; a matrix' planes are together
    uint16_t* to;
    float* parts;                                       // of a gram matrix with splits: tiles on and above the diagonal
    void* out;                                          // of the last step, in the caller's type
    int64_t m, n, m8, n8;
    // Units of the planes are powers of two: of a gram matrix in X's square, of A^2 and A in P's, of P X and X in X's, of the next X in this one's
    // (which with coefficients that are known to keep singular values small are the usual ones), and the last X in the caller's.
    float to_a, square, linear, product, keep, next, back;
    unsigned mt, nt, splits;
    bool tall, grid;
};

// Tiles on and above the diagonal of a square of them, row by row.
__device__ __forceinline__ void upper_tile(unsigned t, unsigned mt, unsigned& mi, unsigned& ni) {
    mi = 0;
    while (t >= mt - mi) { t -= mt - mi; ++mi; }
    ni = mi + t;
}

// W elements of two planes from `at` on.
template <int W> __device__ __forceinline__ void load_planes(const uint16_t* p, int64_t plane, int64_t at, int64_t n, int64_t end, float (&x)[W]) {
#pragma unroll
    for (int i = 0; i < W; i += 8) {
        u32x4 hi = {}, lo = {};
        if (n + i < end) {
            hi = *reinterpret_cast<const u32x4*>(p + at + i);
            lo = *reinterpret_cast<const u32x4*>(p + plane + at + i);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int s = j % 2 * 16;
            x[i + j] = as_float<true>(hi[j / 2] >> s & 0xffff) + as_float<true>(lo[j / 2] >> s & 0xffff);
        }
    }
}

enum { kGram, kGramParts, kPoly, kUpdate };
template <class T, int WHAT, int KIND> __global__ __launch_bounds__(T::THREADS, T::waves(1)) void step_kernel(StepArgs a) {
    __shared__ __attribute__((aligned(256))) char lds[T::lds_bytes(1)];
    unsigned mi, ni;
    if constexpr (WHAT == kGramParts) upper_tile(blockIdx.x, a.mt, mi, ni);
    else tile_of(blockIdx.x, a.mt, a.nt, mi, ni);
    constexpr bool GRAM = WHAT == kGram || WHAT == kGramParts;
    const int64_t m0 = (int64_t)mi * T::BM, n0 = (int64_t)ni * T::BN, batch = blockIdx.z;
    const int64_t wide = a.m * a.n8, square = a.m * a.m8;
    const uint16_t *x = a.x + batch * 2 * wide, *sq = a.sq + batch * 2 * square, *poly = a.poly + batch * 2 * square;
    Sums<T, 1> acc = {};
    const Side sx = {x, a.n8, wide}, sa = {sq, a.m8, square}, sp = {poly, a.m8, square};
    using Stream = OneStream<T, true, WHAT != kUpdate, 1>;
    Stream stream;
    const Side b[1] = {WHAT == kPoly ? sa : sx};
    const int64_t depth = GRAM ? a.n : a.m, steps = cut_into(depth, T::BK);
    const int64_t first = WHAT == kGramParts ? steps * blockIdx.y / a.splits : 0, last = WHAT == kGramParts ? steps * (blockIdx.y + 1) / a.splits : steps;
    stream.flow.start(GRAM ? sx : WHAT == kPoly ? sa : sp, b, m0, a.m, n0, WHAT == kUpdate ? a.n8 : a.m, first * T::BK,
                      last * T::BK < depth ? last * T::BK : depth);
    Ring<T, T::stage_bytes(1), Stream> ring{lds, stream};
    ring.fill();
    accumulate<T, true, WHAT != kUpdate, 1>(acc, ring, last - first);
    ring.end();
    if constexpr (WHAT == kUpdate) settle<T, 1>(acc);
    each_stretch<T>(m0, n0, [&](int i, int64_t m, int64_t n) {
        constexpr int W = 4 * T::NJ;
        float v[W];
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = acc[0][i][j / 4][j % 4];
        if constexpr (WHAT == kGramParts) {
            float* part = a.parts + ((batch * a.splits + blockIdx.y) * gridDim.x + blockIdx.x) * T::BM * T::BN;
            return store_numbers(part + (m - m0) * T::BN, m < a.m, n - n0, T::BN, true, v);
        }
        if (m >= a.m) return;
        if constexpr (WHAT == kGram) {
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] *= a.to_a;
            store_planes<2, true>(a.to + batch * 2 * square, square, m * a.m8 + n, n, a.m, v);
        } else if constexpr (WHAT == kPoly) {
            float old[W];
            load_planes<W>(sq, square, m * a.m8 + n, n, a.m8, old);
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = fmaf(a.square, v[j], a.linear * old[j]);
            store_planes<2, true>(a.to + batch * 2 * square, square, m * a.m8 + n, n, a.m, v);
        } else {
            float old[W];
            load_planes<W>(x, wide, m * a.n8 + n, n, a.n8, old);
#pragma unroll
            for (int j = 0; j < W; ++j) v[j] = fmaf(a.product, v[j], a.keep * old[j]) * a.next;
            if (!a.out) store_planes<2, true>(a.to + batch * 2 * wide, wide, m * a.n8 + n, n, a.n, v);
            else {
                ElemOf<KIND>* out = static_cast<ElemOf<KIND>*>(a.out) + batch * a.m * a.n;
#pragma unroll
                for (int j = 0; j < W; ++j) v[j] *= a.back;
                if (!a.tall) store_row<KIND>(out, m * a.n, n, a.n, a.grid, v);
                else {
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        const float one[4] = {v[j], 0.0f, 0.0f, 0.0f};
                        if (n + j < a.n) store_row<KIND>(out, (n + j) * a.m, m, m + 1, false, one);
                    }
                }
            }
        }
    });
}

// 64 x 64 of the gram matrix from its parts, and of its other half what mirrors them.  4 elements a lane, whose parts are all asked for at
// once: 1024 x 1024 in seven parts 6.2 us, where 256 lanes with four turns took 8.9.
constexpr int kMirrorThreads = 1024;
__global__ __launch_bounds__(kMirrorThreads) void mirror_kernel(StepArgs a, unsigned tile, unsigned tiles) {
    __shared__ float sum[64][65];
    const unsigned blocks = tile / 64, t = blockIdx.x / (blocks * blocks), at = blockIdx.x % (blocks * blocks), batch = blockIdx.z;
    unsigned mi, ni;
    upper_tile(t, a.mt, mi, ni);
    const int64_t m0 = (int64_t)mi * tile + at / blocks * 64, n0 = (int64_t)ni * tile + at % blocks * 64;
    if (m0 >= a.m || n0 >= a.m) return;
    const int64_t size = (int64_t)tile * tile;
    const float* part = a.parts + (batch * a.splits * tiles + t) * size + (at / blocks * 64) * tile + at % blocks * 64;
    static_assert(kMirrorThreads == 64 * 16, "4 elements a lane");
    {
        const int row = threadIdx.x / 16, col = threadIdx.x % 16 * 4;
        f32x4 x = {};
        if (m0 + row < a.m) {
#pragma unroll 8
            for (unsigned s = 0; s < a.splits; ++s) x += *reinterpret_cast<const f32x4*>(part + s * tiles * size + row * tile + col);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[row][col + j] = x[j] * a.to_a;
    }
    __syncthreads();
    const int64_t square = a.m * a.m8;
    uint16_t* to = a.to + batch * 2 * square;
    // half of the lanes for each side of the diagonal
    const int i = threadIdx.x % 512, row = i / 8, col = i % 8 * 8;
    const bool below = threadIdx.x >= 512;
    const int64_t r0 = below ? n0 : m0, c0 = below ? m0 : n0;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = below ? sum[col + j][row] : sum[row][col + j];
    if ((below && mi == ni) || r0 + row >= a.m) return;
    store_planes<2, true>(to, square, (r0 + row) * a.m8 + c0 + col, c0 + col, a.m, v);
}

template <int CHOICE, int WHAT, int KIND> hipError_t launch_tiles(StepArgs a, int64_t batch, hipStream_t st) {
    using T = OrthoTile<CHOICE>;
    a.mt = (unsigned)cut_into(a.m, T::BM);
    a.nt = (unsigned)cut_into(WHAT == kUpdate ? a.n : a.m, T::BN);
    const unsigned tiles = WHAT == kGramParts ? (unsigned)upper_tiles(a.m, T::BM) : a.mt * a.nt;
    step_kernel<T, WHAT, KIND><<<dim3(tiles, WHAT == kGramParts ? a.splits : 1, (unsigned)batch), dim3(T::THREADS), 0, st>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if constexpr (WHAT == kGramParts)
        mirror_kernel<<<dim3(tiles * (T::BM / 64) * (T::BM / 64), 1, (unsigned)batch), dim3(kMirrorThreads), 0, st>>>(a, T::BM, tiles);
    return hipGetLastError();
}
template <int WHAT, int KIND> hipError_t launch(const StepArgs& a, int64_t batch, int choice, hipStream_t st) {
    return choice == 2 ? launch_tiles<2, WHAT, KIND>(a, batch, st)
         : choice == 1 ? launch_tiles<1, WHAT, KIND>(a, batch, st) : launch_tiles<0, WHAT, KIND>(a, batch, st);
}

template <int KIND> hipError_t run(const OrthoArgs& a, hipStream_t st) {
    const OrthoPlan& p = a.plan;
    squares_kernel<KIND><<<dim3(kOrthoPeaks, (unsigned)a.s.B), dim3(256), 0, st>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    first_kernel<KIND><<<dim3((unsigned)cut_into(a.s.M, 64), (unsigned)cut_into(a.s.N, 64), (unsigned)a.s.B), dim3(256), 0, st>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    StepArgs s{};
    uint16_t* x[2] = {reinterpret_cast<uint16_t*>(a.ws + p.x[0]), reinterpret_cast<uint16_t*>(a.ws + p.x[1])};
    uint16_t *sq = reinterpret_cast<uint16_t*>(a.ws + p.a), *poly = reinterpret_cast<uint16_t*>(a.ws + p.p);
    s.sq = sq; s.poly = poly;
    s.m = p.m; s.n = p.n; s.m8 = p.m8; s.n8 = p.n8;
    s.parts = reinterpret_cast<float*>(a.ws + p.parts);
    s.splits = (unsigned)p.splits;
    s.tall = a.s.M > a.s.N;
    s.grid = reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && p.n * (int64_t)sizeof(ElemOf<KIND>) % 16 == 0;
    for (int i = 0; i < a.steps; ++i) {
        const OrthoUnits& u = a.units[i];
        const float* abc = a.coefficients + 3 * i;
        s.to_a = ldexpf(1.0f, u.a - 2 * u.x);
        s.square = ldexpf(abc[2], u.p - 2 * u.a);
        s.linear = ldexpf(abc[1], u.p - u.a);
        s.product = ldexpf(1.0f, -u.p);
        s.keep = abc[0];
        s.next = i + 1 < a.steps ? ldexpf(1.0f, a.units[i + 1].x - u.x) : 1.0f;
        s.back = ldexpf(a.scale, -u.x);
        s.x = x[i % 2];
        s.to = sq;
        if (hipError_t e = s.splits > 1 ? launch<kGramParts, 0>(s, a.s.B, p.gram, st) : launch<kGram, 0>(s, a.s.B, p.gram, st)) return e;
        s.to = poly;
        if (hipError_t e = launch<kPoly, 0>(s, a.s.B, p.poly, st)) return e;
        s.to = x[(i + 1) % 2];
        s.out = i + 1 == a.steps ? a.out : nullptr;
        if (hipError_t e = launch<kUpdate, KIND>(s, a.s.B, p.update, st)) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t orthogonalize(const OrthoArgs& a, hipStream_t st) {
    return a.s.kind == 0 ? run<0>(a, st) : a.s.kind == 1 ? run<1>(a, st) : run<2>(a, st);
}

}  // namespace fsa
