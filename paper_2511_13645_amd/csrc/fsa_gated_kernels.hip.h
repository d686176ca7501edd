// The gated feed-forward block, one element type a translation unit (fsa_gated_{f32,bf16,f16}.hip).
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wd^T;   dh = gy Wd, dg = dh u act'(g), du = dh act(g)
//   dx = dg Wg + du Wu,  dWd = gy^T h,  dWg = dg^T x,  dWu = du^T x
//
// g and u are made side by side (one x, two tables), so that a lane has both of an element and h is all that is written.  The
// backward makes them again beside dh rather than read copies: g and u in 16 bits would be rounded once more on the way to every
// gradient, in fp32 they would be 16 bytes of traffic an element, which takes as long as 2 D products from D of about 1000 on.
// h, dg and du are rounded to the type once: each gradient is then off by its own rounding and one of a factor, as in any product of
// tensors of that type.  fp32 has three planes and loses nothing.
// fp16: dg and du are kept times the power of two that brings the largest |gy| to [1, 2), which the products take back, so that
// gradients of a small loss scale are not rounded among fp16's subnormal numbers.
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

template <int EDGE> using ProductTile = Tile<NP, kHalf, EDGE, EDGE, BK, 2, 2>;
template <int EDGE> using PairTile = Tile<NP, kHalf, EDGE, 64, BK, 2, 2>;

// ---------------------------------------------------------------------------------------------------------------
// operands laid out as planes: rows of a multiple of 8 elements, zeros behind their end
// ---------------------------------------------------------------------------------------------------------------
struct PackList {
    Matrix from[5];
    uint16_t* to[5];
    int64_t first[6];                                   // pieces of 8 elements before each
    int count;
};
__global__ __launch_bounds__(256) void pack_kernel(PackList l) {
    const int64_t all = l.first[l.count];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        int m = 0;
#pragma unroll
        for (int j = 1; j < 5; ++j) if (j < l.count && i >= l.first[j]) m = j;
        const Matrix from = l.from[m];
        const int64_t pieces = cut_into(from.cols, 8), at = i - l.first[m], row = at / pieces, col = at % pieces * 8;
        const Elem* p = static_cast<const Elem*>(from.p) + row * from.stride + col;
        Elem e[8];
        if (col + 8 <= from.cols) __builtin_memcpy(e, p, sizeof(e));
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = col + j < from.cols ? p[j] : Elem(0);
        }
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

// ---------------------------------------------------------------------------------------------------------------
// fp16: the power of two of the gradients
// ---------------------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void peaks_kernel(Matrix g, float* peaks) {
    __shared__ float lds[4];
    float top = 0.0f;
    for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x)
        for (int64_t c = threadIdx.x; c < g.cols; c += 256) {
            const uint16_t e = static_cast<const uint16_t*>(g.p)[row * g.stride + c];
            const float x = fabsf(as_float<true>(e));
            if (x < __builtin_inff()) top = fmaxf(top, x);
        }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) peaks[blockIdx.x] = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}
// 2^e with max * 2^e in [1, 2); what fp16 holds lies within 2^-24 ... 2^15.
__device__ __forceinline__ int lift_of(const float* peaks) {
    float top = peaks[threadIdx.x & 63];
    static_assert(kGatedPeaks == 64, "one a lane");
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    if (!(top > 0.0f)) return 0;
    return 127 - (int)(__builtin_bit_cast(uint32_t, top) >> 23);
}
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// ---------------------------------------------------------------------------------------------------------------
// activations: value and derivative
// ---------------------------------------------------------------------------------------------------------------
struct Gate { float value, slope; };
__device__ __forceinline__ float inverse(float x) { return kKind == 0 ? 1.0f / x : __builtin_amdgcn_rcpf(x); }
template <int ACT> __device__ __forceinline__ Gate gate_of(float g) {
    if constexpr (ACT == FSA_ACT_SILU) {
        const float p = inverse(1.0f + (kKind == 0 ? expf(-g) : __expf(-g)));
        return {g * p, p * fmaf(g, 1.0f - p, 1.0f)};
    } else if constexpr (ACT == FSA_ACT_GELU) {
        const float p = kKind == 0 ? 0.5f * erfcf(-0.70710678118654752440f * g) : fmaf(0.5f, erff(0.70710678118654752440f * g), 0.5f);
        const float bell = 0.39894228040143267794f * (kKind == 0 ? expf(-0.5f * g * g) : __expf(-0.5f * g * g));
        return {g * p, fmaf(g, bell, p)};
    } else {
        return {g > 0.0f ? g : (g != g ? g : 0.0f), g > 0.0f ? 1.0f : 0.0f};
    }
}

struct HiddenArgs {
    Side x, gate, up, down, grad_y;
    uint16_t *h, *dg, *du;                              // [T, H8] planes
    int64_t T, D, H, O, H8;
    const float* peaks;
    unsigned mt, nt;
};

template <class T, int ACT> __global__ __launch_bounds__(T::THREADS) void hidden_kernel(HiddenArgs a) {
    __shared__ __attribute__((aligned(256))) char lds[T::lds_bytes(2)];
    unsigned mi, ni;
    tile_of(blockIdx.x, a.mt, a.nt, mi, ni);
    const int64_t m0 = (int64_t)mi * T::BM, n0 = (int64_t)ni * T::BN;
    Sums<T, 2> acc = {};
    const Side tables[2] = {a.gate, a.up};
    accumulate<T, true, true, 2>(acc, lds, a.x, tables, m0, a.T, n0, a.H, 0, a.D);
    each_stretch<T>(m0, n0, [&](int i, int64_t m, int64_t n) {
        if (m >= a.T) return;
        float h[4 * T::NJ];
#pragma unroll
        for (int j = 0; j < 4 * T::NJ; ++j) h[j] = gate_of<ACT>(acc[0][i][j / 4][j % 4]).value * acc[1][i][j / 4][j % 4];
        store_planes<T::NP, T::HALF>(a.h, a.T * a.H8, m * a.H8 + n, n, a.H, h);
    });
}

template <class T, int ACT> __global__ __launch_bounds__(T::THREADS) void slopes_kernel(HiddenArgs a) {
    __shared__ __attribute__((aligned(256))) char lds[T::lds_bytes(2)];
    unsigned mi, ni;
    tile_of(blockIdx.x, a.mt, a.nt, mi, ni);
    const int64_t m0 = (int64_t)mi * T::BM, n0 = (int64_t)ni * T::BN;
    Sums<T, 2> acc = {};
    Sums<T, 1> dh = {};
    const Side tables[2] = {a.gate, a.up}, down[1] = {a.down};
    accumulate<T, true, false, 1>(dh, lds, a.grad_y, down, m0, a.T, n0, a.H8, 0, a.O);
    accumulate<T, true, true, 2>(acc, lds, a.x, tables, m0, a.T, n0, a.H, 0, a.D);
    const float lift = kHalf ? power_of_two(lift_of(a.peaks)) : 1.0f;
    each_stretch<T>(m0, n0, [&](int i, int64_t m, int64_t n) {
        if (m >= a.T) return;
        float h[4 * T::NJ], dg[4 * T::NJ], du[4 * T::NJ];
#pragma unroll
        for (int j = 0; j < 4 * T::NJ; ++j) {
            const Gate g = gate_of<ACT>(acc[0][i][j / 4][j % 4]);
            const float u = acc[1][i][j / 4][j % 4], d = kHalf ? dh[0][i][j / 4][j % 4] * lift : dh[0][i][j / 4][j % 4];
            h[j] = g.value * u;
            dg[j] = d * u * g.slope;
            du[j] = d * g.value;
        }
        store_planes<T::NP, T::HALF>(a.h, a.T * a.H8, m * a.H8 + n, n, a.H, h);
        store_planes<T::NP, T::HALF>(a.dg, a.T * a.H8, m * a.H8 + n, n, a.H, dg);
        store_planes<T::NP, T::HALF>(a.du, a.T * a.H8, m * a.H8 + n, n, a.H, du);
    });
}

// ---------------------------------------------------------------------------------------------------------------
// products that leave in the caller's type
// ---------------------------------------------------------------------------------------------------------------
struct ProductArgs {
    Side a[2], b[2];
    void* out[2];
    int64_t M, N, K, out_ld;                            // K: depth of one pair
    int64_t M8, N8;                                     // ends of flat operands
    bool together;                                      // one result, the sum of both pairs' products; else a result each
    bool pairs, grid;
    float* parts;                                       // [results][splits][M][N8], where there are splits
    const float* peaks;                                 // or null
    unsigned mt, nt, splits;
};

template <class T, bool ADEEP, bool BDEEP> __global__ __launch_bounds__(T::THREADS) void product_kernel(ProductArgs a) {
    __shared__ __attribute__((aligned(256))) char lds[T::lds_bytes(1)];
    unsigned mi, ni;
    tile_of(blockIdx.x, a.mt, a.nt, mi, ni);
    const int64_t m0 = (int64_t)mi * T::BM, n0 = (int64_t)ni * T::BN;
    const unsigned split = blockIdx.y, which = blockIdx.z;
    Sums<T, 1> acc = {};
    // this split's steps of all pairs', one pair after the other
    const int64_t steps = cut_into(a.K, T::BK), all = a.together ? 2 * steps : steps;
    const int64_t first = all * split / a.splits, last = all * (split + 1) / a.splits;
    auto add = [&](int pair, int64_t from, int64_t to) {
        const Side b[1] = {a.b[pair]};
        const int64_t end = to * T::BK < a.K ? to * T::BK : a.K;
        accumulate<T, ADEEP, BDEEP, 1>(acc, lds, a.a[pair], b, m0, ADEEP ? a.M : a.M8, n0, BDEEP ? a.N : a.N8, from * T::BK, end);
    };
    if (!a.together) add(which, first, last);
    else
#pragma unroll 1
        for (int pair = 0; pair < 2; ++pair) {
            const int64_t from = first - pair * steps, to = last - pair * steps;
            add(pair, from < 0 ? 0 : from, to < steps ? to : steps);
        }
    const float back = kHalf && a.peaks && a.splits == 1 ? power_of_two(-lift_of(a.peaks)) : 1.0f;
    each_stretch<T>(m0, n0, [&](int i, int64_t m, int64_t n) {
        if (m >= a.M) return;
        float x[4 * T::NJ];
#pragma unroll
        for (int j = 0; j < 4 * T::NJ; ++j) x[j] = kHalf ? acc[0][i][j / 4][j % 4] * back : acc[0][i][j / 4][j % 4];
        if (a.splits > 1) store_row<0>(a.parts + (which * a.splits + split) * a.M * a.N8, m * a.N8, n, a.N8, true, x);
        else store_row<kKind>(a.out[which], m * a.out_ld, n, a.N, a.grid, x);
    });
}

// Splits' parts joined in their order.
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a) {
    const float back = kHalf && a.peaks ? power_of_two(-lift_of(a.peaks)) : 1.0f;
    const int64_t pieces = a.N8 / 4, all = a.M * pieces;
    const float* parts = a.parts + blockIdx.y * a.splits * a.M * a.N8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        f32x4 sum = {};
        for (unsigned s = 0; s < a.splits; ++s) sum += *reinterpret_cast<const f32x4*>(parts + s * a.M * a.N8 + i * 4);
        const float x[4] = {sum[0] * back, sum[1] * back, sum[2] * back, sum[3] * back};
        store_row<kKind>(a.out[blockIdx.y], i / pieces * a.out_ld, i % pieces * 4, a.N, a.grid, x);
    }
}

// Gradients of weights over no rows at all.
__global__ __launch_bounds__(256) void zero_kernel(Elem* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = Elem(0);
}

// ---------------------------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------------------------
bool on_grid(const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (int64_t)sizeof(Elem) % 16 == 0; }

template <class T, bool ADEEP, bool BDEEP> hipError_t launch_product(const ProductArgs& a, hipStream_t st) {
    const unsigned results = a.pairs && !a.together ? 2 : 1;
    product_kernel<T, ADEEP, BDEEP><<<dim3(a.mt * a.nt, a.splits, results), dim3(T::THREADS), 0, st>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.splits > 1) {
        const int64_t blocks = cut_into(a.M * (a.N8 / 4), 256);
        join_kernel<<<dim3((unsigned)(blocks < 4096 ? blocks : 4096), results), dim3(256), 0, st>>>(a);
    }
    return hipGetLastError();
}
template <bool ADEEP, bool BDEEP> hipError_t run_product(ProductArgs a, const ProductCut& c, hipStream_t st) {
    a.mt = (unsigned)c.mt; a.nt = (unsigned)c.nt; a.splits = (unsigned)c.splits;
    a.M8 = up_to(a.M, 8); a.N8 = up_to(a.N, 8);
    a.grid = on_grid(a.out[0], a.out_ld) && (!a.out[1] || on_grid(a.out[1], a.out_ld));
    return c.tile == 128 ? launch_product<ProductTile<128>, ADEEP, BDEEP>(a, st) : launch_product<ProductTile<64>, ADEEP, BDEEP>(a, st);
}

template <class T, int ACT> hipError_t launch_pair(HiddenArgs a, bool forward, hipStream_t st) {
    a.mt = (unsigned)cut_into(a.T, T::BM); a.nt = (unsigned)cut_into(a.H, T::BN);
    if (forward) hidden_kernel<T, ACT><<<dim3(a.mt * a.nt), dim3(T::THREADS), 0, st>>>(a);
    else slopes_kernel<T, ACT><<<dim3(a.mt * a.nt), dim3(T::THREADS), 0, st>>>(a);
    return hipGetLastError();
}
template <int ACT> hipError_t by_edge(const HiddenArgs& a, bool forward, hipStream_t st) {
    return pair_tile(a.T, a.H) == 128 ? launch_pair<PairTile<128>, ACT>(a, forward, st) : launch_pair<PairTile<64>, ACT>(a, forward, st);
}
hipError_t run_pair(const GatedArgs& g, const HiddenArgs& a, bool forward, hipStream_t st) {
    return g.activation == FSA_ACT_SILU ? by_edge<FSA_ACT_SILU>(a, forward, st)
         : g.activation == FSA_ACT_GELU ? by_edge<FSA_ACT_GELU>(a, forward, st) : by_edge<FSA_ACT_RELU>(a, forward, st);
}

struct Operands { Side x, gate, up, down, grad_y; };

hipError_t lay_out(const GatedArgs& a, Operands& o, hipStream_t st) {
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
    if (l.count == 0) return hipSuccess;
    const int64_t blocks = cut_into(l.first[l.count], 256);
    pack_kernel<<<dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, st>>>(l);
    return hipGetLastError();
}

HiddenArgs hidden_args(const GatedArgs& a, const Operands& o) {
    HiddenArgs h{};
    h.x = o.x; h.gate = o.gate; h.up = o.up; h.down = o.down; h.grad_y = o.grad_y;
    h.h = reinterpret_cast<uint16_t*>(a.ws + a.plan.h);
    h.dg = reinterpret_cast<uint16_t*>(a.ws + a.plan.dg);
    h.du = reinterpret_cast<uint16_t*>(a.ws + a.plan.du);
    h.T = a.s.T; h.D = a.s.D; h.H = a.s.H; h.O = a.s.O;
    h.H8 = a.plan.H8;
    h.peaks = reinterpret_cast<const float*>(a.ws + a.plan.peaks);
    return h;
}

hipError_t forward(const GatedArgs& a, hipStream_t st) {
    Operands o{};
    if (hipError_t e = lay_out(a, o, st)) return e;
    const HiddenArgs h = hidden_args(a, o);
    if (hipError_t e = run_pair(a, h, true, st)) return e;
    ProductArgs p{};
    p.a[0] = {h.h, h.H8, a.s.T * h.H8}; p.b[0] = o.down;
    p.out[0] = a.y;
    p.M = a.s.T; p.N = a.s.O; p.K = a.s.H; p.out_ld = a.s.O;
    p.parts = reinterpret_cast<float*>(a.ws + a.plan.parts);
    return run_product<true, true>(p, a.plan.answer, st);
}

hipError_t backward(const GatedArgs& a, hipStream_t st) {
    const bool want_w = a.grad_gate || a.grad_up || a.grad_down;
    if (a.s.T == 0) {
        void* const outs[3] = {a.grad_gate, a.grad_up, a.grad_down};
        const int64_t sizes[3] = {a.s.H * a.s.D, a.s.H * a.s.D, a.s.O * a.s.H};
        for (int i = 0; i < 3; ++i)
            if (outs[i]) {
                const int64_t blocks = cut_into(sizes[i], 256);
                zero_kernel<<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st>>>(static_cast<Elem*>(outs[i]), sizes[i]);
                if (hipError_t e = hipGetLastError()) return e;
            }
        return hipSuccess;
    }
    if (!want_w && !a.grad_x) return hipSuccess;
    Operands o{};
    if (hipError_t e = lay_out(a, o, st)) return e;
    float* peaks = reinterpret_cast<float*>(a.ws + a.plan.peaks);
    if (kHalf) {
        peaks_kernel<<<dim3(kGatedPeaks), dim3(256), 0, st>>>(a.grad_y, peaks);
        if (hipError_t e = hipGetLastError()) return e;
    }
    const HiddenArgs h = hidden_args(a, o);
    if (hipError_t e = run_pair(a, h, false, st)) return e;
    const int64_t plane = a.s.T * h.H8;
    const Side hs = {h.h, h.H8, plane}, dg = {h.dg, h.H8, plane}, du = {h.du, h.H8, plane};
    ProductArgs p{};
    p.parts = reinterpret_cast<float*>(a.ws + a.plan.parts);
    if (a.grad_x) {
        p.a[0] = dg; p.a[1] = du; p.b[0] = o.gate; p.b[1] = o.up;
        p.together = p.pairs = true;
        p.out[0] = a.grad_x; p.out[1] = nullptr;
        p.M = a.s.T; p.N = a.s.D; p.K = a.s.H; p.out_ld = a.s.D;
        p.peaks = kHalf ? peaks : nullptr;
        if (hipError_t e = run_product<true, false>(p, a.plan.dx, st)) return e;
    }
    p.together = p.pairs = false;
    p.K = a.s.T;
    if (a.grad_down) {
        p.a[0] = o.grad_y; p.b[0] = hs;
        p.out[0] = a.grad_down; p.out[1] = nullptr;
        p.M = a.s.O; p.N = a.s.H; p.out_ld = a.s.H;
        p.peaks = nullptr;
        if (hipError_t e = run_product<false, false>(p, a.plan.down_grad, st)) return e;
    }
    if (a.grad_gate || a.grad_up) {
        const bool both = a.grad_gate && a.grad_up;
        p.pairs = both;
        p.a[0] = a.grad_gate ? dg : du; p.a[1] = du; p.b[0] = p.b[1] = o.x;
        p.out[0] = a.grad_gate ? a.grad_gate : a.grad_up; p.out[1] = both ? a.grad_up : nullptr;
        p.M = a.s.H; p.N = a.s.D; p.out_ld = a.s.D;
        p.peaks = kHalf ? peaks : nullptr;
        if (hipError_t e = run_product<false, false>(p, a.plan.gate_grad, st)) return e;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace fsa
#endif
