// Root-mean-square norm of rows, with the residual's addition before it, and its gradients.
//
//   s = x + residual (rounded to the type, as the next layers see it),  y = s * rstd * w,  rstd = (mean s^2 + eps)^-1/2
//   ds = gs + rstd * (gy w - s^ * mean(gy w s^)),  s^ = s rstd,         dw = sum over rows of gy s^
//
// Bound by memory: every element is read once, held in registers by the lanes of its row, and written once; the backward makes
// rstd again from the row that it reads anyway.  Sums over a row are fp32 and meet by shuffles (through LDS for rows of more than
// 1024 elements); dw is summed by lane over the rows of a workgroup, written as one part a workgroup and joined in order
// by a second launch, so that no order of atomics shows.
//
// 65536 x 1024 bfloat16 with a residual: forward 98 us (5.5 TB/s), backward 120 (4.5 TB/s) and 5 that join dw.  Rows held as numbers
// from the first on took 108 and 129, 10007 x 602 fp16 24.7 rather than 19.0: all of a row's reads are asked for before the first
// is unpacked.  The backward's registers leave room for 16 waves a CU, which is what 1024 workgroups need; the next row read ahead
// takes 152 and is no quicker (122), 768, 1280 and 1536 workgroups take 136, 182 and 162 where 1024 take 129: two rounds, or too few reads.
#include "fsa_block_kernels.h"
#include "fsa_product.hip.h"

#include <type_traits>

namespace fsa {
namespace {

template <int KIND> struct Row {
    using Elem = typename std::conditional<KIND == 0, float, uint16_t>::type;
    static constexpr int PER = KIND == 0 ? 4 : 8;       // elements of a 16-byte piece
};

// A piece of a row from element c on, zeros behind D, as it lies in memory: half as many registers for 16-bit rows as numbers take.
template <int KIND> struct Piece {
    using Elem = typename Row<KIND>::Elem;
    static constexpr int PER = Row<KIND>::PER;
    product::u32x4 raw;
    __device__ __forceinline__ void read(const void* base, int64_t at, int c, int D) {
        const Elem* p = static_cast<const Elem*>(base) + at + c;
        if (c + PER <= D) __builtin_memcpy(&raw, p, 16);
        else {
            Elem e[PER];
#pragma unroll
            for (int j = 0; j < PER; ++j) e[j] = c + j < D ? p[j] : Elem(0);
            __builtin_memcpy(&raw, e, 16);
        }
    }
    __device__ __forceinline__ void write(void* base, int64_t at, int c, int D) const {
        Elem* p = static_cast<Elem*>(base) + at + c;
        if (c + PER <= D) __builtin_memcpy(p, &raw, 16);
        else {
            Elem e[PER];
            __builtin_memcpy(e, &raw, 16);
#pragma unroll
            for (int j = 0; j < PER; ++j) if (c + j < D) p[j] = e[j];
        }
    }
    __device__ __forceinline__ float get(int j) const {
        const uint32_t word = raw[j * 4 / PER];
        if constexpr (KIND == 0) return __builtin_bit_cast(float, word);
        else return product::as_float<KIND == 2>(j % 2 ? word >> 16 : word & 0xffff);
    }
    __device__ __forceinline__ void set(const float (&x)[PER]) {       // rounded to the type
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (KIND == 0) raw[i] = __builtin_bit_cast(uint32_t, x[i]);
            else raw[i] = product::pack2<KIND == 2>(x[2 * i], x[2 * i + 1]);
        }
    }
};
__device__ __forceinline__ float weight_at(const void* w, int kind, int c, int D) {
    if (c >= D) return 0.0f;
    if (kind == 0) return static_cast<const float*>(w)[c];
    const uint32_t bits = static_cast<const uint16_t*>(w)[c];
    return kind == 1 ? product::as_float<false>(bits) : product::as_float<true>(bits);
}

// Sum of x over the LANES lanes of a row, in every one of them.
template <int LANES> __device__ __forceinline__ float row_sum(float x, float* lds) {
#pragma unroll
    for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) x += __shfl_xor(x, d, 64);
    if constexpr (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        __syncthreads();                                // (who still reads the last sum's)
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.0f;
        const int first = (threadIdx.x >> 6) / WAVES * WAVES;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) x += lds[first + i];
    }
    return x;
}

// Largest x over the lanes of a row.
template <int LANES> __device__ __forceinline__ float row_most(float x, float* lds) {
#pragma unroll
    for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) x = fmaxf(x, __shfl_xor(x, d, 64));
    if constexpr (LANES > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < LANES / 64; ++i) x = fmaxf(x, lds[i]);         // (a workgroup has one such row)
    }
    return x;
}
// rstd of a row whose squares are summed.  Squares that fp32 cannot hold (of elements beyond 2^60 or, where eps does not outweigh them, below
// 2^-50; fp16 has none) are looked at again: the row's numbers are then times `unit`, the power of two that brings the largest to [1, 2) (or
// to less beside a larger eps), and rstd is that of those numbers, since the row's own may be no number of fp32.
struct Scale { float unit, rstd; };
// What a branch that hardly a row takes makes of pieces is made there, and of nothing that would be held in registers on the way to it.
template <int KIND, int NV> __device__ __forceinline__ void afresh(Piece<KIND> (&s)[NV]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) asm volatile("" : "+v"(s[v].raw));
}
template <int KIND, int LANES, int NV> __device__ __forceinline__ Scale scale_of(Piece<KIND> (&s)[NV], float sum, const NormArgs& a, float* lds) {
    Scale r{1.0f, 1.0f / sqrtf(sum / (float)a.D + a.eps)};
    if constexpr (KIND != 2) {
        const bool odd = !(sum < 0x1p120f) || (sum < 0x1p-100f && a.eps < 0x1p-70f);
        if (__builtin_expect(!__any(odd), 1)) return r;  // (all lanes of a row that several waves have find the same)
        constexpr int PER = Row<KIND>::PER;
        float most = 0.0f, again = 0.0f;
        afresh(s);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < PER; ++j) most = fmaxf(most, fabsf(s[v].get(j)));
        most = fmaxf(row_most<LANES>(most, lds), sqrtf(a.eps));        // (where that is the larger, its square is what counts)
        if (odd && most > 0.0f && most < __builtin_inff()) {
            const int e = 254 - (int)(__builtin_bit_cast(uint32_t, most) >> 23);       // (of subnormal numbers the lowest)
            r.unit = __builtin_bit_cast(float, (uint32_t)(e < 1 ? 1 : e > 253 ? 253 : e) << 23);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float x[PER];
#pragma unroll
            for (int j = 0; j < PER; ++j) x[j] = s[v].get(j) * r.unit;
            s[v].set(x);
#pragma unroll
            for (int j = 0; j < PER; ++j) again = fmaf(x[j], x[j], again);
        }
        again = row_sum<LANES>(again, lds);
        if (odd) r.rstd = 1.0f / sqrtf(again / (float)a.D + a.eps * r.unit * r.unit);
    }
    return r;
}

template <int KIND, int LANES, int NV>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256) void norm_fwd_kernel(NormArgs a) {
    constexpr int PER = Row<KIND>::PER, THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    __shared__ float lds[THREADS / 64];
    const int lane = threadIdx.x % LANES, D = (int)a.D;
    float w[NV][PER];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < PER; ++j) w[v][j] = weight_at(a.weight, a.weight_kind, (v * LANES + lane) * PER + j, D);
    // (every lane of a workgroup makes every turn: the sums of long rows meet at barriers)
    for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < a.T; t0 += (int64_t)gridDim.x * ROWS) {
        const int64_t t = t0 + threadIdx.x / LANES;
        const bool live = t < a.T;
        Piece<KIND> s[NV], r[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * LANES + lane) * PER;
            s[v].raw = r[v].raw = product::u32x4{};
            if (!live || c >= D) continue;
            s[v].read(a.x, t * a.x_stride, c, D);
            if (a.residual) r[v].read(a.residual, t * a.residual_stride, c, D);
        }
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * LANES + lane) * PER;
            if (a.residual) {
                float x[PER];
#pragma unroll
                for (int j = 0; j < PER; ++j) x[j] = s[v].get(j) + r[v].get(j);
                s[v].set(x);
                if (live && c < D) s[v].write(a.s, t * a.D, c, D);
            }
#pragma unroll
            for (int j = 0; j < PER; ++j) sum = fmaf(s[v].get(j), s[v].get(j), sum);
        }
        const float rstd = scale_of<KIND, LANES, NV>(s, row_sum<LANES>(sum, lds), a, lds).rstd;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * LANES + lane) * PER;
            if (!live || c >= D) continue;
            float x[PER];
#pragma unroll
            for (int j = 0; j < PER; ++j) x[j] = s[v].get(j) * rstd * w[v][j];
            s[v].set(x);
            s[v].write(a.y, t * a.D, c, D);
        }
    }
}

template <int KIND, int LANES, int NV>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256, LANES < 256 ? 4 : 1) void norm_bwd_kernel(NormArgs a) {
    constexpr int PER = Row<KIND>::PER, THREADS = LANES > 256 ? LANES : 256, ROWS = THREADS / LANES;
    __shared__ float lds[THREADS / 64];
    __shared__ float join[ROWS > 1 ? LANES * NV * PER : 1];
    const int lane = threadIdx.x % LANES, D = (int)a.D;
    float w[NV][PER], dw[NV][PER];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            w[v][j] = weight_at(a.weight, a.weight_kind, (v * LANES + lane) * PER + j, D);
            dw[v][j] = 0.0f;
        }
    for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < a.T; t0 += (int64_t)gridDim.x * ROWS) {
        const int64_t t = t0 + threadIdx.x / LANES;
        struct { Piece<KIND> s[NV], g[NV], gs[NV]; } row;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * LANES + lane) * PER;
            row.s[v].raw = row.g[v].raw = row.gs[v].raw = product::u32x4{};
            if (t >= a.T || c >= D) continue;
            row.s[v].read(a.x, t * a.x_stride, c, D);
            if (a.grad_y) row.g[v].read(a.grad_y, t * a.D, c, D);
            if (a.grad_s) row.gs[v].read(a.grad_s, t * a.D, c, D);
        }
        float sum = 0.0f, dot = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                sum = fmaf(row.s[v].get(j), row.s[v].get(j), sum);
                dot = fmaf(row.g[v].get(j) * w[v][j], row.s[v].get(j), dot);
            }
        sum = row_sum<LANES>(sum, lds);
        dot = row_sum<LANES>(dot, lds);
        const Scale r = scale_of<KIND, LANES, NV>(row.s, sum, a, lds);
        if (KIND != 2 && __any(r.unit != 1.0f)) {
            dot = 0.0f;
            afresh(row.g);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < PER; ++j) dot = fmaf(row.g[v].get(j) * w[v][j], row.s[v].get(j), dot);
            dot = row_sum<LANES>(dot, lds);
        }
        const float mean = dot * r.rstd / (float)D, rstd = r.rstd * r.unit;         // mean: of gy w s^
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * LANES + lane) * PER;
            if (t >= a.T || c >= D) continue;
            float x[PER];
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const float unit = row.s[v].get(j) * r.rstd;
                dw[v][j] = fmaf(row.g[v].get(j), unit, dw[v][j]);
                x[j] = fmaf(rstd, fmaf(-unit, mean, row.g[v].get(j) * w[v][j]), row.gs[v].get(j));
            }
            if (!a.y) continue;
            Piece<KIND> out;
            out.set(x);
            out.write(a.y, t * a.D, c, D);
        }
    }
    if (!a.grad_weight) return;
    // rows of a workgroup one after another, in LDS
    float* out = a.parts + (int64_t)blockIdx.x * D;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (const int c = (v * LANES + lane) * PER + j; c < D) out[c] = dw[v][j];
    } else {
        // lanes of one wave that have the same columns join first
#pragma unroll
        for (int d = LANES; d < 64; d *= 2)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < PER; ++j) dw[v][j] += __shfl_xor(dw[v][j], d, 64);
        for (int wave = 0; wave < THREADS / 64; ++wave) {
            if ((int)(threadIdx.x >> 6) == wave && (int)(threadIdx.x & 63) < LANES)
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        const int c = (v * LANES + lane) * PER + j;
                        join[c] = wave == 0 ? dw[v][j] : join[c] + dw[v][j];
                    }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < D; c += THREADS) out[c] = join[c];
    }
}

// grad_weight from the workgroups' parts: 64 columns a workgroup, a wave's 16 lanes 4 of them each, the parts in 64 shares.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* parts, int64_t count, int64_t D, void* out, int kind) {
    __shared__ float lds[64][65];
    const int col = (threadIdx.x & 15) * 4, share = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 64 + col;
    float x[4] = {};
    if (c + 4 <= D) {
#pragma unroll 4
        for (int64_t i = share; i < count; i += 64) {
            float p[4];
            __builtin_memcpy(p, parts + i * D + c, 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] += p[j];
        }
    } else
        for (int64_t i = share; i < count; i += 64)
#pragma unroll
            for (int j = 0; j < 4; ++j) if (c + j < D) x[j] += parts[i * D + c + j];
#pragma unroll
    for (int j = 0; j < 4; ++j) lds[share][col + j] = x[j];
    __syncthreads();
    // 16 lanes to a column, 4 shares each
    const int own = threadIdx.x >> 4, part = threadIdx.x & 15;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += lds[part * 4 + i][own];
#pragma unroll
    for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d, 64);
    const int64_t at = (int64_t)blockIdx.x * 64 + own;
    if (part != 0 || at >= D) return;
    if (kind == 0) static_cast<float*>(out)[at] = sum;
    else static_cast<uint16_t*>(out)[at] = (uint16_t)((kind == 1 ? product::pack2<false>(sum, 0.0f) : product::pack2<true>(sum, 0.0f)) & 0xffff);
}

template <int KIND, int LANES, int NV> hipError_t launch(const NormArgs& a, bool forward, hipStream_t st) {
    const NormPlan p = norm_plan(a.D, KIND == 0 ? 4 : 2);
    if (forward) {
        const int64_t blocks = cut_into(a.T, p.rows), most = 256 * (p.threads > 256 ? 2 : 8);     // as many as the chip holds at a time
        norm_fwd_kernel<KIND, LANES, NV><<<dim3((unsigned)(blocks < most ? blocks : most)), dim3(p.threads), 0, st>>>(a);
        return hipGetLastError();
    }
    const int64_t parts = norm_parts(a.T, a.D, KIND == 0 ? 4 : 2);
    norm_bwd_kernel<KIND, LANES, NV><<<dim3((unsigned)parts), dim3(p.threads), 0, st>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.grad_weight)
        norm_join_kernel<<<dim3((unsigned)cut_into(a.D, 64)), dim3(1024), 0, st>>>(a.parts, parts, a.D, a.grad_weight, a.weight_kind);
    return hipGetLastError();
}
template <int KIND, int LANES> hipError_t by_pieces(const NormArgs& a, bool forward, hipStream_t st) {
    const int pieces = norm_plan(a.D, KIND == 0 ? 4 : 2).pieces;
    if constexpr (KIND == 0) if (pieces == 4) return launch<KIND, LANES, 4>(a, forward, st);
    return pieces == 2 ? launch<KIND, LANES, 2>(a, forward, st) : launch<KIND, LANES, 1>(a, forward, st);
}
template <int KIND> hipError_t by_lanes(const NormArgs& a, bool forward, hipStream_t st) {
    switch (norm_plan(a.D, KIND == 0 ? 4 : 2).lanes) {
        case 4: return by_pieces<KIND, 4>(a, forward, st);
        case 16: return by_pieces<KIND, 16>(a, forward, st);
        case 64: return by_pieces<KIND, 64>(a, forward, st);
        case 256: return by_pieces<KIND, 256>(a, forward, st);
        default: return by_pieces<KIND, 1024>(a, forward, st);
    }
}
hipError_t by_kind(const NormArgs& a, bool forward, hipStream_t st) {
    return a.kind == 0 ? by_lanes<0>(a, forward, st) : a.kind == 1 ? by_lanes<1>(a, forward, st) : by_lanes<2>(a, forward, st);
}

}  // namespace

hipError_t norm_forward(const NormArgs& a, hipStream_t st) { return by_kind(a, true, st); }
hipError_t norm_backward(const NormArgs& a, hipStream_t st) { return by_kind(a, false, st); }

}  // namespace fsa
