// Device side of the class losses, one element type a translation unit (fsa_class_{f32,bf16,f16}.hip).
//
// Scores z[t,v] = scale * h[t].w[v] come from 32x32x16 matrix instructions, A = the streamed side (from LDS), B = the
// held side (in registers).  Lane l of the result holds column l%32 (a held row) and rows 8*(i/4) + 4*(l/32) + i%4,
// i = 0..15 (streamed rows).  Fed back as the B operand of the second product, register 8s+j of a lane is its k slot
// (l/32, j) of step s, so with A read transposed at those same rows no lane ever exchanges a probability:
//     acc[d, held] += sum over streamed rows of streamed[row, d] * P[row, held].
//
// fp32 rows are held as two fp16 planes, x * 2^e = hi + lo with 2^e that brings the largest finite |x| of the row to
// [2^14, 2^15): 22 bits of every element down to 2^-16 of the row's largest and never an error over 2^-40 of it, whatever other rows
// hold.  Products take hi*hi + hi*lo + lo*hi; what is left out is below 2^-22 of a product, as is what the split rounds away.
// On the held side 2^-e is in the scores' multiplier, a lane's own.  Streamed rows have it beside their tile: s = 2^-e multiplies
// a score, and the second product takes p s, so that what a running reference follows is p s as well.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include <utility>

#include "fsa_class.h"
#include "fsa_internal.h"

namespace fsa {

struct ClassArgs {
    ClassShape s;
    const void* h; int64_t h_stride;                    // strides in elements
    const void* w; int64_t w_stride;
    float scale;                                        // what multiplies h.w (the temperature divided out)
    const int32_t* ids;                                 // [T,K] targets or the teacher's classes
    const void* teacher; int teacher_kind;              // [T,K] teacher logits, or null: one slot of weight one
    float inv_temperature;
    float* loss; float* lse; float* row_grad;           // forward outputs (row_grad nullable)
    const float* grad_loss; const float* lse_in; const float* row_grad_in;
    void* grad_h; void* grad_w;
    ClassCut cut; ClassPlan plan; ClassBuckets buckets; char* ws;
    template <class T> __host__ __device__ T* at(size_t off) const { return reinterpret_cast<T*>(ws + off); }
};

hipError_t class_forward_f32(const ClassArgs&, hipStream_t);
hipError_t class_forward_bf16(const ClassArgs&, hipStream_t);
hipError_t class_forward_f16(const ClassArgs&, hipStream_t);
hipError_t class_gradient_f32(const ClassArgs&, hipStream_t);
hipError_t class_gradient_bf16(const ClassArgs&, hipStream_t);
hipError_t class_gradient_f16(const ClassArgs&, hipStream_t);

#ifdef FSA_CLASS_KIND
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kKind = FSA_CLASS_KIND;                   // 0 fp32, 1 bfloat16, 2 fp16
constexpr int NS = class_planes(kKind);
constexpr bool kHalf = kKind != 1;                      // planes hold fp16 (bfloat16 otherwise)
constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLog2eDouble = 1.44269504088896340736;
// fp16 probabilities are kept as p * 2^14: 28 binades below the largest stay normal numbers.
constexpr float kLift = kHalf ? 14.0f : 0.0f;
// The running reference of a row follows its maximum only when that is passed by this many binades, so that most tiles
// leave the accumulators alone; 2^(14+1) is in range of fp16, bfloat16 has room.
constexpr float kSlack = kHalf ? 1.0f : 8.0f;
using Elem = typename std::conditional<kKind == 0, float, uint16_t>::type;

__device__ __forceinline__ float as_float(uint16_t b) {
    if constexpr (kHalf) return (float)__builtin_bit_cast(_Float16, b);
    else return __builtin_bit_cast(float, (uint32_t)b << 16);
}
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return as_float(x); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {     // nearest even
    if constexpr (kHalf) { const f16x2 v = {(_Float16)a, (_Float16)b}; return __builtin_bit_cast(uint32_t, v); }
    else { const bf16x2 v = {(__bf16)a, (__bf16)b}; return __builtin_bit_cast(uint32_t, v); }
}
__device__ __forceinline__ float low2(uint32_t p) { return as_float((uint16_t)(p & 0xffff)); }
__device__ __forceinline__ float high2(uint32_t p) { return as_float((uint16_t)(p >> 16)); }

__device__ __forceinline__ f32x16 matmul(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (kHalf)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// a and b of NS planes each: every product but lo*lo.
__device__ __forceinline__ f32x16 matmul(const u32x4 (&a)[NS], const u32x4 (&b)[NS], f32x16 c) {
    if constexpr (NS == 2) { c = matmul(a[1], b[0], c); c = matmul(a[0], b[1], c); }
    return matmul(a[0], b[0], c);
}

// Planes of eight scaled elements.  An infinite element stays infinite (and its rest zero), NaN stays NaN.
__device__ __forceinline__ void split8(const float (&x)[8], float unit, u32x4 (&out)[NS]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = x[2 * i] * unit, b = x[2 * i + 1] * unit;
        out[0][i] = pack2(a, b);
        if constexpr (NS == 2) {
            float ra = a - low2(out[0][i]), rb = b - high2(out[0][i]);
            if (__builtin_isinf(a)) ra = 0.0f;
            if (__builtin_isinf(b)) rb = 0.0f;
            out[1][i] = pack2(ra, rb);
        }
    }
}

// 16 bytes of a row from byte `at` on, zero behind its end: one wide load at whatever alignment the row has, that of the
// row's last 16 bytes shifted down where it ends before.
__device__ __forceinline__ u32x4 load16(const Elem* row, int bytes, int at) {
    const char* p = reinterpret_cast<const char*>(row);
    u32x4 x = {};
    if (at + 16 <= bytes) __builtin_memcpy(&x, p + at, 16);
    else if (at < bytes && bytes >= 16) {
        uint64_t lo, hi;
        __builtin_memcpy(&lo, p + bytes - 16, 8);
        __builtin_memcpy(&hi, p + bytes - 8, 8);
        const int bits = 8 * (at + 16 - bytes);         // 16 ... 112
        lo = bits >= 64 ? hi >> (bits - 64) : lo >> bits | hi << (64 - bits);
        hi = bits >= 64 ? 0 : hi >> bits;
        x = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    } else if (at < bytes) {                            // rows of less than 16 bytes
        uint64_t lo = 0, hi = 0;
#pragma unroll 1
        for (int i = bytes / (int)sizeof(Elem) - 1; i >= at / (int)sizeof(Elem); --i) {
            uint32_t e = 0;
            __builtin_memcpy(&e, row + i, sizeof(Elem));
            hi = hi << 8 * sizeof(Elem) | lo >> (64 - 8 * sizeof(Elem));
            lo = lo << 8 * sizeof(Elem) | e;
        }
        x = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    }
    return x;
}
// Eight elements of a row from column `col` on.
struct Eight { u32x4 v[kKind == 0 ? 2 : 1]; };
__device__ __forceinline__ Eight load8(const Elem* row, int64_t D, int col) {
    Eight e;
    const int bytes = (int)(D * sizeof(Elem));
#pragma unroll
    for (int i = 0; i < (kKind == 0 ? 2 : 1); ++i) e.v[i] = load16(row, bytes, col * (int)sizeof(Elem) + 16 * i);
    return e;
}
__device__ __forceinline__ void planes_of(const Eight& e, float unit, u32x4 (&out)[NS]) {
    if constexpr (kKind == 0) {
        float x[8];
        __builtin_memcpy(x, &e, sizeof(x));
        split8(x, unit, out);
    } else out[0] = e.v[0];
}

// Four elements of a row as numbers, zero behind its D.
__device__ __forceinline__ f32x4 load4(const Elem* row, int64_t D, int col) {
    f32x4 x = {};
    if (col + 4 <= D) {
        Elem e[4];
        __builtin_memcpy(e, row + col, sizeof(e));
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = value(e[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) if (col + j < D) x[j] = value(row[col + j]);
    }
    return x;
}

// Chunk (of 8 elements, 16 bytes) c of row r of a tile lies at chunk c ^ turn(r) of its row.  LDS serves 256 bytes at a time:
// 16 rows of one chunk (the first product's reads) and 4 rows of four neighbouring ones (the transposing reads) then lie
// on different banks.
template <int DP> __device__ __forceinline__ int turn(int r) {
    return DP == 64 ? 4 * ((r >> 1) & 1) + ((r >> 2) & 3) : 4 * (r & 3) + ((r >> 2) & 3);
}

__device__ __forceinline__ u32x2 read_transposed(const uint16_t* p) {
    using lds_s16x4 = __attribute__((address_space(3))) s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
}

__device__ __forceinline__ void store_elem(void* p, int64_t i, float x) {
    if constexpr (kKind == 0) static_cast<float*>(p)[i] = x;
    else static_cast<uint16_t*>(p)[i] = (uint16_t)(pack2(x, 0.0f) & 0xffff);
}
__device__ __forceinline__ void store4(void* p, int64_t i, f32x4 x) {
    if constexpr (kKind == 0) __builtin_memcpy(static_cast<float*>(p) + i, &x, 16);
    else {
        const u32x2 v = {pack2(x[0], x[1]), pack2(x[2], x[3])};
        __builtin_memcpy(static_cast<uint16_t*>(p) + i, &v, 8);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// powers of two that bring the largest finite element of a row to [2^14, 2^15)
// ---------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ int unit_exponent(float peak, int most) {
    if (!(peak > 0.0f)) return 0;
    int e = 0;
    frexpf(peak, &e);                                   // peak = m * 2^e, m in [0.5, 1)
    e = 15 - e;
    return e < -126 ? -126 : e > most ? most : e;
}
__device__ __forceinline__ float unit_of(float peak, int most = 126) { return ldexpf(1.0f, unit_exponent(peak, most)); }
// Streamed rows: at most 2^80, so that p, of p s, stays in range.  Rows whose largest element is below 2^-82 have fewer bits than 22.
constexpr int kMostUnit = 80;
// What a tile of streamed rows has beside it: s of every row and, in the forward, the binary logarithm of s 2^15 and its inverse
// (2^15: the logarithms of rows with elements around one are small, and a score that one is added to loses nothing).
__device__ __forceinline__ float log_scale(float s) { return (float)((int)(__builtin_bit_cast(uint32_t, s) >> 23) - 127 + 15); }
template <int ROWS> struct Scales {
    float s[ROWS], log[ROWS], inverse[ROWS];
    __device__ __forceinline__ void put(int r, float scale) {
        s[r] = scale;
        log[r] = log_scale(scale);
        inverse[r] = 0x1p-15f / scale;
    }
};
// What scores of scaled tables are multiplied by, at least 2^-126: they are below 2^40, and -inf, a class that there is not, stays.
__device__ __forceinline__ float not_zero(float x) { return fmaxf(x, 0x1p-126f); }
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < __builtin_inff() ? a : 0.0f;
}
// Largest of n partial peaks, by the whole workgroup; `room` is a word of LDS per wave.
template <int WAVES>
__device__ __forceinline__ float block_peak(const float* peaks, int n, float* room) {
    float m = 0.0f;
    for (int i = threadIdx.x; i < n; i += WAVES * 64) m = fmaxf(m, peaks[i]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) m = fmaxf(m, room[i]);
    __syncthreads();
    return m;
}
// Unit of the gradients: of |g| s over rows that live, for fp32 rows, or of |g|.
template <int WAVES = kClassWaves>
__device__ __forceinline__ float grad_unit(const ClassArgs& a, float* room) {
    // bfloat16 has the range as it is: 24 binades keep products that its subnormals can still hold out of fp32's
    if constexpr (!kHalf) return 0x1p24f;
    return unit_of(block_peak<WAVES>(a.at<const float>(a.plan.peaks), kPeaks, room));
}
// The largest finite |x| that a lane holds of a row.
__device__ __forceinline__ float peak_of(const Eight& e) {
    float m = 0.0f;
    if constexpr (kKind == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t bits = e.v[i][j];        // (hipcc casts the vector's first element for e.v[i][j] itself)
                m = fmaxf(m, finite_abs(__builtin_bit_cast(float, bits)));
            }
    }
    return m;
}
__device__ __forceinline__ float wave_max(float m) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    return m;
}

// Logit of slot i of [T,K], before the temperature; -inf: an empty slot, or one that the teacher gives nothing.
__device__ __forceinline__ float slot_score(const ClassArgs& a, int64_t i) {
    if (a.ids[i] < 0) return -__builtin_inff();
    if (!a.teacher) return 0.0f;
    if (a.teacher_kind == 0) return static_cast<const float*>(a.teacher)[i];
    if (a.teacher_kind == 1) return __builtin_bit_cast(float, (uint32_t)static_cast<const uint16_t*>(a.teacher)[i] << 16);
    return (float)static_cast<const _Float16*>(a.teacher)[i];
}
// Whether row t has a slot of any weight, asked by a whole wave.
__device__ __forceinline__ bool row_lives(const ClassArgs& a, int64_t t, int lane) {
    return __any(lane < a.s.K && slot_score(a, t * a.s.K + lane) != -__builtin_inff());
}

// Largest |g| s of fp32 rows that live, or |g|, a part per workgroup.
__global__ __launch_bounds__(kClassThreads) void class_peaks_kernel(ClassArgs a) {
    __shared__ float room[kClassWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float m = 0.0f;
    for (int64_t t = (int64_t)blockIdx.x * kClassWaves + wave; t < a.s.T; t += (int64_t)gridDim.x * kClassWaves) {
        if (!row_lives(a, t, lane)) continue;
        float peak = 0.0f;
        if constexpr (kKind == 0)
            for (int d = lane; d < a.s.D; d += 64) peak = fmaxf(peak, finite_abs(value(static_cast<const Elem*>(a.h)[t * a.h_stride + d])));
        const int e = kKind == 0 ? unit_exponent(wave_max(peak), kMostUnit) : 0;
        m = fmaxf(m, fminf(ldexpf(finite_abs(a.grad_loss[t]), -e), 0x1.fffffep127f));
    }
    if (lane == 0) room[wave] = m;
    __syncthreads();
    if (threadIdx.x == 0) a.at<float>(a.plan.peaks)[blockIdx.x] = fmaxf(fmaxf(room[0], room[1]), fmaxf(room[2], room[3]));
}

// Where chunk c of row r lies in planes of rows of DP elements, in elements.  Wide planes lie as a wave fetches them: by
// tiles of 32 rows, quarters of the row, and 64 chunks an instruction (chunks lane%4 + 4 (i/2) of rows lane/4 + 16 (i%2)).
template <int DP> __device__ __forceinline__ int64_t plane_place(int64_t r, int c) {
    if constexpr (narrow_depth(DP)) return r * DP + c * 8;
    constexpr int chunks = DP / kClassWaves / 8, each = kBlock * chunks / 64;
    const int q = c / chunks, cc = c % chunks, rr = (int)(r % kBlock);
    return (((r / kBlock * kClassWaves + q) * each + 2 * (cc / 4) + rr / 16) * 64 + rr % 16 * 4 + cc % 4) * 8;
}

// ---------------------------------------------------------------------------------------------------------------
// backward, ahead of the products: planes of h (rows without a slot are zero, whatever they hold), what a row brings
// along, the slots sorted, and the gradient of h
// ---------------------------------------------------------------------------------------------------------------
// The teacher's weights of row t over its slots, in lanes 0..K-1 (K <= 64): a softmax over the slots that name a class.
__device__ __forceinline__ float slot_weight(const ClassArgs& a, int64_t t, int lane, int& id, float& log_weight) {
    id = -1;
    float x = -__builtin_inff();
    if (lane < a.s.K) {
        const int64_t i = t * a.s.K + lane;
        id = a.ids[i];
        x = slot_score(a, i);
    }
    log_weight = 0.0f;
    if (!a.teacher) return id >= 0 ? 1.0f : 0.0f;
    float top = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    if (top == -__builtin_inff()) top = 0.0f;           // no slot, or none with any weight
    x = (x - top) * a.inv_temperature;                  // differences alone: a logit over the temperature may be out of range
    const float e = id < 0 ? 0.0f : expf(x);
    float sum = e;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (sum == 0.0f) { id = -1; return 0.0f; }          // teacher gives its classes no weight: as a row without slots
    log_weight = x - logf(sum);
    return e / sum;
}

// What the gradient knows of 32 rows' slots in one bucket: where they lie, how many, and whether any of the rows has a
// negative gradient.
struct SlotWord {
    uint32_t w;
    __device__ __forceinline__ int start() const { return w & 2047; }
    __device__ __forceinline__ int count() const { return w >> 11 & 4095; }
    __device__ __forceinline__ bool negative() const { return w >> 31; }
};
// A slot: its row of the 32 above 27 bits of class, and g (q - p), sorted with the units of the gradient and never zero.
struct Slot { uint32_t key; float pull; };

constexpr int kRowThreads = 1024, kRowWaves = kRowThreads / 64, kRowsEach = kBlock / kRowWaves;

// Row t of grad_h, by a wave: what the forward made of it, times the gradient of its loss.
__device__ __forceinline__ void write_row_grad(const ClassArgs& a, int64_t t, float g, bool lives, int lane) {
    for (int d = lane; d < a.s.D; d += 64)
        store_elem(a.grad_h, t * a.s.D + d, lives ? g * a.row_grad_in[t * a.s.D + d] : 0.0f);
}
__global__ __launch_bounds__(kClassThreads) void class_row_grad_kernel(ClassArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * kClassWaves + (threadIdx.x >> 6);
    if (t >= a.s.T) return;
    int id;
    float log_weight;
    slot_weight(a, t, lane, id, log_weight);
    write_row_grad(a, t, a.grad_loss[t], __any(id >= 0), lane);
}

// Scores of slots' classes are sums in 64 bits, few as they are: in fp32 the rounding of a score near 20 would be 1e-6 of p.
__device__ __forceinline__ float probability(double score, double lse) {
    const float p = exp2f((float)((score - lse) * kLog2eDouble));
    return p > 1.0f ? 1.0f : p;                         // (NaN stays)
}
__device__ __forceinline__ double dot4(f32x4 x, f32x4 y) {
    return ((double)x[0] * y[0] + (double)x[1] * y[1]) + ((double)x[2] * y[2] + (double)x[3] * y[3]);
}
// A class that several slots of a row name is the first one's, with the weights in slot order; false for the others, and for
// slots that name no class of the table.  IDs and weights in lanes 0..K-1.
__device__ __forceinline__ bool merge_slots(const ClassArgs& a, int id, float& q) {
    const int lane = threadIdx.x & 63;
    const float own = q;
    bool first = id >= 0 && id < a.s.V;
    for (int j = 0; j < a.s.K && a.s.K > 1; ++j) {
        const int other = __builtin_amdgcn_readlane(id, j);
        const float more = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, own), j));
        if (other == id && j < lane) first = false;
        if (other == id && j > lane) q += more;
    }
    return first;
}
// p of the classes that lanes [from, to) name for row t (an ID behind the last class: 0), by the dot product of the elements
// themselves; `lanes` of the wave to a class, four classes to a group of them at a time.
__device__ __forceinline__ float slot_probability(const ClassArgs& a, int64_t t, int id, int lane, int lanes, int from, int to) {
    const Elem *h = static_cast<const Elem*>(a.h) + t * a.h_stride, *w = static_cast<const Elem*>(a.w);
    const int groups = 64 / lanes, group = lane / lanes, l = lane % lanes;
    const bool known = id >= 0 && id < a.s.V;
    double z = 0.0;
    for (int j = from; j < to; j += 4 * groups) {
        const Elem* row[4];
        double dot[4] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = j + i * groups + group, of = __shfl(known ? id : -1, k & 63);
            row[i] = of >= 0 && k < to ? w + of * a.w_stride : nullptr;
        }
        for (int c = 4 * l; c < a.s.D; c += 4 * lanes) {
            const f32x4 x = load4(h, a.s.D, c);
            f32x4 y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = row[i] ? load4(row[i], a.s.D, c) : f32x4{};
#pragma unroll
            for (int i = 0; i < 4; ++i) dot[i] += dot4(x, y[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            for (int d = 1; d < lanes; d *= 2) dot[i] += __shfl_xor(dot[i], d);
            const int k = j + i * groups;
            const double mine = __shfl(dot[i], (lane - k) * lanes & 63);
            if (lane >= k && lane < k + groups) z = mine;
        }
    }
    return known ? probability(z * a.scale, a.lse_in[t]) : 0.0f;
}
// The same of rows [t, t + N) of one slot each, the whole wave to a class, all rows at a time.
template <int N> __device__ __forceinline__ void target_probability(const ClassArgs& a, int64_t t, int lane, float (&p)[N]) {
    const Elem *h[N], *w[N];
    double dot[N] = {};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int id = t + k < a.s.T ? a.ids[t + k] : -1;
        h[k] = static_cast<const Elem*>(a.h) + (t + k) * a.h_stride;
        w[k] = id >= 0 && id < a.s.V ? static_cast<const Elem*>(a.w) + id * a.w_stride : nullptr;
    }
    for (int c = 4 * lane; c < a.s.D; c += 256) {
        f32x4 x[N] = {}, y[N] = {};
#pragma unroll
        for (int k = 0; k < N; ++k) if (w[k]) { x[k] = load4(h[k], a.s.D, c); y[k] = load4(w[k], a.s.D, c); }
#pragma unroll
        for (int k = 0; k < N; ++k) dot[k] += dot4(x[k], y[k]);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < N; ++k) dot[k] += __shfl_xor(dot[k], d);
#pragma unroll
    for (int k = 0; k < N; ++k) p[k] = w[k] ? probability(dot[k] * a.scale, a.lse_in[t + k]) : 0.0f;
}

// The slots of a row that the gradient sorts, in lanes 0..K-1, as their class (-1: none) and g (q - p): places of the classes that
// a row names are left out of the products, which round p, because of a row that has learned its class only p - q is left.
// Each place of [row][class] is one slot's.
__device__ __forceinline__ Slot row_slot(const ClassArgs& a, int id, float q, float p, float g) {
    const bool some = merge_slots(a, id, q);
    return Slot{some ? (uint32_t)id : ~0u, g * (q - p)};
}

// Rows of more than one slot, ahead of the sorting: one workgroup per row, as many slots to a wave as it scores at a time.  Bound by the reads of
// the classes' rows: 4096 rows of 32 slots, 128 bfloat16 (33 MB of rows) 28 us.
__global__ __launch_bounds__(kRowThreads) void class_slots_kernel(ClassArgs a, int lanes) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = blockIdx.x;
    const int each = 4 * (64 / lanes), from = wave * each, to = from + each < a.s.K ? from + each : a.s.K;
    int id;
    float log_weight;
    const float weight = slot_weight(a, t, lane, id, log_weight);
    const bool lives = __any(id >= 0);
    const float p = lives ? slot_probability(a, t, id, lane, lanes, from, to) : 0.0f;
    const Slot s = row_slot(a, id, weight, p, lives ? a.grad_loss[t] : 0.0f);
    if (lane >= from && lane < to) a.at<Slot>(a.plan.row_slots)[t * a.s.K + lane] = s;
}

// One workgroup per 32 rows, two to a wave.  Latency alone, 11 to 24 us: the chain from IDs over logits or the classes' rows to
// the sorted slots.
template <int DP>
__global__ __launch_bounds__(kRowThreads) void class_rows_kernel(ClassArgs a, int64_t padded) {
    __shared__ float room[kRowWaves];
    __shared__ uint32_t signs, counts[kMostBuckets], sums[kRowWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const ClassBuckets bk = a.buckets;
    if (threadIdx.x == 0) signs = 0;
    for (int i = threadIdx.x; i < bk.count; i += kRowThreads) counts[i] = 0;
    const float unit = grad_unit<kRowWaves>(a, room);
    uint16_t* planes = a.at<uint16_t>(a.plan.rows);
    __syncthreads();
    int ids[kRowsEach];
    float pulls[kRowsEach], target[kRowsEach] = {};
    if (!a.plan.row_slots) target_probability(a, (int64_t)blockIdx.x * kBlock + wave * kRowsEach, lane, target);
#pragma unroll
    for (int k = 0; k < kRowsEach; ++k) {
        const int q = wave * kRowsEach + k;
        const int64_t t = (int64_t)blockIdx.x * kBlock + q;
        int id = -1;
        float log_weight, weight = 0.0f;
        if (t < a.s.T) weight = slot_weight(a, t, lane, id, log_weight);
        const bool lives = __any(id >= 0);
        constexpr int kEach = (DP / 8 + 63) / 64;
        Eight e[kEach];
        float peak = 0.0f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = lane + 64 * i;
            e[i] = Eight{};
            if (lives && c * 8 < a.s.D) e[i] = load8(static_cast<const Elem*>(a.h) + t * a.h_stride, a.s.D, c * 8);
            peak = fmaxf(peak, peak_of(e[i]));
        }
        const int exponent = kKind == 0 ? unit_exponent(wave_max(peak), kMostUnit) : 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int c = lane + 64 * i;
            if (c >= DP / 8) break;
            u32x4 p[NS];
            planes_of(e[i], ldexpf(1.0f, exponent), p);
#pragma unroll
            for (int n = 0; n < NS; ++n) *reinterpret_cast<u32x4*>(planes + (int64_t)n * padded * DP + plane_place<DP>(t, c)) = p[n];
        }
        const int up = (kKind == 0 ? (int)(__builtin_bit_cast(uint32_t, unit) >> 23) - 127 : 0) - exponent;       // the unit times s
        const float loss_grad = lives ? a.grad_loss[t] : 0.0f, g = kKind == 0 ? ldexpf(loss_grad, up) : loss_grad * unit;
        if (a.grad_h && t < a.s.T) write_row_grad(a, t, loss_grad, lives, lane);
        // P = |g| * softmax = 2^(score * log2e + start), its sign apart
        if (lane == 0) {
            a.at<float>(a.plan.start)[t] = lives ? log2f(fabsf(g)) - a.lse_in[t] * kLog2e : -__builtin_inff();
            if constexpr (kKind == 0) a.at<float>(a.plan.scales)[t] = ldexpf(1.0f, -exponent);
            if (g < 0.0f) atomicOr(&signs, 1u << q);
        }
        Slot own{~0u, 0.0f};
        if (!a.plan.row_slots) own = row_slot(a, id, weight, target[k], loss_grad);
        else if (t < a.s.T && lane < a.s.K) own = a.at<const Slot>(a.plan.row_slots)[t * a.s.K + lane];
        ids[k] = (int)own.key;
        pulls[k] = kKind == 0 ? ldexpf(own.pull, up) : own.pull * unit;
        if (pulls[k] == 0.0f) pulls[k] = 0x1p-126f;     // (a place that is named is told by not being zero)
        if (ids[k] >= 0) atomicAdd(&counts[(uint32_t)ids[k] / kBlock / (uint32_t)bk.per], 1u);
    }
    __syncthreads();
    // counts to places, four buckets to a thread
    static_assert(kMostBuckets <= 4 * kRowThreads, "a thread has four buckets");
    uint32_t mine[4], before = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = 4 * threadIdx.x + j;
        mine[j] = i < bk.count ? counts[i] : 0;
        before += mine[j];
    }
    const uint32_t total = before;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(before, d);
        if (lane >= d) before += o;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    before -= total;
    for (int i = 0; i < wave; ++i) before += sums[i];
    uint32_t* words = a.at<uint32_t>(a.plan.buckets) + (int64_t)blockIdx.x * bk.count;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = 4 * threadIdx.x + j;
        if (i < bk.count) {
            words[i] = (mine[j] ? before : 0) | mine[j] << 11 | (signs ? 1u << 31 : 0);
            counts[i] = before;
        }
        before += mine[j];
    }
    __syncthreads();
    Slot* slots = a.at<Slot>(a.plan.slots) + (int64_t)blockIdx.x * kBlock * a.s.K;
#pragma unroll
    for (int k = 0; k < kRowsEach; ++k)
        if (ids[k] >= 0)
            slots[atomicAdd(&counts[(uint32_t)ids[k] / kBlock / (uint32_t)bk.per], 1u)] = Slot{(uint32_t)(wave * kRowsEach + k) << 27 | (uint32_t)ids[k], pulls[k]};
    if (threadIdx.x == 0) a.at<uint32_t>(a.plan.signs)[blockIdx.x] = signs;
}

// The slots that a wave's (or a wide workgroup's) 32 classes have in the streamed blocks, M blocks of a tile: words are
// asked for two tiles ahead, slots one, so that nothing of it is waited for.
template <int M>
struct SlotFeed {
    const uint32_t* words;                              // of this bucket, a block of rows apart
    const Slot* slots;
    int64_t buckets, block_slots, blocks;
    uint32_t first_class;
    SlotWord ahead[M], next[M], now[M];
    Slot next_slot[M], slot[M];
    __device__ __forceinline__ SlotFeed(const ClassArgs& a, int64_t padded, int64_t v0) {
        const ClassBuckets bk = a.buckets;
        const uint32_t block = (uint32_t)(v0 < a.s.V ? v0 / kBlock : 0);
        words = a.at<const uint32_t>(a.plan.buckets) + block / (uint32_t)bk.per;
        slots = a.at<const Slot>(a.plan.slots);
        buckets = bk.count; block_slots = (int64_t)kBlock * a.s.K; blocks = padded / kBlock;
        first_class = (uint32_t)v0;
    }
    __device__ __forceinline__ void ask_words(int64_t block) {
#pragma unroll
        for (int m = 0; m < M; ++m) ahead[m].w = block + m < blocks ? words[(block + m) * buckets] : 0;
    }
    __device__ __forceinline__ void ask_slots(int64_t block, int lane) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            next[m].w = __builtin_amdgcn_readfirstlane(ahead[m].w);
            next_slot[m] = Slot{~0u, 0.0f};
            if (lane < next[m].count()) next_slot[m] = slots[(block + m) * block_slots + next[m].start() + lane];
        }
    }
    __device__ __forceinline__ void turn() {
#pragma unroll
        for (int m = 0; m < M; ++m) { now[m] = next[m]; slot[m] = next_slot[m]; }
    }
    // What the slots of block m take, into cells[row][class]; whether there was one (wave-uniform).
    __device__ __forceinline__ bool gather(int m, int64_t block, int lane, float* cells) const {
        if (now[m].count() == 0) return false;
        bool hit = false;
        Slot s = slot[m];
        for (int e = lane;;) {
            const uint32_t c = (s.key & 0x7ffffffu) - first_class;
            if (e < now[m].count() && c < (uint32_t)kBlock) {
                cells[(s.key >> 27) * kBlock + c] = s.pull;
                hit = true;
            }
            e += 64;
            if (e - lane >= now[m].count()) break;
            if (e < now[m].count()) s = slots[block * block_slots + now[m].start() + e];
        }
        return __any(hit);
    }
};

// The table as planes of padded rows, zero behind its last row and element, and s of fp32 rows.  Bound by memory: 2.5 M x 128 fp32,
// 1.28 GB in and out each, 0.47 ms (5.4 TB/s).
template <int DP>
__global__ __launch_bounds__(kClassThreads) void class_pack_kernel(ClassArgs a, int64_t rows) {
    uint16_t* planes = a.at<uint16_t>(a.plan.table);
    if constexpr (kKind == 0 && !narrow_depth(DP)) {    // tiles of 32 rows, a quarter to a wave, as its planes lie
        constexpr int chunks = DP / kClassWaves / 8, each = kBlock * chunks / 64;
        __shared__ float room[kClassWaves][kBlock];
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        for (int64_t tile = blockIdx.x; tile < rows / kBlock; tile += gridDim.x) {
            Eight e[each];
            float peak[2] = {}, unit[2];
#pragma unroll
            for (int i = 0; i < each; ++i) {
                const int64_t v = tile * kBlock + (lane >> 2) + 16 * (i & 1);
                const int c = wave * chunks + (lane & 3) + 4 * (i >> 1);
                e[i] = Eight{};
                if (v < a.s.V && c * 8 < a.s.D) e[i] = load8(static_cast<const Elem*>(a.w) + v * a.w_stride, a.s.D, c * 8);
                peak[i & 1] = fmaxf(peak[i & 1], peak_of(e[i]));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                peak[i] = fmaxf(peak[i], __shfl_xor(peak[i], 1));
                peak[i] = fmaxf(peak[i], __shfl_xor(peak[i], 2));
                if ((lane & 3) == 0) room[wave][(lane >> 2) + 16 * i] = peak[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = (lane >> 2) + 16 * i;
                unit[i] = unit_of(fmaxf(fmaxf(room[0][r], room[1][r]), fmaxf(room[2][r], room[3][r])), kMostUnit);
                if (wave == 0 && (lane & 3) == 0) a.at<float>(a.plan.table_scales)[tile * kBlock + r] = 1.0f / unit[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < each; ++i) {
                u32x4 p[NS];
                planes_of(e[i], unit[i & 1], p);
#pragma unroll
                for (int n = 0; n < NS; ++n)
                    *reinterpret_cast<u32x4*>(planes + (int64_t)n * rows * DP + (((tile * kClassWaves + wave) * each + i) * 64 + lane) * 8) = p[n];
            }
        }
        return;
    }
    for (int64_t q = (int64_t)blockIdx.x * kClassThreads + threadIdx.x; q < rows * (DP / 8); q += (int64_t)gridDim.x * kClassThreads) {
        int64_t v = q / (DP / 8);                       // chunk q of the planes, in their own order
        int c = (int)(q % (DP / 8));
        if constexpr (!narrow_depth(DP)) {
            constexpr int chunks = DP / kClassWaves / 8, each = kBlock * chunks / 64;
            const int lane = (int)(q % 64);
            const int64_t load = q / 64, i = load % each, quarter = load / each % kClassWaves;
            v = load / each / kClassWaves * kBlock + (lane >> 2) + 16 * (i & 1);
            c = (int)(quarter * chunks + (lane & 3) + 4 * (i >> 1));
        }
        Eight e = {};
        if (v < a.s.V && c * 8 < a.s.D) e = load8(static_cast<const Elem*>(a.w) + v * a.w_stride, a.s.D, c * 8);
        float unit = 1.0f;
        if constexpr (kKind == 0) {                     // DP / 8 neighbouring lanes have a row
            float peak = peak_of(e);
#pragma unroll
            for (int d = 1; d < DP / 8; d *= 2) peak = fmaxf(peak, __shfl_xor(peak, d));
            unit = unit_of(peak, kMostUnit);
            if (c == 0) a.at<float>(a.plan.table_scales)[v] = 1.0f / unit;
        }
        u32x4 p[NS];
        planes_of(e, unit, p);
#pragma unroll
        for (int n = 0; n < NS; ++n) *reinterpret_cast<u32x4*>(planes + (int64_t)n * rows * DP + q * 8) = p[n];
    }
}

// ---------------------------------------------------------------------------------------------------------------
// the streamed side in LDS: ROWS rows of DP elements, NS planes
// ---------------------------------------------------------------------------------------------------------------
template <int DP, int ROWS>
struct Tile {
    static constexpr int kChunks = ROWS * DP / 8, kEach = kChunks / kClassThreads;
    static constexpr int kPlane = ROWS * DP;            // elements
    static_assert(kChunks % kClassThreads == 0, "threads share a tile evenly");

    // Rows [first, first + ROWS) of the table, those behind its last row repeat it.
    struct FromTable {
        Eight e[kEach];
        __device__ __forceinline__ void load(const Elem* w, int64_t stride, int64_t V, int64_t D, int64_t first) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int q = i * kClassThreads + threadIdx.x, r = q / (DP / 8), c = q % (DP / 8);
                const int64_t v = first + r < V ? first + r : V - 1;
                e[i] = load8(w + v * stride, D, c * 8);
            }
        }
        // (DP / 8 neighbouring lanes have a row)
        __device__ __forceinline__ void store(uint16_t* lds, Scales<ROWS>* scales) const {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int q = i * kClassThreads + threadIdx.x, r = q / (DP / 8), c = q % (DP / 8);
                float unit = 1.0f;
                if constexpr (kKind == 0) {
                    float peak = peak_of(e[i]);
#pragma unroll
                    for (int d = 1; d < DP / 8; d *= 2) peak = fmaxf(peak, __shfl_xor(peak, d));
                    unit = unit_of(peak, kMostUnit);
                    if (c == 0) scales->put(r, 1.0f / unit);
                }
                u32x4 p[NS];
                planes_of(e[i], unit, p);
#pragma unroll
                for (int n = 0; n < NS; ++n) *reinterpret_cast<u32x4*>(lds + n * kPlane + r * DP + (c ^ turn<DP>(r)) * 8) = p[n];
            }
        }
    };
    // The same of 16-bit planes of rows of DP elements on the 16-byte grid, `rows` of them; a thread's share lies at fixed
    // places from the tile's first row on.
    struct FromPlanes {
        static constexpr int kStep = kClassThreads / (DP / 8);     // rows from one of a thread's chunks to the next
        u32x4 p[NS][kEach];
        __device__ __forceinline__ void load(const char* planes, int row_bytes, int64_t plane_bytes, int64_t rows, int64_t first) {
            const uint32_t place = threadIdx.x / (DP / 8) * row_bytes + threadIdx.x % (DP / 8) * 16;
            if (first + ROWS <= rows) {
#pragma unroll
                for (int n = 0; n < NS; ++n)
#pragma unroll
                    for (int i = 0; i < kEach; ++i)
                        p[n][i] = *reinterpret_cast<const u32x4*>(planes + n * plane_bytes + (first + i * kStep) * row_bytes + place);
            } else {
                asm volatile("");                       // the last tile of a table as it is
#pragma unroll
                for (int n = 0; n < NS; ++n)
#pragma unroll
                    for (int i = 0; i < kEach; ++i) {
                        int64_t r = first + i * kStep + threadIdx.x / (DP / 8);
                        if (r >= rows) r = rows - 1;
                        p[n][i] = *reinterpret_cast<const u32x4*>(planes + n * plane_bytes + r * row_bytes + threadIdx.x % (DP / 8) * 16);
                    }
            }
        }
        __device__ __forceinline__ void store(uint16_t* lds) const {
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const int q = i * kClassThreads + threadIdx.x, r = q / (DP / 8), c = q % (DP / 8);
                    *reinterpret_cast<u32x4*>(lds + n * kPlane + r * DP + (c ^ turn<DP>(r)) * 8) = p[n][i];
                }
        }
    };

    // A operand of the first product: block b, step ks of 16 elements.
    static __device__ __forceinline__ void rows(const uint16_t* lds, int b, int ks, int lane, u32x4 (&out)[NS]) {
        const int r = b * kBlock + (lane & 31), c = 2 * ks + (lane >> 5);
#pragma unroll
        for (int n = 0; n < NS; ++n) out[n] = *reinterpret_cast<const u32x4*>(lds + n * kPlane + r * DP + (c ^ turn<DP>(r)) * 8);
    }
    // A operand of the second: elements 32*db.., step s of 16 rows of block b, the rows in the order of a result's registers.
    static __device__ __forceinline__ void columns(const uint16_t* lds, int b, int s, int db, int lane, u32x4 (&out)[NS]) {
        const int i = lane & 15, r = b * kBlock + 16 * s + 4 * (lane >> 5) + (i >> 2);
        const int c = 4 * db + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const int t = c ^ turn<DP>(r);              // row r + 8 turns by 2 more
            const uint16_t* p = lds + n * kPlane + r * DP + (i & 1) * 4;
            const u32x2 a = read_transposed(p + t * 8), z = read_transposed(p + 8 * DP + (t ^ 2) * 8);
            out[n] = u32x4{a[0], a[1], z[0], z[1]};
        }
    }
};

// P of a block as the second product's B operand, its two steps; planes of what fp16 or bfloat16 takes of it, nearest even.
__device__ __forceinline__ void operand_of(const float (&p)[16], u32x4 (&out)[2][NS]) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = p[8 * s + j];
        split8(x, 1.0f, out[s]);
    }
}

// P's operand without the places that slots name: bit i of `named` is register i of this lane's result.
__device__ __forceinline__ void leave_out(uint32_t named, u32x4 (&q)[2][NS]) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t two = named >> (8 * s + 2 * j), keep = ((two & 1) - 1 & 0xffffu) | ((two >> 1 & 1) - 1 & 0xffff0000u);
#pragma unroll
            for (int n = 0; n < NS; ++n) q[s][n][j] &= keep;
        }
}

// Row that register i of a result stands for, in its block.
__device__ __forceinline__ int row_of(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

// Columns [col0, col0 + 16 KS) of a row as B operands, and the row's unit: that of what `join` makes of the peak of a lane's columns.
template <int KS, class Join>
__device__ __forceinline__ float hold(const Elem* row, int64_t D, int col0, int lane, u32x4 (&held)[KS][NS], Join join) {
    Eight e[KS];
    float peak = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int col = col0 + 16 * ks + 8 * (lane >> 5);
        e[ks] = Eight{};
        if (col < D) e[ks] = load8(row, D, col);
        peak = fmaxf(peak, peak_of(e[ks]));
    }
    const float unit = kKind == 0 ? unit_of(join(peak)) : 1.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) planes_of(e[ks], unit, held[ks]);
    return unit;
}
// The peak of a row that two lanes hold.
__device__ __forceinline__ float both_halves(float peak) { return fmaxf(peak, __shfl_xor(peak, 32)); }
// Row `row` of h, or its last one.
__device__ __forceinline__ const Elem* held_row(const ClassArgs& a, int64_t row) {
    return static_cast<const Elem*>(a.h) + (row < a.s.T ? row : a.s.T - 1) * a.h_stride;
}
// Two values of P, registers 2j and 2j + 1 of step s, into that step's B operand; planes of what fp16 or bfloat16 takes of
// them, nearest even.
__device__ __forceinline__ void put2(float a, float b, int j, u32x4 (&out)[NS]) {
    out[0][j] = pack2(a, b);
    if constexpr (NS == 2) out[1][j] = pack2(a - low2(out[0][j]), b - high2(out[0][j]));
}

template <int N> using number = std::integral_constant<int, N>;
template <class F, int... I> __device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) { (f(number<I>{}), ...); }
// f(number<0>), ..., f(number<N - 1>)
template <int N, class F> __device__ __forceinline__ void each(F f) { each_of(f, std::make_integer_sequence<int, N>{}); }

// One tile further: the scores of the tile `ahead` and the products of the tile `tile` with P, which element(m, i) makes of
// the scores that `tile` had, a matrix instruction at a time.  Between two of them stand the reads for three further on
// and a share of the exponentials, a block's own while the products before it run, so that the matrix unit, LDS and the
// vector unit work side by side; the compiler's own order waited for every read.  ready(m, q) sees a block's operand.
//
// WITHIN: scores and products of one tile (ahead == tile); a block is exponentiated while the next one's scores, or the
// products of the one before, run.  It keeps no scores from one tile to the next.
template <int DP, int BLOCKS, int MY, bool PRODUCT, bool WITHIN, class Element, class Ready>
__device__ __forceinline__ void advance(const uint16_t* ahead, const uint16_t* tile, int block0, int lane,
                                        const u32x4 (&held)[DP / 16][NS], f32x16 (&score)[MY], f32x16* acc, Element element, Ready ready) {
    constexpr int KS = DP / 16, DB = DP / 32;
    constexpr int S = MY * KS, EACH = 2 * DB, ALL = S + (PRODUCT ? MY * EACH : 0), R = 4;
    using T = Tile<DP, BLOCKS * kBlock>;
    u32x4 ring[R][NS], q[2][2][NS];
    float even = 0.0f;
    auto load = [&](auto at) {
        constexpr int k = at();
        if constexpr (k < S) T::rows(ahead, block0 + (WITHIN ? k / KS : k % MY), WITHIN ? k % KS : k / MY, lane, ring[k % R]);
        else if constexpr (k < ALL) T::columns(tile, block0 + (k - S) / EACH, (k - S) % EACH / DB, (k - S) % DB, lane, ring[k % R]);
    };
    auto elements = [&](auto block, auto from, auto to) {
        constexpr int m = block(), first = from();
        each<to() - first>([&](auto n) {
            constexpr int i = first + n();
            const float p = element(m, i);
            if constexpr (i & 1) put2(even, p, i / 2 % 4, q[m & 1][i / 8]);
            even = p;
        });
    };
    each<R - 1>([&](auto k) { load(k); });
    each<ALL>([&](auto at) {
        constexpr int k = at();
        load(number<k + R - 1>{});
        if constexpr (k < S) {
            constexpr int m = WITHIN ? k / KS : k % MY, ks = WITHIN ? k % KS : k / MY;
            score[m] = matmul(ring[k % R], held[ks], ks == 0 ? f32x16{} : score[m]);
            if constexpr (WITHIN) {
                if constexpr (m == 1) elements(number<0>{}, number<16 * ks / KS>{}, number<16 * (ks + 1) / KS>{});
                else if constexpr (MY == 1 && k == S - 1) elements(number<0>{}, number<0>{}, number<16>{});
            } else if constexpr (PRODUCT) elements(number<0>{}, number<16 * k / S>{}, number<16 * (k + 1) / S>{});
            else each<MY>([&](auto j) {                 // no products to hide other blocks' behind
                elements(j, number<16 * k / S>{}, number<16 * (k + 1) / S>{});
            });
        } else {
            constexpr int o = k - S, m = o / EACH;
            acc[o % DB] = matmul(ring[k % R], q[m & 1][o % EACH / DB], acc[o % DB]);
            if constexpr (m + 1 < MY) elements(number<m + 1>{}, number<16 * (o % EACH) / EACH>{}, number<16 * (o % EACH + 1) / EACH>{});
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (PRODUCT && k == S - 1) ready(0, q[0]);
        if constexpr (PRODUCT && k >= S && (k - S) % EACH == EACH - 1 && (k - S) / EACH + 1 < MY) {
            constexpr int m = (k - S) / EACH + 1;
            ready(m, q[m & 1]);
        }
    });
}

// ---------------------------------------------------------------------------------------------------------------
// classes that the held rows' slots name, for the forward
// ---------------------------------------------------------------------------------------------------------------
// Their places are left out of the sums of p and of p w (theirs are added when the parts are joined).  A wave
// asks for the next tile that has one with one comparison of scalars: looking at every tile's slots, or masking P between the
// products, took the loop's registers and up to half of its speed.
// Up to two slots a row lie in a register of the wave; more of them in a list for every 32 rows in the order of the classes, class *
// 32 + row, that a launch ahead sorts, but for workgroups of few tiles, which look all of them through.  Latency alone, 10 us (10 slots a row) to 21 (64).
__global__ __launch_bounds__(kRowThreads) void class_named_kernel(ClassArgs a, int classes) {
    __shared__ uint32_t keys[kBlock * 64];
    __shared__ int count;
    const int64_t t0 = (int64_t)blockIdx.x * kBlock;
    int size = 2 * kRowThreads;                         // a power of two
    while (size / 2 >= kBlock * a.s.K) size /= 2;
    for (int e = threadIdx.x; e < size; e += kRowThreads) keys[e] = ~0u;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    for (int e = threadIdx.x; e < kBlock * a.s.K; e += kRowThreads) {
        const int row = e / a.s.K;
        const int id = t0 + row < a.s.T ? a.ids[t0 * a.s.K + e] : -1;
        if (id >= 0 && id < a.s.V) { keys[e] = (uint32_t)id << 5 | (uint32_t)row; atomicAdd(&count, 1); }
    }
    for (int run = 2; run <= size; run *= 2)            // bitonic: runs of this length in turns up and down
        for (int d = run / 2; d > 0; d /= 2) {
            // (pairs up to 64 apart stay within the 128 keys of a wave)
            if (d >= 64 || run == 2) __syncthreads();
            else __builtin_amdgcn_wave_barrier();
            const int i = threadIdx.x / d * 2 * d + threadIdx.x % d;
            if (i < size) {
                const uint32_t x = keys[i], y = keys[i + d];
                if ((x > y) == ((i & run) == 0)) { keys[i] = y; keys[i + d] = x; }
            }
        }
    __syncthreads();
    const int n = count;
    uint32_t* list = a.at<uint32_t>(a.plan.named) + (int64_t)blockIdx.x * kBlock * a.s.K;
    for (int e = threadIdx.x; e < n; e += kRowThreads) list[e] = keys[e];
    uint32_t* starts = a.at<uint32_t>(a.plan.named_starts) + (int64_t)blockIdx.x * (a.cut.parts + 1);
    for (int p = threadIdx.x; p <= a.cut.parts; p += kRowThreads) {
        const int64_t from = p < a.cut.parts ? (int64_t)a.cut.place((unsigned)p).first * classes : a.s.V;
        int lo = 0, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if ((int64_t)(keys[mid] >> 5) < from) lo = mid + 1;
            else hi = mid;
        }
        starts[p] = lo;
    }
}
// What 32 rows name within a workgroup's part of the classes, tiles of CLASSES at a time.
template <int CLASSES> struct Named {
    static constexpr uint32_t kNone = 0x7fffffff;
    const uint32_t* list;                               // null: a lane has a class of its own (negative: none)
    uint32_t keys;                                      // that class, or 64 keys of the list
    int at, end, most;                                  // wave-uniform, as
    uint32_t next;                                      // the next tile that has one
    int last;
    __device__ __forceinline__ void load(int lane) { keys = (at & ~63) + lane < most ? list[(at & ~63) + lane] : 0; }
    // From tile `from` on.
    __device__ __forceinline__ void look(int from) {
        if (list) next = at < end ? ((uint32_t)__builtin_amdgcn_readlane((int)keys, at & 63) >> 5) / CLASSES : kNone;
        else {
            const int tile = (int)keys >= 0 ? (int)(keys / CLASSES) : -1;
            uint32_t m = tile >= from && tile < last ? tile : kNone;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) { const uint32_t o = __shfl_xor(m, d); m = o < m ? o : m; }
            next = __builtin_amdgcn_readfirstlane(m);
        }
    }
    __device__ __forceinline__ Named(const ClassArgs& a, int64_t block, int part, int first, int last_, int lane) : last(last_) {
        most = kBlock * a.s.K;
        if (!a.row_grad) {                              // no gradients wanted: nothing is left out
            list = nullptr;
            next = kNone;
            return;
        }
        if (a.plan.named) {
            list = a.at<const uint32_t>(a.plan.named) + block * most;
            const uint32_t* starts = a.at<const uint32_t>(a.plan.named_starts) + block * (a.cut.parts + 1) + part;
            at = __builtin_amdgcn_readfirstlane(starts[0]);
            end = __builtin_amdgcn_readfirstlane(starts[1]);
            load(lane);
        } else if (a.s.K > kWaveSlots) {
            list = nullptr;
            next = first;
            return;
        } else {
            list = nullptr;
            const int64_t t = block * kBlock + (lane & 31);
            const int id = t < a.s.T && lane < most ? a.ids[t * a.s.K + (lane >> 5)] : -1;
            keys = id < a.s.V ? id : -1;
        }
        look(first);
    }
    // f(whether a lane has one, its row and class of the tile) for up to 64 of tile `it`, the next, at a time.
    template <class F> __device__ __forceinline__ void take_many(const ClassArgs& a, int64_t block, int it, int lane, F f) {
        if (!list) {                                    // few tiles: every slot is looked at for each
            const int64_t rows = a.s.T - block * kBlock;
            const int n = (int)(rows < kBlock ? rows : kBlock) * a.s.K;
#pragma unroll 4
            for (int e = lane; e < n; e += 64) {
                const int id = a.ids[block * most + e];
                f(id >= 0 && id < a.s.V && id / CLASSES == it, e / a.s.K, id % CLASSES);
            }
            next = it + 1;
            return;
        }
        do {
            const int now = __builtin_amdgcn_readfirstlane(at), i = (now & ~63) + lane;
            const bool has = (keys >> 5) / CLASSES == (uint32_t)it && i >= now && i < end;
            f(has, (int)(keys & 31), (int)((keys >> 5) % CLASSES));
            at = now + __popcll(__ballot(has));
            if ((at & 63) == 0 && at < end) load(lane);
            look(it);
        } while (next == (uint32_t)it);
    }
    // f(rows that name it, a bit each, class of the tile) for every class of tile `it`, the next; all of it in scalars, as the
    // waves have no registers left.
    template <class F> __device__ __forceinline__ void take(int it, int lane, F f) {
        if (list) {
            int now = __builtin_amdgcn_readfirstlane(at);
            const int stop = __builtin_amdgcn_readfirstlane(end);
            uint32_t key = __builtin_amdgcn_readlane((int)keys, now & 63), tile;
            do {
                const uint32_t cls = key >> 5;
                uint32_t rows = 0;
                do {
                    rows |= 1u << (key & 31);
                    if ((++now & 63) == 0 && now < stop) { at = now; load(lane); }
                    key = __builtin_amdgcn_readlane((int)keys, now & 63);
                } while (now < stop && key >> 5 == cls);
                f(rows, (int)(cls % CLASSES));
                tile = now < stop ? (key >> 5) / CLASSES : kNone;
            } while (tile == (uint32_t)it);
            at = now;
            next = tile;
        } else {
            for (uint64_t some = __ballot((int)keys >= 0 && keys / CLASSES == (uint32_t)it); some;) {
                const uint32_t cls = __builtin_amdgcn_readlane((int)keys, __builtin_ctzll(some));
                const uint64_t same = __ballot(keys == cls);
                f((uint32_t)(same | same >> 32), (int)(cls % CLASSES));
                some &= ~same;
            }
            look(it + 1);
        }
    }
};

// ---------------------------------------------------------------------------------------------------------------
// forward: a wave holds 32 rows of h, the table streams by
// ---------------------------------------------------------------------------------------------------------------
// Mathematics: p = 2^(score * log2e - ref), ref following a row's maximum; the sum of p and, for the gradient of the row,
// the sum of p times the table's rows, both without the classes that the row's slots name (where gradients are wanted: theirs
// are added, to p with its sum and with p - q, when the parts are joined: of a row that has learned its class 1 - p is far
// below the roundings of p and of its score), all in one pass.
// What bounds it: two products of T V D multiply-adds on the matrix units beside an exponential a score, which takes 16
// cycles for 64 of them, as long as half a product of 128 elements.  4096 rows x 2.5 M classes x 128 bfloat16: 5.06 to 5.4 ms,
// 1.04 to 0.97 PFLOP/s as the card holds its clock, matrix units busy a little over half of the time; a large bfloat16 product of
// the library runs at 1.29.  8 rows, one read of the table: 104 us, 6.0 TB/s.  fp32 rows of up to 64 elements and 16-bit ones of up
// to 128 have no register left: 4 to 41 are spilled around the loop (fp32 64: 14 reads of them a tile).
// Why this way: rows stay in registers and the table streams, because a row's statistics then never leave its lane (an
// accumulator column) until the end; a wave has 32 of them, two waves fit a SIMD (with one: 8.1 ms against 5.6, before the order of advance()).  Few rows: the
// waves of a workgroup share the streamed blocks instead (WY).
//
// Named classes: few of them are taken out of a tile's scores one after the other, 0.3 to 0.6 us each; CROWDED, all of them together,
// which costs every tile registers (1024 x 47 x 100 fp32, 10 slots: 47.9 us and 19.4; 4096 x 2.5 M x
// 128 bfloat16: 5.3 ms and 6.4).
template <int DP, int WY, bool MEAN, bool STRAIGHT, bool CROWDED = false>
__global__ __launch_bounds__(kClassThreads, DP * NS <= 128 ? 2 : 1) void class_forward_kernel(ClassArgs a, int64_t padded) {
    constexpr int NB = blocks_per_tile(WY, DP, kKind), MY = NB / WY, WX = kClassWaves / WY;   // blocks of a tile, a wave's own of them
    using T = Tile<DP, NB * kBlock>;
    constexpr bool AHEAD = WY == 1;
    constexpr int TILES = AHEAD ? 3 : 2;
    __shared__ __align__(16) uint16_t lds[TILES][NS * T::kPlane];
    using Beside = Scales<NB * kBlock>;
    __shared__ __align__(16) Beside scales[kKind == 0 ? TILES : 1];
    __shared__ uint32_t places[CROWDED ? kClassWaves : 1][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, x = wave % WX, y = wave / WX;
    const ClassCut::Place place = a.cut.place(blockIdx.x);
    const int part = place.part, group = place.group, first = place.first, last = place.last;
    if constexpr (CROWDED) places[wave][lane] = 0;
    const int64_t row0 = ((int64_t)group * WX + x) * kBlock, row = row0 + (lane & 31);   // of h, held by this lane
    const bool live = row0 < padded;                      // wave-uniform
    u32x4 held[DP / 16][NS];
    const float to_log2 = not_zero(a.scale * kLog2e / hold<DP / 16>(held_row(a, row), a.s.D, 0, lane, held, both_halves));

    float ref = -3e38f, sum = 0.0f;                     // P = 2^(score - ref); ref = followed maximum - kLift
    f32x16 acc[MEAN ? DP / 32 : 1];
#pragma unroll
    for (auto& f : acc) f = f32x16{};

    // the table as planes (those of the call, or 16-bit rows as they are), or rows of any kind
    typename std::conditional<STRAIGHT, typename T::FromPlanes, typename T::FromTable>::type next;
    const char* planes = a.plan.packed ? a.ws + a.plan.table : static_cast<const char*>(a.w);
    const int row_bytes = 2 * (a.plan.packed ? DP : (int)a.w_stride);
    const int64_t table_rows = a.plan.packed ? padded_rows(a.s.V) : a.s.V;
    float next_scale = 1.0f;
    auto fetch = [&](int it) {
        if (it >= last) return;
        if constexpr (STRAIGHT) next.load(planes, row_bytes, table_rows * row_bytes, table_rows, (int64_t)it * NB * kBlock);
        else next.load(static_cast<const Elem*>(a.w), a.w_stride, a.s.V, a.s.D, (int64_t)it * NB * kBlock);
        if constexpr (kKind == 0 && STRAIGHT)
            if (threadIdx.x < NB * kBlock) next_scale = a.at<const float>(a.plan.table_scales)[(int64_t)it * NB * kBlock + threadIdx.x];
    };
    auto store = [&](int slot) {
        if constexpr (STRAIGHT) {
            next.store(lds[slot]);
            if constexpr (kKind == 0) if (threadIdx.x < NB * kBlock) scales[slot].put(threadIdx.x, next_scale);
        } else next.store(lds[slot], &scales[kKind == 0 ? slot : 0]);
    };
    f32x16 score[MY];
    float top;                                          // of this lane's scores of a tile
    auto scores = [&](const uint16_t* tile) {
#pragma unroll
        for (int m = 0; m < MY; ++m) {
            score[m] = f32x16{};
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) {
                u32x4 f[NS];
                T::rows(tile, y * MY + m, ks, lane, f);
                score[m] = matmul(f, held[ks], score[m]);
            }
        }
    };
    // fp32: the scores become binary logarithms of p s here (with a mean to make or not: the same sums), 16-bit scores those of p when
    // they are exponentiated.
    auto find_top = [&](int it, int slot) {
        if constexpr (kKind == 0)
#pragma unroll
            for (int m = 0; m < MY; ++m)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int r = (y * MY + m) * kBlock + row_of(i, lane);
                    const f32x4 s = *reinterpret_cast<const f32x4*>(&scales[slot].s[r]) * to_log2;
                    const f32x4 l = *reinterpret_cast<const f32x4*>(&scales[slot].log[r]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) score[m][i + j] = fmaf(score[m][i + j], s[j], l[j]);
                }
        if ((int64_t)(it + 1) * NB * kBlock > a.s.V) {  // the last tile: classes that there are not
            asm volatile("");                           // a branch, not sixteen selects in every tile
            const int left = (int)(a.s.V - (int64_t)it * NB * kBlock) - y * MY * kBlock;
#pragma unroll
            for (int m = 0; m < MY; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) if (m * kBlock + row_of(i, lane) >= left) score[m][i] = -__builtin_inff();
        }
        top = score[0][0];
#pragma unroll
        for (int m = 0; m < MY; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, score[m][i]);
        if constexpr (kKind != 0) top *= to_log2;
    };
    auto power = [&](float z) { return __builtin_amdgcn_exp2f(kKind == 0 ? z - ref : fmaf(z, to_log2, -ref)); };

    // Ahead: a tile's scores are made while the tile before it is exponentiated and multiplied; its table rows lie in the
    // next of three LDS tiles by then, those of the tile after it are on their way in registers.
    int slot = 0;
    fetch(first);
    using Places = Named<NB * kBlock>;
    typename std::conditional<MEAN, Places, int>::type named = [&] {
        if constexpr (MEAN) return Places(a, live ? row0 / kBlock : 0, part, first, last, lane);
        else return 0;
    }();
    if constexpr (AHEAD) {
        store(0);
        fetch(first + 1);
        __syncthreads();
        if (live) {
            scores(lds[0]);
            find_top(first, 0);
        }
    }
    for (int it = first; it < last; ++it) {
        const int at = slot;
        uint16_t* tile = lds[at];
        slot = slot + 1 == TILES ? 0 : slot + 1;
        uint16_t* ahead = lds[slot];
        if constexpr (AHEAD) {
            if (it + 1 < last) store(slot);
        } else store(at);
        __syncthreads();
        fetch(it + (AHEAD ? 2 : 1));
        if (!live) continue;
        if constexpr (!AHEAD) {
            scores(tile);
            find_top(it, at);
        }
        if (__any(top - ref > kLift + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float to = top - ref > kLift + kSlack ? top - kLift : ref, by = exp2f(ref - to);     // (of this row alone)
            ref = to;
            sum *= by;
            if constexpr (MEAN)
#pragma unroll
                for (auto& f : acc) f *= by;
        }
        if constexpr (CROWDED) {
            if (named.next == (uint32_t)it) {
                named.take_many(a, row0 / kBlock, it, lane, [&](bool has, int r, int c) {
                    const int b = c / kBlock - y * MY;
                    if (has && b >= 0 && b < MY)
                        atomicOr(&places[wave][r + 32 * (c >> 2 & 1)], 1u << (16 * b + 4 * (c % kBlock >> 3) + (c & 3)));
                });
                __builtin_amdgcn_wave_barrier();
                const uint32_t out = places[wave][lane];        // bit 16 m + i: register i of block m is named
                places[wave][lane] = 0;
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int m = 0; m < MY; ++m)
#pragma unroll
                    for (int i = 0; i < 16; ++i) if (out >> (16 * m + i) & 1) score[m][i] = -__builtin_inff();
            }
        } else if constexpr (MEAN)
            if (named.next == (uint32_t)it)
                named.take(it, lane, [&](uint32_t rows, int c) {
                    const int b = c / kBlock - (WY == 1 ? 0 : __builtin_amdgcn_readfirstlane(y)) * MY, i = 4 * (c % kBlock >> 3) + (c & 3);
                    const bool mine = lane >> 5 == (c >> 2 & 1) && rows >> (lane & 31) & 1;
                    each<MY>([&](auto m) {
                        if (b != m()) return;
                        const float z = score[m()][i];
                        score[m()][i] = mine ? -__builtin_inff() : z;
                    });
                });
        if constexpr (AHEAD) {
            f32x16 now[MY];
#pragma unroll
            for (int m = 0; m < MY; ++m) now[m] = score[m];
            float some[2] = {};                         // (behind the last tile the scores are of no use, and unused)
            f32x4 back[MEAN ? 1 : MY] = {};             // (of a block at a time where products follow, of all in turn otherwise)
            advance<DP, NB, MY, MEAN, false>(ahead, tile, 0, lane, held, score, acc, [&](int m, int i) {
                const float p = power(now[m][i]);
                if constexpr (kKind == 0) {     // p of p s
                    f32x4& b = back[MEAN ? 0 : m];
                    if (i % 4 == 0) b = *reinterpret_cast<const f32x4*>(&scales[at].inverse[m * kBlock + row_of(i, lane)]);
                    some[i & 1] = fmaf(p, b[i % 4], some[i & 1]);
                } else some[i & 1] += p;
                return p;
            }, [](int, u32x4 (&)[2][NS]) {});
            sum += some[0] + some[1];
            find_top(it + 1, slot);
            continue;
        }
#pragma unroll
        for (int m = 0; m < MY; ++m) {
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = power(score[m][i]);
            f32x4 s4 = {};
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                f32x4 four{p[i], p[i + 1], p[i + 2], p[i + 3]};
                if constexpr (kKind == 0) four *= *reinterpret_cast<const f32x4*>(&scales[at].inverse[(y * MY + m) * kBlock + row_of(i, lane)]);
                s4 += four;
            }
            sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
            if constexpr (MEAN) {
                u32x4 b[2][NS];
                operand_of(p, b);
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int db = 0; db < DP / 32; ++db) {
                        u32x4 f[NS];
                        T::columns(tile, y * MY + m, s, db, lane, f);
                        acc[db] = matmul(f, b[s], acc[db]);
                    }
            }
        }
    }
    if (!live) return;
    sum += __shfl_xor(sum, 32);
    const int64_t place_of = (int64_t)(part * WY + y) * padded + row;
    if (lane < 32) {                                    // a row's slices lie together
        const int64_t stat = row * a.cut.slices() + part * WY + y;
        a.at<float>(a.plan.top)[stat] = ref;
        a.at<float>(a.plan.sum)[stat] = sum;
    }
    if constexpr (MEAN) {
        float* out = a.at<float>(a.plan.mean_parts) + place_of * DP + 4 * (lane >> 5);
        const float back = kKind == 0 ? 0x1p-15f : 1.0f;
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(out + 32 * db + 8 * i) =
                    f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]} * back;
    }
}

// One workgroup per row.  LOSS: the parts joined, the row's slots scored again (sums in 64 bits of the elements themselves), its
// loss.  ROWS: the gradient of its loss, scale * (sum of p w over classes that no slot names + sum of (p - q) w over those), from
// parts that carry their own reference (LOSS as well) or that are normalised already.
// The workgroup is cut into groups of `lanes` lanes that cover four elements each; slots and parts go around them.  Bound by
// the latency of its reads: 4096 rows x 128 with 16 parts 24 us, 8 rows 6.
constexpr int kMostSlices = 4096;
template <bool LOSS, bool ROWS>
__global__ __launch_bounds__(kClassThreads) void class_finish_kernel(ClassArgs a, int64_t padded, int depth, int slices, int lanes) {
    __shared__ float room[kClassWaves], slot_pull[64];
    __shared__ double slot_z[64];
    __shared__ int slot_id[64], alive;
    __shared__ float weight[LOSS && ROWS ? kMostSlices : 1];
    __shared__ __align__(16) f32x4 gathered[ROWS ? kClassThreads : 1];
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float* tops = a.at<const float>(a.plan.top) + t * slices;
    const float* sums = a.at<const float>(a.plan.sum) + t * slices;
    float top = -3e38f, sum = 1.0f;
    if constexpr (LOSS)
#pragma unroll 4
        for (int p = threadIdx.x; p < slices; p += kClassThreads) if (sums[p] != 0.0f) top = fmaxf(top, tops[p]);    // (a reference may be a named class's)
    int id = -1;
    float q = 0.0f, log_weight = 0.0f;                  // of lane's slot, in wave 0
    if (wave == 0) {
        q = slot_weight(a, t, lane, id, log_weight);
        slot_id[lane] = id;
        slot_z[lane] = 0.0f;
        if constexpr (!LOSS) slot_pull[lane] = lane < a.s.K ? a.at<const float>(a.plan.pulls)[t * a.s.K + lane] : 0.0f;
        const bool lives = __any(id >= 0);
        if (lane == 0) alive = lives;
    }
    if constexpr (LOSS) {
        top = wave_max(top);
        if (lane == 0) room[wave] = top;
    }
    __syncthreads();
    if (!alive) {                                       // nothing of the row is used, whatever it holds
        if (LOSS && threadIdx.x == 0) {
            a.loss[t] = 0.0f; a.lse[t] = 0.0f;
            if (!ROWS && a.row_grad) a.at<float>(a.plan.norm)[t] = __builtin_inff();
        }
        if constexpr (ROWS)
            for (int d = threadIdx.x; d < a.s.D; d += kClassThreads) a.row_grad[t * a.s.D + d] = 0.0f;
        return;
    }
    const int groups = kClassThreads / lanes, group = threadIdx.x / lanes, l = threadIdx.x % lanes;
    const Elem* w = static_cast<const Elem*>(a.w);
    if constexpr (LOSS) {
        top = fmaxf(fmaxf(room[0], room[1]), fmaxf(room[2], room[3]));
        __syncthreads();
        sum = 0.0f;
#pragma unroll 4
        for (int p = threadIdx.x; p < slices; p += kClassThreads) {
            const float e = sums[p] != 0.0f ? exp2f(tops[p] - top) : 0.0f;
            sum += sums[p] * e;
            if constexpr (ROWS) weight[p] = e;
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        if (lane == 0) room[wave] = sum;
        const Elem* h = static_cast<const Elem*>(a.h) + t * a.h_stride;
        for (int j = group; j < a.s.K; j += groups) {
            const int id = slot_id[j];
            if (id < 0) continue;
            double dot = id < a.s.V ? 0.0 : __builtin_nan("");       // a class that there is not
            if (id < a.s.V)
                for (int c = 4 * l; c < a.s.D; c += 4 * lanes) {
                    dot += dot4(load4(h, a.s.D, c), load4(w + id * a.w_stride, a.s.D, c));
                }
            for (int d = 1; d < lanes; d *= 2) dot += __shfl_xor(dot, d);
            if (l == 0) slot_z[j] = dot;
        }
        __syncthreads();
        if (wave == 0) {
            sum = (room[0] + room[1]) + (room[2] + room[3]);
            // where gradients are wanted the named classes are not in the sums yet
            const bool apart = ROWS || a.row_grad;
            const double z = slot_z[lane] * a.scale, z2 = z * kLog2eDouble;
            float pull = q;
            const bool named = apart && merge_slots(a, id, pull);
            double most = named && z2 > top ? z2 : (double)top;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) { const double o = __shfl_xor(most, d); most = o > most ? o : most; }
            double own = named ? exp2(z2 - most) : 0.0;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) own += __shfl_xor(own, d);
            const double log2_sum = most + log2(sum * exp2(top - most) + own), lse = log2_sum / kLog2eDouble;
            float loss = id >= 0 && q != 0.0f ? q * (log_weight + (float)(lse - z)) : 0.0f;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) loss += __shfl_xor(loss, d);
            const float rest = (float)exp2(top - log2_sum);     // what the others' sums are relative to, as a share
            if (lane == 0) {
                a.loss[t] = loss; a.lse[t] = (float)lse;
                if constexpr (ROWS) room[0] = rest;
                // where means are made in a launch of their own: what they are relative to
                else if (a.row_grad) { a.at<float>(a.plan.norm)[t] = top - kLift; a.at<float>(a.plan.back)[t] = rest; }
            }
            if (apart) {
                pull = named ? probability(z, lse) - pull : 0.0f;
                if constexpr (ROWS) slot_pull[lane] = pull;
                else if (lane < a.s.K) a.at<float>(a.plan.pulls)[t * a.s.K + lane] = pull;
            }
        }
        if constexpr (ROWS) __syncthreads();
    }
    if constexpr (ROWS) {
        const float* parts = a.at<const float>(a.plan.mean_parts);
        const float back = LOSS ? room[0] : a.at<const float>(a.plan.back)[t];
        for (int c0 = 0; c0 < a.s.D; c0 += 4 * lanes) {
            const int c = c0 + 4 * l;
            f32x4 e = {};
            if (c < a.s.D) {
#pragma unroll 4
                for (int p = group; p < slices; p += groups) {
                    const f32x4 x = *reinterpret_cast<const f32x4*>(parts + (p * padded + t) * depth + c);
                    e += LOSS ? x * weight[p] : x;
                }
                e *= back;
#pragma unroll 4
                for (int j = group; j < a.s.K; j += groups) {
                    const float pull = slot_pull[j];    // 0 of an empty slot
                    if (pull != 0.0f) e += pull * load4(w + slot_id[j] * a.w_stride, a.s.D, c);
                }
            }
            gathered[threadIdx.x] = e;
            __syncthreads();
            if (group == 0 && c < a.s.D) {
                for (int g = 1; g < groups; ++g) e += gathered[g * lanes + l];
                for (int j = 0; j < 4; ++j) if (c + j < a.s.D) a.row_grad[t * a.s.D + c + j] = a.scale * e[j];
            }
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// gradients
// ---------------------------------------------------------------------------------------------------------------
// A wave holds 32 classes, the rows stream by:
//   grad_w[v] = scale * sum_t g_t (p[t,v] - sum over t's slots j that name v of q_j) h[t]
// Scores are made again from the table and the rows, 2 T V D operations, because keeping them would move 6 bytes a score: 12
// times what the classes and their gradients move at 128 elements.  A class's row is written once, by the wave that holds it,
// or in parts that a second launch joins where there are fewer classes than waves.
// 4096 x 2.5 M x 128 bfloat16: 5.46 ms, 0.96 PFLOP/s; what slots add costs by the slot (4096 x 169,343, 32 slots a row: 0.59
// ms, where the classes alone would take 0.37 at that rate).
// P = 2^(score * by + start), P s for fp32 rows: at most 2^15 there, which a row of enormous scores, whose log-sum-exp is rounded,
// would exceed.
template <bool BOUNDED> __device__ __forceinline__ float power_of(float score, float by, float start) {
    const float e = fmaf(score, by, start);
    return __builtin_amdgcn_exp2f(BOUNDED && e > 15.0f ? 15.0f : e);    // (NaN stays)
}
template <int DP, int WY>
__global__ __launch_bounds__(kClassThreads, DP * NS <= 128 && WY < 4 ? 2 : 1) void class_gradient_kernel(ClassArgs a, int64_t padded) {
    constexpr int NB = blocks_per_tile(WY, DP, kKind), MY = NB / WY, WX = kClassWaves / WY;
    using T = Tile<DP, NB * kBlock>;
    __shared__ __align__(16) uint16_t lds[2][NS * T::kPlane];
    __shared__ __align__(16) float starts[2][NB * kBlock], scales[2][kKind == 0 ? NB * kBlock : 1];
    __shared__ float cells[kClassWaves][MY][kBlock * kBlock];
    __shared__ float room[kClassWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, x = wave % WX, y = wave / WX;
    const ClassCut::Place place = a.cut.place(blockIdx.x);
    const int part = place.part, group = place.group, first = place.first, last = place.last;
    const float unit = grad_unit(a, room);
    const int64_t v0 = ((int64_t)group * WX + x) * kBlock, v = v0 + (lane & 31);
    const bool live = v0 < a.s.V;                       // wave-uniform

    u32x4 held[DP / 16][NS];
    const float to_log2 = not_zero(a.scale * kLog2e /
        hold<DP / 16>(static_cast<const Elem*>(a.w) + (v < a.s.V ? v : a.s.V - 1) * a.w_stride, a.s.D, 0, lane, held, both_halves));
    f32x16 acc[DP / 32];
#pragma unroll
    for (auto& f : acc) f = f32x16{};
    float* cell = cells[wave][0];                       // what slots take of a tile's blocks, [row][class]
    for (int i = lane; i < MY * kBlock * kBlock; i += 64) cell[i] = 0.0f;

    const float* start = a.at<const float>(a.plan.start);
    typename T::FromPlanes next;
    float next_start = 0.0f, next_scale = 1.0f;
    SlotFeed<MY> feed(a, padded, v0);
    auto fetch = [&](int it) {
        if (it >= last) return;
        next.load(a.ws + a.plan.rows, 2 * DP, padded * 2 * DP, padded, (int64_t)it * NB * kBlock);   // (padded to whole tiles)
        if (threadIdx.x < NB * kBlock) {
            next_start = start[(int64_t)it * NB * kBlock + threadIdx.x];
            if constexpr (kKind == 0) next_scale = a.at<const float>(a.plan.scales)[(int64_t)it * NB * kBlock + threadIdx.x];
        }
    };
    auto store = [&](int slot) {
        next.store(lds[slot]);
        if (threadIdx.x < NB * kBlock) {
            starts[slot][threadIdx.x] = next_start;
            if constexpr (kKind == 0) scales[slot][threadIdx.x] = next_scale;
        }
    };
    auto product = [&](const uint16_t* tile, int b, const u32x4 (&q)[2][NS]) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int db = 0; db < DP / 32; ++db) {
                u32x4 f[NS];
                T::columns(tile, b, s, db, lane, f);
                acc[db] = matmul(f, q[s], acc[db]);
            }
    };
    // Where rows of block t have negative gradients: their signs into P's operand, whose step s and word j hold registers
    // 8s + 2j and 8s + 2j + 1.
    auto sign = [&](int64_t block, u32x4 (&q)[2][NS]) {
        const uint32_t signs = a.at<const uint32_t>(a.plan.signs)[block];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = row_of(8 * s + 2 * j, lane);
                const uint32_t flip = (signs >> r & 1) << 15 | (signs >> (r + 1)) << 31;
#pragma unroll
                for (int n = 0; n < NS; ++n) q[s][n][j] ^= flip;
            }
    };
    // Places that slots name are left out of the block's own product, whose rounding of p would be far above p - q of a row
    // that has learned its class: p - q of them, made in fp32, is added by a product of its own, for 16-bit types in two
    // roundings (of a row that has not learned its class it is most of what the class gets).
    bool hit[MY];                                       // whether they are in a block of the tile, wave-uniform
    uint32_t named[MY];                                 // registers of a lane whose places are named
    auto gather = [&](int64_t block) {
        feed.turn();
#pragma unroll
        for (int m = 0; m < MY; ++m) {
            hit[m] = feed.gather(m, block + m, lane, cell + m * kBlock * kBlock);
            if (!hit[m]) continue;
            __builtin_amdgcn_wave_barrier();
            named[m] = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) named[m] |= (cell[(m * kBlock + row_of(i, lane)) * kBlock + (lane & 31)] != 0.0f ? 1u : 0u) << i;
        }
    };
    auto pull = [&](const uint16_t* tile, int m) {
        float c[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float& at = cell[(m * kBlock + row_of(i, lane)) * kBlock + (lane & 31)];
            c[i] = -at;
            at = 0.0f;
        }
#pragma unroll 1
        for (int n = 0; n < 2 / NS; ++n) {
            u32x4 q[2][NS];
            operand_of(c, q);
            product(tile, y * MY + m, q);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    c[8 * s + 2 * j] -= low2(q[s][0][j]);
                    c[8 * s + 2 * j + 1] -= high2(q[s][0][j]);
                }
        }
        __builtin_amdgcn_wave_barrier();
    };

    int slot = 0;
    fetch(first);
    if (first < last) {
        feed.ask_words((int64_t)first * NB + y * MY);
        feed.ask_slots((int64_t)first * NB + y * MY, lane);
        feed.ask_words((int64_t)(first + 1) * NB + y * MY);
        if (live) gather((int64_t)first * NB + y * MY);
    }
    for (int it = first; it < last; ++it) {
        const int at = slot;
        const uint16_t* tile = lds[at];
        slot ^= 1;
        store(at);                                      // the other tile may still be read
        __syncthreads();
        fetch(it + 1);
        feed.ask_slots((int64_t)(it + 1) * NB + y * MY, lane);
        feed.ask_words((int64_t)(it + 2) * NB + y * MY);
        if (!live) continue;
        const int64_t block0 = (int64_t)it * NB + y * MY;          // of rows
        f32x16 score[MY];
        f32x4 s = {}, by = {};
        advance<DP, NB, MY, true, true>(tile, tile, y * MY, lane, held, score, acc, [&](int m, int i) {
            const int r = (y * MY + m) * kBlock + row_of(i, lane);
            if (i % 4 == 0) {
                s = *reinterpret_cast<const f32x4*>(&starts[at][r]);
                if constexpr (kKind == 0) by = *reinterpret_cast<const f32x4*>(&scales[at][r]) * to_log2;
            }
            return power_of<kKind == 0>(score[m][i], kKind == 0 ? by[i % 4] : to_log2, s[i % 4]);
        }, [&](int m, u32x4 (&q)[2][NS]) {
            if (feed.now[m].negative()) sign(block0 + m, q);
            if (hit[m]) leave_out(named[m], q);
        });
#pragma unroll
        for (int m = 0; m < MY; ++m)
            if (hit[m]) pull(tile, m);
        if (it + 1 < last) gather(block0 + NB);         // what was asked for has come by now
    }
    if (!live) return;
    const float back = a.scale / unit;
    if (a.cut.slices() > 1) {
        const int64_t rows = ceil_div(a.s.V, kBlock) * kBlock;
        float* out = a.at<float>(a.plan.grad_parts) + ((int64_t)(part * WY + y) * rows + v) * DP + 4 * (lane >> 5);
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(out + 32 * db + 8 * i) =
                    f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]} * back;
        return;
    }
    if (v >= a.s.V) return;
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = 32 * db + 8 * i + 4 * (lane >> 5);
            const f32x4 g = f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]} * back;
            if (d + 4 <= a.s.D) store4(a.grad_w, v * a.s.D + d, g);
            else
                for (int j = 0; j < 4; ++j) if (d + j < a.s.D) store_elem(a.grad_w, v * a.s.D + d + j, g[j]);
        }
}

// ---------------------------------------------------------------------------------------------------------------
// wide rows: the four waves of a workgroup hold a quarter of the elements each
// ---------------------------------------------------------------------------------------------------------------
// A wave's quarter of 32 streamed rows in LDS, its own: no other wave reads it.  Rows of 32 chunks turn as in the narrow
// kernels' tiles; others, of 4 or 12 chunks more than a multiple of 16, lie close but for one chunk more after every four of
// them, which parts the same reads.
template <int Q>
struct Quarter {
    static constexpr int kChunks = Q / 8, kEach = kBlock * kChunks / 64;
    // Lane l fetches and stores chunks l%4 + 4 (i/2) of rows l/4 + 16 (i%2): 64 bytes of a row together, and places that
    // follow from one by constants.
    static __device__ __forceinline__ int row(int i, int lane) { return (lane >> 2) + 16 * (i & 1); }
    static __device__ __forceinline__ int chunk(int i, int lane) { return (lane & 3) + 4 * (i >> 1); }
    static constexpr bool kTurns = kChunks == 32;
    static constexpr int kPlane = kBlock * Q + (kTurns ? 0 : 64);
    static_assert(kTurns || kChunks % 16 == 4 || kChunks % 16 == 12, "rows part on banks");
    static_assert((kBlock * kChunks) % 64 == 0 && kChunks % 4 == 0, "lanes share rows evenly");
    static __device__ __forceinline__ int place(int r, int c) {
        return kTurns ? r * Q + (c ^ turn<Q>(r)) * 8 : r * Q + (r >> 2) * 8 + c * 8;
    }
    static __device__ __forceinline__ void rows(const uint16_t* lds, int ks, int lane, u32x4 (&out)[NS]) {
#pragma unroll
        for (int n = 0; n < NS; ++n)
            out[n] = *reinterpret_cast<const u32x4*>(lds + n * kPlane + place(lane & 31, 2 * ks + (lane >> 5)));
    }
    static __device__ __forceinline__ void columns(const uint16_t* lds, int s, int db, int lane, u32x4 (&out)[NS]) {
        const int i = lane & 15, r = 16 * s + 4 * (lane >> 5) + (i >> 2), c = 4 * db + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const uint16_t* p = lds + n * kPlane + (i & 1) * 4;
            const u32x2 a = read_transposed(p + place(r, c)), z = read_transposed(p + place(r + 8, c));
            out[n] = u32x4{a[0], a[1], z[0], z[1]};
        }
    }
};

// Steps load(k, f), use(k, f) for k = 0 ... N - 1, every load three uses ahead of its own.
template <int N, class Load, class Use> __device__ __forceinline__ void ahead_of(Load load, Use use) {
    constexpr int R = 4;
    u32x4 ring[R][NS];
    each<R - 1>([&](auto k) { if constexpr (k() < N) load(k, ring[k()]); });
    each<N>([&](auto k) {
        if constexpr (k() + R - 1 < N) load(number<k() + R - 1>{}, ring[(k() + R - 1) % R]);
        use(k, ring[k() % R]);
        __builtin_amdgcn_sched_barrier(0);
    });
}

enum WideMode { kStats, kMean, kGradient };

// Rows of more than 256 elements do not fit a wave's registers beside their accumulators.  Split over four waves, each adds
// its quarter of every score; a wave then sums the four partial scores of a quarter of the streamed rows, so that every
// exponential is taken once, and P goes back to all through LDS: 3 KB of LDS traffic a wave for 32 x 32 scores.  The forward is
// two launches, statistics first: a common running maximum would cost the four waves another meeting a tile.
// Bound by the meetings (two barriers a tile) and, for the statistics, by the table's way to the CUs, once for every 32 rows.
// 1024 x 232,965 x 602 fp16: 0.64 + 0.92 + 0.97 ms (0.45, 0.63, 0.59 PFLOP/s); fp32, 257 rows: 0.67 + 0.80 + 1.10 ms, of which
// one workgroup fits a CU, so that its meetings are waited for: 1.35 times the plain products in fp32, the furthest from the floor.
// fp32 rows of more than 640 elements spill up to 77 registers.
// kStats: running maximum and sum of every held row of h, one pair per wave (a quarter of the streamed classes each).
// kMean: sum of the table's rows under 2^(score - norm).  kGradient: as the narrow kernel.
template <int Q, WideMode MODE, bool STRAIGHT>
__global__ __launch_bounds__(kClassThreads, Q * NS <= 192 ? 2 : 1) void class_wide_kernel(ClassArgs a, int64_t padded) {
    using S = Quarter<Q>;
    constexpr int DEPTH = Q * kClassWaves;
    __shared__ __align__(16) uint16_t quarters[kClassWaves][NS * S::kPlane];
    constexpr int MEETS = MODE == kStats && Q * NS < 160 ? 2 : 1;         // one more barrier a tile where two cost a workgroup
    __shared__ __align__(16) f32x4 partial[MEETS][kClassWaves][4][64];
    constexpr int PS = MODE == kStats ? 1 : MODE == kGradient ? 2 : NS;   // planes of P; 16-bit types use the second after a hit
    __shared__ __align__(16) u32x2 shared_p[PS][2][64][2];
    __shared__ int hit;                                 // the tile that last had a slot of these classes
    __shared__ uint32_t places[MODE != kGradient ? kClassWaves : 1][64];
    __shared__ float cells[MODE == kGradient ? kBlock * kBlock : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col0 = wave * Q;
    const ClassCut::Place place = a.cut.place(blockIdx.x);
    const int part = place.part, group = place.group, first = place.first, last = place.last;
    float* room = reinterpret_cast<float*>(partial);
    const float unit = MODE == kGradient ? grad_unit(a, room) : 1.0f;
    const int64_t x0 = (int64_t)group * kBlock, x = x0 + (lane & 31);
    const Elem* w = static_cast<const Elem*>(a.w);
    const uint16_t* planes = a.at<const uint16_t>(a.plan.rows);
    uint16_t* lds = quarters[wave];

    u32x4 held[Q / 16][NS];
    auto join = [&](float peak) {                       // of a row that four waves hold
        peak = both_halves(peak);
        if (lane < kBlock) room[wave * kBlock + lane] = peak;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kClassWaves; ++i) peak = fmaxf(peak, room[i * kBlock + (lane & 31)]);
        __syncthreads();
        return peak;
    };
    const Elem* own = MODE == kGradient ? w + (x < a.s.V ? x : a.s.V - 1) * a.w_stride : held_row(a, x);
    const float to_log2 = not_zero(a.scale * kLog2e / hold<Q / 16>(own, a.s.D, col0, lane, held, join));
    if constexpr (MODE == kGradient) {
        for (int i = threadIdx.x; i < kBlock * kBlock; i += kClassThreads) cells[i] = 0.0f;
        if (threadIdx.x == 0) hit = -1;
        __syncthreads();
    }
    if constexpr (MODE != kGradient) places[wave][lane] = 0;
    using Places = Named<kBlock>;
    typename std::conditional<MODE != kGradient, Places, int>::type named = [&] {
        if constexpr (MODE != kGradient) return Places(a, group, part, first, last, lane);
        else return 0;
    }();
    const float norm = MODE == kMean && x < a.s.T ? a.at<const float>(a.plan.norm)[x] : __builtin_inff();
    float ref = -3e38f, sum = 0.0f;
    f32x16 acc[MODE == kStats ? 1 : Q / 32];
#pragma unroll
    for (auto& f : acc) f = f32x16{};

    // the next tile's quarter: rows of the table as they are, or planes
    constexpr bool FROM_PLANES = MODE == kGradient || STRAIGHT;
    static_assert(kKind != 0 || FROM_PLANES, "fp32 tables are laid out first: a wave has no row whole, to make its unit of");
    struct { Eight e[FROM_PLANES ? 1 : S::kEach]; u32x4 p[FROM_PLANES ? NS : 1][FROM_PLANES ? S::kEach : 1]; } next;
    const bool as_is = MODE != kGradient && !a.plan.packed;
    const uint16_t* streamed = MODE == kGradient ? planes : as_is ? reinterpret_cast<const uint16_t*>(w) : a.at<const uint16_t>(a.plan.table);
    const int64_t plane = (MODE == kGradient ? padded : padded_rows(a.s.V)) * DEPTH;
    const int lane_place = as_is ? S::row(0, lane) * (int)a.w_stride + S::chunk(0, lane) * 8 : lane * 8;
    const int step_row = as_is ? 16 * (int)a.w_stride : 512, step_chunk = as_is ? 32 : 1024;
    SlotFeed<1> feed(a, padded, MODE == kGradient ? x0 : 0);
    f32x4 next_start = {}, next_scale = {};
    const float* scales = kKind == 0 ? a.at<const float>(MODE == kGradient ? a.plan.scales : a.plan.table_scales) : nullptr;
    auto fetch = [&](int it) {
        if constexpr (MODE == kGradient)
            if (wave == 0) {                            // one wave looks after the slots of the workgroup's classes
                feed.ask_slots(it, lane);
                feed.ask_words(it + 1);
            }
        const uint16_t* at = streamed + (as_is ? (int64_t)it * kBlock * a.w_stride + col0 : ((int64_t)it * kClassWaves + wave) * S::kEach * 512);
        const int left = as_is ? (int)(a.s.V - 1 - (int64_t)it * kBlock) : kBlock;       // planes have whole tiles
#pragma unroll
        for (int i = 0; i < S::kEach; ++i) {
            const int c = S::chunk(i, lane);
            const int64_t row = (int64_t)it * kBlock + S::row(i, lane);
            if constexpr (FROM_PLANES) {
                int place = lane_place + (i & 1) * step_row + (i >> 1) * step_chunk;
                if (left < kBlock) {
                    asm volatile("");                   // the last tile of a table as it is: rows behind its last one repeat it
                    const int r = S::row(i, lane);
                    place = (r < left ? r : left) * (int)a.w_stride + c * 8;
                }
#pragma unroll
                for (int n = 0; n < NS; ++n) next.p[n][i] = *reinterpret_cast<const u32x4*>(at + n * plane + place);
            } else next.e[i] = load8(w + (row < a.s.V ? row : a.s.V - 1) * a.w_stride, a.s.D, col0 + c * 8);
        }
        if constexpr (MODE == kGradient)
            next_start = *reinterpret_cast<const f32x4*>(a.at<const float>(a.plan.start) + (int64_t)it * kBlock + 8 * wave + 4 * (lane >> 5));
        if constexpr (kKind == 0) next_scale = *reinterpret_cast<const f32x4*>(scales + (int64_t)it * kBlock + 8 * wave + 4 * (lane >> 5));
    };
    if (first < last) {
        if (MODE == kGradient && wave == 0) feed.ask_words(first);
        fetch(first);
    }
    for (int it = first; it < last; ++it) {
        if (MODE == kGradient && wave == 0) feed.turn();
#pragma unroll
        for (int i = 0; i < S::kEach; ++i) {
            const int r = S::row(i, lane), c = S::chunk(i, lane);
            u32x4 p[NS];
            if constexpr (FROM_PLANES) {
#pragma unroll
                for (int n = 0; n < NS; ++n) p[n] = next.p[n][i];
            } else planes_of(next.e[i], 1.0f, p);
#pragma unroll
            for (int n = 0; n < NS; ++n) *reinterpret_cast<u32x4*>(lds + n * S::kPlane + S::place(r, c)) = p[n];
        }
        const f32x4 start = next_start, scale = next_scale;
        __builtin_amdgcn_wave_barrier();
        if (it + 1 < last) fetch(it + 1);
        f32x16 score = {};
        ahead_of<Q / 16>([&](auto k, u32x4 (&f)[NS]) { S::rows(lds, k(), lane, f); },
                         [&](auto k, const u32x4 (&f)[NS]) { score = matmul(f, held[k()], score); });
        auto& meet = partial[MEETS == 2 ? (it - first) & 1 : 0];
#pragma unroll
        for (int i = 0; i < 4; ++i) meet[wave][i][lane] = f32x4{score[4 * i], score[4 * i + 1], score[4 * i + 2], score[4 * i + 3]};
        const int64_t y0 = (int64_t)it * kBlock;
        if (MODE == kGradient && wave == 0)
            if (feed.gather(0, it, lane, cells) && lane == 0) hit = it;
        __syncthreads();
        f32x4 z = (meet[0][wave][lane] + meet[1][wave][lane]) + (meet[2][wave][lane] + meet[3][wave][lane]);   // rows 8*wave + 4*(lane/32) + j
        const int y = 8 * wave + 4 * (lane >> 5);
        f32x4 back = {1.0f, 1.0f, 1.0f, 1.0f};          // p of p s
        if constexpr (kKind == 0 && MODE != kGradient) {        // to binary logarithms of p s 2^15, as in the narrow kernel
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float s = scale[j];
                z[j] = fmaf(z[j], s * to_log2, log_scale(s));
                back[j] = 0x1p-15f / s;
            }
        }
        if (MODE != kGradient && y0 + kBlock > a.s.V) {
            asm volatile("");
#pragma unroll
            for (int j = 0; j < 4; ++j) if (y0 + y + j >= a.s.V) z[j] = -__builtin_inff();
        }
        if constexpr (MODE != kGradient) {
            if (named.next == (uint32_t)it && a.s.K > kWaveSlots) {
                named.take_many(a, group, it, lane, [&](bool has, int r, int c) {
                    if (has && c >> 3 == wave) atomicOr(&places[wave][r + 32 * (c >> 2 & 1)], 1u << (c & 3));
                });
                __builtin_amdgcn_wave_barrier();
                const uint32_t mine = places[wave][lane];
                places[wave][lane] = 0;
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int j = 0; j < 4; ++j) if (mine >> j & 1) z[j] = -__builtin_inff();
            } else if (named.next == (uint32_t)it)
                named.take(it, lane, [&](uint32_t rows, int c) {
                    const bool mine = c >> 3 == wave && lane >> 5 == (c >> 2 & 1) && rows >> (lane & 31) & 1;
#pragma unroll
                    for (int j = 0; j < 4; ++j) if (mine && j == (c & 3)) z[j] = -__builtin_inff();
                });
        }
        if constexpr (MODE == kStats) {
            if constexpr (kKind != 0) z *= to_log2;
            const float top = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
            if (__any(top > ref + kSlack)) {            // (what the mean's P is relative to)
                const float to = top > ref + kSlack ? top : ref;
                sum *= exp2f(ref - to);
                ref = to;
            }
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = __builtin_amdgcn_exp2f(z[j] - ref) * back[j];
            sum += (e[0] + e[1]) + (e[2] + e[3]);
            if constexpr (MEETS == 1) __syncthreads();
        } else {
            float p[4];
            if constexpr (MODE == kMean) {
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = __builtin_amdgcn_exp2f(kKind == 0 ? z[j] - norm : fmaf(z[j], to_log2, -norm));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) p[j] = power_of<kKind == 0>(z[j], kKind == 0 ? scale[j] * to_log2 : to_log2, start[j]);
                const uint32_t signs = a.at<const uint32_t>(a.plan.signs)[it];
                if (signs) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) if (signs >> (y + j) & 1) p[j] = -p[j];
                }
                if (hit == it) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float& c = cells[(y + j) * kBlock + (lane & 31)];
                        if (c != 0.0f) p[j] = -c;       // p - q of a place that a slot names, as in the narrow kernel
                        c = 0.0f;
                    }
                }
            }
            const uint32_t p0 = pack2(p[0], p[1]), p1 = pack2(p[2], p[3]);
            shared_p[0][wave >> 1][lane][wave & 1] = u32x2{p0, p1};
            const bool rest = MODE == kGradient && NS == 1 && hit == it;        // as in the narrow kernel
            if (NS == 2 || rest)
                shared_p[PS - 1][wave >> 1][lane][wave & 1] =
                    u32x2{pack2(p[0] - low2(p0), p[1] - high2(p0)), pack2(p[2] - low2(p1), p[3] - high2(p1))};
            __syncthreads();
            constexpr int DB = Q / 32;
            u32x4 b[2][NS];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int n = 0; n < NS; ++n) b[s][n] = *reinterpret_cast<const u32x4*>(&shared_p[n][s][lane][0]);
            auto products = [&] {
                ahead_of<2 * DB>([&](auto k, u32x4 (&f)[NS]) { S::columns(lds, k() / DB, k() % DB, lane, f); },
                                 [&](auto k, const u32x4 (&f)[NS]) { acc[k() % DB] = matmul(f, b[k() / DB], acc[k() % DB]); });
            };
            products();
            if (rest) {
#pragma unroll
                for (int s = 0; s < 2; ++s) b[s][0] = *reinterpret_cast<const u32x4*>(&shared_p[PS - 1][s][lane][0]);
                products();
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    if constexpr (MODE == kStats) {                     // both halves of the wave hold a row's classes
        const float other = __shfl_xor(ref, 32), to = fmaxf(ref, other);
        sum = sum * exp2f(ref - to);
        sum += __shfl_xor(sum, 32);
        const int64_t at = x * (a.cut.parts * kClassWaves) + part * kClassWaves + wave;
        if (lane < 32) {
            a.at<float>(a.plan.top)[at] = to;
            a.at<float>(a.plan.sum)[at] = sum;
        }
    } else {
        const float back = MODE == kGradient ? a.scale / unit : exp2f(kKind == 0 ? -kLift - 15.0f : -kLift);
        const int64_t rows = MODE == kGradient ? ceil_div(a.s.V, kBlock) * kBlock : padded;
        const bool joined = MODE == kMean || a.cut.parts > 1;
        float* out = a.at<float>(MODE == kGradient ? a.plan.grad_parts : a.plan.mean_parts);
#pragma unroll
        for (int db = 0; db < Q / 32; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = col0 + 32 * db + 8 * i + 4 * (lane >> 5);
                const f32x4 g = f32x4{acc[db][4 * i], acc[db][4 * i + 1], acc[db][4 * i + 2], acc[db][4 * i + 3]} * back;
                if (joined) *reinterpret_cast<f32x4*>(out + ((int64_t)part * rows + x) * DEPTH + d) = g;
                else if (x < a.s.V) {
                    if (d + 4 <= a.s.D) store4(a.grad_w, x * a.s.D + d, g);
                    else
                        for (int j = 0; j < 4; ++j) if (d + j < a.s.D) store_elem(a.grad_w, x * a.s.D + d + j, g[j]);
                }
            }
    }
}

// Parts of grad_w joined in part order.
__global__ __launch_bounds__(kClassThreads) void class_join_kernel(ClassArgs a, int depth, int slices) {
    const int64_t rows = ceil_div(a.s.V, kBlock) * kBlock, n = a.s.V * a.s.D;
    const float* parts = a.at<const float>(a.plan.grad_parts);
    for (int64_t i = (int64_t)blockIdx.x * kClassThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kClassThreads) {
        const int64_t v = i / a.s.D, d = i % a.s.D;
        float g = 0.0f;
#pragma unroll 8
        for (int p = 0; p < slices; ++p) g += parts[(p * rows + v) * depth + d];
        store_elem(a.grad_w, i, g);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------------------------------------------
template <class F> hipError_t with_depth(int depth, F f) {
    switch (depth) {
        case 64: f(std::integral_constant<int, 64>{}); break;
        case 128: f(std::integral_constant<int, 128>{}); break;
        case 256: f(std::integral_constant<int, 256>{}); break;
        case 384: f(std::integral_constant<int, 384>{}); break;
        case 640: f(std::integral_constant<int, 640>{}); break;
        case 1024: f(std::integral_constant<int, 1024>{}); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

// Lanes that share a row, four elements each.
inline int row_lanes(int64_t D) {
    int lanes = 1;
    while (lanes < 64 && 4 * lanes < D) lanes *= 2;
    return lanes;
}

template <int DP, bool MEAN> void launch_forward(const ClassArgs& a, int64_t padded, hipStream_t stream) {
    const unsigned grid = (unsigned)(a.cut.groups * a.cut.parts);
    const bool straight = a.plan.packed || a.plan.straight;
    if constexpr (!narrow_depth(DP)) {
        if (straight || kKind == 0) class_wide_kernel<DP / kClassWaves, MEAN ? kMean : kStats, true><<<grid, kClassThreads, 0, stream>>>(a, padded);
        else if constexpr (kKind != 0) class_wide_kernel<DP / kClassWaves, MEAN ? kMean : kStats, false><<<grid, kClassThreads, 0, stream>>>(a, padded);
    } else {
        const bool crowded = MEAN && crowded_tiles(a.s);
        auto run = [&](auto wy) {
            if (crowded) class_forward_kernel<DP, wy(), MEAN, false, MEAN><<<grid, kClassThreads, 0, stream>>>(a, padded);
            else if (straight && wy() != 2) class_forward_kernel<DP, wy(), MEAN, wy() != 2><<<grid, kClassThreads, 0, stream>>>(a, padded);
            else class_forward_kernel<DP, wy(), MEAN, false><<<grid, kClassThreads, 0, stream>>>(a, padded);
        };
        if (a.cut.wy == 1) run(number<1>{});
        else if (a.cut.wy == 2) run(number<2>{});
        else if constexpr (DP * NS <= 256) run(number<4>{});
    }
}
template <int DP> void launch_gradient(const ClassArgs& a, int64_t padded, hipStream_t stream) {
    const unsigned grid = (unsigned)(a.cut.groups * a.cut.parts);
    if constexpr (!narrow_depth(DP)) class_wide_kernel<DP / kClassWaves, kGradient, true><<<grid, kClassThreads, 0, stream>>>(a, padded);
    else if (a.cut.wy == 1) class_gradient_kernel<DP, 1><<<grid, kClassThreads, 0, stream>>>(a, padded);
    else if (a.cut.wy == 2) class_gradient_kernel<DP, 2><<<grid, kClassThreads, 0, stream>>>(a, padded);
    else if constexpr (DP * NS <= 256) class_gradient_kernel<DP, 4><<<grid, kClassThreads, 0, stream>>>(a, padded);
}

hipError_t forward(ClassArgs a, hipStream_t stream) {
    const int64_t padded = padded_rows(a.s.T);
    const int depth = class_depth(a.s.D);
    const bool wide = !narrow_depth(depth), rows = a.row_grad != nullptr;
    a.cut = forward_cut(a.s);
    const int slices = (int)a.cut.slices();
    const int lanes = row_lanes(a.s.D);
    auto run = [&](bool mean) {
        return with_depth(depth, [&](auto dp) {
            mean ? launch_forward<dp(), true>(a, padded, stream) : launch_forward<dp(), false>(a, padded, stream);
        });
    };
    if (a.plan.packed) {
        const int64_t table = padded_rows(a.s.V), grid = ceil_div(table * depth / 8, kClassThreads);
        if (hipError_t e = with_depth(depth, [&](auto dp) {
                class_pack_kernel<dp()><<<(unsigned)(grid < 8192 ? grid : 8192), kClassThreads, 0, stream>>>(a, table);
            })) return e;
    }
    if (a.plan.named)
        class_named_kernel<<<(unsigned)(padded / kBlock), kRowThreads, 0, stream>>>(a, wide ? kBlock : blocks_per_tile(a.cut.wy, depth, kKind) * kBlock);
    if (hipError_t e = run(rows && !wide)) return e;
    const unsigned T = (unsigned)a.s.T;
    if (rows && !wide) class_finish_kernel<true, true><<<T, kClassThreads, 0, stream>>>(a, padded, depth, slices, lanes);
    else class_finish_kernel<true, false><<<T, kClassThreads, 0, stream>>>(a, padded, depth, wide ? slices * kClassWaves : slices, lanes);
    if (!rows || !wide) return hipGetLastError();
    if (hipError_t e = run(true)) return e;
    class_finish_kernel<false, true><<<T, kClassThreads, 0, stream>>>(a, padded, depth, slices, lanes);
    return hipGetLastError();
}

hipError_t gradient(ClassArgs a, hipStream_t stream) {
    const int64_t padded = padded_rows(a.s.T);
    const int depth = class_depth(a.s.D);
    if (!a.grad_w) {
        if (a.grad_h && a.s.T) class_row_grad_kernel<<<(unsigned)ceil_div(a.s.T, kClassWaves), kClassThreads, 0, stream>>>(a);
        return hipGetLastError();
    }
    a.cut = gradient_cut(a.s);
    a.buckets = buckets_of(a.s.V, a.s.K);
    if constexpr (kHalf) class_peaks_kernel<<<kPeaks, kClassThreads, 0, stream>>>(a);
    if (a.plan.row_slots && a.s.T) {
        const int lanes = row_lanes(a.s.D);
        class_slots_kernel<<<(unsigned)a.s.T, 64 * (unsigned)ceil_div(a.s.K, 4 * (64 / lanes)), 0, stream>>>(a, lanes);
    }
    if (hipError_t e = with_depth(depth, [&](auto dp) {
            if (padded) class_rows_kernel<dp()><<<padded / kBlock, kRowThreads, 0, stream>>>(a, padded);
        })) return e;
    if (hipError_t e = with_depth(depth, [&](auto dp) { launch_gradient<dp()>(a, padded, stream); })) return e;
    if (a.cut.slices() > 1) {
        const int64_t n = ceil_div(a.s.V * a.s.D, kClassThreads);
        class_join_kernel<<<(unsigned)(n < 4096 ? n : 4096), kClassThreads, 0, stream>>>(a, depth, (int)a.cut.slices());
    }
    return hipGetLastError();
}

}  // namespace
#endif

}  // namespace fsa
