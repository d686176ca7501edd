// The C ABI of the residual norm, the gated feed-forward block and the orthogonalised update declared in include/fsa.h: host-side
// validation, workspace sizes, dispatch by type.  Nothing here allocates, synchronises or keeps anything.
#include "../../include/fsa.h"
#include "fsa_block_kernels.h"

#include <cmath>

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool known(int dtype) { return dtype == FSA_F32 || dtype == FSA_BF16 || dtype == FSA_F16; }
int elem_bytes(int dtype) { return dtype == FSA_F32 ? 4 : 2; }
bool not_negative(float x) { return std::isfinite(x) && x >= 0.0f; }
bool in(int64_t n, int64_t low, int64_t high) { return n >= low && n <= high; }
constexpr int64_t kMostStride = (int64_t)1 << 31;
int status_of(hipError_t e) { return e == hipSuccess ? FSA_OK : FSA_ERR_HIP; }

int take_room(void* workspace, int64_t bytes, size_t need) {
    if (bytes < 0) return FSA_ERR_ARG;
    if (need == 0) return FSA_OK;
    if ((size_t)bytes < need || !workspace) return FSA_ERR_WORKSPACE;
    return aligned(workspace, 16) ? FSA_OK : FSA_ERR_ALIGN;
}

// ---------------------------------------------------------------------------------------------------------------
// norm
// ---------------------------------------------------------------------------------------------------------------
bool norm_sizes(int64_t T, int64_t D) { return in(T, 0, FSA_NORM_TMAX) && in(D, 1, FSA_NORM_DMAX); }
static_assert(FSA_NORM_DMAX == fsa::kNormDmax && FSA_ORTHO_STEPS == fsa::kMostSteps, "");

size_t norm_room(int64_t T, int64_t D, int dtype) { return (size_t)(fsa::norm_parts(T, D, elem_bytes(dtype)) * D) * 4; }

// ---------------------------------------------------------------------------------------------------------------
// gated feed-forward
// ---------------------------------------------------------------------------------------------------------------
bool gated_sizes(int64_t T, int64_t D, int64_t H, int64_t O) {
    return in(T, 0, FSA_GATED_TMAX) && in(D, 1, FSA_GATED_MOST) && in(H, 1, FSA_GATED_MOST) && in(O, 1, FSA_GATED_MOST);
}
// Whether a product can read a matrix in place: what starts on the 16-byte grid and ends on a multiple of 8 elements, and of which a
// tile's rows lie within 31 bits of bytes.
bool in_place(const fsa::Matrix& m, int dtype) {
    return dtype != FSA_F32 && aligned(m.p, 16) && m.stride % 8 == 0 && m.cols % 8 == 0 && m.stride <= (1 << 21);
}
constexpr int kAllPacked = 31;
int type_of(int dtype) { return dtype & ~FSA_GATED_FINE; }
fsa::GatedShape gated_shape(int64_t T, int64_t D, int64_t H, int64_t O, int dtype) {
    return {T, D, H, O, type_of(dtype), (dtype & FSA_GATED_FINE) != 0};
}
bool gated_known(int64_t T, int64_t D, int64_t H, int64_t O, int dtype) { return known(type_of(dtype)) && gated_sizes(T, D, H, O); }

int gated_take(fsa::GatedArgs& a, const void* x, int64_t x_stride, const void* gate, int64_t gate_stride, const void* up, int64_t up_stride,
               const void* down, int64_t down_stride, int dtype, int activation, int64_t T, int64_t D, int64_t H, int64_t O) {
    if (!gate || !up || !down || (T > 0 && !x)) return FSA_ERR_NULL;
    if (!known(type_of(dtype))) return FSA_ERR_DTYPE;
    if (!gated_sizes(T, D, H, O) || !in(activation, FSA_ACT_SILU, FSA_ACT_RELU)) return FSA_ERR_ARG;
    if (!in(x_stride, D, kMostStride) || !in(gate_stride, D, kMostStride) || !in(up_stride, D, kMostStride) || !in(down_stride, H, kMostStride))
        return FSA_ERR_ARG;
    const int eb = elem_bytes(type_of(dtype));
    if (!aligned(x, eb) || !aligned(gate, eb) || !aligned(up, eb) || !aligned(down, eb)) return FSA_ERR_ALIGN;
    a.s = gated_shape(T, D, H, O, dtype);
    a.activation = activation;
    a.x = {x, x_stride, T, D};
    a.gate = {gate, gate_stride, H, D};
    a.up = {up, up_stride, H, D};
    a.down = {down, down_stride, O, H};
    return FSA_OK;
}
int packs_of(const fsa::GatedArgs& a, bool backward) {
    const fsa::Matrix* m[5] = {&a.x, &a.gate, &a.up, &a.down, &a.grad_y};
    int packs = 0;
    for (int i = 0; i < (backward ? 5 : 4); ++i) packs |= in_place(*m[i], a.s.kind) ? 0 : 1 << i;
    if ((packs & 6) != 0 || a.gate.stride != a.up.stride) packs |= 6;       // both tables lie alike
    return packs;
}

}  // namespace

extern "C" {

int fsa_norm_fwd(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                 const void* weight, int dtype, int weight_dtype, int64_t T, int64_t D, float eps,
                 void* out_y, void* out_s, void* stream) {
    if (!weight || (T > 0 && (!x || !out_y || (residual && !out_s)))) return FSA_ERR_NULL;
    if (!known(dtype) || !known(weight_dtype)) return FSA_ERR_DTYPE;
    if (!norm_sizes(T, D) || !not_negative(eps) || !in(x_stride, D, kMostStride) || (!residual && out_s)) return FSA_ERR_ARG;
    if (residual && !in(residual_stride, D, kMostStride)) return FSA_ERR_ARG;
    const int eb = elem_bytes(dtype);
    if (!aligned(x, eb) || !aligned(residual, eb) || !aligned(out_y, eb) || !aligned(out_s, eb) || !aligned(weight, elem_bytes(weight_dtype)))
        return FSA_ERR_ALIGN;
    if (T == 0) return FSA_OK;
    fsa::NormArgs a{};
    a.x = x; a.x_stride = x_stride; a.residual = residual; a.residual_stride = residual_stride; a.weight = weight;
    a.kind = dtype; a.weight_kind = weight_dtype; a.T = T; a.D = D; a.eps = eps;
    a.y = out_y; a.s = out_s;
    (void)hipGetLastError();                            // an error that the caller left pending is not this call's
    return status_of(fsa::norm_forward(a, static_cast<hipStream_t>(stream)));
}

int64_t fsa_norm_bwd_workspace_bytes(int64_t T, int64_t D, int dtype) {
    return known(dtype) && norm_sizes(T, D) ? (int64_t)norm_room(T, D, dtype) : 0;
}

int fsa_norm_bwd(const void* grad_y, const void* grad_s, const void* s, int64_t s_stride,
                 const void* weight, int dtype, int weight_dtype, int64_t T, int64_t D, float eps,
                 void* grad_x, void* grad_weight, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!weight || (T > 0 && !s)) return FSA_ERR_NULL;
    if (!known(dtype) || !known(weight_dtype)) return FSA_ERR_DTYPE;
    if (!norm_sizes(T, D) || !not_negative(eps) || !in(s_stride, D, kMostStride)) return FSA_ERR_ARG;
    const int eb = elem_bytes(dtype), wb = elem_bytes(weight_dtype);
    if (!aligned(grad_y, eb) || !aligned(grad_s, eb) || !aligned(s, eb) || !aligned(grad_x, eb) || !aligned(weight, wb) || !aligned(grad_weight, wb))
        return FSA_ERR_ALIGN;
    if (int rc = take_room(workspace, workspace_bytes, grad_weight ? norm_room(T, D, dtype) : 0)) return rc;
    if ((T == 0 || !grad_x) && !grad_weight) return FSA_OK;
    fsa::NormArgs a{};
    a.x = s; a.x_stride = s_stride; a.weight = weight; a.grad_y = grad_y; a.grad_s = grad_s;
    a.kind = dtype; a.weight_kind = weight_dtype; a.T = T; a.D = D; a.eps = eps;
    a.y = grad_x; a.grad_weight = grad_weight; a.parts = static_cast<float*>(workspace);
    (void)hipGetLastError();
    return status_of(fsa::norm_backward(a, static_cast<hipStream_t>(stream)));
}

// The sizes alone do not say where operands lie: room to lay all of them out.
int64_t fsa_gated_fwd_workspace_bytes(int64_t T, int64_t D, int64_t H, int64_t O, int dtype) {
    if (!gated_known(T, D, H, O, dtype)) return 0;
    return (int64_t)fsa::gated_plan(gated_shape(T, D, H, O, dtype), false, false, kAllPacked).bytes;
}
int64_t fsa_gated_bwd_workspace_bytes(int64_t T, int64_t D, int64_t H, int64_t O, int dtype) {
    if (!gated_known(T, D, H, O, dtype)) return 0;
    return (int64_t)fsa::gated_plan(gated_shape(T, D, H, O, dtype), true, false, kAllPacked).bytes;
}

int fsa_gated_keep_pays(int64_t T, int64_t D, int64_t H, int64_t O, int dtype) {
    return gated_known(T, D, H, O, dtype) && fsa::gated_keep_pays(gated_shape(T, D, H, O, dtype)) ? 1 : 0;
}

int64_t fsa_gated_kept_bytes(int64_t T, int64_t D, int64_t H, int64_t O, int dtype) {
    return gated_known(T, D, H, O, dtype) ? (int64_t)fsa::kept_plan(gated_shape(T, D, H, O, dtype)).bytes : 0;
}

int fsa_gated_fwd(const void* x, int64_t x_stride, const void* w_gate, int64_t gate_stride, const void* w_up, int64_t up_stride,
                  const void* w_down, int64_t down_stride, int dtype, int activation, int64_t T, int64_t D, int64_t H, int64_t O,
                  void* out_y, void* out_kept, void* workspace, int64_t workspace_bytes, void* stream) {
    fsa::GatedArgs a{};
    if (T > 0 && !out_y) return FSA_ERR_NULL;
    if (int rc = gated_take(a, x, x_stride, w_gate, gate_stride, w_up, up_stride, w_down, down_stride, dtype, activation, T, D, H, O)) return rc;
    if (!aligned(out_y, elem_bytes(a.s.kind)) || !aligned(out_kept, 16)) return FSA_ERR_ALIGN;
    if (T == 0) return FSA_OK;
    a.packs = packs_of(a, false);
    a.plan = fsa::gated_plan(a.s, false, false, a.packs);
    if (int rc = take_room(workspace, workspace_bytes, a.plan.bytes)) return rc;
    a.y = out_y; a.kept = static_cast<char*>(out_kept); a.ws = static_cast<char*>(workspace);
    (void)hipGetLastError();
    hipStream_t st = static_cast<hipStream_t>(stream);
    return status_of(a.s.kind == FSA_F32 ? fsa::gated_forward_f32(a, st) : a.s.kind == FSA_BF16 ? fsa::gated_forward_bf16(a, st)
                                                                                               : fsa::gated_forward_f16(a, st));
}

int fsa_gated_bwd(const void* grad_y, int64_t grad_y_stride, const void* x, int64_t x_stride,
                  const void* w_gate, int64_t gate_stride, const void* w_up, int64_t up_stride, const void* w_down, int64_t down_stride,
                  int dtype, int activation, int64_t T, int64_t D, int64_t H, int64_t O, const void* kept,
                  void* grad_x, void* grad_gate, void* grad_up, void* grad_down,
                  void* workspace, int64_t workspace_bytes, void* stream) {
    fsa::GatedArgs a{};
    if (T > 0 && !grad_y) return FSA_ERR_NULL;
    if (int rc = gated_take(a, x, x_stride, w_gate, gate_stride, w_up, up_stride, w_down, down_stride, dtype, activation, T, D, H, O)) return rc;
    if (!in(grad_y_stride, O, kMostStride)) return FSA_ERR_ARG;
    const int eb = elem_bytes(a.s.kind);
    if (!aligned(grad_y, eb) || !aligned(grad_x, eb) || !aligned(grad_gate, eb) || !aligned(grad_up, eb) || !aligned(grad_down, eb) ||
        !aligned(kept, 16))
        return FSA_ERR_ALIGN;
    a.grad_y = {grad_y, grad_y_stride, T, O};
    a.kept = static_cast<char*>(const_cast<void*>(kept));                     // (read)
    a.grad_x = grad_x; a.grad_gate = grad_gate; a.grad_up = grad_up; a.grad_down = grad_down;
    if (T > 0) {
        a.packs = packs_of(a, true);
        a.plan = fsa::gated_plan(a.s, true, kept != nullptr, a.packs);
        if (int rc = take_room(workspace, workspace_bytes, a.plan.bytes)) return rc;
        a.ws = static_cast<char*>(workspace);
    }
    (void)hipGetLastError();
    hipStream_t st = static_cast<hipStream_t>(stream);
    return status_of(a.s.kind == FSA_F32 ? fsa::gated_backward_f32(a, st) : a.s.kind == FSA_BF16 ? fsa::gated_backward_bf16(a, st)
                                                                                                : fsa::gated_backward_f16(a, st));
}

int64_t fsa_orthogonalize_workspace_bytes(int64_t B, int64_t M, int64_t N, int dtype) {
    if (!known(dtype) || !in(B, 0, FSA_ORTHO_BMAX) || !in(M, 1, FSA_ORTHO_MOST) || !in(N, 1, FSA_ORTHO_MOST)) return 0;
    return (int64_t)fsa::ortho_plan({B, M, N, dtype}).bytes;
}

int fsa_orthogonalize(const void* g, int64_t batch_stride, int64_t stride, int dtype, int64_t B, int64_t M, int64_t N,
                      const float* coefficients, int32_t steps, float eps, float scale,
                      void* out, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!coefficients || (B > 0 && (!g || !out))) return FSA_ERR_NULL;
    if (!known(dtype)) return FSA_ERR_DTYPE;
    if (!in(B, 0, FSA_ORTHO_BMAX) || !in(M, 1, FSA_ORTHO_MOST) || !in(N, 1, FSA_ORTHO_MOST) || !in(steps, 1, FSA_ORTHO_STEPS) ||
        !not_negative(eps) || !std::isfinite(scale) || !in(stride, N, kMostStride) || (B > 1 && batch_stride < 0))
        return FSA_ERR_ARG;
    fsa::OrthoArgs a{};
    for (int i = 0; i < 3 * steps; ++i) a.coefficients[i] = coefficients[i];
    if (!fsa::ortho_units(a.coefficients, steps, FSA_ORTHO_COEFFICIENT, a.units)) return FSA_ERR_ARG;
    if (!aligned(g, elem_bytes(dtype)) || !aligned(out, elem_bytes(dtype))) return FSA_ERR_ALIGN;
    if (B == 0) return FSA_OK;
    a.s = {B, M, N, dtype};
    a.plan = fsa::ortho_plan(a.s);
    if (int rc = take_room(workspace, workspace_bytes, a.plan.bytes)) return rc;
    a.g = g; a.batch_stride = batch_stride; a.stride = stride; a.steps = steps; a.eps = eps; a.scale = scale;
    a.out = out; a.ws = static_cast<char*>(workspace);
    (void)hipGetLastError();
    return status_of(fsa::orthogonalize(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
