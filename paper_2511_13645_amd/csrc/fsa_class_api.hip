// The C ABI of the class losses declared in include/fsa.h: host-side validation, workspace sizes, dispatch by type.
// Nothing here allocates, synchronises or keeps anything.
#include "../../include/fsa.h"
#include "fsa_class_kernels.hip.h"

#include <cmath>

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool known(int dtype) { return dtype == FSA_F32 || dtype == FSA_BF16 || dtype == FSA_F16; }
int elem_bytes(int dtype) { return dtype == FSA_F32 ? 4 : 2; }
bool sizes_ok(int64_t T, int64_t V, int64_t D, int32_t K) {
    return T >= 0 && T <= FSA_CLASS_TMAX && V >= 1 && V <= FSA_CLASS_VMAX && D >= 1 && D <= FSA_CLASS_DMAX && K >= 1 &&
           K <= FSA_KMAX;
}
constexpr int64_t kMostStride = 1 << 24;             // a block of 32 rows stays within 32-bit byte offsets

bool positive(float x) { return std::isfinite(x) && x > 0.0f; }

// What every entry point takes, checked; `a` is filled in but for outputs and workspace.
int take(fsa::ClassArgs& a, const void* h, int64_t h_stride, const void* w, int64_t w_stride, int dtype, int64_t T, int64_t V,
         int64_t D, float scale, float temperature, const int32_t* ids, const void* teacher, int teacher_dtype, int32_t K) {
    if (!w || (T > 0 && (!h || !ids))) return FSA_ERR_NULL;
    if (!known(dtype) || !known(teacher_dtype)) return FSA_ERR_DTYPE;
    if (!sizes_ok(T, V, D, K) || h_stride < D || w_stride < D || h_stride > kMostStride || w_stride > kMostStride)
        return FSA_ERR_ARG;
    if (!positive(scale) || !positive(temperature) || !positive(scale / temperature) || !positive(1.0f / temperature)) return FSA_ERR_ARG;
    if (!aligned(h, elem_bytes(dtype)) || !aligned(w, elem_bytes(dtype)) || !aligned(ids, 4) ||
        !aligned(teacher, elem_bytes(teacher_dtype)))
        return FSA_ERR_ALIGN;
    a.s = {T, V, D, dtype, K};
    a.h = h; a.h_stride = h_stride; a.w = w; a.w_stride = w_stride;
    a.scale = scale / temperature; a.inv_temperature = 1.0f / temperature;
    a.ids = ids; a.teacher = teacher; a.teacher_kind = teacher_dtype;
    return FSA_OK;
}

// Rows of a whole depth that all start on the 16-byte grid are read as they are.
bool straight(const fsa::ClassArgs& a) {
    return a.s.kind != FSA_F32 && a.s.D == fsa::class_depth(a.s.D) && aligned(a.w, 16) && a.w_stride % 8 == 0;
}

int take_room(fsa::ClassArgs& a, void* workspace, int64_t bytes) {
    if (bytes < 0) return FSA_ERR_ARG;
    if ((size_t)bytes < a.plan.bytes || !workspace) return FSA_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return FSA_ERR_ALIGN;
    a.ws = static_cast<char*>(workspace);
    return FSA_OK;
}

int status_of(hipError_t e) { return e == hipSuccess ? FSA_OK : FSA_ERR_HIP; }

hipError_t forward_of(const fsa::ClassArgs& a, hipStream_t st) {
    return a.s.kind == FSA_F32 ? fsa::class_forward_f32(a, st) : a.s.kind == FSA_BF16 ? fsa::class_forward_bf16(a, st)
                                                                                     : fsa::class_forward_f16(a, st);
}
hipError_t gradient_of(const fsa::ClassArgs& a, hipStream_t st) {
    return a.s.kind == FSA_F32 ? fsa::class_gradient_f32(a, st) : a.s.kind == FSA_BF16 ? fsa::class_gradient_bf16(a, st)
                                                                                      : fsa::class_gradient_f16(a, st);
}

int forward(fsa::ClassArgs& a, float* loss, float* lse, float* row_grad, void* workspace, int64_t bytes, void* stream) {
    if (a.s.T > 0 && (!loss || !lse)) return FSA_ERR_NULL;
    if (!aligned(loss, 4) || !aligned(lse, 4) || !aligned(row_grad, 4)) return FSA_ERR_ALIGN;
    if (a.s.T == 0) return FSA_OK;
    a.plan = fsa::plan_of(a.s, straight(a), true, row_grad != nullptr, false);
    if (int rc = take_room(a, workspace, bytes)) return rc;
    a.loss = loss; a.lse = lse; a.row_grad = row_grad;
    (void)hipGetLastError();                            // an error that the caller left pending is not this call's
    return status_of(forward_of(a, static_cast<hipStream_t>(stream)));
}

int backward(fsa::ClassArgs& a, const float* grad_loss, const float* lse, const float* row_grad, void* grad_h, void* grad_w,
             void* workspace, int64_t bytes, void* stream) {
    if (a.s.T > 0 && (!grad_loss || !lse)) return FSA_ERR_NULL;
    const int eb = elem_bytes(a.s.kind);
    if (!aligned(grad_loss, 4) || !aligned(lse, 4) || !aligned(row_grad, 4) || !aligned(grad_h, eb) || !aligned(grad_w, eb))
        return FSA_ERR_ALIGN;
    const bool again = grad_h && !row_grad && a.s.T > 0;
    a.plan = fsa::plan_of(a.s, straight(a), again, again, grad_w != nullptr);
    if (int rc = take_room(a, workspace, bytes)) return rc;
    (void)hipGetLastError();
    hipStream_t st = static_cast<hipStream_t>(stream);
    a.grad_loss = grad_loss; a.lse_in = lse; a.row_grad_in = row_grad; a.grad_h = grad_h; a.grad_w = grad_w;
    if (again) {                                        // losses and log-sum-exps of this run are not wanted
        fsa::ClassArgs f = a;
        f.row_grad = a.at<float>(a.plan.row_grad);
        f.loss = a.at<float>(a.plan.loss); f.lse = f.loss + fsa::padded_rows(a.s.T);
        a.row_grad_in = f.row_grad;
        if (hipError_t e = forward_of(f, st)) return status_of(e);
    }
    return status_of(gradient_of(a, st));
}

// The sizes alone do not say where the table lies: room for a table off the grid.
int64_t room_for(const fsa::ClassShape& s, bool forward, bool with_row_grad, bool with_grad_w) {
    return (int64_t)fsa::plan_of(s, false, forward, with_row_grad, with_grad_w).bytes;
}

}  // namespace

extern "C" {

int64_t fsa_class_fwd_workspace_bytes(int64_t T, int64_t V, int64_t D, int dtype, int32_t K, int with_row_grad) {
    if (!known(dtype) || !sizes_ok(T, V, D, K)) return 0;
    return room_for({T, V, D, dtype, K}, true, with_row_grad != 0, false);
}

int64_t fsa_class_bwd_workspace_bytes(int64_t T, int64_t V, int64_t D, int dtype, int32_t K, int with_row_grad, int with_grad_w) {
    if (!known(dtype) || !sizes_ok(T, V, D, K)) return 0;
    return room_for({T, V, D, dtype, K}, with_row_grad != 0, with_row_grad != 0, with_grad_w != 0);
}

int fsa_xent_fwd(const void* h, int64_t h_stride, const void* w, int64_t w_stride, int dtype,
                 int64_t T, int64_t V, int64_t D, float scale, const int32_t* targets,
                 float* out_loss, float* out_lse, float* out_row_grad,
                 void* workspace, int64_t workspace_bytes, void* stream) {
    fsa::ClassArgs a{};
    if (int rc = take(a, h, h_stride, w, w_stride, dtype, T, V, D, scale, 1.0f, targets, nullptr, FSA_F32, 1)) return rc;
    return forward(a, out_loss, out_lse, out_row_grad, workspace, workspace_bytes, stream);
}

int fsa_xent_bwd(const float* grad_loss, const void* h, int64_t h_stride, const void* w, int64_t w_stride, int dtype,
                 int64_t T, int64_t V, int64_t D, float scale, const int32_t* targets,
                 const float* lse, const float* row_grad, void* grad_h, void* grad_w,
                 void* workspace, int64_t workspace_bytes, void* stream) {
    fsa::ClassArgs a{};
    if (int rc = take(a, h, h_stride, w, w_stride, dtype, T, V, D, scale, 1.0f, targets, nullptr, FSA_F32, 1)) return rc;
    return backward(a, grad_loss, lse, row_grad, grad_h, grad_w, workspace, workspace_bytes, stream);
}

int fsa_distill_fwd(const void* h, int64_t h_stride, const void* w, int64_t w_stride, int dtype,
                    int64_t T, int64_t V, int64_t D, float scale, float temperature,
                    const int32_t* teacher_ids, const void* teacher_logits, int teacher_dtype, int32_t K,
                    float* out_loss, float* out_lse, float* out_row_grad,
                    void* workspace, int64_t workspace_bytes, void* stream) {
    fsa::ClassArgs a{};
    if (T > 0 && !teacher_logits) return FSA_ERR_NULL;
    if (int rc = take(a, h, h_stride, w, w_stride, dtype, T, V, D, scale, temperature, teacher_ids, teacher_logits, teacher_dtype, K))
        return rc;
    return forward(a, out_loss, out_lse, out_row_grad, workspace, workspace_bytes, stream);
}

int fsa_distill_bwd(const float* grad_loss, const void* h, int64_t h_stride, const void* w, int64_t w_stride, int dtype,
                    int64_t T, int64_t V, int64_t D, float scale, float temperature,
                    const int32_t* teacher_ids, const void* teacher_logits, int teacher_dtype, int32_t K,
                    const float* lse, const float* row_grad, void* grad_h, void* grad_w,
                    void* workspace, int64_t workspace_bytes, void* stream) {
    fsa::ClassArgs a{};
    if (T > 0 && !teacher_logits) return FSA_ERR_NULL;
    if (int rc = take(a, h, h_stride, w, w_stride, dtype, T, V, D, scale, temperature, teacher_ids, teacher_logits, teacher_dtype, K))
        return rc;
    return backward(a, grad_loss, lse, row_grad, grad_h, grad_w, workspace, workspace_bytes, stream);
}

}  // extern "C"
