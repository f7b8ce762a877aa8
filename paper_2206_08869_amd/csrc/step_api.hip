// C entry points of the two ends of a training step: checks of the arguments, then the launches (loss.hip, orth.hip).
#include "../../include/iodf.h"

#include "block.h"
#include "step.h"

using namespace iodf;

namespace {

bool a_type(int t) { return t == IODF_T_F32 || t == IODF_T_BF16 || t == IODF_T_F16; }
int size_of(int t) { return t == IODF_T_F32 ? 4 : 2; }
bool a_tensor(const void* p, int type, int64_t stride, int cols) {
    return p && ((uintptr_t)p & (size_of(type) - 1)) == 0 && stride >= cols && stride <= (1ll << 40);
}
bool words(const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

int check_loss(const iodf_class_loss* a) {
    if (!a || !a_type(a->type) || a->rows < 0 || a->rows > (1 << 24) || a->classes < 1 || a->classes > (1 << 20) || a->cols < 1 || a->cols > 65536)
        return IODF_E_ARG;
    if (a->rows * a->cols > (1ll << 34) || (int64_t)a->classes * a->cols > (1ll << 34) || a->rows * a->classes > (1ll << 38)) return IODF_E_ARG;
    return IODF_OK;
}

// What both directions read, and the workspace.
int check_loss_call(const iodf_class_loss* a, int backward, const void* work, int64_t work_bytes) {
    int64_t need = 0;
    const int rc = iodf_class_loss_workspace(a, backward, &need);
    if (rc != IODF_OK) return rc;
    if (need && (!work || !words(work, 16) || work_bytes < need)) return IODF_E_ARG;
    if (a->rows == 0) return IODF_OK;
    if (!a_tensor(a->u, a->type, a->u_stride, a->cols) || !a_tensor(a->w, a->type, a->w_stride, a->cols) || !a->target || !words(a->target, 8))
        return IODF_E_ARG;
    return a->lse && words(a->lse, 4) ? IODF_OK : IODF_E_ARG;
}

// Polynomials, sizes and types that orthogonalising takes.
bool check_orth_sizes(int64_t count, int rows, int cols, float eps) {
    if (rows < 1 || cols < 1 || rows > 65536 || cols > 65536 || (rows < cols ? rows : cols) > 16384) return false;
    const int64_t padded = ((int64_t)rows + 63) / 64 * 64 * (((int64_t)cols + 63) / 64 * 64);
    return count >= 0 && count * padded <= (1ll << 32) && eps > 0.f && eps < 3e38f;
}

}  // namespace

extern "C" {

int iodf_class_loss_workspace(const iodf_class_loss* a, int backward, int64_t* bytes) {
    const int rc = check_loss(a);
    if (rc != IODF_OK) return rc;
    if (!bytes) return IODF_E_ARG;
    *bytes = a->rows ? (int64_t)class_loss_workspace(*a, backward != 0) : 0;
    return IODF_OK;
}

int iodf_class_loss_forward(const iodf_class_loss* a, void* work, int64_t work_bytes, void* stream) {
    const int rc = check_loss_call(a, 0, work, work_bytes);
    if (rc != IODF_OK || a->rows == 0) return rc;
    if (!a->loss || !words(a->loss, 4)) return IODF_E_ARG;
    return report_hip(launch_class_loss(*a, work, (hipStream_t)stream));
}

int iodf_class_loss_backward(const iodf_class_loss* a, void* work, int64_t work_bytes, void* stream) {
    const int rc = check_loss_call(a, 1, work, work_bytes);
    if (rc != IODF_OK) return rc;
    if (!words(a->dloss, 4) || !words(a->dlse, 4)) return IODF_E_ARG;
    if ((a->du && a->rows && !a_tensor(a->du, a->type, a->du_stride, a->cols)) || (a->dw && !a_tensor(a->dw, a->type, a->dw_stride, a->cols)))
        return IODF_E_ARG;
    if (!a->dw && (!a->du || a->rows == 0)) return IODF_OK;
    return report_hip(launch_class_loss_backward(*a, work, (hipStream_t)stream));
}

int iodf_orthogonalise_workspace(const iodf_orth* a, int64_t* bytes) {
    if (!a || !bytes || !a_type(a->in_type) || !a_type(a->out_type) || a->count > 4096 || !check_orth_sizes(a->count, a->rows, a->cols, a->eps))
        return IODF_E_ARG;
    *bytes = a->count ? (int64_t)orth_workspace(*a) : 0;
    return IODF_OK;
}

int iodf_orthogonalise(const iodf_orth* a, void* work, int64_t work_bytes, void* stream) {
    int64_t need = 0;
    OrthSteps s;
    const int rc = iodf_orthogonalise_workspace(a, &need);
    if (rc != IODF_OK) return rc;
    if (!orth_steps(a->steps, a->coefficients, s)) return IODF_E_ARG;
    if (a->count == 0) return IODF_OK;
    if (!work || !words(work, 16) || work_bytes < need) return IODF_E_ARG;
    if (!a_tensor(a->in, a->in_type, a->in_stride, a->cols) || !a_tensor(a->out, a->out_type, a->out_stride, a->cols)) return IODF_E_ARG;
    if (a->count > 1) {
        if (a->in_batch < 1 || a->out_batch < 1 || a->in_batch > (1ll << 40) || a->out_batch > (1ll << 40)) return IODF_E_ARG;
        // one behind the other, or side by side between the rows of the first
        if (a->out_batch < (a->rows - 1) * a->out_stride + a->cols && (a->out_batch < a->cols || (a->count - 1) * a->out_batch + a->cols > a->out_stride))
            return IODF_E_ARG;
    }
    iodf_orth run = *a;
    if (a->count == 1) run.in_batch = run.out_batch = 1;  // one matrix: they are multiplied with 0
    return report_hip(launch_orthogonalise(run, s, work, (hipStream_t)stream));
}

int iodf_muon_workspace(const iodf_muon* a, int64_t* bytes) {
    if (!a || !bytes || !a_type(a->weight_type) || !a_type(a->grad_type) || a->count < 0 || a->count > kMaxUpdates || !check_orth_sizes(1, a->rows, a->cols, a->eps))
        return IODF_E_ARG;
    *bytes = a->count ? (int64_t)muon_workspace(*a) : 0;
    return IODF_OK;
}

int iodf_muon_step(const iodf_muon* a, void* work, int64_t work_bytes, void* stream) {
    int64_t need = 0;
    OrthSteps s;
    const int rc = iodf_muon_workspace(a, &need);
    if (rc != IODF_OK) return rc;
    if (!orth_steps(a->steps, a->coefficients, s)) return IODF_E_ARG;
    const float numbers[4] = {a->rate, a->beta, a->decay, a->scale};
    for (float v : numbers)
        if (!(v > -3e38f && v < 3e38f)) return IODF_E_ARG;
    if (a->count == 0) return IODF_OK;
    if (!work || !words(work, 16) || work_bytes < need || !a->weights || !a->grads || !a->momenta) return IODF_E_ARG;
    for (int64_t k = 0; k < a->count; ++k)
        if (!a_tensor(a->weights[k], a->weight_type, a->weight_stride, a->cols) || !a_tensor(a->grads[k], a->grad_type, a->grad_stride, a->cols) ||
            !a->momenta[k] || !words(a->momenta[k], 4))
            return IODF_E_ARG;
    return report_hip(launch_muon_step(*a, s, work, (hipStream_t)stream));
}

}  // extern "C"
