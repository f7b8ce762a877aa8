// C entry points of the training operators: checks of the arguments, then the launches (block_*.hip).
#include "../../include/iodf.h"

#include "block.h"

using namespace iodf;

namespace {

// what a launch can count (less than 2^32 threads): the backward pass of a join has at least one workgroup for each shared gate
constexpr int64_t kMaxRows = 1ll << 30, kMaxElems = 1ll << 34, kMaxGates = 1ll << 21;
constexpr int kMaxCols = 65536;

bool a_type(int t) { return t == IODF_T_F32 || t == IODF_T_BF16 || t == IODF_T_F16; }
bool a_shape(int64_t rows, int cols, int most) { return rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= most && rows * code_pitch(cols) <= kMaxElems; }
// a pointer to elements of `type`, strided; code rows are read and written 16 bytes at a time
bool a_tensor(const void* p, int type, int64_t stride, int cols) {
    return p && ((uintptr_t)p & (type == IODF_T_F32 ? 3 : 1)) == 0 && stride >= cols && stride <= (1ll << 40);
}
bool a_code(const int8_t* q, const uint8_t* e) { return q && e && ((uintptr_t)q & 15) == 0; }
bool floats(const void* p) { return ((uintptr_t)p & 3) == 0; }

int check_join(const iodf_join* a) {
    if (!a || !a_shape(a->rows, a->cols, kJoinMaxCols) || !a_type(a->block_type) || !(a->eps > 0.f) || !(a->eps < 3e38f)) return IODF_E_ARG;
    if (a->stream_type != a->block_type && a->stream_type != IODF_T_F32) return IODF_E_ARG;
    if (a->gate && a->gate_rows < 1 && a->rows) return IODF_E_ARG;
    if (!floats(a->alpha) || !floats(a->gate) || !floats(a->w_post) || !floats(a->w_pre)) return IODF_E_ARG;
    return IODF_OK;
}

int check_glu(const iodf_glu* a) {
    if (!a || !a_shape(a->rows, a->cols, kMaxCols) || !a_type(a->type)) return IODF_E_ARG;
    return a->act == IODF_ACT_RELU || a->act == IODF_ACT_SILU || a->act == IODF_ACT_GELU ? IODF_OK : IODF_E_ARG;
}

int check_wgrad(const iodf_wgrad* a) {
    if (!a || !a_shape(a->rows, a->cols, kMaxCols) || !a_shape(a->rows, a->out, kMaxCols) || !a_type(a->dy_type)) return IODF_E_ARG;
    return IODF_OK;
}

}  // namespace

extern "C" {

int iodf_pack(const void* x, int x_type, int64_t x_stride, int64_t rows, int cols, const uint8_t* live, int8_t* q, uint8_t* e,
              void* stream) {
    if (!a_type(x_type) || !a_shape(rows, cols, kMaxCols)) return IODF_E_ARG;
    if (rows == 0) return IODF_OK;
    if (!a_tensor(x, x_type, x_stride, cols) || !a_code(q, e)) return IODF_E_ARG;
    return report_hip(launch_pack(x, x_type, x_stride, rows, cols, live, q, e, (hipStream_t)stream));
}

int iodf_unpack(const int8_t* q, const uint8_t* e, int64_t rows, int cols, void* y, int y_type, int64_t y_stride, void* stream) {
    if ((y_type != IODF_T_F32 && y_type != IODF_T_BF16) || !a_shape(rows, cols, kMaxCols)) return IODF_E_ARG;
    if (rows == 0) return IODF_OK;
    if (!a_tensor(y, y_type, y_stride, cols) || !a_code(q, e)) return IODF_E_ARG;
    return report_hip(launch_unpack(q, e, rows, cols, y, y_type, y_stride, (hipStream_t)stream));
}

int iodf_join_forward(const iodf_join* a, void* stream) {
    const int rc = check_join(a);
    if (rc != IODF_OK || a->rows == 0) return rc;
    const int ts = a->stream_type, tb = a->block_type;
    if (!a_tensor(a->in_stream, ts, a->in_stream_stride, a->cols) || !a_tensor(a->out_stream, ts, a->out_stream_stride, a->cols) ||
        !a_tensor(a->in_block, tb, a->in_block_stride, a->cols) || (a->w_pre && !a_tensor(a->out_block, tb, a->out_block_stride, a->cols)))
        return IODF_E_ARG;
    if (a->in_stream == a->out_stream && a->in_stream_stride != a->out_stream_stride) return IODF_E_ARG;
    iodf_join run = *a;
    if (a->nq) {  // a checkpoint: whole or not at all
        if (!a_code(a->nq, a->ne) || (a->w_post && !a->inv_post) || (a->w_pre && (!a_code(a->xq, a->xe) || !a->inv_pre))) return IODF_E_ARG;
        if (!floats(a->inv_pre) || !floats(a->inv_post)) return IODF_E_ARG;
        if (!a->w_pre) run.xq = nullptr, run.inv_pre = nullptr;
    } else if (a->xq) {
        return IODF_E_ARG;
    } else {
        run.inv_pre = run.inv_post = nullptr;
    }
    return report_hip(launch_join_forward(run, (hipStream_t)stream));
}

int iodf_join_workspace(const iodf_join* a, int64_t* bytes) {
    const int rc = check_join(a);
    if (rc != IODF_OK) return rc;
    if (!bytes || (a->gate && a->gate_rows > 1 && (a->rows - 1) / a->gate_rows >= kMaxGates)) return IODF_E_ARG;
    *bytes = (int64_t)join_workspace(a->rows, a->cols, a->gate ? a->gate_rows : a->rows);
    return IODF_OK;
}

int iodf_join_backward(const iodf_join* a, void* work, int64_t work_bytes, void* stream) {
    int64_t need = 0;
    const int rc = iodf_join_workspace(a, &need);
    if (rc != IODF_OK) return rc;
    if (!work || ((uintptr_t)work & 15) || work_bytes < need) return IODF_E_ARG;
    if (!a->alpha != !a->dalpha || !a->gate != !a->dgate || !a->w_post != !a->dw_post || !a->w_pre != !a->dw_pre) return IODF_E_ARG;
    if (!floats(a->dalpha) || !floats(a->dgate) || !floats(a->dw_post) || !floats(a->dw_pre)) return IODF_E_ARG;
    if (a->rows) {
        const int ts = a->stream_type, tb = a->block_type;
        if (!a_tensor(a->in_stream, ts, a->in_stream_stride, a->cols) || !a_tensor(a->out_stream, ts, a->out_stream_stride, a->cols) ||
            !a_tensor(a->out_block, tb, a->out_block_stride, a->cols) || !a_code(a->nq, a->ne) || (a->w_post && !a->inv_post))
            return IODF_E_ARG;
        if (a->w_pre && (!a_tensor(a->in_block, tb, a->in_block_stride, a->cols) || !a_code(a->xq, a->xe) || !a->inv_pre)) return IODF_E_ARG;
        if (!floats(a->inv_pre) || !floats(a->inv_post)) return IODF_E_ARG;
    }
    return report_hip(launch_join_backward(*a, work, (hipStream_t)stream));
}

int iodf_glu_forward(const iodf_glu* a, void* stream) {
    const int rc = check_glu(a);
    if (rc != IODF_OK || a->rows == 0) return rc;
    if (!a_tensor(a->a, a->type, a->a_stride, a->cols) || !a_tensor(a->b, a->type, a->b_stride, a->cols) ||
        !a_tensor(a->y, a->type, a->y_stride, a->cols))
        return IODF_E_ARG;
    if ((a->aq || a->bq) && (!a_code(a->aq, a->ae) || !a_code(a->bq, a->be))) return IODF_E_ARG;
    return report_hip(launch_glu_forward(*a, (hipStream_t)stream));
}

int iodf_glu_backward(const iodf_glu* a, void* stream) {
    const int rc = check_glu(a);
    if (rc != IODF_OK || a->rows == 0) return rc;
    if (!a_tensor(a->dy, a->type, a->dy_stride, a->cols) || !a_tensor(a->da, a->type, a->da_stride, a->cols) ||
        !a_tensor(a->db, a->type, a->db_stride, a->cols) || !a_code(a->aq, a->ae) || !a_code(a->bq, a->be) || (a->yq && !a_code(a->yq, a->ye)))
        return IODF_E_ARG;
    return report_hip(launch_glu_backward(*a, (hipStream_t)stream));
}

int iodf_weight_grad_workspace(const iodf_wgrad* a, int64_t* bytes) {
    const int rc = check_wgrad(a);
    if (rc != IODF_OK) return rc;
    if (!bytes) return IODF_E_ARG;
    *bytes = (int64_t)wgrad_workspace(*a);
    return IODF_OK;
}

int iodf_weight_grad(const iodf_wgrad* a, void* work, int64_t work_bytes, void* stream) {
    int64_t need = 0;
    const int rc = iodf_weight_grad_workspace(a, &need);
    if (rc != IODF_OK) return rc;
    if (need && (!work || ((uintptr_t)work & 15) || work_bytes < need)) return IODF_E_ARG;
    if (!a_tensor(a->dw, IODF_T_F32, a->dw_stride, a->cols) || !floats(a->col_scale)) return IODF_E_ARG;
    if (a->rows && (!a_tensor(a->dy, a->dy_type, a->dy_stride, a->out) || !a_code(a->q, a->e))) return IODF_E_ARG;
    return report_hip(launch_weight_grad(*a, work, (hipStream_t)stream));
}

}  // extern "C"
