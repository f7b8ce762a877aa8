// Launchers of the training operators of residual blocks: 8-bit activation checkpoints (block_rows.hip, block_gate.hip) and the
// weight gradient taken from them (block_wgrad.hip). All pointers are device memory; every call only enqueues on `st`.
// The callers (block_api.hip) have checked types, sizes and pointers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/iodf.h"

namespace iodf {

constexpr int kCodeGroup = 32;          // columns that share an exponent
constexpr int kJoinMaxCols = 16384;     // widest row of a join: two vectors of eight columns to each of 1024 threads

inline int code_pitch(int cols) { return (cols + kCodeGroup - 1) / kCodeGroup * kCodeGroup; }

hipError_t launch_pack(const void* x, int type, long long stride, long long rows, int cols, const uint8_t* live, int8_t* q,
                       uint8_t* e, hipStream_t st);
hipError_t launch_unpack(const int8_t* q, const uint8_t* e, long long rows, int cols, void* y, int type, long long stride,
                         hipStream_t st);

hipError_t launch_join_forward(const iodf_join& a, hipStream_t st);
// `work` holds join_workspace(a) bytes.
hipError_t launch_join_backward(const iodf_join& a, void* work, hipStream_t st);
size_t join_workspace(long long rows, int cols, long long gate_rows);

hipError_t launch_glu_forward(const iodf_glu& a, hipStream_t st);
hipError_t launch_glu_backward(const iodf_glu& a, hipStream_t st);

hipError_t launch_weight_grad(const iodf_wgrad& a, void* work, hipStream_t st);
size_t wgrad_workspace(const iodf_wgrad& a);

// The code of a HIP error, kept for iodf_last_hip_error; IODF_OK for hipSuccess.
int report_hip(hipError_t e);

}  // namespace iodf
