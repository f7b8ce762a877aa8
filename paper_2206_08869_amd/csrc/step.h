// Launchers of the two ends of a training step: the loss over a table of classes (loss.hip) and orthogonalised updates (orth.hip). All pointers
// are device memory; every call only enqueues on `st`. The callers (step_api.hip) have checked types, sizes and pointers.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/iodf.h"

namespace iodf {

constexpr int kMaxUpdates = IODF_MUON_MOST;

hipError_t launch_class_loss(const iodf_class_loss& a, void* work, hipStream_t st);
hipError_t launch_class_loss_backward(const iodf_class_loss& a, void* work, hipStream_t st);
size_t class_loss_workspace(const iodf_class_loss& a, bool backward);

// What the products of an orthogonalising need of its polynomials: how large numbers get, checked by the caller.
struct OrthSteps {
    int n;
    float a[IODF_ORTH_MOST], b[IODF_ORTH_MOST], c[IODF_ORTH_MOST];
    int x_exp[IODF_ORTH_MOST + 1], a_exp[IODF_ORTH_MOST], b_exp[IODF_ORTH_MOST];  // powers of two that 16-bit numbers are held times
};
// false: the polynomials let numbers grow past what 16 bits hold
bool orth_steps(int steps, const float* coefficients, OrthSteps& s);

hipError_t launch_orthogonalise(const iodf_orth& a, const OrthSteps& s, void* work, hipStream_t st);
size_t orth_workspace(const iodf_orth& a);
hipError_t launch_muon_step(const iodf_muon& a, const OrthSteps& s, void* work, hipStream_t st);
size_t muon_workspace(const iodf_muon& a);

}  // namespace iodf
