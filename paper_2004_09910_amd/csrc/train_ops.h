// Internal launcher interface of the operators around a stage's tasks: layer
// normalisation, orthogonalised updates, weight steps.  As in kernels.h,
// every launcher enqueues on `st` and returns the launch status, and dt is
// the storage type (0 = bfloat16, 1 = float32).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tgp.h"

namespace tgpk {

// One layer norm: rows x C, consecutive rows of each tensor ld* elements apart.
struct NormShape {
  long rows;
  int C;
};
hipError_t layer_norm_forward(int dt, const NormShape& s, const void* x, long ldx,
                              const float* gain, const float* bias, float eps, void* y, long ldy,
                              float* stats, hipStream_t st);
// Floats of the partial column sums that the backward may leave in `part`.
size_t layer_norm_partial_floats(int dt, const NormShape& s);
hipError_t layer_norm_backward(int dt, const NormShape& s, const void* dy, long lddy,
                               const void* x, long ldx, const float* gain, const float* stats,
                               void* dx, long lddx, float* dgain, float* dbias, bool overwrite,
                               float* part, hipStream_t st);

// Workspace bytes of the matrices t[0 .. n), and the update of all of them.
size_t muon_bytes(int n, const tgp_muon_tensor* t);
hipError_t muon_update(int n, const tgp_muon_tensor* t, float mu, bool nesterov, int steps,
                       float eps, void* ws, hipStream_t st);

hipError_t weight_step(int n, const tgp_step_tensor* t, float decay, hipStream_t st);
// c1, c2: the bias corrections 1 / (1 - beta^step).
hipError_t adamw_step(int n, const tgp_adamw_tensor* t, float rate, float beta1, float beta2,
                      float eps, float decay, float c1, float c2, hipStream_t st);

}  // namespace tgpk
