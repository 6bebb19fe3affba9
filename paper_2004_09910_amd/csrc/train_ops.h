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

// A gated block, checked: bytes of a call's workspace, and the calls.
struct Gated {
  tgp_gated_shape s;
  long rows;
  tgp_gated_weights w;
};
size_t gated_bytes(const tgp_gated_shape& s, long rows, bool backward);
hipError_t gated_forward(const Gated& g, const void* x, long ldx, void* y, long ldy, void* ws,
                         hipStream_t st);
hipError_t gated_backward(const Gated& g, const void* dy, long lddy, const void* x, long ldx,
                          void* dx, long lddx, const tgp_gated_grads& grads, bool overwrite,
                          void* ws, hipStream_t st);

// The norms around a residual block: tensors and their row distances.
struct Rows {
  void* p;
  long ld;
};
struct ResidualForward {
  tgp_residual_shape s;
  tgp_residual_params w;
  Rows r, f, gate, out, z;
  float* stats;
};
struct ResidualBackward {
  tgp_residual_shape s;
  tgp_residual_params w;
  Rows dz, dout, out, f, gate;
  const float* stats;
  Rows dr, df, dgate;
  tgp_residual_grads g;
  bool overwrite;
  float* part;   // partial column sums
};
constexpr int kResidualMaxC = 32768;
hipError_t residual_norm_forward(const ResidualForward& a, hipStream_t st);
size_t residual_norm_partial_floats(const tgp_residual_shape& s);
hipError_t residual_norm_backward(const ResidualBackward& a, hipStream_t st);

// Workspace bytes of the matrices t[0 .. n), and the update of all of them.
size_t muon_bytes(int n, const tgp_muon_tensor* t);
hipError_t muon_update(int n, const tgp_muon_tensor* t, float mu, bool nesterov, int steps,
                       float eps, void* ws, hipStream_t st);

hipError_t weight_step(int n, const tgp_step_tensor* t, float decay, hipStream_t st);
// c1, c2: the bias corrections 1 / (1 - beta^step).
hipError_t adamw_step(int n, const tgp_adamw_tensor* t, float rate, float beta1, float beta2,
                      float eps, float decay, float c1, float c2, hipStream_t st);

// rc2: sqrt(1 / (1 - beta2^step)).
hipError_t adamw8_step(int n, const tgp_adamw8_tensor* t, float rate, double beta1, double beta2,
                       float eps, float decay, float c1, float rc2, uint64_t seed, hipStream_t st);

}  // namespace tgpk
