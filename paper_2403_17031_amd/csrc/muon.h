// Launchers of muon.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rlhf {

// One matrix [rows, cols], contiguous.  Either src (float, or bfloat16 with src_bf16) is orthogonalised into out (bfloat16), or
// (src null) an optimizer step runs: grad and moment give the matrix, param and param_bf16 (may be null) take the update.
struct MuonMatrix {
  const void* src;
  uint16_t* out;
  float* param;
  const float* grad;
  float* moment;
  uint16_t* param_bf16;
  int rows, cols;
};
struct MuonScalars {
  int src_bf16, nesterov, steps;
  float beta, omb, grad_scale;  // moment = beta moment + omb grad_scale grad
  float decay;                  // param = decay param - lr rms sqrt(max(rows, cols)) O
  double lr_rms, eps;
};
constexpr int kMuonGroup = 48;  // most matrices of a call
// Workspace bytes of a call on matrices of these sizes.
size_t muon_workspace_bytes(const MuonMatrix* ms, int count);
hipError_t launch_muon(const MuonMatrix* ms, int count, const MuonScalars& c, void* workspace, hipStream_t s);

}  // namespace rlhf
