// Launch interface of the expert feed-forward block and its gradient (expert_ffn.hip,
// expert_ffn_f32.hip).  Not part of the public ABI.
#pragma once

#include "checkpoint.h"
#include "groups.h"

namespace trimmoe {

struct ExpertFfnArgs {
  bool bf16, gated;
  int keep;  // TRIMMOE_KEEP_*
  int d, F;
  Groups groups;
  const void *w_up, *w_gate, *w_down;
  const void* x;        // [n, d]
  // kept pre-activations: written by the forward, read by the backward
  void *up, *gate;      // [n, F], values or codes
  uint8_t *up_scale, *gate_scale;
  void* y;              // [n, d], forward
  // backward
  const uint8_t* x_scale;  // x holds codes, or NULL
  const void* dy;
  void *dx, *dw_up, *dw_gate, *dw_down;  // each may be NULL
  char* ws;
  int n_cu;
};

size_t expert_ffn_ws(bool bf16, bool gated, int keep, int E, int d, int F, int n);
size_t expert_ffn_backward_ws(bool bf16, bool gated, bool x_packed, int E, int d, int F, int n);
hipError_t launch_expert_ffn(const ExpertFfnArgs& a, hipStream_t st);
hipError_t launch_expert_ffn_backward(const ExpertFfnArgs& a, hipStream_t st);

// The arrays of the workspace.  `elem`: bytes of a value
inline size_t ffn_align(size_t x) { return (x + 255) & ~(size_t)255; }
inline size_t ffn_array(int n, int cols, int elem) { return ffn_align((size_t)n * cols * elem); }

// the fp32 side; bytes of the sums of K's pieces of n rows times M columns over K
size_t row_parts_f32(const Groups& g, int M, long K);
hipError_t launch_expert_ffn_f32(const ExpertFfnArgs& a, hipStream_t st);
hipError_t launch_expert_ffn_backward_f32(const ExpertFfnArgs& a, hipStream_t st);

}  // namespace trimmoe
