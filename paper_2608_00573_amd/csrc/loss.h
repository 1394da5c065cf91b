// Launch interface of the training losses (head_loss.hip, balance.hip).
// Not part of the public ABI.
#pragma once

#include "common.h"

namespace trimmoe {

// ------------------------------------------ cross entropy of a vocabulary head --
struct HeadLossArgs {
  bool bf16;
  int V, d, T;
  const void* w;          // [V, d]
  const float* b;         // [V] or NULL
  const void* h;          // [T, d]
  const int32_t* target;  // [T]
  // forward
  float* loss;  // [T]
  float* lse;   // [T] (backward: read)
  // backward
  const float* dloss;  // [T]
  void* dh;            // [T, d] or NULL
  void* dw;            // [V, d] or NULL
  float* db;           // [V] or NULL
  char* ws;
  int n_cu;
};

// softmax pairs (max z log2 e, sum exp(z - max z)) of a bf16 head per row and
// vocabulary tile, NaN logits kept (gemm.hip)
hipError_t launch_head_loss_partials(const void* W, const float* bias, const void* H, int n_rows,
                                     int V, int K, int n_vtiles, float2* partials, int n_cu,
                                     hipStream_t st);

size_t head_loss_ws(bool bf16, int V, int d, int T);
size_t head_loss_backward_ws(bool bf16, int V, int d, int T);
hipError_t launch_head_loss(const HeadLossArgs& a, hipStream_t st);
hipError_t launch_head_loss_backward(const HeadLossArgs& a, hipStream_t st);

// ------------------------------------------------------ balance of a router --
struct BalanceArgs {
  bool bf16;
  int E, k, d, T;
  const void* w;          // [E, d]
  const float* b;         // [E] or NULL
  const void* h;          // [T, d]
  const int16_t* target;  // [T, k]
  float* prob;            // [T, E] (backward: read)
  int32_t* counts;        // [E + 1] (backward: read)
  // forward
  float* prob_sum;  // [E]
  float* loss;      // [1]
  // backward
  const float* dloss;  // [1]
  void* dh;            // [T, d] or NULL
  void* dw;            // [E, d] or NULL
  float* db;           // [E] or NULL
  char* ws;
};

size_t balance_ws(bool bf16, int E, int d, int T);
size_t balance_backward_ws(bool bf16, int E, int d, int T);
hipError_t launch_balance(const BalanceArgs& a, hipStream_t st);
hipError_t launch_balance_backward(const BalanceArgs& a, hipStream_t st);

}  // namespace trimmoe
