// Arguments and launchers of the training-side operators (token
// log-probabilities, losses, AdamW, factored moments, norms,
// embedding, Muon).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "bergson.h"

namespace bergson {

constexpr int kStateBlock = BERGSON_STATE_BLOCK;   // elements per scale of an 8-bit state

struct LogprobArgs {
  const void* x;              // [rows, ld] logits
  int dtype;
  int64_t rows, V, ld;
  const int64_t* targets;
  double tau;
  float* logp;                // [rows] each; entropy or nullptr
  float* lse;
  float* entropy;
  int* status;
};
cudaError_t launch_token_logprobs(const LogprobArgs& a, cudaStream_t s);

struct LogprobGradArgs {
  const void* x;
  int dtype;
  int64_t rows, V, ld;
  const int64_t* targets;
  double tau;
  const float* lse;
  const float* entropy;       // with d_entropy
  const float* d_logp;        // nullptr: 0
  const float* d_entropy;     // nullptr: 0
  void* dx;                   // [rows, ld_d]
  int64_t ld_d;
  int* status;
};
cudaError_t launch_token_logprobs_backward(const LogprobGradArgs& a, cudaStream_t s);

size_t policy_workspace(int64_t B, int64_t T);
cudaError_t launch_policy_loss(const bergson_policy_args& a, void* ws, cudaStream_t s);
cudaError_t launch_preference_loss(const bergson_preference_args& a, cudaStream_t s);

struct AdamwScalars {
  double lr, beta1, beta2, eps;
  int64_t step;
  uint64_t seed;
  const float* grad_scale;    // device, or nullptr
};
cudaError_t launch_adamw(const bergson_adamw_tensor* t, int n, const AdamwScalars& a,
                         cudaStream_t s);
cudaError_t launch_state_values(const uint8_t* codes, const float* scale, int64_t n, int moment,
                                float* out, cudaStream_t s);

size_t moments_workspace(const bergson_moment_matrix* m, int n);
cudaError_t launch_factor_moments(const bergson_moment_matrix* m, int n, double correction,
                                  double floor, void* ws, cudaStream_t s);

cudaError_t launch_norm(const bergson_norm_args& a, cudaStream_t s);
size_t norm_backward_workspace(int64_t rows, int64_t d);
cudaError_t launch_norm_backward(const bergson_norm_grad_args& a, void* ws, cudaStream_t s);

cudaError_t launch_embedding(const bergson_embedding_args& a, int* status, cudaStream_t s);
size_t embedding_backward_workspace(int64_t rows, int64_t V, int64_t d);
cudaError_t launch_embedding_backward(const bergson_embedding_grad_args& a, void* ws, int* status,
                                      cudaStream_t s);

struct MuonScalars {
  double lr, beta;
  bool nesterov;
  const double* coefficients;  // [iterations, 3]
  int iterations;
  int products;                // 1 or 3
  const float* grad_scale;     // device, or nullptr
};
// Whether a matrix's counter holds its products' tiles, at their widest.
bool muon_counts(int64_t rows, int64_t cols, int products, int iterations);
size_t muon_workspace(const bergson_muon_tensor* t, int n, int products);
cudaError_t launch_muon(const bergson_muon_tensor* t, int n, const MuonScalars& a, void* ws,
                        int* status, int sms, cudaStream_t s);

}  // namespace bergson
