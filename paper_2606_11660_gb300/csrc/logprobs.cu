// Token log-probabilities of logits and their backward pass.
//
//   z = x / tau,  lse = log sum_v exp(z_v),  logp = z_t - lse,
//   H = -sum_v p_v log p_v = log s - w / s  with  m = max z,
//   s = sum exp(z_v - m),  w = sum exp(z_v - m) (z_v - m),
//   dx_v = (d_logp ([v = t] - p_v) - d_H p_v (log p_v + H)) / tau.
//
// The forward pass goes over a row once, with the running maximum and the two
// sums rescaled when the maximum grows.

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 256;
constexpr float kInf = __builtin_huge_valf();
constexpr float kNoRow = -1e30f;               // a row's lse below this: it has no entries

struct RowSums {
  float m = -kInf, s = 0.0f, w = 0.0f;
};

// w about a maximum that is larger by -d, f = exp(d).  Where f is 0 nothing is left,
// also where s d would pass the range (or the side is empty, d = -inf).
__device__ __forceinline__ float shifted(float w, float s, float f, float d) {
  return f > 0.0f ? f * (w + s * d) : 0.0f;
}

__device__ __forceinline__ void merge(RowSums& a, const RowSums& b) {
  const float m = fmaxf(a.m, b.m);
  const float da = a.m == m ? 0.0f : a.m - m, db = b.m == m ? 0.0f : b.m - m;
  const float fa = expf(da), fb = expf(db);
  a.w = shifted(a.w, a.s, fa, da) + shifted(b.w, b.s, fb, db);
  a.s = a.s * fa + b.s * fb;
  a.m = m;
}

__device__ __forceinline__ RowSums shuffle(const RowSums& a, int o) {
  RowSums r;
  r.m = __shfl_xor_sync(0xffffffffu, a.m, o);
  r.s = __shfl_xor_sync(0xffffffffu, a.s, o);
  r.w = __shfl_xor_sync(0xffffffffu, a.w, o);
  return r;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(
    const T* __restrict__ x, int64_t V, int64_t ld, const int64_t* __restrict__ targets,
    float inv_tau, float* __restrict__ logp, float* __restrict__ lse,
    float* __restrict__ entropy, int* status) {
  __shared__ RowSums red[kThreads / 32];
  const int64_t r = blockIdx.x;
  const int64_t t = targets[r];
  if (t < 0) {
    if (threadIdx.x == 0) {
      logp[r] = 0.0f;
      lse[r] = 0.0f;
      if (entropy != nullptr) entropy[r] = 0.0f;
    }
    return;
  }
  const T* row = x + r * ld;
  RowSums a;
  for (int64_t v = threadIdx.x; v < V; v += kThreads) {
    const float z = to_f32(row[v]) * inv_tau;
    if (z == -kInf) continue;
    if (z > a.m) {
      const float d = a.m - z, f = expf(d);
      a.w = shifted(a.w, a.s, f, d);
      a.s *= f;
      a.m = z;
    }
    const float d = z - a.m, e = expf(d);
    a.s += e;
    a.w += e > 0.0f ? e * d : e;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) merge(a, shuffle(a, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kThreads / 32; ++i) merge(a, red[i]);
    const float nan = __int_as_float(0x7fffffff);
    const bool none = a.m == -kInf && a.s == 0.0f;
    const bool bad = !(a.m < kInf) || a.s != a.s;
    const float ls = logf(a.s);
    lse[r] = none ? -kInf : bad ? nan : a.m + ls;
    if (entropy != nullptr) entropy[r] = none ? 0.0f : bad ? nan : ls - a.w / a.s;
    if (t >= V && status != nullptr) atomicCAS(status, 0, BERGSON_EINVAL);
    logp[r] = none && t < V ? -kInf
              : bad || t >= V ? nan : (to_f32(row[t]) * inv_tau - a.m) - ls;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprobs_backward_kernel(
    const T* x, int64_t V, int64_t ld, const int64_t* __restrict__ targets, float inv_tau,
    const float* __restrict__ lse, const float* __restrict__ entropy,
    const float* __restrict__ d_logp, const float* __restrict__ d_entropy, T* dx, int64_t ld_d,
    int* status) {
  const int64_t r = blockIdx.x;
  const int64_t t = targets[r];
  const T* row = x + r * ld;
  T* out = dx + r * ld_d;
  const float w = d_logp != nullptr ? d_logp[r] : 0.0f;
  const float h = d_entropy != nullptr ? d_entropy[r] : 0.0f;
  const float l = lse[r];
  if (t >= V) {
    if (threadIdx.x == 0 && status != nullptr) atomicCAS(status, 0, BERGSON_EINVAL);
    for (int64_t v = threadIdx.x; v < V; v += kThreads)
      out[v] = from_f32<T>(__int_as_float(0x7fffffff));
    return;
  }
  if (t < 0 || (w == 0.0f && h == 0.0f) || l < kNoRow) {
    for (int64_t v = threadIdx.x; v < V; v += kThreads) out[v] = from_f32<T>(0.0f);
    return;
  }
  const float ent = d_entropy != nullptr ? entropy[r] : 0.0f;
  for (int64_t v = threadIdx.x; v < V; v += kThreads) {
    const float q = to_f32(row[v]) * inv_tau - l;
    const float p = expf(q);
    float d = -w * p;
    if (p > 0.0f) d -= h * p * (q + ent);
    if (v == t) d += w;
    out[v] = from_f32<T>(d * inv_tau);
  }
}

template <typename T>
cudaError_t run_forward(const LogprobArgs& a, cudaStream_t s) {
  logprobs_kernel<T><<<static_cast<unsigned>(a.rows), kThreads, 0, s>>>(
      static_cast<const T*>(a.x), a.V, a.ld, a.targets, static_cast<float>(1.0 / a.tau), a.logp,
      a.lse, a.entropy, a.status);
  return cudaGetLastError();
}

template <typename T>
cudaError_t run_backward(const LogprobGradArgs& a, cudaStream_t s) {
  logprobs_backward_kernel<T><<<static_cast<unsigned>(a.rows), kThreads, 0, s>>>(
      static_cast<const T*>(a.x), a.V, a.ld, a.targets, static_cast<float>(1.0 / a.tau), a.lse,
      a.entropy, a.d_logp, a.d_entropy, static_cast<T*>(a.dx), a.ld_d, a.status);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_token_logprobs(const LogprobArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case BERGSON_BF16: return run_forward<__nv_bfloat16>(a, s);
    case BERGSON_F16: return run_forward<__half>(a, s);
    default: return run_forward<float>(a, s);
  }
}

cudaError_t launch_token_logprobs_backward(const LogprobGradArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case BERGSON_BF16: return run_backward<__nv_bfloat16>(a, s);
    case BERGSON_F16: return run_backward<__half>(a, s);
    default: return run_backward<float>(a, s);
  }
}

}  // namespace bergson
