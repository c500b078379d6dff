// One AdamW step over many tensors, states in 32 or 8 bits.
//
// The tensors' records travel in the kernel's parameters (up to 32 KB), so a
// launch needs no table on the device.  A warp takes 256 consecutive elements
// of one tensor, which is the block that shares a scale of an 8-bit state.
//
// m and v are formed by multiplications and additions that are each rounded
// (no fused multiply-add): the codes of an 8-bit state then follow from the
// formula alone, whichever program computes them.

#include <cmath>

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxEntries = 300;

struct Entry {
  void* p;
  const void* g;
  float* master;
  void* m;
  void* v;
  float* ms;
  float* vs;
  int64_t n;
  uint64_t key;                // start of the tensor's SplitMix64 sequence
  float lr, wd;                // lr lr_scale, weight decay
  uint8_t pt, gt, st, pad[5];
};

struct StepParams {
  Entry e[kMaxEntries];
  uint32_t begin[kMaxEntries + 1];   // first block of each tensor in the launch
  int n;
  float b1, b2, a1, a2;        // beta, 1 - beta
  float c1, c2, eps;           // bias corrections 1 / (1 - beta^step)
  const float* grad_scale;
};

__device__ __forceinline__ float load_as_f32(const void* p, int type, int64_t i) {
  if (type == BERGSON_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  if (type == BERGSON_F16) return __half2float(static_cast<const __half*>(p)[i]);
  return static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_from_f32(void* p, int type, int64_t i, float x) {
  if (type == BERGSON_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
  else if (type == BERGSON_F16) static_cast<__half*>(p)[i] = __float2half_rn(x);
  else static_cast<float*>(p)[i] = x;
}

__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ StepParams s) {
  const uint32_t block = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (block >= s.begin[s.n]) return;
  int lo = 0, hi = s.n;                          // begin[lo] <= block < begin[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (s.begin[mid] <= block) lo = mid; else hi = mid;
  }
  const Entry& e = s.e[lo];
  const int64_t first = static_cast<int64_t>(block - s.begin[lo]) * kStateBlock;
  const int lane = threadIdx.x & 31;
  const float gs = s.grad_scale != nullptr ? *s.grad_scale : 1.0f;
  const bool eight = e.st == BERGSON_STATE_8BIT;
  const float ms = eight ? e.ms[first / kStateBlock] : 0.0f;
  const float vs = eight ? e.vs[first / kStateBlock] : 0.0f;
  float m[8], v[8], top_m = 0.0f, top_v = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int64_t i = first + lane + 32 * k;
    m[k] = v[k] = 0.0f;
    if (i >= e.n) continue;
    const float g = __fmul_rn(load_as_f32(e.g, e.gt, i), gs);
    float m0, v0;
    if (eight) {
      m0 = __fmul_rn(decode_first(static_cast<const uint8_t*>(e.m)[i]), ms);
      v0 = __fmul_rn(decode_second(static_cast<const uint8_t*>(e.v)[i]), vs);
    } else {
      m0 = static_cast<const float*>(e.m)[i];
      v0 = static_cast<const float*>(e.v)[i];
    }
    m[k] = __fadd_rn(__fmul_rn(m0, s.b1), __fmul_rn(g, s.a1));
    v[k] = __fadd_rn(__fmul_rn(v0, s.b2), __fmul_rn(__fmul_rn(g, g), s.a2));
    const float w = e.master != nullptr ? e.master[i] : load_as_f32(e.p, e.pt, i);
    const float step = (m[k] * s.c1) / (sqrtf(v[k] * s.c2) + s.eps);
    const float w1 = w - e.lr * (step + e.wd * w);
    if (e.master != nullptr) e.master[i] = w1;
    store_from_f32(e.p, e.pt, i, w1);
    if (!eight) {
      static_cast<float*>(e.m)[i] = m[k];
      static_cast<float*>(e.v)[i] = v[k];
    }
    // of the bits, so that a NaN is the largest
    top_m = __uint_as_float(max(__float_as_uint(top_m), __float_as_uint(fabsf(m[k]))));
    top_v = __uint_as_float(max(__float_as_uint(top_v), __float_as_uint(fabsf(v[k]))));
  }
  if (!eight) return;
  top_m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top_m)));
  top_v = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top_v)));
  const float ms1 = block_scale(top_m), vs1 = block_scale(top_v);
  const float im = block_inverse(ms1), iv = block_inverse(vs1);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int64_t i = first + lane + 32 * k;
    if (i >= e.n) continue;
    const uint64_t h = mix64(e.key + (static_cast<uint64_t>(i >> 2) + 1) * kSplitMixGamma);
    const uint32_t chance = static_cast<uint32_t>(h >> (16 * (i & 3))) & 0xffffu;
    static_cast<uint8_t*>(e.m)[i] = static_cast<uint8_t>(encode_first(m[k], im, chance));
    static_cast<uint8_t*>(e.v)[i] = static_cast<uint8_t>(encode_second(v[k], iv, chance));
  }
  if (lane == 0) {
    e.ms[first / kStateBlock] = ms1;
    e.vs[first / kStateBlock] = vs1;
  }
}

__global__ void __launch_bounds__(kThreads) state_values_kernel(
    const uint8_t* __restrict__ codes, const float* __restrict__ scale, int64_t n, int moment,
    float* __restrict__ out) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= n) return;
  const float y = moment == BERGSON_MOMENT_FIRST ? decode_first(codes[i]) : decode_second(codes[i]);
  out[i] = __fmul_rn(y, scale[i / kStateBlock]);
}

}  // namespace

cudaError_t launch_adamw(const bergson_adamw_tensor* t, int n, const AdamwScalars& a,
                         cudaStream_t s) {
  StepParams p;
  p.b1 = static_cast<float>(a.beta1);
  p.b2 = static_cast<float>(a.beta2);
  p.a1 = static_cast<float>(1.0 - a.beta1);
  p.a2 = static_cast<float>(1.0 - a.beta2);
  p.c1 = static_cast<float>(1.0 / (1.0 - std::pow(a.beta1, static_cast<double>(a.step))));
  p.c2 = static_cast<float>(1.0 / (1.0 - std::pow(a.beta2, static_cast<double>(a.step))));
  p.eps = static_cast<float>(a.eps);
  p.grad_scale = a.grad_scale;
  const uint64_t base = mix64(a.seed ^ mix64(static_cast<uint64_t>(a.step)));
  constexpr int64_t kMaxBlocks = int64_t{1} << 31;   // of a launch
  p.n = 0;
  p.begin[0] = 0;
  const auto flush = [&]() -> cudaError_t {
    if (p.n == 0) return cudaSuccess;
    adamw_kernel<<<(p.begin[p.n] + kWarps - 1) / kWarps, kThreads, 0, s>>>(p);
    p.n = 0;
    return cudaGetLastError();
  };
  for (int i = 0; i < n; ++i) {
    if (t[i].n == 0) continue;
    const int64_t blocks = (t[i].n + kStateBlock - 1) / kStateBlock;
    if (p.n == kMaxEntries || (p.n > 0 && p.begin[p.n] + blocks > kMaxBlocks)) {
      const cudaError_t e = flush();
      if (e != cudaSuccess) return e;
    }
    Entry& e = p.e[p.n];
    e.p = t[i].param;
    e.g = t[i].grad;
    e.master = t[i].master;
    e.m = t[i].m;
    e.v = t[i].v;
    e.ms = t[i].m_scale;
    e.vs = t[i].v_scale;
    e.n = t[i].n;
    e.key = mix64(static_cast<uint64_t>(i) ^ base);
    e.lr = static_cast<float>(a.lr * t[i].lr_scale);
    e.wd = t[i].weight_decay;
    e.pt = static_cast<uint8_t>(t[i].param_dtype);
    e.gt = static_cast<uint8_t>(t[i].grad_dtype);
    e.st = static_cast<uint8_t>(t[i].state_kind);
    p.begin[p.n + 1] = p.begin[p.n] + static_cast<uint32_t>(blocks);
    ++p.n;
  }
  return flush();
}

cudaError_t launch_state_values(const uint8_t* codes, const float* scale, int64_t n, int moment,
                                float* out, cudaStream_t s) {
  if (n == 0) return cudaSuccess;
  state_values_kernel<<<static_cast<unsigned>((n + kThreads - 1) / kThreads), kThreads, 0, s>>>(
      codes, scale, n, moment, out);
  return cudaGetLastError();
}

}  // namespace bergson
