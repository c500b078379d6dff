// One AdamW step over many tensors, states in 32 or 8 bits.
//
// The tensors' records travel in the kernel's parameters (up to 32 KB), so a
// launch needs no table on the device.  A warp takes 256 consecutive elements
// of one tensor at a time, which is the block that shares a scale of an 8-bit
// state; a lane has 8 of them, in loads of 8 to 32 bytes.  The step is bound by its
// bytes: 2 + 2 + 16 an element with 16-bit parameters and gradients and 32-bit
// states, 2 + 2 + 2 + 4 with 8-bit ones, 8 more with a master copy (2 less read).  201M
// elements with masters and 32-bit states: 798 us, 7.1 TB/s.  With 8-bit states
// some 70 instructions an element stand beside the bytes, half of them on the integer
// pipe: 50M elements with masters 128 us (6.3 TB/s, two thirds of the issue slots), without 116
// (4.4 TB/s, three quarters of them).
//
// m and v are formed by multiplications and additions that are each rounded
// (no fused multiply-add): the codes of an 8-bit state then follow from the
// formula alone, whichever program computes them.  The step itself takes the
// short square root and reciprocal (1 unit each), which no state sees.

#include <cmath>

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
// Tensors of a kind share a launch: fp32 states; 8-bit states without and with a master
// copy.  A warp takes kRun blocks of them.  Without a master copy two blocks share what comes
// before them (50M elements, 1 / 2 / 4 blocks: 136 / 115 / 121 us); with one the loop's
// registers cost more (1 / 2: 127 / 138).
enum class Kind { kWide, kEight, kEightMaster };
template <Kind kKind>
constexpr int kRun = kKind == Kind::kEight ? 2 : 1;
constexpr int kFew = 24, kMany = 300;          // records a launch can take

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
  float lr_c1, lr_wd;          // lr lr_scale / (1 - beta1^step), lr lr_scale weight_decay
  uint8_t pt, gt, st;
  uint8_t vec;                 // every pointer fits loads of 8 elements
  uint8_t pad[4];
};

struct StepScalars {
  float b1, b2, a1, a2;        // beta, 1 - beta
  float c2, eps;               // 1 / (1 - beta2^step)
  int n;                       // tensors
  const float* grad_scale;
};

template <int N>
struct StepParams {
  StepScalars s;
  uint32_t begin[N + 1];       // first CTA of each tensor in the launch
  Entry e[N];
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

// 8 elements from i on, as they lie in memory (16 bytes, or 32 of fp32).
__device__ __forceinline__ void load8(const void* p, int type, int64_t i, uint32_t (&r)[8]) {
  if (type == BERGSON_F32) {
    load32(static_cast<const float*>(p) + i, r);
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    r[0] = u.x; r[1] = u.y; r[2] = u.z; r[3] = u.w;
  }
}
__device__ __forceinline__ void to_floats(const uint32_t (&r)[8], int type, float (&x)[8]) {
  if (type == BERGSON_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = __uint_as_float(r[k] << 16);
      x[2 * k + 1] = __uint_as_float(r[k] & 0xffff0000u);
    }
  } else if (type == BERGSON_F16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r[k]));
      x[2 * k] = f.x;
      x[2 * k + 1] = f.y;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(r[k]);
  }
}
__device__ __forceinline__ void store8(void* p, int type, int64_t i, const float (&x)[8]) {
  if (type == BERGSON_F32) {
    uint32_t r[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = __float_as_uint(x[k]);
    store32(static_cast<float*>(p) + i, r);
    return;
  }
  uint4 u;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (type == BERGSON_BF16)
      pack2(u, k, make_float2(x[2 * k], x[2 * k + 1]), static_cast<const __nv_bfloat16*>(nullptr));
    else
      pack2(u, k, make_float2(x[2 * k], x[2 * k + 1]), static_cast<const __half*>(nullptr));
  }
  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) = u;
}

__device__ __forceinline__ float next_first(const StepScalars& s, float m, float g) {
  return __fadd_rn(__fmul_rn(m, s.b1), __fmul_rn(g, s.a1));
}
__device__ __forceinline__ float next_second(const StepScalars& s, float v, float g) {
  return __fadd_rn(__fmul_rn(v, s.b2), __fmul_rn(__fmul_rn(g, g), s.a2));
}
// w - lr (c1 m / (sqrt(vc) + eps) + wd w), vc = c2 v.  It counts at least as the normal range's
// end: 0 / 0 cannot arise.
__device__ __forceinline__ float next_weight(const StepScalars& s, const Entry& e, float w, float m,
                                             float vc) {
  const float root = sqrt_approx(at_least(vc, 1.17549435e-38f));
  return fmaf(-e.lr_c1 * m, rcp_approx(root + s.eps), fmaf(-e.lr_wd, w, w));
}
__device__ __forceinline__ float block_top(float top) {     // of the warp's lanes, NaN the largest
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
}

// A whole block of a tensor whose pointers fit.
template <Kind kKind>
__device__ __forceinline__ void block_vectors(const StepScalars& s, const Entry& e, int64_t first,
                                              float gs) {
  const int lane = threadIdx.x & 31;
  const int64_t i = first + 8 * lane;
  constexpr bool kEight = kKind != Kind::kWide;
  const bool master =
      kKind == Kind::kEightMaster || (kKind == Kind::kWide && e.master != nullptr);
  uint32_t rw[8], rg[8], rm[8], rv[8];
  load8(e.g, e.gt, i, rg);
  if (master) load32(e.master + i, rw); else load8(e.p, e.pt, i, rw);
  float ms = 0.0f, vs = 0.0f;
  if (kEight) {
    const uint2 um = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(e.m) + i);
    const uint2 uv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(e.v) + i);
    rm[0] = um.x; rm[1] = um.y;
    rv[0] = uv.x; rv[1] = uv.y;
    ms = e.ms[first / kStateBlock];
    vs = e.vs[first / kStateBlock];
  } else {
    load32(static_cast<const float*>(e.m) + i, rm);
    load32(static_cast<const float*>(e.v) + i, rv);
  }
  float g[8], w[8], m[8], v[8];
  to_floats(rg, e.gt, g);
  to_floats(rw, master ? BERGSON_F32 : e.pt, w);
  if (kEight) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      decode_nonzero_first4(rm[q], m + 4 * q);
      decode_nonzero_second4(rv[q], v + 4 * q);
    }
    // codes of 0 are rare but where there is no gradient: a branch of the warp
    if (__any_sync(0xffffffffu, (zero_bytes(rm[0] & 0x7f7f7f7fu) | zero_bytes(rm[1] & 0x7f7f7f7fu) |
                                 zero_bytes(rv[0]) | zero_bytes(rv[1])) != 0)) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        put_zeros4(rm[q] & 0x7f7f7f7fu, m + 4 * q);
        put_zeros4(rv[q], v + 4 * q);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m[k] = __uint_as_float(rm[k]);
      v[k] = __uint_as_float(rv[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < 8; k += 2) {               // next_first and next_second, two lanes at once
    const float2 g2 = mul2(make_float2(g[k], g[k + 1]), pair(gs));
    float2 m2 = make_float2(m[k], m[k + 1]), v2 = make_float2(v[k], v[k + 1]);
    if (kEight) {
      m2 = mul2(m2, pair(ms));
      v2 = mul2(v2, pair(vs));
    }
    m2 = mul2(m2, pair(s.b1));
    v2 = mul2(v2, pair(s.b2));
    const float2 mg = mul2(g2, pair(s.a1)), vg = mul2(mul2(g2, g2), pair(s.a2));
    // one lane each: a sum of two lanes would be merged with the products before it
    m[k] = __fadd_rn(m2.x, mg.x); m[k + 1] = __fadd_rn(m2.y, mg.y);
    v[k] = __fadd_rn(v2.x, vg.x); v[k + 1] = __fadd_rn(v2.y, vg.y);
    const float2 vc = mul2(make_float2(v[k], v[k + 1]), pair(s.c2));
    w[k] = next_weight(s, e, w[k], m[k], vc.x);
    w[k + 1] = next_weight(s, e, w[k + 1], m[k + 1], vc.y);
  }
  if (master) store8(e.master, BERGSON_F32, i, w);
  store8(e.p, e.pt, i, w);
  if (!kEight) {
    store8(e.m, BERGSON_F32, i, m);
    store8(e.v, BERGSON_F32, i, v);
    return;
  }
  float top_m = 0.0f, top_v = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    top_m = max_nan(top_m, m[k]);
    top_v = max_nan(top_v, v[k]);
  }
  // the lower lanes take m's scale and its inverse, the upper ones v's
  const float all_m = block_top(top_m), all_v = block_top(top_v);
  const float scale = block_scale(lane < 16 ? all_m : all_v), inverse = block_inverse(scale);
  const float im = __shfl_sync(0xffffffffu, inverse, 0), iv = __shfl_sync(0xffffffffu, inverse, 16);
  uint32_t cm[2], cv[2];
  const uint64_t at = e.key + (static_cast<uint64_t>(i >> 2) + 1) * kSplitMixGamma;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    uint32_t c[4];
    chances(mix64(at + q * kSplitMixGamma), c);
    cm[q] = encode_first4(m + 4 * q, im, c);
    cv[q] = encode_second4(v + 4 * q, iv, c);
  }
  if (__any_sync(0xffffffffu, (zero_bytes(cv[0]) | zero_bytes(cv[1])) != 0)) {
    cv[0] = raise_zeros4(cv[0], v);
    cv[1] = raise_zeros4(cv[1], v + 4);
  }
  *reinterpret_cast<uint2*>(static_cast<uint8_t*>(e.m) + i) = make_uint2(cm[0], cm[1]);
  *reinterpret_cast<uint2*>(static_cast<uint8_t*>(e.v) + i) = make_uint2(cv[0], cv[1]);
  if (lane % 16 == 0) (lane == 0 ? e.ms : e.vs)[first / kStateBlock] = scale;
}

// Any block: element by element, neighbouring lanes at neighbouring elements.
__device__ __noinline__ void block_elements(const StepScalars& s, const Entry& e, int64_t first,
                                            float gs) {
  const int lane = threadIdx.x & 31;
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
    m[k] = next_first(s, m0, g);
    v[k] = next_second(s, v0, g);
    const float w = next_weight(
        s, e, e.master != nullptr ? e.master[i] : load_as_f32(e.p, e.pt, i), m[k],
        v[k] * s.c2);
    if (e.master != nullptr) e.master[i] = w;
    store_from_f32(e.p, e.pt, i, w);
    if (!eight) {
      static_cast<float*>(e.m)[i] = m[k];
      static_cast<float*>(e.v)[i] = v[k];
    }
    top_m = max_nan(top_m, m[k]);
    top_v = max_nan(top_v, v[k]);
  }
  if (!eight) return;
  const float ms1 = block_scale(block_top(top_m)), vs1 = block_scale(block_top(top_v));
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

// Nine CTAs an SM: 56 registers (10 spill: 134 against 127 us for 50M 8-bit elements with
// masters).
template <int N, Kind kKind>
__global__ void __launch_bounds__(kThreads, 9) adamw_kernel(
    const __grid_constant__ StepParams<N> p) {
  int lo = 0, hi = p.s.n;                        // begin[lo] <= CTA < begin[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (p.begin[mid] <= blockIdx.x) lo = mid; else hi = mid;
  }
  const Entry& e = p.e[lo];
  griddep_wait();
  const float gs = p.s.grad_scale != nullptr ? *p.s.grad_scale : 1.0f;
  int64_t first = (static_cast<int64_t>(blockIdx.x - p.begin[lo]) * (kWarps * kRun<kKind>) +
                   (threadIdx.x >> 5)) * kStateBlock;
#pragma unroll 1
  for (int k = 0; k < kRun<kKind>; ++k, first += kWarps * kStateBlock) {
    if (first >= e.n) return;
    if (!e.vec || first + kStateBlock > e.n) block_elements(p.s, e, first, gs);
    else block_vectors<kKind>(p.s, e, first, gs);
  }
}

// 8 codes a thread where the pointers allow it.
__global__ void __launch_bounds__(kThreads) state_values_kernel(
    const uint8_t* __restrict__ codes, const float* __restrict__ scale, int64_t n, int moment,
    int vec, float* __restrict__ out) {
  const int64_t i = 8 * (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x);
  griddep_wait();
  if (i >= n) return;
  const float sc = scale[i / kStateBlock];
  if (vec && i + 8 <= n) {
    const uint2 u = *reinterpret_cast<const uint2*>(codes + i);
    float x[8];
    if (moment == BERGSON_MOMENT_FIRST) {
      decode_first4(u.x, x);
      decode_first4(u.y, x + 4);
    } else {
      decode_second4(u.x, x);
      decode_second4(u.y, x + 4);
    }
    uint32_t r[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = __float_as_uint(__fmul_rn(x[k], sc));
    store32(out + i, r);
    return;
  }
  for (int k = 0; k < 8 && i + k < n; ++k) {
    const uint32_t c = codes[i + k];
    out[i + k] = __fmul_rn(moment == BERGSON_MOMENT_FIRST ? decode_first(c) : decode_second(c), sc);
  }
}

bool on(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool fits_vectors(const bergson_adamw_tensor& t) {
  const size_t state = t.state_kind == BERGSON_STATE_8BIT ? 8 : 32;
  return on(t.param, t.param_dtype == BERGSON_F32 ? 32 : 16) &&
         on(t.grad, t.grad_dtype == BERGSON_F32 ? 32 : 16) && on(t.master, 32) && on(t.m, state) &&
         on(t.v, state);
}

Kind kind_of(const bergson_adamw_tensor& t) {
  return t.state_kind == BERGSON_STATE_F32 ? Kind::kWide
         : t.master == nullptr             ? Kind::kEight
                                           : Kind::kEightMaster;
}

int64_t blocks_of(int64_t n) { return (n + kStateBlock - 1) / kStateBlock; }

// The tensors of one kind.
template <int N, Kind kKind>
cudaError_t run_adamw(const bergson_adamw_tensor* t, int n, const AdamwScalars& a, cudaStream_t s) {
  StepParams<N> p;
  p.s.b1 = static_cast<float>(a.beta1);
  p.s.b2 = static_cast<float>(a.beta2);
  p.s.a1 = static_cast<float>(1.0 - a.beta1);
  p.s.a2 = static_cast<float>(1.0 - a.beta2);
  const double c1 = 1.0 / (1.0 - std::pow(a.beta1, static_cast<double>(a.step)));
  p.s.c2 = static_cast<float>(1.0 / (1.0 - std::pow(a.beta2, static_cast<double>(a.step))));
  p.s.eps = static_cast<float>(a.eps);
  p.s.grad_scale = a.grad_scale;
  const uint64_t base = mix64(a.seed ^ mix64(static_cast<uint64_t>(a.step)));
  constexpr int64_t cta_blocks = kWarps * kRun<kKind>;
  constexpr int64_t kMaxCtas = INT32_MAX;       // of a launch
  int k = 0;
  p.begin[0] = 0;
  const auto flush = [&]() -> cudaError_t {
    if (k == 0) return cudaSuccess;
    p.s.n = k;
    const dim3 grid(p.begin[k]);
    k = 0;
    return launch_dependent(adamw_kernel<N, kKind>, grid, dim3(kThreads), 0, s, p);
  };
  for (int i = 0; i < n; ++i) {
    if (t[i].n == 0 || kind_of(t[i]) != kKind) continue;
    const int64_t ctas = (blocks_of(t[i].n) + cta_blocks - 1) / cta_blocks;
    if (k == N || (k > 0 && p.begin[k] + ctas > kMaxCtas)) {
      const cudaError_t e = flush();
      if (e != cudaSuccess) return e;
    }
    Entry& e = p.e[k];
    e.p = t[i].param;
    e.g = t[i].grad;
    e.master = t[i].master;
    e.m = t[i].m;
    e.v = t[i].v;
    e.ms = t[i].m_scale;
    e.vs = t[i].v_scale;
    e.n = t[i].n;
    e.key = mix64(static_cast<uint64_t>(i) ^ base);
    e.lr_c1 = static_cast<float>(a.lr * t[i].lr_scale * c1);
    e.lr_wd = static_cast<float>(a.lr * t[i].lr_scale * t[i].weight_decay);
    e.pt = static_cast<uint8_t>(t[i].param_dtype);
    e.gt = static_cast<uint8_t>(t[i].grad_dtype);
    e.st = static_cast<uint8_t>(t[i].state_kind);
    e.vec = fits_vectors(t[i]) ? 1 : 0;
    p.begin[k + 1] = p.begin[k] + static_cast<uint32_t>(ctas);
    ++k;
  }
  return flush();
}

template <Kind kKind>
cudaError_t run_kind(const bergson_adamw_tensor* t, int n, int count, const AdamwScalars& a,
                     cudaStream_t s) {
  if (count == 0) return cudaSuccess;
  return count <= kFew ? run_adamw<kFew, kKind>(t, n, a, s) : run_adamw<kMany, kKind>(t, n, a, s);
}

}  // namespace

cudaError_t launch_adamw(const bergson_adamw_tensor* t, int n, const AdamwScalars& a,
                         cudaStream_t s) {
  int count[3] = {0, 0, 0};
  for (int i = 0; i < n; ++i) {
    if (t[i].n > 0) ++count[static_cast<int>(kind_of(t[i]))];
  }
  cudaError_t e = run_kind<Kind::kWide>(t, n, count[0], a, s);
  if (e == cudaSuccess) e = run_kind<Kind::kEight>(t, n, count[1], a, s);
  if (e == cudaSuccess) e = run_kind<Kind::kEightMaster>(t, n, count[2], a, s);
  return e;
}

cudaError_t launch_state_values(const uint8_t* codes, const float* scale, int64_t n, int moment,
                                float* out, cudaStream_t s) {
  const int64_t grid = (n + 8 * kThreads - 1) / (8 * kThreads);
  return launch_dependent(state_values_kernel, dim3(static_cast<unsigned>(grid)), dim3(kThreads),
                          0, s, codes, scale, n, moment, on(codes, 8) && on(out, 32) ? 1 : 0, out);
}

}  // namespace bergson
