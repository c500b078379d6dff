// Token log-probabilities of logits and their backward pass.
//
//   z = x / tau,  lse = log sum_v exp(z_v),  logp = z_t - lse,
//   H = -sum_v p_v log p_v = ln 2 (log2 s - w / s)  with  m = max x,  u = (x - m) log2(e) / tau,
//   s = sum 2^u,  w = sum u 2^u,
//   dx_v = (d_logp ([v = t] - p_v) - d_H p_v (log p_v + H)) / tau.
//
// The forward pass reads a row once.  A thread takes four 16-byte vectors at a
// time: their largest element first (in the logits' own type), its two sums are
// rescaled where the maximum has grown, then a subtraction, a product, an ex2
// and two accumulations an element, in pairs of fp32 lanes.  Differences from
// the maximum are formed before anything is scaled, so that entries at a type's
// lowest value take no other path.
//
// The backward pass takes p from x / tau - lse, where fp32 holds what lse has to say of the
// sum; a row whose lse is far from 0 (logits at a large common offset, a finite mask over all
// of them) is summed again about its largest element.
//
// Both passes are bound by the logits' bytes: 8192 x 131,072 bf16 with entropies 288 us
// (6.7 TB/s, the measured copy rate; ex2 and the conversions fill half of the
// issue slots), the gradients at 8192 x 65,536, half of whose rows are left out and only
// written, 235 us (6.8 TB/s).

#include <type_traits>

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                     // vectors a thread has on the way
// 64 registers hold them and their sums.  8192 x 131,072 bf16 with entropies, us:
// 4 vectors at 3 / 4 CTAs an SM 320 / 290, 3 at 4: 311, 2 at 5 / 6: 319 / 317.
constexpr int kFwdCtas = 4;
// 48 registers, of which the rare second sum of a far row takes its share (1031 x 32,003 fp16 with
// entropies at 5 / 6: 20.9 / 21.8 us).
constexpr int kBwdCtas = 5;
constexpr float kInf = __builtin_huge_valf();
constexpr float kNoRow = -1e30f;               // a row's lse below this: it has no entries
// From here on an fp32 lse says too little of the sum: its half unit, 1.5e-5 below 512, is p's
// relative error, and from 2^24 on log V is lost beside it.  8192 x 65,536 bf16 with all rows below
// / above: 306 / 461 us.
constexpr float kFarLse = 512.0f;
constexpr float kLog2e = 1.44269504f;
constexpr float kLn2 = 0.693147181f;

struct RowSums {
  float m = -kInf, s = 0.0f, w = 0.0f;
};

// w about a maximum that is larger by -d, f = 2^d.  Where f is 0 nothing is left,
// also where s d would pass the range (or the side is empty, d = -inf).
__device__ __forceinline__ float shifted(float w, float s, float f, float d) {
  return f > 0.0f ? f * (w + s * d) : 0.0f;
}

__device__ __forceinline__ void merge(RowSums& a, const RowSums& b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float da = a.m == m ? 0.0f : (a.m - m) * c, db = b.m == m ? 0.0f : (b.m - m) * c;
  const float fa = exp2_approx(da), fb = exp2_approx(db);
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

template <typename T, int N>
__device__ __forceinline__ float largest(const uint4 (&v)[N]) {
  if constexpr (sizeof(T) == 4) {
    float m = vec_max(v[0], static_cast<const float*>(nullptr));
#pragma unroll
    for (int k = 1; k < N; ++k) m = fmaxf(m, vec_max(v[k], static_cast<const float*>(nullptr)));
    return m;
  } else {
    using H2 = typename std::conditional<std::is_same<T, __half>::value, __half2,
                                         __nv_bfloat162>::type;
    H2 m = vec_max2<H2>(v[0]);
#pragma unroll
    for (int k = 1; k < N; ++k) m = __hmax2(m, vec_max2<H2>(v[k]));
    return fmaxf(to_f32(m.x), to_f32(m.y));
  }
}

// A thread's running sums, two lanes each.
template <typename T, bool kEntropy>
struct Accumulator {
  float m = -kInf;
  float2 s = {0.0f, 0.0f}, w = {0.0f, 0.0f};

  __device__ __forceinline__ void raise(float top, float c) {
    const float d = (m - top) * c;             // -inf from the start
    const float f = exp2_approx(d);
    if (kEntropy) {
      w.x = shifted(w.x, s.x, f, d);
      w.y = shifted(w.y, s.y, f, d);
    }
    s.x *= f;
    s.y *= f;
    m = top;
  }

  template <int N>
  __device__ __forceinline__ void take(const uint4 (&v)[N], float c) {
    const float top = largest<T>(v);
    if (top > m) raise(top, c);
    const float2 neg = pair(m == -kInf ? 0.0f : -m), cc = pair(c);
    const float2 w0 = w;
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
      for (int j = 0; j < Vec16<T>::kPairs; ++j) {
        const float2 u = mul2(add2(unpack2(v[k], j, static_cast<const T*>(nullptr)), neg), cc);
        const float2 e = make_float2(exp2_approx(u.x), exp2_approx(u.y));
        s = add2(s, e);
        if (kEntropy) w = fma2(e, u, w);
      }
    }
    // an entry of -inf (or one that the scale takes there) made 0 * inf: once more
    // with its product left out; a NaN among the logits is in s already
    if (kEntropy && !(w.x == w.x && w.y == w.y)) {
      w = w0;
      for (int k = 0; k < N; ++k) {
        for (int j = 0; j < Vec16<T>::kPairs; ++j) {
          const float2 u = mul2(add2(unpack2(v[k], j, static_cast<const T*>(nullptr)), neg), cc);
          const float ex = exp2_approx(u.x), ey = exp2_approx(u.y);
          if (ex > 0.0f) w.x = fmaf(ex, u.x, w.x);
          if (ey > 0.0f) w.y = fmaf(ey, u.y, w.y);
        }
      }
    }
  }

  __device__ __forceinline__ void take_one(T x, float c) {
    const float f = to_f32(x);
    if (f > m) raise(f, c);
    const float u = (f - (m == -kInf ? 0.0f : m)) * c;
    const float e = exp2_approx(u);
    s.x += e;
    if (kEntropy && e > 0.0f) w.x = fmaf(e, u, w.x);
  }

  __device__ __forceinline__ RowSums sums() const {
    RowSums r;
    r.m = m;
    r.s = s.x + s.y;
    r.w = w.x + w.y;
    return r;
  }
};

// Elements before the first 16-byte boundary of a row (at most V).
template <typename T>
__device__ __forceinline__ int64_t head_of(const T* row, int64_t V) {
  const int64_t h = ((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(T);
  return h < V ? h : V;
}

// What thread `at` of `n` finds in its share of a row: every n-th vector of [first,
// last), kVecs of them on the way, and the elements outside the vectors where `edges` is set.
template <typename T, bool kEntropy, int kVecs>
__device__ __forceinline__ RowSums scan_row(const T* row, int64_t V, float c, int at, int n,
                                            int part, int parts) {
  constexpr int E = Vec16<T>::kElems;
  const int64_t head = head_of(row, V);
  const int64_t vecs = (V - head) / E;
  const int64_t per = (vecs + parts - 1) / parts;
  const int64_t last = min(vecs, per * (part + 1));
  const uint4* body = reinterpret_cast<const uint4*>(row + head);
  Accumulator<T, kEntropy> a;
  int64_t i = per * part + at;
  for (; i + (kVecs - 1) * n < last; i += kVecs * n) {
    uint4 v[kVecs];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) v[k] = __ldcs(body + i + k * n);
    a.take(v, c);
  }
  if constexpr (kVecs > 1) {
    uint4 v[kVecs - 1][1];
#pragma unroll
    for (int k = 0; k < kVecs - 1; ++k)
      if (i + k * n < last) v[k][0] = __ldcs(body + i + k * n);
#pragma unroll
    for (int k = 0; k < kVecs - 1; ++k)
      if (i + k * n < last) a.take(v[k], c);
  }
  if (part == 0) {
    if (at < head) a.take_one(row[at], c);
    const int64_t tail = head + vecs * E + at;
    if (tail < V) a.take_one(row[tail], c);
  }
  return a.sums();
}

// n < E elements lie before the first vector and after the last: fewer than a warp's lanes.
static_assert(Vec16<__half>::kElems <= 32, "edges are taken by one pass of a warp");

struct ForwardParams {
  const void* x;
  int64_t rows, V, ld;
  const int64_t* targets;
  float inv_tau, c;            // 1 / tau, log2(e) / tau
  float* logp;
  float* lse;
  float* entropy;
  int* status;
};

template <typename T>
__device__ __forceinline__ void write_row(const ForwardParams& p, int64_t r, int64_t t,
                                          const RowSums& a) {
  const float nan = __int_as_float(0x7fffffff);
  const bool none = a.m == -kInf && a.s == 0.0f;
  const bool bad = !(a.m < kInf) || a.s != a.s;
  const float ls = log2f(a.s) * kLn2;
  p.lse[r] = none ? -kInf : bad ? nan : fmaf(a.m, p.inv_tau, ls);
  if (p.entropy != nullptr) p.entropy[r] = none ? 0.0f : bad ? nan : ls - a.w / a.s * kLn2;
  if (t >= p.V) {
    if (p.status != nullptr) atomicCAS(p.status, 0, BERGSON_EINVAL);
    p.logp[r] = nan;
  } else if (none || bad) {
    p.logp[r] = none ? -kInf : nan;
  } else {
    p.logp[r] = (to_f32(static_cast<const T*>(p.x)[r * p.ld + t]) - a.m) * p.inv_tau - ls;
  }
}

__device__ __forceinline__ void write_left_out(const ForwardParams& p, int64_t r) {
  p.logp[r] = 0.0f;
  p.lse[r] = 0.0f;
  if (p.entropy != nullptr) p.entropy[r] = 0.0f;
}

// A CTA (or the CTAs of a cluster, each its part) takes a row.
template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kThreads, kFwdCtas) logprobs_row_kernel(const ForwardParams p) {
  __shared__ RowSums red[kThreads / 32];
  __shared__ RowSums ranks[8];
  const int parts = static_cast<int>(cluster_size());
  const int part = static_cast<int>(blockIdx.x) % parts;
  const int64_t r = blockIdx.x / parts;
  griddep_wait();
  const int64_t t = p.targets[r];
  if (t < 0) {
    if (threadIdx.x == 0 && part == 0) write_left_out(p, r);
    return;
  }
  const T* row = static_cast<const T*>(p.x) + r * p.ld;
  if (parts > 1) cluster_arrive();
  RowSums a = scan_row<T, kEntropy, kUnroll>(row, p.V, p.c, threadIdx.x, kThreads, part, parts);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) merge(a, shuffle(a, o), p.c);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
  __syncthreads();
  if (threadIdx.x < 32) {
    a = red[threadIdx.x & (kThreads / 32 - 1)];
#pragma unroll
    for (int o = kThreads / 64; o > 0; o >>= 1) merge(a, shuffle(a, o), p.c);
  }
  if (parts > 1) {
    cluster_wait();                            // the first CTA has started
    if (threadIdx.x == 0) {
      st_cluster(&ranks[part].m, 0, a.m);
      st_cluster(&ranks[part].s, 0, a.s);
      st_cluster(&ranks[part].w, 0, a.w);
    }
    cluster_barrier();
    if (part != 0) return;
    if (threadIdx.x == 0) {
      a = ranks[0];
      for (int k = 1; k < parts; ++k) merge(a, ranks[k], p.c);
    }
  }
  if (threadIdx.x == 0) write_row<T>(p, r, t, a);
}

// A warp takes a row.
template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kThreads, kFwdCtas) logprobs_warp_kernel(const ForwardParams p) {
  griddep_wait();
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  if (r >= p.rows) return;
  const int lane = threadIdx.x & 31;
  const int64_t t = p.targets[r];
  if (t < 0) {
    if (lane == 0) write_left_out(p, r);
    return;
  }
  const T* row = static_cast<const T*>(p.x) + r * p.ld;
  RowSums a = scan_row<T, kEntropy, kUnroll>(row, p.V, p.c, lane, 32, 0, 1);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) merge(a, shuffle(a, o), p.c);
  if (lane == 0) write_row<T>(p, r, t, a);
}

// ---------------------------------------------------------------- backward

struct BackwardParams {
  const void* x;
  int64_t rows, V, ld;
  const int64_t* targets;
  float inv_tau, c;            // 1 / tau, log2(e) / tau
  const float* lse;
  const float* entropy;
  const float* d_logp;
  const float* d_entropy;
  void* dx;
  int64_t ld_d;
  int slices;                  // CTAs a row
  int* status;
};

// One row's constants.  log p_v = q - rest, q = x_v / tau - lse; rest is 0 but for far rows.
struct RowGrad {
  float inv_tau, lse;
  float rest2;                 // -rest log2(e)
  float a, b;                  // dx_v = p_v (a + b q) + [v = t] hit
  float hit;
};

template <typename T, bool kEntropy>
__device__ __forceinline__ float2 grad2(float2 x, const RowGrad& g) {
  float2 q = fma2(x, pair(g.inv_tau), pair(-g.lse));
  if (kEntropy) {              // exp(-150) is 0, and so is its product with any a + b q
    q.x = fmaxf(q.x, -150.0f);
    q.y = fmaxf(q.y, -150.0f);
  }
  const float2 u = fma2(q, pair(kLog2e), pair(g.rest2));
  const float2 e = make_float2(exp2_approx(u.x), exp2_approx(u.y));
  return kEntropy ? mul2(e, fma2(q, pair(g.b), pair(g.a))) : mul2(e, pair(g.a));
}

template <typename T, bool kEntropy>
__device__ __forceinline__ T grad1(T x, const RowGrad& g, bool hit) {
  const float d = grad2<T, kEntropy>(pair(to_f32(x)), g).x;
  return from_f32<T>(hit ? d + g.hit : d);
}

// The gradients of a vector whose first element is v0; t is the target.
template <typename T, bool kEntropy>
__device__ __forceinline__ uint4 grad_vec(const uint4& x, const RowGrad& g, int64_t v0, int64_t t) {
  constexpr int E = Vec16<T>::kElems;
  uint4 o;
  const int at = t >= v0 && t < v0 + E ? static_cast<int>(t - v0) : -1;
#pragma unroll
  for (int j = 0; j < Vec16<T>::kPairs; ++j) {
    float2 d = grad2<T, kEntropy>(unpack2(x, j, static_cast<const T*>(nullptr)), g);
    if (at >= 0) {
      if (at == 2 * j) d.x += g.hit;
      if (at == 2 * j + 1) d.y += g.hit;
    }
    pack2(o, j, d, static_cast<const T*>(nullptr));
  }
  return o;
}

// What a far row's rounded lse leaves out: the row's largest element and sum once more, by a warp
// or a CTA; the same in every thread, and none leaves before all have read the row.
template <typename T, bool kWarp>
__device__ __noinline__ float rest_of(const T* row, int64_t V, float c, float inv_tau, float lse) {
  RowSums a = kWarp ? scan_row<T, false, 1>(row, V, c, threadIdx.x & 31, 32, 0, 1)
                    : scan_row<T, false, 1>(row, V, c, threadIdx.x, kThreads, 0, 1);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) merge(a, shuffle(a, o), c);
  if (!kWarp) {
    __shared__ RowSums red[kThreads / 32];
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
    __syncthreads();
    a = red[threadIdx.x & (kThreads / 32 - 1)];
#pragma unroll
    for (int o = kThreads / 64; o > 0; o >>= 1) merge(a, shuffle(a, o), c);
  }
  return fmaf(a.m, inv_tau, -lse) + log2f(a.s) * kLn2;
}

// Part `part` of a row, by a warp or a CTA.
template <typename T, bool kEntropy, bool kWarp>
__device__ __forceinline__ void backward_row(const BackwardParams& p, int64_t r, int part) {
  constexpr int E = Vec16<T>::kElems;
  constexpr int n = kWarp ? 32 : kThreads;
  const int at = kWarp ? threadIdx.x & 31 : threadIdx.x;
  const T* row = static_cast<const T*>(p.x) + r * p.ld;
  T* out = static_cast<T*>(p.dx) + r * p.ld_d;
  const int64_t t = p.targets[r];
  const float w = p.d_logp != nullptr ? p.d_logp[r] : 0.0f;
  const float h = p.d_entropy != nullptr ? p.d_entropy[r] : 0.0f;
  const float l = p.lse[r];
  const bool nan = t >= p.V;
  const bool none = nan || t < 0 || (w == 0.0f && h == 0.0f) || l < kNoRow;
  float rest = 0.0f;
  int slices = p.slices;
  if (!none && fabsf(l) >= kFarLse) {
    // by the row's first CTA alone: d_logits may be the logits
    if (part != 0) return;
    slices = 1;
    rest = rest_of<T, kWarp>(row, p.V, p.c, p.inv_tau, l);
  }
  const int64_t head = head_of(out, p.V);
  const int64_t vecs = (p.V - head) / E;
  const int64_t per = (vecs + slices - 1) / slices;
  const int64_t first = per * part, last = min(vecs, first + per);
  const int64_t tail = head + vecs * E + at;
  uint4* body = reinterpret_cast<uint4*>(out + head);
  if (none) {
    const float f = nan ? __int_as_float(0x7fffffff) : 0.0f;
    if (nan && part == 0 && at == 0 && p.status != nullptr)
      atomicCAS(p.status, 0, BERGSON_EINVAL);
    uint4 v;
#pragma unroll
    for (int j = 0; j < Vec16<T>::kPairs; ++j) pack2(v, j, pair(f), static_cast<const T*>(nullptr));
    for (int64_t i = first + at; i < last; i += n) __stcs(body + i, v);
    if (part == 0) {
      if (at < head) out[at] = from_f32<T>(f);
      if (tail < p.V) out[tail] = from_f32<T>(f);
    }
    return;
  }
  RowGrad g;
  g.inv_tau = p.inv_tau;
  g.lse = l;
  g.rest2 = -kLog2e * rest;
  g.b = -h * p.inv_tau;
  g.a = fmaf(-g.b, rest, -(w + (kEntropy ? h * p.entropy[r] : 0.0f)) * p.inv_tau);
  g.hit = w * p.inv_tau;
  if (((reinterpret_cast<uintptr_t>(row + head)) & 15) == 0) {
    const uint4* in = reinterpret_cast<const uint4*>(row + head);
    for (int64_t i = first + at; i < last; i += kUnroll * n) {
      uint4 v[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (i + k * n < last) v[k] = __ldcs(in + i + k * n);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (i + k * n < last)
          __stcs(body + i + k * n, grad_vec<T, kEntropy>(v[k], g, head + (i + k * n) * E, t));
    }
  } else {
    // the rows of the two tensors start at different places within 16 bytes
    for (int64_t i = first + at; i < last; i += n) {
      uint4 o;
      const int64_t v0 = head + i * E;
      T* e = reinterpret_cast<T*>(&o);
#pragma unroll
      for (int k = 0; k < E; ++k) e[k] = grad1<T, kEntropy>(row[v0 + k], g, v0 + k == t);
      __stcs(body + i, o);
    }
  }
  if (part == 0) {
    if (at < head) out[at] = grad1<T, kEntropy>(row[at], g, at == t);
    if (tail < p.V) out[tail] = grad1<T, kEntropy>(row[tail], g, tail == t);
  }
}

template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kThreads, kBwdCtas) logprobs_backward_kernel(const BackwardParams p) {
  griddep_wait();
  backward_row<T, kEntropy, false>(p, blockIdx.x / p.slices,
                                   static_cast<int>(blockIdx.x % p.slices));
}

template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kThreads) logprobs_backward_warp_kernel(const BackwardParams p) {
  griddep_wait();
  const int64_t r = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  if (r < p.rows) backward_row<T, kEntropy, true>(p, r, 0);
}

// ------------------------------------------------------------------- host

// Rows of up to kWarpRowBytes go to warps, of up to kManyRowBytes where there are kManyRows.
// us by CTAs / by warps: 4096 x 4096 bf16 19.8 / 8.8, 8192 x 2000 fp32 31.0 / 14.5, but 1000 x
// 8000 bf16 8.6 / 9.2 and 2048 x 32,003 bf16 28.6 / 32.3.
constexpr int64_t kWarpRowBytes = 4096;
constexpr int64_t kManyRowBytes = 16384, kManyRows = 1216;
// Few rows are split over a cluster down to kPartBytes (1 / 100 rows of 131,072 bf16: 6.5 / 9.0
// us, 9.6 / 16.2 whole), the backward pass's always into slices (8192 x 65,536, us: 16 KB
// 254, 32 KB 238, 64 KB 239).
constexpr int64_t kPartBytes = 32768;
constexpr int64_t kSliceBytes = 32768;

bool rows_to_warps(int64_t rows, int64_t bytes) {
  return bytes <= (rows >= kManyRows ? kManyRowBytes : kWarpRowBytes);
}

template <typename T, bool kEntropy>
cudaError_t run_forward(const LogprobArgs& a, cudaStream_t s) {
  const ForwardParams p{a.x, a.rows, a.V, a.ld, a.targets, static_cast<float>(1.0 / a.tau),
                        static_cast<float>(1.4426950408889634 / a.tau), a.logp, a.lse, a.entropy,
                        a.status};
  const int64_t bytes = a.V * static_cast<int64_t>(sizeof(T));
  if (rows_to_warps(a.rows, bytes)) {
    const int64_t grid = (a.rows + kThreads / 32 - 1) / (kThreads / 32);
    return launch_dependent(logprobs_warp_kernel<T, kEntropy>, dim3(static_cast<unsigned>(grid)),
                            dim3(kThreads), 0, s, p);
  }
  // Few rows: the CTAs of a cluster share one.
  int parts = 1;
  while (parts < 8 && a.rows * parts < 2 * kPlanCTAs && bytes / parts >= kPartBytes) parts *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.rows * parts));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = parts;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, logprobs_row_kernel<T, kEntropy>, p);
}

template <typename T, bool kEntropy>
cudaError_t run_backward(const LogprobGradArgs& a, cudaStream_t s) {
  BackwardParams p{a.x, a.rows, a.V, a.ld, a.targets, static_cast<float>(1.0 / a.tau),
                   static_cast<float>(1.4426950408889634 / a.tau), a.lse, a.entropy, a.d_logp,
                   a.d_entropy, a.dx, a.ld_d, 1, a.status};
  const int64_t bytes = a.V * static_cast<int64_t>(sizeof(T));
  if (rows_to_warps(a.rows, bytes)) {
    const int64_t grid = (a.rows + kThreads / 32 - 1) / (kThreads / 32);
    return launch_dependent(logprobs_backward_warp_kernel<T, kEntropy>,
                            dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, s, p);
  }
  const int64_t slices = (bytes + kSliceBytes - 1) / kSliceBytes;
  p.slices = static_cast<int>(slices * a.rows < INT32_MAX ? slices : 1);
  return launch_dependent(logprobs_backward_kernel<T, kEntropy>,
                          dim3(static_cast<unsigned>(a.rows * p.slices)), dim3(kThreads), 0, s, p);
}

template <typename T>
cudaError_t run_forward(const LogprobArgs& a, cudaStream_t s) {
  return a.entropy != nullptr ? run_forward<T, true>(a, s) : run_forward<T, false>(a, s);
}
template <typename T>
cudaError_t run_backward(const LogprobGradArgs& a, cudaStream_t s) {
  return a.d_entropy != nullptr ? run_backward<T, true>(a, s) : run_backward<T, false>(a, s);
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
