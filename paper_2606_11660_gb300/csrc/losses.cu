// The clipped policy loss and the preference loss, forward and backward: one
// pass over the tokens, whose gradients follow from their own values and a weight.

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kSegment = 512;                  // tokens of a row a warp takes at once

// ---------------------------------------------------------------- policy

struct PolicyParams {
  bergson_policy_args a;
  int64_t segments;            // per row
  unsigned* counts;            // valid tokens: per row
  float4* sums;                // [B, segments] of l, k, clipped, valid tokens
  float low, high, kl, ent;
};

__global__ void __launch_bounds__(kThreads) policy_count_kernel(const PolicyParams p) {
  const int64_t b = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (b >= p.a.B) return;
  const uint8_t* row = p.a.mask + b * p.a.ld_mask;
  unsigned n = 0;
  for (int64_t t = threadIdx.x & 31; t < p.a.T; t += 32) n += row[t] != 0;
  n = __reduce_add_sync(0xffffffffu, n);
  if ((threadIdx.x & 31) == 0) p.counts[b] = n;
}

__device__ __forceinline__ double policy_weight(const PolicyParams& p, int64_t b, double total) {
  switch (p.a.reduction) {
    case BERGSON_POLICY_TOKEN_MEAN: return 1.0 / fmax(total, 1.0);
    case BERGSON_POLICY_SEQ_MEAN: {
      const double n = p.a.mask != nullptr ? p.counts[b] : p.a.T;
      return 1.0 / (p.a.B * fmax(n, 1.0));
    }
    default: return 1.0 / (p.a.B * p.a.norm_tokens);
  }
}

// Valid tokens of the batch, in every thread.
__device__ __forceinline__ double policy_total(const PolicyParams& p, double* red) {
  if (p.a.mask == nullptr) return static_cast<double>(p.a.B) * p.a.T;
  double n = 0.0;
  for (int64_t b = threadIdx.x; b < p.a.B; b += blockDim.x) n += p.counts[b];
  return block_sum(n, red);
}

__global__ void __launch_bounds__(kThreads) policy_kernel(const PolicyParams p) {
  __shared__ double red[kWarps];
  const double total =
      p.a.reduction == BERGSON_POLICY_TOKEN_MEAN ? policy_total(p, red) : 0.0;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (item >= p.a.B * p.segments) return;
  const int64_t b = item / p.segments, seg = item % p.segments;
  const float w = static_cast<float>(policy_weight(p, b, total));
  const int64_t end = min(p.a.T, (seg + 1) * kSegment);
  float loss = 0.0f, kls = 0.0f, clipped = 0.0f, valid = 0.0f;
  for (int64_t t = seg * kSegment + (threadIdx.x & 31); t < end; t += 32) {
    const bool on = p.a.mask == nullptr || p.a.mask[b * p.a.ld_mask + t] != 0;
    float grad = 0.0f, l = 0.0f;
    if (on) {
      const float lp = p.a.logp[b * p.a.ld_logp + t];
      const float adv = p.a.advantages[p.a.ld_adv == 0 ? b : b * p.a.ld_adv + t];
      const float ratio = expf(lp - p.a.old_logp[b * p.a.ld_old + t]);
      const float free = ratio * adv;
      const float held = fminf(fmaxf(ratio, p.low), p.high) * adv;
      const bool clip = free > held;
      l = clip ? -held : -free;
      grad = clip ? 0.0f : -free;
      if (p.a.ref_logp != nullptr) {
        const float gap = p.a.ref_logp[b * p.a.ld_ref + t] - lp;
        const float up = expm1f(gap);
        const float k = up - gap;
        l += p.kl * k;
        grad -= p.kl * up;
        kls += k;
      }
      if (p.a.entropy != nullptr) l -= p.ent * p.a.entropy[b * p.a.ld_entropy + t];
      loss += l;
      clipped += clip ? 1.0f : 0.0f;
      valid += 1.0f;
    }
    p.a.d_logp[b * p.a.ld_d + t] = on ? w * grad : 0.0f;
    if (p.a.d_entropy != nullptr) p.a.d_entropy[b * p.a.ld_de + t] = on ? -w * p.ent : 0.0f;
  }
  loss = warp_sum(loss);
  kls = warp_sum(kls);
  clipped = warp_sum(clipped);
  valid = warp_sum(valid);
  if ((threadIdx.x & 31) == 0) p.sums[item] = make_float4(loss, kls, clipped, valid);
}

__global__ void __launch_bounds__(1024) policy_finish_kernel(const PolicyParams p) {
  __shared__ double red[32];
  const double total =
      p.a.reduction == BERGSON_POLICY_TOKEN_MEAN ? policy_total(p, red) : 0.0;
  double loss = 0.0, kl = 0.0, clipped = 0.0, valid = 0.0;
  for (int64_t b = threadIdx.x; b < p.a.B; b += blockDim.x) {
    double l = 0.0;
    for (int64_t i = b * p.segments; i < (b + 1) * p.segments; ++i) {
      const float4 v = p.sums[i];
      l += v.x;
      kl += v.y;
      clipped += v.z;
      valid += v.w;
    }
    l *= policy_weight(p, b, total);
    if (p.a.seq_loss != nullptr) p.a.seq_loss[b] = static_cast<float>(l);
    loss += l;
  }
  loss = block_sum(loss, red);
  kl = block_sum(kl, red);
  clipped = block_sum(clipped, red);
  valid = block_sum(valid, red);
  if (threadIdx.x == 0) {
    *p.a.loss = static_cast<float>(loss);
    if (p.a.stats != nullptr) {
      p.a.stats[0] = static_cast<float>(kl / fmax(valid, 1.0));
      p.a.stats[1] = static_cast<float>(clipped / fmax(valid, 1.0));
      p.a.stats[2] = static_cast<float>(valid);
    }
  }
}

// ------------------------------------------------------------ preference

struct PreferenceParams {
  bergson_preference_args a;
};

// f(x) and its slope.
__device__ __forceinline__ void preference_f(int kind, float x, float beta, float* f, float* df) {
  if (kind == BERGSON_PREFERENCE_SIGMOID) {
    const float e = expf(-fabsf(x));
    *f = fmaxf(-x, 0.0f) + log1pf(e);
    *df = -(x >= 0.0f ? e : 1.0f) / (1.0f + e);
  } else if (kind == BERGSON_PREFERENCE_HINGE) {
    *f = fmaxf(1.0f - x, 0.0f);
    *df = x < 1.0f ? -1.0f : 0.0f;
    if (x != x) *f = *df = x;
  } else {
    const float y = (x - 0.5f) / beta;
    *f = y * y;
    *df = 2.0f * y / beta;
  }
}

__global__ void __launch_bounds__(kThreads) preference_kernel(const PreferenceParams p) {
  __shared__ double red[kWarps];
  const int64_t pair = blockIdx.x;
  double s[2], n[2];
  for (int side = 0; side < 2; ++side) {
    const int64_t r = pair + side * p.a.P;
    float sum = 0.0f, count = 0.0f;
    for (int64_t t = threadIdx.x; t < p.a.T; t += kThreads) {
      if (p.a.mask != nullptr && p.a.mask[r * p.a.ld_mask + t] == 0) continue;
      float v = p.a.logp[r * p.a.ld_logp + t];
      if (p.a.ref_logp != nullptr) v -= p.a.ref_logp[r * p.a.ld_ref + t];
      sum += v;
      count += 1.0f;
    }
    s[side] = block_sum(static_cast<double>(sum), red);
    n[side] = p.a.mean_logp ? fmax(block_sum(static_cast<double>(count), red), 1.0) : 1.0;
    s[side] /= n[side];
  }
  const float beta = static_cast<float>(p.a.beta);
  const float x = static_cast<float>(p.a.beta * (s[0] - s[1]) - p.a.margin);
  const float eps = static_cast<float>(p.a.label_smoothing);
  float f, df, g, dg;
  preference_f(p.a.kind, x, beta, &f, &df);
  preference_f(p.a.kind, -x, beta, &g, &dg);
  // a side of weight 0 takes no part, even where it is infinite
  const float loss = (eps < 1.0f ? (1.0f - eps) * f : 0.0f) + (eps > 0.0f ? eps * g : 0.0f);
  const float slope = (eps < 1.0f ? (1.0f - eps) * df : 0.0f) - (eps > 0.0f ? eps * dg : 0.0f);
  if (threadIdx.x == 0) {
    p.a.pair_loss[pair] = loss;
    if (p.a.rewards != nullptr) {
      p.a.rewards[pair] = static_cast<float>(p.a.beta * s[0]);
      p.a.rewards[pair + p.a.P] = static_cast<float>(p.a.beta * s[1]);
    }
  }
  for (int side = 0; side < 2; ++side) {
    const int64_t r = pair + side * p.a.P;
    const float d = static_cast<float>((side ? -1.0 : 1.0) * slope * p.a.beta /
                                       (static_cast<double>(p.a.P) * n[side]));
    for (int64_t t = threadIdx.x; t < p.a.T; t += kThreads) {
      const bool on = p.a.mask == nullptr || p.a.mask[r * p.a.ld_mask + t] != 0;
      p.a.d_logp[r * p.a.ld_d + t] = on ? d : 0.0f;
    }
  }
}

__global__ void __launch_bounds__(1024) preference_finish_kernel(const float* pair_loss,
                                                                 int64_t P, float* loss) {
  __shared__ double red[32];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < P; i += blockDim.x) s += pair_loss[i];
  s = block_sum(s, red);
  if (threadIdx.x == 0) *loss = P > 0 ? static_cast<float>(s / static_cast<double>(P)) : 0.0f;
}

int64_t segments_of(int64_t T) { return (T + kSegment - 1) / kSegment; }

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t policy_workspace(int64_t B, int64_t T) {
  return 256 + align256(4 * static_cast<size_t>(B)) +
         align256(16 * static_cast<size_t>(B) * static_cast<size_t>(segments_of(T)));
}

cudaError_t launch_policy_loss(const bergson_policy_args& a, void* ws, cudaStream_t s) {
  PolicyParams p;
  p.a = a;
  p.segments = segments_of(a.T);
  p.counts = static_cast<unsigned*>(ws);
  p.sums = reinterpret_cast<float4*>(static_cast<char*>(ws) +
                                     align256(4 * static_cast<size_t>(a.B)));
  p.low = static_cast<float>(1.0 - a.clip_low);
  p.high = static_cast<float>(1.0 + a.clip_high);
  p.kl = static_cast<float>(a.kl_coef);
  p.ent = static_cast<float>(a.entropy_coef);
  if (a.kl_coef == 0.0) p.a.ref_logp = nullptr;
  if (a.entropy_coef == 0.0) p.a.entropy = nullptr;
  const int64_t items = a.B * p.segments;
  if (items > 0) {
    if (a.mask != nullptr && a.reduction != BERGSON_POLICY_SUM_NORM)
      policy_count_kernel<<<static_cast<unsigned>((a.B + kWarps - 1) / kWarps), kThreads, 0, s>>>(p);
    policy_kernel<<<static_cast<unsigned>((items + kWarps - 1) / kWarps), kThreads, 0, s>>>(p);
  } else {
    // nothing reads the counts of a batch without tokens: every loss is 0
    p.a.mask = nullptr;
  }
  policy_finish_kernel<<<1, 1024, 0, s>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_preference_loss(const bergson_preference_args& a, int, cudaStream_t s) {
  PreferenceParams p;
  p.a = a;
  if (a.P > 0) preference_kernel<<<static_cast<unsigned>(a.P), kThreads, 0, s>>>(p);
  preference_finish_kernel<<<1, 1024, 0, s>>>(a.pair_loss, a.P, a.loss);
  return cudaGetLastError();
}

}  // namespace bergson
