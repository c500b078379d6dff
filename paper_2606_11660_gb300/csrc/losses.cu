// The clipped policy loss and the preference loss, forward and backward.
//
// Both read every valid token once and write its gradient: 4 bytes a tensor and one of
// mask, some 30 operations, so they are bound by memory, and below some 10^5 tokens by
// their launches.  A token's gradient needs a weight that depends on others: the
// policy loss counts the valid tokens beforehand (a byte a token), the preference
// loss holds a pair in a CTA (or a cluster that shares its sums) and comes back to
// write.  Sums over tokens follow an order fixed by the sizes, the leading dimensions and the
// tensors' alignment.
//
// Policy loss of 2048 x 16,384 tokens, KL and entropy terms, a token mean: 123 us (the
// count 10, the tokens 109, the finish 8), 6.8 TB/s of the 25 bytes a token; masked
// tokens' inputs are not read, and of what moves with 54% of them valid it is 0.72 of
// the copy rate.  Preference loss of 256 pairs of 32,768 tokens without a reference: 29 us, 0.77
// of 9 bytes a token at the copy rate and 0.61 of what moves; what is left are the two
// phases' latencies with a pair's CTAs in step.

#include <algorithm>

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// ------------------------------------------------ several tokens of a row a lane
//
// A warp takes 32 N tokens of a row at a time, N (4 or 8) a lane: neighbours in one
// load where the rows allow it (kVec), else 32 apart in loads of one.  Their mask
// bytes stay in words; tokens outside the row have mask 0.  Masked tokens are not read
// (in a vector, where all of it is masked).
//
// Rows of any length start off a vector's boundary, but where the tensors' bases are
// aligned and their leading dimensions the same modulo N, row b of each of them starts
// s = b ld mod N elements past one.  A row is then taken from token -s on.

template <int N>
struct Mask {
  uint32_t w[N / 4];
  __device__ __forceinline__ bool on(int j) const {
    return (w[j / 4] & (0xffu << (8 * (j % 4)))) != 0;
  }
  __device__ __forceinline__ bool any() const {
    return N == 4 ? w[0] != 0 : (w[0] | w[N / 4 - 1]) != 0;
  }
  __device__ __forceinline__ int count() const {
    int c = 0;
#pragma unroll
    for (int k = 0; k < N / 4; ++k)
      c += __popc((w[k] | ((w[k] & 0x7f7f7f7fu) + 0x7f7f7f7fu)) & 0x80808080u);
    return c;
  }
};

template <int N, bool kVec>
__device__ __forceinline__ int token_of(int t0, int j) {
  const int lane = threadIdx.x & 31;
  return kVec ? t0 + N * lane + j : t0 + lane + 32 * j;
}
// Whether all of a lane's tokens lie in [0, T), and in one vector.
template <int N, bool kVec>
__device__ __forceinline__ bool whole(int t0, int T) {
  return kVec && token_of<N, kVec>(t0, 0) >= 0 && token_of<N, kVec>(t0, N - 1) < T;
}
// How far past a vector's boundary row b starts.
template <int N, bool kVec>
__device__ __forceinline__ int shift_of(int64_t b, int64_t ld) {
  return kVec ? static_cast<int>((b * ld) & (N - 1)) : 0;
}

template <int N, bool kVec>
__device__ __forceinline__ Mask<N> load_mask(const uint8_t* mask, int t0, int T) {
  Mask<N> m;
  if (whole<N, kVec>(t0, T)) {
    if (mask == nullptr) {
#pragma unroll
      for (int k = 0; k < N / 4; ++k) m.w[k] = 0x01010101u;
    } else if constexpr (N == 8) {
      const uint2 u = *reinterpret_cast<const uint2*>(mask + token_of<N, kVec>(t0, 0));
      m.w[0] = u.x;
      m.w[1] = u.y;
    } else {
      m.w[0] = *reinterpret_cast<const uint32_t*>(mask + token_of<N, kVec>(t0, 0));
    }
    return m;
  }
#pragma unroll
  for (int k = 0; k < N / 4; ++k) m.w[k] = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int t = token_of<N, kVec>(t0, j);
    if (t >= 0 && t < T)
      m.w[j / 4] |= (mask == nullptr ? 1u : static_cast<uint32_t>(mask[t])) << (8 * (j % 4));
  }
  return m;
}

// The values of the tokens that are on (others: anything).
template <int N, bool kVec>
__device__ __forceinline__ void load_tokens(const float* row, int t0, int T, const Mask<N>& m,
                                            float (&x)[N]) {
  if (whole<N, kVec>(t0, T)) {
    if (!m.any()) return;
    const float* at = row + token_of<N, kVec>(t0, 0);
    if constexpr (N == 8) {
      uint32_t r[8];
      load32(at, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(r[j]);
    } else {
      const float4 f = __ldcs(reinterpret_cast<const float4*>(at));
      x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (m.on(j)) x[j] = __ldcs(row + token_of<N, kVec>(t0, j));
}

template <int N, bool kVec>
__device__ __forceinline__ void store_tokens(float* row, int t0, int T, const float (&x)[N]) {
  if (whole<N, kVec>(t0, T)) {
    float* at = row + token_of<N, kVec>(t0, 0);
    if constexpr (N == 8) {
      uint32_t r[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] = __float_as_uint(x[j]);
      store32(at, r);
    } else {
      __stcs(reinterpret_cast<float4*>(at), make_float4(x[0], x[1], x[2], x[3]));
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int t = token_of<N, kVec>(t0, j);
    if (t >= 0 && t < T) __stcs(row + t, x[j]);
  }
}

// Nonzero bytes among n from p, counted by a warp (the sum is in every lane).
__device__ __forceinline__ unsigned count_bytes(const uint8_t* p, int64_t n) {
  const int lane = threadIdx.x & 31;
  int64_t head = (16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15;
  head = head < n ? head : n;
  const int64_t vecs = (n - head) / 16;
  const uint4* body = reinterpret_cast<const uint4*>(p + head);
  unsigned c = 0;
  for (int64_t i = lane; i < vecs; i += 4 * 32) {
    uint4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = i + 32 * j < vecs ? body[i + 32 * j] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t w = word(v[j], k);
        c += __popc((w | ((w & 0x7f7f7f7fu) + 0x7f7f7f7fu)) & 0x80808080u);
      }
    }
  }
  const int64_t tail = head + 16 * vecs + lane;
  if (lane < head) c += p[lane] != 0;
  if (tail < n) c += p[tail] != 0;
  return __reduce_add_sync(0xffffffffu, c);
}

// ---------------------------------------------------------------- policy

// Tokens of a row a warp takes: the longer ones where there is one for every resident
// warp.  us at 1024 / 256: 32 x 32,768 tokens 15.9 / 13.5, 512 x 4000 20.3 / 17.6,
// 2048 x 4096 39.8 / 42.1, 2048 x 16,384 (without entropies) 103 / 128.
constexpr int kSegment = 1024, kShortSegment = 256;
constexpr int64_t kLongItems = 152 * 32;
constexpr int kCountSegment = 4096;            // mask bytes a warp counts at once
constexpr int kCountCtas = 1216;
constexpr int kPolicyPerSm = 4;                // CTAs an SM holds (123 us; 3: 129, 5: 126)
constexpr int kFinishCtas = 152;
// The one-launch form: at most so many segments of the shorter kind.  us in one launch / in
// three: 8 x 97 tokens 9.1 / 12.9, 64 x 1000 10.1 / 13.5; of 512 segments, 64 x 2000, 17.6 / 12.9.
constexpr int kSmallItems = 256;
constexpr int kSmallThreads = 512, kSmallWarps = kSmallThreads / 32;
constexpr int kSmallCount = 2048;              // mask bytes a warp counts at once there

struct Totals {
  Sum2 loss, kl;
  unsigned long long clipped = 0, valid = 0;
  __device__ __forceinline__ void add(const float4& v) {  // a segment's sums
    loss.add(v.x);
    kl.add(v.y);
    clipped += static_cast<unsigned>(v.z);
    valid += static_cast<unsigned>(v.w);
  }
  __device__ __forceinline__ void add(const Totals& o) {
    loss.add(o.loss);
    kl.add(o.kl);
    clipped += o.clipped;
    valid += o.valid;
  }
};
__device__ __forceinline__ Totals totals_sum(const Totals& t) {
  Totals r;
  r.loss = warp_sum(t.loss);
  r.kl = warp_sum(t.kl);
  r.clipped = warp_sum(t.clipped);
  r.valid = warp_sum(t.valid);
  return r;
}

struct PolicyParams {
  bergson_policy_args a;
  int segment;                                 // tokens of a row a warp takes
  int64_t segments, count_segments;            // per row
  unsigned* counts;            // valid tokens: per CTA (TOKEN_MEAN) or [B, count_segments]
  int n_counts;                // CTAs that counted (TOKEN_MEAN), a multiple of 4
  float4* sums;                // [B, segments] of l, k, clipped, valid tokens
  Totals* totals;              // [kFinishCtas] of the same, l weighed
  unsigned* ticket;
  float low, high, kl, ent;
  float norm;                  // 1 / (B norm_tokens) (SUM_NORM)
};

__global__ void __launch_bounds__(kThreads) policy_count_kernel(const PolicyParams p) {
  __shared__ unsigned red[kWarps];
  griddep_wait();
  const int64_t items = p.a.B * p.count_segments;
  const int64_t warps = static_cast<int64_t>(gridDim.x) * kWarps;
  unsigned mine = 0;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); i < items;
       i += warps) {
    const int64_t b = i / p.count_segments, t = (i % p.count_segments) * kCountSegment;
    const int64_t n = min(p.a.T - t, static_cast<int64_t>(kCountSegment));
    const unsigned c = count_bytes(p.a.mask + b * p.a.ld_mask + t, n);
    if (p.a.reduction == BERGSON_POLICY_SEQ_MEAN) {
      if ((threadIdx.x & 31) == 0) p.counts[i] = c;
    }
    mine += c;
  }
  if (p.a.reduction != BERGSON_POLICY_TOKEN_MEAN) return;
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned c = 0;                            // 2^40 tokens over 1216 CTAs fit 32 bits
    for (int w = 0; w < kWarps; ++w) c += red[w];
    p.counts[blockIdx.x] = c;
  }
}

// The token weight where the batch (TOKEN_MEAN) or the row (SEQ_MEAN) has n valid tokens.
__device__ __forceinline__ float weight_of(const PolicyParams& p, unsigned long long n) {
  if (p.a.reduction == BERGSON_POLICY_SUM_NORM) return p.norm;
  n = n > 1 ? n : 1;
  if (p.a.reduction == BERGSON_POLICY_SEQ_MEAN) n *= static_cast<unsigned long long>(p.a.B);
  return 1.0f / static_cast<float>(n);
}

// What the counts before say: of the batch, and of row b, in every lane of a warp.
__device__ __forceinline__ unsigned long long counted_batch(const PolicyParams& p) {
  if (p.a.reduction != BERGSON_POLICY_TOKEN_MEAN) return 0;
  if (p.a.mask == nullptr) return static_cast<unsigned long long>(p.a.B) * p.a.T;
  unsigned long long n = 0;
  const uint4* counts = reinterpret_cast<const uint4*>(p.counts);
#pragma unroll 4
  for (int i = threadIdx.x & 31; i < p.n_counts / 4; i += 32) {
    const uint4 c = counts[i];
    n += static_cast<unsigned long long>(c.x) + c.y + c.z + c.w;
  }
  return warp_sum(n);
}
__device__ __forceinline__ unsigned long long counted_row(const PolicyParams& p, int64_t b) {
  if (p.a.mask == nullptr) return static_cast<unsigned long long>(p.a.T);
  unsigned long long n = 0;
  if (p.count_segments <= 8) {
    for (int i = 0; i < static_cast<int>(p.count_segments); ++i)
      n += p.counts[b * p.count_segments + i];
    return n;
  }
  for (int64_t i = threadIdx.x & 31; i < p.count_segments; i += 32)
    n += p.counts[b * p.count_segments + i];
  return warp_sum(n);
}
__device__ __forceinline__ float counted_weight(const PolicyParams& p, unsigned long long batch,
                                                int64_t b) {
  return weight_of(p, p.a.reduction == BERGSON_POLICY_SEQ_MEAN ? counted_row(p, b) : batch);
}

// up = exp(g) - 1 and k = up - g.  Below 1/4 by the series of k = g^2 (1/2 + g/6 + ...),
// where the difference would cancel (six terms: 2^-24 of up); above, exp's 2 units of error are at
// most 5e-7 of exp(g) and 1e-5 of k, at any gap (a base-2 exponential of the rounded g log2(e)
// would lose |g| units: 2e-6 at 30).
__device__ __forceinline__ void kl_of(float g, float* k, float* up) {
  float s = fmaf(g, 1.0f / 5040.0f, 1.0f / 720.0f);
  s = fmaf(g, s, 1.0f / 120.0f);
  s = fmaf(g, s, 1.0f / 24.0f);
  s = fmaf(g, s, 1.0f / 6.0f);
  s = fmaf(g, s, 0.5f);
  s *= g * g;
  const float e = expf(g) - 1.0f;
  const bool small = fabsf(g) < 0.25f;
  *k = small ? s : e - g;
  *up = small ? s + g : e;
}

// A warp takes a segment of row b with token weight w; the segment's sums are in every lane.
template <bool kVec>
__device__ __forceinline__ float4 policy_segment(const PolicyParams& p, int64_t b, int seg,
                                                 float w) {
  const int T = static_cast<int>(p.a.T);
  const uint8_t* mask = p.a.mask == nullptr ? nullptr : p.a.mask + b * p.a.ld_mask;
  const bool by_token = p.a.ld_adv != 0;
  const float adv_row = by_token ? 0.0f : p.a.advantages[b];
  const float minus_we = -w * p.ent;
  float loss = 0.0f, kls = 0.0f;
  int clipped = 0, valid = 0;
  int t0 = seg * p.segment - shift_of<4, kVec>(b, p.a.ld_logp);
  Mask<4> next = load_mask<4, kVec>(mask, t0, T);
#pragma unroll 1
  for (int left = min(T - t0, p.segment); left > 0; left -= 128, t0 += 128) {
    const Mask<4> m = next;
    if (left > 128) next = load_mask<4, kVec>(mask, t0 + 128, T);
    float lp[4], old[4], adv[4], ref[4], ent[4], d[4], dh[4];
    load_tokens<4, kVec>(p.a.logp + b * p.a.ld_logp, t0, T, m, lp);
    load_tokens<4, kVec>(p.a.old_logp + b * p.a.ld_old, t0, T, m, old);
    if (p.a.ref_logp != nullptr)
      load_tokens<4, kVec>(p.a.ref_logp + b * p.a.ld_ref, t0, T, m, ref);
    if (p.a.entropy != nullptr)
      load_tokens<4, kVec>(p.a.entropy + b * p.a.ld_entropy, t0, T, m, ent);
    if (by_token) load_tokens<4, kVec>(p.a.advantages + b * p.a.ld_adv, t0, T, m, adv);
    valid += m.count();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      d[j] = dh[j] = 0.0f;
      if (!m.on(j)) continue;
      const float a = by_token ? adv[j] : adv_row;
      const float ratio = expf(lp[j] - old[j]);
      const float free = ratio * a;
      const float held = fminf(fmaxf(ratio, p.low), p.high) * a;
      const bool clip = free > held;
      float l = clip ? -held : -free;
      float grad = clip ? 0.0f : -free;
      if (p.a.ref_logp != nullptr) {
        float k, up;
        kl_of(ref[j] - lp[j], &k, &up);
        kls += k;
        if (p.kl != 0.0f) {                    // 0: k is watched alone, also where it is infinite
          l = fmaf(p.kl, k, l);
          grad = fmaf(-p.kl, up, grad);
        }
      }
      if (p.a.entropy != nullptr) l = fmaf(-p.ent, ent[j], l);
      loss += l;
      clipped += clip ? 1 : 0;
      d[j] = w * grad;
      dh[j] = minus_we;
    }
    store_tokens<4, kVec>(p.a.d_logp + b * p.a.ld_d, t0, T, d);
    if (p.a.d_entropy != nullptr)
      store_tokens<4, kVec>(p.a.d_entropy + b * p.a.ld_de, t0, T, dh);
  }
  return make_float4(warp_sum(loss), warp_sum(kls),
                     static_cast<float>(__reduce_add_sync(0xffffffffu, clipped)),
                     static_cast<float>(__reduce_add_sync(0xffffffffu, valid)));
}

__device__ __forceinline__ void write_stats(const PolicyParams& p, const Totals& t) {
  *p.a.loss = t.loss.value();
  if (p.a.stats == nullptr) return;
  const float n = static_cast<float>(t.valid > 1 ? t.valid : 1);
  p.a.stats[0] = t.kl.value() / n;
  p.a.stats[1] = static_cast<float>(t.clipped) / n;
  p.a.stats[2] = static_cast<float>(t.valid);
}

// A warp's sums over the segments of row b, as `part`(i) gives them.
template <typename F>
__device__ __forceinline__ Totals row_totals(int64_t segments, F part) {
  Totals r;
  for (int64_t i = threadIdx.x & 31; i < segments; i += 32) r.add(part(i));
  return totals_sum(r);
}

template <bool kVec>
__global__ void __launch_bounds__(kThreads, kPolicyPerSm) policy_kernel(const PolicyParams p) {
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  griddep_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.ticket = 0;      // for the grid after this one
  if (item >= p.a.B * p.segments) return;
  const int64_t b = item / p.segments;
  const float4 s = policy_segment<kVec>(p, b, static_cast<int>(item - b * p.segments),
                                        counted_weight(p, counted_batch(p), b));
  if ((threadIdx.x & 31) == 0) p.sums[item] = s;
}

// Rows' losses, a warp each; the last CTA to finish adds the CTAs' totals in order.
__global__ void __launch_bounds__(kThreads) policy_finish_kernel(const PolicyParams p) {
  __shared__ Totals red[kWarps];
  __shared__ bool last;
  const int lane = threadIdx.x & 31;
  griddep_wait();
  const unsigned long long batch = counted_batch(p);
  Totals t;
  for (int64_t b = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); b < p.a.B;
       b += static_cast<int64_t>(gridDim.x) * kWarps) {
    Totals r = row_totals(p.segments, [&](int64_t i) { return p.sums[b * p.segments + i]; });
    const float l = r.loss.value() * counted_weight(p, batch, b);
    if (p.a.seq_loss != nullptr && lane == 0) p.a.seq_loss[b] = l;
    r.loss = Sum2();
    r.loss.add(l);
    t.add(r);
  }
  if (lane == 0) red[threadIdx.x >> 5] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    t = red[0];
    for (int w = 1; w < kWarps; ++w) t.add(red[w]);
    p.totals[blockIdx.x] = t;
    __threadfence();
    last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last || threadIdx.x >= 32) return;
  __threadfence();
  t = Totals();
  for (int i = lane; i < static_cast<int>(gridDim.x); i += 32) t.add(p.totals[i]);
  t = totals_sum(t);
  if (lane == 0) write_stats(p, t);
}

// The whole of a small batch in one cluster: the CTAs count the rows' valid tokens together,
// each takes its share of the segments and leaves their sums with the first, which finishes.
template <bool kVec>
__global__ void __launch_bounds__(kSmallThreads) policy_small_kernel(const PolicyParams p) {
  __shared__ unsigned counts[kSmallItems];               // per row
  __shared__ float4 sums[kSmallItems];
  __shared__ Totals red[kSmallWarps];
  const int parts = static_cast<int>(cluster_size()), rank = static_cast<int>(blockIdx.x);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int B = static_cast<int>(p.a.B), T = static_cast<int>(p.a.T);
  const int segments = static_cast<int>(p.segments);
  const bool counted = p.a.reduction != BERGSON_POLICY_SUM_NORM;
  for (int b = threadIdx.x; b < B; b += kSmallThreads)
    counts[b] = p.a.mask == nullptr ? static_cast<unsigned>(T) : 0u;
  cluster_barrier();                                        // every CTA has started, with zeros
  griddep_wait();
  unsigned total = 0;
  if (counted) {
    if (p.a.mask != nullptr) {
      const int per = (T + kSmallCount - 1) / kSmallCount;
      for (int i = rank * kSmallWarps + warp; i < B * per; i += parts * kSmallWarps) {
        const int b = i / per, t = (i - b * per) * kSmallCount;
        const unsigned c =
            count_bytes(p.a.mask + b * p.a.ld_mask + t, min(T - t, kSmallCount));
        if (lane < parts) add_cluster(&counts[b], lane, c);
      }
      cluster_barrier();
    }
    if (p.a.reduction == BERGSON_POLICY_TOKEN_MEAN) {
      for (int b = lane; b < B; b += 32) total += counts[b];
      total = __reduce_add_sync(0xffffffffu, total);
    }
  }
  const auto weight = [&](int b) {
    return weight_of(p, p.a.reduction == BERGSON_POLICY_SEQ_MEAN ? counts[b] : total);
  };
  for (int i = rank * kSmallWarps + warp; i < B * segments; i += parts * kSmallWarps) {
    const int b = i / segments;
    const float4 s = policy_segment<kVec>(p, b, i - b * segments, weight(b));
    if (lane < 4) {
      const float x = lane == 0 ? s.x : lane == 1 ? s.y : lane == 2 ? s.z : s.w;
      st_cluster(reinterpret_cast<float*>(&sums[i]) + lane, 0, x);
    }
  }
  cluster_barrier();
  if (rank != 0) return;
  Totals t;
  const auto take_row = [&](int b, Totals r) {
    const float x = r.loss.value() * weight(b);
    if (p.a.seq_loss != nullptr) p.a.seq_loss[b] = x;
    r.loss = Sum2();
    r.loss.add(x);
    t.add(r);
  };
  if (segments <= 4) {                                   // a row a thread
    for (int b = threadIdx.x; b < B; b += kSmallThreads) {
      Totals r;
      for (int i = b * segments; i < (b + 1) * segments; ++i) r.add(sums[i]);
      take_row(b, r);
    }
  } else {                                               // a row a warp
    for (int b = warp; b < B; b += kSmallWarps) {
      const Totals r = row_totals(segments, [&](int64_t i) { return sums[b * segments + i]; });
      if (lane == 0) take_row(b, r);
    }
  }
  t = totals_sum(t);
  if (lane == 0) red[warp] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    t = red[0];
    for (int w = 1; w < kSmallWarps; ++w) t.add(red[w]);
    write_stats(p, t);
  }
}

// ------------------------------------------------------------ preference

constexpr int kPairThreads = 256;
constexpr int kPairWarps = kPairThreads / 32;
constexpr int kPairPerSm = 5, kPairPerSmRef = 4;
// A pair is split, into shares of more than half of kPairTokens, up to kPairCtas CTAs an SM:
// 1 / 32 pairs of 32,768 tokens split 11.0 / 10.9 us, whole 17.4 / 18.2; more shares wait
// longer for each other (256 pairs in 8 shares each 37 us, in 2 33).
constexpr int kPairCtas = 2;
constexpr int64_t kPairTokens = 2048;

// From kManyPairs on, pairs of up to kShortPair tokens go to a warp each: 2048 of 100 / 600 /
// 1000 tokens 7.8 / 9.4 / 13.4 us, to a CTA each 15.6 / 22.1 / 23.6; 700 of 1000 9.2 and 11.9,
// of 2000 13.8 and 12.1.
constexpr int64_t kManyPairs = 608;
constexpr int64_t kShortPair = 1024;

struct PreferenceParams {
  bergson_preference_args a;
};

// f(x) and its slope.
__device__ __forceinline__ void preference_f(int kind, float x, float beta, float* f, float* df) {
  if (kind == BERGSON_PREFERENCE_SIGMOID) {
    const float e = expf(-fabsf(x));
    *f = fmaxf(-x, 0.0f) + log1pf(e);
    *df = -(x >= 0.0f ? e : 1.0f) / (1.0f + e);
    if (x != x) *f = *df = x;
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

// The sums over places [t0, t1) of a pair's rows (token t of a row has place t + its shift;
// t0 a multiple of 256) by a group of kGroup warps: a warp by itself, or the CTA
// through red and counts.
template <int N, bool kVec, bool kRef, int kGroup>
__device__ __forceinline__ void pair_sums(const PreferenceParams& p, int64_t pair, int t0, int t1,
                                          Sum2 (*red)[2], int (*counts)[2], Sum2* sum, int* count) {
  const int lane = threadIdx.x & 31, warp = kGroup == 1 ? 0 : threadIdx.x >> 5;
  constexpr int kStride = 32 * N * kGroup;
  const uint8_t* mask[2];
  const float* x[2];
  const float* ref[2];
  Sum2 s[2];
  int n[2] = {0, 0}, shift[2], end[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t r = pair + k * p.a.P;
    shift[k] = shift_of<N, kVec>(r, p.a.ld_logp);
    end[k] = min(static_cast<int>(p.a.T), t1 - shift[k]);
    mask[k] = p.a.mask == nullptr ? nullptr : p.a.mask + r * p.a.ld_mask;
    x[k] = p.a.logp + r * p.a.ld_logp;
    ref[k] = kRef ? p.a.ref_logp + r * p.a.ld_ref : nullptr;
  }
  int t = t0 + 32 * N * warp, left = t1 - t;
  Mask<N> next[2];
  if (left > 0) {
    next[0] = load_mask<N, kVec>(mask[0], t - shift[0], end[0]);
    next[1] = load_mask<N, kVec>(mask[1], t - shift[1], end[1]);
  }
#pragma unroll 1
  for (; left > 0; left -= kStride, t += kStride) {
    float v[2][N], u[2][N];
    const Mask<N> m[2] = {next[0], next[1]};
    load_tokens<N, kVec>(x[0], t - shift[0], end[0], m[0], v[0]);
    load_tokens<N, kVec>(x[1], t - shift[1], end[1], m[1], v[1]);
    if (kRef) {
      load_tokens<N, kVec>(ref[0], t - shift[0], end[0], m[0], u[0]);
      load_tokens<N, kVec>(ref[1], t - shift[1], end[1], m[1], u[1]);
    }
    if (left > kStride) {
      next[0] = load_mask<N, kVec>(mask[0], t + kStride - shift[0], end[0]);
      next[1] = load_mask<N, kVec>(mask[1], t + kStride - shift[1], end[1]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float f = 0.0f;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (m[k].on(j)) f += kRef ? v[k][j] - u[k][j] : v[k][j];
      n[k] += m[k].count();
      s[k].add(f);
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    s[k] = warp_sum(s[k]);
    n[k] = __reduce_add_sync(0xffffffffu, n[k]);
    if (kGroup == 1) {
      sum[k] = s[k];
      count[k] = n[k];
    } else if (lane == 0) {
      red[warp][k] = s[k];
      counts[warp][k] = n[k];
    }
  }
  if (kGroup == 1) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    sum[k] = red[0][k];
    count[k] = counts[0][k];
#pragma unroll
    for (int w = 1; w < kGroup; ++w) {
      sum[k].add(red[w][k]);
      count[k] += counts[w][k];
    }
  }
}

// What follows from a pair's sums, in every thread.
struct PairGrad {
  float loss, d[2], reward[2];
};

__device__ __forceinline__ PairGrad pair_grad(const bergson_preference_args& a, const Sum2* sum,
                                              const int* count) {
  const float beta = static_cast<float>(a.beta), eps = static_cast<float>(a.label_smoothing);
  float n[2], s[2], gap;
  for (int k = 0; k < 2; ++k) {
    n[k] = a.mean_logp && count[k] > 1 ? static_cast<float>(count[k]) : 1.0f;
    s[k] = sum[k].value() / n[k];
  }
  // without means the sums' second parts still count in their difference
  gap = a.mean_logp ? s[0] - s[1] : sum[0].hi - sum[1].hi;
  if (!a.mean_logp && gap - gap == 0.0f) gap += sum[0].lo - sum[1].lo;
  const float x = fmaf(beta, gap, -static_cast<float>(a.margin));
  float f, df, g, dg;
  preference_f(a.kind, x, beta, &f, &df);
  preference_f(a.kind, -x, beta, &g, &dg);
  PairGrad o;
  // a side of weight 0 takes no part, even where it is infinite
  o.loss = (eps < 1.0f ? (1.0f - eps) * f : 0.0f) + (eps > 0.0f ? eps * g : 0.0f);
  const float slope = (eps < 1.0f ? (1.0f - eps) * df : 0.0f) - (eps > 0.0f ? eps * dg : 0.0f);
  for (int k = 0; k < 2; ++k) {
    o.d[k] = (k ? -slope : slope) * beta / (static_cast<float>(a.P) * n[k]);
    o.reward[k] = beta * s[k];
  }
  return o;
}

template <int N, bool kVec, int kGroup>
__device__ __forceinline__ void write_pair(const PreferenceParams& p, int64_t pair, int t0, int t1,
                                           const float* d) {
  const int warp = kGroup == 1 ? 0 : threadIdx.x >> 5;
  constexpr int kStride = 32 * N * kGroup;
  const uint8_t* mask[2];
  float* out[2];
  int shift[2], end[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t r = pair + k * p.a.P;
    shift[k] = shift_of<N, kVec>(r, p.a.ld_logp);
    end[k] = min(static_cast<int>(p.a.T), t1 - shift[k]);
    mask[k] = p.a.mask == nullptr ? nullptr : p.a.mask + r * p.a.ld_mask;
    out[k] = p.a.d_logp + r * p.a.ld_d;
  }
  int t = t0 + 32 * N * warp;
#pragma unroll 2
  for (int left = t1 - t; left > 0; left -= kStride, t += kStride) {
    const Mask<N> m[2] = {load_mask<N, kVec>(mask[0], t - shift[0], end[0]),
                          load_mask<N, kVec>(mask[1], t - shift[1], end[1])};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float x[N];
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = m[k].on(j) ? d[k] : 0.0f;
      store_tokens<N, kVec>(out[k], t - shift[k], end[k], x);
    }
  }
}

__device__ __forceinline__ void write_rewards(const bergson_preference_args& a, int64_t pair,
                                              const PairGrad& g) {
  a.pair_loss[pair] = g.loss;
  if (a.rewards == nullptr) return;
  a.rewards[pair] = g.reward[0];
  a.rewards[pair + a.P] = g.reward[1];
}

// Places that the rows' tokens may have, whatever their shifts.
template <int N>
__device__ __forceinline__ int places(int64_t T) {
  return T > 0 ? static_cast<int>(T) + N - 1 : 0;
}

// Many short pairs: one a warp.
template <int N, bool kVec, bool kRef>
__global__ void __launch_bounds__(kPairThreads) preference_warp_kernel(const PreferenceParams p) {
  const int64_t pair = static_cast<int64_t>(blockIdx.x) * kPairWarps + (threadIdx.x >> 5);
  griddep_wait();
  if (pair >= p.a.P) return;
  const int T = places<N>(p.a.T);
  Sum2 sum[2];
  int count[2];
  pair_sums<N, kVec, kRef, 1>(p, pair, 0, T, nullptr, nullptr, sum, count);
  const PairGrad g = pair_grad(p.a, sum, count);
  if ((threadIdx.x & 31) == 0) write_rewards(p.a, pair, g);
  write_pair<N, kVec, 1>(p, pair, 0, T, g.d);
}

// kTogether: a pair a CTA, all of them in one cluster, whose first CTA adds the losses.
// Else a pair a cluster, its CTAs each a share of the tokens.
template <int N, bool kVec, bool kRef, bool kTogether>
__global__ void __launch_bounds__(kPairThreads, kRef ? kPairPerSmRef : kPairPerSm)
    preference_kernel(const PreferenceParams p) {
  __shared__ Sum2 red[kPairWarps][2];
  __shared__ int counts[kPairWarps][2];
  __shared__ float shared[8][6];               // from each CTA: two sums and counts
  const int parts = static_cast<int>(cluster_size());
  const int rank = static_cast<int>(blockIdx.x) % parts;
  const int64_t pair = kTogether ? blockIdx.x : blockIdx.x / parts;
  const bool live = pair < p.a.P;
  const int T = places<N>(p.a.T), blocks = (T - 1) / 256 + 1;
  const int per = kTogether ? blocks : (blocks + parts - 1) / parts;
  const int t0 =
      kTogether ? 0 : static_cast<int>(min(static_cast<int64_t>(T), int64_t{256} * per * rank));
  const int t1 = static_cast<int>(min(static_cast<int64_t>(T), t0 + int64_t{256} * per));
  Sum2 sum[2];
  int count[2] = {};
  griddep_wait();
  if (live) pair_sums<N, kVec, kRef, kPairWarps>(p, pair, t0, t1, red, counts, sum, count);
  if (!kTogether && parts > 1) {
    cluster_barrier();                            // every CTA has started
    if (threadIdx.x < parts) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        st_cluster(&shared[rank][3 * k], threadIdx.x, sum[k].hi);
        st_cluster(&shared[rank][3 * k + 1], threadIdx.x, sum[k].lo);
        st_cluster(&shared[rank][3 * k + 2], threadIdx.x, __int_as_float(count[k]));
      }
    }
    cluster_barrier();
    for (int k = 0; k < 2; ++k) {
      sum[k] = Sum2();
      count[k] = 0;
      for (int c = 0; c < parts; ++c) {
        Sum2 o;
        o.hi = shared[c][3 * k];
        o.lo = shared[c][3 * k + 1];
        sum[k].add(o);
        count[k] += __float_as_int(shared[c][3 * k + 2]);
      }
    }
  }
  PairGrad g = {};
  if (live) {
    g = pair_grad(p.a, sum, count);
    if (threadIdx.x == 0 && (kTogether || rank == 0)) write_rewards(p.a, pair, g);
  }

  if (live) write_pair<N, kVec, kPairWarps>(p, pair, t0, t1, g.d);
  if (kTogether) {
    cluster_barrier();                            // every CTA has started
    if (threadIdx.x == 0) st_cluster(&shared[rank][0], 0, g.loss);
    cluster_barrier();
    if (rank == 0 && threadIdx.x == 0) {
      Sum2 l;
      for (int c = 0; c < static_cast<int>(p.a.P); ++c) l.add(shared[c][0]);
      *p.a.loss = l.value() / static_cast<float>(p.a.P);
    }
  }
}

__global__ void __launch_bounds__(1024) preference_finish_kernel(const float* pair_loss,
                                                                 int64_t P, float* loss) {
  __shared__ Sum2 red[32];
  griddep_wait();
  Sum2 s;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < P; i += blockDim.x) s.add(pair_loss[i]);
  s = block_sum(s, red);
  if (threadIdx.x == 0) *loss = P > 0 ? s.value() / static_cast<float>(P) : 0.0f;
}

// ------------------------------------------------------------------- host

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t align256(size_t n) { return (n + 255) / 256 * 256; }
size_t counts_bytes(int64_t B, int64_t T) {
  const int64_t n = std::max<int64_t>(kCountCtas, B * ceil_div(T, kCountSegment));
  return align256(4 * static_cast<size_t>(n));
}

// Rows whose vectors of n tokens lie where those of a tensor of leading dimension ld0 do.
bool fits(const void* p, int64_t ld, size_t elem, int n, int64_t ld0) {
  return p == nullptr ||
         (reinterpret_cast<uintptr_t>(p) % (n * elem) == 0 && (ld - ld0) % n == 0);
}

template <typename K, typename P>
cudaError_t launch_cluster(K kernel, int64_t grid, int threads, int cluster, const P& p,
                           cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <bool kVec>
cudaError_t run_policy(PolicyParams p, cudaStream_t s) {
  if (p.segment == kShortSegment && p.a.B * p.segments <= kSmallItems) {
    int parts = 1;
    while (parts < 8 && parts * kSmallWarps < p.a.B * p.segments) parts *= 2;
    return launch_cluster(policy_small_kernel<kVec>, parts, kSmallThreads, parts, p, s);
  }
  const int64_t items = p.a.B * p.segments;
  if (p.a.mask != nullptr && p.a.reduction != BERGSON_POLICY_SUM_NORM) {
    p.n_counts = static_cast<int>(
        std::min<int64_t>(kCountCtas, 4 * ceil_div(p.a.B * p.count_segments, 4 * kWarps)));
    const cudaError_t e =
        launch_dependent(policy_count_kernel, dim3(p.n_counts), dim3(kThreads), 0, s, p);
    if (e != cudaSuccess) return e;
  }
  cudaError_t e = launch_dependent(policy_kernel<kVec>,
                                   dim3(static_cast<unsigned>(ceil_div(items, kWarps))),
                                   dim3(kThreads), 0, s, p);
  if (e != cudaSuccess) return e;
  const int64_t finish = std::min<int64_t>(kFinishCtas, ceil_div(p.a.B, kWarps));
  return launch_dependent(policy_finish_kernel, dim3(static_cast<unsigned>(finish)),
                          dim3(kThreads), 0, s, p);
}

template <int N, bool kVec, bool kRef>
cudaError_t run_preference(const PreferenceParams& p, cudaStream_t s) {
  const int64_t P = p.a.P;
  // few short pairs: one launch, their losses added through the cluster (4 x 383 tokens
  // 8.0 us, 9.9 with the second grid)
  if (P <= 8 && 2 * p.a.T <= 8192) {
    int n = 1;
    while (n < P) n *= 2;
    return launch_cluster(preference_kernel<N, kVec, kRef, true>, n, kPairThreads, n, p, s);
  }
  int parts = 1;
  while (parts < 8 && P * parts < kPairCtas * kPlanCTAs && p.a.T / parts > kPairTokens) parts *= 2;
  cudaError_t e;
  if (P >= kManyPairs && p.a.T <= kShortPair)
    e = launch_dependent(preference_warp_kernel<N, kVec, kRef>,
                         dim3(static_cast<unsigned>(ceil_div(P, kPairWarps))),
                         dim3(kPairThreads), 0, s, p);
  else
    e = launch_cluster(preference_kernel<N, kVec, kRef, false>, P * parts, kPairThreads, parts, p,
                       s);
  if (e != cudaSuccess) return e;
  return launch_dependent(preference_finish_kernel, dim3(1), dim3(1024), 0, s,
                          static_cast<const float*>(p.a.pair_loss), P, p.a.loss);
}

template <int N, bool kVec>
cudaError_t run_preference(const PreferenceParams& p, cudaStream_t s) {
  return p.a.ref_logp != nullptr ? run_preference<N, kVec, true>(p, s)
                                 : run_preference<N, kVec, false>(p, s);
}

}  // namespace

// Segments of a row, from its shift on.
static int64_t segments_of(int64_t T, int segment) { return (T + 3 + segment - 1) / segment; }

// counts, the totals and their ticket, the segments' sums
size_t policy_workspace(int64_t B, int64_t T) {
  return counts_bytes(B, T) + align256(sizeof(Totals) * kFinishCtas) + 256 +
         align256(sizeof(float4) * static_cast<size_t>(B * segments_of(T, kShortSegment)));
}

cudaError_t launch_policy_loss(const bergson_policy_args& a, void* ws, cudaStream_t s) {
  PolicyParams p;
  p.a = a;
  p.segment = a.B * ceil_div(a.T, kSegment) >= kLongItems ? kSegment : kShortSegment;
  p.count_segments = ceil_div(a.T, kCountSegment);
  p.n_counts = 0;
  char* at = static_cast<char*>(ws);
  p.counts = reinterpret_cast<unsigned*>(at);
  at += counts_bytes(a.B, a.T);
  p.totals = reinterpret_cast<Totals*>(at);
  at += align256(sizeof(Totals) * kFinishCtas);
  p.ticket = reinterpret_cast<unsigned*>(at);
  p.sums = reinterpret_cast<float4*>(at + 256);
  p.low = static_cast<float>(1.0 - a.clip_low);
  p.high = static_cast<float>(1.0 + a.clip_high);
  p.kl = static_cast<float>(a.kl_coef);
  p.ent = static_cast<float>(a.entropy_coef);
  p.norm = static_cast<float>(1.0 / (static_cast<double>(a.B) * a.norm_tokens));
  if (a.kl_coef == 0.0 && a.stats == nullptr) p.a.ref_logp = nullptr;
  if (a.entropy_coef == 0.0) p.a.entropy = nullptr;
  if (a.B == 0 || a.T == 0) {                  // no token: zeros
    cudaError_t e = cudaMemsetAsync(a.loss, 0, sizeof(float), s);
    if (e == cudaSuccess && a.stats != nullptr)
      e = cudaMemsetAsync(a.stats, 0, 3 * sizeof(float), s);
    if (e == cudaSuccess && a.seq_loss != nullptr && a.B > 0)
      e = cudaMemsetAsync(a.seq_loss, 0, sizeof(float) * static_cast<size_t>(a.B), s);
    return e;
  }
  const auto fit = [&](const void* x, int64_t ld, size_t elem) {
    return fits(x, ld, elem, 4, a.ld_logp);
  };
  const bool vec = fit(a.logp, a.ld_logp, 4) && fit(a.old_logp, a.ld_old, 4) &&
                   fit(p.a.ref_logp, a.ld_ref, 4) && fit(p.a.entropy, a.ld_entropy, 4) &&
                   (a.ld_adv == 0 || fit(a.advantages, a.ld_adv, 4)) &&
                   fit(a.mask, a.ld_mask, 1) && fit(a.d_logp, a.ld_d, 4) &&
                   fit(a.d_entropy, a.ld_de, 4);
  // rows that start on boundaries need no room for a shift
  p.segments = vec && a.ld_logp % 4 != 0 ? segments_of(a.T, p.segment) : ceil_div(a.T, p.segment);
  return vec ? run_policy<true>(p, s) : run_policy<false>(p, s);
}

cudaError_t launch_preference_loss(const bergson_preference_args& a, cudaStream_t s) {
  if (a.P == 0) {
    preference_finish_kernel<<<1, 1024, 0, s>>>(a.pair_loss, 0, a.loss);
    return cudaGetLastError();
  }
  PreferenceParams p;
  p.a = a;
  const auto all_fit = [&](int n) {
    return fits(a.logp, a.ld_logp, 4, n, a.ld_logp) &&
           fits(a.ref_logp, a.ld_ref, 4, n, a.ld_logp) &&
           fits(a.mask, a.ld_mask, 1, n, a.ld_logp) && fits(a.d_logp, a.ld_d, 4, n, a.ld_logp);
  };
  if (all_fit(8)) return run_preference<8, true>(p, s);
  return all_fit(4) ? run_preference<4, true>(p, s) : run_preference<4, false>(p, s);
}

}  // namespace bergson
