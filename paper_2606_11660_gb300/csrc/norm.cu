// Layer norm (and its form without a mean), forward and backward.
//
//   forward   y = (x - mu) rstd w + b,   rstd = (mean (x - mu)^2 + eps)^-1/2
//   backward  h = dy w,  n = (x - mu) rstd,
//             dx = rstd (h - mean h - n mean (h n)),  dw = sum_r dy n,  db = sum_r dy
//
// (mu = 0 and no mean of h without a mean).  Both are bound by their bytes: a
// row is read once, stays in the registers of the 4 .. 32 lanes (up to 512 columns; forward
// up to 1024) or the CTA that have it, 8 to 32 columns a thread, and the next rows are on
// their way while this one is reduced.  A thread keeps its columns from row to row, so that weights
// are loaded once a CTA and the backward pass sums dw and db in registers; one row of both a CTA
// goes to the workspace, and a second kernel adds these up in order.
// 65,536 x 2048 bf16: 91 us forward (5.9 TB/s) and 139 backward (135 and 4; 6.0 TB/s); the forward
// pass fills 68% of the issue slots, and did so at 77% in 127 us before its arithmetic went in pairs.

#include <algorithm>
#include <atomic>
#include <cmath>

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kCols = 16;                      // columns a thread
constexpr int kShortCols = 32 * 8;             // up to here 8 columns a lane, as few lanes as do
constexpr int kWarpCols = 32 * kCols;          // up to here a warp takes a row, 16 columns a lane
constexpr int kLongCols = 64 * kCols;          // forward, with vectors, up to here, 32 columns a lane
constexpr int kWarps = 4;                      // warps of such a CTA
constexpr int kMidCols = 8192;                 // up to here dw, db and the next row stay in registers
constexpr int kMaxCols = 16384;                // up to here a row stays in registers
constexpr int kLoopThreads = 512;              // of the kernels for longer rows
constexpr int kSlabRows = 512;                 // rows of a CTA that sums columns of such rows

// Sums of one value or two over the threads that share a row, in each of them: G lanes side by
// side, or the CTA by way of `red` (N values for each of 32 warps, not in use by the row before or
// after, zeros at first).  Two go through the warp as one: its halves take one each after the first
// step.
template <bool kCta, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int G, float* red) {
  static_assert(N == 1 || N == 2, "one value or two");
  if constexpr (!kCta) {
    for (int o = G >> 1; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
  } else {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    float s;
    if constexpr (N == 2) {
      const bool upper = lane >= 16;
      s = upper ? v[1] : v[0];
      s += __shfl_xor_sync(0xffffffffu, upper ? v[0] : v[1], 16);
    } else {
      s = v[0] + __shfl_xor_sync(0xffffffffu, v[0], 16);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane % (32 / N) == 0) red[N * warp + lane / (32 / N)] = s;
    __syncthreads();
    // four at a time; what stands behind the last warp's is 0
    float4 t = *reinterpret_cast<const float4*>(red);
    for (int w = 4; w < N * warps; w += 4) {
      const float4 y = *reinterpret_cast<const float4*>(red + w);
      t.x += y.x; t.y += y.y; t.z += y.z; t.w += y.w;
    }
    if constexpr (N == 1) {
      v[0] = (t.x + t.y) + (t.z + t.w);
    } else {
      v[0] = t.x + t.z;
      v[1] = t.y + t.w;
    }
  }
}
// rstd of a mean square with eps added: NaN where that is infinite, so that a row which holds an
// infinity is NaN without a mean too (1 / sqrt(inf) = 0 would make its other entries zeros).
__device__ __forceinline__ float inverse_root(float square) {
  return __frcp_rn(__fsqrt_rn(square)) + (square - square);
}
// Clears the places of row_sums.
__device__ __forceinline__ void clear_sums(float* red, int n) {
  for (int i = threadIdx.x; i < n; i += blockDim.x) red[i] = 0.0f;
  __syncthreads();
}

// Rows on their way to a thread.  In vectors: by asynchronous copies to places of its own in
// shared memory, kSlots rows ahead, so that no thread waits for another and no register is
// held (a row at a time in registers: too few bytes in flight, 65,536 x 2048 at 4.1 TB/s with 6
// CTAs an SM).  A vector past the end copies what there is and zeros.  By elements: one row ahead,
// in registers.
template <typename T, int kB, int C, int kSlots>
struct Feed {
  using R = RowPart<T, kB, C>;
  static constexpr bool kVec = kB > 0;
  static constexpr int kBytes = R::kPer * kB;    // of a row, a thread
  uint32_t base;
  int slot = 0;
  int bytes[kVec ? R::kPer : 1];                 // of the thread's vectors that are within a row
  R row;
  __device__ __forceinline__ Feed(const void* smem, int part, int d, int t, int G)
      : base(kVec ? smem_u32(smem) + part * kSlots * kBytes * blockDim.x + kB * threadIdx.x : 0) {
    if constexpr (kVec) {
#pragma unroll
      for (int k = 0; k < R::kPer; ++k)
        bytes[k] = max(0, min(kB, (d - R::col(t, G, k)) * static_cast<int>(sizeof(T))));
    }
  }
  __device__ __forceinline__ uint32_t at(int k) const {
    return base + (slot * R::kPer + k) * kB * blockDim.x;
  }
  // Sends for row r, which starts at p, into the slot that was read last (in: it is a row at all).
  __device__ __forceinline__ void send(const T* first, int64_t r, int64_t ld, bool in, int d, int t,
                                       int G) {
    const T* p = in ? first + r * ld : first;
    if constexpr (kVec) {
      p += R::E * t;
#pragma unroll
      for (int k = 0; k < R::kPer; ++k) {
        const int n = in ? bytes[k] : 0;
        const T* from = n > 0 ? p + k * R::E * G : first;
        if constexpr (kB == 16)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at(k)), "l"(from), "r"(n)
                       : "memory");
        else
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(at(k)), "l"(from), "r"(n)
                       : "memory");
      }
    } else {
      row.load(p, in ? d : 0, t, G);
    }
  }
  __device__ __forceinline__ void next() { slot = slot + 1 == kSlots ? 0 : slot + 1; }
  // The values of the slot's row (which must have arrived).
  __device__ __forceinline__ void take(float2 (&x)[C / 2]) {
    if constexpr (kVec) {
#pragma unroll
      for (int k = 0; k < R::kPer; ++k) {
        if constexpr (kB == 16) {
          uint32_t* r = row.raw + 4 * k;
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                       : "r"(at(k))
                       : "memory");
        } else {
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(row.raw[k]) : "r"(at(k)) : "memory");
        }
      }
    }
    row.pairs(x);
  }
};
template <bool kVec>
__device__ __forceinline__ void feed_commit() {
  if constexpr (kVec) asm volatile("cp.async.commit_group;" ::: "memory");
}
template <bool kVec>
__device__ __forceinline__ void feed_end() {
  if constexpr (kVec) asm volatile("cp.async.wait_group 0;" ::: "memory");
}
template <bool kVec, int kSlots>
__device__ __forceinline__ void feed_wait() {
  if constexpr (kVec) asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 1) : "memory");
}

// The rows of a thread: its first one, and how far apart they are.  All lanes of a warp make
// the same number of turns; a row past the last is of no columns.
struct Turns {
  int G, t;                    // threads that share a row, place among them
  int64_t first, step;         // rows of the warp's (CTA's) first lane
  int sub;                     // rows behind that
};
template <bool kCta>
__device__ __forceinline__ Turns turns(int lanes) {
  Turns u;
  if (kCta) {
    u.G = blockDim.x;
    u.t = threadIdx.x;
    u.first = blockIdx.x;
    u.step = gridDim.x;
    u.sub = 0;
  } else {
    const int per = 32 / lanes;
    u.G = lanes;
    u.t = threadIdx.x & (lanes - 1);
    u.first = (static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * per;
    u.step = static_cast<int64_t>(gridDim.x) * kWarps * per;
    u.sub = (threadIdx.x & 31) / lanes;
  }
  return u;
}

struct NormParams {
  const void* x;
  const void* w;               // or nullptr: ones
  const void* b;               // or nullptr: zeros
  void* y;
  float* mean;                 // or nullptr
  float* rstd;                 // or nullptr
  int64_t rows, ld_x, ld_y;
  int64_t d;
  int lanes;                   // that share a row, of kernels without kCta: 4 .. 32
  int wt;
  int layer;
  float eps, inv_d;
};

constexpr int kForwardSlots = 3, kBackwardSlots = 2;

template <typename T, int kB, bool kCta, bool kWide, int C>
__global__ void __launch_bounds__(kWide ? 1024 : kCta ? 512 : 32 * kWarps)
    norm_kernel(const __grid_constant__ NormParams p) {
  using R = RowPart<T, kB, C>;
  constexpr bool kVec = kB > 0;
  constexpr int kSlots = kVec ? kForwardSlots : 1;
  constexpr int H = C / 2;
  extern __shared__ __align__(16) uint8_t slots[];
  __shared__ __align__(16) float red[2][2][32];
  const Turns u = turns<kCta>(p.lanes);
  const int G = u.G, t = u.t, d = static_cast<int>(p.d);
  const bool whole = R::column(t, G, C - 1) < d;       // all of the thread's columns are
  if (kCta) clear_sums(&red[0][0][0], 128);
  griddep_wait();
  const T* xs = static_cast<const T*>(p.x);
  Feed<T, kB, C, kSlots> feed(slots, 0, d, t, G);
  const auto send = [&](int64_t r) {
    feed.send(xs, r, p.ld_x, r < p.rows, d, t, G);
    feed_commit<kVec>();
  };
#pragma unroll
  for (int k = 0; k < kSlots; ++k) {
    send(u.first + k * u.step + u.sub);
    feed.next();
  }
  float2 w[H], b[H];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = R::column(t, G, i);
    const float wi = p.w != nullptr && c < d ? load_any(p.w, p.wt, c) : 1.0f;
    const float bi = p.b != nullptr && c < d ? load_any(p.b, p.wt, c) : 0.0f;
    (i % 2 == 0 ? w[i / 2].x : w[i / 2].y) = wi;
    (i % 2 == 0 ? b[i / 2].x : b[i / 2].y) = bi;
  }
  int turn = 0;
  for (int64_t first = u.first; first < p.rows; first += u.step, turn ^= 1) {
    const int64_t r = first + u.sub;
    float2 x[H];
    feed_wait<kVec, kSlots>();
    feed.take(x);
    send(r + kSlots * u.step);
    feed.next();
    float mean = 0.0f;
    if (p.layer) {
      float2 s2 = x[0];
#pragma unroll
      for (int i = 1; i < H; ++i) s2 = add2(s2, x[i]);
      float s[1] = {s2.x + s2.y};
      row_sums<kCta>(s, G, red[turn][0]);
      mean = s[0] * p.inv_d;
      const float2 less = pair(-mean);
#pragma unroll
      for (int i = 0; i < H; ++i) x[i] = add2(x[i], less);
      if (!whole) {
#pragma unroll
        for (int i = 0; i < C; ++i)
          if (R::column(t, G, i) >= d) (i % 2 == 0 ? x[i / 2].x : x[i / 2].y) = 0.0f;
      }
    }
    float2 q2 = mul2(x[0], x[0]);
#pragma unroll
    for (int i = 1; i < H; ++i) q2 = fma2(x[i], x[i], q2);
    float q[1] = {q2.x + q2.y};
    row_sums<kCta>(q, G, red[turn][1]);
    const float rstd = inverse_root(fmaf(q[0], p.inv_d, p.eps));
#pragma unroll
    for (int i = 0; i < H; ++i) x[i] = fma2(mul2(x[i], pair(rstd)), w[i], b[i]);
    R::store_pairs(static_cast<T*>(p.y) + r * p.ld_y, r < p.rows ? d : 0, t, G, x);
    if (t == 0 && r < p.rows) {
      if (p.mean != nullptr && p.layer) p.mean[r] = mean;
      if (p.rstd != nullptr) p.rstd[r] = rstd;
    }
  }
  feed_end<kVec>();
}

// Rows too long for registers: a CTA a row, read once a sum and once more.
template <typename T>
__global__ void __launch_bounds__(kLoopThreads) norm_loop_kernel(
    const __grid_constant__ NormParams p) {
  __shared__ float red[2][32];
  griddep_wait();
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(p.x) + r * p.ld_x;
    T* y = static_cast<T*>(p.y) + r * p.ld_y;
    float mean = 0.0f;
    if (p.layer) {
      CompensatedSum s;
      for (int64_t c = threadIdx.x; c < p.d; c += kLoopThreads) s.add(to_f32(x[c]));
      mean = block_sum(s.s, red[0]) * p.inv_d;
    }
    CompensatedSum q;
    for (int64_t c = threadIdx.x; c < p.d; c += kLoopThreads) {
      const float v = to_f32(x[c]) - mean;
      q.add(v * v);
    }
    const float rstd = inverse_root(fmaf(block_sum(q.s, red[1]), p.inv_d, p.eps));
    for (int64_t c = threadIdx.x; c < p.d; c += kLoopThreads) {
      const float w = p.w != nullptr ? load_any(p.w, p.wt, c) : 1.0f;
      const float b = p.b != nullptr ? load_any(p.b, p.wt, c) : 0.0f;
      y[c] = from_f32<T>(fmaf((to_f32(x[c]) - mean) * rstd, w, b));
    }
    if (threadIdx.x == 0) {
      if (p.mean != nullptr && p.layer) p.mean[r] = mean;
      if (p.rstd != nullptr) p.rstd[r] = rstd;
    }
  }
}

// ------------------------------------------------------------------ backward

struct GradParams {
  const void* x;
  const void* w;               // or nullptr: ones
  const float* mean;           // layer norm only
  const float* rstd;
  const void* dy;
  void* dx;
  float* part;                 // [CTAs, 2, d] sums of dy n and dy, or nullptr: none wanted
  int64_t rows, ld_x, ld_dy, ld_dx;
  int64_t d;
  int lanes;                   // that share a row, of kernels without kCta: 4 .. 32
  int wt;
  int layer;
  float inv_d;
};

// kWide: 8192 < d <= 16384, 1024 threads of 64 registers: dw, db and the weights stand
// in shared memory (192 KB at the longest), and no row is read ahead.
template <typename T, int kB, bool kCta, bool kWide, int C>
__global__ void __launch_bounds__(kWide ? 1024 : kCta ? 512 : 32 * kWarps)
    norm_backward_kernel(const __grid_constant__ GradParams p) {
  using R = RowPart<T, kB, C>;
  // kWide: the rows are read as they are needed
  constexpr bool kFed = kB > 0 && !kWide;
  constexpr int kSlots = kFed ? kBackwardSlots : 1;
  constexpr int H = C / 2;
  __shared__ __align__(16) float red[2][64];
  // kWide: weights, dw, db; else the rows on their way, and at the end [2, d] of a CTA's warps to
  // add up
  extern __shared__ __align__(16) float wide[];
  const Turns u = turns<kCta>(p.lanes);
  const int G = u.G, t = u.t, d = static_cast<int>(p.d);
  if (kCta) clear_sums(&red[0][0], 128);
  griddep_wait();
  // where thread t's pair i stands in shared memory: neighbouring threads side by side
  float2* wide2 = reinterpret_cast<float2*>(wide);
  const auto at = [&](int i) { return i * G + t; };
  const int n = H * G;
  float2 w[kWide ? 1 : H], dw[kWide ? 1 : H], db[kWide ? 1 : H];
  const T* xs = static_cast<const T*>(p.x);
  const T* dys = static_cast<const T*>(p.dy);
  Feed<T, kB, C, kSlots> nx(wide, 0, d, t, G), ny(wide, 1, d, t, G);
  RowPart<T, kB, C> rx, ry;                  // kWide
  float mean_next[kSlots], rstd_next[kSlots];
  const auto send = [&](int k, int64_t row) {
    const bool in = row < p.rows;
    if constexpr (kWide) {
      rx.load(xs + (in ? row * p.ld_x : 0), in ? d : 0, t, G);
      ry.load(dys + (in ? row * p.ld_dy : 0), in ? d : 0, t, G);
    } else {
      nx.send(xs, row, p.ld_x, in, d, t, G);
      ny.send(dys, row, p.ld_dy, in, d, t, G);
    }
    feed_commit<kFed>();
    mean_next[k] = p.layer && in ? p.mean[row] : 0.0f;
    rstd_next[k] = in ? p.rstd[row] : 0.0f;
  };
#pragma unroll
  for (int k = 0; k < kSlots; ++k) {
    send(k, u.first + k * u.step + u.sub);
    nx.next();
    ny.next();
  }
#pragma unroll
  for (int i = 0; i < H; ++i) {
    float2 v;
    const int c0 = R::column(t, G, 2 * i), c1 = R::column(t, G, 2 * i + 1);
    v.x = p.w != nullptr && c0 < d ? load_any(p.w, p.wt, c0) : 1.0f;
    v.y = p.w != nullptr && c1 < d ? load_any(p.w, p.wt, c1) : 1.0f;
    if constexpr (kWide) {
      wide2[at(i)] = v;
      wide2[n + at(i)] = wide2[2 * n + at(i)] = pair(0.0f);
    } else {
      w[i] = v;
      dw[i] = db[i] = pair(0.0f);
    }
  }
  int turn = 0;
  for (int64_t first = u.first; first < p.rows; first += u.step, turn ^= 1) {
    const int64_t r = first + u.sub;
    float2 x[H], g[H];
    feed_wait<kFed, kSlots>();
    if constexpr (kWide) {
      rx.pairs(x);
      ry.pairs(g);
    } else {
      nx.take(x);
      ny.take(g);
    }
    const float mean = mean_next[0], rstd = rstd_next[0];
#pragma unroll
    for (int k = 1; k < kSlots; ++k) {
      mean_next[k - 1] = mean_next[k];
      rstd_next[k - 1] = rstd_next[k];
    }
    if constexpr (!kWide) {
      send(kSlots - 1, r + kSlots * u.step);
      nx.next();
      ny.next();
    }
    // past the row's end dy is 0: nothing there counts
    float2 along2 = pair(0.0f), level2 = pair(0.0f);
#pragma unroll
    for (int i = 0; i < H; ++i) {
      x[i] = mul2(add2(x[i], pair(-mean)), pair(rstd));
      if constexpr (kWide) {
        wide2[n + at(i)] = fma2(g[i], x[i], wide2[n + at(i)]);
        wide2[2 * n + at(i)] = add2(wide2[2 * n + at(i)], g[i]);
        g[i] = mul2(g[i], wide2[at(i)]);
      } else {
        dw[i] = fma2(g[i], x[i], dw[i]);
        db[i] = add2(db[i], g[i]);
        g[i] = mul2(g[i], w[i]);
      }
      along2 = fma2(g[i], x[i], along2);
      level2 = add2(level2, g[i]);
    }
    float s[2] = {along2.x + along2.y, level2.x + level2.y};
    row_sums<kCta>(s, G, red[turn]);
    const float2 along = pair(-s[0] * p.inv_d), level = pair(p.layer ? -s[1] * p.inv_d : 0.0f);
#pragma unroll
    for (int i = 0; i < H; ++i) x[i] = mul2(add2(fma2(x[i], along, g[i]), level), pair(rstd));
    R::store_pairs(static_cast<T*>(p.dx) + r * p.ld_dx, r < p.rows ? d : 0, t, G, x);
    if constexpr (kWide) send(0, r + u.step);
  }
  feed_end<kFed>();
  if (p.part == nullptr) return;
  float* part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * d;
  const auto put = [&](float* to, int i, const float2& v) {
    const int c0 = R::column(t, G, 2 * i), c1 = R::column(t, G, 2 * i + 1);
    if (c0 < d) to[c0] = v.x;
    if (c1 < d) to[c1] = v.y;
  };
  if constexpr (kWide) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      put(part, i, wide2[n + at(i)]);
      put(part + d, i, wide2[2 * n + at(i)]);
    }
  } else if constexpr (kCta) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      put(part, i, dw[i]);
      put(part + d, i, db[i]);
    }
  } else {
    __syncthreads();                           // the slots are free
    for (int o = G; o < 32; o <<= 1) {         // the warp's rows
#pragma unroll
      for (int i = 0; i < H; ++i) {
        dw[i].x += __shfl_xor_sync(0xffffffffu, dw[i].x, o);
        dw[i].y += __shfl_xor_sync(0xffffffffu, dw[i].y, o);
        db[i].x += __shfl_xor_sync(0xffffffffu, db[i].x, o);
        db[i].y += __shfl_xor_sync(0xffffffffu, db[i].y, o);
      }
    }
    const int warp = threadIdx.x >> 5;         // one warp after the other: a fixed order
    for (int k = 0; k < kWarps; ++k) {
      if (warp == k && u.sub == 0) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const int c = R::column(t, G, i);
          if (c < d) {
            const float vw = i % 2 == 0 ? dw[i / 2].x : dw[i / 2].y;
            const float vb = i % 2 == 0 ? db[i / 2].x : db[i / 2].y;
            wide[c] = k == 0 ? vw : wide[c] + vw;
            wide[d + c] = k == 0 ? vb : wide[d + c] + vb;
          }
        }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * d; c += blockDim.x) part[c] = wide[c];
  }
}

// dx of rows too long for registers.
template <typename T>
__global__ void __launch_bounds__(kLoopThreads) norm_backward_loop_kernel(
    const __grid_constant__ GradParams p) {
  __shared__ float red[2][32];
  griddep_wait();
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(p.x) + r * p.ld_x;
    const T* dy = static_cast<const T*>(p.dy) + r * p.ld_dy;
    T* dx = static_cast<T*>(p.dx) + r * p.ld_dx;
    const float mean = p.layer ? p.mean[r] : 0.0f, rstd = p.rstd[r];
    CompensatedSum hn, h;
    for (int64_t c = threadIdx.x; c < p.d; c += kLoopThreads) {
      const float w = p.w != nullptr ? load_any(p.w, p.wt, c) : 1.0f;
      const float g = to_f32(dy[c]) * w;
      hn.add(g * ((to_f32(x[c]) - mean) * rstd));
      h.add(g);
    }
    const float along = block_sum(hn.s, red[0]) * p.inv_d;
    const float level = p.layer ? block_sum(h.s, red[1]) * p.inv_d : 0.0f;
    for (int64_t c = threadIdx.x; c < p.d; c += kLoopThreads) {
      const float w = p.w != nullptr ? load_any(p.w, p.wt, c) : 1.0f;
      const float n = (to_f32(x[c]) - mean) * rstd;
      dx[c] = from_f32<T>(rstd * (to_f32(dy[c]) * w - fmaf(n, along, level)));
    }
  }
}

// Sums of dy n and dy of such rows: a thread a column, a CTA kSlabRows rows at a time.
template <typename T>
__global__ void __launch_bounds__(128) norm_columns_kernel(const __grid_constant__ GradParams p) {
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 128 + threadIdx.x;
  griddep_wait();
  if (c >= p.d) return;
  CompensatedSum dw, db;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.y) * kSlabRows; r0 < p.rows;
       r0 += static_cast<int64_t>(gridDim.y) * kSlabRows) {
    const int64_t end = min(r0 + kSlabRows, p.rows);
    for (int64_t r = r0; r < end; ++r) {
      const float g = to_f32(static_cast<const T*>(p.dy)[r * p.ld_dy + c]);
      const float x = to_f32(static_cast<const T*>(p.x)[r * p.ld_x + c]);
      dw.add(g * ((x - (p.layer ? p.mean[r] : 0.0f)) * p.rstd[r]));
      db.add(g);
    }
  }
  float* part = p.part + static_cast<int64_t>(blockIdx.y) * 2 * p.d;
  part[c] = dw.s;
  part[p.d + c] = db.s;
}

// dw and db from the CTAs' sums: 32 columns a CTA, a warp every 32nd of them.
constexpr int kPartWarps = 32;
__global__ void __launch_bounds__(32 * kPartWarps) norm_parts_kernel(
    const float* __restrict__ part, int n, int64_t d, float* dw, float* db) {
  __shared__ float red[kPartWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c0 = static_cast<int64_t>(blockIdx.x) * 32;
  float* out = blockIdx.y == 0 ? dw : db;
  griddep_wait();
  if (out == nullptr) return;
  const float* p = part + blockIdx.y * d + c0 + lane;
  float s = 0.0f;
  if (c0 + lane < d) {
    for (int k0 = warp; k0 < n; k0 += 8 * kPartWarps) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = k0 + i * kPartWarps;
        x[i] = k < n ? p[2 * d * k] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s += x[i];
    }
  }
  red[warp][lane] = s;
  __syncthreads();
  // column `warp`, its 32 sums across the lanes
  s = warp_sum(red[lane][warp]);
  if (lane == 0 && c0 + warp < d) out[c0 + warp] = s;
}

// Threads that share a row of the CTA kernels.
int row_threads(int64_t d) { return static_cast<int>(ceil_div(ceil_div(d, kCols), 32) * 32); }

// Lanes that share a row of up to kWarpCols columns.
int row_lanes(int64_t d) {
  int lanes = 32;
  while (lanes > 4 && d <= 4 * lanes) lanes /= 2;
  return lanes;
}

// CTAs of the forward kernels, which go over the rows: as many as are resident (one more than that
// would wait for all of another's rows: 65,536 x 2048 at 7 CTAs an SM where 6 fit 160 us, not 103).
template <typename Kernel>
cudaError_t resident_ctas(std::atomic<int>* known, Kernel kernel, int threads, size_t smem,
                          int64_t* ctas) {
  int n = known[threads / 32].load(std::memory_order_relaxed);
  if (n == 0) {
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem);
    if (e != cudaSuccess) return e;
    known[threads / 32].store(n, std::memory_order_relaxed);
  }
  *ctas = static_cast<int64_t>(kPlanCTAs) * std::max(1, n);
  return cudaSuccess;
}

// The most CTAs of the backward pass, which launches as many of them as are resident (65,536 x 512:
// 51 us; 5 an SM for every length 68).  It takes three rows a CTA at least: a CTA's sums cost about
// as much as a row.
int64_t backward_ctas(int64_t rows, int64_t d) {
  if (d <= kWarpCols)
    return std::min(ceil_div(rows, 3 * kWarps * 32 / row_lanes(d)), int64_t{kPlanCTAs} * 7);
  const int g = row_threads(d);
  return std::min(ceil_div(rows, 3), kPlanCTAs * std::max<int64_t>(1, 512 / g));
}
int64_t column_slabs(int64_t rows) { return std::min<int64_t>(ceil_div(rows, kSlabRows), 64); }

// Bytes of a kernel's rows on their way, and the most that a kernel of C columns a thread takes.
template <typename T, int kB, int C, int kSlots>
constexpr size_t slot_bytes(int threads, int parts) {
  return static_cast<size_t>(parts) * kSlots * Feed<T, kB, C, kSlots>::kBytes * threads;
}

template <typename T, int kB, bool kCta, bool kWide, int C>
cudaError_t run_norm_rows(const NormParams& p, int threads, int64_t units, cudaStream_t s) {
  static std::atomic<int> known[33];
  static PerDeviceOnce attr;
  const auto kernel = norm_kernel<T, kB, kCta, kWide, C>;
  constexpr int kMost = kWide ? 1024 : kCta ? 512 : 32 * kWarps;
  const size_t smem = slot_bytes<T, kB, C, kForwardSlots>(threads, 1);
  cudaError_t e = smem_attr_once(
      attr, kernel, static_cast<int>(slot_bytes<T, kB, C, kForwardSlots>(kMost, 1)));
  int64_t ctas = 0;
  if (e == cudaSuccess) e = resident_ctas(known, kernel, threads, smem, &ctas);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3(static_cast<unsigned>(std::min(units, ctas))), dim3(threads),
                          smem, s, p);
}

template <typename T, int kB>
cudaError_t run_norm(const NormParams& p, cudaStream_t s) {
  const int64_t units = ceil_div(p.rows, kWarps * 32 / p.lanes);       // of kernels without kCta
  if constexpr (kB != 4)
    if (p.d <= kShortCols) return run_norm_rows<T, kB, false, false, 8>(p, 32 * kWarps, units, s);
  if (p.d <= kWarpCols) return run_norm_rows<T, kB, false, false, kCols>(p, 32 * kWarps, units, s);
  // No barrier a row: 65,536 x 768 52 us, by CTAs 56; 65,536 x 640 38 and 44.  The backward
  // pass has no registers for it (32,768 x 1024 fp32 88 us, by CTAs 74).
  if constexpr (kB == 16)
    if (p.d <= kLongCols)
      return run_norm_rows<T, kB, false, false, 2 * kCols>(p, 32 * kWarps, units, s);
  if (p.d <= kMidCols) return run_norm_rows<T, kB, true, false, kCols>(p, row_threads(p.d), p.rows, s);
  return run_norm_rows<T, kB, true, true, kCols>(p, row_threads(p.d), p.rows, s);
}

template <typename T>
cudaError_t run_norm_any(const NormParams& p, cudaStream_t s) {
  if (p.d > kMaxCols)
    return launch_dependent(norm_loop_kernel<T>,
                            dim3(static_cast<unsigned>(std::min<int64_t>(p.rows, 4 * kPlanCTAs))),
                            dim3(kLoopThreads), 0, s, p);
  const auto fits = [&](size_t n) {
    return on_bytes(p.x, p.ld_x, sizeof(T), n) && on_bytes(p.y, p.ld_y, sizeof(T), n);
  };
  if (fits(16)) return run_norm<T, 16>(p, s);
  // Two 16-bit elements at once: 20,000 x 4090 82 us, by elements 121; up to 256 columns no faster
  // (100,000 x 90 26 us, by elements 23).
  if constexpr (sizeof(T) == 2)
    if (p.d > kShortCols && fits(4)) return run_norm<T, 4>(p, s);
  return run_norm<T, 0>(p, s);
}

template <typename T, int kB, bool kCta, bool kWide, int C>
cudaError_t run_backward_rows(const GradParams& p, int64_t* parts, int threads, cudaStream_t s) {
  const auto kernel = norm_backward_kernel<T, kB, kCta, kWide, C>;
  constexpr int kMost = kWide ? 1024 : kCta ? 512 : 32 * kWarps;
  const auto bytes = [](int n) {
    if (kWide) return 3 * kCols * sizeof(float) * n;
    const size_t sums = kCta ? 0 : 2 * 32 * C * sizeof(float);
    return std::max(sums, slot_bytes<T, kB, C, kBackwardSlots>(n, 2));
  };
  static std::atomic<int> known[33];
  static PerDeviceOnce attr;
  cudaError_t e = smem_attr_once(attr, kernel, static_cast<int>(bytes(kMost)));
  int64_t ctas = 0;
  if (e == cudaSuccess) e = resident_ctas(known, kernel, threads, bytes(threads), &ctas);
  if (e != cudaSuccess) return e;
  *parts = std::min(*parts, ctas);
  return launch_dependent(kernel, dim3(static_cast<unsigned>(*parts)), dim3(threads), bytes(threads),
                          s, p);
}

template <typename T, int kB>
cudaError_t run_backward(const GradParams& p, int64_t* parts, cudaStream_t s) {
  if constexpr (kB != 4)
    if (p.d <= kShortCols) return run_backward_rows<T, kB, false, false, 8>(p, parts, 32 * kWarps, s);
  if (p.d <= kWarpCols) return run_backward_rows<T, kB, false, false, kCols>(p, parts, 32 * kWarps, s);
  if (p.d <= kMidCols) return run_backward_rows<T, kB, true, false, kCols>(p, parts, row_threads(p.d), s);
  return run_backward_rows<T, kB, true, true, kCols>(p, parts, row_threads(p.d), s);
}

template <typename T>
cudaError_t run_backward_any(const GradParams& p, int64_t* parts, cudaStream_t s) {
  if (p.d > kMaxCols) {
    // the column sums first: dx may take the place of x or dy
    if (p.part != nullptr) {
      const dim3 grid(static_cast<unsigned>(ceil_div(p.d, 128)), static_cast<unsigned>(*parts));
      const cudaError_t e = launch_dependent(norm_columns_kernel<T>, grid, dim3(128), 0, s, p);
      if (e != cudaSuccess) return e;
    }
    return launch_dependent(norm_backward_loop_kernel<T>,
                            dim3(static_cast<unsigned>(std::min<int64_t>(p.rows, 4 * kPlanCTAs))),
                            dim3(kLoopThreads), 0, s, p);
  }
  const auto fits = [&](size_t n) {
    return on_bytes(p.x, p.ld_x, sizeof(T), n) && on_bytes(p.dy, p.ld_dy, sizeof(T), n) &&
           on_bytes(p.dx, p.ld_dx, sizeof(T), n);
  };
  if (fits(16)) return run_backward<T, 16>(p, parts, s);
  // as the forward pass: 5000 x 10,002 119 us, by elements 146; 100,000 x 90 35, by elements 31
  if constexpr (sizeof(T) == 2)
    if (p.d > kShortCols && fits(4)) return run_backward<T, 4>(p, parts, s);
  return run_backward<T, 0>(p, parts, s);
}

int64_t backward_parts(int64_t rows, int64_t d) {
  return d > kMaxCols ? column_slabs(rows) : backward_ctas(rows, d);
}

}  // namespace

cudaError_t launch_norm(const bergson_norm_args& a, cudaStream_t s) {
  NormParams p = {};
  p.x = a.x;
  p.w = a.weight;
  p.b = a.bias;
  p.y = a.y;
  p.mean = a.mean;
  p.rstd = a.rstd;
  p.rows = a.rows;
  p.d = a.d;
  p.ld_x = a.ld_x;
  p.ld_y = a.ld_y;
  p.lanes = row_lanes(a.d);
  p.wt = a.w_dtype;
  p.layer = a.kind == BERGSON_NORM_LAYER ? 1 : 0;
  p.eps = static_cast<float>(a.eps);
  p.inv_d = static_cast<float>(1.0 / static_cast<double>(a.d));
  if (a.dtype == BERGSON_BF16) return run_norm_any<__nv_bfloat16>(p, s);
  if (a.dtype == BERGSON_F16) return run_norm_any<__half>(p, s);
  return run_norm_any<float>(p, s);
}

size_t norm_backward_workspace(int64_t rows, int64_t d) {
  const size_t bytes = static_cast<size_t>(backward_parts(rows, d)) * 2 * d * sizeof(float);
  return std::max<size_t>(256, (bytes + 255) / 256 * 256);
}

cudaError_t launch_norm_backward(const bergson_norm_grad_args& a, void* ws, cudaStream_t s) {
  const bool sums = a.d_weight != nullptr || a.d_bias != nullptr;
  if (a.rows == 0) {
    cudaError_t e = cudaSuccess;
    if (a.d_weight != nullptr) e = cudaMemsetAsync(a.d_weight, 0, a.d * sizeof(float), s);
    if (e == cudaSuccess && a.d_bias != nullptr) e = cudaMemsetAsync(a.d_bias, 0, a.d * sizeof(float), s);
    return e;
  }
  int64_t parts = backward_parts(a.rows, a.d);
  GradParams p = {};
  p.x = a.x;
  p.w = a.weight;
  p.mean = a.mean;
  p.rstd = a.rstd;
  p.dy = a.dy;
  p.dx = a.dx;
  p.part = sums ? static_cast<float*>(ws) : nullptr;
  p.rows = a.rows;
  p.d = a.d;
  p.ld_x = a.ld_x;
  p.ld_dy = a.ld_dy;
  p.ld_dx = a.ld_dx;
  p.lanes = row_lanes(a.d);
  p.wt = a.w_dtype;
  p.layer = a.kind == BERGSON_NORM_LAYER ? 1 : 0;
  p.inv_d = static_cast<float>(1.0 / static_cast<double>(a.d));
  cudaError_t e = a.dtype == BERGSON_BF16  ? run_backward_any<__nv_bfloat16>(p, &parts, s)
                  : a.dtype == BERGSON_F16 ? run_backward_any<__half>(p, &parts, s)
                                           : run_backward_any<float>(p, &parts, s);
  if (e != cudaSuccess || !sums) return e;
  const dim3 grid(static_cast<unsigned>(ceil_div(a.d, 32)), 2);
  return launch_dependent(norm_parts_kernel, grid, dim3(32 * kPartWarps), 0, s,
                          static_cast<const float*>(ws), static_cast<int>(parts), a.d, a.d_weight, a.d_bias);
}

}  // namespace bergson
