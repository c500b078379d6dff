// Layer norm (and its form without a mean), forward and backward.
//
//   forward   y = (x - mu) rstd w + b,   rstd = (mean (x - mu)^2 + eps)^-1/2
//   backward  h = dy w,  n = (x - mu) rstd,
//             dx = rstd (h - mean h - n mean (h n)),  dw = sum_r dy n,  db = sum_r dy
//
// (mu = 0 and no mean of h without a mean).  Both are bound by their bytes: a
// row is read once, stays in the registers of the 4 .. 32 lanes (up to 512 columns)
// or the CTA that have it, 8 or 16 columns a thread, and the next row's loads are on their way while this
// one is reduced.  A thread keeps its columns from row to row, so that weights are
// loaded once a CTA and the backward pass sums dw and db in registers; one row
// of both a CTA goes to the workspace, and a second kernel adds these up in order.

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kCols = 16;                      // columns a thread
constexpr int kShortCols = 32 * 8;             // up to here 8 columns a lane, as few lanes as do
constexpr int kWarpCols = 32 * kCols;          // up to here a warp takes a row
constexpr int kWarps = 4;                      // warps of such a CTA
constexpr int kMidCols = 8192;                 // up to here dw, db and the next row stay in registers
constexpr int kMaxCols = 16384;                // up to here a row stays in registers
constexpr int kLoopThreads = 512;              // of the kernels for longer rows
constexpr int kSlabRows = 512;                 // rows of a CTA that sums columns of such rows

// Sums over the threads that share a row, in each of them: G lanes side by side, or the
// CTA by way of `red` (32 values each, not in use by the row before or after).
template <bool kCta, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int G, float* red) {
  if constexpr (!kCta) {
    for (int o = G >> 1; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) red[32 * i + (threadIdx.x >> 5)] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < warps ? red[32 * i + lane] : 0.0f);
  }
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

template <typename T, bool kVec, bool kCta, bool kWide, int C>
__global__ void __launch_bounds__(kWide ? 1024 : kCta ? 512 : 32 * kWarps)
    norm_kernel(const __grid_constant__ NormParams p) {
  using R = RowPart<T, kVec, C>;
  __shared__ float red[2][2][32];
  const Turns u = turns<kCta>(p.lanes);
  const int G = u.G, t = u.t, d = static_cast<int>(p.d);
  griddep_wait();
  float w[C], b[C];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = R::column(t, G, i);
    w[i] = p.w != nullptr && c < d ? load_any(p.w, p.wt, c) : 1.0f;
    b[i] = p.b != nullptr && c < d ? load_any(p.b, p.wt, c) : 0.0f;
  }
  const T* xs = static_cast<const T*>(p.x);
  R next;
  const auto fetch = [&](int64_t r) { next.load(xs + r * p.ld_x, r < p.rows ? d : 0, t, G); };
  fetch(u.first + u.sub);
  int turn = 0;
  for (int64_t first = u.first; first < p.rows; first += u.step, turn ^= 1) {
    const int64_t r = first + u.sub;
    const R row = next;
    fetch(r + u.step);
    float x[C];
    row.floats(x);
    float mean = 0.0f;
    if (p.layer) {
      float s[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < C; ++i) s[0] += x[i];
      row_sums<kCta>(s, G, red[turn][0]);
      mean = s[0] * p.inv_d;
#pragma unroll
      for (int i = 0; i < C; ++i) x[i] = R::column(t, G, i) < d ? x[i] - mean : 0.0f;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < C; ++i) q[0] = fmaf(x[i], x[i], q[0]);
    row_sums<kCta>(q, G, red[turn][1]);
    const float rstd = __frcp_rn(__fsqrt_rn(fmaf(q[0], p.inv_d, p.eps)));
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = fmaf(x[i] * rstd, w[i], b[i]);
    R::store(static_cast<T*>(p.y) + r * p.ld_y, r < p.rows ? d : 0, t, G, x);
    if (t == 0 && r < p.rows) {
      if (p.mean != nullptr && p.layer) p.mean[r] = mean;
      if (p.rstd != nullptr) p.rstd[r] = rstd;
    }
  }
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
    const float rstd = __frcp_rn(__fsqrt_rn(fmaf(block_sum(q.s, red[1]), p.inv_d, p.eps)));
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
template <typename T, bool kVec, bool kCta, bool kWide, int C>
__global__ void __launch_bounds__(kWide ? 1024 : kCta ? 512 : 32 * kWarps)
    norm_backward_kernel(const __grid_constant__ GradParams p) {
  using R = RowPart<T, kVec, C>;
  __shared__ float red[2][64];
  extern __shared__ float wide[];              // kWide: weights, dw, db; warps of rows: [2, d] to add up
  const Turns u = turns<kCta>(p.lanes);
  const int G = u.G, t = u.t, d = static_cast<int>(p.d);
  griddep_wait();
  // where thread t's value i stands in shared memory: neighbouring threads side by side
  const auto at = [&](int i) { return i * G + t; };
  const int n = C * G;
  float w[kWide ? 1 : C], dw[kWide ? 1 : C], db[kWide ? 1 : C];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = R::column(t, G, i);
    const float v = p.w != nullptr && c < d ? load_any(p.w, p.wt, c) : 1.0f;
    if constexpr (kWide) {
      wide[at(i)] = v;
      wide[n + at(i)] = wide[2 * n + at(i)] = 0.0f;
    } else {
      w[i] = v;
      dw[i] = db[i] = 0.0f;
    }
  }
  const T* xs = static_cast<const T*>(p.x);
  const T* dys = static_cast<const T*>(p.dy);
  R nx, ny;
  float mean_next = 0.0f, rstd_next = 0.0f;
  const auto fetch = [&](int64_t row) {
    const bool in = row < p.rows;
    nx.load(xs + row * p.ld_x, in ? d : 0, t, G);
    ny.load(dys + row * p.ld_dy, in ? d : 0, t, G);
    if (p.layer) mean_next = in ? p.mean[row] : 0.0f;
    rstd_next = in ? p.rstd[row] : 0.0f;
  };
  fetch(u.first + u.sub);
  int turn = 0;
  for (int64_t first = u.first; first < p.rows; first += u.step, turn ^= 1) {
    const int64_t r = first + u.sub;
    float x[C], g[C];
    nx.floats(x);
    ny.floats(g);
    const float mean = mean_next, rstd = rstd_next;
    if constexpr (!kWide) fetch(r + u.step);
    float s[2] = {0.0f, 0.0f};                 // of h n and h
#pragma unroll
    for (int i = 0; i < C; ++i) {
      x[i] = R::column(t, G, i) < d ? (x[i] - mean) * rstd : 0.0f;
      if constexpr (kWide) {
        wide[n + at(i)] = fmaf(g[i], x[i], wide[n + at(i)]);
        wide[2 * n + at(i)] += g[i];
        g[i] *= wide[at(i)];
      } else {
        dw[i] = fmaf(g[i], x[i], dw[i]);
        db[i] += g[i];
        g[i] *= w[i];
      }
      s[0] = fmaf(g[i], x[i], s[0]);
      s[1] += g[i];
    }
    row_sums<kCta>(s, G, red[turn]);
    const float along = s[0] * p.inv_d, level = p.layer ? s[1] * p.inv_d : 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = rstd * (g[i] - fmaf(x[i], along, level));
    R::store(static_cast<T*>(p.dx) + r * p.ld_dx, r < p.rows ? d : 0, t, G, x);
    if constexpr (kWide) fetch(r + u.step);
  }
  if (p.part == nullptr) return;
  float* part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * d;
  if constexpr (kWide) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = R::column(t, G, i);
      if (c < d) {
        part[c] = wide[n + at(i)];
        part[d + c] = wide[2 * n + at(i)];
      }
    }
  } else if constexpr (kCta) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = R::column(t, G, i);
      if (c < d) {
        part[c] = dw[i];
        part[d + c] = db[i];
      }
    }
  } else {
    for (int o = G; o < 32; o <<= 1) {         // the warp's rows
#pragma unroll
      for (int i = 0; i < C; ++i) {
        dw[i] += __shfl_xor_sync(0xffffffffu, dw[i], o);
        db[i] += __shfl_xor_sync(0xffffffffu, db[i], o);
      }
    }
    const int warp = threadIdx.x >> 5;         // one warp after the other: a fixed order
    for (int k = 0; k < kWarps; ++k) {
      if (warp == k && u.sub == 0) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const int c = R::column(t, G, i);
          if (c < d) {
            wide[c] = k == 0 ? dw[i] : wide[c] + dw[i];
            wide[d + c] = k == 0 ? db[i] : wide[d + c] + db[i];
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

// dw and db from the CTAs' sums: 32 columns a CTA, its 8 warps every eighth of them.
__global__ void __launch_bounds__(256) norm_parts_kernel(const float* __restrict__ part, int n,
                                                         int64_t d, float* dw, float* db) {
  __shared__ float red[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
  float* out = blockIdx.y == 0 ? dw : db;
  griddep_wait();
  if (out == nullptr) return;
  const float* p = part + blockIdx.y * d + c;
  float s = 0.0f;
  if (c < d) {
#pragma unroll 8
    for (int k = warp; k < n; k += 8) s += p[2 * d * k];
  }
  red[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < d) {
    float t = red[0][lane];
#pragma unroll
    for (int k = 1; k < 8; ++k) t += red[k][lane];
    out[c] = t;
  }
}

// Threads that share a row of the CTA kernels.
int row_threads(int64_t d) { return static_cast<int>(ceil_div(ceil_div(d, kCols), 32) * 32); }

// Lanes that share a row of up to kWarpCols columns.
int row_lanes(int64_t d) {
  int lanes = 32;
  while (lanes > 4 && d <= 4 * lanes) lanes /= 2;
  return lanes;
}

// CTAs of the kernels whose CTAs go over the rows: as many as are resident.
int64_t forward_ctas(int64_t rows, int64_t d) {
  if (d <= kWarpCols)
    return std::min(ceil_div(rows, kWarps * 32 / row_lanes(d)), int64_t{kPlanCTAs} * 8);
  const int g = row_threads(d);
  return std::min(rows, kPlanCTAs * std::max<int64_t>(1, 896 / g));
}
int64_t backward_ctas(int64_t rows, int64_t d) {
  if (d <= kWarpCols)
    return std::min(ceil_div(rows, kWarps * 32 / row_lanes(d)), int64_t{kPlanCTAs} * 5);
  const int g = row_threads(d);
  return std::min(rows, kPlanCTAs * std::max<int64_t>(1, 512 / g));
}
int64_t column_slabs(int64_t rows) { return std::min<int64_t>(ceil_div(rows, kSlabRows), 64); }

template <typename T, bool kVec>
cudaError_t run_norm(const NormParams& p, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>(forward_ctas(p.rows, p.d)));
  if (p.d <= kShortCols)
    return launch_dependent(norm_kernel<T, kVec, false, false, 8>, grid, dim3(32 * kWarps), 0, s,
                            p);
  if (p.d <= kWarpCols)
    return launch_dependent(norm_kernel<T, kVec, false, false, kCols>, grid, dim3(32 * kWarps), 0,
                            s, p);
  const auto kernel = p.d <= kMidCols ? norm_kernel<T, kVec, true, false, kCols>
                                      : norm_kernel<T, kVec, true, true, kCols>;
  return launch_dependent(kernel, grid, dim3(row_threads(p.d)), 0, s, p);
}

template <typename T>
cudaError_t run_norm_any(const NormParams& p, cudaStream_t s) {
  if (p.d > kMaxCols)
    return launch_dependent(norm_loop_kernel<T>,
                            dim3(static_cast<unsigned>(std::min<int64_t>(p.rows, 4 * kPlanCTAs))),
                            dim3(kLoopThreads), 0, s, p);
  const bool vec = on16(p.x, p.ld_x, sizeof(T)) && on16(p.y, p.ld_y, sizeof(T));
  return vec ? run_norm<T, true>(p, s) : run_norm<T, false>(p, s);
}

template <typename T, bool kVec, bool kWide>
cudaError_t run_backward_cta(const GradParams& p, dim3 grid, size_t smem, cudaStream_t s) {
  const auto kernel = norm_backward_kernel<T, kVec, true, kWide, kCols>;
  if (kWide) {
    static PerDeviceOnce attr;
    const cudaError_t e = smem_attr_once(attr, kernel, 3 * kMaxCols * sizeof(float));
    if (e != cudaSuccess) return e;
  }
  return launch_dependent(kernel, grid, dim3(row_threads(p.d)), smem, s, p);
}

template <typename T, bool kVec>
cudaError_t run_backward(const GradParams& p, int64_t ctas, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>(ctas));
  const size_t sums = 2 * p.d * sizeof(float);
  if (p.d <= kShortCols)
    return launch_dependent(norm_backward_kernel<T, kVec, false, false, 8>, grid,
                            dim3(32 * kWarps), sums, s, p);
  if (p.d <= kWarpCols)
    return launch_dependent(norm_backward_kernel<T, kVec, false, false, kCols>, grid,
                            dim3(32 * kWarps), sums, s, p);
  if (p.d <= kMidCols) return run_backward_cta<T, kVec, false>(p, grid, 0, s);
  return run_backward_cta<T, kVec, true>(
      p, grid, 3 * kCols * static_cast<size_t>(row_threads(p.d)) * sizeof(float), s);
}

template <typename T>
cudaError_t run_backward_any(const GradParams& p, int64_t parts, cudaStream_t s) {
  if (p.d > kMaxCols) {
    // the column sums first: dx may take the place of x or dy
    if (p.part != nullptr) {
      const dim3 grid(static_cast<unsigned>(ceil_div(p.d, 128)), static_cast<unsigned>(parts));
      const cudaError_t e = launch_dependent(norm_columns_kernel<T>, grid, dim3(128), 0, s, p);
      if (e != cudaSuccess) return e;
    }
    return launch_dependent(norm_backward_loop_kernel<T>,
                            dim3(static_cast<unsigned>(std::min<int64_t>(p.rows, 4 * kPlanCTAs))),
                            dim3(kLoopThreads), 0, s, p);
  }
  const bool vec = on16(p.x, p.ld_x, sizeof(T)) && on16(p.dy, p.ld_dy, sizeof(T)) &&
                   on16(p.dx, p.ld_dx, sizeof(T));
  return vec ? run_backward<T, true>(p, parts, s) : run_backward<T, false>(p, parts, s);
}

int64_t backward_parts(int64_t rows, int64_t d) {
  return d > kMaxCols ? column_slabs(rows) : backward_ctas(rows, d);
}

}  // namespace

cudaError_t launch_norm(const NormArgs& a, cudaStream_t s) {
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

cudaError_t launch_norm_backward(const NormGradArgs& a, void* ws, cudaStream_t s) {
  const bool sums = a.dw != nullptr || a.db != nullptr;
  if (a.rows == 0) {
    cudaError_t e = cudaSuccess;
    if (a.dw != nullptr) e = cudaMemsetAsync(a.dw, 0, a.d * sizeof(float), s);
    if (e == cudaSuccess && a.db != nullptr) e = cudaMemsetAsync(a.db, 0, a.d * sizeof(float), s);
    return e;
  }
  const int64_t parts = backward_parts(a.rows, a.d);
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
  cudaError_t e = a.dtype == BERGSON_BF16  ? run_backward_any<__nv_bfloat16>(p, parts, s)
                  : a.dtype == BERGSON_F16 ? run_backward_any<__half>(p, parts, s)
                                           : run_backward_any<float>(p, parts, s);
  if (e != cudaSuccess || !sums) return e;
  const dim3 grid(static_cast<unsigned>(ceil_div(a.d, 32)), 2);
  return launch_dependent(norm_parts_kernel, grid, dim3(256), 0, s,
                          static_cast<const float*>(ws), static_cast<int>(parts), a.d, a.dw, a.db);
}

}  // namespace bergson
