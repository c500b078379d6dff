// Factored second moments of AdamW's v: the row and column means of every
// matrix, in one pass over tiles and a second small one over their sums.

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMostRows = 32, kLeastRows = 4;  // rows a warp takes (a power of two between)
constexpr int kRows = 4;                       // of them on the way at once
constexpr int kTileCtas = 3;
constexpr int kStrip = 256;                    // columns of a tile, 8 a lane
constexpr int kFew = 24, kMany = 300;          // records a launch can take

struct Entry {
  const void* v;
  const float* vs;
  int64_t rows, cols;
  float* r;
  float* c;
  float* row_part;             // [strips, rows]
  float* col_part;             // [bands, cols]
  float* tile_part;            // [bands, strips]
  int bands, strips;           // tiles of kWarps warp_rows rows and kStrip columns
  int warp_rows;
  int st;
  int vec;                     // rows start on boundaries of a lane's 8 elements
};

template <int N>
struct MomentParams {
  float correction, floor;
  int n;
  uint32_t tiles[N + 1];               // first CTA of each matrix in the first pass
  uint32_t outs[N + 1];                // ... and in the second
  Entry e[N];
};

__device__ __forceinline__ int find(const uint32_t* begin, int n, uint32_t at) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (begin[mid] <= at) lo = mid; else hi = mid;
  }
  return lo;
}

// The sums over the lanes of each of N values: lane l has that of value l / (32 / N).
template <int N>
__device__ __forceinline__ float sum_each(float (&x)[N]) {
  const int lane = threadIdx.x & 31;
  int o = 16;
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2) {
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const float give = up ? x[k] : x[k + n];
      x[k] = (up ? x[k + n] : x[k]) + __shfl_xor_sync(0xffffffffu, give, o);
    }
    o /= 2;
  }
  float t = x[0];
  for (; o > 0; o /= 2) t += __shfl_xor_sync(0xffffffffu, t, o);
  return t;
}

// A warp's rows r0 .. r0 + e.warp_rows of a tile: lane sums of the columns in col[], the
// rows' sums to row_part.  Vectors: columns c0 + 8 lane + k; else c0 + lane + 32 k.
template <bool kEight, bool kVec>
__device__ __forceinline__ void take_rows(const Entry& e, int64_t r0, int64_t c0, float* row_part,
                                          float (&col)[8]) {
  const int lane = threadIdx.x & 31;
  float2 col2[4] = {};
#pragma unroll 1
  for (int64_t r = r0; r < r0 + e.warp_rows && r < e.rows; r += kRows) {
    float sums[kRows];
    if constexpr (kVec && !kEight) {
      uint32_t x[kRows][8];
      const int64_t c = c0 + 8 * lane;
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[k][j] = 0;
        if (r + k < e.rows && c < e.cols)
          load32(static_cast<const float*>(e.v) + (r + k) * e.cols + c, x[k]);
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        float2 s = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 y = make_float2(__uint_as_float(x[k][2 * j]), __uint_as_float(x[k][2 * j + 1]));
          col2[j] = add2(col2[j], y);
          s = add2(s, y);
        }
        sums[k] = s.x + s.y;
      }
    } else if constexpr (kVec) {
      uint2 u[kRows];
      float sc[kRows];
      const int64_t c = c0 + 8 * lane;
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        u[k] = make_uint2(0, 0);
        sc[k] = 0.0f;
        if (r + k < e.rows && c < e.cols) {
          const int64_t i = (r + k) * e.cols + c;
          u[k] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(e.v) + i);
          sc[k] = e.vs[i / kStateBlock];
        }
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        float y[8];
        decode_second4(u[k].x, y);
        decode_second4(u[k].y, y + 4);
        float2 s = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 y2 = make_float2(y[2 * j], y[2 * j + 1]);
          col2[j] = fma2(y2, pair(sc[k]), col2[j]);
          s = add2(s, y2);
        }
        sums[k] = (s.x + s.y) * sc[k];
      }
    } else {
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        float y[8];
        const int64_t row = (r + k) * e.cols;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int64_t c = c0 + lane + 32 * j;
          y[j] = 0.0f;
          if (r + k < e.rows && c < e.cols)
            y[j] = kEight ? decode_second(static_cast<const uint8_t*>(e.v)[row + c]) *
                                e.vs[(row + c) / kStateBlock]
                          : static_cast<const float*>(e.v)[row + c];
        }
        float2 s = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 y2 = make_float2(y[2 * j], y[2 * j + 1]);
          col2[j] = add2(col2[j], y2);
          s = add2(s, y2);
        }
        sums[k] = s.x + s.y;
      }
    }
    const float t = sum_each(sums);
    const int k = lane / (32 / kRows);
    if (lane % (32 / kRows) == 0 && r + k < e.rows) row_part[r + k] = t;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    col[2 * j] = col2[j].x;
    col[2 * j + 1] = col2[j].y;
  }
}

template <int N>
__global__ void __launch_bounds__(kThreads, kTileCtas) moment_tiles_kernel(
    const __grid_constant__ MomentParams<N> p) {
  __shared__ float cols[kWarps][kStrip];
  __shared__ float red[kWarps];
  const int at = find(p.tiles, p.n, blockIdx.x);
  const Entry& e = p.e[at];
  const uint32_t tile = blockIdx.x - p.tiles[at];
  griddep_wait();
  const int band = tile / e.strips, strip = tile % e.strips;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t r0 = (static_cast<int64_t>(band) * kWarps + warp) * e.warp_rows;
  const int64_t c0 = static_cast<int64_t>(strip) * kStrip;
  float* row_part = e.row_part + static_cast<int64_t>(strip) * e.rows;
  float col[8];
  if (e.st == BERGSON_STATE_8BIT) {
    if (e.vec) take_rows<true, true>(e, r0, c0, row_part, col);
    else take_rows<true, false>(e, r0, c0, row_part, col);
  } else {
    if (e.vec) take_rows<false, true>(e, r0, c0, row_part, col);
    else take_rows<false, false>(e, r0, c0, row_part, col);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) cols[warp][e.vec ? 8 * lane + j : lane + 32 * j] = col[j];
  __syncthreads();
  float x = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) x += cols[w][threadIdx.x];
  const int64_t c = c0 + threadIdx.x;
  if (c < e.cols) e.col_part[static_cast<int64_t>(band) * e.cols + c] = x;
  x = block_sum(x, red);
  if (threadIdx.x == 0) e.tile_part[tile] = x;
}
static_assert(kStrip == kThreads, "a thread sums a column of the tile");

template <int N>
__global__ void __launch_bounds__(kThreads) moment_finish_kernel(
    const __grid_constant__ MomentParams<N> p) {
  __shared__ float red[kWarps];
  const int at = find(p.outs, p.n, blockIdx.x);
  const Entry& e = p.e[at];
  const int64_t i = static_cast<int64_t>(blockIdx.x - p.outs[at]) * kThreads + threadIdx.x;
  griddep_wait();
  const bool row = i < e.rows;
  const int64_t j = i - e.rows;
  CompensatedSum x;
  if (row || j < e.cols) {
    const float* part = row ? e.row_part + i : e.col_part + j;
    const int64_t step = row ? e.rows : e.cols;
    const int n = row ? e.strips : e.bands;
    for (int k = 0; k < n; k += 8) {
      float v[8];
#pragma unroll
      for (int o = 0; o < 8; ++o) v[o] = k + o < n ? part[(k + o) * step] : 0.0f;
#pragma unroll
      for (int o = 0; o < 8; ++o) x.add(v[o]);
    }
  }
  CompensatedSum sum;
  const int64_t tiles = static_cast<int64_t>(e.bands) * e.strips;
  for (int64_t k = threadIdx.x; k < tiles; k += kThreads) sum.add(e.tile_part[k]);
  const float all = block_sum(sum.s, red);
  const float rows = static_cast<float>(e.rows), cols = static_cast<float>(e.cols);
  if (row) e.r[i] = x.s / cols * p.correction + p.floor;
  else if (j < e.cols)
    e.c[j] = (x.s / rows * p.correction + p.floor) / (all / rows / cols * p.correction + p.floor);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rows a warp takes of a matrix, by its own size alone (so that its sums are the same
// in any company): as many as leave kTilesWanted tiles.
constexpr int64_t kTilesWanted = 64;
int warp_rows_of(const bergson_moment_matrix& m) {
  int rows = kMostRows;
  while (rows > kLeastRows &&
         ceil_div(m.d_out, kWarps * rows) * ceil_div(m.d_in, kStrip) < kTilesWanted)
    rows /= 2;
  return rows;
}

size_t floats_of(const bergson_moment_matrix& m) {
  const size_t bands = ceil_div(m.d_out, kWarps * warp_rows_of(m));
  const size_t strips = ceil_div(m.d_in, kStrip);
  return strips * m.d_out + bands * m.d_in + bands * strips;
}

template <int N>
cudaError_t run_moments(const bergson_moment_matrix* m, int n, double correction, double floor,
                        void* ws, cudaStream_t s) {
  MomentParams<N> p;
  p.correction = static_cast<float>(correction);
  p.floor = static_cast<float>(floor);
  int k = 0;
  p.tiles[0] = p.outs[0] = 0;
  float* at = static_cast<float*>(ws);
  const auto flush = [&]() -> cudaError_t {
    if (k == 0) return cudaSuccess;
    p.n = k;
    const cudaError_t e = launch_dependent(moment_tiles_kernel<N>, dim3(p.tiles[k]),
                                           dim3(kThreads), 0, s, p);
    if (e != cudaSuccess) return e;
    const dim3 grid(p.outs[k]);
    k = 0;
    return launch_dependent(moment_finish_kernel<N>, grid, dim3(kThreads), 0, s, p);
  };
  for (int i = 0; i < n; ++i) {
    const int warp_rows = warp_rows_of(m[i]);
    const int64_t bands = ceil_div(m[i].d_out, kWarps * warp_rows);
    const int64_t strips = ceil_div(m[i].d_in, kStrip);
    const int64_t outs = ceil_div(m[i].d_out + m[i].d_in, kThreads);
    if (k == N ||
        (k > 0 && (p.tiles[k] + bands * strips > INT32_MAX || p.outs[k] + outs > INT32_MAX))) {
      const cudaError_t e = flush();
      if (e != cudaSuccess) return e;
    }
    Entry& e = p.e[k];
    e.v = m[i].v;
    e.vs = m[i].v_scale;
    e.rows = m[i].d_out;
    e.cols = m[i].d_in;
    e.r = m[i].r;
    e.c = m[i].c;
    e.st = m[i].state_kind;
    e.vec = m[i].d_in % 8 == 0 &&
            reinterpret_cast<uintptr_t>(m[i].v) % (e.st == BERGSON_STATE_8BIT ? 8 : 32) == 0;
    e.warp_rows = warp_rows;
    e.bands = static_cast<int>(bands);
    e.strips = static_cast<int>(strips);
    e.row_part = at;
    e.col_part = e.row_part + strips * e.rows;
    e.tile_part = e.col_part + bands * e.cols;
    at = e.tile_part + bands * strips;
    p.tiles[k + 1] = p.tiles[k] + static_cast<uint32_t>(bands * strips);
    p.outs[k + 1] = p.outs[k] + static_cast<uint32_t>(outs);
    ++k;
  }
  return flush();
}

}  // namespace

size_t moments_workspace(const bergson_moment_matrix* m, int n) {
  size_t total = 0;
  for (int i = 0; i < n; ++i) total += floats_of(m[i]);
  return (total * sizeof(float) + 255) / 256 * 256 + 256;
}

cudaError_t launch_factor_moments(const bergson_moment_matrix* m, int n, double correction,
                                  double floor, void* ws, cudaStream_t s) {
  return n <= kFew ? run_moments<kFew>(m, n, correction, floor, ws, s)
                   : run_moments<kMany>(m, n, correction, floor, ws, s);
}

}  // namespace bergson
