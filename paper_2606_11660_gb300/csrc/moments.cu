// Factored second moments of AdamW's v: the row and column means of every
// matrix, in one pass over tiles and a second small one over their sums.

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kBand = 64;                      // rows of a tile
constexpr int kStrip = kThreads;               // columns of a tile
constexpr int kMaxEntries = 300;

struct Entry {
  const void* v;
  const float* vs;
  int64_t rows, cols;
  float* r;
  float* c;
  float* row_part;             // [strips, rows]
  float* col_part;             // [bands, cols]
  float* tile_part;            // [bands, strips]
  int bands, strips;
  int st, pad;
};

struct MomentParams {
  Entry e[kMaxEntries];
  uint32_t tiles[kMaxEntries + 1];
  uint32_t outs[kMaxEntries + 1];      // CTAs of the second pass
  int n;
  float correction, floor;
};

__device__ __forceinline__ int find(const uint32_t* begin, int n, uint32_t at) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (begin[mid] <= at) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kThreads) moment_tiles_kernel(
    const __grid_constant__ MomentParams p) {
  __shared__ float rows[kWarps][kBand];
  __shared__ float red[kWarps];
  const Entry& e = p.e[find(p.tiles, p.n, blockIdx.x)];
  const uint32_t tile = blockIdx.x - p.tiles[find(p.tiles, p.n, blockIdx.x)];
  const int band = tile / e.strips, strip = tile % e.strips;
  const int64_t c = static_cast<int64_t>(strip) * kStrip + threadIdx.x;
  const int64_t r0 = static_cast<int64_t>(band) * kBand;
  float col = 0.0f;
  for (int k = 0; k < kBand; ++k) {
    float x = 0.0f;
    if (r0 + k < e.rows && c < e.cols) {
      const int64_t i = (r0 + k) * e.cols + c;
      x = e.st == BERGSON_STATE_8BIT
              ? __fmul_rn(decode_second(static_cast<const uint8_t*>(e.v)[i]), e.vs[i / kStateBlock])
              : static_cast<const float*>(e.v)[i];
    }
    col += x;
    x = warp_sum(x);
    if ((threadIdx.x & 31) == 0) rows[threadIdx.x >> 5][k] = x;
  }
  if (c < e.cols) e.col_part[static_cast<int64_t>(band) * e.cols + c] = col;
  __syncthreads();
  if (threadIdx.x < kBand && r0 + threadIdx.x < e.rows) {
    float x = 0.0f;
    for (int w = 0; w < kWarps; ++w) x += rows[w][threadIdx.x];
    e.row_part[static_cast<int64_t>(strip) * e.rows + r0 + threadIdx.x] = x;
  }
  const float all = block_sum(col, red);
  if (threadIdx.x == 0) e.tile_part[tile] = all;
}

__global__ void __launch_bounds__(kThreads) moment_finish_kernel(
    const __grid_constant__ MomentParams p) {
  __shared__ float red[kWarps];
  const int at = find(p.outs, p.n, blockIdx.x);
  const Entry& e = p.e[at];
  const int64_t i = static_cast<int64_t>(blockIdx.x - p.outs[at]) * kThreads + threadIdx.x;
  CompensatedSum sum;
  for (int64_t k = threadIdx.x; k < static_cast<int64_t>(e.bands) * e.strips; k += kThreads)
    sum.add(e.tile_part[k]);
  const float all = block_sum(sum.s, red);
  const float rows = static_cast<float>(e.rows), cols = static_cast<float>(e.cols);
  const float mean = all / rows / cols * p.correction + p.floor;
  if (i < e.rows) {
    CompensatedSum x;
    for (int k = 0; k < e.strips; ++k) x.add(e.row_part[k * e.rows + i]);
    e.r[i] = x.s / cols * p.correction + p.floor;
  } else if (i - e.rows < e.cols) {
    const int64_t j = i - e.rows;
    CompensatedSum x;
    for (int k = 0; k < e.bands; ++k) x.add(e.col_part[k * e.cols + j]);
    e.c[j] = (x.s / rows * p.correction + p.floor) / mean;
  }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

size_t floats_of(const bergson_moment_matrix& m) {
  const size_t bands = ceil_div(m.d_out, kBand), strips = ceil_div(m.d_in, kStrip);
  return strips * m.d_out + bands * m.d_in + bands * strips;
}

}  // namespace

size_t moments_workspace(const bergson_moment_matrix* m, int n) {
  size_t total = 0;
  for (int i = 0; i < n; ++i) total += floats_of(m[i]);
  return (total * sizeof(float) + 255) / 256 * 256 + 256;
}

cudaError_t launch_factor_moments(const bergson_moment_matrix* m, int n, double correction,
                                  double floor, void* ws, cudaStream_t s) {
  MomentParams p;
  p.correction = static_cast<float>(correction);
  p.floor = static_cast<float>(floor);
  p.n = 0;
  p.tiles[0] = p.outs[0] = 0;
  float* at = static_cast<float*>(ws);
  const auto flush = [&]() -> cudaError_t {
    if (p.n == 0) return cudaSuccess;
    moment_tiles_kernel<<<p.tiles[p.n], kThreads, 0, s>>>(p);
    moment_finish_kernel<<<p.outs[p.n], kThreads, 0, s>>>(p);
    p.n = 0;
    return cudaGetLastError();
  };
  for (int i = 0; i < n; ++i) {
    const int64_t bands = ceil_div(m[i].d_out, kBand), strips = ceil_div(m[i].d_in, kStrip);
    const int64_t outs = ceil_div(m[i].d_out + m[i].d_in, kThreads);
    if (p.n == kMaxEntries ||
        (p.n > 0 && (p.tiles[p.n] + bands * strips > INT32_MAX || p.outs[p.n] + outs > INT32_MAX))) {
      const cudaError_t e = flush();
      if (e != cudaSuccess) return e;
    }
    Entry& e = p.e[p.n];
    e.v = m[i].v;
    e.vs = m[i].v_scale;
    e.rows = m[i].d_out;
    e.cols = m[i].d_in;
    e.r = m[i].r;
    e.c = m[i].c;
    e.st = m[i].state_kind;
    e.bands = static_cast<int>(bands);
    e.strips = static_cast<int>(strips);
    e.row_part = at;
    e.col_part = e.row_part + strips * e.rows;
    e.tile_part = e.col_part + bands * e.cols;
    at = e.tile_part + bands * strips;
    p.tiles[p.n + 1] = p.tiles[p.n] + static_cast<uint32_t>(bands * strips);
    p.outs[p.n + 1] = p.outs[p.n] + static_cast<uint32_t>(outs);
    ++p.n;
  }
  return flush();
}

}  // namespace bergson
