// Factored second moments of AdamW's v: the row and column means of every
// matrix, in one pass over tiles and a second small one over their sums.

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMostRows = 32, kLeastRows = 4;  // rows a warp takes (a power of two between)
// Rows on the way at once, fp32 and 8-bit (1 KB and 256 bytes a row), and CTAs an SM.
// 201M fp32 elements, us: 8 rows at 3 CTAs 157, 4 at 1 / 3 / 4 CTAs 149 / 136 / 142.
constexpr int kRows32 = 4, kRows8 = 8;
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

// The 8 codes from element i on, which may lie across two 8-byte words and two scales.
// A word that reaches past the matrix is read byte by byte.
__device__ __forceinline__ uint2 load_codes(const uint8_t* v, int64_t i, int count, int64_t n) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(v) + i, base = at & ~uintptr_t{7};
  const int skip = static_cast<int>(at & 7);
  if (base < reinterpret_cast<uintptr_t>(v) || base + 16 > reinterpret_cast<uintptr_t>(v) + n) {
    uint2 u = make_uint2(0, 0);
    for (int j = 0; j < count; ++j) {
      const uint32_t c = v[i + j];
      if (j < 4) u.x |= c << (8 * j); else u.y |= c << (8 * (j - 4));
    }
    return u;
  }
  const uint2 a = *reinterpret_cast<const uint2*>(base), b = *reinterpret_cast<const uint2*>(base + 8);
  const uint32_t w[4] = {a.x, a.y, b.x, b.y};
  const bool far = skip >= 4;
  const uint32_t w0 = far ? w[1] : w[0], w1 = far ? w[2] : w[1], w2 = far ? w[3] : w[2];
  uint2 u;
  u.x = __funnelshift_r(w0, w1, 8 * (skip & 3));
  u.y = __funnelshift_r(w1, w2, 8 * (skip & 3));
  // codes past the row's end belong to the next one
  if (count < 8) {
    u.y = count <= 4 ? 0u : u.y & ((1u << (8 * (count - 4))) - 1u);
    if (count < 4) u.x &= (1u << (8 * count)) - 1u;
  }
  return u;
}

// The values of a lane's 8 codes added up, and to the columns.  By all lanes of a warp;
// one that has none gives scale 0.
__device__ __forceinline__ float add_codes(uint2 u, float scale, float2 (&col)[4]) {
  float y[8];
  decode_nonzero_second4(u.x, y);
  decode_nonzero_second4(u.y, y + 4);
  if (__any_sync(0xffffffffu, (zero_bytes(u.x) | zero_bytes(u.y)) != 0)) {
    put_zeros4(u.x, y);
    put_zeros4(u.y, y + 4);
  }
  float2 s = {0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 y2 = make_float2(y[2 * j], y[2 * j + 1]);
    col[j] = fma2(y2, pair(scale), col[j]);
    s = add2(s, y2);
  }
  return (s.x + s.y) * scale;
}

// A warp's rows r0 .. r0 + e.warp_rows of a tile: lane sums of the columns in col[], the
// rows' sums to row_part.  Columns c0 + 8 lane + k, or of fp32 rows that start off a
// lane's 32 bytes c0 + lane + 32 k.
template <bool kEight, bool kVec>
__device__ __forceinline__ void take_rows(const Entry& e, int64_t r0, int64_t c0, float* row_part,
                                          float (&col)[8]) {
  constexpr int kRows = kEight ? kRows8 : kRows32;
  const int lane = threadIdx.x & 31;
  const int64_t r1 = min(e.rows, r0 + e.warp_rows);
  const int64_t c = c0 + 8 * lane;
  const int count = static_cast<int>(min(static_cast<int64_t>(8), e.cols - c));   // of the lane's
  float2 col2[4] = {};
#pragma unroll 1
  for (int64_t r = r0; r < r1; r += kRows) {
    float sums[kRows];
    if constexpr (!kEight) {
      uint32_t x[kRows][8];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[k][j] = 0;
        if (r + k >= r1) continue;
        const float* row = static_cast<const float*>(e.v) + (r + k) * e.cols;
        if (kVec) {
          if (count > 0) load32(row + c, x[k]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (c0 + lane + 32 * j < e.cols) x[k][j] = __float_as_uint(row[c0 + lane + 32 * j]);
        }
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
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        u[k] = make_uint2(0x01010101u, 0x01010101u);
        sc[k] = 0.0f;
        if (r + k < r1 && count > 0) {
          const uint64_t i = (r + k) * e.cols + c;
          u[k] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(e.v) + i);
          sc[k] = e.vs[i / kStateBlock];
        }
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) sums[k] = add_codes(u[k], sc[k], col2);
    } else {
      const int64_t n = e.rows * e.cols;
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        uint2 u = make_uint2(0x01010101u, 0x01010101u), v = u;
        float sc = 0.0f, sc2 = 0.0f;
        if (r + k < r1 && count > 0) {
          const uint64_t i = (r + k) * e.cols + c;
          const int near = kStateBlock - static_cast<int>(i % kStateBlock);   // with the first scale
          u = load_codes(static_cast<const uint8_t*>(e.v), i, count, n);
          sc = e.vs[i / kStateBlock];
          if (near < count) {                    // below 8 here
            const uint32_t lo = near >= 4 ? 0xffffffffu : (1u << (8 * near)) - 1u;
            const uint32_t hi = near <= 4 ? 0u : (1u << (8 * (near - 4))) - 1u;
            v.x = u.x & ~lo;
            v.y = u.y & ~hi;
            u.x &= lo;
            u.y &= hi;
            sc2 = e.vs[i / kStateBlock + 1];
          }
        }
        sums[k] = add_codes(u, sc, col2);
        if (__any_sync(0xffffffffu, sc2 != 0.0f)) sums[k] += add_codes(v, sc2, col2);
      }
    }
    const float t = sum_each(sums);
    const int k = lane / (32 / kRows);
    if (lane % (32 / kRows) == 0 && r + k < r1) row_part[r + k] = t;
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
  for (int j = 0; j < 8; ++j)
    cols[warp][e.vec || e.st == BERGSON_STATE_8BIT ? 8 * lane + j : lane + 32 * j] = col[j];
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
