// Factored second moments of AdamW's v: the row and column means of every
// matrix, in one pass over tiles and a second small one over their sums.
//
// A warp takes up to 32 rows of a strip, with its lanes' columns in registers; the
// rows' sums of four or eight rows at a time go through one butterfly over the lanes.  fp32
// matrices are bound by their bytes: 201M elements in 16 matrices 128 us, 6.3 TB/s.
// 8-bit ones are bound by the instructions that take codes apart (7.6 an element, 0.57 of
// the issue slots at a third of the warps): 68 us, 3.0 TB/s.

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
// Columns of a tile: 32 bytes of fp32 a lane, 16 codes of 8 bits.
constexpr int kStrip32 = 256, kStrip8 = 512;
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
  int bands, strips;           // tiles of kWarps warp_rows rows and `strip` columns
  int warp_rows, strip;
  int st;
  int vec;                     // rows start on boundaries of a lane's vector
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
  const uint2 a = *reinterpret_cast<const uint2*>(base);
  const uint2 b = *reinterpret_cast<const uint2*>(base + 8);
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

constexpr uint4 kNoCodes = {0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u};

// The values of a lane's 16 codes added up, and to the columns.  By all lanes of a warp;
// one that has none gives kNoCodes and scale 0.
__device__ __forceinline__ float add_codes(const uint4& u, float scale, float2 (&col)[8]) {
  float y[16];
#pragma unroll
  for (int q = 0; q < 4; ++q) decode_nonzero_second4(word(u, q), y + 4 * q);
  if (__any_sync(0xffffffffu, (zero_bytes(u.x) | zero_bytes(u.y) | zero_bytes(u.z) |
                               zero_bytes(u.w)) != 0)) {
#pragma unroll
    for (int q = 0; q < 4; ++q) put_zeros4(word(u, q), y + 4 * q);
  }
  float2 s = {0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float2 y2 = make_float2(y[2 * j], y[2 * j + 1]);
    col[j] = fma2(y2, pair(scale), col[j]);
    s = add2(s, y2);
  }
  return (s.x + s.y) * scale;
}

// The first `near` of 16 codes, the others 0.
__device__ __forceinline__ uint4 first_codes(const uint4& u, int near) {
  uint4 a;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int n = near - 4 * q;
    set_word(a, q, n >= 4 ? word(u, q) : n <= 0 ? 0u : word(u, q) & ((1u << (8 * n)) - 1u));
  }
  return a;
}

// A warp's rows r0 .. r0 + e.warp_rows of a tile: the rows' sums to row_part, and in col[]
// the lane's columns c0 + kCols lane + k, or of fp32 rows that start off a lane's 32
// bytes c0 + lane + 32 k.
template <bool kEight, bool kVec, int kCols>
__device__ __forceinline__ void take_rows(const Entry& e, int64_t r0, int64_t c0, float* row_part,
                                          float2 (&col)[kCols / 2]) {
  constexpr int kRows = kEight ? kRows8 : kRows32;
  const int lane = threadIdx.x & 31;
  const int64_t c = c0 + kCols * lane;
  const int cols = static_cast<int>(e.cols);
  // the lane's columns that the matrix has
  const int count = static_cast<int>(min(static_cast<int64_t>(kCols), e.cols - c));
  int left = static_cast<int>(min(e.rows - r0, static_cast<int64_t>(e.warp_rows)));
#pragma unroll
  for (int j = 0; j < kCols / 2; ++j) col[j] = {0.0f, 0.0f};
  uint64_t i = static_cast<uint64_t>(r0) * cols + c;      // the lane's first element of a row
  row_part += r0;
#pragma unroll 1
  for (; left > 0; left -= kRows, i += static_cast<uint64_t>(kRows) * cols, row_part += kRows) {
    float sums[kRows];
    if constexpr (!kEight) {
      uint32_t x[kRows][8];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[k][j] = 0;
        if (k >= left) continue;
        const float* row = static_cast<const float*>(e.v) + (i + static_cast<uint64_t>(k) * cols);
        if (kVec) {
          if (count > 0) load32(row, x[k]);
        } else {
          row -= 8 * lane;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (c0 + lane + 32 * j < cols) x[k][j] = __float_as_uint(row[lane + 32 * j]);
        }
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        float2 s = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 y =
              make_float2(__uint_as_float(x[k][2 * j]), __uint_as_float(x[k][2 * j + 1]));
          col[j] = add2(col[j], y);
          s = add2(s, y);
        }
        sums[k] = s.x + s.y;
      }
    } else if constexpr (kVec) {
      uint4 u[kRows];
      float sc[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        u[k] = kNoCodes;
        sc[k] = 0.0f;
        if (k < left && count > 0) {
          const uint64_t at = i + static_cast<uint64_t>(k) * cols;
          u[k] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(e.v) + at));
          sc[k] = e.vs[at / kStateBlock];
        }
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) sums[k] = add_codes(u[k], sc[k], col);
    } else {
      const int64_t n = e.rows * e.cols;
      const uint8_t* v = static_cast<const uint8_t*>(e.v);
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        uint4 u = kNoCodes, u2 = kNoCodes;
        float sc = 0.0f, sc2 = 0.0f;
        if (k < left && count > 0) {
          const uint64_t at = i + static_cast<uint64_t>(k) * cols;
          const uint2 a = load_codes(v, at, min(count, 8), n);
          const uint2 b = count > 8 ? load_codes(v, at + 8, count - 8, n) : make_uint2(0, 0);
          u = make_uint4(a.x, a.y, b.x, b.y);
          const int near = kStateBlock - static_cast<int>(at % kStateBlock);   // of one scale
          sc = e.vs[at / kStateBlock];
          if (near < count) {
            const uint4 f = first_codes(u, near);
            u2 = make_uint4(u.x ^ f.x, u.y ^ f.y, u.z ^ f.z, u.w ^ f.w);
            u = f;
            sc2 = e.vs[at / kStateBlock + 1];
          }
        }
        sums[k] = add_codes(u, sc, col);
        if (__any_sync(0xffffffffu, sc2 != 0.0f)) sums[k] += add_codes(u2, sc2, col);
      }
    }
    const float t = sum_each(sums);
    const int k = lane / (32 / kRows);
    if (lane % (32 / kRows) == 0 && k < left) row_part[k] = t;
  }
}

// ... and the columns' sums of the warp to shared memory.
template <bool kEight, bool kVec>
__device__ __forceinline__ void take_tile(const Entry& e, int64_t r0, int64_t c0, float* row_part,
                                          float* cols) {
  constexpr int kCols = kEight ? kStrip8 / 32 : kStrip32 / 32;
  const int lane = threadIdx.x & 31;
  float2 col[kCols / 2];
  take_rows<kEight, kVec, kCols>(e, r0, c0, row_part, col);
#pragma unroll
  for (int j = 0; j < kCols; ++j)
    cols[kEight || kVec ? kCols * lane + j : lane + 32 * j] = j % 2 ? col[j / 2].y : col[j / 2].x;
}

template <int N>
__global__ void __launch_bounds__(kThreads, kTileCtas) moment_tiles_kernel(
    const __grid_constant__ MomentParams<N> p) {
  __shared__ float cols[kWarps][kStrip8];
  __shared__ float red[kWarps];
  const int at = find(p.tiles, p.n, blockIdx.x);
  const Entry& e = p.e[at];
  const uint32_t tile = blockIdx.x - p.tiles[at];
  griddep_wait();
  const int band = tile / e.strips, strip = tile % e.strips;
  const int warp = threadIdx.x >> 5;
  const int64_t r0 = (static_cast<int64_t>(band) * kWarps + warp) * e.warp_rows;
  const int64_t c0 = static_cast<int64_t>(strip) * e.strip;
  float* row_part = e.row_part + static_cast<int64_t>(strip) * e.rows;
  if (e.st == BERGSON_STATE_8BIT) {
    if (e.vec) take_tile<true, true>(e, r0, c0, row_part, cols[warp]);
    else take_tile<true, false>(e, r0, c0, row_part, cols[warp]);
  } else {
    if (e.vec) take_tile<false, true>(e, r0, c0, row_part, cols[warp]);
    else take_tile<false, false>(e, r0, c0, row_part, cols[warp]);
  }
  __syncthreads();
  float all = 0.0f;
  for (int k = threadIdx.x; k < e.strip; k += kThreads) {
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) x += cols[w][k];
    if (c0 + k < e.cols) e.col_part[static_cast<int64_t>(band) * e.cols + c0 + k] = x;
    all += x;
  }
  all = block_sum(all, red);
  if (threadIdx.x == 0) e.tile_part[tile] = all;
}

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
// in any company): as many as leave kTilesWanted tiles.  Four 8-bit matrices of 72 x 72 to
// 288 x 72: 8.2 us, 26 with 32 rows always; 16 of 2048 x 2048 and more: 68, 83 with 256 tiles.
constexpr int64_t kTilesWanted = 64;
int strip_of(const bergson_moment_matrix& m) {
  return m.state_kind == BERGSON_STATE_8BIT ? kStrip8 : kStrip32;
}
int warp_rows_of(const bergson_moment_matrix& m) {
  int rows = kMostRows;
  while (rows > kLeastRows &&
         ceil_div(m.d_out, kWarps * rows) * ceil_div(m.d_in, strip_of(m)) < kTilesWanted)
    rows /= 2;
  return rows;
}

size_t floats_of(const bergson_moment_matrix& m) {
  const size_t bands = ceil_div(m.d_out, kWarps * warp_rows_of(m));
  const size_t strips = ceil_div(m.d_in, strip_of(m));
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
    const int64_t strips = ceil_div(m[i].d_in, strip_of(m[i]));
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
    const bool eight = e.st == BERGSON_STATE_8BIT;
    e.vec = m[i].d_in % (eight ? 16 : 8) == 0 &&
            reinterpret_cast<uintptr_t>(m[i].v) % (eight ? 16 : 32) == 0;
    e.strip = strip_of(m[i]);
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
