// One Muon step over many matrices: momentum, orthogonalisation of the update by
// Newton-Schulz products, weight update.
//
//   m <- beta m + (1 - beta) g,   u = m, or beta m + (1 - beta) g,   X = u / |u|_F,
//   per iteration (a, b, c):  A = X X^T,  X <- (a I + b A + c A^2) X,
//   w <- w - lr (ortho_scale X + weight_decay w)
//
// for the short side first; a matrix with more rows than columns takes A = X^T X and
// X <- X (..), and none is ever transposed.  The polynomial is taken as
//
//   A' = A + h I,   B = c A'^2 + (a - c h^2) I,   X <- B X,     h = b / 2c
//
// (c = 0: B = b A + a I at once), so that no product reads anything but its two operands.
//
// The products run on the tensor cores with fp16 operands and fp32 sums.  An operand is held as
// one fp16 plane (products = 1) or as the sum of two, hi = fp16(v), lo = fp16(v - hi) (products =
// 3: hi hi + hi lo + lo hi; what is left out is below 2^-22), in 1024 times its value: entries are
// 1 / 32768 and smaller at first, of the size of 1 / sqrt(columns) later.  By that hi has its 11
// bits down to entries of 2^-24, and both have 22 down to some 2^-12; below, lo is subnormal and an
// entry is off by up to 2^-35, beside |X|_F = 1.
//
// Matrices of one shape form a group, their planes stacked in the workspace under one
// tensor map.  All products of all iterations are one launch of persistent CTA pairs over 256-row
// tiles, handed out step by step, longest products first; a matrix's tiles wait for its own earlier
// ones alone.  An operand is read with its rows as they lie (K-major) or across (MN-major)
// by the tensor cores' own descriptors.  A' and B are symmetric: only tiles on and below the
// diagonal are computed and stored, and a read above it takes the mirror image across.
//
// Bound: with two planes an accumulator of 256 columns is 12 MMAs of 128 cycles a stage for 64 KB
// of loads, with one plane two of them are 8 for 48 KB; a CTA's loads come at 39 to 47 bytes a
// cycle when all SMs load, so that both forms wait for them a little (1.0 to 1.3 of the MMAs'
// time).  The smallest steps wait for one another: 15 products at 5 to 11 us, a chain of planes
// written, counted, seen and loaded.  Four blocks of d 2048 at one plane: 5.5 ms, 1.25 PFLOP/s
// under the power cap; ten of d 640 at two: 1.8 ms, 0.87 PFLOP/s of MMAs (six of 2048 rows: 84% of
// the tensor pipe's cycles, 69% at one plane).

#include <algorithm>
#include <cmath>
#include <functional>
#include <memory>
#include <vector>

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

constexpr float kPlaneScale = 1024.0f;         // of what the planes hold
constexpr int kMaxGroups = 8;                  // shapes of a batch of matrices
constexpr int kMaxMats = 300;                  // matrices of a batch
constexpr int64_t kBatchElements = 1ll << 29;  // of X planes where a batch ends: bounds the workspace

int64_t round_to(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// ------------------------------------------------------------------ momentum

constexpr int kMomentThreads = 256;
constexpr int64_t kMomentChunk = 8 * kMomentThreads;   // elements of a CTA's turn
constexpr float kUp = 0x1p100f, kDown = 0x1p-100f;

struct MomentEntry {
  const void* g;
  float* m;
  __half* x;                   // planes
  int64_t n, plane;            // elements; planes apart
  int32_t cols, ld;
  int32_t gt;
  int32_t vec;                 // g and m take vectors of 8, and rows are whole ones
};
struct WeightEntry {
  void* p;
  float* master;
  const __half* x;
  int64_t n, plane;
  int32_t cols, ld;
  float lr_ortho, lr_decay;    // lr lr_scale ortho_scale / 1024, lr lr_scale weight_decay
  int32_t pt;
  int32_t vec;
};

template <int N>
struct MomentParams {
  float beta, alpha;           // alpha = 1 - beta
  int nesterov;
  int n;
  const float* grad_scale;
  float3* part;                // a CTA's sums of squares
  int* counters;               // of the products: cleared by the first CTA
  int64_t chunk;               // elements a CTA
  uint32_t begin[N + 1];       // first CTA of each matrix
  MomentEntry e[N];
};
template <int N>
struct WeightParams {
  int n;
  int64_t chunk;
  uint32_t begin[N + 1];
  WeightEntry e[N];
};

template <typename Params>
__device__ __forceinline__ int entry_of(const Params& p) {
  int lo = 0, hi = p.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (p.begin[mid] <= blockIdx.x) lo = mid; else hi = mid;
  }
  return lo;
}

// 8 elements from i on as floats; those from n on are 0.
__device__ __forceinline__ void load_eight(const void* p, int type, bool vec, int64_t i, int64_t n,
                                           float (&x)[8]) {
  if (vec && i + 8 <= n) {
    if (type == BERGSON_F32) {
      uint32_t r[8];
      load32(static_cast<const float*>(p) + i, r);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(r[k]);
      return;
    }
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = type == BERGSON_BF16 ? unpack2(u, k, static_cast<const __nv_bfloat16*>(nullptr))
                                            : unpack2(u, k, static_cast<const __half*>(nullptr));
      x[2 * k] = f.x;
      x[2 * k + 1] = f.y;
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = i + k < n ? load_any(p, type, i + k) : 0.0f;
}

// Where a thread's 8 elements of a CTA's 2048 stand: side by side in vectors, else 256 apart, so
// that neighbouring threads take neighbouring elements.
__device__ __forceinline__ int64_t place(bool vec, int64_t at, int k) {
  return vec ? at + 8 * threadIdx.x + k : at + threadIdx.x + static_cast<int64_t>(kMomentThreads) * k;
}
__device__ __forceinline__ void load_turn(const void* p, int type, bool vec, int64_t at, int64_t n,
                                          float (&x)[8]) {
  if (vec) {
    load_eight(p, type, true, place(true, at, 0), n, x);
    return;
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int64_t i = place(false, at, k);
    x[k] = i < n ? load_any(p, type, i) : 0.0f;
  }
}
// Where element i of a matrix stands in its planes.
__device__ __forceinline__ int64_t in_plane(int64_t i, int cols, int ld) {
  const int64_t row = i <= INT32_MAX ? static_cast<uint32_t>(i) / static_cast<uint32_t>(cols) : i / cols;
  return row * ld + (i - row * cols);
}

// m's update and the sums of the squares of 2^100 u, u and 2^-100 u.  The first that is finite
// holds the norm of any u that fp32 does, with all its digits: the smallest u, 2^-149, has a square
// of 2^-98 in the first sum, and where a sum of up to 2^36 squares passed 2^128, the largest is
// 2^-108 or more in the next one.  Bound by its bytes all the same: 201M elements 305 us, 6.6 TB/s.
template <int N>
__global__ void __launch_bounds__(kMomentThreads) moment_kernel(
    const __grid_constant__ MomentParams<N> p) {
  __shared__ float red[2][32];
  const int k = entry_of(p);
  const MomentEntry& e = p.e[k];
  griddep_wait();
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i <= p.n; i += kMomentThreads) p.counters[i] = 0;
  const float gs = p.grad_scale != nullptr ? *p.grad_scale : 1.0f;
  const int64_t begin = static_cast<int64_t>(blockIdx.x - p.begin[k]) * p.chunk;
  const int64_t end = min(begin + p.chunk, e.n);
  CompensatedSum up, mid, down;
  for (int64_t at = begin; at < end; at += kMomentChunk) {
    float g[8], m[8];
    load_turn(e.g, e.gt, e.vec, at, end, g);
    load_turn(e.m, BERGSON_F32, e.vec, at, end, m);
    float su = 0.0f, sm = 0.0f, sd = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = p.alpha * (g[j] * gs);
      m[j] = fmaf(p.beta, m[j], a);
      const float u = p.nesterov ? fmaf(p.beta, m[j], a) : m[j];
      su = fmaf(u * kUp, u * kUp, su);
      sm = fmaf(u, u, sm);
      sd = fmaf(u * kDown, u * kDown, sd);
    }
    up.add(su);
    mid.add(sm);
    down.add(sd);
    if (e.vec) {
      if (place(true, at, 0) < end) {
        uint32_t r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = __float_as_uint(m[j]);
        store32(e.m + place(true, at, 0), r);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (place(false, at, j) < end) e.m[place(false, at, j)] = m[j];
    }
  }
  const float a = block_sum(up.s, red[0]), b = block_sum(mid.s, red[1]);
  const float c = block_sum(down.s, red[0]);
  if (threadIdx.x == 0) p.part[blockIdx.x] = make_float3(a, b, c);
}

// The planes of 1024 u / |u|_F, as (2^k u) (1024 / |2^k u|_F) with the k of the sum that holds the
// norm: 1024 / |u|_F alone would pass fp32 below 3e-36, and the norm itself above 3.4e38.  A matrix
// of zeros stays one; one that holds NaN or an infinity is NaN.
template <int N, int P>
__global__ void __launch_bounds__(kMomentThreads) planes_kernel(
    const __grid_constant__ MomentParams<N> p) {
  __shared__ float red[2][32];
  const int k = entry_of(p);
  const MomentEntry& e = p.e[k];
  griddep_wait();
  float a = 0.0f, b = 0.0f, c = 0.0f;
  for (uint32_t i = p.begin[k] + threadIdx.x; i < p.begin[k + 1]; i += kMomentThreads) {
    const float3 s = p.part[i];
    a += s.x;
    b += s.y;
    c += s.z;
  }
  a = block_sum(a, red[0]);
  b = block_sum(b, red[1]);
  c = block_sum(c, red[0]);
  const bool small = a - a == 0.0f, medium = b - b == 0.0f;
  const float shift = small ? kUp : medium ? 1.0f : kDown, square = small ? a : medium ? b : c;
  const float scale = square - square != 0.0f ? __int_as_float(0x7fffffff)
                      : square == 0.0f        ? 0.0f
                                              : kPlaneScale * __frcp_rn(__fsqrt_rn(square));
  const float gs = p.grad_scale != nullptr ? *p.grad_scale : 1.0f;
  const int64_t begin = static_cast<int64_t>(blockIdx.x - p.begin[k]) * p.chunk;
  const int64_t end = min(begin + p.chunk, e.n);
  for (int64_t at = begin; at < end; at += kMomentChunk) {
    float u[8];
    load_turn(e.m, BERGSON_F32, e.vec, at, end, u);
    if (p.nesterov) {
      float g[8];
      load_turn(e.g, e.gt, e.vec, at, end, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = fmaf(p.beta, u[j], p.alpha * (g[j] * gs));
    }
    if (e.vec) {                                 // the eight are of one row
      const int64_t i = place(true, at, 0);
      if (i >= end) continue;
      uint4 hi, lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 v = make_float2(u[2 * j] * shift * scale, u[2 * j + 1] * shift * scale);
        pack2(hi, j, v, static_cast<const __half*>(nullptr));
        const float2 h = unpack2(hi, j, static_cast<const __half*>(nullptr));
        pack2(lo, j, make_float2(v.x - h.x, v.y - h.y), static_cast<const __half*>(nullptr));
      }
      __half* x = e.x + in_plane(i, e.cols, e.ld);
      *reinterpret_cast<uint4*>(x) = hi;
      if (P == 2) *reinterpret_cast<uint4*>(x + e.plane) = lo;
      continue;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t i = place(false, at, j);
      if (i >= end) break;
      const float v = u[j] * shift * scale;
      const __half hi = __float2half_rn(v);
      __half* x = e.x + in_plane(i, e.cols, e.ld);
      *x = hi;
      if (P == 2) x[e.plane] = __float2half_rn(v - __half2float(hi));
    }
  }
}

// w <- w - lr (ortho_scale X + weight_decay w).  In a pass of its own: in the last product's
// epilogue the scattered rows of a tile cost as much (49M elements with masters: 100 us either
// way).
template <int N, int P>
__global__ void __launch_bounds__(kMomentThreads) weights_kernel(
    const __grid_constant__ WeightParams<N> p) {
  const int k = entry_of(p);
  const WeightEntry& e = p.e[k];
  griddep_wait();
  const int64_t begin = static_cast<int64_t>(blockIdx.x - p.begin[k]) * p.chunk;
  const int64_t end = min(begin + p.chunk, e.n);
  const void* from = e.master != nullptr ? e.master : e.p;
  const int type = e.master != nullptr ? static_cast<int>(BERGSON_F32) : e.pt;
  for (int64_t at = begin; at < end; at += kMomentChunk) {
    float w[8], x[8];
    load_turn(from, type, e.vec, at, end, w);
    const int64_t i0 = place(true, at, 0);
    if (e.vec) {
      if (i0 >= end) continue;
      const __half* s = e.x + in_plane(i0, e.cols, e.ld);
      load_eight(s, BERGSON_F16, true, 0, 8, x);
      if (P == 2) {
        float lo[8];
        load_eight(s + e.plane, BERGSON_F16, true, 0, 8, lo);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += lo[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int64_t i = place(false, at, j);
        x[j] = 0.0f;
        if (i >= end) continue;
        const __half* s = e.x + in_plane(i, e.cols, e.ld);
        x[j] = __half2float(*s);
        if (P == 2) x[j] += __half2float(s[e.plane]);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = fmaf(-e.lr_ortho, x[j], fmaf(-e.lr_decay, w[j], w[j]));
    if (e.vec) {
      uint32_t r[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] = __float_as_uint(w[j]);
      if (e.master != nullptr) store32(e.master + i0, r);
      if (e.pt == BERGSON_F32) {
        store32(static_cast<float*>(e.p) + i0, r);
        continue;
      }
      uint4 u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 y = make_float2(w[2 * j], w[2 * j + 1]);
        if (e.pt == BERGSON_BF16) pack2(u, j, y, static_cast<__nv_bfloat16*>(nullptr));
        else pack2(u, j, y, static_cast<__half*>(nullptr));
      }
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(e.p) + i0) = u;
      continue;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t i = place(false, at, j);
      if (i >= end) break;
      if (e.master != nullptr) e.master[i] = w[j];
      if (e.pt == BERGSON_BF16) static_cast<__nv_bfloat16*>(e.p)[i] = __float2bfloat16_rn(w[j]);
      else if (e.pt == BERGSON_F16) static_cast<__half*>(e.p)[i] = __float2half_rn(w[j]);
      else static_cast<float*>(e.p)[i] = w[j];
    }
  }
}

// ------------------------------------------------------------------ products

constexpr int kTileM = 256;                    // rows of a pair's tile, 128 a CTA
constexpr int kTileN = 256;                    // columns of an accumulator, at most
constexpr int kTileK = 64;                     // a stage: one 128-byte row of fp16
constexpr int kBoxBytes = 64 * 128;
constexpr int kPlaneBytes = 2 * kBoxBytes;     // of 128 rows of an operand's plane in a stage
constexpr int kEpilogueWarps = 16;             // four to a quarter of the rows: 64 columns a thread
constexpr int kFirstEpilogue = 4;              // warps: A's loads, MMA, B's loads, schedule, epilogue
constexpr int kThreads = 32 * (kFirstEpilogue + kEpilogueWarps);
constexpr int kChain = 4;                      // stages of an accumulation chain with two planes
constexpr int kOutTile = 32 * 64;              // bytes
constexpr int kBarBytes = 256;
constexpr int kTmemCols = 2 * kTileN;          // two accumulators
constexpr uint64_t kDrainTimeoutNs = 2000000000ull;

// With one plane a tile is two accumulators wide: a stage's loads (48 KB a CTA for 8 MMAs of 128
// cycles) then keep up with the MMAs, which those of one (32 KB for 4) do not, at some 2.4
// cycles a row of 128 bytes.  With two planes an accumulator has 12 MMAs for 64 KB.
template <int P>
struct ProdCfg {
  static constexpr int kSub = P == 2 ? 1 : 2;
  static constexpr int kABytes = P * kPlaneBytes;
  static constexpr int kStageBytes = kABytes + kSub * P * kPlaneBytes;
  static constexpr int kStages = P == 2 ? 3 : 4;
  // one plane: a warp's 32 rows and columns on their way out
  static constexpr int kOutBytes = P == 2 ? 0 : kEpilogueWarps * kOutTile;
  static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kOutBytes + kBarBytes;
};

// How an operand [rows, K] of a product lies in memory.
enum : int { kRowMajor = 0, kAcross = 1, kSymmetric = 2 };

// The three products of an iteration: A' = X X^T + h I, B = c A'^2 + .., X' = B X.
constexpr int kParts = 3;

struct ProdGroup {             // of a shape's product
  int begin;                   // first tile of the shape within the product's step
  int per_mat;                 // tiles of a matrix
  int n_mt, n_nt, tn;          // tiles of ProdCfg::kSub times tn columns
  int M, N, K;                 // of D [M, N]
  int a_kind, b_kind;
  int chunks_b;                // 64-row chunks of a box of B's across; 0: one each, tn % 128 != 0
  int lower;                   // only tiles that reach the diagonal or lie below
};
struct ShapeInfo {
  ProdGroup part[kParts];
  int first_mat;
  int ld[2];                   // of X's planes, and of A' and B's
  int64_t plane[2];
  __half* buf[4];              // X, X', A', B
};
// An operand's boxes: of the rows as they lie, and across.
struct Side {
  CUtensorMap rows, across;
};
struct ShapeMaps {
  Side a[5], b[5];             // of the first product by X's buffer, the second, the third by X's buffer
  CUtensorMap out[4];          // of buf, boxes of 32 rows and columns (one plane)
};
__host__ __device__ constexpr int side_of(int part, int cur) {
  return part == 0 ? cur : part == 1 ? 2 : 3 + cur;
}
struct Step {
  int begin;                   // first tile
  float alpha, gamma;          // D' = alpha acc + gamma I
  uint8_t part, cur, dst;      // product, X's buffer, buf it writes
  uint8_t before[kParts];      // steps before this one, by product
  uint8_t pad[2];
};

template <int G, int S>
struct ProdParams {
  ShapeMaps maps[G];
  ShapeInfo info[G];
  Step step[S];
  int n, n_steps, n_tiles;
  int* counters;               // tiles handed out; then per matrix, epilogue warps that are through with a tile
  int* status;
  uint64_t timeout_ns;
};

struct Tile {
  int step, group, mat, mt, nt;
  int subs;                    // accumulators that are needed: columns within D and not above the diagonal
};

// Tile t, which is of step `step` or a later one.
template <int P, int G, int S>
__device__ __forceinline__ Tile tile_of(const ProdParams<G, S>& p, int t, int step) {
  constexpr int kSub = ProdCfg<P>::kSub;
  Tile o;
  while (step + 1 < p.n_steps && p.step[step + 1].begin <= t) ++step;
  o.step = step;
  const int part = p.step[step].part;
  t -= p.step[step].begin;
  o.group = 0;
  while (o.group + 1 < p.n && p.info[o.group + 1].part[part].begin <= t) ++o.group;
  const ProdGroup& g = p.info[o.group].part[part];
  t -= g.begin;
  o.mat = t / g.per_mat;
  t -= o.mat * g.per_mat;
  int width = g.N;                               // of the tile's row of tiles
  if (g.lower) {
    o.mt = 0;
    for (;;) {
      width = min((o.mt + 1) * kTileM, g.N);
      const int n = (width + kSub * g.tn - 1) / (kSub * g.tn);
      if (t < n) break;
      t -= n;
      ++o.mt;
    }
    o.nt = t;
  } else {
    constexpr int kSide = 8;                     // near-square blocks of tiles share panels in L2
    const int per = kSide * g.n_nt, block = t / per, r = t - block * per;
    const int rows = min(kSide, g.n_mt - block * kSide);
    o.mt = block * kSide + r % rows;
    o.nt = r / rows;
  }
  o.subs = kSub == 1 ? 1 : min(kSub, (width - o.nt * kSub * g.tn + g.tn - 1) / g.tn);
  return o;
}

// ---- The schedule.  Tiles are handed out in order, step by step, to pairs as they become free: a
// warp of each pair takes the next one and passes it to the pair's others through a ring in shared
// memory.  A matrix's tiles wait for all tiles of its earlier steps, which were handed out before:
// whichever pairs run, the first unfinished tile can proceed, so that no pair needs another to be
// resident.
constexpr int kSlots = 2;                      // tiles a pair has taken and not begun
constexpr int kTakers = 2 * (2 + kEpilogueWarps) + 1;    // loads and epilogue of both CTAs, MMA

struct Ring {                  // in each CTA; `empty` counts in the even one
  uint64_t full[kSlots], empty[kSlots];
  int tile[kSlots];
};

__device__ __forceinline__ void store_remote(uint32_t cluster_addr, int v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}

// Hands out tiles, from one thread of the even CTA.
__device__ __forceinline__ bool hand_out(Ring* ring, int* counter, int n_tiles, uint64_t tmo,
                                         const volatile int* abort_flag) {
  uint32_t ph = 0;
  for (int slot = 0;;) {
    if (!mbar_wait_cluster(smem_u32(&ring->empty[slot]), ph ^ 1, tmo, abort_flag)) return false;
    const int t = atomicAdd(counter, 1);
    const int tile = t < n_tiles ? t : -1;
    for (uint32_t r = 0; r < 2; ++r) {
      store_remote(mapa_shared(smem_u32(&ring->tile[slot]), r), tile);
      mbar_arrive_cluster(mapa_shared(smem_u32(&ring->full[slot]), r));
    }
    if (tile < 0) return true;
    if (++slot == kSlots) { slot = 0; ph ^= 1; }
  }
}

// A taker's place in the ring; next() is called by one lane: the tile, -1 at the end, -2 when it
// gave up.
struct Taker {
  int slot = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ int next(Ring* ring, uint64_t tmo, const volatile int* abort_flag) {
    if (!mbar_wait_cluster(smem_u32(&ring->full[slot]), ph, tmo, abort_flag)) return -2;
    const int t = *reinterpret_cast<volatile int*>(&ring->tile[slot]);
    mbar_arrive_cluster(mapa_shared(smem_u32(&ring->empty[slot]), 0));
    if (++slot == kSlots) { slot = 0; ph ^= 1; }
    return t;
  }
  __device__ __forceinline__ int next_warp(Ring* ring, uint64_t tmo, const volatile int* abort_flag) {
    int t = 0;
    if ((threadIdx.x & 31) == 0) t = next(ring, tmo, abort_flag);
    return __shfl_sync(0xffffffffu, t, 0);
  }
};

// Waits until `need` epilogue warps are through with the matrix's earlier steps, whose planes
// may be loaded then.
__device__ __forceinline__ bool wait_matrix(const int* done, int need, uint64_t tmo,
                                            const volatile int* abort_flag) {
  const uint64_t t0 = global_timer_ns();
  for (uint32_t it = 0;; ++it) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(done) : "memory");
    if (v >= need) break;
    if (abort_flag != nullptr && *abort_flag) return false;
    if (it == (1u << 30) || global_timer_ns() - t0 > tmo) return false;
  }
  asm volatile("fence.proxy.async;" ::: "memory");
  return true;
}

// The stage from which on the operand rows from row0 on (a tile's first) are read across.
__device__ __forceinline__ int across_from(int kind, int row0) {
  return kind == kRowMajor ? INT32_MAX
         : kind == kAcross ? 0
                           : (row0 / kTileM + 1) * (kTileM / kTileK);
}

__device__ __forceinline__ void tma_load_rows(uint32_t dst, const void* tmap, uint32_t bar, int k,
                                              int row, int plane, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      ".L2::cache_hint [%0], [%1, {%3, %4, %5}], [%2], %6;" ::"r"(dst),
      "l"(tmap), "r"(bar), "r"(k), "r"(row), "r"(plane), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void tma_load_across(uint32_t dst, const void* tmap, uint32_t bar,
                                                int row, int k, int plane, int chunk,
                                                uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      ".L2::cache_hint [%0], [%1, {%3, %4, %5, %6}], [%2], %7;" ::"r"(dst),
      "l"(tmap), "r"(bar), "r"(row), "r"(k), "r"(plane), "r"(chunk), "l"(policy)
      : "memory");
}

// Shared-memory descriptors of the two ways, 128-byte swizzle, as their low words (the upper one is
// the same: 1024 bytes from one group of 8 to the next).  Rows as they lie: 128 bytes of K each, 8
// rows a group.  Across: 64 rows side by side in 128 bytes, 8 columns of K a group; a chunk's P
// planes come one after the other, the next 64 rows behind them.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
template <int P>
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr, bool x) {
  return (saddr >> 4) | (x ? static_cast<uint32_t>(P * kBoxBytes >> 4) : 1u) << 16;
}
__device__ __forceinline__ void umma_pair_low(uint32_t d_tmem, uint32_t a_low, uint32_t b_low,
                                              uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
      "setp.ne.b32 p, %5, 0;\n\t"
      "mov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %4, p;\n\t}" ::"r"(d_tmem),
      "r"(a_low), "r"(b_low), "r"(kDescHigh), "r"(idesc), "r"(accumulate)
      : "memory");
}
// True in one lane of a whole warp, the same each time.
__device__ __forceinline__ bool elect_lane() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r != 0;
}

// One side's loads of all the tiles of a CTA, by one thread.
template <int P, bool kSideB, int G, int S>
__device__ __forceinline__ void load_side(const ProdParams<G, S>& p, int rank, Ring* ring,
                                          uint32_t sbase, uint64_t* full, uint64_t* empty,
                                          volatile int* s_abort) {
  using C = ProdCfg<P>;
  const uint64_t tmo = p.timeout_ns;
  const uint64_t pol = policy_evict_normal();
  Taker taker;
  int stage = 0, step = 0;
  uint32_t ph = 0;
  uint32_t issued = 0, issued_par = 0;
  bool ok = true;
  while (ok) {
    const int t = taker.next(ring, tmo, s_abort);
    if (t < 0) {
      ok = t == -1;
      break;
    }
    const Tile o = tile_of<P>(p, t, step);
    step = o.step;
    const Step& st = p.step[step];
    const ShapeInfo& info = p.info[o.group];
    const ProdGroup& g = info.part[st.part];
    int need = 0;
#pragma unroll
    for (int k = 0; k < kParts; ++k)
      need += st.before[k] * info.part[k].per_mat * (2 * kEpilogueWarps);
    const ShapeMaps& maps = p.maps[o.group];
    const Side& side = kSideB ? maps.b[side_of(st.part, st.cur)] : maps.a[side_of(st.part, st.cur)];
    const void* rows_map = &side.rows;
    const void* across_map = &side.across;
    const int kind = kSideB ? g.b_kind : g.a_kind;
    if (kind != kAcross) prefetch_tmap(rows_map);
    if (kind != kRowMajor) prefetch_tmap(across_map);
    if (need > 0 && !wait_matrix(p.counters + 1 + info.first_mat + o.mat, need, tmo, s_abort)) {
      ok = false;
      break;
    }
    const int z = o.mat * P;
    const int subs = kSideB ? o.subs : 1;
    const int wide = kSideB ? g.tn : kTileM;       // rows over the pair
    const int half = wide / 2;
    const int first = kSideB ? o.nt * C::kSub * g.tn : o.mt * kTileM;
    const int chunks = kSideB ? g.chunks_b : 2;
    const int boxes = (half + 63) / 64;            // without whole chunks
    const int x_from = across_from(kind, first), inner = g.K;
    for (int k0 = 0; k0 < inner; k0 += kTileK) {
      if (!mbar_wait(smem_u32(&empty[stage]), ph ^ 1, tmo, s_abort)) { ok = false; break; }
      const bool x = k0 / kTileK >= x_from;
      const uint32_t fb_local = smem_u32(&full[stage]);
      const uint32_t fb = mapa_shared(fb_local, 0);
      if (rank == 0) {
        const uint32_t bytes = x ? (chunks > 0 ? chunks : boxes) * P * kBoxBytes : half * 128 * P;
        mbar_arrive_expect_tx(fb_local, 2 * subs * bytes);
      }
      uint32_t dst = sbase + stage * C::kStageBytes + (kSideB ? C::kABytes : 0);
      int r = first + rank * half;
      for (int h = 0; h < subs; ++h, r += wide, dst += P * kPlaneBytes) {
        if (!x) {
          tma_load_rows(dst, rows_map, fb, k0, r, z, pol);
        } else if (chunks > 0) {
          tma_load_across(dst, across_map, fb, 0, k0, z, r / 64, pol);
        } else {
          for (int q = 0; q < boxes; ++q)
            tma_load_across(dst + q * P * kBoxBytes, across_map, fb, r + 64 * q, k0, z, 0, pol);
        }
      }
      issued |= 1u << stage;
      issued_par = (issued_par & ~(1u << stage)) | (ph << stage);
      if (++stage == C::kStages) { stage = 0; ph ^= 1; }
    }
  }
  if (!ok) {
    raise_device_error(p.status, s_abort, kStatusTimeout);
    if (rank == 0) {
      for (int s = 0; s < C::kStages; ++s)
        if (issued >> s & 1)
          mbar_wait(smem_u32(&full[s]), (issued_par >> s) & 1, kDrainTimeoutNs, nullptr);
    } else {
      const uint64_t t0 = global_timer_ns();      // its loads complete on the other CTA's barrier
      while (global_timer_ns() - t0 < 1000000ull) {
      }
    }
  }
}

__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint64_t tmo,
                                          const volatile int* abort_flag) {
  bool ok = true;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait_inline(bar, parity, tmo, abort_flag);
  return __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
}

// 16 columns of a row to their two planes.
__device__ __forceinline__ void put_planes(__half* d, int64_t plane, const float* v) {
  uint32_t hi[8], lo[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(v[2 * k] - f.x, v[2 * k + 1] - f.y);
    hi[k] = *reinterpret_cast<const uint32_t*>(&h);
    lo[k] = *reinterpret_cast<const uint32_t*>(&l);
  }
  store32(d, hi);
  store32(d + plane, lo);
}

// All steps' D[i, j] = alpha <a_i, b_j> + gamma [i == j] over persistent CTA pairs, synchronised
// as the other pair kernels: the odd CTA's loads complete on the even CTA's `full`, the
// even CTA's MMA thread frees a stage in both CTAs and hands accumulators to both
// epilogues by multicast commits, and every epilogue warp of both CTAs releases an
// accumulator on the even CTA's `tempty`.  Every wait is bounded.
//
// The tensor cores' fp32 sums round toward zero.  With two planes, an accumulation chain is kChain
// stages (48 MMAs, a stage's smallest terms first) and the epilogue adds the chains in registers
// while the next one runs; with one plane the operands' own rounding is 2^-12 and a tile is one
// chain, which loses up to 2^-23 an MMA: 2^-27 a column of K.
template <int P, int G, int S>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    products_kernel(const __grid_constant__ ProdParams<G, S> p) {
  using C = ProdCfg<P>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  const uint32_t sbase = smem_u32(smem);
  uint64_t* full =
      reinterpret_cast<uint64_t*>(smem + C::kStages * C::kStageBytes + C::kOutBytes);
  uint64_t* empty = full + C::kStages;
  uint64_t* tfull = empty + C::kStages;
  uint64_t* tempty = tfull + 2;
  uint64_t* drain = tempty + 2;
  Ring* ring = reinterpret_cast<Ring*>(drain + 1);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(ring + 1);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);

  const int rank = static_cast<int>(cluster_ctarank());
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  griddep_launch_dependents();   // the next grid sets itself up and waits for this one to end
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(smem_u32(&full[s]), 2);              // A's and B's loads
      mbar_init(smem_u32(&empty[s]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&tfull[i]), 1);
      mbar_init(smem_u32(&tempty[i]), 2 * kEpilogueWarps);     // of both CTAs
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(smem_u32(&ring->full[i]), 1);
      mbar_init(smem_u32(&ring->empty[i]), kTakers);
    }
    mbar_init(smem_u32(drain), 1);
    *s_abort = 0;
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(s_tmem), kTmemCols);
    tmem_relinquish_pair();
  }
  __syncwarp();
  tc_fence_before();
  cluster_sync();
  tc_fence_after();
  griddep_wait();                // the operands come from earlier grids
  const uint32_t tmem = *s_tmem;
  const uint64_t tmo = p.timeout_ns;

  if (warp == 0) {
    if (lane == 0) load_side<P, false>(p, rank, ring, sbase, full, empty, s_abort);
    __syncwarp();
  } else if (warp == 2) {
    if (lane == 0) load_side<P, true>(p, rank, ring, sbase, full, empty, s_abort);
    __syncwarp();
  } else if (warp == 3) {
    if (rank == 0 && lane == 0 && !hand_out(ring, p.counters, p.n_tiles, tmo, s_abort))
      raise_device_error(p.status, s_abort, kStatusTimeout);
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (even CTA)
    // The whole warp goes through the loop and one lane issues: descriptors then are the warp's
    // own, and an MMA takes 18 cycles to issue instead of 62 in a branch of one lane.
    if (rank == 0) {
      const bool lead = elect_lane();
      int stage = 0;
      uint32_t ph = 0;
      int ab = 0;                                    // the tile's first accumulator, its round's parity
      uint32_t aph = 0;
      bool ok = true;
      Taker taker;
      int step = 0;
      while (ok) {
        const int t = taker.next_warp(ring, tmo, s_abort);
        if (t < 0) {
          ok = t == -1;
          break;
        }
        const Tile o = tile_of<P>(p, t, step);
        step = o.step;
        const ProdGroup& g = p.info[o.group].part[p.step[step].part];
        const int subs = o.subs, tn = g.tn, stages = (g.K + kTileK - 1) / kTileK;
        // stages from which on an operand is read across
        const int xa_from = across_from(g.a_kind, o.mt * kTileM);
        const int xb_from = across_from(g.b_kind, o.nt * C::kSub * tn);
        const uint32_t base_idesc = make_idesc_f16(kTileM, tn, false);
        bool fresh = true;                           // the accumulators hold nothing yet
        // A tile of two accumulators begins with a ring of stages for the first and then for the
        // second, which the epilogue is still reading at that time.
        for (int kb = 0, len; ok && kb < stages; kb += len) {
          len = C::kSub == 2 && kb == 0 && subs == 2 ? min(C::kStages, stages) : 1;
          const bool ends = kb + len == stages || (P == 2 && kb % kChain == kChain - 1);
          int cab = ab;
          uint32_t caph = aph;
#pragma unroll
          for (int h = 0; h < C::kSub; ++h) {
            if (h >= subs) break;
            if (fresh) {
              ok = warp_wait(smem_u32(&tempty[cab]), caph ^ 1, tmo, s_abort);
              if (!ok) break;
            }
            int st = stage;
            uint32_t sph = ph;
            for (int kc = kb; kc < kb + len; ++kc) {
              if (h == 0) {
                ok = warp_wait(smem_u32(&full[st]), sph, tmo, s_abort);
                if (!ok) break;
              }
              const bool xa = kc >= xa_from, xb = kc >= xb_from;
              tc_fence_after();
              if (lead) {
                const uint32_t sa = sbase + st * C::kStageBytes;
                const uint32_t da = desc_low<P>(sa, xa);
                const uint32_t db = desc_low<P>(sa + C::kABytes + h * P * kPlaneBytes, xb);
                // 16 columns of K: 32 bytes of a row, or 16 rows of 128 bytes
                const uint32_t step_a = xa ? 128 : 2, step_b = xb ? 128 : 2;
                const uint32_t plane_a = (xa ? kBoxBytes : kPlaneBytes) / 16;
                const uint32_t plane_b = (xb ? kBoxBytes : tn / 2 * 128) / 16;
                const uint32_t idesc = base_idesc | (xa ? 1u << 15 : 0u) | (xb ? 1u << 16 : 0u);
                const uint32_t d = tmem + cab * kTileN;
                const bool first = fresh && kc == kb;
                constexpr int kTerms = P == 2 ? 3 : 1;
#pragma unroll
                for (int q = 0; q < kTerms; ++q) {   // lo hi, hi lo, hi hi
                  const uint32_t at = da + (P == 2 && q == 0 ? plane_a : 0);
                  const uint32_t bt = db + (P == 2 && q == 1 ? plane_b : 0);
#pragma unroll
                  for (int kk = 0; kk < kTileK / 16; ++kk)
                    umma_pair_low(d, at + kk * step_a, bt + kk * step_b, idesc,
                                  !first || q != 0 || kk != 0);
                }
                // A commit stands in the branch of the MMAs that it follows.  In a branch of its
                // own behind the warp's barrier, by the same lane, it did not arrive; why is not
                // known.
                if (ends && kc == kb + len - 1) umma_commit_pair(smem_u32(&tfull[cab]), 0x3);
                if (h == subs - 1) umma_commit_pair(smem_u32(&empty[st]), 0x3);
              }
              __syncwarp();
              if (++st == C::kStages) { st = 0; sph ^= 1; }
            }
            if (!ok) break;
            if (++cab == 2) { cab = 0; caph ^= 1; }
          }
          if (!ok) break;
          fresh = ends;
          if (ends) { ab = cab; aph = caph; }
          stage += len;
          if (stage >= C::kStages) { stage -= C::kStages; ph ^= 1; }
        }
      }
      if (lead) {
        if (!ok) raise_device_error(p.status, s_abort, kStatusTimeout);
        umma_commit_pair(smem_u32(drain), 0x1);
        mbar_wait(smem_u32(drain), 0, kDrainTimeoutNs, nullptr);
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ epilogue
    // Thread = a row of this CTA's half (TMEM lane) and up to 64 of an accumulator's columns:
    // summed up in registers, so that the accumulator is free again before anything is written.  A
    // thread writes whole 32-byte sectors of its row.
    const int ew = warp - kFirstEpilogue;
    const int quarter = warp & 3;
    uint8_t* out = smem + C::kStages * C::kStageBytes + ew * kOutTile;
    int ab = 0;
    uint32_t aph = 0;
    bool aborted = false;
    Taker taker;
    int step = 0;
    while (!aborted) {
      const int t = taker.next_warp(ring, tmo, s_abort);
      if (t < 0) {
        if (t != -1) raise_device_error(p.status, s_abort, kStatusTimeout);
        break;
      }
      const Tile o = tile_of<P>(p, t, step);
      step = o.step;
      const Step& st = p.step[step];
      const ShapeInfo& info = p.info[o.group];
      const ProdGroup& g = info.part[st.part];
      const int which = st.part == 2 ? 0 : 1;        // planes of X's, or of A' and B's
      const int pieces = g.tn / 16, first = pieces * (ew >> 2) / 4;      // of 16 columns
      const int mine = pieces * ((ew >> 2) + 1) / 4 - first;             // up to 4
      const int row = o.mt * kTileM + rank * (kTileM / 2) + 32 * quarter + lane;
      const int chains = P == 2 ? (g.K + kTileK * kChain - 1) / (kTileK * kChain) : 1;
      for (int h = 0; h < o.subs && !aborted; ++h) {
        const int col0 = (o.nt * C::kSub + h) * g.tn + 16 * first;
        const int left = row < g.M ? min(16 * mine, g.N - col0) : 0;     // columns to write
        constexpr int kAcc = kTileN / 4;
        float acc[kAcc];
        if constexpr (P == 2) {
#pragma unroll
          for (int j = 0; j < kAcc; ++j) acc[j] = 0.0f;  // 0 + v = v: the first chain lands unchanged
        }
        for (int ch = 0; ch < chains; ++ch) {
          if (!warp_wait(smem_u32(&tfull[ab]), aph, tmo, s_abort)) {
            raise_device_error(p.status, s_abort, kStatusTimeout);
            aborted = true;
            break;
          }
          tc_fence_after();
          const uint32_t tb = tmem + (static_cast<uint32_t>(32 * quarter) << 16) + ab * kTileN +
                              16 * first;
          if constexpr (P == 1) {                    // 32 columns or 64
            tmem_ld64(tb, acc);
          } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              if (u < mine) {
                float v[16];
                tmem_ld16(tb + 16 * u, v);
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                  const float2 x = add2(make_float2(acc[16 * u + j], acc[16 * u + j + 1]),
                                        make_float2(v[j], v[j + 1]));
                  acc[16 * u + j] = x.x;
                  acc[16 * u + j + 1] = x.y;
                }
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(mapa_shared(smem_u32(&tempty[ab]), 0));
          if (++ab == 2) { ab = 0; aph ^= 1; }
        }
        if (aborted) break;
        const float2 alpha = pair(st.alpha);
#pragma unroll
        for (int j = 0; j < kAcc; j += 2) {
          const float2 x = mul2(make_float2(acc[j], acc[j + 1]), alpha);
          acc[j] = x.x;
          acc[j + 1] = x.y;
        }
        const int row0 = row - lane;
        if (st.gamma != 0.0f && row0 < col0 + kAcc && row0 + 32 > col0) {     // on the diagonal
          const float gamma = st.gamma;
#pragma unroll
          for (int j = 0; j < kAcc; ++j) acc[j] += row == col0 + j ? gamma : 0.0f;
        }
        if constexpr (P == 1) {
#pragma unroll
          for (int u = 0; u < 4; u += 2) {
            if (u >= mine) break;
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
#pragma unroll
            for (int c = 0; c < 4; ++c) {          // 8 columns each, 64-byte swizzle
              uint4 v;
#pragma unroll
              for (int j = 0; j < 4; ++j)
                pack2(v, j, make_float2(acc[16 * u + 8 * c + 2 * j], acc[16 * u + 8 * c + 2 * j + 1]),
                      static_cast<const __half*>(nullptr));
              *reinterpret_cast<uint4*>(out + 64 * lane + 16 * (c ^ ((lane >> 1) & 3))) = v;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0 && row0 < g.M && col0 + 16 * u < g.N) {
              asm volatile(
                  "cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                  ::"l"(&p.maps[o.group].out[st.dst]), "r"(smem_u32(out)), "r"(col0 + 16 * u), "r"(row0),
                    "r"(o.mat)
                  : "memory");
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          }
        } else {
          __half* d = info.buf[st.dst] + static_cast<int64_t>(o.mat) * P * info.plane[which] +
                      static_cast<int64_t>(row) * info.ld[which] + col0;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (16 * u >= left) break;
            put_planes(d + 16 * u, info.plane[which], acc + 16 * u);
          }
        }
        __syncwarp();
      }
      if (aborted) break;
      // Through with the tile: its planes may be loaded, by whoever sees the count.  Two planes:
      // the warp's barrier puts all lanes' stores before lane 0's release, and the thread that
      // loads has its proxy fence behind its acquire (wait_matrix): one on the way from the stores
      // to the copies is enough.  One plane: the copies out have ended before the release.
      if (P == 1 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
      __syncwarp();
      if (lane == 0)
        asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(p.counters + 1 + info.first_mat +
                                                                    o.mat)
                     : "memory");
    }
    // one that gave up may have copies out of shared memory on their way
    if (P == 1 && aborted && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
  }

  tc_fence_before();
  cluster_sync();              // no MMA, commit or remote arrival is still in flight
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, kTmemCols);
  }
}

// ------------------------------------------------------------------ host

struct Shape {
  int64_t rows, cols;
  std::vector<int> mats;       // indices into the caller's array
};

// The tensors by their shape, the longest products first, cut into batches.
struct Batch {
  std::vector<Shape> shapes;
  int mats = 0;
  int64_t elements = 0, held = 0;                // of the matrices, and of an X plane of each
};

// Rows of a plane are whole chunks of 64 columns.
int64_t leading(int64_t cols) { return round_to(cols, 64); }

std::vector<Batch> batches_of(const bergson_muon_tensor* t, int n) {
  std::vector<Shape> shapes;
  for (int i = 0; i < n; ++i) {
    size_t k = 0;
    while (k < shapes.size() && (shapes[k].rows != t[i].rows || shapes[k].cols != t[i].cols)) ++k;
    if (k == shapes.size()) shapes.push_back({t[i].rows, t[i].cols, {}});
    shapes[k].mats.push_back(i);
  }
  std::stable_sort(shapes.begin(), shapes.end(), [](const Shape& a, const Shape& b) {
    return std::max(a.rows, a.cols) > std::max(b.rows, b.cols);
  });
  std::vector<Batch> out;
  for (const Shape& s : shapes) {
    // A' and B take no more than X: their short side squared, padded alike
    const int64_t each = s.rows * s.cols, held = s.rows * leading(s.cols);
    bool open = false;                           // the shape is the last of the last batch
    for (int i : s.mats) {
      if (out.empty() || out.back().mats == kMaxMats ||
          (out.back().mats > 0 && out.back().held + held > kBatchElements) ||
          (!open && out.back().shapes.size() == kMaxGroups)) {
        out.emplace_back();
        open = false;
      }
      Batch& b = out.back();
      if (!open) b.shapes.push_back({s.rows, s.cols, {}});
      open = true;
      b.shapes.back().mats.push_back(i);
      ++b.mats;
      b.elements += each;
      b.held += held;
    }
  }
  return out;
}

// Where a shape's planes stand in the workspace: X twice, A and B.
struct Planes {
  size_t x[2], a, b;
  int64_t x_ld, x_plane, s_ld, s_plane;
};

struct BatchLayout {
  std::vector<Planes> shapes;
  size_t part = 0, counters = 0, total = 0;
  int64_t chunk = 0, ctas = 0;
};

BatchLayout layout_of(const Batch& b, int P) {
  BatchLayout l;
  size_t at = 0;
  const auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += static_cast<size_t>(round_to(bytes, 256));
    return here;
  };
  l.chunk = std::max(2 * kMomentChunk,
                     round_to(ceil_div(b.elements, kPlanCTAs * 16), kMomentChunk));
  for (const Shape& s : b.shapes)
    l.ctas += ceil_div(s.rows * s.cols, l.chunk) * static_cast<int64_t>(s.mats.size());
  l.part = take(l.ctas * static_cast<int64_t>(sizeof(float3)));
  l.counters = take((1 + b.mats) * static_cast<int64_t>(sizeof(int)));
  for (const Shape& s : b.shapes) {
    Planes p;
    const int64_t m = std::min(s.rows, s.cols), n = static_cast<int64_t>(s.mats.size()) * P * 2;
    p.x_ld = leading(s.cols);
    p.x_plane = s.rows * p.x_ld;
    p.s_ld = leading(m);
    p.s_plane = m * p.s_ld;
    p.x[0] = take(n * p.x_plane);
    p.x[1] = take(n * p.x_plane);
    p.a = take(n * p.s_plane);
    p.b = take(n * p.s_plane);
    l.shapes.push_back(p);
  }
  l.total = at;
  return l;
}

// Columns of an accumulator for D [m, n] (lower: the tiles that reach the diagonal or lie below),
// at most `most`: what computes least that is not needed.  An accumulator pays some 40 columns'
// time beside its own.  With one plane they are whole chunks.
struct Columns {
  int tn;
  int64_t accs;                // accumulators of a matrix
};
Columns tile_columns(int64_t m, int64_t n, bool lower, int P, int most) {
  Columns best{most, 0};
  int64_t cost = INT64_MAX;
  for (int tn = most; tn >= std::min(128, most); tn -= P == 2 ? 32 : 128) {
    int64_t c = 0;
    for (int64_t r = kTileM; r < m + kTileM; r += kTileM)
      c += ceil_div(lower ? std::min(r, n) : n, tn);
    if (c * (tn + 40) < cost) {
      cost = c * (tn + 40);
      best = {tn, c};
    }
  }
  return best;
}

// The D of a shape's product: 0 A', 1 B, 2 X'.
struct Dims {
  int64_t m, n, k;
};
Dims dims_of(const Shape& s, int part) {
  const int64_t m = std::min(s.rows, s.cols);
  return part == 2 ? Dims{s.rows, s.cols, m} : Dims{m, m, part == 0 ? std::max(s.rows, s.cols) : m};
}

// The same for all shapes of a launch, with the width that leaves the clusters least time: wide
// tiles read less for a product, narrow ones are more.  In cycles: MMAs of 1 / 2 a column and 57
// at least, loads of 2.6 a 128-byte row, 4000 a tile.
std::vector<int> launch_columns(const Batch& b, int part, int P, int clusters) {
  std::vector<int> best(b.shapes.size()), now(b.shapes.size());
  double least = INFINITY;
  for (int most : {256, 128, 64}) {
    if (P == 1 && most < 128) break;
    double all = 0.0, longest = 0.0;
    for (size_t i = 0; i < b.shapes.size(); ++i) {
      const Dims d = dims_of(b.shapes[i], part);
      const Columns c = tile_columns(d.m, d.n, part < 2, P, most);
      now[i] = c.tn;
      const double mma = (P == 2 ? 12 : 4) * std::max(57.0, c.tn / 2.0);
      const double load = 2.6 * P * (128 + c.tn / 2);
      const double tile = 4000.0 + static_cast<double>(ceil_div(d.k, kTileK)) * std::max(mma, load);
      all += tile * static_cast<double>(c.accs) * static_cast<double>(b.shapes[i].mats.size());
      longest = std::max(longest, tile);
    }
    const double time = std::max(all / clusters, longest);
    if (time < 0.97 * least) {
      least = time;
      best = now;
    }
  }
  return best;
}

template <int N>
cudaError_t run_moments(const bergson_muon_tensor* t, const Batch& b, const BatchLayout& l,
                        const MuonScalars& a, uint8_t* ws, cudaStream_t s) {
  const int P = a.products == 3 ? 2 : 1;
  MomentParams<N> p;
  p.beta = static_cast<float>(a.beta);
  p.alpha = static_cast<float>(1.0 - a.beta);
  p.nesterov = a.nesterov ? 1 : 0;
  p.n = b.mats;
  p.grad_scale = a.grad_scale;
  p.part = reinterpret_cast<float3*>(ws + l.part);
  p.counters = reinterpret_cast<int*>(ws + l.counters);
  p.chunk = l.chunk;
  p.begin[0] = 0;
  int k = 0;
  for (size_t g = 0; g < b.shapes.size(); ++g) {
    const Shape& sh = b.shapes[g];
    const Planes& pl = l.shapes[g];
    for (size_t z = 0; z < sh.mats.size(); ++z, ++k) {
      const bergson_muon_tensor& x = t[sh.mats[z]];
      MomentEntry& e = p.e[k];
      e.g = x.grad;
      e.m = x.m;
      e.x = reinterpret_cast<__half*>(ws + pl.x[0]) + static_cast<int64_t>(z) * P * pl.x_plane;
      e.n = sh.rows * sh.cols;
      e.plane = pl.x_plane;
      e.cols = static_cast<int32_t>(sh.cols);
      e.ld = static_cast<int32_t>(pl.x_ld);
      e.gt = x.grad_dtype;
      e.vec = sh.cols % 8 == 0 && on16(x.grad, 0, 1) && reinterpret_cast<uintptr_t>(x.m) % 32 == 0 &&
              (x.grad_dtype != BERGSON_F32 || reinterpret_cast<uintptr_t>(x.grad) % 32 == 0);
      p.begin[k + 1] = p.begin[k] + static_cast<uint32_t>(ceil_div(e.n, l.chunk));
    }
  }
  const dim3 grid(p.begin[k]), block(kMomentThreads);
  cudaError_t e = launch_dependent(moment_kernel<N>, grid, block, 0, s, p);
  if (e != cudaSuccess) return e;
  return P == 2 ? launch_dependent(planes_kernel<N, 2>, grid, block, 0, s, p)
                : launch_dependent(planes_kernel<N, 1>, grid, block, 0, s, p);
}

template <int N>
cudaError_t run_weights(const bergson_muon_tensor* t, const Batch& b, const BatchLayout& l,
                        const MuonScalars& a, uint8_t* ws, cudaStream_t s) {
  const int P = a.products == 3 ? 2 : 1;
  WeightParams<N> p;
  p.n = b.mats;
  p.chunk = l.chunk;
  p.begin[0] = 0;
  int k = 0;
  for (size_t g = 0; g < b.shapes.size(); ++g) {
    const Shape& sh = b.shapes[g];
    const Planes& pl = l.shapes[g];
    for (size_t z = 0; z < sh.mats.size(); ++z, ++k) {
      const bergson_muon_tensor& x = t[sh.mats[z]];
      WeightEntry& e = p.e[k];
      e.p = x.param;
      e.master = x.master;
      e.x = reinterpret_cast<const __half*>(ws + pl.x[a.iterations & 1]) +
            static_cast<int64_t>(z) * P * pl.x_plane;
      e.n = sh.rows * sh.cols;
      e.plane = pl.x_plane;
      e.cols = static_cast<int32_t>(sh.cols);
      e.ld = static_cast<int32_t>(pl.x_ld);
      const double lr = a.lr * x.lr_scale;
      e.lr_ortho = static_cast<float>(lr * x.ortho_scale / kPlaneScale);
      e.lr_decay = static_cast<float>(lr * x.weight_decay);
      e.pt = x.param_dtype;
      e.vec = sh.cols % 8 == 0 && reinterpret_cast<uintptr_t>(x.master) % 32 == 0 &&
              reinterpret_cast<uintptr_t>(x.param) % (x.param_dtype == BERGSON_F32 ? 32 : 16) == 0;
      p.begin[k + 1] = p.begin[k] + static_cast<uint32_t>(ceil_div(e.n, l.chunk));
    }
  }
  const dim3 grid(p.begin[k]), block(kMomentThreads);
  return P == 2 ? launch_dependent(weights_kernel<N, 2>, grid, block, 0, s, p)
                : launch_dependent(weights_kernel<N, 1>, grid, block, 0, s, p);
}

// The maps that a kind of operand is read by.  rows: of a box of rows; chunks: of a box across
// (0: a chunk at any row).
bool encode_side(Side* s, int kind, const void* ptr, int64_t cols, int64_t rows, int64_t planes,
                 int64_t ld, int P, int box_rows, int chunks) {
  return (kind == kAcross ||
          encode_tmap_stack(&s->rows, ptr, cols, rows, planes, ld, box_rows, P) == CUDA_SUCCESS) &&
         (kind == kRowMajor ||
          encode_tmap_across(&s->across, ptr, cols, rows, planes, ld, P, chunks) == CUDA_SUCCESS);
}

constexpr int64_t kMostOfMatrix = INT32_MAX / (2 * kEpilogueWarps);     // tiles, in its counter

using Launch = std::function<cudaError_t(cudaStream_t)>;

// All products of a batch, as `launch`: tensor maps, schedule and limits are done with before
// anything of the step is enqueued, so that what fails here leaves m and the weights alone.
template <int P, int G, int S>
cudaError_t prepare_products(const Batch& b, const BatchLayout& l, const MuonScalars& a,
                             uint8_t* ws, int* status, int sms, Launch* launch) {
  const int most_clusters = std::max(1, sms / 2);
  std::vector<int> columns[kParts];
  for (int part = 0; part < kParts; ++part)
    columns[part] = launch_columns(b, part, P, most_clusters);
  static_assert(sizeof(ProdParams<G, S>) <= 32'000, "a launch's parameters");
  const auto params = std::make_shared<ProdParams<G, S>>();
  ProdParams<G, S>& p = *params;
  p.n = static_cast<int>(b.shapes.size());
  p.counters = reinterpret_cast<int*>(ws + l.counters);
  p.status = status;
  p.timeout_ns = kWaitTimeoutNs;
  int first = 0;
  int64_t tiles[kParts] = {0, 0, 0};             // of a step
  for (int k = 0; k < p.n; ++k) {
    const Shape& sh = b.shapes[k];
    const Planes& pl = l.shapes[k];
    const int64_t m = std::min(sh.rows, sh.cols), n = static_cast<int64_t>(sh.mats.size()) * P;
    const bool tall = sh.rows > sh.cols;
    ShapeInfo& info = p.info[k];
    ShapeMaps& maps = p.maps[k];
    info.first_mat = first;
    first += static_cast<int>(sh.mats.size());
    info.ld[0] = static_cast<int>(pl.x_ld);
    info.ld[1] = static_cast<int>(pl.s_ld);
    info.plane[0] = pl.x_plane;
    info.plane[1] = pl.s_plane;
    const size_t at[4] = {pl.x[0], pl.x[1], pl.a, pl.b};
    bool good = true;
    for (int i = 0; i < 4; ++i) {
      info.buf[i] = reinterpret_cast<__half*>(ws + at[i]);
      if (P == 1) good = good && encode_tmap_out(&maps.out[i], ws + at[i], i < 2 ? sh.cols : m,
                                     i < 2 ? sh.rows : m, n, i < 2 ? pl.x_ld : pl.s_ld) == CUDA_SUCCESS;
    }
    for (int part = 0; part < kParts; ++part) {
      const Dims d = dims_of(sh, part);
      ProdGroup& g = info.part[part];
      g.M = static_cast<int>(d.m);
      g.N = static_cast<int>(d.n);
      g.K = static_cast<int>(d.k);
      g.lower = part < 2 ? 1 : 0;
      g.a_kind = part == 1 ? kSymmetric : part == 0 ? (tall ? kAcross : kRowMajor)
                                                    : (tall ? kRowMajor : kSymmetric);
      g.b_kind = part == 1 ? kSymmetric : part == 0 ? (tall ? kAcross : kRowMajor)
                                                    : (tall ? kSymmetric : kAcross);
      g.tn = columns[part][k];
      g.chunks_b = g.tn % 128 == 0 ? g.tn / 128 : 0;
      const int width = ProdCfg<P>::kSub * g.tn;
      g.n_mt = static_cast<int>(ceil_div(g.M, kTileM));
      g.n_nt = static_cast<int>(ceil_div(g.N, width));
      g.per_mat = 0;
      for (int mt = 0; mt < g.n_mt; ++mt)
        g.per_mat += g.lower ? static_cast<int>(ceil_div(std::min((mt + 1) * kTileM, g.N), width))
                             : g.n_nt;
      g.begin = static_cast<int>(tiles[part]);
      tiles[part] += static_cast<int64_t>(g.per_mat) * static_cast<int64_t>(sh.mats.size());
      // the operands: X [rows, cols] or the symmetric A', B [m, m]
      for (int cur = 0; cur < (part == 1 ? 1 : 2); ++cur) {
        const auto operand = [&](Side* sides, int kind, int rows, int chunks) {
          Side* side = &sides[side_of(part, cur)];
          if (kind == kSymmetric && cur == 1) {
            *side = sides[side_of(part, 0)];
            return;
          }
          const bool x = kind != kSymmetric;
          const size_t from = x ? pl.x[cur] : part == 1 ? pl.a : pl.b;
          good = good && encode_side(side, kind, ws + from, x ? sh.cols : m, x ? sh.rows : m, n,
                                     x ? pl.x_ld : pl.s_ld, P, rows, chunks);
        };
        operand(maps.a, g.a_kind, kTileM / 2, 2);
        operand(maps.b, g.b_kind, g.tn / 2, g.chunks_b);
      }
    }
    if (!good) return cudaErrorInvalidValue;
  }
  int64_t total = 0;
  int before[kParts] = {0, 0, 0};
  for (int it = 0; it < a.iterations; ++it) {
    const double ca = a.coefficients[3 * it], cb = a.coefficients[3 * it + 1],
                 cc = a.coefficients[3 * it + 2];
    const double h = cc != 0.0 ? cb / (2.0 * cc) : 0.0;
    for (int part = 0; part < kParts; ++part) {
      if (part == 1 && cc == 0.0) continue;
      const double alpha = part == 0 ? (cc != 0.0 ? 1.0 : cb) : part == 1 ? cc : 1.0;
      const double gamma = part == 0 ? (cc != 0.0 ? h : ca) : part == 1 ? ca - cc * h * h : 0.0;
      Step& st = p.step[p.n_steps++];
      st.begin = static_cast<int>(total);
      st.alpha = static_cast<float>(alpha / kPlaneScale);
      st.gamma = static_cast<float>(gamma * kPlaneScale);
      st.part = static_cast<uint8_t>(part);
      st.cur = static_cast<uint8_t>(it & 1);
      st.dst = static_cast<uint8_t>(part == 2 ? (it & 1) ^ 1 : part == 0 && cc != 0.0 ? 2 : 3);
      for (int k = 0; k < kParts; ++k) st.before[k] = static_cast<uint8_t>(before[k]);
      ++before[part];
      total += tiles[part];
    }
  }
  // the counters: tiles handed out (one past the last a pair), and a matrix's epilogue warps
  bool counted = total <= INT32_MAX - most_clusters;
  for (int k = 0; k < p.n; ++k) {
    int64_t of_mat = 0;
    for (int part = 0; part < kParts; ++part)
      of_mat += static_cast<int64_t>(before[part]) * p.info[k].part[part].per_mat;
    counted = counted && of_mat <= kMostOfMatrix;
  }
  if (!counted) return cudaErrorInvalidConfiguration;
  p.n_tiles = static_cast<int>(total);
  const int64_t widest = std::max(tiles[0], std::max(tiles[1], tiles[2]));
  const int64_t clusters = std::max<int64_t>(1, std::min<int64_t>(most_clusters, widest));
  const auto kernel = products_kernel<P, G, S>;
  static PerDeviceOnce attr;
  const cudaError_t e = smem_attr_once(attr, kernel, ProdCfg<P>::kSmemBytes);
  if (e != cudaSuccess) return e;
  *launch = [kernel, params, clusters](cudaStream_t s) {
    return launch_dependent(kernel, dim3(static_cast<unsigned>(2 * clusters)), dim3(kThreads),
                            ProdCfg<P>::kSmemBytes, s, *params);
  };
  return cudaSuccess;
}

// Sizes of the launches' parameters: few and most.
constexpr int kFewGroups = 4, kFewMats = 48, kFewSteps = 18, kMaxSteps = kParts * 64;

}  // namespace

size_t muon_workspace(const bergson_muon_tensor* t, int n, int products) {
  size_t most = 256;
  for (const Batch& b : batches_of(t, n))
    most = std::max(most, layout_of(b, products == 3 ? 2 : 1).total);
  return most;
}

bool muon_counts(int64_t rows, int64_t cols, int products, int iterations) {
  const int64_t m = std::min(rows, cols), width = products == 3 ? kTileN : 2 * kTileN;
  int64_t tiles = ceil_div(rows, kTileM) * ceil_div(cols, width);
  for (int64_t r = kTileM; r < m + kTileM; r += kTileM)
    tiles += 2 * ceil_div(std::min(r, m), width);
  return tiles * iterations <= kMostOfMatrix;
}

cudaError_t launch_muon(const bergson_muon_tensor* t, int n, const MuonScalars& a, void* ws,
                        int* status, int sms, cudaStream_t s) {
  uint8_t* w = static_cast<uint8_t*>(ws);
  const std::vector<Batch> batches = batches_of(t, n);
  std::vector<BatchLayout> layouts;
  std::vector<Launch> products(batches.size());
  for (size_t i = 0; i < batches.size(); ++i) {
    const Batch& b = batches[i];
    layouts.push_back(layout_of(b, a.products == 3 ? 2 : 1));
    const BatchLayout& l = layouts.back();
    const bool short_run = b.shapes.size() <= kFewGroups && 3 * a.iterations <= kFewSteps;
    Launch* to = &products[i];
    cudaError_t e;
    if (a.products == 3)
      e = short_run ? prepare_products<2, kFewGroups, kFewSteps>(b, l, a, w, status, sms, to)
                    : prepare_products<2, kMaxGroups, kMaxSteps>(b, l, a, w, status, sms, to);
    else
      e = short_run ? prepare_products<1, kFewGroups, kFewSteps>(b, l, a, w, status, sms, to)
                    : prepare_products<1, kMaxGroups, kMaxSteps>(b, l, a, w, status, sms, to);
    if (e != cudaSuccess) return e;
  }
  for (size_t i = 0; i < batches.size(); ++i) {
    const Batch& b = batches[i];
    const BatchLayout& l = layouts[i];
    const bool few = b.mats <= kFewMats;
    cudaError_t e = few ? run_moments<kFewMats>(t, b, l, a, w, s)
                        : run_moments<kMaxMats>(t, b, l, a, w, s);
    if (e != cudaSuccess) return e;
    e = products[i](s);
    if (e != cudaSuccess) return e;
    e = few ? run_weights<kFewMats>(t, b, l, a, w, s) : run_weights<kMaxMats>(t, b, l, a, w, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace bergson
