// Embedding lookup with a scale, and its gradient.
//
//   forward   out_r = s table[id_r]
//   backward  dT[v] = s sum_{r: id_r = v} dy_r   (+ dT[v])
//
// Both are bound by their bytes.  The gradient is summed in fp32 and without
// atomics, so that it has the same bits every time: the rows are put in the order of
// their tokens, and what shares a token is added up in the order of the rows.
//
// Up to 4096 rows, one launch: the CTA of a token's first row finds the
// others by comparing tokens and adds them all (4096 rows of one token at d 2048: 253 us;
// 4097, by the sort, 81), and CTAs of their own write zeros to the rest of the table.  Above, a
// radix sort of (token, row), 9 bits a pass: counts per tile of rows, then every tile places its
// rows behind those of the tiles before it.  The sorted rows are added up 8 to 64 at a time, a run:
// a token whose rows all lie within such a run is done there; what it has of the tokens that cross
// its ends goes to the workspace and is joined by a last kernel.  There no run is longer than
// another, however often a token comes.
// 65,536 x 4096 bf16 lookups 111 us (6.2 TB/s); the gradient of 65,536 x 2048 into 50,304 rows
// 110 us: the sort 25 (latency), sums and zeros 75 (6.0 TB/s), joining 11.

#include <algorithm>

#include "internal.h"
#include "train.cuh"

namespace bergson {

namespace {

// ------------------------------------------------------------------ forward

constexpr int kLookupThreads = 128;

struct LookupParams {
  const void* table;
  const int64_t* ids;
  void* out;
  int64_t V, rows, ld_t, ld_o;
  int d, slabs;
  float scale;
  int* status;
};

// A warp takes 32 * C columns of a row.
template <typename T, bool kVec>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(
    const __grid_constant__ LookupParams p) {
  constexpr int C = kVec ? 4 * Vec16<T>::kElems : 8;
  using R = RowPart<T, kVec ? 16 : 0, C>;
  const int lane = threadIdx.x & 31;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kLookupThreads / 32) + (threadIdx.x >> 5);
  const int64_t r = unit / p.slabs;
  const int c0 = static_cast<int>(unit % p.slabs) * 32 * C;
  griddep_wait();
  if (r >= p.rows) return;
  const int64_t id = p.ids[r];
  const int d = min(p.d - c0, 32 * C);
  float x[C];
  if (id < 0 || id >= p.V) {
    if (id >= p.V && lane == 0 && c0 == 0) raise_device_error(p.status, nullptr, BERGSON_EINVAL);
    const float v = id < 0 ? 0.0f : __int_as_float(0x7fffffff);
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = v;
  } else {
    R row;
    row.load(static_cast<const T*>(p.table) + id * p.ld_t + c0, d, lane, 32);
    row.floats(x);
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] *= p.scale;
  }
  R::store(static_cast<T*>(p.out) + r * p.ld_o + c0, d, lane, 32, x);
}

// ------------------------------------------------------------------ backward

constexpr int kFewRows = 4096;                 // up to here one launch does it all
constexpr int kFewThreads = 512;
constexpr int kFewZeros = 512;                 // rows of the table a CTA of zeros looks after, at most,
constexpr int64_t kZeroBytes = 64 << 10;       //   and what they hold, about
constexpr int kMinRun = 8, kMaxRun = 64;       // sorted rows added up by one CTA
constexpr int64_t kManyRuns = 1000;            // CTAs that are worth longer runs
constexpr int kSumThreads = 128;
constexpr int kCols = 8;                       // columns a thread
constexpr int kFewAhead = 4;                   // rows on their way
constexpr int kJoinThreads = 256;               // a warp joins the token that a run ends in
constexpr int kJoinCols = 128;
constexpr int kShortParts = 16;                // of so many runs
constexpr int kSortThreads = 1024;
constexpr int kSortItems = 2048;               // items of a step of the sort
constexpr int kDigitBits = 9;
constexpr int kBins = 1 << kDigitBits;
constexpr int kMaxTiles = 128;
constexpr int kMaxPasses = 4;

struct GradOut {
  void* table;                 // [V, ld]
  int64_t ld;
  int type;
  int vec;                     // its rows take 16-byte accesses
  int add;
  float scale;
};

// E (1, 4 or 8) neighbouring columns of the table's row v, as they are.
template <int E>
__device__ __forceinline__ void get_columns(const GradOut& o, int64_t v, int col, int d, float* x) {
  const int64_t at = v * o.ld + col;
  if (E == 1 || !o.vec || col + E > d) {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = col + i < d ? load_any(o.table, o.type, at + i) : 0.0f;
    return;
  }
  if constexpr (E > 1) {
#pragma unroll
    for (int k = 0; k < E / 4; ++k) {
      if (o.type == BERGSON_F32) {
        const float4 z = reinterpret_cast<const float4*>(static_cast<const float*>(o.table) + at)[k];
        x[4 * k] = z.x; x[4 * k + 1] = z.y; x[4 * k + 2] = z.z; x[4 * k + 3] = z.w;
      } else {
        const uint2 z = reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(o.table) + at)[k];
        const uint4 w = make_uint4(z.x, z.y, 0, 0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 f = o.type == BERGSON_BF16
                               ? unpack2(w, h, static_cast<const __nv_bfloat16*>(nullptr))
                               : unpack2(w, h, static_cast<const __half*>(nullptr));
          x[4 * k + 2 * h] = f.x;
          x[4 * k + 2 * h + 1] = f.y;
        }
      }
    }
  }
}
// Sets them to x.
template <int E>
__device__ __forceinline__ void set_columns(const GradOut& o, int64_t v, int col, int d,
                                            const float* x) {
  const int64_t at = v * o.ld + col;
  if (E == 1 || !o.vec || col + E > d) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if (col + i >= d) return;
      if (o.type == BERGSON_BF16)
        static_cast<__nv_bfloat16*>(o.table)[at + i] = __float2bfloat16_rn(x[i]);
      else if (o.type == BERGSON_F16) static_cast<__half*>(o.table)[at + i] = __float2half_rn(x[i]);
      else static_cast<float*>(o.table)[at + i] = x[i];
    }
    return;
  }
  if constexpr (E > 1) {
    if (o.type == BERGSON_F32) {
      float4* t = reinterpret_cast<float4*>(static_cast<float*>(o.table) + at);
#pragma unroll
      for (int k = 0; k < E / 4; ++k)
        t[k] = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
      return;
    }
    uint4 w;
#pragma unroll
    for (int h = 0; h < E / 2; ++h) {
      const float2 f = make_float2(x[2 * h], x[2 * h + 1]);
      if (o.type == BERGSON_BF16) pack2(w, h, f, static_cast<const __nv_bfloat16*>(nullptr));
      else pack2(w, h, f, static_cast<const __half*>(nullptr));
    }
    uint16_t* t = static_cast<uint16_t*>(o.table) + at;
    if constexpr (E == 8) *reinterpret_cast<uint4*>(t) = w;
    else *reinterpret_cast<uint2*>(t) = make_uint2(w.x, w.y);
  }
}
// Their sum times the scale, added to what is there with o.add.
template <int E>
__device__ __forceinline__ void put_columns(const GradOut& o, int64_t v, int col, int d,
                                            const float* sum) {
  float x[E];
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = 0.0f;
  if (o.add) get_columns<E>(o, v, col, d, x);
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = fmaf(sum[i], o.scale, x[i]);
  set_columns<E>(o, v, col, d, x);
}

// A thread's columns of a slab of the table's row v.
template <typename R>
__device__ __forceinline__ void get_row(const GradOut& o, int64_t v, int c0, int d, int t, int G,
                                        float (&x)[kCols]) {
#pragma unroll
  for (int k = 0; k < R::kPer; ++k)
    if (c0 + R::col(t, G, k) < d) get_columns<R::E>(o, v, c0 + R::col(t, G, k), d, x + R::E * k);
}
// Sets them to the sum times the scale on top of `old`.
template <typename R>
__device__ __forceinline__ void put_row(const GradOut& o, int64_t v, int c0, int d, int t, int G,
                                        const float (&sum)[kCols], const float (&old)[kCols]) {
  float x[kCols];
#pragma unroll
  for (int i = 0; i < kCols; ++i) x[i] = fmaf(sum[i], o.scale, old[i]);
#pragma unroll
  for (int k = 0; k < R::kPer; ++k)
    if (c0 + R::col(t, G, k) < d) set_columns<R::E>(o, v, c0 + R::col(t, G, k), d, x + R::E * k);
}

// Zeros in the table's row v, by `n` threads of which this is the t-th: 16 bytes at a time between
// the row's first and last 16-byte boundaries.
__device__ __forceinline__ void zero_row(const GradOut& o, int64_t v, int d, int t, int n) {
  const int64_t size = o.type == BERGSON_F32 ? 4 : 2;
  uint8_t* row = static_cast<uint8_t*>(o.table) + v * o.ld * size;
  const int64_t bytes = d * size;
  const int64_t head = min(bytes, static_cast<int64_t>(-reinterpret_cast<uintptr_t>(row) & 15));
  const int64_t vecs = (bytes - head) / 16, tail = head + 16 * vecs;
  uint4* whole = reinterpret_cast<uint4*>(row + head);
  for (int64_t i = t; i < vecs; i += n) whole[i] = make_uint4(0, 0, 0, 0);
  if (2 * t < head) reinterpret_cast<uint16_t*>(row)[t] = 0;
  if (2 * t < bytes - tail) reinterpret_cast<uint16_t*>(row + tail)[t] = 0;
}

struct FewParams {
  const void* dy;
  const int64_t* ids;
  GradOut out;
  int64_t V, ld_dy;
  int rows, d, slabs, group;   // threads of a row's slab
  int zeros;                   // rows of the table a CTA of zeros looks after
  int* status;
};

// CTA r * slabs + k: the token whose first row is r, slab k.  The CTAs behind: zeros.
template <typename T, bool kVec>
__global__ void __launch_bounds__(kFewThreads, 3) few_rows_kernel(
    const __grid_constant__ FewParams p) {
  using R = RowPart<T, kVec ? 16 : 0, kCols>;
  __shared__ uint16_t list[kFewRows];
  __shared__ int counts[kFewThreads / 32];
  __shared__ float joined[kFewThreads * kCols];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  griddep_wait();
  const int n_sum = p.rows * p.slabs;
  if (static_cast<int>(blockIdx.x) >= n_sum) {
    uint8_t* touched = reinterpret_cast<uint8_t*>(list);
    for (int i = tid; i < p.zeros; i += kFewThreads) touched[i] = 0;
    __syncthreads();
    const int64_t v0 = static_cast<int64_t>(blockIdx.x - n_sum) * p.zeros;
    for (int j = tid; j < p.rows; j += kFewThreads) {
      const int64_t id = p.ids[j];
      if (id >= v0 && id < v0 + p.zeros) touched[id - v0] = 1;
    }
    __syncthreads();
    if (p.zeros < kFewThreads / 32) {              // few wide rows: all threads for each
      for (int i = 0; i < p.zeros && v0 + i < p.V; ++i)
        if (!touched[i]) zero_row(p.out, v0 + i, p.d, tid, kFewThreads);
      return;
    }
    for (int i = warp; i < p.zeros && v0 + i < p.V; i += kFewThreads / 32)
      if (!touched[i]) zero_row(p.out, v0 + i, p.d, lane, 32);
    return;
  }
  const int r = blockIdx.x / p.slabs, slab = blockIdx.x % p.slabs;
  const int64_t id = p.ids[r];
  if (id < 0) return;
  if (id >= p.V) {
    if (tid == 0 && slab == 0) raise_device_error(p.status, nullptr, BERGSON_EINVAL);
    return;
  }
  for (int j0 = 0; j0 < r; j0 += kFewThreads)      // frequent tokens end early
    if (__syncthreads_or(j0 + tid < r && p.ids[j0 + tid] == id)) return;
  int n = 0;
  for (int j0 = r; j0 < p.rows; j0 += kFewThreads) {
    const bool mine = j0 + tid < p.rows && p.ids[j0 + tid] == id;
    const unsigned votes = __ballot_sync(0xffffffffu, mine);
    if (lane == 0) counts[warp] = __popc(votes);
    __syncthreads();
    const int c = lane < kFewThreads / 32 ? counts[lane] : 0;
    const int below = __reduce_add_sync(0xffffffffu, lane < warp ? c : 0);
    const int all = __reduce_add_sync(0xffffffffu, c);
    if (mine) list[n + below + __popc(votes & ((1u << lane) - 1))] = static_cast<uint16_t>(j0 + tid);
    n += all;
    __syncthreads();
  }
  // `groups` of threads take parts of the list, joined in order
  const int groups = kFewThreads / p.group, g = tid / p.group, t = tid % p.group;
  const int per = (n + groups - 1) / groups;
  const int c0 = slab * p.group * kCols;
  float old[kCols];
#pragma unroll
  for (int i = 0; i < kCols; ++i) old[i] = 0.0f;
  if (p.out.add && g == 0) get_row<R>(p.out, id, c0, p.d, t, p.group, old);
  float sum[kCols];
#pragma unroll
  for (int i = 0; i < kCols; ++i) sum[i] = 0.0f;
  if (g < groups) {
    const int end = min(n, (g + 1) * per);
    for (int k0 = g * per; k0 < end; k0 += kFewAhead) {
      R row[kFewAhead];
#pragma unroll
      for (int k = 0; k < kFewAhead; ++k) {
        const int64_t at = k0 + k < end ? list[k0 + k] : 0;
        row[k].load(static_cast<const T*>(p.dy) + at * p.ld_dy + c0, k0 + k < end ? p.d - c0 : 0, t,
                    p.group);
      }
#pragma unroll
      for (int k = 0; k < kFewAhead; ++k) {
        if (k0 + k >= end) break;
        float x[kCols];
        row[k].floats(x);
#pragma unroll
        for (int i = 0; i < kCols; ++i) sum[i] += x[i];
      }
    }
  }
  if (n > 1) {
#pragma unroll
    for (int i = 0; i < kCols; ++i) joined[i * kFewThreads + tid] = sum[i];
    __syncthreads();
    if (g == 0) {
      for (int k = 1; k < groups && k * per < n; ++k) {
#pragma unroll
        for (int i = 0; i < kCols; ++i) sum[i] += joined[i * kFewThreads + k * p.group + t];
      }
    }
  }
  if (g == 0) put_row<R>(p.out, id, c0, p.d, t, p.group, sum, old);
}

// ---- the sort.  Keys are tokens; rows that take no part have V, behind all others.

struct SortParams {
  const int64_t* ids;
  const uint32_t* key_in;      // nullptr: ids, of rows 0, 1, ..
  const int* row_in;
  uint32_t* key_out;
  int* row_out;
  int* table;                  // [tiles, kBins] of this pass
  int* next_table;             // of the next pass, or nullptr: the last one
  uint8_t* touched;            // [V]
  int64_t V, rows;
  int64_t tile;                // rows of a tile, a multiple of kSortItems
  int tiles, shift, next_shift;
  int64_t clear_words;         // of next tables, 4-byte words from clear on
  int* clear;
  int* status;
};

__device__ __forceinline__ uint32_t sort_key(const SortParams& p, int64_t i) {
  if (p.key_in != nullptr) return p.key_in[i];
  const int64_t id = p.ids[i];
  return static_cast<uint32_t>(id >= 0 && id < p.V ? id : p.V);
}

// The first pass's counts per tile; also clears the later passes' and the marks of touched rows.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(
    const __grid_constant__ SortParams p) {
  __shared__ int bins[kBins];
  griddep_wait();
  const int64_t step = static_cast<int64_t>(gridDim.x) * kSortThreads;
  const int64_t me = static_cast<int64_t>(blockIdx.x) * kSortThreads + threadIdx.x;
  for (int64_t i = me; i < p.clear_words; i += step) p.clear[i] = 0;
  if (static_cast<int>(blockIdx.x) >= p.tiles) return;
  if (threadIdx.x < kBins) bins[threadIdx.x] = 0;
  __syncthreads();
  const int64_t end = min((blockIdx.x + 1) * p.tile, p.rows);
  for (int64_t i = blockIdx.x * p.tile + threadIdx.x; i < end; i += kSortThreads) {
    if (p.ids[i] >= p.V) raise_device_error(p.status, nullptr, BERGSON_EINVAL);
    atomicAdd(&bins[(sort_key(p, i) >> p.shift) & (kBins - 1)], 1);
  }
  __syncthreads();
  if (threadIdx.x < kBins) p.table[blockIdx.x * kBins + threadIdx.x] = bins[threadIdx.x];
}

// Places a tile's items: behind those of smaller digits and those of the tiles before it.
__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(
    const __grid_constant__ SortParams p) {
  constexpr int kWarps = kSortThreads / 32;
  constexpr int kRounds = kSortItems / kSortThreads;
  __shared__ uint16_t hist[kWarps][kBins];
  __shared__ int base[kBins];
  __shared__ int part[2][2][kBins];
  __shared__ int scan[kBins / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t begin = blockIdx.x * p.tile, end = min(begin + p.tile, p.rows);
  griddep_wait();
  uint32_t key[kRounds];
  int row[kRounds];
  const auto fetch = [&](int64_t i0) {
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const int64_t i = i0 + (warp * kRounds + k) * 32 + lane;
      key[k] = i < end ? sort_key(p, i) : 0;
      row[k] = p.row_in != nullptr && i < end ? p.row_in[i] : static_cast<int>(i);
    }
  };
  fetch(begin);
  {
    // what stands before this tile and in all: two halves of the tiles a digit
    const int digit = tid & (kBins - 1), half = tid / kBins;
    int before = 0, all = 0;
#pragma unroll 8
    for (int t = half; t < p.tiles; t += kSortThreads / kBins) {
      const int c = p.table[t * kBins + digit];
      all += c;
      before += t < static_cast<int>(blockIdx.x) ? c : 0;
    }
    part[half][0][digit] = before;
    part[half][1][digit] = all;
    __syncthreads();
    int total = 0, incl = 0;
    if (tid < kBins) {
      before = part[0][0][tid] + part[1][0][tid];
      total = part[0][1][tid] + part[1][1][tid];
      incl = total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) scan[warp] = incl;
    }
    __syncthreads();
    if (tid < kBins) {
      for (int w = 0; w < warp; ++w) incl += scan[w];
      base[tid] = incl - total + before;
    }
  }
  for (int64_t i0 = begin; i0 < end; i0 += kSortItems) {
    for (int i = tid; i < kWarps * kBins / 2; i += kSortThreads)
      reinterpret_cast<uint32_t*>(hist)[i] = 0;
    __syncthreads();
    unsigned same[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const int64_t i = i0 + (warp * kRounds + k) * 32 + lane;
      // an item past the end has a digit of its own
      const uint32_t digit = i < end ? (key[k] >> p.shift) & (kBins - 1) : kBins;
      same[k] = __match_any_sync(0xffffffffu, digit);
      if (i < end && lane == __ffs(same[k]) - 1) hist[warp][digit] += __popc(same[k]);
      __syncwarp();
    }
    __syncthreads();
    int sum = 0;
    if (tid < kBins) {
#pragma unroll 8
      for (int w = 0; w < kWarps; ++w) {
        const int c = hist[w][tid];
        hist[w][tid] = static_cast<uint16_t>(sum);
        sum += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const int64_t i = i0 + (warp * kRounds + k) * 32 + lane;
      const uint32_t digit = (key[k] >> p.shift) & (kBins - 1);
      int at = 0;
      if (i < end) at = base[digit] + hist[warp][digit] + __popc(same[k] & ((1u << lane) - 1));
      __syncwarp();
      if (i < end) {
        if (lane == __ffs(same[k]) - 1) hist[warp][digit] += __popc(same[k]);
        p.key_out[at] = key[k];
        p.row_out[at] = row[k];
        if (p.next_table != nullptr)
          atomicAdd(&p.next_table[at / p.tile * kBins + ((key[k] >> p.next_shift) & (kBins - 1))], 1);
        else if (p.touched != nullptr && key[k] < p.V)
          p.touched[key[k]] = 1;
      }
      __syncwarp();
    }
    __syncthreads();
    if (tid < kBins) base[tid] += sum;
    if (i0 + kSortItems < end) fetch(i0 + kSortItems);
  }
}

// ---- sums of the sorted rows

struct SumParams {
  const void* dy;
  const uint32_t* key;
  const int* row;
  const uint8_t* touched;      // nullptr: no zeros
  float* part;                 // [runs, 2, ld_part]
  GradOut out;
  int64_t V, rows, ld_dy, ld_part;
  int64_t runs;
  int64_t n_sum;               // CTAs that add
  int d, slabs;
  int run;                     // rows of a run, a multiple of 8
};

// kAdd: the table's rows that are done here come with the rows that are added to them.
template <typename T, bool kVec, bool kAdd>
__global__ void __launch_bounds__(kSumThreads) sum_kernel(const __grid_constant__ SumParams p) {
  constexpr int kAhead = kAdd ? 4 : 8;           // rows on their way
  using R = RowPart<T, kVec ? 16 : 0, kCols>;
  __shared__ uint32_t keys[kMaxRun + 2];         // one before, one behind
  __shared__ int rows[kMaxRun];
  const int tid = threadIdx.x, G = blockDim.x, length = p.run;
  griddep_wait();
  if (blockIdx.x >= p.n_sum) {
    const int64_t step = static_cast<int64_t>(gridDim.x - p.n_sum) * (G / 32);
    for (int64_t v = (blockIdx.x - p.n_sum) * (G / 32) + (tid >> 5); v < p.V; v += step)
      if (!p.touched[v]) zero_row(p.out, v, p.d, tid & 31, 32);
    return;
  }
  const uint32_t none = static_cast<uint32_t>(p.V);
  const int64_t run = blockIdx.x / p.slabs, p0 = run * length;
  const int c0 = static_cast<int>(blockIdx.x % p.slabs) * G * kCols;
  for (int i = tid; i < length + 2; i += G) {
    const int64_t at = p0 + i - 1;
    keys[i] = at >= 0 && at < p.rows ? p.key[at] : none;
    if (i < length) rows[i] = p0 + i < p.rows ? p.row[p0 + i] : 0;
  }
  __syncthreads();
  bool open = keys[0] == keys[1];                // the first token began before
  float sum[kCols];
#pragma unroll
  for (int i = 0; i < kCols; ++i) sum[i] = 0.0f;
  for (int j0 = 0; j0 < length; j0 += kAhead) {
    if (keys[j0 + 1] == none) break;
    R row[kAhead];
    float old[kAdd ? kAhead : 1][kCols];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t v = keys[j0 + k + 1];
      row[k].load(static_cast<const T*>(p.dy) + rows[j0 + k] * p.ld_dy + c0, v != none ? p.d - c0 : 0,
                  tid, G);
      if constexpr (kAdd) {
        // a token that ends here and did not begin before the run
        if (v != none && keys[j0 + k + 2] != v && v != keys[0])
          get_row<R>(p.out, v, c0, p.d, tid, G, old[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int j = j0 + k;
      const uint32_t v = keys[j + 1];
      if (v == none) break;
      float x[kCols];
      row[k].floats(x);
#pragma unroll
      for (int i = 0; i < kCols; ++i) sum[i] += x[i];
      const bool ends = keys[j + 2] != v;
      if (!ends && j < length - 1) continue;
      if (open || !ends) {
        float* part = p.part + (2 * run + (open ? 0 : 1)) * p.ld_part;
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          const int c = c0 + R::column(tid, G, i);
          if (c < p.d) part[c] = sum[i];
        }
      } else {
        float zero[kCols];
#pragma unroll
        for (int i = 0; i < kCols; ++i) zero[i] = 0.0f;
        if constexpr (kAdd) put_row<R>(p.out, v, c0, p.d, tid, G, sum, old[k]);
        else put_row<R>(p.out, v, c0, p.d, tid, G, sum, zero);
      }
      open = false;
#pragma unroll
      for (int i = 0; i < kCols; ++i) sum[i] = 0.0f;
    }
  }
}

// The part sums [begin, end) of a token that begins in `run`: 0 is that run's second sum, q the
// first of run + q.  Four columns a lane.
__device__ __forceinline__ float4 add_parts(const SumParams& p, int64_t run, int64_t begin,
                                            int64_t end, int col) {
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  constexpr int kParts = 8;                      // on their way
  for (int64_t q0 = begin; q0 < end; q0 += kParts) {
    float4 x[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int64_t q = q0 + k;
      x[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (q < end)
        x[k] = *reinterpret_cast<const float4*>(
            p.part + (2 * (run + q) + (q == 0 ? 1 : 0)) * p.ld_part + col);
    }
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      sum.x += x[k].x; sum.y += x[k].y; sum.z += x[k].z; sum.w += x[k].w;
    }
  }
  return sum;
}

// The tokens that cross ends of runs: the warp of the run where a token begins adds what that
// run and the next ones have of it.  What more than kShortParts runs have is added by all the CTA's
// warps, a stretch each, joined in order.
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ SumParams p) {
  constexpr int kWarps = kJoinThreads / 32;
  __shared__ float4 red[kWarps][32];
  __shared__ int64_t parts[kWarps];              // of the warps' tokens that are left
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = static_cast<int>(blockIdx.y) * kJoinCols + 4 * lane;
  const bool mine = col < p.ld_part;
  const uint32_t none = static_cast<uint32_t>(p.V);
  griddep_wait();
  const int64_t run0 = static_cast<int64_t>(blockIdx.x) * kWarps, run = run0 + warp;
  const int64_t last = run * p.run + p.run - 1;
  int64_t n = 0;                                 // part sums, if a token that goes on begins here
  uint32_t v = none;
  if (last + 1 < p.rows) {
    v = p.key[last];
    const uint32_t next = p.key[last + 1];
    const uint32_t before = run > 0 ? p.key[run * p.run - 1] : none;
    if (v != none && next == v && before != v) {
      // does run + n hold some too?  128 runs a step
      for (n = 2;; n += 128) {
        uint32_t first[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t at = (run + n + 32 * k + lane) * p.run;
          first[k] = at < p.rows ? p.key[at] : none;
        }
        int more = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const unsigned votes = __ballot_sync(0xffffffffu, first[k] == v);
          if (more == 32 * k) more += votes == 0xffffffffu ? 32 : __ffs(~votes) - 1;
        }
        if (more < 128) {
          n += more;
          break;
        }
      }
    }
  }
  const bool many = n > kShortParts;
  if (n > 0 && !many && mine) {
    const float4 s = add_parts(p, run, 0, n, col);
    const float sum[4] = {s.x, s.y, s.z, s.w};
    if (col < p.d) put_columns<4>(p.out, v, col, p.d, sum);
  }
  if (lane == 0) parts[warp] = many ? n : 0;
  if (!__syncthreads_or(many)) return;
  for (int k = 0; k < kWarps; ++k) {
    const int64_t all = parts[k];
    if (all == 0) continue;
    const int64_t per = (all + kWarps - 1) / kWarps;
    const int64_t begin = min(warp * per, all), end = min(begin + per, all);
    __syncthreads();                             // the last token's sums have been read
    if (mine) red[warp][lane] = add_parts(p, run0 + k, begin, end, col);
    __syncthreads();
    if (warp == 0 && col < p.d) {
      float4 s = red[0][lane];
      for (int w = 1; w < kWarps; ++w) {
        const float4 x = red[w][lane];
        s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
      }
      const float sum[4] = {s.x, s.y, s.z, s.w};
      put_columns<4>(p.out, p.key[(run0 + k + 1) * p.run - 1], col, p.d, sum);
    }
  }
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Threads of a row's slab: 8 columns each.
int slab_threads(int64_t d) {
  return static_cast<int>(std::min<int64_t>(kSumThreads, ceil_div(ceil_div(d, kCols), 32) * 32));
}

struct SortPlan {
  int passes = 1, tiles = 1, run = kMinRun;
  int64_t tile = kSortItems, runs = 0, ld_part = 0;
  size_t table = 0, touched = 0, key[2] = {0, 0}, row[2] = {0, 0}, part = 0, total = 0;
  int64_t clear_words = 0;     // from the second pass's table to the end of `touched`
};

// Long runs have less to join, short ones more rows on their way when there are few: 32 rows a run
// for all had 5009 x 437 at 41 us and 33,799 x 5463 at 146; by this rule 32 and 129.  With rows
// of the table beside them (add) a run takes twice the turns.
int run_rows(int64_t rows, int64_t d, bool add) {
  const int64_t ctas = rows * ceil_div(d, slab_threads(d) * kCols);      // of runs of one row
  const int64_t many = add ? 2 * kManyRuns : kManyRuns;
  int run = kMinRun;
  while (run < (add ? kMaxRun / 2 : kMaxRun) && ctas >= 2 * run * many) run *= 2;
  return run;
}

SortPlan sort_plan(int64_t rows, int64_t V, int64_t d, bool add) {
  SortPlan s;
  int bits = 1;
  while ((V >> bits) != 0) ++bits;             // keys are 0 .. V
  s.passes = static_cast<int>(ceil_div(bits, kDigitBits));
  s.tile = ceil_div(ceil_div(rows, kMaxTiles), kSortItems) * kSortItems;
  s.tiles = static_cast<int>(ceil_div(rows, s.tile));
  s.run = run_rows(rows, d, add);
  s.runs = ceil_div(rows, s.run);
  s.ld_part = ceil_div(d, 8) * 8;
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round256(bytes);
    return here;
  };
  const size_t one = static_cast<size_t>(s.tiles) * kBins * sizeof(int);
  s.table = take(one * s.passes);
  s.touched = take(static_cast<size_t>(V));
  s.clear_words = static_cast<int64_t>((at - s.table - one) / 4);
  for (int i = 0; i < 2; ++i) {
    s.key[i] = take(static_cast<size_t>(rows) * 4);
    s.row[i] = take(static_cast<size_t>(rows) * 4);
  }
  s.part = take(static_cast<size_t>(s.runs) * 2 * s.ld_part * sizeof(float));
  s.total = at;
  return s;
}

template <typename T, bool kVec>
cudaError_t run_few(const bergson_embedding_grad_args& a, const GradOut& out, int* status,
                    cudaStream_t s) {
  FewParams p = {};
  p.dy = a.dy;
  p.ids = a.ids;
  p.out = out;
  p.V = a.V;
  p.ld_dy = a.ld_dy;
  p.rows = static_cast<int>(a.rows);
  p.d = static_cast<int>(a.d);
  p.group = slab_threads(a.d);
  p.slabs = static_cast<int>(ceil_div(a.d, p.group * kCols));
  p.status = status;
  const int64_t row_bytes = a.d * (a.t_dtype == BERGSON_F32 ? 4 : 2);
  p.zeros = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kFewZeros, kZeroBytes / row_bytes)));
  const int64_t grid = a.rows * p.slabs + (a.add ? 0 : ceil_div(a.V, p.zeros));
  return launch_dependent(few_rows_kernel<T, kVec>, dim3(static_cast<unsigned>(grid)),
                          dim3(kFewThreads), 0, s, p);
}

template <typename T, bool kVec>
cudaError_t run_sums(const bergson_embedding_grad_args& a, SumParams p, cudaStream_t s) {
  const int threads = slab_threads(a.d);
  p.slabs = static_cast<int>(ceil_div(a.d, threads * kCols));
  p.n_sum = p.runs * p.slabs;
  const int64_t zeros =
      a.add ? 0 : std::min<int64_t>(ceil_div(a.V, threads / 32), 4 * kPlanCTAs);
  const auto kernel = a.add ? sum_kernel<T, kVec, true> : sum_kernel<T, kVec, false>;
  return launch_dependent(kernel, dim3(static_cast<unsigned>(p.n_sum + zeros)), dim3(threads), 0, s,
                          p);
}

cudaError_t run_sorted(const bergson_embedding_grad_args& a, const GradOut& out, bool vec,
                       uint8_t* ws, int* status, cudaStream_t s) {
  const SortPlan plan = sort_plan(a.rows, a.V, a.d, a.add != 0);
  SortParams p = {};
  p.ids = a.ids;
  p.table = reinterpret_cast<int*>(ws + plan.table);
  p.V = a.V;
  p.rows = a.rows;
  p.tile = plan.tile;
  p.tiles = plan.tiles;
  p.clear = p.table + plan.tiles * kBins;
  p.clear_words = a.add ? static_cast<int64_t>(plan.passes - 1) * plan.tiles * kBins
                        : plan.clear_words;
  p.status = status;
  const int64_t ctas =
      std::max<int64_t>(plan.tiles, std::min<int64_t>(kPlanCTAs, p.clear_words / 8192));
  cudaError_t e = launch_dependent(sort_count_kernel, dim3(static_cast<unsigned>(ctas)),
                                   dim3(kSortThreads), 0, s, p);
  for (int k = 0; k < plan.passes && e == cudaSuccess; ++k) {
    const bool last = k == plan.passes - 1;
    p.key_in = k == 0 ? nullptr : p.key_out;
    p.row_in = k == 0 ? nullptr : p.row_out;
    p.key_out = reinterpret_cast<uint32_t*>(ws + plan.key[k & 1]);
    p.row_out = reinterpret_cast<int*>(ws + plan.row[k & 1]);
    p.table = reinterpret_cast<int*>(ws + plan.table) + k * plan.tiles * kBins;
    p.next_table = last ? nullptr : p.table + plan.tiles * kBins;
    p.shift = k * kDigitBits;
    p.next_shift = p.shift + kDigitBits;
    p.touched = a.add ? nullptr : ws + plan.touched;
    e = launch_dependent(sort_place_kernel, dim3(static_cast<unsigned>(plan.tiles)),
                         dim3(kSortThreads), 0, s, p);
  }
  if (e != cudaSuccess) return e;
  SumParams q = {};
  q.dy = a.dy;
  q.key = p.key_out;
  q.row = p.row_out;
  q.touched = p.touched;
  q.part = reinterpret_cast<float*>(ws + plan.part);
  q.out = out;
  q.V = a.V;
  q.rows = a.rows;
  q.ld_dy = a.ld_dy;
  q.ld_part = plan.ld_part;
  q.runs = plan.runs;
  q.run = plan.run;
  q.d = static_cast<int>(a.d);
  if (a.dtype == BERGSON_BF16)
    e = vec ? run_sums<__nv_bfloat16, true>(a, q, s) : run_sums<__nv_bfloat16, false>(a, q, s);
  else if (a.dtype == BERGSON_F16)
    e = vec ? run_sums<__half, true>(a, q, s) : run_sums<__half, false>(a, q, s);
  else
    e = vec ? run_sums<float, true>(a, q, s) : run_sums<float, false>(a, q, s);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>(ceil_div(plan.runs, kJoinThreads / 32)),
                  static_cast<unsigned>(ceil_div(a.d, kJoinCols)));
  return launch_dependent(join_kernel, grid, dim3(kJoinThreads), 0, s, q);
}

template <typename T>
cudaError_t run_lookup(const bergson_embedding_args& a, int* status, cudaStream_t s) {
  const bool vec = on16(a.table, a.ld_t, sizeof(T)) && on16(a.out, a.ld_o, sizeof(T));
  LookupParams p = {};
  p.table = a.table;
  p.ids = a.ids;
  p.out = a.out;
  p.V = a.V;
  p.rows = a.rows;
  p.ld_t = a.ld_t;
  p.ld_o = a.ld_o;
  p.d = static_cast<int>(a.d);
  p.slabs = static_cast<int>(ceil_div(a.d, 32 * (vec ? 4 * Vec16<T>::kElems : 8)));
  p.scale = static_cast<float>(a.scale);
  p.status = status;
  const int64_t grid = ceil_div(a.rows * p.slabs, kLookupThreads / 32);
  if (grid > INT32_MAX) return cudaErrorInvalidConfiguration;
  const auto kernel = vec ? lookup_kernel<T, true> : lookup_kernel<T, false>;
  return launch_dependent(kernel, dim3(static_cast<unsigned>(grid)), dim3(kLookupThreads), 0, s, p);
}

}  // namespace

cudaError_t launch_embedding(const bergson_embedding_args& a, int* status, cudaStream_t s) {
  if (a.dtype == BERGSON_BF16) return run_lookup<__nv_bfloat16>(a, status, s);
  if (a.dtype == BERGSON_F16) return run_lookup<__half>(a, status, s);
  return run_lookup<float>(a, status, s);
}

size_t embedding_backward_workspace(int64_t rows, int64_t V, int64_t d) {
  return rows <= kFewRows ? 256 : sort_plan(rows, V, d, true).total;
}

cudaError_t launch_embedding_backward(const bergson_embedding_grad_args& a, void* ws, int* status,
                                      cudaStream_t s) {
  GradOut out = {};
  out.table = a.d_table;
  out.ld = a.ld_t;
  out.type = a.t_dtype;
  out.vec = on16(a.d_table, a.ld_t, a.t_dtype == BERGSON_F32 ? 4 : 2) ? 1 : 0;
  out.add = a.add ? 1 : 0;
  out.scale = static_cast<float>(a.scale);
  const bool vec = on16(a.dy, a.ld_dy, a.dtype == BERGSON_F32 ? 4 : 2);
  if (a.rows > kFewRows) return run_sorted(a, out, vec, static_cast<uint8_t*>(ws), status, s);
  if (a.rows == 0 && a.add) return cudaSuccess;
  if (a.dtype == BERGSON_BF16)
    return vec ? run_few<__nv_bfloat16, true>(a, out, status, s)
               : run_few<__nv_bfloat16, false>(a, out, status, s);
  if (a.dtype == BERGSON_F16)
    return vec ? run_few<__half, true>(a, out, status, s)
               : run_few<__half, false>(a, out, status, s);
  return vec ? run_few<float, true>(a, out, status, s) : run_few<float, false>(a, out, status, s);
}

}  // namespace bergson
