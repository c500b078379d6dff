// Device helpers of the training-side operators: element types, a thread's part of
// a row, block sums and the codes of 8-bit optimiser states.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "ptx.cuh"
#include "train.h"

namespace bergson {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---- two fp32 lanes at once (sm_100 and later issue them as one instruction)
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{.reg .b64 a, b, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 r, a, b;\n\tmov.b64 {%0, %1}, r;}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{.reg .b64 a, b, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mul.rn.f32x2 r, a, b;\n\tmov.b64 {%0, %1}, r;}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{.reg .b64 a, b, c, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mov.b64 c, {%6, %7};\n\tfma.rn.f32x2 r, a, b, c;\n\tmov.b64 {%0, %1}, r;}"
      : "=f"(r.x), "=f"(r.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 pair(float x) { return make_float2(x, x); }

__device__ __forceinline__ float exp2_approx(float x) {     // 2 units; 0 below 2^-126
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- 16 bytes of a tensor as pairs of fp32, and back
template <typename T>
struct Vec16 {
  static constexpr int kElems = 16 / sizeof(T);
  static constexpr int kPairs = kElems / 2;
};
__device__ __forceinline__ float2 unpack2(const uint4& v, int k, const float*) {
  return k == 0 ? make_float2(__uint_as_float(v.x), __uint_as_float(v.y))
                : make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int k) {
  return k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w;
}
__device__ __forceinline__ float2 unpack2(const uint4& v, int k, const __nv_bfloat16*) {
  const uint32_t u = word(v, k);
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(const uint4& v, int k, const __half*) {
  const uint32_t u = word(v, k);
  return __half22float2(*reinterpret_cast<const __half2*>(&u));
}
__device__ __forceinline__ void pack2(uint4& v, int k, float2 x, const float*) {
  if (k == 0) { v.x = __float_as_uint(x.x); v.y = __float_as_uint(x.y); }
  else { v.z = __float_as_uint(x.x); v.w = __float_as_uint(x.y); }
}
__device__ __forceinline__ void set_word(uint4& v, int k, uint32_t u) {
  if (k == 0) v.x = u; else if (k == 1) v.y = u; else if (k == 2) v.z = u; else v.w = u;
}
__device__ __forceinline__ void pack2(uint4& v, int k, float2 x, const __nv_bfloat16*) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
  set_word(v, k, *reinterpret_cast<const uint32_t*>(&h));
}
__device__ __forceinline__ void pack2(uint4& v, int k, float2 x, const __half*) {
  const __half2 h = __floats2half2_rn(x.x, x.y);
  set_word(v, k, *reinterpret_cast<const uint32_t*>(&h));
}
// The largest of the elements (NaN is passed over).
__device__ __forceinline__ float vec_max(const uint4& v, const float*) {
  return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)),
               fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
template <typename H2>
__device__ __forceinline__ H2 vec_max2(const uint4& v) {
  const H2* h = reinterpret_cast<const H2*>(&v);
  return __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
}

// Host helpers of the launchers.
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Rows of a matrix that can be accessed 16 (4) bytes at a time.
inline bool on_bytes(const void* p, int64_t ld, size_t size, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0 && ld * size % n == 0;
}
inline bool on16(const void* p, int64_t ld, size_t size) { return on_bytes(p, ld, size, 16); }

__device__ __forceinline__ float load_any(const void* p, int type, int64_t i) {
  if (type == BERGSON_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  if (type == BERGSON_F16) return __half2float(static_cast<const __half*>(p)[i]);
  return static_cast<const float*>(p)[i];
}

// A thread's columns of a row and how they lie in it: kPer vectors of kB bytes (16; 4, of two 16-bit
// elements; 0: an element), vector k at column E (t + k G) for thread t of the G that share the row.
template <typename T, int kB, int C>
struct RowPart {
  static_assert(kB == 16 || (kB == 4 && sizeof(T) == 2) || kB == 0, "vectors of 16 or 4 bytes");
  static constexpr bool kVec = kB == 16;
  static constexpr int E = kB == 0 ? 1 : kB / static_cast<int>(sizeof(T));
  static constexpr int kPer = C / E;
  // As they lie in memory.
  static constexpr int kWords = kVec ? 4 * kPer : kPer;
  uint32_t raw[kWords];

  __device__ __forceinline__ static int col(int t, int G, int k) { return E * (t + k * G); }
  // The column of element i of the thread's C.
  __device__ __forceinline__ static int column(int t, int G, int i) {
    return col(t, G, i / E) + i % E;
  }

  __device__ __forceinline__ void load(const T* row, int d, int t, int G) {
    const T* p = row + E * t;
    const int left = d - E * t, step = E * G;    // columns from the thread's first one on
#pragma unroll
    for (int k = 0; k < kPer; ++k, p += step) {
      const int n = left - k * step;
      if constexpr (kVec) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (n >= E) {
          v = *reinterpret_cast<const uint4*>(p);
        } else if (n > 0) {
          __align__(16) T part[E];
#pragma unroll
          for (int i = 0; i < E; ++i) part[i] = i < n ? p[i] : T(0.0f);
          v = *reinterpret_cast<const uint4*>(part);
        }
        raw[4 * k] = v.x; raw[4 * k + 1] = v.y; raw[4 * k + 2] = v.z; raw[4 * k + 3] = v.w;
      } else if constexpr (kB == 4) {
        raw[k] = n >= 2 ? *reinterpret_cast<const uint32_t*>(p)
                 : n == 1 ? *reinterpret_cast<const uint16_t*>(p) : 0;
      } else {
        raw[k] = 0;
        if (n > 0) {
          if constexpr (sizeof(T) == 2) raw[k] = *reinterpret_cast<const uint16_t*>(p);
          else raw[k] = __float_as_uint(*p);
        }
      }
    }
  }
  // Pairs of neighbours among the thread's C.
  __device__ __forceinline__ void pairs(float2 (&x)[C / 2]) const {
    if constexpr (kVec) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const uint4 v = make_uint4(raw[4 * k], raw[4 * k + 1], raw[4 * k + 2], raw[4 * k + 3]);
#pragma unroll
        for (int i = 0; i < E / 2; ++i)
          x[E / 2 * k + i] = unpack2(v, i, static_cast<const T*>(nullptr));
      }
    } else if constexpr (kB == 4) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        x[k] = unpack2(make_uint4(raw[k], 0, 0, 0), 0, static_cast<const T*>(nullptr));
    } else {
#pragma unroll
      for (int k = 0; k < C / 2; ++k) x[k] = make_float2(one(raw[2 * k]), one(raw[2 * k + 1]));
    }
  }
  __device__ __forceinline__ static float one(uint32_t w) {
    if constexpr (sizeof(T) == 2) {
      const uint16_t u = static_cast<uint16_t>(w);
      return to_f32(*reinterpret_cast<const T*>(&u));
    } else {
      return __uint_as_float(w);
    }
  }
  __device__ __forceinline__ void floats(float (&x)[C]) const {
    float2 y[C / 2];
    pairs(y);
#pragma unroll
    for (int i = 0; i < C / 2; ++i) {
      x[2 * i] = y[i].x;
      x[2 * i + 1] = y[i].y;
    }
  }
  __device__ __forceinline__ static void store_pairs(T* row, int d, int t, int G,
                                                     const float2 (&x)[C / 2]) {
    T* p = row + E * t;
    const int left = d - E * t, step = E * G;
#pragma unroll
    for (int k = 0; k < kPer; ++k, p += step) {
      const int n = left - k * step;
      if constexpr (kVec) {
        uint4 v;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) pack2(v, i, x[E / 2 * k + i], static_cast<const T*>(nullptr));
        if (n >= E) {
          *reinterpret_cast<uint4*>(p) = v;
        } else if (n > 0) {
#pragma unroll
          for (int i = 0; i < E; ++i) {
            const float2 y = x[E / 2 * k + i / 2];
            if (i < n) p[i] = from_f32<T>(i % 2 == 0 ? y.x : y.y);
          }
        }
      } else if constexpr (kB == 4) {
        uint4 v = make_uint4(0, 0, 0, 0);
        pack2(v, 0, x[k], static_cast<const T*>(nullptr));
        if (n >= 2) *reinterpret_cast<uint32_t*>(p) = v.x;
        else if (n == 1) *p = from_f32<T>(x[k].x);
      } else if (n > 0) {
        *p = from_f32<T>(k % 2 == 0 ? x[k / 2].x : x[k / 2].y);
      }
    }
  }
  __device__ __forceinline__ static void store(T* row, int d, int t, int G, const float (&x)[C]) {
    float2 y[C / 2];
#pragma unroll
    for (int i = 0; i < C / 2; ++i) y[i] = make_float2(x[2 * i], x[2 * i + 1]);
    store_pairs(row, d, t, G, y);
  }
};

// 32 bytes at once, from and to 32-byte boundaries.
__device__ __forceinline__ void load32(const void* p, uint32_t (&r)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
                 "=r"(r[6]), "=r"(r[7]) : "l"(p));
}
__device__ __forceinline__ void store32(void* p, const uint32_t (&r)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ float sqrt_approx(float x) {     // 2^-23 relative, of normal x
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {      // 1 unit, of normal x up to 2^126
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The larger of a and |b|; NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(fabsf(b)));
  return y;
}
// The larger of two; NaN if one is.
__device__ __forceinline__ float at_least(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// Four bytes, x0 the lowest, of integers held to [0, 255].
__device__ __forceinline__ uint32_t pack_bytes(int x0, int x1, int x2, int x3) {
  uint32_t hi, d;
  asm("cvt.pack.sat.u8.s32.b32 %0, %1, %2, %3;" : "=r"(hi) : "r"(x3), "r"(x2), "r"(0));
  asm("cvt.pack.sat.u8.s32.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(x1), "r"(x0), "r"(hi));
  return d;
}

// ---- clusters
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
  return r;
}
// cluster_sync() after code in which a warp's lanes may have parted, and its two halves for
// work between them (the barrier wants whole warps).
__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();
  cluster_sync();
}
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Stores to the shared memory of the cluster's CTA `rank`, at the address that `p` has here.
__device__ __forceinline__ void st_cluster(float* p, uint32_t rank, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(p), rank)), "f"(v)
               : "memory");
}

// Adds to a word of the shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ void add_cluster(unsigned* p, uint32_t rank, unsigned v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(
                   mapa_shared(smem_u32(p), rank)), "r"(v)
               : "memory");
}

// Kahan-compensated running sum.
struct CompensatedSum {
  float s = 0.0f, c = 0.0f;
  __device__ __forceinline__ void add(float x) {
    const float y = x - c;
    const float t = s + y;
    c = (t - s) - y;
    s = t;
  }
};

// A sum held as two fp32 numbers (some 48 bits): fp64 arithmetic, at two operations a
// clock and SM, would take longer than the loads.  An overflow or NaN shows in hi.
struct Sum2 {
  float hi = 0.0f, lo = 0.0f;
  __device__ __forceinline__ void add(float x) {
    const float t = hi + x, y = t - hi;
    lo += (hi - (t - y)) + (x - y);
    hi = t;
  }
  __device__ __forceinline__ void add(const Sum2& o) {
    add(o.hi);
    lo += o.lo;
  }
  __device__ __forceinline__ float value() const { return hi - hi == 0.0f ? hi + lo : hi; }
};
__device__ __forceinline__ Sum2 warp_sum(Sum2 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sum2 x;
    x.hi = __shfl_xor_sync(0xffffffffu, v.hi, o);
    x.lo = __shfl_xor_sync(0xffffffffu, v.lo, o);
    v.add(x);
  }
  return v;
}

// The sum over the CTA (whole warps, at most 32), in every thread; `red` holds a
// value per warp and may be reused after the call.
template <typename F>
__device__ __forceinline__ F block_sum(F v, F* red) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  F t = (threadIdx.x & 31) < (blockDim.x >> 5) ? red[threadIdx.x & 31] : F();
  t = warp_sum(t);
  __syncthreads();
  return t;
}

// ---- 8-bit states.  A code is the top bits of a positive float below its sign,
// less those of the smallest magnitude held: truncating the bits and adding chance
// below the cut rounds up with a probability equal to the part cut off.  Code 0 has the place of
// the magnitude below code 1's but stands for zero: an m of up to 2^-15 of the scale is dropped, a
// v > 0 takes code 1 at least.
constexpr int kCodeShift = 20;                 // three bits of mantissa stay
constexpr int kFirstBase = 112 << 3;           // m: exponents 2^-15 .. 2^0 in 7 bits
constexpr int kSecondBase = 96 << 3;           // v: exponents 2^-31 .. 2^0 in 8 bits
constexpr float kTopInverse = static_cast<float>(1.0 / 1.875);   // 1.875: the largest code

__device__ __forceinline__ float decode_first(uint32_t code) {
  const uint32_t mag = code & 127u;
  const uint32_t bits = ((mag + kFirstBase) << kCodeShift) | ((code & 128u) << 24);
  return mag != 0 ? __uint_as_float(bits) : __uint_as_float((code & 128u) << 24);
}
__device__ __forceinline__ float decode_second(uint32_t code) {
  return code != 0 ? __uint_as_float((code + kSecondBase) << kCodeShift) : 0.0f;
}
// The scale of a block whose largest magnitude is `top`, and its inverse (0 for a block of zeros).
__device__ __forceinline__ float block_scale(float top) {
  return top > 0.0f ? fmaxf(__fmul_rn(top, kTopInverse), 1.17549435e-38f) : top;
}
__device__ __forceinline__ float block_inverse(float scale) {
  return scale > 0.0f ? __frcp_rn(scale) : 0.0f;
}
// `chance`: 16 random bits.
__device__ __forceinline__ uint32_t encode_first(float m, float inv, uint32_t chance) {
  const float y = __fmul_rn(fabsf(m), inv);
  int code = ((__float_as_int(y) + static_cast<int>(chance << 4)) >> kCodeShift) - kFirstBase;
  code = min(max(code, 0), 127);
  return static_cast<uint32_t>(code) | (m < 0.0f ? 128u : 0u);
}
__device__ __forceinline__ uint32_t encode_second(float v, float inv, uint32_t chance) {
  const float y = __fmul_rn(v, inv);
  int code = ((__float_as_int(y) + static_cast<int>(chance << 4)) >> kCodeShift) - kSecondBase;
  code = min(max(code, 1), 255);
  return v > 0.0f ? static_cast<uint32_t>(code) : 0u;
}

// ---- four codes at once: byte k of `w` is element k.  The bases' bits are those
// that no code sets, so they are put in by an OR; a code of 0 is a matter of its own.
template <int K>
__device__ __forceinline__ uint32_t byte_to_code_bits(uint32_t w) {   // byte K at bit 20 on
  return K == 0 ? w << 20 : K == 1 ? w << 12 : K == 2 ? w << 4 : w >> 4;
}
// Nonzero where a byte of w is 0.
__device__ __forceinline__ uint32_t zero_bytes(uint32_t w) {
  return (w - 0x01010101u) & ~w & 0x80808080u;
}
template <int K>
__device__ __forceinline__ float first_bits(uint32_t w) {
  return __uint_as_float((byte_to_code_bits<K>(w) & 0x07f00000u) |
                         static_cast<uint32_t>(kFirstBase << kCodeShift) |
                         ((w << (24 - 8 * K)) & 0x80000000u));
}
template <int K>
__device__ __forceinline__ float second_bits(uint32_t w) {
  return __uint_as_float((byte_to_code_bits<K>(w) & 0x0ff00000u) |
                         static_cast<uint32_t>(kSecondBase << kCodeShift));
}
// The values of codes of which none is 0 (a 0 would read as the smallest magnitude) ...
__device__ __forceinline__ void decode_nonzero_first4(uint32_t w, float* x) {
  x[0] = first_bits<0>(w);
  x[1] = first_bits<1>(w);
  x[2] = first_bits<2>(w);
  x[3] = first_bits<3>(w);
}
__device__ __forceinline__ void decode_nonzero_second4(uint32_t w, float* x) {
  x[0] = second_bits<0>(w);
  x[1] = second_bits<1>(w);
  x[2] = second_bits<2>(w);
  x[3] = second_bits<3>(w);
}
// ... and zeros where the bytes of w say so.
__device__ __forceinline__ void put_zeros4(uint32_t w, float* x) {
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (((w >> (8 * k)) & 255u) == 0) x[k] = 0.0f;
}
__device__ __forceinline__ void decode_first4(uint32_t w, float* x) {
  decode_nonzero_first4(w, x);
  put_zeros4(w & 0x7f7f7f7fu, x);
}
__device__ __forceinline__ void decode_second4(uint32_t w, float* x) {
  decode_nonzero_second4(w, x);
  put_zeros4(w, x);
}
// Where the four elements' chances stand below the cut: bits 4 .. 19.
__device__ __forceinline__ void chances(uint64_t h, uint32_t (&c)[4]) {
  const uint32_t lo = static_cast<uint32_t>(h), hi = static_cast<uint32_t>(h >> 32);
  c[0] = (lo << 4) & 0xffff0u;
  c[1] = (lo >> 12) & 0xffff0u;
  c[2] = (hi << 4) & 0xffff0u;
  c[3] = (hi >> 12) & 0xffff0u;
}
// encode_first and encode_second (but for raise_zeros4) of four elements.  The first's
// magnitudes are packed with one bit more, so that holding them to a byte holds them to 7 bits.
__device__ __forceinline__ uint32_t encode_first4(const float* m, float inv, const uint32_t* c) {
  int x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    x[k] = (__float_as_int(__fmul_rn(fabsf(m[k]), inv)) + static_cast<int>(c[k]) -
            (kFirstBase << kCodeShift)) >> (kCodeShift - 1);
  const uint32_t mag = (pack_bytes(x[0], x[1], x[2], x[3]) >> 1) & 0x7f7f7f7fu;
  const uint32_t s01 = __byte_perm(__float_as_uint(m[0]), __float_as_uint(m[1]), 0x0073);
  const uint32_t s23 = __byte_perm(__float_as_uint(m[2]), __float_as_uint(m[3]), 0x0073);
  return mag | (__byte_perm(s01, s23, 0x5410) & 0x80808080u);
}
__device__ __forceinline__ uint32_t encode_second4(const float* v, float inv, const uint32_t* c) {
  int x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    x[k] = (__float_as_int(__fmul_rn(v[k], inv)) + static_cast<int>(c[k]) -
            (kSecondBase << kCodeShift)) >> kCodeShift;
  return pack_bytes(x[0], x[1], x[2], x[3]);
}
// Only a v of 0 takes code 0: others get the smallest.
__device__ __forceinline__ uint32_t raise_zeros4(uint32_t w, const float* v) {
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (((w >> (8 * k)) & 255u) == 0 && v[k] > 0.0f) w |= 1u << (8 * k);
  return w;
}

// The SplitMix64 finaliser (Steele, Lea and Flood 2014) and its sequence's increment.
constexpr uint64_t kSplitMixGamma = 0x9E3779B97F4A7C15ull;
__host__ __device__ __forceinline__ uint64_t mix64(uint64_t x) {
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return x ^ (x >> 31);
}

}  // namespace bergson
