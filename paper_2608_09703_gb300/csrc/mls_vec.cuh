// 16-byte vectors of bf16 or fp32 values and warp sums, shared by the row-norm
// kernels (mls_junction.cu, mls_norm.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace mls {

// 16 bytes of E <-> N fp32 values.
template <typename E>
struct Vec;
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = *reinterpret_cast<const __nv_bfloat162*>(&w[i]);
      const float2 v = __bfloat1622float2(h);
      f[2 * i] = v.x;
      f[2 * i + 1] = v.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x);
    f[1] = __uint_as_float(u.y);
    f[2] = __uint_as_float(u.z);
    f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
  }
};

__device__ __forceinline__ uint4 ld16(const void* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void st16(void* p, const uint4& v) { *reinterpret_cast<uint4*>(p) = v; }

// Tells the compiler the cached vectors may have changed, so it re-unpacks
// them after the reductions instead of keeping 8 floats per vector alive.
template <int R>
__device__ __forceinline__ void keep_packed(uint4 (&v)[R]) {
#pragma unroll
  for (int j = 0; j < R; ++j) asm volatile("" : "+r"(v[j].x), "+r"(v[j].y), "+r"(v[j].z), "+r"(v[j].w));
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}


// Two fp32 values in a 64-bit register pair: one instruction works on both.
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ F2 f2(float v) { return f2(v, v); }
__device__ __forceinline__ void f2_split(F2 v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ float f2_sum(F2 v) {
  float lo, hi;
  f2_split(v, lo, hi);
  return lo + hi;
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// The same vectors as pairs: 4 of bf16, 2 of fp32.
template <typename E>
struct Vec2;
template <>
struct Vec2<__nv_bfloat16> {
  static constexpr int N = 4;
  static constexpr uint32_t kOne = 0x3f803f80u;  // two ones
  static __device__ __forceinline__ void unpack(const uint4& u, F2 (&f)[4]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 pack(const F2 (&f)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      f2_split(f[i], lo, hi);
      const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Vec2<float> {
  static constexpr int N = 2;
  static constexpr uint32_t kOne = 0x3f800000u;
  static __device__ __forceinline__ void unpack(const uint4& u, F2 (&f)[2]) {
    f[0] = f2(__uint_as_float(u.x), __uint_as_float(u.y));
    f[1] = f2(__uint_as_float(u.z), __uint_as_float(u.w));
  }
  static __device__ __forceinline__ uint4 pack(const F2 (&f)[2]) {
    float a, b, c, d;
    f2_split(f[0], a, b);
    f2_split(f[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
};

// A sum in two fp32 words: what rounding the first loses goes to the second (Knuth's
// two-sum), so a long sum keeps some 45 bits.  An SM adds two 64-bit values a clock
// and 128 fp32 ones.  Once the first word is infinite or NaN the second means nothing.
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ void pair_add(Pair& a, float hi, float lo) {
  const float s = a.hi + hi, b = s - a.hi;
  a.lo += ((a.hi - (s - b)) + (hi - b)) + lo;
  a.hi = s;
}
__device__ __forceinline__ Pair warp_sum_pair(Pair a) {  // valid in lane 0
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    pair_add(a, __shfl_down_sync(0xffffffffu, a.hi, o), __shfl_down_sync(0xffffffffu, a.lo, o));
  return a;
}
__device__ __forceinline__ Pair pair_scaled(const Pair& a, float c) {
  const float hi = a.hi * c;
  return {hi, isfinite(hi) ? fmaf(a.hi, c, -hi) + a.lo * c : 0.f};
}
__device__ __forceinline__ float pair_float(const Pair& a) { return isfinite(a.hi) ? a.hi + a.lo : a.hi; }
__device__ __forceinline__ double pair_value(const Pair& a) {
  return isfinite(a.hi) ? static_cast<double>(a.hi) + static_cast<double>(a.lo) : static_cast<double>(a.hi);
}

}  // namespace mls
