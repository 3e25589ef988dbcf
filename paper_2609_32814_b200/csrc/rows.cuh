// What the row-wise kernels around the projections share: eight consecutive values of a row in either type, and the
// host's checks of their operands.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "algproj.h"

namespace algproj {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f32(float v, float *dst) { *dst = v; }
__device__ __forceinline__ void from_f32(float v, __nv_bfloat16 *dst) { *dst = __float2bfloat16_rn(v); }

// Eight consecutive values as they lie in memory: 16 bytes of bf16, 32 of fp32.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16 *p) { a = *(const uint4 *)p; }
  __device__ __forceinline__ void load4(int half, const __nv_bfloat16 *p) {   // four of them
    const uint2 v = *(const uint2 *)p;
    if (half) a.z = v.x, a.w = v.y;
    else a.x = v.x, a.y = v.y;
  }
  __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[2 * j] = __uint_as_float(w[j] << 16), f[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float *p) { a = ((const float4 *)p)[0], b = ((const float4 *)p)[1]; }
  __device__ __forceinline__ void load4(int half, const float *p) { (half ? b : a) = *(const float4 *)p; }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
    w[j] = *(const uint32_t *)&v;
  }
  *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float a, float b, float c, float d) {
  const __nv_bfloat162 u = __floats2bfloat162_rn(a, b), v = __floats2bfloat162_rn(c, d);
  *(uint2 *)p = make_uint2(*(const uint32_t *)&u, *(const uint32_t *)&v);
}
__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) { *(float4 *)p = make_float4(a, b, c, d); }
__device__ __forceinline__ void store8(float *p, const float (&f)[8]) {
  if (((uintptr_t)p & 31u) == 0) {   // whole sectors: 16 bytes and 16 more would write each twice
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]),
                 "f"(f[7])
                 : "memory");
  } else {
    ((float4 *)p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    ((float4 *)p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
}

// Eight values as four pairs, for the packed fp32 instructions: half as many issue slots as one value at a time.
struct F8 {
  uint64_t p[4];
};
// (moves between a pair and its halves, not shifts and ors: those cost instructions)
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void halves(uint64_t p, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ uint64_t pair_mul(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ F8 all8(float v) {
  const uint64_t p = pair(v, v);
  return {{p, p, p, p}};
}
__device__ __forceinline__ F8 operator*(const F8 &a, const F8 &b) {
  return {{pair_mul(a.p[0], b.p[0]), pair_mul(a.p[1], b.p[1]), pair_mul(a.p[2], b.p[2]), pair_mul(a.p[3], b.p[3])}};
}
__device__ __forceinline__ F8 operator+(const F8 &a, const F8 &b) {
  return {{pair_add(a.p[0], b.p[0]), pair_add(a.p[1], b.p[1]), pair_add(a.p[2], b.p[2]), pair_add(a.p[3], b.p[3])}};
}
__device__ __forceinline__ F8 operator*(const F8 &a, float b) { return a * all8(b); }
__device__ __forceinline__ F8 operator+(const F8 &a, float b) { return a + all8(b); }
__device__ __forceinline__ F8 fma8(const F8 &a, const F8 &b, const F8 &c) {
  return {{pair_fma(a.p[0], b.p[0], c.p[0]), pair_fma(a.p[1], b.p[1], c.p[1]), pair_fma(a.p[2], b.p[2], c.p[2]), pair_fma(a.p[3], b.p[3], c.p[3])}};
}
__device__ __forceinline__ F8 fma8(const F8 &a, float b, const F8 &c) { return fma8(a, all8(b), c); }
__device__ __forceinline__ F8 from8(const float (&f)[8]) { return {{pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7])}}; }
__device__ __forceinline__ void to8(const F8 &a, float (&f)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) halves(a.p[j], f[2 * j], f[2 * j + 1]);
}
__device__ __forceinline__ float sum8(const F8 &a) {
  float lo, hi;
  halves(pair_add(pair_add(a.p[0], a.p[1]), pair_add(a.p[2], a.p[3])), lo, hi);
  return lo + hi;
}
// The sum of eight products.
__device__ __forceinline__ float dot8(const F8 &a, const F8 &b) {
  float lo, hi;
  halves(pair_add(pair_fma(a.p[0], b.p[0], pair_mul(a.p[1], b.p[1])), pair_fma(a.p[2], b.p[2], pair_mul(a.p[3], b.p[3]))), lo, hi);
  return lo + hi;
}
// 1 / (1 + exp(-x)), by two approximations of the special function unit: off by 7 units of 2^-24, and below 0 by 2 |x| more from the rounding of x log2 e.
__device__ __forceinline__ float sigmoid(float x) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}
// The same, and what makes its slope a product, s (s e): s (1 - s) loses its bits as s nears 1 (0.9 % at x = 12, all from 17 on).
// (Below -88.4, where s is 0 already, e would become infinite.)
__device__ __forceinline__ float sigmoid(float x, float &e) {
  float r;
  asm("max.NaN.f32 %0, %1, 0fC2B0CCCD;" : "=f"(r) : "f"(x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(r * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}

constexpr long long kLandCycles = 2000000;   // about a millisecond, in which any copy lands
constexpr int kMaxStall = 1 << 16;             // of ALG_OPT_TEST_STALL_BYTES: what a barrier counts stays below 2^20
constexpr int64_t kMaxLd = 1 << 30;   // (the kernels count the bytes between rows in 32 bits)
inline size_t elem_size(alg_dtype_t t) { return t == ALG_BF16 ? 2 : 4; }
inline bool on_16(const void *p, int64_t ld, size_t elem) { return ((uintptr_t)p & 15u) == 0 && ((size_t)ld * elem) % 16 == 0; }
inline bool on_element(const void *p, size_t elem) { return (uintptr_t)p % elem == 0; }

// M rows of `width` bytes, `pitch` bytes apart.
struct RowSpan {
  uintptr_t at;
  size_t pitch, width;
  int64_t rows;
  uintptr_t end() const { return at + (size_t)(rows - 1) * pitch + width; }
};
inline RowSpan span(const void *p, int64_t ld, int64_t cols, size_t elem, int64_t M) {
  return {(uintptr_t)p, (size_t)ld * elem, (size_t)cols * elem, M};
}
// Whether two matrices may share a byte (column slices of one buffer do not).
inline bool meet(const RowSpan &a, const RowSpan &b) {
  if (!a.at || !b.at || a.rows <= 0 || b.rows <= 0 || a.end() <= b.at || b.end() <= a.at) return false;
  if (a.pitch != b.pitch) return true;
  const RowSpan &lo = a.at <= b.at ? a : b, &hi = a.at <= b.at ? b : a;
  const size_t d = (hi.at - lo.at) % a.pitch;
  return d < lo.width || d + hi.width > a.pitch;
}
inline bool same_rows(const RowSpan &a, const RowSpan &b) { return a.at == b.at && a.pitch == b.pitch && a.width == b.width; }

// The options of handles whose only ones are about their waits.
inline alg_status_t wait_option(long long *limit, uint32_t *stall, alg_option_t option, int64_t value) {
  if (option == ALG_OPT_WAIT_LIMIT_CYCLES && value >= 1000) *limit = value;
  else if (option == ALG_OPT_TEST_STALL_BYTES && value >= 0 && value <= kMaxStall && value % 16 == 0) *stall = (uint32_t)value;
  else return ALG_ERR_INVALID_ARG;
  return ALG_OK;
}

// The current device, which has to be the one a handle was made on, and of the kind the kernels are built for.
inline alg_status_t kernel_device(int *dev, int *num_sms) {
  int major = 0;
  if (cudaGetDevice(dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev) != cudaSuccess ||
      cudaDeviceGetAttribute(num_sms, cudaDevAttrMultiProcessorCount, *dev) != cudaSuccess)
    return ALG_ERR_CUDA;
  return major == 10 ? ALG_OK : ALG_ERR_UNSUPPORTED_SHAPE;
}
inline bool is_current(int device) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == device;
}

}  // namespace algproj
