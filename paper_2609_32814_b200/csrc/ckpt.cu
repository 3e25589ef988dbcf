// Activations kept in 8 bits between the two passes of a training step, and the activation that goes with them.
//
// A block of 32 columns of a row shares a power of two 2^e, the smallest with max|x| <= top * 2^e (top = 448 for e4m3, 127
// for int8); the code of x is x * 2^-e rounded to the format.  With max|x| = f 2^p, 1 <= f < 2, and top = t 2^P, that is
// e = p - P + (f > t): a carry out of the mantissa, found by one addition on the bits.  Products with 2^-e and 2^e are exact,
// so a code depends on nothing but the values.
//
// One pass over memory either way, eight columns (16 bytes of bf16) a thread: four neighbouring threads are a block and
// find its maximum by two shuffles.  Bound by HBM.
#include <cuda_fp8.h>

#include <new>

#include "common.cuh"
#include "rows.cuh"

using namespace algproj;

struct alg_ckpt_s {
  int cols = 0, parts = 1, padded = 0;   // columns of a part, parts, columns of a part as the records hold them
  alg_q8_t format = ALG_Q8_E4M3;
  alg_act_t act = ALG_ACT_NONE;
  int device = 0, num_sms = 148;
  int64_t row_bytes = 0;
};

namespace algproj {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 32;       // columns that share a scale
constexpr int kMinExp = -120;    // of a scale: it and its inverse stay normal numbers

enum { kStore, kLoad, kForward, kBackward };

struct CkptArgs {
  const void *in;        // X, Z or dA
  void *out, *again;     // X, A or dZ; the activation of the backward pass
  uint8_t *ckpt;
  int64_t ld_in, ld_out, ld_again, row_bytes;
  int64_t M;
  int cols, padded, parts;
  int units;             // padded / 8: threads' pieces of a row
  uint32_t inv_units;    // ceil(2^32 / units)
  int tile_rows;         // rows a CTA takes at a time
  int int8;
};

// The largest magnitude of eight values, as bits: one that is not finite is above all others.
__device__ __forceinline__ uint32_t largest8(const Raw8<__nv_bfloat16> &r) {
  const uint32_t m = 0x7FFF7FFFu;
  const uint32_t v = __vmaxu2(__vmaxu2(r.a.x & m, r.a.y & m), __vmaxu2(r.a.z & m, r.a.w & m));
  return max(v << 16, v & 0x7FFF0000u);
}
__device__ __forceinline__ uint32_t largest8(const Raw8<float> &r) {
  auto most = [](float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(fabsf(a)), "f"(fabsf(b)));
    return d;
  };
  return __float_as_uint(most(most(most(r.a.x, r.a.y), most(r.a.z, r.a.w)), most(most(r.b.x, r.b.y), most(r.b.z, r.b.w))));
}
// Codes of eight values whose block's largest magnitude has the bits `top`; the scale byte.  Integers without a conversion: x * 2^-e plus
// 1.5 * 2^23 is rounded to a whole number, whose low byte is the code; back the same way from 2^23 + 128 + code, exactly.
__device__ __forceinline__ uint2 encode8(const F8 &x, uint32_t top, int int8, int *scale) {
  if (top >= 0x7F800000u) {   // an infinity or a NaN
    *scale = 255;
    return make_uint2(0u, 0u);
  }
  // mantissas above that of 448 = 1.75 * 2^8 (127 = 1.984375 * 2^6) carry into the exponent
  const int e = max(kMinExp, (int)((top + (int8 ? 0x7FFFFFu - 0x7E0000u : 0x7FFFFFu - 0x600000u)) >> 23) - 127 - (int8 ? 6 : 8));
  *scale = e + 127;
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
  float f[8];
  if (int8) {
    to8(fma8(x, inv, all8(12582912.f)), f);
    auto pack = [](float a, float b, float c, float d) {
      return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
    };
    return make_uint2(pack(f[0], f[1], f[2], f[3]), pack(f[4], f[5], f[6], f[7]));
  }
  to8(x * inv, f);
  auto pack = [](float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    return lo | (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3) << 16;
  };
  return make_uint2(pack(f[0], f[1], f[2], f[3]), pack(f[4], f[5], f[6], f[7]));
}
__device__ __forceinline__ F8 decode8(uint2 c, int s, int int8) {
  const float scale = s == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)s << 23);
  float f[8];
  if (int8) {
    const uint32_t lo = c.x ^ 0x80808080u, hi = c.y ^ 0x80808080u;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(__byte_perm(j < 4 ? lo : hi, 0x4B000000u, 0x7440 | (j & 3)));
    return (from8(f) + -8388736.f) * scale;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((j < 2 ? c.x : c.y) >> (16 * (j & 1)) & 0xFFFFu), __NV_E4M3);
    const float2 v = __half22float2(*(const __half2 *)&h);
    f[2 * j] = v.x, f[2 * j + 1] = v.y;
  }
  return from8(f) * scale;
}

__device__ __forceinline__ F8 each(const F8 &x, float (*g)(float)) {
  float f[8];
  to8(x, f);
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = g(f[j]);
  return from8(f);
}
__device__ __forceinline__ float exp2_(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ F8 minus(const F8 &a) { return a * -1.f; }

// act(z), and its derivative where `slope` is not null.
template <typename T, int ACT>
__device__ __forceinline__ F8 act8(const F8 &z, F8 *slope) {
  const float log2e = 1.4426950408889634f;
  if (ACT == ALG_ACT_SILU) {
    const F8 p = each(each(z * -log2e, exp2_) + 1.f, reciprocal), a = z * p;
    if (slope) *slope = fma8(a, minus(p) + 1.f, p);
    return a;
  }
  if (ACT == ALG_ACT_GELU_TANH) {   // (1 + tanh u) / 2 = 1 / (1 + exp(-2u)), 2u = 2k z (1 + c z^2)
    const float k2 = 2.f * 0.7978845608028654f, c = 0.044715f;
    const F8 zz = z * z, p = each(each(z * fma8(zz, -log2e * k2 * c, all8(-log2e * k2)), exp2_) + 1.f, reciprocal), a = z * p;
    if (slope) *slope = fma8(a * (minus(p) + 1.f), fma8(zz, 3.f * k2 * c, all8(k2)), p);
    return a;
  }
  if (ACT == ALG_ACT_GELU_ERF) {
    float f[8], t[8], d[8];
    to8(z, f);
    if (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j) t[j] = fmaf(0.5f, erff(f[j] * 0.70710678118654752f), 0.5f);
      const F8 p = from8(t);
      if (slope) *slope = fma8(z * 0.39894228040143268f, each(z * z * (-0.5f * log2e), exp2_), p);
      return z * p;
    }
    // bf16 results: the lower tail 2^p(|z|) of the projection kernels' epilogues, off by 2.4e-6 at most
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = fminf(fabsf(f[j]), 6.f), d[j] = fabsf(f[j]), f[j] = fmaxf(f[j], 0.f);
    const F8 u = from8(t);
    F8 q = fma8(u, all8(3.3093889e-05f), all8(-7.6922908e-04f));
    q = fma8(q, u, all8(8.0807470e-03f));
    q = fma8(q, u, all8(-5.3412151e-02f));
    q = fma8(q, u, all8(-4.5877093e-01f));
    q = fma8(q, u, all8(-1.1512017f));
    q = fma8(q, u, all8(-0.99999309f));
    const F8 tail = each(q, exp2_), a = fma8(minus(from8(d)), tail, from8(f));
    if (slope) {
      float h[8], zf[8];
      to8(minus(tail) + 0.5f, h);
      to8(z, zf);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[j] = copysignf(h[j], zf[j]);
      *slope = fma8(z * 0.39894228040143268f, each(z * z * (-0.5f * log2e), exp2_), from8(h) + 0.5f);
    }
    return a;
  }
  if (slope) *slope = all8(1.f);
  return z;
}

// Eight columns of a row from column c on, zero past `cols`.
template <typename T, bool VEC>
__device__ __forceinline__ void fetch8(Raw8<T> &r, const T *row, int c, int cols) {
  if (VEC) {
    if (c < cols) r.load(row + c);   // (cols is a multiple of 8)
    else r.zero();
  } else {
    r.zero();
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < cols) r.set(j, row[c + j]);
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void put8(T *row, int c, int cols, const F8 &a) {
  float f[8];
  to8(a, f);
  if (VEC) {
    if (c < cols) store8(row + c, f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < cols) from_f32(f[j], row + c + j);
  }
}

// Whole warps call this: the maximum of a block is found among its four threads.
template <typename T>
__device__ __forceinline__ void keep8(const Raw8<T> &r, const F8 &x, uint8_t *codes, uint8_t *scale, bool on, int int8) {
  uint32_t top = largest8(r);
  top = max(top, __shfl_xor_sync(~0u, top, 1));
  top = max(top, __shfl_xor_sync(~0u, top, 2));
  int s;
  const uint2 w = encode8(x, top, int8, &s);
  if (!on) return;
  *(uint2 *)codes = w;
  if ((threadIdx.x & 3) == 0) *scale = (uint8_t)s;
}

template <typename T, int OP, int ACT, bool GATED, bool VEC>
__global__ void __launch_bounds__(kThreads) ckpt_kernel(const CkptArgs a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int codes = a.parts * a.padded;
  for (int64_t row0 = (int64_t)blockIdx.x * a.tile_rows; row0 < a.M; row0 += (int64_t)gridDim.x * a.tile_rows) {
    const int n = (int)min((int64_t)a.tile_rows, a.M - row0) * a.units;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
      const int i = i0 + threadIdx.x;
      const bool on = i < n;                                   // (n is a multiple of 4: a block is whole)
      const int r = on && a.units > 1 ? (int)__umulhi((uint32_t)i, a.inv_units) : 0;
      const int64_t b = row0 + r;
      const int u = on ? i - r * a.units : 0, c = u * 8;
      uint8_t *rec = a.ckpt + b * a.row_bytes;
      const int limit = on ? a.cols : 0;
      auto eight = [](const Raw8<T> &r) {
        float f[8];
        r.get(f);
        return from8(f);
      };
      if (OP == kStore || OP == kForward) {
        const T *row = (const T *)a.in + b * a.ld_in;
        Raw8<T> raw, raw2;
        fetch8<T, VEC>(raw, row, c, limit);
        if (GATED) fetch8<T, VEC>(raw2, row + a.cols, c, limit);
        const F8 z = eight(raw);
        F8 up;
        if (GATED) up = eight(raw2);
        if (OP == kForward) {
          F8 f = act8<T, ACT>(z, nullptr);
          if (GATED) f = f * up;
          put8<T, VEC>((T *)a.out + b * a.ld_out, c, limit, f);
        }
        if (OP == kStore || a.ckpt) {
          keep8(raw, z, rec + c, rec + codes + (u >> 2), on, a.int8);
          if (GATED) keep8(raw2, up, rec + a.padded + c, rec + codes + (a.padded >> 5) + (u >> 2), on, a.int8);
        }
      } else if (on) {
        const uint2 w = *(const uint2 *)(rec + c);
        const int s = rec[codes + (u >> 2)];
        uint2 w2;
        int s2;
        if (GATED) w2 = *(const uint2 *)(rec + a.padded + c), s2 = rec[codes + (a.padded >> 5) + (u >> 2)];
        if (OP == kLoad) {
          put8<T, VEC>((T *)a.out + b * a.ld_out, c, limit, decode8(w, s, a.int8));
        } else {
          Raw8<T> raw;
          fetch8<T, VEC>(raw, (const T *)a.in + b * a.ld_in, c, limit);
          const F8 z = decode8(w, s, a.int8), d = eight(raw);
          F8 slope, f = act8<T, ACT>(z, &slope);
          T *out = (T *)a.out + b * a.ld_out;
          if (GATED) {
            const F8 up = decode8(w2, s2, a.int8);
            put8<T, VEC>(out + a.cols, c, limit, f * d);
            slope = slope * up, f = f * up;
          }
          put8<T, VEC>(out, c, limit, slope * d);
          if (a.again) put8<T, VEC>((T *)a.again + b * a.ld_again, c, limit, f);
        }
      }
    }
  }
}

template <typename T, int OP, int ACT, bool GATED>
cudaError_t launch_ckpt(const alg_ckpt_s &h, CkptArgs a, bool vec, cudaStream_t st) {
  a.row_bytes = h.row_bytes;
  a.cols = h.cols, a.padded = h.padded, a.parts = h.parts;
  a.units = h.padded / 8;
  a.inv_units = (uint32_t)((0x100000000ull + a.units - 1) / a.units);
  a.int8 = h.format == ALG_Q8_INT8;
  // tiles of about four pieces a thread
  a.tile_rows = a.units >= 4 * kThreads ? 1 : 4 * kThreads / a.units;
  const int64_t tiles = (a.M + a.tile_rows - 1) / a.tile_rows;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles < (int64_t)h.num_sms * 64 ? tiles : (int64_t)h.num_sms * 64));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  const cudaError_t e = vec ? cudaLaunchKernelEx(&cfg, ckpt_kernel<T, OP, ACT, GATED, true>, a)
                            : cudaLaunchKernelEx(&cfg, ckpt_kernel<T, OP, ACT, GATED, false>, a);
  if (e == cudaSuccess) count_launch(1);
  return e;
}
template <typename T, int OP>
cudaError_t launch_act(const alg_ckpt_s &h, const CkptArgs &a, bool vec, cudaStream_t st) {
  const bool g = h.parts == 2;
  switch (h.act) {
    case ALG_ACT_NONE: return g ? launch_ckpt<T, OP, ALG_ACT_NONE, true>(h, a, vec, st) : launch_ckpt<T, OP, ALG_ACT_NONE, false>(h, a, vec, st);
    case ALG_ACT_GELU_ERF: return g ? launch_ckpt<T, OP, ALG_ACT_GELU_ERF, true>(h, a, vec, st) : launch_ckpt<T, OP, ALG_ACT_GELU_ERF, false>(h, a, vec, st);
    case ALG_ACT_GELU_TANH: return g ? launch_ckpt<T, OP, ALG_ACT_GELU_TANH, true>(h, a, vec, st) : launch_ckpt<T, OP, ALG_ACT_GELU_TANH, false>(h, a, vec, st);
    default: return g ? launch_ckpt<T, OP, ALG_ACT_SILU, true>(h, a, vec, st) : launch_ckpt<T, OP, ALG_ACT_SILU, false>(h, a, vec, st);
  }
}

// Rows on 16 bytes, and both halves of a gated one.
bool vectors(const alg_ckpt_s &h, const void *p, int64_t ld, size_t elem) { return !p || (h.cols % 8 == 0 && on_16(p, ld, elem)); }
bool dtype_ok(alg_dtype_t t) { return t == ALG_F32 || t == ALG_BF16; }
RowSpan records(const alg_ckpt_s &h, const void *ckpt, int64_t M) { return span(ckpt, h.row_bytes, h.row_bytes, 1, M); }

}  // namespace
}  // namespace algproj

extern "C" {

alg_status_t alg_ckpt_create(alg_ckpt_t *out, int cols, alg_q8_t format, alg_act_t act, int gated) {
  if (!out) return ALG_ERR_INVALID_ARG;
  *out = nullptr;
  if (cols < 1 || cols > ALG_CKPT_MAX_COLS || (format != ALG_Q8_E4M3 && format != ALG_Q8_INT8) || (int)act < 0 || (int)act > ALG_ACT_SILU)
    return ALG_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  const alg_status_t s = kernel_device(&dev, &sms);
  if (s != ALG_OK) return s;
  alg_ckpt_s *h = new (std::nothrow) alg_ckpt_s();
  if (!h) return ALG_ERR_INVALID_ARG;
  h->cols = cols, h->parts = gated ? 2 : 1;
  h->padded = (cols + kBlock - 1) / kBlock * kBlock;
  h->format = format, h->act = act;
  h->device = dev, h->num_sms = sms;
  h->row_bytes = ((int64_t)h->parts * (h->padded + h->padded / kBlock) + 31) / 32 * 32;
  *out = h;
  return ALG_OK;
}

alg_status_t alg_ckpt_destroy(alg_ckpt_t h) {
  if (!h) return ALG_ERR_INVALID_ARG;
  delete h;
  return ALG_OK;
}

alg_status_t alg_ckpt_row_bytes(alg_ckpt_t h, size_t *bytes) {
  if (!h || !bytes) return ALG_ERR_INVALID_ARG;
  *bytes = (size_t)h->row_bytes;
  return ALG_OK;
}

static alg_status_t ckpt_common(alg_ckpt_t h, int64_t M, alg_dtype_t dtype) {
  return !h || M < 0 || M > (1 << 30) || !dtype_ok(dtype) ? ALG_ERR_INVALID_ARG : ALG_OK;
}
static alg_status_t ckpt_done(cudaError_t e) { return e == cudaSuccess ? ALG_OK : ALG_ERR_CUDA; }

alg_status_t alg_ckpt_store(alg_ckpt_t h, const void *X, int64_t ldx, alg_dtype_t x_dtype, int64_t M, void *ckpt, void *stream) {
  alg_status_t s = ckpt_common(h, M, x_dtype);
  if (s != ALG_OK || M == 0) return s;
  const size_t e = elem_size(x_dtype);
  if (h->parts != 1 || !X || !ckpt || ldx < h->cols || !on_element(X, e) || ((uintptr_t)ckpt & 15u)) return ALG_ERR_INVALID_ARG;
  if (meet(span(X, ldx, h->cols, e, M), records(*h, ckpt, M)) || !is_current(h->device)) return ALG_ERR_INVALID_ARG;
  CkptArgs a = {};
  a.in = X, a.ld_in = ldx, a.ckpt = (uint8_t *)ckpt, a.M = M;
  const bool vec = vectors(*h, X, ldx, e);
  cudaStream_t st = (cudaStream_t)stream;
  return ckpt_done(x_dtype == ALG_BF16 ? launch_ckpt<__nv_bfloat16, kStore, ALG_ACT_NONE, false>(*h, a, vec, st)
                                       : launch_ckpt<float, kStore, ALG_ACT_NONE, false>(*h, a, vec, st));
}

alg_status_t alg_ckpt_load(alg_ckpt_t h, const void *ckpt, int64_t M, void *X, int64_t ldx, alg_dtype_t x_dtype, void *stream) {
  alg_status_t s = ckpt_common(h, M, x_dtype);
  if (s != ALG_OK || M == 0) return s;
  const size_t e = elem_size(x_dtype);
  if (h->parts != 1 || !X || !ckpt || ldx < h->cols || !on_element(X, e) || ((uintptr_t)ckpt & 15u)) return ALG_ERR_INVALID_ARG;
  if (meet(span(X, ldx, h->cols, e, M), records(*h, ckpt, M)) || !is_current(h->device)) return ALG_ERR_INVALID_ARG;
  CkptArgs a = {};
  a.out = X, a.ld_out = ldx, a.ckpt = (uint8_t *)ckpt, a.M = M;
  const bool vec = vectors(*h, X, ldx, e);
  cudaStream_t st = (cudaStream_t)stream;
  return ckpt_done(x_dtype == ALG_BF16 ? launch_ckpt<__nv_bfloat16, kLoad, ALG_ACT_NONE, false>(*h, a, vec, st)
                                       : launch_ckpt<float, kLoad, ALG_ACT_NONE, false>(*h, a, vec, st));
}

alg_status_t alg_ckpt_act_forward(alg_ckpt_t h, const void *Z, int64_t ldz, int64_t M, void *A, int64_t lda, alg_dtype_t dtype, void *ckpt,
                                  void *stream) {
  alg_status_t s = ckpt_common(h, M, dtype);
  if (s != ALG_OK || M == 0) return s;
  const size_t e = elem_size(dtype);
  const int64_t wide = (int64_t)h->parts * h->cols;
  if (!Z || !A || ldz < wide || lda < h->cols || !on_element(Z, e) || !on_element(A, e) || ((uintptr_t)ckpt & 15u)) return ALG_ERR_INVALID_ARG;
  const RowSpan z = span(Z, ldz, wide, e, M), out = span(A, lda, h->cols, e, M), rec = records(*h, ckpt, M);
  if ((meet(out, z) && !same_rows(out, z)) || meet(rec, z) || meet(rec, out) || !is_current(h->device)) return ALG_ERR_INVALID_ARG;
  CkptArgs a = {};
  a.in = Z, a.ld_in = ldz, a.out = A, a.ld_out = lda, a.ckpt = (uint8_t *)ckpt, a.M = M;
  const bool vec = vectors(*h, Z, ldz, e) && vectors(*h, A, lda, e);
  cudaStream_t st = (cudaStream_t)stream;
  return ckpt_done(dtype == ALG_BF16 ? launch_act<__nv_bfloat16, kForward>(*h, a, vec, st) : launch_act<float, kForward>(*h, a, vec, st));
}

alg_status_t alg_ckpt_act_backward(alg_ckpt_t h, const void *ckpt, const void *dA, int64_t ldda, int64_t M, void *dZ, int64_t lddz, void *A,
                                   int64_t lda, alg_dtype_t dtype, void *stream) {
  alg_status_t s = ckpt_common(h, M, dtype);
  if (s != ALG_OK || M == 0) return s;
  const size_t e = elem_size(dtype);
  const int64_t wide = (int64_t)h->parts * h->cols;
  if (!ckpt || !dA || !dZ || ldda < h->cols || lddz < wide || (A && lda < h->cols) || !on_element(dA, e) || !on_element(dZ, e) || !on_element(A, e) ||
      ((uintptr_t)ckpt & 15u))
    return ALG_ERR_INVALID_ARG;
  const RowSpan g = span(dA, ldda, h->cols, e, M), out = span(dZ, lddz, wide, e, M), again = span(A, lda, h->cols, e, M), rec = records(*h, ckpt, M);
  if ((meet(out, g) && !same_rows(out, g)) || meet(again, g) || meet(again, out) || meet(rec, g) || meet(rec, out) || meet(rec, again) ||
      !is_current(h->device))
    return ALG_ERR_INVALID_ARG;
  CkptArgs a = {};
  a.in = dA, a.ld_in = ldda, a.out = dZ, a.ld_out = lddz, a.again = A, a.ld_again = lda, a.ckpt = (uint8_t *)ckpt, a.M = M;
  const bool vec = vectors(*h, dA, ldda, e) && vectors(*h, dZ, lddz, e) && vectors(*h, A, lda, e);
  cudaStream_t st = (cudaStream_t)stream;
  return ckpt_done(dtype == ALG_BF16 ? launch_act<__nv_bfloat16, kBackward>(*h, a, vec, st) : launch_act<float, kBackward>(*h, a, vec, st));
}

}  // extern "C"
