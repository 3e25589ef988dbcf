// Activations kept in 8 bits between the two passes of a training step, and the activation that goes with them.
//
// A block of 32 columns of a row shares a power of two 2^e, the smallest with max|x| <= top * 2^e (top = 448 for e4m3, 127
// for int8); the code of x is x * 2^-e rounded to the format.  With max|x| = f 2^p, 1 <= f < 2, and top = t 2^P, that is
// e = p - P + (f > t): a carry out of the mantissa, found by one addition on the bits.  Products with 2^-e and 2^e are exact,
// so a code depends on nothing but the values.
//
// One pass over memory either way, eight columns (16 bytes of bf16) a thread: four neighbouring threads are a block and
// find its maximum by two shuffles.  Bound by HBM: 16384 x 7168 fp32 stored and loaded 180 us (6.57 TB/s), SwiGLU 16384 x 6144 both
// passes 283 us (6.45), GELU 8003 x 4096 69 us (5.76; with erff and one value an instruction 113, bound by the arithmetic), in fp32 114 (6.3).
#include <cuda_fp8.h>

#include <new>

#include "common.cuh"
#include "rows.cuh"

using namespace algproj;

struct alg_ckpt_s {
  int cols = 0, parts = 1, padded = 0;   // columns of a part, parts, columns of a part as the records hold them
  alg_q8_t format = ALG_Q8_E4M3;
  alg_act_t act = ALG_ACT_NONE;
  int device = 0;
  int64_t row_bytes = 0;
};

namespace algproj {
namespace {

constexpr int kThreads = 128;
constexpr int kBlock = 32;       // columns that share a scale
constexpr int kMinExp = -120;    // of a scale: it and its inverse stay normal numbers

enum { kStore, kLoad, kForward, kBackward };

struct CkptArgs {
  const uint8_t *in;     // X, Z or dA
  uint8_t *out, *again;  // X, A or dZ; the activation of the backward pass
  uint8_t *ckpt;
  uint32_t pitch_in, pitch_out, pitch_again, row_bytes;   // bytes between rows
  int64_t M;
  int cols, padded, codes, scales;   // codes of a row; scales of a part
  int units;             // padded / 8: threads' pieces of a row
  uint32_t inv_units;    // ceil(2^32 / units)
  int tile_rows;         // rows of a CTA
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

__device__ __forceinline__ uint64_t both(float v) { return pair(v, v); }
__device__ __forceinline__ uint64_t exp2_of(uint64_t x) {
  float lo, hi;
  halves(x, lo, hi);
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(lo));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(hi));
  return pair(lo, hi);
}
__device__ __forceinline__ uint64_t one_over(uint64_t x) {
  float lo, hi;
  halves(x, lo, hi);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(lo));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(hi));
  return pair(lo, hi);
}

// Phi(n), the normal distribution's lower tail, for n <= 0, and e = exp(-n^2 / 2).  However small it is, the tail keeps its bits.
// bf16 results: 2^q(n), q of degree eight fitted to log2 Phi(n) on [-13.3, 0] (beyond, the tail is 0 in fp32): 8.1e-4 of the value at most, a fifth of half a
// step, and 5.6e-7 at most.
// fp32: Phi(n) / e falls smoothly from 1/2 towards 0.4 / |n|: it is t P(t) with t = 1 / (1 - 0.275 n) and P of degree eight, fitted to 3.9e-8 of its value, 8
// units of 2^-24 with its own roundings; what grows is the rounding of n^2, n^2 units.  (For bf16 that took 74 us of both passes over 8003 x 4096, where 2^q takes 71.)
template <typename T>
__device__ __forceinline__ uint64_t normal_tail(uint64_t n, uint64_t e) {
  uint64_t p;
  if (sizeof(T) == 2) {
    p = pair_fma(n, both(4.11549252e-08f), both(2.46185356e-06f));
    p = pair_fma(p, n, both(6.28251626e-05f));
    p = pair_fma(p, n, both(9.06560959e-04f));
    p = pair_fma(p, n, both(8.35534306e-03f));
    p = pair_fma(p, n, both(5.36305293e-02f));
    p = pair_fma(p, n, both(-4.58744711e-01f));
    p = pair_fma(p, n, both(1.1511728f));
    return exp2_of(pair_fma(p, n, both(-0.999998488f)));
  }
  const uint64_t t = one_over(pair_fma(n, both(-0.275f), both(1.f)));
  p = pair_fma(t, both(0.0262493369f), both(-0.106020485f));
  p = pair_fma(p, t, both(0.120182197f));
  p = pair_fma(p, t, both(-0.0233438075f));
  p = pair_fma(p, t, both(0.0796022513f));
  p = pair_fma(p, t, both(0.0826022953f));
  p = pair_fma(p, t, both(0.10123601f));
  p = pair_fma(p, t, both(0.109789479f));
  p = pair_fma(p, t, both(0.109702743f));
  return pair_mul(pair_mul(p, t), e);
}

// act(z) of two values, and its derivative.  (Two at a time and packed at once: eight would hold 56 registers where 40 do, and threads
// are what keeps the memory busy.)
template <typename T, int ACT>
__device__ __forceinline__ uint64_t act2(uint64_t z, uint64_t *slope) {
  const float log2e = 1.4426950408889634f;
  if (ACT == ALG_ACT_SILU) {
    const uint64_t p = one_over(pair_add(exp2_of(pair_mul(z, both(-log2e))), both(1.f))), a = pair_mul(z, p);
    *slope = pair_fma(a, pair_fma(p, both(-1.f), both(1.f)), p);
    return a;
  }
  if (ACT == ALG_ACT_GELU_TANH) {   // (1 + tanh u) / 2 = 1 / (1 + exp(-2u)), 2u = 2k z (1 + c z^2)
    const float k2 = 2.f * 0.7978845608028654f, c = 0.044715f;
    // (squares that would be infinite: 0 * infinity in the slope; far behind where 1 - p is 0)
    float s0, s1;
    halves(pair_mul(z, z), s0, s1);
    const uint64_t zz = pair(fminf(s0, 1e30f), fminf(s1, 1e30f)), u = pair_mul(z, pair_fma(zz, both(-log2e * k2 * c), both(-log2e * k2)));
    const uint64_t p = one_over(pair_add(exp2_of(u), both(1.f))), a = pair_mul(z, p);
    *slope = pair_fma(pair_mul(a, pair_fma(p, both(-1.f), both(1.f))), pair_fma(zz, both(3.f * k2 * c), both(k2)), p);
    return a;
  }
  if (ACT == ALG_ACT_GELU_ERF) {
    float lo, hi;
    halves(z, lo, hi);
    const uint64_t n = pair(fmaxf(-fabsf(lo), -13.3f), fmaxf(-fabsf(hi), -13.3f));   // (whose tail is 0, as that of an infinity should be)
    const uint64_t e = exp2_of(pair_mul(pair_mul(n, n), both(-0.5f * log2e))), tail = normal_tail<T>(n, e);
    // Phi(z) is the tail or 1 - tail, never a difference of two halves: that would leave nothing of it from -5.5 on
    float t0, t1, h0, h1;
    halves(tail, t0, t1);
    halves(pair_fma(tail, both(-1.f), both(1.f)), h0, h1);
    *slope = pair_fma(pair_mul(z, both(0.39894228040143268f)), e, pair(lo < 0.f ? t0 : h0, hi < 0.f ? t1 : h1));
    auto above = [](float v) {   // max(v, 0), NaN for NaN
      float r;
      asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(v));
      return r;
    };
    return pair_fma(n, tail, pair(above(lo), above(hi)));   // z - |z| tail above 0, -|z| tail below
  }
  *slope = both(1.f);
  return z;
}

// Eight results on their way out.
template <typename T>
struct Out8;
template <>
struct Out8<__nv_bfloat16> {
  uint32_t w[4];
  __device__ __forceinline__ void set(int j, uint64_t p) {
    float lo, hi;
    halves(p, lo, hi);
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    w[j] = *(const uint32_t *)&v;
  }
  __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]); }
  __device__ __forceinline__ void stage(__nv_bfloat16 *p) const { store(p); }   // into shared memory
};
template <>
struct Out8<float> {
  float f[8];
  __device__ __forceinline__ void set(int j, uint64_t p) { halves(p, f[2 * j], f[2 * j + 1]); }
  __device__ __forceinline__ void store(float *p) const { store8(p, f); }
  __device__ __forceinline__ void stage(float *p) const {
    ((float4 *)p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    ((float4 *)p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// Eight columns of a row from column c on, zero past `cols` (a multiple of 8), of rows on 16 bytes.
template <typename T>
__device__ __forceinline__ void fetch8(Raw8<T> &r, const T *row, int c, int cols) {
  if (c < cols) r.load(row + c);
  else r.zero();
}
template <typename T>
__device__ __forceinline__ void put8(T *row, int c, int cols, const Out8<T> &o) {
  if (c < cols) o.store(row + c);
}
// The same of any rows, by whole warps: value by value, neighbouring threads on neighbouring columns, and turned round in the warp's part of
// shared memory (eight values a thread straight from memory would be eight requests for the same sectors: 9000 x 4001 GELU 293 us).
// r, c: the thread's row and column; c past the row for a thread without one.
template <typename T>
__device__ __forceinline__ void fetch_any(Raw8<T> &raw, T *turn, const uint8_t *base, uint32_t pitch, int first, uint32_t r, int c, int cols) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int from = j * 4 + (lane >> 3), col = __shfl_sync(~0u, c, from) + (lane & 7);
    const uint32_t row = __shfl_sync(~0u, r, from);
    T v = T(0.f);
    if (col < cols) v = ((const T *)(base + (uint64_t)row * pitch))[first + col];
    turn[j * 32 + lane] = v;
  }
  __syncwarp();
  raw.load(turn + lane * 8);
  __syncwarp();
}
template <typename T>
__device__ __forceinline__ void put_any(const Out8<T> &o, T *turn, uint8_t *base, uint32_t pitch, int first, uint32_t r, int c, int cols) {
  const int lane = threadIdx.x & 31;
  o.stage(turn + lane * 8);
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int from = j * 4 + (lane >> 3), col = __shfl_sync(~0u, c, from) + (lane & 7);
    const uint32_t row = __shfl_sync(~0u, r, from);
    if (col < cols) ((T *)(base + (uint64_t)row * pitch))[first + col] = turn[j * 32 + lane];
  }
  __syncwarp();
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

template <typename T>
__device__ __forceinline__ F8 eight(const Raw8<T> &r) {
  float f[8];
  r.get(f);
  return from8(f);
}

// A thread's piece on its way: eight columns of a row (and the eight that go with them, of a gated matrix).
template <typename T, int OP, bool GATED, bool VEC>
struct Piece {
  uint32_t r;     // row
  int u;          // piece of the row
  bool on;
  Raw8<T> raw, raw2;
  uint2 w, w2;
  int s, s2;

  __device__ __forceinline__ T *row(uint8_t *p, uint32_t pitch) const { return (T *)(p + (uint64_t)r * pitch); }
  __device__ __forceinline__ uint8_t *record(const CkptArgs &a) const { return a.ckpt + (uint64_t)r * a.row_bytes; }
  __device__ __forceinline__ int column() const { return on ? u * 8 : 1 << 30; }
  __device__ __forceinline__ void fetch(Raw8<T> &v, const CkptArgs &a, int first, T *turn) const {
    if (VEC) fetch8(v, row(const_cast<uint8_t *>(a.in), a.pitch_in) + first, column(), a.cols);
    else fetch_any(v, turn, a.in, a.pitch_in, first, r, column(), a.cols);
  }
  __device__ __forceinline__ void put(const Out8<T> &v, const CkptArgs &a, uint8_t *to, uint32_t pitch, int first, T *turn) const {
    if (VEC) put8(row(to, pitch) + first, column(), a.cols, v);
    else put_any(v, turn, to, pitch, first, r, column(), a.cols);
  }
  // piece i of n; whole warps
  __device__ __forceinline__ void ask(const CkptArgs &a, uint32_t row0, int i, int n, T *turn) {
    on = i < n;
    r = on ? __umulhi((uint32_t)i, a.inv_units) : 0u;
    u = on ? i - (int)r * a.units : 0;
    r += row0;
    if (OP == kLoad || OP == kBackward) {
      w = w2 = make_uint2(0u, 0u), s = s2 = 0;
      if (on) {
        const uint8_t *rec = record(a);
        w = *(const uint2 *)(rec + u * 8);
        s = rec[a.codes + (u >> 2)];
        if (GATED) w2 = *(const uint2 *)(rec + a.padded + u * 8), s2 = rec[a.codes + a.scales + (u >> 2)];
      }
    }
    if (OP == kLoad) return;
    fetch(raw, a, 0, turn);
    if (OP == kForward && GATED) fetch(raw2, a, a.cols, turn);
  }
  template <int ACT>
  __device__ __forceinline__ void finish(const CkptArgs &a, T *turn) {
    uint64_t slope;
    if (OP == kStore || OP == kForward) {
      if (OP == kForward) {
        const F8 z = eight(raw);
        Out8<T> o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint64_t f = act2<T, ACT>(z.p[j], &slope);
          if (GATED) f = pair_mul(f, eight(raw2).p[j]);
          o.set(j, f);
        }
        put(o, a, a.out, a.pitch_out, 0, turn);
      }
      if (OP == kStore || a.ckpt) {
        uint8_t *rec = record(a);
        keep8(raw, eight(raw), rec + u * 8, rec + a.codes + (u >> 2), on, a.int8);
        if (GATED) keep8(raw2, eight(raw2), rec + a.padded + u * 8, rec + a.codes + a.scales + (u >> 2), on, a.int8);
      }
      return;
    }
    const F8 z = decode8(w, s, a.int8);
    Out8<T> dz, du, f;
    if (OP == kLoad) {
#pragma unroll
      for (int j = 0; j < 4; ++j) dz.set(j, z.p[j]);
      put(dz, a, a.out, a.pitch_out, 0, turn);
      return;
    }
    F8 up;
    if (GATED) up = decode8(w2, s2, a.int8);
    const F8 d = eight(raw);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t v = act2<T, ACT>(z.p[j], &slope);
      if (GATED) {
        du.set(j, pair_mul(v, d.p[j]));
        dz.set(j, pair_mul(pair_mul(slope, up.p[j]), d.p[j]));
        f.set(j, pair_mul(v, up.p[j]));
      } else {
        dz.set(j, pair_mul(slope, d.p[j]));
        f.set(j, v);
      }
    }
    put(dz, a, a.out, a.pitch_out, 0, turn);
    if (GATED) put(du, a, a.out, a.pitch_out, a.cols, turn);
    if (a.again) put(f, a, a.again, a.pitch_again, 0, turn);
  }
};

// Two pieces of a thread are on their way at a time; one of a gated matrix, whose registers are better spent on threads (two: 312 us against
// 300 at 16384 x 6144).  Small CTAs, as many as there are tiles: 512 threads 331 us, 256 302, 128 295, forty registers or more alike.
template <typename T, int OP, int ACT, bool GATED, bool VEC>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 12 : 9) ckpt_kernel(const CkptArgs a) {
  __shared__ __align__(32) T turns[VEC ? 1 : kThreads / 32][VEC ? 1 : 256];
  T *const turn = turns[VEC ? 0 : threadIdx.x >> 5];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t row0 = blockIdx.x * a.tile_rows;
  const int n = (int)min((uint32_t)a.tile_rows, (uint32_t)a.M - row0) * a.units;   // (a multiple of four: a block is whole)
  for (int i = threadIdx.x; i - (int)threadIdx.x < n; i += (GATED ? 1 : 2) * kThreads) {
    Piece<T, OP, GATED, VEC> p, q;
    p.ask(a, row0, i, n, turn);
    if (!GATED) q.ask(a, row0, i + kThreads, n, turn);
    p.template finish<ACT>(a, turn);
    if (!GATED) q.template finish<ACT>(a, turn);
  }
}

template <typename T, int OP, int ACT, bool GATED>
cudaError_t launch_ckpt(const alg_ckpt_s &h, CkptArgs a, bool vec, cudaStream_t st) {
  a.row_bytes = (uint32_t)h.row_bytes;
  a.cols = h.cols, a.padded = h.padded, a.codes = h.parts * h.padded, a.scales = h.padded / kBlock;
  a.units = h.padded / 8;
  a.inv_units = (uint32_t)((0x100000000ull + a.units - 1) / a.units);
  a.int8 = h.format == ALG_Q8_INT8;
  // tiles of about four pieces a thread
  a.tile_rows = a.units >= 4 * kThreads ? 1 : 4 * kThreads / a.units;
  const int64_t tiles = (a.M + a.tile_rows - 1) / a.tile_rows;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)tiles);   // (2^30 rows at most)
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
  h->device = dev;
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
  if (h->parts != 1 || !X || !ckpt || ldx < h->cols || ldx >= kMaxLd || !on_element(X, e) || ((uintptr_t)ckpt & 15u)) return ALG_ERR_INVALID_ARG;
  if (meet(span(X, ldx, h->cols, e, M), records(*h, ckpt, M)) || !is_current(h->device)) return ALG_ERR_INVALID_ARG;
  CkptArgs a = {};
  a.in = (const uint8_t *)X, a.pitch_in = (uint32_t)(ldx * e), a.ckpt = (uint8_t *)ckpt, a.M = M;
  const bool vec = vectors(*h, X, ldx, e);
  cudaStream_t st = (cudaStream_t)stream;
  return ckpt_done(x_dtype == ALG_BF16 ? launch_ckpt<__nv_bfloat16, kStore, ALG_ACT_NONE, false>(*h, a, vec, st)
                                       : launch_ckpt<float, kStore, ALG_ACT_NONE, false>(*h, a, vec, st));
}

alg_status_t alg_ckpt_load(alg_ckpt_t h, const void *ckpt, int64_t M, void *X, int64_t ldx, alg_dtype_t x_dtype, void *stream) {
  alg_status_t s = ckpt_common(h, M, x_dtype);
  if (s != ALG_OK || M == 0) return s;
  const size_t e = elem_size(x_dtype);
  if (h->parts != 1 || !X || !ckpt || ldx < h->cols || ldx >= kMaxLd || !on_element(X, e) || ((uintptr_t)ckpt & 15u)) return ALG_ERR_INVALID_ARG;
  if (meet(span(X, ldx, h->cols, e, M), records(*h, ckpt, M)) || !is_current(h->device)) return ALG_ERR_INVALID_ARG;
  CkptArgs a = {};
  a.out = (uint8_t *)X, a.pitch_out = (uint32_t)(ldx * e), a.ckpt = (uint8_t *)ckpt, a.M = M;
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
  if (!Z || !A || ldz < wide || lda < h->cols || ldz >= kMaxLd || lda >= kMaxLd || !on_element(Z, e) || !on_element(A, e) || ((uintptr_t)ckpt & 15u)) return ALG_ERR_INVALID_ARG;
  const RowSpan z = span(Z, ldz, wide, e, M), out = span(A, lda, h->cols, e, M), rec = records(*h, ckpt, M);
  if ((meet(out, z) && !same_rows(out, z)) || meet(rec, z) || meet(rec, out) || !is_current(h->device)) return ALG_ERR_INVALID_ARG;
  CkptArgs a = {};
  a.in = (const uint8_t *)Z, a.pitch_in = (uint32_t)(ldz * e), a.out = (uint8_t *)A, a.pitch_out = (uint32_t)(lda * e), a.ckpt = (uint8_t *)ckpt, a.M = M;
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
  if (!ckpt || !dA || !dZ || ldda < h->cols || lddz < wide || (A && lda < h->cols) || ldda >= kMaxLd || lddz >= kMaxLd || lda >= kMaxLd || !on_element(dA, e) || !on_element(dZ, e) || !on_element(A, e) ||
      ((uintptr_t)ckpt & 15u))
    return ALG_ERR_INVALID_ARG;
  const RowSpan g = span(dA, ldda, h->cols, e, M), out = span(dZ, lddz, wide, e, M), again = span(A, lda, h->cols, e, M), rec = records(*h, ckpt, M);
  if ((meet(out, g) && !same_rows(out, g)) || meet(again, g) || meet(again, out) || meet(rec, g) || meet(rec, out) || meet(rec, again) ||
      !is_current(h->device))
    return ALG_ERR_INVALID_ARG;
  CkptArgs a = {};
  a.in = (const uint8_t *)dA, a.pitch_in = (uint32_t)(ldda * e), a.out = (uint8_t *)dZ, a.pitch_out = (uint32_t)(lddz * e), a.again = (uint8_t *)A,
  a.pitch_again = (uint32_t)(lda * e), a.ckpt = (uint8_t *)ckpt, a.M = M;
  const bool vec = vectors(*h, dA, ldda, e) && vectors(*h, dZ, lddz, e) && vectors(*h, A, lda, e);
  cudaStream_t st = (cudaStream_t)stream;
  return ckpt_done(dtype == ALG_BF16 ? launch_act<__nv_bfloat16, kBackward>(*h, a, vec, st) : launch_act<float, kBackward>(*h, a, vec, st));
}

}  // extern "C"
