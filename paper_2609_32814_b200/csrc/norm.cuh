// A block's border: Y = R + alpha * scale * g * (norm(F) * w + b) and N = norm(Y) * w' + b', and the gradients of both.
//
// A row is D <= 8192 features, read and written once: bound by HBM, if the arithmetic is kept short (72 instructions a value
// took twice the time of the bytes).  A group of T threads takes a row at a time, sixteen columns a thread (eight in the gradients of LayerNorm to 4096); the rows of its
// operands come into shared memory by the bulk copy engine, `stages` rows ahead, so that what is in flight does not depend on how
// many registers the arithmetic takes.  Vectors are folded once a CTA (alpha * scale * post_weight, ...) and kept in shared memory; arithmetic is on
// pairs; up to four sums cross the group in one exchange.
// Gradient of v = (x - mean) r, r = 1 / sqrt(var + eps), for a gradient h of v:
//     dx = r (h - mean(h) - v mean(h v))       (RMS: without mean(h), mean(x) = 0)
// Column sums: with a = dR * g every vector behind F needs only P = sum_b a v and Q = sum_b a:
//     d_post_weight = alpha scale P,  d_post_bias = alpha scale Q,  d_scale = alpha (post_weight P + post_bias Q).
// A thread keeps the sums of its columns over all rows of its group in registers, the groups of a CTA meet in shared memory at the end, and
// a second launch adds the CTAs' sums in CTA order.
// Measured, back to back: forward, 32768 x 4096 bf16, RMS, gate of each element 205 to 210 us (6.4 TB/s); backward, LayerNorm, 16384 x 4096, fp32
// stream, gate of each element 285 us (5.2 TB/s: the sums leave eight columns a thread, three exchanges a row); one row 4 us.
#pragma once

#include "common.cuh"
#include "rows.cuh"
#include "tc_common.cuh"

namespace algproj {

struct NormArgs;
// A translation unit each for a direction and type of the residual stream (F, gate and N bf16), and in the backward pass for a norm: the kernels with their form as a constant.
// types: 2 for an fp32 stream, + 1 for fp32 F, gate and N; alike: see NormArgs::off; exact:
// rows of whole 16-byte words, on 16 bytes.
cudaError_t launch_norm_forward_any(NormArgs &a, int types, bool alike, bool exact, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_backward_any(NormArgs &a, int types, bool alike, bool exact, int grid, size_t smem, cudaStream_t st);   // rows of eight columns a thread
cudaError_t launch_norm_backward_any_wide(NormArgs &a, int types, bool alike, bool exact, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_forward_bf16(NormArgs &a, int form, bool layer, bool on16, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_forward_f32(NormArgs &a, int form, bool layer, bool on16, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_backward_rms_bf16(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_backward_layer_bf16(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_backward_layer_wide_bf16(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_backward_rms_f32(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_backward_layer_f32(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st);
cudaError_t launch_norm_backward_layer_wide_f32(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st);


constexpr int kMaxStages = 4;
constexpr int kMaxGroups = 15;             // named barriers 1 .. 15
constexpr int kBudget = 224 * 1024;        // shared memory of a CTA for its vectors and rows
constexpr int kNarrow = 4096;              // widest row of eight columns a thread
constexpr int kThreads = 512;              // of a CTA, at most
constexpr int kSums = 4;                   // column sums: dN * v, dN, P, Q

enum { kX, kT, kN, kF, kG, kOps };          // operands: R or Y, dY, dN, F, gate of each element
struct NormArgs {
  uint32_t M;
  int D, T, G, stages;
  int flags, layer;
  float eps, alpha;
  const uint8_t *op[kOps];      // rows of the operands, nullptr for none
  uint32_t pitch[kOps], bytes[kOps];   // bytes between rows, of a row
  int at[kOps], stage_bytes;    // where a row lies in a stage
  int period, off, ld_off;      // rows whose first value lies off a granule of 4 or 8: by (off + row * ld_off) mod granule, the same every `period` rows
  const void *gate;             // of each row
  const float *post_w, *post_b, *scale, *pre_w, *pre_b;
  uint8_t *y, *out;             // forward: Y, N; backward: dR, dF
  uint8_t *dg;                  // backward: gradient of the gate
  uint32_t pitch_y, pitch_out, pitch_dg;
  int kept;                     // the folded vectors a kernel reads, a bit each
  int vectors;                  // their bytes in shared memory; 0: read where they lie
  float *part;                  // [CTAs][kSums][D]
  int *status;
  long long wait_limit;
  uint32_t stall;               // test aid: bytes that are expected of a row beside its own, and never come
};

// The form of a call: what it does, as a constant of a kernel (kAny: found out at run time, with every branch that costs: gradients of
// 16384 x 4096 rows 467 us against 320).
enum { kFormPre = 1, kFormPost = 2, kFormJoin = 4, kFormGate = 8, kAny = -1 };   // + kFormGate * gate
// gate of each element: whether through a sigmoid is part of the form, asked at run time it kept registers alive that the backward pass
// spilled (LayerNorm of 16384 x 4096: 4 % more); a row's gate asks at run time
enum { kGateNone, kGateRow, kGateElement, kGateSigmoid };

namespace {

// Shared memory of a CTA: barriers, the reductions' two slots, then the rows.
constexpr int kBarBytes = kMaxGroups * kMaxStages * 8;
constexpr int kRedBytes = 2 * 32 * 16;   // two slots of one float4 for each warp
constexpr int kRowsAt = (kBarBytes + kRedBytes + 127) / 128 * 128;

__device__ __forceinline__ void group_barrier(int g, int T) {
  if (T == 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(g + 1), "r"(T) : "memory");
}
// Sums of up to four values over the group's threads, to all of them.  In a warp the lanes halve the values between them (six
// exchanges for four values, not twenty), then each lane fetches one value of every eighth warp.  Two slots in turn: a thread that
// writes a slot again has passed the barrier behind everybody's reading of it.
template <int K>
__device__ __forceinline__ void group_sum(float (&v)[K], float4 *red, int &turn, int g, int T) {
  const int lane = threadIdx.x & 31;
  float r;   // of value lane & 3 (K > 2), lane & 1 (K = 2), or the only one
  if (K == 1) {
    r = v[0];
  } else {
    float a0, a1;
    if (K > 2) {
      const float hi0 = v[K > 2 ? 2 : 0], hi1 = K > 3 ? v[K > 3 ? 3 : 0] : 0.f, lo0 = v[0], lo1 = v[K > 1 ? 1 : 0];
      const bool up = lane & 2;
      a0 = (up ? hi0 : lo0) + __shfl_xor_sync(~0u, up ? lo0 : hi0, 2);
      a1 = (up ? hi1 : lo1) + __shfl_xor_sync(~0u, up ? lo1 : hi1, 2);
    } else {
      a0 = v[0], a1 = v[K > 1 ? 1 : 0];
    }
    const bool odd = lane & 1;
    r = (odd ? a1 : a0) + __shfl_xor_sync(~0u, odd ? a0 : a1, 1);
  }
  if (K == 1) r += __shfl_xor_sync(~0u, r, 1);
  if (K <= 2) r += __shfl_xor_sync(~0u, r, 2);
  r += __shfl_xor_sync(~0u, r, 4);
  r += __shfl_xor_sync(~0u, r, 8);
  r += __shfl_xor_sync(~0u, r, 16);
  constexpr int kValues = K > 2 ? 4 : K;
  if (T > 32) {
    const int warps = T >> 5, first = g * warps, mine = (threadIdx.x >> 5) - first;
    float *slot = (float *)(red + turn * 32 + first);
    turn ^= 1;
    if (lane < kValues) slot[mine * kValues + lane] = r;
    group_barrier(g, T);
    r = lane < warps * kValues ? slot[lane] : 0.f;
    if (kValues > 2 && lane + 32 < warps * kValues) r += slot[lane + 32];   // (sixteen warps at most)
#pragma unroll
    for (int o = kValues; o < 32; o <<= 1) r += __shfl_xor_sync(~0u, r, o);
  } else {
    __syncwarp();   // (a barrier of the group, as callers count on)
  }
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = K == 1 ? r : __shfl_sync(~0u, r, k);
}

// A thread's pieces of eight columns.  Rows on 16 bytes: eight consecutive ones, or, where operands are fp32, four and four that lie
// T * 4 columns apart (eight fp32 values in a row would have every second thread's 16 bytes meet in the same banks).  Else every T-th
// column, whose scalar accesses coalesce.
// Rows need not begin on a granule (eight bf16 values, four fp32): where all operands lie off it alike, a CTA takes rows that lie off it by the same
// `shift`, and column c is at c + shift of the granules, so that accesses are whole ones all the same; threads at a row's ends mask theirs.
// kExact: no shift, and every row is whole 16-byte words of each type; all rows and vectors lie on 16 bytes.  kWhole: and inside, all of them
// (nothing is asked, which the backward pass has no registers for: gradients of 16384 x 4096 rows 265 us against 311).
enum { kScalar, kEight, kFours, kExact = 4, kWhole = 8 + kExact };
template <int HOW>
struct Cols {
  static constexpr int MAP = HOW & 3;
  int t, T, shift, end;   // end: D + shift
  __device__ __forceinline__ int at(int v, int j) const {
    return MAP == kEight ? (v * T + t) * 8 + j : MAP == kFours ? ((2 * v + (j >> 2)) * T + t) * 4 + (j & 3) : t + (v * 8 + j) * T;
  }
  __device__ __forceinline__ bool on(int v, int j) const {
    if ((HOW & kWhole) == kWhole) return true;
    if (HOW & kExact) return at(v, MAP == kEight ? 0 : j & 4) < end;
    return at(v, j) >= shift && at(v, j) < end;
  }
  // granule `from` (its first value's place) of `n`: some of it inside the row; all of it
  __device__ __forceinline__ bool some(int from) const { return (HOW & kWhole) == kWhole || from < end; }
  __device__ __forceinline__ bool all(int from, int n) const { return HOW & kExact ? some(from) : from >= shift && from + n <= end; }
  template <typename T_>
  __device__ __forceinline__ F8 load(const T_ *row, int v) const {   // zero outside the row
    float f[8];
    if (MAP == kScalar) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = on(v, j) ? to_f32(row[at(v, j)]) : 0.f;
      return from8(f);
    }
    Raw8<T_> r;
    if (MAP == kEight) {
      if (some(at(v, 0))) r.load(row + at(v, 0));
      else r.zero();
    } else {
      if ((HOW & kWhole) != kWhole) r.zero();
      if (some(at(v, 0))) r.load4(0, row + at(v, 0));
      if (some(at(v, 4))) r.load4(1, row + at(v, 4));
    }
    r.get(f);
    return HOW & kExact ? from8(f) : inside(from8(f), v);
  }
  template <typename T_>
  __device__ __forceinline__ void store(T_ *row, int v, const F8 &a) const {
    float f[8];
    to8(a, f);
    if (HOW & kExact) {
      if (MAP == kEight) {
        if (some(at(v, 0))) store8(row + at(v, 0), f);
      } else {
        if (some(at(v, 0))) store4(row + at(v, 0), f[0], f[1], f[2], f[3]);
        if (some(at(v, 4))) store4(row + at(v, 4), f[4], f[5], f[6], f[7]);
      }
    } else if (MAP == kEight && all(at(v, 0), 8)) {
      store8(row + at(v, 0), f);
    } else if (MAP == kFours && all(at(v, 0), 4) && all(at(v, 4), 4)) {
      store4(row + at(v, 0), f[0], f[1], f[2], f[3]);
      store4(row + at(v, 4), f[4], f[5], f[6], f[7]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (on(v, j)) from_f32(f[j], row + at(v, j));
    }
  }
  // `a` inside the row, zero outside
  __device__ __forceinline__ F8 inside(const F8 &a, int v) const {
    if ((HOW & kWhole) == kWhole) return a;
    if (HOW & kExact && MAP == kEight) return some(at(v, 0)) ? a : all8(0.f);
    if (MAP == kEight && all(at(v, 0), 8)) return a;
    if (MAP == kFours && all(at(v, 0), 4) && all(at(v, 4), 4)) return a;
    float f[8];
    to8(a, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = on(v, j) ? f[j] : 0.f;
    return from8(f);
  }
  // Where the folded vectors keep a place: for consecutive eights in two planes of fours, again for the banks.
  __device__ __forceinline__ static int kept(int c, int pieces) { return MAP == kEight ? ((c >> 2 & 1) * pieces + (c >> 3)) * 4 + (c & 3) : c; }
  __device__ __forceinline__ F8 load_kept(const float *vec, int v, int pieces) const {
    float f[8];
    if (MAP == kScalar) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = vec[at(v, j)];
      return from8(f);
    }
    const float4 a = *(const float4 *)(vec + (MAP == kEight ? (v * T + t) * 4 : at(v, 0))), b = *(const float4 *)(vec + (MAP == kEight ? (pieces + v * T + t) * 4 : at(v, 4)));
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    return from8(f);
  }
};
template <int HOW>
__device__ __forceinline__ int shift_of(const NormArgs &a) {
  if (HOW & kExact || HOW == kScalar) return 0;
  return (a.off + (int)(blockIdx.x % a.period) * a.ld_off) & ((HOW & 3) == kEight ? 7 : 3);
}

// The vectors of a call, folded: in shared memory where that leaves room for the rows, else read from where they lie.
enum { kVecW, kVecB, kVecPreW, kVecPreB };   // alpha * scale * post_weight, alpha * scale * post_bias, pre_weight, pre_bias
struct Vectors {
  const float *at[4];   // in shared memory
  __device__ __forceinline__ static float value(const NormArgs &a, int which, int c) {
    if (which == kVecPreW) return a.pre_w ? a.pre_w[c] : 1.f;
    if (which == kVecPreB) return a.pre_b ? a.pre_b[c] : 0.f;
    const float s = a.alpha * (a.scale ? a.scale[c] : 1.f);
    return which == kVecW ? s * (a.post_w ? a.post_w[c] : 1.f) : a.post_b ? s * a.post_b[c] : 0.f;
  }
  __device__ __forceinline__ static float4 value4(const NormArgs &a, int which, int c) {
    auto four = [&](const float *p, float none) { return p ? *(const float4 *)(p + c) : make_float4(none, none, none, none); };
    if (which >= kVecPreW) return which == kVecPreW ? four(a.pre_w, 1.f) : four(a.pre_b, 0.f);
    const float4 s = four(a.scale, 1.f), v = which == kVecW ? four(a.post_w, 1.f) : four(a.post_b, 0.f);
    return make_float4(a.alpha * s.x * v.x, a.alpha * s.y * v.y, a.alpha * s.z * v.z, a.alpha * s.w * v.w);
  }
};
// Which of them a kernel keeps; all threads, before the rows.
template <int MAP, int V>
__device__ __forceinline__ Vectors fold_vectors(const NormArgs &a, uint8_t *smem) {
  Vectors vec = {{nullptr, nullptr, nullptr, nullptr}};
  float *to = (float *)(smem + kRowsAt);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!(a.kept >> k & 1) || !a.vectors) continue;
    const int shift = shift_of<MAP>(a);
    if (MAP & kExact) {
#pragma unroll 4
      for (int c = threadIdx.x * 4; c < a.T * V * 8; c += blockDim.x * 4)
        *(float4 *)(to + Cols<MAP>::kept(c, a.T * V)) = c < a.D ? Vectors::value4(a, k, c) : make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
#pragma unroll 4
      for (int c = threadIdx.x; c < a.T * V * 8; c += blockDim.x)
        to[Cols<MAP>::kept(c, a.T * V)] = c >= shift && c < a.D + shift ? Vectors::value(a, k, c - shift) : 0.f;
    }
    vec.at[k] = to;
    to += a.T * V * 8;
  }
  return vec;
}
template <int MAP, int V, int FORM>
__device__ __forceinline__ F8 vector8(const NormArgs &a, const Vectors &vec, int which, const Cols<MAP> &cols, int v) {
  if (V == 1 || FORM != kAny || a.vectors) return cols.load_kept(vec.at[which], v, a.T * V);
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = cols.on(v, j) ? Vectors::value(a, which, cols.at(v, j) - cols.shift) : 0.f;
  return from8(f);
}

// A row of the operands on its way into shared memory.  The warps of a group share the asking: a copy takes its thread about 150
// cycles, and a warp that asked for all five would have the others wait at the next barrier.  (What has landed before it is expected
// only makes the barrier's count negative for a while.)  A row off 16 bytes comes with the rest of the 16-byte words that hold its ends, and lies
// as far into its place in the stage as it does into the first of them.
template <bool OFF>
__device__ __forceinline__ void issue_row(const NormArgs &a, uint32_t stage, uint32_t bar, uint32_t row, int t) {
  if (t & 31) return;
  auto from = [&](int k) { return a.op[k] + (uint64_t)row * a.pitch[k]; };
  auto bytes = [&](int k) { return OFF ? (((uint32_t)(uintptr_t)from(k) & 15u) + a.bytes[k] + 15u) & ~15u : a.bytes[k]; };
  if (t == 0) {
    uint32_t total = a.stall;
#pragma unroll
    for (int k = 0; k < kOps; ++k) total += a.op[k] ? bytes(k) : 0u;
    tc::mbar_expect_tx(bar, total);
  }
  for (int k = t >> 5; k < kOps; k += a.T >> 5)
    if (a.op[k])
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(stage + a.at[k]),
                   "l"((uintptr_t)from(k) & ~(uintptr_t)15), "r"(bytes(k)), "r"(bar)
                   : "memory");
}
template <typename T, int MAP>
__device__ __forceinline__ const T *staged(const NormArgs &a, const uint8_t *stage, int k, uint32_t row, int shift) {
  if (MAP & kExact) return (const T *)(stage + a.at[k]);
  return (const T *)(stage + a.at[k] + (int)(((uint32_t)(uintptr_t)a.op[k] + row * a.pitch[k]) & 15u) - shift * (int)sizeof(T));
}

// A group's rows: those of its CTA's shift (the grid is a multiple of the period).
__device__ __forceinline__ uint32_t row_step(const NormArgs &a) { return gridDim.x * a.G; }
__device__ __forceinline__ uint32_t first_row(const NormArgs &a, int g) { return blockIdx.x % a.period + a.period * (blockIdx.x / a.period * a.G + g); }

// The loop over a group's rows: body(row, stage, release); release() once the row's operands are read and a barrier of the group has
// followed.  A wait that runs out says so in the status word.  From then on nothing is right and nothing more is asked for, but every thread still goes
// the same way to the end, where it gives the copies on their way time to land: the CTA's shared memory is not handed on before.
template <int MAP, int V, typename XT, typename BT, typename Body>
__device__ __forceinline__ void each_row(const NormArgs &a, uint8_t *smem, Vectors *vec, Body body) {
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  uint8_t *const rows = smem + kRowsAt + a.vectors + g * a.stages * a.stage_bytes;
  const uint32_t bar = tc::smem_u32(smem) + g * a.stages * 8, rows_at = tc::smem_u32(rows);
  if (t == 0) {
    for (int s = 0; s < a.stages; ++s) tc::mbar_init(bar + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  group_barrier(g, a.T);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t first = first_row(a, g), step = row_step(a);
  for (int s = 0; s < a.stages; ++s)
    if (first + s * step < a.M) issue_row<!(MAP & kExact)>(a, rows_at + s * a.stage_bytes, bar + 8 * s, first + s * step, t);
  *vec = fold_vectors<MAP, V>(a, smem);
  __syncthreads();
  int s = 0;
  uint32_t parity = 0;
  bool failed = false;
  for (uint32_t row = first; row < a.M; row += step) {
    if (!tc::mbar_try_wait(bar + 8 * s, parity) && !failed) {
      const long long t0 = clock64();
      while (!tc::mbar_try_wait(bar + 8 * s, parity))
        if (clock64() - t0 > a.wait_limit) {
          failed = true;
          atomicExch(a.status, (int)ALG_ERR_DEVICE_TIMEOUT);
          break;
        }
    }
    body(row, (const uint8_t *)rows + s * a.stage_bytes, [&] {
      if (!failed && row + a.stages * step < a.M) issue_row<!(MAP & kExact)>(a, rows_at + s * a.stage_bytes, bar + 8 * s, row + a.stages * step, t);
    });
    if (++s == a.stages) s = 0, parity ^= 1;
  }
  if (failed)
    for (const long long t0 = clock64(); clock64() - t0 < kLandCycles;) {
    }
}

// The gate of a row, asked for one row ahead.
template <typename BT>
__device__ __forceinline__ float next_gate(const BT *gate, uint32_t row, const NormArgs &a, float &ahead) {
  const uint32_t step = row_step(a);
  const float now = row < step ? to_f32(gate[row]) : ahead;   // (a group's first row is below the step)
  if (row + step < a.M) ahead = to_f32(gate[row + step]);
  return now;
}

// FULL: LayerNorm, or with biases or their gradients; LayerNorm where the form is a constant.
template <typename XT, typename BT, int MAP, int V, bool FULL, int FORM>
__global__ void __launch_bounds__(kThreads, 1) norm_forward_kernel(const NormArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  float4 *red = (float4 *)(smem + kBarBytes);
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  const int shift = shift_of<MAP>(a);
  const Cols<MAP> cols = {t, a.T, shift, a.D + shift};
  const float inv_d = 1.f / (float)a.D;
  constexpr bool any = FORM == kAny;
  constexpr int gate_of = any ? 0 : FORM / kFormGate;
  const bool pre = any ? a.flags & ALG_NORM_PRE : FORM & kFormPre, join = any ? a.flags & ALG_NORM_JOIN : FORM & kFormJoin;
  const bool post = any ? a.flags & ALG_NORM_POST : FORM & kFormPost, layer = any ? FULL && a.layer : FULL;
  const bool gate_row = any ? a.flags & ALG_NORM_GATE_ROW : gate_of == kGateRow, gate_el = any ? a.flags & ALG_NORM_GATE_ELEMENT : gate_of >= kGateElement;
  const bool sig = any || gate_of == kGateRow ? a.flags & ALG_NORM_GATE_SIGMOID : gate_of == kGateSigmoid;
  int turn = 0;
  Vectors vec;
  float gate_ahead = 0.f;
  each_row<MAP, V, XT, BT>(a, smem, &vec, [&](uint32_t row, const uint8_t *st, auto release) {
    F8 y[V], f[V], q[V];
    bool held = true;
    const float gate = gate_row ? next_gate((const BT *)a.gate, row, a, gate_ahead) : 1.f;
    // takes the mean off z and finds 1 / sqrt(var + eps)
    auto stat = [&](F8 (&z)[V]) {
      if (layer) {
        float m[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) m[0] += sum8(z[v]);
        group_sum(m, red, turn, g, a.T);
        if (held) release(), held = false;
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = cols.inside(z[v] + -m[0] * inv_d, v);
      }
      float s[1] = {0.f};
#pragma unroll
      for (int v = 0; v < V; ++v) s[0] += dot8(z[v], z[v]);
      group_sum(s, red, turn, g, a.T);
      if (held) release(), held = false;
      return rsqrtf(s[0] * inv_d + a.eps);
    };
#pragma unroll
    for (int v = 0; v < V; ++v) y[v] = cols.load(staged<XT, MAP>(a, st, kX, row, shift), v);
    if (join) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        f[v] = cols.load(staged<BT, MAP>(a, st, kF, row, shift), v);
        if (gate_el) q[v] = cols.load(staged<BT, MAP>(a, st, kG, row, shift), v);
      }
      const float rf = post ? stat(f) : 1.f, g1 = gate_row && sig ? sigmoid(gate) : gate;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const F8 w = vector8<MAP, V, FORM>(a, vec, kVecW, cols, v);
        F8 n = f[v] * w * rf;
        if (FULL) n = n + vector8<MAP, V, FORM>(a, vec, kVecB, cols, v);
        if (gate_el) {
          if (sig) {
            float e[8];
            to8(q[v], e);
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = sigmoid(e[j]);
            q[v] = from8(e);
          }
          y[v] = fma8(n, q[v], y[v]);
        } else {
          y[v] = fma8(n, g1, y[v]);
        }
        cols.store((XT *)(a.y + (uint64_t)row * a.pitch_y) - shift, v, y[v]);
      }
    }
    if (pre) {
      const float ry = stat(y);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        F8 n = y[v] * ry * vector8<MAP, V, FORM>(a, vec, kVecPreW, cols, v);
        if (FULL) n = n + vector8<MAP, V, FORM>(a, vec, kVecPreB, cols, v);
        cols.store((BT *)(a.out + (uint64_t)row * a.pitch_out) - shift, v, n);
      }
    }
    if (held) {
      group_barrier(g, a.T);
      release();
    }
  });
}

template <typename XT, typename BT, int MAP, int V, bool FULL, int FORM>
__global__ void __launch_bounds__(kThreads, 1) norm_backward_kernel(const NormArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  float4 *red = (float4 *)(smem + kBarBytes);
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  const int shift = shift_of<MAP>(a);
  const Cols<MAP> cols = {t, a.T, shift, a.D + shift};
  const float inv_d = 1.f / (float)a.D;
  constexpr bool any = FORM == kAny;
  constexpr int gate_of = any ? 0 : FORM / kFormGate;
  const bool pre = any ? a.flags & ALG_NORM_PRE : FORM & kFormPre, join = any ? a.flags & ALG_NORM_JOIN : FORM & kFormJoin;
  const bool post = any ? a.flags & ALG_NORM_POST : FORM & kFormPost, layer = any ? FULL && a.layer : FULL;
  const bool gate_row = any ? a.flags & ALG_NORM_GATE_ROW : gate_of == kGateRow, gate_el = any ? a.flags & ALG_NORM_GATE_ELEMENT : gate_of >= kGateElement;
  const bool sig = any || gate_of == kGateRow ? a.flags & ALG_NORM_GATE_SIGMOID : gate_of == kGateSigmoid;
  // (a form that is a constant comes with dY and with every gradient wanted)
  const bool has_dy = any ? a.op[kT] != nullptr : true, to_f = any ? a.out != nullptr : true, to_gate = any ? a.dg != nullptr : true;
  F8 sum[kSums][V];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int v = 0; v < V; ++v) sum[k][v] = all8(0.f);
  int turn = 0;
  Vectors vec;
  float gate_ahead = 0.f;
  each_row<MAP, V, XT, BT>(a, smem, &vec, [&](uint32_t row, const uint8_t *st, auto release) {
    // a row of eight columns a thread stays in registers, a wider one is read from its stage as needed
    F8 hx, hn, hf, hh;   // (hh: dN * pre_weight)
    auto x_of = [&](int v) { return V == 1 ? hx : cols.load(staged<XT, MAP>(a, st, kX, row, shift), v); };
    auto n_of = [&](int v) { return V == 1 ? hn : cols.load(staged<BT, MAP>(a, st, kN, row, shift), v); };
    auto h_of = [&](int v) { return V == 1 ? hh : n_of(v) * vector8<MAP, V, FORM>(a, vec, kVecPreW, cols, v); };
    auto f_of = [&](int v) { return V == 1 ? hf : cols.load(staged<BT, MAP>(a, st, kF, row, shift), v); };
    F8 d[V], q[V];   // dY, then the gradient of R; the gate
    bool held = V == 1;
    const float gate_1 = gate_row ? next_gate((const BT *)a.gate, row, a, gate_ahead) : 1.f;
    if (V == 1) {
      if (pre) hx = cols.load(staged<XT, MAP>(a, st, kX, row, shift), 0), hn = cols.load(staged<BT, MAP>(a, st, kN, row, shift), 0), hh = hn * vector8<MAP, V, FORM>(a, vec, kVecPreW, cols, 0);
      if (join) hf = cols.load(staged<BT, MAP>(a, st, kF, row, shift), 0);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      d[v] = has_dy ? cols.load(staged<XT, MAP>(a, st, kT, row, shift), v) : all8(0.f);
      if (V == 1 && gate_el) q[v] = cols.load(staged<BT, MAP>(a, st, kG, row, shift), v);
    }
    // statistics of Y and F, and the means of h = dN * pre_weight and of h times the normed Y
    float mx = 0.f, mf = 0.f, mh = 0.f;
    if (layer && (pre || post)) {
      float m[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (pre) m[0] += sum8(x_of(v)), m[2] += sum8(h_of(v));
        if (post) m[1] += sum8(f_of(v));
      }
      group_sum(m, red, turn, g, a.T);
      if (held) release(), held = false;
      mx = m[0] * inv_d, mf = m[1] * inv_d, mh = m[2] * inv_d;
      if (V == 1) {
        if (pre) hx = cols.inside(hx + -mx, 0);
        if (post) hf = cols.inside(hf + -mf, 0);
      }
    }
    // (x and f without their means)
    auto xc_of = [&](int v) { return V == 1 || !layer ? x_of(v) : cols.inside(x_of(v) + -mx, v); };
    auto fc_of = [&](int v) { return V == 1 || !layer || !post ? f_of(v) : cols.inside(f_of(v) + -mf, v); };
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (pre) {
        const F8 x = xc_of(v);
        s[0] += dot8(x, x);
        s[2] += dot8(x, h_of(v));
      }
      if (post) {
        const F8 f = fc_of(v);
        s[1] += dot8(f, f);
      }
    }
    if (pre || post) {
      group_sum(s, red, turn, g, a.T);
      if (held) release(), held = false;
    }
    const float rx = rsqrtf(s[0] * inv_d + a.eps), rf = post ? rsqrtf(s[1] * inv_d + a.eps) : 1.f;
    const float mhv = s[2] * inv_d * rx;
    // the row's gate and its slope
    float gr = gate_1, gs = 1.f;
    if (gate_row && sig) {
      float e1;
      gr = sigmoid(gate_1, e1), gs = gr * (gr * e1);
    }
    F8 e[V];   // gradient of V
    float m[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (pre) {
        const F8 x = xc_of(v) * rx, n = n_of(v);
        sum[0][v] = fma8(n, x, sum[0][v]);
        if (FULL) sum[1][v] = sum[1][v] + n;
        F8 h = h_of(v);
        if (layer) h = h + -mh;
        d[v] = fma8(fma8(x, -mhv, h), rx, d[v]);
        if (layer) d[v] = cols.inside(d[v], v);
      }
      cols.store((XT *)(a.y + (uint64_t)row * a.pitch_y) - shift, v, d[v]);
      if (!join) continue;
      const F8 f = fc_of(v) * rf, w = vector8<MAP, V, FORM>(a, vec, kVecW, cols, v);
      F8 dg = d[v] * gr;   // the gradient behind the gate
      auto of_gate = [&] {
        F8 b = f * w;
        if (FULL) b = b + vector8<MAP, V, FORM>(a, vec, kVecB, cols, v);
        return b * d[v];
      };
      if (gate_el) {
        F8 z = V == 1 ? q[v] : cols.load(staged<BT, MAP>(a, st, kG, row, shift), v);
        if (sig) {   // the gate's gradient pair by pair: with the slopes kept for later the narrow LayerNorm spills (16384 x 4096: 330 us, so 285)
          F8 b, add;
          if (FULL) add = vector8<MAP, V, FORM>(a, vec, kVecB, cols, v);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float lo, hi, e0, e1;
            halves(z.p[j], lo, hi);
            lo = sigmoid(lo, e0), hi = sigmoid(hi, e1);
            z.p[j] = pair(lo, hi);
            b.p[j] = pair_mul(f.p[j], w.p[j]);
            if (FULL) b.p[j] = pair_add(b.p[j], add.p[j]);
            b.p[j] = pair_mul(pair_mul(b.p[j], d[v].p[j]), pair_mul(z.p[j], pair_mul(z.p[j], pair(e0, e1))));
          }
          if (to_gate) cols.store((BT *)(a.dg + (uint64_t)row * a.pitch_dg) - shift, v, b);
        }
        dg = d[v] * z;
      }
      sum[2][v] = fma8(dg, f, sum[2][v]);
      if (FULL) sum[3][v] = sum[3][v] + dg;
      e[v] = dg * w;
      if (gate_row) m[2] += sum8(of_gate());
      else if (gate_el && to_gate && !sig) cols.store((BT *)(a.dg + (uint64_t)row * a.pitch_dg) - shift, v, of_gate());
      if (post) {
        if (layer) m[0] += sum8(e[v]);
        m[1] += dot8(e[v], f);
      } else if (to_f) {
        cols.store((BT *)(a.out + (uint64_t)row * a.pitch_out) - shift, v, e[v]);
      }
    }
    if (join && ((post && to_f) || (gate_row && to_gate))) {
      group_sum(m, red, turn, g, a.T);
      if (held) release(), held = false;
      if (gate_row && to_gate && t == 0) from_f32(m[2] * gs, (BT *)a.dg + row);
      if (post && to_f) {
        const float me = m[0] * inv_d, mev = m[1] * inv_d;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          F8 o = fma8(fc_of(v) * rf, -mev, e[v]);
          if (layer) o = o + -me;
          cols.store((BT *)(a.out + (uint64_t)row * a.pitch_out) - shift, v, o * rf);
        }
      }
    }
    if (V > 1 || held) {
      group_barrier(g, a.T);
      release();
    }
  });
  if (!a.part) return;
  // the groups' sums meet where the rows were, [groups][D], and are added in their order
  float *acc = (float *)(smem + kRowsAt + a.vectors);
  float *part = a.part + (size_t)blockIdx.x * kSums * a.D;
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    if ((k < 2 ? !pre : !join) || (!FULL && (k & 1))) continue;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float f[8];
      to8(sum[k][v], f);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (cols.on(v, j)) acc[g * a.D + cols.at(v, j) - shift] = f[j];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += blockDim.x) {
      float s = 0.f;
      for (int i = 0; i < a.G; ++i) s += acc[i * a.D + c];
      part[(size_t)k * a.D + c] = s;
    }
  }
}

inline cudaError_t launch_norm_kernel(const void *kernel, int grid, int threads, size_t smem, cudaStream_t st, void **params) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel, params);
  if (e == cudaSuccess) count_launch(1);
  return e;
}

constexpr int kSmemMax = kRowsAt + kBudget;

template <bool BACK, typename XT, typename BT, int MAP, int V, bool FULL, int FORM>
cudaError_t launch_rows(NormArgs &a, int grid, size_t smem, cudaStream_t st) {
  static OncePerDevice once;
  const void *k;
  if constexpr (BACK) k = (const void *)norm_backward_kernel<XT, BT, MAP, V, FULL, FORM>;
  else k = (const void *)norm_forward_kernel<XT, BT, MAP, V, FULL, FORM>;
  const cudaError_t e = once([&] { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax); });
  if (e != cudaSuccess) return e;
  void *params[] = {&a};
  return launch_norm_kernel(k, grid, a.T * a.G, smem, st, params);
}

// The kernel of a form.
template <bool BACK, typename XT, int V, bool LAYER, int FORM>
cudaError_t launch_form(NormArgs &a, bool on16, int grid, size_t smem, cudaStream_t st) {
  constexpr int kMap = sizeof(XT) == 4 ? kFours : kEight;
  // forward: rows of whole 16-byte words (of F in bf16: eights) on 16 bytes; backward: such as fill the threads' pieces
  if (on16 && (BACK ? a.D == a.T * V * 8 : a.D % 8 == 0))
    return launch_rows<BACK, XT, __nv_bfloat16, kMap | (BACK ? kWhole : kExact), V, LAYER, FORM>(a, grid, smem, st);
  return launch_rows<BACK, XT, __nv_bfloat16, kMap, V, LAYER, FORM>(a, grid, smem, st);
}
template <bool BACK, typename XT, int V, bool LAYER, int BASE>
cudaError_t launch_gate(NormArgs &a, int gate, bool on16, int grid, size_t smem, cudaStream_t st) {
  switch (gate) {
    case kGateNone: return launch_form<BACK, XT, V, LAYER, BASE>(a, on16, grid, smem, st);
    case kGateRow: return launch_form<BACK, XT, V, LAYER, BASE + kFormGate * kGateRow>(a, on16, grid, smem, st);
    case kGateElement: return launch_form<BACK, XT, V, LAYER, BASE + kFormGate * kGateElement>(a, on16, grid, smem, st);
    default: return launch_form<BACK, XT, V, LAYER, BASE + kFormGate * kGateSigmoid>(a, on16, grid, smem, st);
  }
}
template <bool BACK, typename XT, int V, bool LAYER>
cudaError_t launch_forms(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st) {
  const int gate = form / kFormGate;
  switch (form % kFormGate) {
    case kFormJoin | kFormPost | kFormPre: return launch_gate<BACK, XT, V, LAYER, kFormJoin | kFormPost | kFormPre>(a, gate, on16, grid, smem, st);
    case kFormJoin | kFormPost: return launch_gate<BACK, XT, V, LAYER, kFormJoin | kFormPost>(a, gate, on16, grid, smem, st);
    case kFormJoin | kFormPre: return launch_gate<BACK, XT, V, LAYER, kFormJoin | kFormPre>(a, gate, on16, grid, smem, st);
    default: return launch_form<BACK, XT, V, LAYER, kFormPre>(a, on16, grid, smem, st);
  }
}

}  // namespace
}  // namespace algproj
