// A block's border: Y = R + alpha * scale * g * (norm(F) * w + b) and N = norm(Y) * w' + b', and the gradients of both.
//
// A row is D <= 8192 features, read and written once: bound by HBM, if the arithmetic is kept short (72 instructions a value
// took twice the time of the bytes).  A group of T threads takes a row at a time, eight columns a thread (16 past 4096); the rows of its
// operands come into shared memory by the bulk copy engine, `stages` rows ahead, so that what is in flight does not depend on how
// many registers the arithmetic takes.  Vectors are folded once a CTA (alpha * scale * post_weight, ...) and kept in shared memory; arithmetic is on
// pairs; up to four sums cross the group in one exchange.
// Gradient of v = (x - mean) r, r = 1 / sqrt(var + eps), for a gradient h of v:
//     dx = r (h - mean(h) - v mean(h v))       (RMS: without mean(h), mean(x) = 0)
// Column sums: with a = dR * g every vector behind F needs only P = sum_b a v and Q = sum_b a:
//     d_post_weight = alpha scale P,  d_post_bias = alpha scale Q,  d_scale = alpha (post_weight P + post_bias Q).
// A thread keeps the sums of its columns over all rows of its group in registers, the groups of a CTA meet in shared memory at the end, and
// a second launch adds the CTAs' sums in CTA order.
#include <cmath>
#include <new>

#include "common.cuh"
#include "rows.cuh"
#include "tc_common.cuh"

using namespace algproj;

struct alg_norm_s {
  int D = 0, flags = 0;
  alg_norm_kind_t kind = ALG_NORM_RMS;
  float eps = 0.f;
  alg_dtype_t stream_dtype = ALG_BF16, dtype = ALG_BF16;
  int device = 0, num_sms = 148;
  int *d_status = nullptr;
};

namespace algproj {
namespace {

constexpr int kMaxStages = 4;
constexpr int kMaxGroups = 15;             // named barriers 1 .. 15
constexpr int kBudget = 224 * 1024;        // shared memory of a CTA for its vectors and rows
constexpr int kVectorBytes = 64 * 1024;    // folded vectors that are kept in shared memory
constexpr int kNarrow = 4096;              // widest row of eight columns a thread
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
  const void *gate;             // of each row
  const float *post_w, *post_b, *scale, *pre_w, *pre_b;
  uint8_t *y, *out;             // forward: Y, N; backward: dR, dF
  uint8_t *dg;                  // backward: gradient of the gate
  uint32_t pitch_y, pitch_out, pitch_dg;
  int vectors;                  // bytes of the folded vectors in shared memory; 0: read where they lie
  float *part;                  // [CTAs][kSums][D]
  int *status;
  long long wait_limit;
};

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
    r = 0.f;
    for (int i = lane; i < warps * kValues; i += 32) r += slot[i];
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
// kWhole: every thread's pieces are inside the row, nothing is asked.
enum { kScalar, kEight, kFours, kWhole = 4 };
template <int HOW>
struct Cols {
  static constexpr int MAP = HOW & 3;
  int t, T, D;
  __device__ __forceinline__ int at(int v, int j) const {
    return MAP == kEight ? (v * T + t) * 8 + j : MAP == kFours ? ((2 * v + (j >> 2)) * T + t) * 4 + (j & 3) : t + (v * 8 + j) * T;
  }
  __device__ __forceinline__ bool on(int v, int j) const { return HOW & kWhole || at(v, MAP == kEight ? 0 : MAP == kFours ? j & 4 : j) < D; }
  template <typename T_>
  __device__ __forceinline__ F8 load(const T_ *row, int v) const {   // zero past the row's end
    float f[8];
    if (MAP == kEight) {
      Raw8<T_> r;
      if (on(v, 0)) r.load(row + at(v, 0));
      else r.zero();
      r.get(f);
    } else if (MAP == kFours) {
      Raw8<T_> r;
      r.zero();
      if (on(v, 0)) r.load4(0, row + at(v, 0));
      if (on(v, 4)) r.load4(1, row + at(v, 4));
      r.get(f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = on(v, j) ? to_f32(row[at(v, j)]) : 0.f;
    }
    return from8(f);
  }
  template <typename T_>
  __device__ __forceinline__ void store(T_ *row, int v, const F8 &a) const {
    float f[8];
    to8(a, f);
    if (MAP == kEight) {
      if (on(v, 0)) store8(row + at(v, 0), f);
    } else if (MAP == kFours) {
      if (on(v, 0)) store4(row + at(v, 0), f[0], f[1], f[2], f[3]);
      if (on(v, 4)) store4(row + at(v, 4), f[4], f[5], f[6], f[7]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (on(v, j)) from_f32(f[j], row + at(v, j));
    }
  }
  // `a` inside the row, zero past its end
  __device__ __forceinline__ F8 inside(const F8 &a, int v) const {
    if (HOW & kWhole) return a;
    if (MAP == kEight) return on(v, 0) ? a : all8(0.f);
    float f[8];
    to8(a, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = on(v, j) ? f[j] : 0.f;
    return from8(f);
  }
  // Where the folded vectors keep a column: for consecutive eights in two planes of fours, again for the banks.
  __device__ __forceinline__ static int kept(int c, int pieces) { return MAP == kEight ? ((c >> 2 & 1) * pieces + (c >> 3)) * 4 + (c & 3) : c; }
  __device__ __forceinline__ F8 load_kept(const float *vec, int v, int pieces) const {
    if (MAP != kEight) return load(vec, v);
    float f[8];
    const float4 a = *(const float4 *)(vec + (v * T + t) * 4), b = *(const float4 *)(vec + (pieces + v * T + t) * 4);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    return from8(f);
  }
};

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
};
// Which of them a kernel keeps; all threads, before the rows.
template <int MAP, int V>
__device__ __forceinline__ Vectors fold_vectors(const NormArgs &a, uint8_t *smem, bool full) {
  Vectors vec = {{nullptr, nullptr, nullptr, nullptr}};
  float *to = (float *)(smem + kRowsAt);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const bool used = (k < 2 ? a.flags & ALG_NORM_JOIN : a.flags & ALG_NORM_PRE) && (full || !(k & 1));
    if (!used || !a.vectors) continue;
    for (int c = threadIdx.x; c < a.T * V * 8; c += blockDim.x) to[Cols<MAP>::kept(c, a.T * V)] = c < a.D ? Vectors::value(a, k, c) : 0.f;
    vec.at[k] = to;
    to += a.T * V * 8;
  }
  return vec;
}
template <int MAP, int V>
__device__ __forceinline__ F8 vector8(const NormArgs &a, const Vectors &vec, int which, const Cols<MAP> &cols, int v) {
  if (V == 1 || a.vectors) return cols.load_kept(vec.at[which], v, a.T * V);
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = cols.on(v, j) ? Vectors::value(a, which, cols.at(v, j)) : 0.f;
  return from8(f);
}

// A row of the operands on its way into shared memory; one thread.
__device__ __forceinline__ void issue_row(const NormArgs &a, uint32_t stage, uint32_t bar, uint32_t row) {
  uint32_t total = 0;
#pragma unroll
  for (int k = 0; k < kOps; ++k) total += a.op[k] ? a.bytes[k] : 0u;
  tc::mbar_expect_tx(bar, total);
#pragma unroll
  for (int k = 0; k < kOps; ++k)
    if (a.op[k])
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(stage + a.at[k]),
                   "l"(a.op[k] + (uint64_t)row * a.pitch[k]), "r"(a.bytes[k]), "r"(bar)
                   : "memory");
}
// Unaligned rows: the group copies them itself.
template <typename XT, typename BT>
__device__ __forceinline__ void copy_row(const NormArgs &a, uint8_t *stage, uint32_t row, int t) {
#pragma unroll
  for (int k = 0; k < kOps; ++k) {
    if (!a.op[k]) continue;
    const uint8_t *p = a.op[k] + (uint64_t)row * a.pitch[k];
    for (int c = t; c < a.D; c += a.T) {
      if (k < kN) ((XT *)(stage + a.at[k]))[c] = ((const XT *)p)[c];
      else ((BT *)(stage + a.at[k]))[c] = ((const BT *)p)[c];
    }
  }
}

// The loop over a group's rows: body(row, stage, release); release() once the row's operands are read and a barrier of the group has
// followed.
template <int MAP, int V, typename XT, typename BT, typename Body>
__device__ __forceinline__ void each_row(const NormArgs &a, uint8_t *smem, Vectors *vec, bool full, Body body) {
  constexpr bool copies = MAP == kScalar;
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  uint8_t *const rows = smem + kRowsAt + a.vectors + g * a.stages * a.stage_bytes;
  const uint32_t bar = tc::smem_u32(smem) + g * a.stages * 8, rows_at = tc::smem_u32(rows);
  if (!copies && t == 0) {
    for (int s = 0; s < a.stages; ++s) tc::mbar_init(bar + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t first = blockIdx.x * a.G + g, step = gridDim.x * a.G;
  if (!copies && t == 0)
    for (int s = 0; s < a.stages; ++s)
      if (first + s * step < a.M) issue_row(a, rows_at + s * a.stage_bytes, bar + 8 * s, first + s * step);
  *vec = fold_vectors<MAP, V>(a, smem, full);
  __syncthreads();
  int s = 0;
  uint32_t parity = 0;
  bool failed = false;   // after a wait that ran out nothing is right, but every thread still goes the same way to the end
  for (uint32_t row = first; row < a.M; row += step) {
    if (copies) {
      group_barrier(g, a.T);   // (the row before it is read)
      copy_row<XT, BT>(a, rows, row, t);
      group_barrier(g, a.T);
    } else if (!tc::mbar_try_wait(bar + 8 * s, parity) && !failed) {
      const long long t0 = clock64();
      while (!tc::mbar_try_wait(bar + 8 * s, parity))
        if (clock64() - t0 > a.wait_limit) {
          failed = true;
          atomicExch(a.status, (int)ALG_ERR_DEVICE_TIMEOUT);
          break;
        }
    }
    body(row, (const uint8_t *)rows + s * a.stage_bytes, [&] {
      if (!copies && t == 0 && row + a.stages * step < a.M) issue_row(a, rows_at + s * a.stage_bytes, bar + 8 * s, row + a.stages * step);
    });
    if (!copies && ++s == a.stages) s = 0, parity ^= 1;
  }
}

// FULL: LayerNorm, or with biases or their gradients.
template <typename XT, typename BT, int MAP, int V, bool FULL>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512, 1) norm_forward_kernel(const NormArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  float4 *red = (float4 *)(smem + kBarBytes);
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  const Cols<MAP> cols = {t, a.T, a.D};
  const float inv_d = 1.f / (float)a.D;
  const bool layer = FULL && a.layer, sig = a.flags & ALG_NORM_GATE_SIGMOID;
  int turn = 0;
  Vectors vec;
  each_row<MAP, V, XT, BT>(a, smem, &vec, FULL, [&](uint32_t row, const uint8_t *st, auto release) {
    F8 y[V], f[V], q[V];
    bool held = true;
    const float gate = a.flags & ALG_NORM_GATE_ROW ? to_f32(((const BT *)a.gate)[row]) : 1.f;
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
    for (int v = 0; v < V; ++v) y[v] = cols.load((const XT *)(st + a.at[kX]), v);
    if (a.flags & ALG_NORM_JOIN) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        f[v] = cols.load((const BT *)(st + a.at[kF]), v);
        if (a.flags & ALG_NORM_GATE_ELEMENT) q[v] = cols.load((const BT *)(st + a.at[kG]), v);
      }
      const float rf = a.flags & ALG_NORM_POST ? stat(f) : 1.f, g1 = a.flags & ALG_NORM_GATE_ROW && sig ? sigmoid(gate) : gate;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const F8 w = vector8<MAP, V>(a, vec, kVecW, cols, v);
        F8 n = f[v] * w * rf;
        if (FULL) n = n + vector8<MAP, V>(a, vec, kVecB, cols, v);
        if (a.flags & ALG_NORM_GATE_ELEMENT) {
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
        cols.store((XT *)(a.y + (uint64_t)row * a.pitch_y), v, y[v]);
      }
    }
    if (a.flags & ALG_NORM_PRE) {
      const float ry = stat(y);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        F8 n = y[v] * ry * vector8<MAP, V>(a, vec, kVecPreW, cols, v);
        if (FULL) n = n + vector8<MAP, V>(a, vec, kVecPreB, cols, v);
        cols.store((BT *)(a.out + (uint64_t)row * a.pitch_out), v, n);
      }
    }
    if (held) {
      group_barrier(g, a.T);
      release();
    }
  });
}

template <typename XT, typename BT, int MAP, int V, bool FULL>
__global__ void __launch_bounds__(512, 1) norm_backward_kernel(const NormArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  float4 *red = (float4 *)(smem + kBarBytes);
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  const Cols<MAP> cols = {t, a.T, a.D};
  const float inv_d = 1.f / (float)a.D;
  const bool pre = a.flags & ALG_NORM_PRE, join = a.flags & ALG_NORM_JOIN, post = a.flags & ALG_NORM_POST, layer = FULL && a.layer;
  const bool sig = a.flags & ALG_NORM_GATE_SIGMOID, gate_row = a.flags & ALG_NORM_GATE_ROW, gate_el = a.flags & ALG_NORM_GATE_ELEMENT;
  F8 sum[kSums][V];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int v = 0; v < V; ++v) sum[k][v] = all8(0.f);
  int turn = 0;
  Vectors vec;
  each_row<MAP, V, XT, BT>(a, smem, &vec, FULL, [&](uint32_t row, const uint8_t *st, auto release) {
    // a row of eight columns a thread stays in registers, a wider one is read from its stage as needed
    F8 hx, hn, hf;
    auto x_of = [&](int v) { return V == 1 ? hx : cols.load((const XT *)(st + a.at[kX]), v); };
    auto n_of = [&](int v) { return V == 1 ? hn : cols.load((const BT *)(st + a.at[kN]), v); };
    auto f_of = [&](int v) { return V == 1 ? hf : cols.load((const BT *)(st + a.at[kF]), v); };
    F8 d[V], q[V];   // dY, then the gradient of R; the gate
    bool held = V == 1;
    const float gate_1 = gate_row ? to_f32(((const BT *)a.gate)[row]) : 1.f;
    if (V == 1) {
      if (pre) hx = cols.load((const XT *)(st + a.at[kX]), 0), hn = cols.load((const BT *)(st + a.at[kN]), 0);
      if (join) hf = cols.load((const BT *)(st + a.at[kF]), 0);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      d[v] = a.op[kT] ? cols.load((const XT *)(st + a.at[kT]), v) : all8(0.f);
      if (V == 1 && gate_el) q[v] = cols.load((const BT *)(st + a.at[kG]), v);
    }
    // statistics of Y and F, and the means of h = dN * pre_weight and of h times the normed Y
    float mx = 0.f, mf = 0.f, mh = 0.f;
    if (layer) {
      float m[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (pre) m[0] += sum8(x_of(v)), m[2] += dot8(n_of(v), vector8<MAP, V>(a, vec, kVecPreW, cols, v));
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
        s[2] += dot8(x * n_of(v), vector8<MAP, V>(a, vec, kVecPreW, cols, v));
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
    const float gr = gate_row && sig ? sigmoid(gate_1) : gate_1, gs = sig ? gr * (1.f - gr) : 1.f;
    F8 e[V];   // gradient of V
    float m[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (pre) {
        const F8 x = xc_of(v) * rx, n = n_of(v);
        sum[0][v] = fma8(n, x, sum[0][v]);
        if (FULL) sum[1][v] = sum[1][v] + n;
        F8 h = n * vector8<MAP, V>(a, vec, kVecPreW, cols, v);
        if (layer) h = h + -mh;
        d[v] = fma8(fma8(x, -mhv, h), rx, d[v]);
        if (layer) d[v] = cols.inside(d[v], v);
      }
      cols.store((XT *)(a.y + (uint64_t)row * a.pitch_y), v, d[v]);
      if (!join) continue;
      const F8 f = fc_of(v) * rf, w = vector8<MAP, V>(a, vec, kVecW, cols, v);
      F8 dg = d[v] * gr;   // the gradient behind the gate
      F8 slope;
      if (gate_el) {
        F8 z = V == 1 ? q[v] : cols.load((const BT *)(st + a.at[kG]), v);
        if (sig) {
          float p[8];
          to8(z, p);
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = sigmoid(p[j]);
          z = from8(p);
          slope = fma8(z * z, -1.f, z);
        }
        dg = d[v] * z;
      }
      sum[2][v] = fma8(dg, f, sum[2][v]);
      if (FULL) sum[3][v] = sum[3][v] + dg;
      e[v] = dg * w;
      if (gate_row || (gate_el && a.dg)) {
        F8 b = f * w;
        if (FULL) b = b + vector8<MAP, V>(a, vec, kVecB, cols, v);
        b = b * d[v];
        if (gate_el) {
          if (sig) b = b * slope;
          cols.store((BT *)(a.dg + (uint64_t)row * a.pitch_dg), v, b);
        } else {
          m[2] += sum8(b);
        }
      }
      if (post) {
        if (layer) m[0] += sum8(e[v]);
        m[1] += dot8(e[v], f);
      } else if (a.out) {
        cols.store((BT *)(a.out + (uint64_t)row * a.pitch_out), v, e[v]);
      }
    }
    if (join && ((post && a.out) || (gate_row && a.dg))) {
      group_sum(m, red, turn, g, a.T);
      if (held) release(), held = false;
      if (gate_row && a.dg && t == 0) from_f32(m[2] * gs, (BT *)a.dg + row);
      if (post && a.out) {
        const float me = m[0] * inv_d, mev = m[1] * inv_d;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          F8 o = fma8(fc_of(v) * rf, -mev, e[v]);
          if (layer) o = o + -me;
          cols.store((BT *)(a.out + (uint64_t)row * a.pitch_out), v, o * rf);
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
        if (cols.on(v, j)) acc[g * a.D + cols.at(v, j)] = f[j];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += blockDim.x) {
      float s = 0.f;
      for (int i = 0; i < a.G; ++i) s += acc[i * a.D + c];
      part[(size_t)k * a.D + c] = s;
    }
  }
}

struct SumsArgs {
  int ctas, D, flags, full;
  float alpha;
  const float *part, *post_w, *post_b, *scale;
  float *d_post_w, *d_post_b, *d_scale, *d_pre_w, *d_pre_b;
};
// 32 columns a CTA, 32 slices of the CTAs' sums.
constexpr int kSlices = 32;
__global__ void __launch_bounds__(32 * kSlices) norm_sums_kernel(const SumsArgs a) {
  __shared__ float slice[kSums][kSlices][33];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  const bool used[kSums] = {(a.flags & ALG_NORM_PRE) != 0, (a.flags & ALG_NORM_PRE) && a.full, (a.flags & ALG_NORM_JOIN) != 0,
                            (a.flags & ALG_NORM_JOIN) && a.full};
  float s[kSums] = {0.f, 0.f, 0.f, 0.f};
  if (c < a.D)
#pragma unroll 2
    for (int i = y; i < a.ctas; i += kSlices) {
      const float *p = a.part + (size_t)i * kSums * a.D + c;
#pragma unroll
      for (int k = 0; k < kSums; ++k)
        if (used[k]) s[k] += p[(size_t)k * a.D];
    }
#pragma unroll
  for (int k = 0; k < kSums; ++k) slice[k][y][x] = s[k];
  __syncthreads();
  if (y >= kSums) return;
  // warp y adds up sum y of its columns
  float r = 0.f;
#pragma unroll 8
  for (int i = 0; i < kSlices; ++i) r += slice[y][i][x];
  slice[y][0][x] = r;
  asm volatile("bar.sync 1, %0;" ::"n"(32 * kSums) : "memory");
  if (c >= a.D) return;
  const float scale = a.alpha * (a.scale ? a.scale[c] : 1.f), w = a.alpha * (a.post_w ? a.post_w[c] : 1.f), b = a.alpha * (a.post_b ? a.post_b[c] : 0.f);
  if (y == 0 && a.d_pre_w) a.d_pre_w[c] = r;
  if (y == 1 && a.d_pre_b) a.d_pre_b[c] = r;
  if (y == 2 && a.d_post_w) a.d_post_w[c] = scale * r;
  if (y == 2 && a.d_scale) a.d_scale[c] = fmaf(w, r, b * slice[3][0][x]);
  if (y == 3 && a.d_post_b) a.d_post_b[c] = scale * r;
}

cudaError_t launch_pdl(const void *kernel, int grid, int threads, size_t smem, cudaStream_t st, void **params) {
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

template <bool BACK, typename XT, typename BT, int MAP, int V, bool FULL>
cudaError_t launch_rows(NormArgs &a, int grid, size_t smem, cudaStream_t st) {
  static OncePerDevice once;
  const void *k = BACK ? (const void *)norm_backward_kernel<XT, BT, MAP, V, FULL> : (const void *)norm_forward_kernel<XT, BT, MAP, V, FULL>;
  const cudaError_t e = once([&] { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax); });
  if (e != cudaSuccess) return e;
  void *params[] = {&a};
  return launch_pdl(k, grid, a.T * a.G, smem, st, params);
}
template <bool BACK, typename XT, typename BT, int V>
cudaError_t launch_wide(NormArgs &a, bool vec, bool full, int grid, size_t smem, cudaStream_t st) {
  constexpr int kMap = sizeof(XT) == 4 || sizeof(BT) == 4 ? kFours : kEight;
  if (!vec) return launch_rows<BACK, XT, BT, kScalar, V, true>(a, grid, smem, st);
  if (a.D == a.T * V * 8)
    return full ? launch_rows<BACK, XT, BT, kMap | kWhole, V, true>(a, grid, smem, st) : launch_rows<BACK, XT, BT, kMap | kWhole, V, false>(a, grid, smem, st);
  return full ? launch_rows<BACK, XT, BT, kMap, V, true>(a, grid, smem, st) : launch_rows<BACK, XT, BT, kMap, V, false>(a, grid, smem, st);
}
template <bool BACK, typename XT, typename BT>
cudaError_t launch_typed(NormArgs &a, bool vec, bool full, int grid, size_t smem, cudaStream_t st) {
  return a.D <= kNarrow ? launch_wide<BACK, XT, BT, 1>(a, vec, full, grid, smem, st) : launch_wide<BACK, XT, BT, 2>(a, vec, full, grid, smem, st);
}

// Threads of a row, rows a CTA works on at once, rows on their way; the grid.
int shape_rows(const alg_norm_s &h, NormArgs &a, bool back, bool full, size_t *smem) {
  const bool narrow = a.D <= kNarrow;
  const int pieces = (a.D + (narrow ? 7 : 15)) / (narrow ? 8 : 16);
  a.T = (pieces + 31) / 32 * 32;
  a.stage_bytes = 0;
  for (int k = 0; k < kOps; ++k) {
    a.at[k] = a.stage_bytes;
    a.bytes[k] = (uint32_t)(a.D * elem_size(k < kN ? h.stream_dtype : h.dtype));
    if (a.op[k]) a.stage_bytes += (int)((a.bytes[k] + 15) / 16 * 16);
  }
  const size_t stage = a.stage_bytes;
  const int kept = ((a.flags & ALG_NORM_JOIN ? 1 : 0) + (a.flags & ALG_NORM_PRE ? 1 : 0)) * (full ? 2 : 1);
  a.vectors = kept * a.T * (narrow ? 1 : 2) * 32;
  if (a.vectors > kVectorBytes) a.vectors = 0;   // (only rows of sixteen columns a thread have as many)
  const size_t budget = (size_t)kBudget - a.vectors;
  const int threads = back || !narrow ? 512 : 1024;
  int groups = threads / a.T;
  if (groups > kMaxGroups) groups = kMaxGroups;
  const int64_t per_sm = (a.M + h.num_sms - 1) / h.num_sms;
  if (groups > per_sm) groups = (int)per_sm;
  while (groups > 1 && 2 * groups * stage > budget) --groups;   // (a row ahead of each)
  a.G = groups;
  int stages = (int)(budget / (groups * stage));
  if (stages > kMaxStages) stages = kMaxStages;
  const int64_t rows = (a.M + (int64_t)groups * h.num_sms - 1) / ((int64_t)groups * h.num_sms);
  if (stages > rows) stages = (int)rows;
  a.stages = stages;
  size_t bytes = (size_t)groups * stages * stage;
  if (back && bytes < (size_t)groups * a.D * 4) bytes = (size_t)groups * a.D * 4;   // the groups' sums meet there
  *smem = kRowsAt + a.vectors + bytes;
  const int64_t ctas = (a.M + groups - 1) / groups;
  return (int)(ctas < h.num_sms ? ctas : h.num_sms);
}

template <bool BACK>
cudaError_t launch_norm(const alg_norm_s &h, NormArgs &a, bool vec, bool *full, int *grid, cudaStream_t st) {
  size_t smem = 0;
  *full = *full || a.layer || a.post_b || a.pre_b || !vec;
  *grid = shape_rows(h, a, BACK, *full, &smem);
  if (h.stream_dtype == ALG_BF16)
    return h.dtype == ALG_BF16 ? launch_typed<BACK, __nv_bfloat16, __nv_bfloat16>(a, vec, *full, *grid, smem, st)
                               : launch_typed<BACK, __nv_bfloat16, float>(a, vec, *full, *grid, smem, st);
  return h.dtype == ALG_BF16 ? launch_typed<BACK, float, __nv_bfloat16>(a, vec, *full, *grid, smem, st)
                             : launch_typed<BACK, float, float>(a, vec, *full, *grid, smem, st);
}

constexpr int64_t kMaxLd = 1 << 30;   // (the kernels count the bytes between rows in 32 bits)
void put_operand(NormArgs &a, int k, const void *p, int64_t ld, size_t e) { a.op[k] = (const uint8_t *)p, a.pitch[k] = (uint32_t)(ld * e); }
// One matrix operand: its span, whether it is well formed, whether its rows lie on 16 bytes.
struct Operand {
  RowSpan s;
  bool ok, vec;
};
Operand operand(const void *p, int64_t ld, int64_t cols, size_t e, int64_t M) {
  if (!p) return {span(nullptr, 0, 0, 1, 0), true, true};
  return {span(p, ld, cols, e, M), ld >= cols && ld < kMaxLd && on_element(p, e), on_16(p, ld, e)};
}
bool vector_ok(const float *p) { return on_element(p, 4); }
bool vector_16(const float *p) { return ((uintptr_t)p & 15u) == 0; }
size_t sums_bytes(const alg_norm_s &h) { return (size_t)h.num_sms * kSums * h.D * sizeof(float); }

}  // namespace
}  // namespace algproj

extern "C" {

alg_status_t alg_norm_create(alg_norm_t *out, int D, alg_norm_kind_t kind, int flags, float eps, alg_dtype_t stream_dtype, alg_dtype_t dtype) {
  if (!out) return ALG_ERR_INVALID_ARG;
  *out = nullptr;
  if (D < 1 || (kind != ALG_NORM_RMS && kind != ALG_NORM_LAYER) || !(eps >= 0.f) || !std::isfinite(eps)) return ALG_ERR_INVALID_ARG;
  if ((stream_dtype != ALG_F32 && stream_dtype != ALG_BF16) || (dtype != ALG_F32 && dtype != ALG_BF16)) return ALG_ERR_INVALID_ARG;
  const bool join = flags & ALG_NORM_JOIN, row = flags & ALG_NORM_GATE_ROW, el = flags & ALG_NORM_GATE_ELEMENT;
  if (flags < 0 || flags > 63 || !(flags & (ALG_NORM_JOIN | ALG_NORM_PRE)) || (!join && (flags & ~ALG_NORM_PRE)) || (row && el) ||
      ((flags & ALG_NORM_GATE_SIGMOID) && !row && !el))
    return ALG_ERR_INVALID_ARG;
  if (D > ALG_NORM_MAX_D) return ALG_ERR_UNSUPPORTED_SHAPE;
  int dev = 0, sms = 0;
  const alg_status_t s = kernel_device(&dev, &sms);
  if (s != ALG_OK) return s;
  alg_norm_s *h = new (std::nothrow) alg_norm_s();
  if (!h) return ALG_ERR_INVALID_ARG;
  h->D = D, h->kind = kind, h->flags = flags, h->eps = eps;
  h->stream_dtype = stream_dtype, h->dtype = dtype;
  h->device = dev, h->num_sms = sms;
  if (cudaMalloc(&h->d_status, 4 * sizeof(int)) != cudaSuccess || cudaMemset(h->d_status, 0, 4 * sizeof(int)) != cudaSuccess ||
      cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess) {
    if (h->d_status) cudaFree(h->d_status);
    delete h;
    return ALG_ERR_CUDA;
  }
  *out = h;
  return ALG_OK;
}

alg_status_t alg_norm_destroy(alg_norm_t h) {
  if (!h) return ALG_ERR_INVALID_ARG;
  cudaFree(h->d_status);
  delete h;
  return ALG_OK;
}

alg_status_t alg_norm_workspace_bytes(alg_norm_t h, size_t *bytes) {
  if (!h || !bytes) return ALG_ERR_INVALID_ARG;
  *bytes = (sums_bytes(*h) + 255) / 256 * 256;
  return ALG_OK;
}

alg_status_t alg_norm_forward(alg_norm_t h, const void *R, int64_t ldr, const void *F, int64_t ldf, const void *gate, int64_t ldg,
                              const float *post_weight, const float *post_bias, const float *scale, float alpha, const float *pre_weight,
                              const float *pre_bias, int64_t M, void *Y, int64_t ldy, void *N, int64_t ldn, void *stream) {
  if (!h || M < 0 || M > (1 << 30)) return ALG_ERR_INVALID_ARG;
  if (M == 0) return ALG_OK;
  const bool join = h->flags & ALG_NORM_JOIN, pre = h->flags & ALG_NORM_PRE, post = h->flags & ALG_NORM_POST;
  const bool row = h->flags & ALG_NORM_GATE_ROW, el = h->flags & ALG_NORM_GATE_ELEMENT;
  if (!R || join != (F != nullptr) || join != (Y != nullptr) || pre != (N != nullptr) || (row || el) != (gate != nullptr)) return ALG_ERR_INVALID_ARG;
  if ((!post && (post_weight || post_bias)) || (!join && scale) || (!pre && (pre_weight || pre_bias))) return ALG_ERR_INVALID_ARG;
  const size_t ex = elem_size(h->stream_dtype), eb = elem_size(h->dtype);
  const int D = h->D;
  const Operand in[3] = {operand(R, ldr, D, ex, M), operand(F, ldf, D, eb, M), row ? operand(gate, 1, 1, eb, M) : operand(gate, ldg, D, eb, M)};
  const Operand to[2] = {operand(Y, ldy, D, ex, M), operand(N, ldn, D, eb, M)};
  bool vec = D % 8 == 0;
  for (const Operand &o : to) {
    if (!o.ok) return ALG_ERR_INVALID_ARG;
    vec = vec && o.vec;
    for (const Operand &i : in)
      if (meet(o.s, i.s) && !same_rows(o.s, i.s)) return ALG_ERR_INVALID_ARG;
  }
  for (int k = 0; k < 3; ++k) {
    if (!in[k].ok) return ALG_ERR_INVALID_ARG;
    vec = vec && (in[k].vec || (k == 2 && row));
  }
  if (meet(to[0].s, to[1].s)) return ALG_ERR_INVALID_ARG;
  for (const float *v : {post_weight, post_bias, scale, pre_weight, pre_bias}) {
    if (!vector_ok(v)) return ALG_ERR_INVALID_ARG;
    vec = vec && vector_16(v);
    for (const Operand &o : to)
      if (v && meet(o.s, span(v, D, D, 4, 1))) return ALG_ERR_INVALID_ARG;
  }
  if (!is_current(h->device)) return ALG_ERR_INVALID_ARG;
  NormArgs a = {};
  a.M = (uint32_t)M, a.D = D, a.flags = h->flags, a.layer = h->kind == ALG_NORM_LAYER, a.eps = h->eps, a.alpha = alpha;
  put_operand(a, kX, R, ldr, ex), put_operand(a, kF, F, ldf, eb), put_operand(a, kG, el ? gate : nullptr, ldg, eb);
  a.gate = row ? gate : nullptr;
  a.post_w = post_weight, a.post_b = post_bias, a.scale = scale, a.pre_w = pre_weight, a.pre_b = pre_bias;
  a.y = (uint8_t *)Y, a.pitch_y = (uint32_t)(ldy * ex), a.out = (uint8_t *)N, a.pitch_out = (uint32_t)(ldn * eb);
  a.status = h->d_status, a.wait_limit = kDefaultWaitLimit;
  int grid = 0;
  bool full = false;
  return launch_norm<false>(*h, a, vec, &full, &grid, (cudaStream_t)stream) == cudaSuccess ? ALG_OK : ALG_ERR_CUDA;
}

alg_status_t alg_norm_backward(alg_norm_t h, const void *Y, int64_t ldy, const void *dY, int64_t lddy, const void *dN, int64_t lddn, const void *F,
                               int64_t ldf, const void *gate, int64_t ldg, const float *post_weight, const float *post_bias, const float *scale,
                               float alpha, const float *pre_weight, int64_t M, void *dR, int64_t lddr, void *dF, int64_t lddf, void *dgate,
                               int64_t lddg, float *d_post_weight, float *d_post_bias, float *d_scale, float *d_pre_weight, float *d_pre_bias,
                               void *workspace, size_t workspace_bytes, void *stream) {
  if (!h || M < 0 || M > (1 << 30)) return ALG_ERR_INVALID_ARG;
  const bool join = h->flags & ALG_NORM_JOIN, pre = h->flags & ALG_NORM_PRE, post = h->flags & ALG_NORM_POST;
  const bool row = h->flags & ALG_NORM_GATE_ROW, el = h->flags & ALG_NORM_GATE_ELEMENT;
  const bool sums = d_post_weight || d_post_bias || d_scale || d_pre_weight || d_pre_bias;
  if ((!post && (post_weight || post_bias || d_post_weight || d_post_bias)) || (!join && (scale || d_scale || dF)) ||
      (!pre && (pre_weight || d_pre_weight || d_pre_bias)) || (!row && !el && dgate))
    return ALG_ERR_INVALID_ARG;
  const int D = h->D;
  float *const vectors_out[5] = {d_post_weight, d_post_bias, d_scale, d_pre_weight, d_pre_bias};
  const float *const vectors_in[4] = {post_weight, post_bias, scale, pre_weight};
  bool vec = D % 8 == 0;
  for (const float *v : vectors_out)
    if (!vector_ok(v)) return ALG_ERR_INVALID_ARG;
  for (const float *v : vectors_in) {
    if (!vector_ok(v)) return ALG_ERR_INVALID_ARG;
    vec = vec && vector_16(v);
  }
  if (sums && (!workspace || ((uintptr_t)workspace & 255u))) return ALG_ERR_INVALID_ARG;
  if (sums && workspace_bytes < sums_bytes(*h)) return ALG_ERR_WORKSPACE_TOO_SMALL;
  NormArgs a = {};
  if (M > 0) {
    if ((pre && !Y) || !dR || pre != (dN != nullptr) || join != (F != nullptr) || (row || el) != (gate != nullptr) || (!pre && !dY)) return ALG_ERR_INVALID_ARG;
    const size_t ex = elem_size(h->stream_dtype), eb = elem_size(h->dtype);
    const Operand in[5] = {operand(Y, ldy, D, ex, M), operand(dY, lddy, D, ex, M), operand(dN, lddn, D, eb, M), operand(F, ldf, D, eb, M),
                           row ? operand(gate, 1, 1, eb, M) : operand(gate, ldg, D, eb, M)};
    const Operand to[3] = {operand(dR, lddr, D, ex, M), operand(dF, lddf, D, eb, M),
                           row ? operand(dgate, 1, 1, eb, M) : operand(dgate, lddg, D, eb, M)};
    const RowSpan ws = sums ? span(workspace, 0, (int64_t)sums_bytes(*h), 1, 1) : span(nullptr, 0, 0, 1, 0);
    for (int k = 0; k < 5; ++k) {
      if (!in[k].ok || meet(ws, in[k].s)) return ALG_ERR_INVALID_ARG;
      vec = vec && (in[k].vec || (k == 4 && row));
      for (const float *v : vectors_out)
        if (v && meet(in[k].s, span(v, D, D, 4, 1))) return ALG_ERR_INVALID_ARG;
    }
    for (int k = 0; k < 3; ++k) {
      if (!to[k].ok || meet(ws, to[k].s)) return ALG_ERR_INVALID_ARG;
      vec = vec && (to[k].vec || (k == 2 && row));
      for (const Operand &i : in)
        if (meet(to[k].s, i.s) && !same_rows(to[k].s, i.s)) return ALG_ERR_INVALID_ARG;
      for (int l = 0; l < k; ++l)
        if (meet(to[k].s, to[l].s)) return ALG_ERR_INVALID_ARG;
      for (const float *v : vectors_out)
        if (v && meet(to[k].s, span(v, D, D, 4, 1))) return ALG_ERR_INVALID_ARG;
      for (const float *v : vectors_in)
        if (v && meet(to[k].s, span(v, D, D, 4, 1))) return ALG_ERR_INVALID_ARG;
    }
    put_operand(a, kX, pre ? Y : nullptr, ldy, ex);   // (Y is not needed without a norm behind it)
    put_operand(a, kT, dY, lddy, ex), put_operand(a, kN, dN, lddn, eb), put_operand(a, kF, F, ldf, eb);
    put_operand(a, kG, el ? gate : nullptr, ldg, eb);
    a.gate = row ? gate : nullptr;
    a.y = (uint8_t *)dR, a.pitch_y = (uint32_t)(lddr * ex), a.out = (uint8_t *)dF, a.pitch_out = (uint32_t)(lddf * eb);
    a.dg = (uint8_t *)dgate, a.pitch_dg = (uint32_t)(lddg * eb);
  }
  if (!is_current(h->device)) return ALG_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  a.M = (uint32_t)M, a.D = D, a.flags = h->flags, a.layer = h->kind == ALG_NORM_LAYER, a.eps = h->eps, a.alpha = alpha;
  a.post_w = post_weight, a.post_b = post_bias, a.scale = scale, a.pre_w = pre_weight;
  a.part = sums ? (float *)workspace : nullptr;
  a.status = h->d_status, a.wait_limit = kDefaultWaitLimit;
  int grid = 0;
  bool full = d_post_bias || d_pre_bias;
  if (M > 0 && launch_norm<true>(*h, a, vec, &full, &grid, st) != cudaSuccess) return ALG_ERR_CUDA;
  if (!sums) return ALG_OK;
  SumsArgs b = {grid, D, h->flags, full, alpha, a.part, post_weight, post_bias, scale, d_post_weight, d_post_bias, d_scale, d_pre_weight, d_pre_bias};
  void *params[] = {&b};
  return launch_pdl((const void *)norm_sums_kernel, (D + 31) / 32, 32 * kSlices, 0, st, params) == cudaSuccess ? ALG_OK : ALG_ERR_CUDA;
}

alg_status_t alg_norm_last_status(alg_norm_t h, void *stream, alg_status_t *status) {
  if (!h || !status) return ALG_ERR_INVALID_ARG;
  int v = 0;
  if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess || cudaMemcpy(&v, h->d_status, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess)
    return ALG_ERR_CUDA;
  if (v && (cudaMemset(h->d_status, 0, sizeof(int)) != cudaSuccess || cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess)) return ALG_ERR_CUDA;
  *status = (alg_status_t)v;
  return ALG_OK;
}

}  // extern "C"
