// A block's border: Y = R + alpha * scale * g * (norm(F) * w + b) and N = norm(Y) * w' + b', and the gradients of both.
//
// A row is D <= 8192 features, read and written once: bound by HBM.  A group of T threads takes a row at a time; the
// rows of its operands come into shared memory by the bulk copy engine, `stages` rows ahead, so that what is in flight does not
// depend on how many registers the arithmetic takes, and stay there while the row's statistics are found and used.
// Gradient of v = (x - mean) r, r = 1 / sqrt(var + eps), for a gradient h of v:
//     dx = r (h - mean(h) - v mean(h v))       (RMS: without mean(h), mean(x) = 0)
// Column sums: with a = alpha * dR * g every vector behind F needs only P = sum_b a v and Q = sum_b a:
//     d_post_weight = scale P,  d_post_bias = scale Q,  d_scale = post_weight P + post_bias Q.
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
constexpr int kStageBudget = 200 * 1024;   // shared memory for the rows of a CTA
constexpr int kSums = 4;                   // column sums: dN * v, dN, P, Q

struct NormArgs {
  int64_t M;
  int D, T, G, stages;
  int flags, layer;
  float eps, alpha;
  // forward: x = R, f = F, g = gate; backward: x = Y, t = dY, n = dN, f = F, g = gate
  const void *x, *t, *n, *f, *g;
  int64_t ldx, ldt, ldn, ldf, ldg;
  const float *post_w, *post_b, *scale, *pre_w, *pre_b;
  void *y, *out;                // forward: Y, N
  int64_t ldy, ldo;
  void *dr, *df, *dg;           // backward
  int64_t lddr, lddf, lddg;
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
// Sums over the group's threads, to all of them.  Two slots in turn: a thread that writes a slot again has passed the barrier
// behind everybody's reading of it.
template <int K>
__device__ __forceinline__ void group_sum(float (&v)[K], float4 *red, int &turn, int g, int T) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(~0u, v[k], o);
  if (T == 32) return;
  const int warps = T >> 5, first = g * warps, lane = threadIdx.x & 31;
  float4 *slot = red + turn * 32 + first;
  turn ^= 1;
  if (lane == 0) slot[(threadIdx.x >> 5) - first] = make_float4(v[0], K > 1 ? v[K > 1 ? 1 : 0] : 0.f, K > 2 ? v[K > 2 ? 2 : 0] : 0.f, 0.f);
  group_barrier(g, T);
  const float4 p = lane < warps ? slot[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
  v[0] = p.x;
  if (K > 1) v[K > 1 ? 1 : 0] = p.y;
  if (K > 2) v[K > 2 ? 2 : 0] = p.z;
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(~0u, v[k], o);
}

// A thread's pieces of eight: consecutive columns where rows lie on 16 bytes, else every T-th column (whose scalar accesses coalesce).
template <bool VEC>
struct Cols {
  int t, T, D;
  __device__ __forceinline__ int at(int v, int j) const { return VEC ? (v * T + t) * 8 + j : t + (v * 8 + j) * T; }
  __device__ __forceinline__ bool on(int v, int j) const { return at(v, j) < D; }
  template <typename T_>
  __device__ __forceinline__ void load(const T_ *row, int v, float (&f)[8], float none = 0.f) const {
    if (VEC) {
      if (at(v, 0) < D) {
        Raw8<T_> r;
        r.load(row + at(v, 0));
        r.get(f);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = none;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = on(v, j) ? to_f32(row[at(v, j)]) : none;
    }
  }
  template <typename T_>
  __device__ __forceinline__ void store(T_ *row, int v, const float (&f)[8]) const {
    if (VEC) {
      if (at(v, 0) < D) store8(row + at(v, 0), f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (on(v, j)) from_f32(f[j], row + at(v, j));
    }
  }
};

__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }

// The rows of one group on their way through shared memory.
template <bool VEC>
struct RowPipe {
  static constexpr int kOps = 5;
  const uint8_t *src[kOps];
  int64_t pitch[kOps];
  int bytes[kOps], at[kOps];   // of a row; its place in a stage
  int stage_bytes;
  uint32_t bar;                // shared address of the group's first barrier
  uint8_t *rows;
  bool failed = false;

  __device__ __forceinline__ const uint8_t *stage(int s) const { return rows + s * stage_bytes; }
  __device__ __forceinline__ void issue(int s, int64_t row) const {   // one thread
    int total = 0;
#pragma unroll
    for (int k = 0; k < kOps; ++k) total += src[k] ? bytes[k] : 0;
    tc::mbar_expect_tx(bar + 8 * s, total);
#pragma unroll
    for (int k = 0; k < kOps; ++k)
      if (src[k])
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                         tc::smem_u32(rows + s * stage_bytes + at[k])),
                     "l"(src[k] + row * pitch[k]), "r"(bytes[k]), "r"(bar + 8 * s)
                     : "memory");
  }
  // Unaligned rows: the group copies them itself.
  template <typename XT, typename BT>
  __device__ __forceinline__ void copy(int64_t row, int t, int T, int D) const {
#pragma unroll
    for (int k = 0; k < kOps; ++k) {
      if (!src[k]) continue;
      if (k < 2) {
        const XT *p = (const XT *)(src[k] + row * pitch[k]);
        for (int c = t; c < D; c += T) ((XT *)(rows + at[k]))[c] = p[c];
      } else {
        const BT *p = (const BT *)(src[k] + row * pitch[k]);
        for (int c = t; c < D; c += T) ((BT *)(rows + at[k]))[c] = p[c];
      }
    }
  }
  // After a wait that ran out nothing is right, but every thread still goes the same way to the end.
  __device__ __forceinline__ void wait(int s, uint32_t parity, int *status, long long limit) {
    if (tc::mbar_try_wait(bar + 8 * s, parity) || failed) return;
    const long long t0 = clock64();
    while (!tc::mbar_try_wait(bar + 8 * s, parity))
      if (clock64() - t0 > limit) {
        failed = true;
        atomicExch(status, (int)ALG_ERR_DEVICE_TIMEOUT);
        return;
      }
  }
};

template <bool VEC, typename XT, typename BT>
__device__ __forceinline__ RowPipe<VEC> make_pipe(const NormArgs &a, uint8_t *smem, int g) {
  RowPipe<VEC> p;
  const void *src[5] = {a.x, a.t, a.n, a.f, a.flags & ALG_NORM_GATE_ELEMENT ? a.g : nullptr};
  const int64_t ld[5] = {a.ldx, a.ldt, a.ldn, a.ldf, a.ldg};
  int off = 0;
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    const int e = k < 2 ? (int)sizeof(XT) : (int)sizeof(BT);
    p.src[k] = (const uint8_t *)src[k];
    p.pitch[k] = ld[k] * e;
    p.bytes[k] = a.D * e;
    p.at[k] = off;
    if (src[k]) off += (a.D * e + 15) / 16 * 16;
  }
  p.stage_bytes = off;
  p.bar = tc::smem_u32(smem) + g * a.stages * 8;
  p.rows = smem + kRowsAt + (size_t)g * a.stages * off;
  return p;
}

// The loop over a group's rows: body(row, stage base).
template <bool VEC, typename XT, typename BT, typename Body>
__device__ __forceinline__ void each_row(const NormArgs &a, uint8_t *smem, Body body) {
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  RowPipe<VEC> pipe = make_pipe<VEC, XT, BT>(a, smem, g);
  if (VEC) {
    if (t == 0) {
      for (int s = 0; s < a.stages; ++s) tc::mbar_init(pipe.bar + 8 * s, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      tc::fence_async_smem();
    }
    group_barrier(g, a.T);
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t first = (int64_t)blockIdx.x * a.G + g, step = (int64_t)gridDim.x * a.G;
  if (VEC && t == 0)
    for (int s = 0; s < a.stages; ++s)
      if (first + s * step < a.M) pipe.issue(s, first + s * step);
  int s = 0;
  uint32_t parity = 0;
  for (int64_t row = first; row < a.M; row += step) {
    if (VEC) {
      pipe.wait(s, parity, a.status, a.wait_limit);
    } else {
      pipe.template copy<XT, BT>(row, t, a.T, a.D);
      group_barrier(g, a.T);
    }
    const uint8_t *st = pipe.stage(s);
    body(row, st, pipe);
    group_barrier(g, a.T);   // everybody is done with the stage
    if (VEC) {
      if (t == 0 && row + a.stages * step < a.M) pipe.issue(s, row + a.stages * step);
      if (++s == a.stages) s = 0, parity ^= 1;
    }
  }
}

// Sum and sum of squares about the mean: r = 1 / sqrt(var + eps), mean.
struct Stat {
  float mean, r;
};

template <typename XT, typename BT, bool VEC, int V>
__global__ void __launch_bounds__(V == 1 ? 1024 : 512, 1) norm_forward_kernel(const NormArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  float4 *red = (float4 *)(smem + kBarBytes);
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  const Cols<VEC> cols = {t, a.T, a.D};
  const float inv_d = 1.f / (float)a.D;
  int turn = 0;
  // mean and factor of the group's row held in z
  auto stat = [&](const float (&z)[V][8]) {
    Stat st = {0.f, 0.f};
    if (a.layer) {
      float m[1] = {0.f};
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) m[0] += z[v][j];
      group_sum(m, red, turn, g, a.T);
      st.mean = m[0] * inv_d;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = z[v][j] - st.mean;
        q[0] += cols.on(v, j) ? d * d : 0.f;
      }
    group_sum(q, red, turn, g, a.T);
    st.r = rsqrtf(q[0] * inv_d + a.eps);
    return st;
  };
  each_row<VEC, XT, BT>(a, smem, [&](int64_t row, const uint8_t *st, const RowPipe<VEC> &pipe) {
    float y[V][8];
    const float gate = a.flags & ALG_NORM_GATE_ROW ? to_f32(((const BT *)a.g)[row]) : 1.f;
#pragma unroll
    for (int v = 0; v < V; ++v) cols.load((const XT *)(st + pipe.at[0]), v, y[v]);
    if (a.flags & ALG_NORM_JOIN) {
      float f[V][8];
#pragma unroll
      for (int v = 0; v < V; ++v) cols.load((const BT *)(st + pipe.at[3]), v, f[v]);
      Stat sf = {0.f, 1.f};
      if (a.flags & ALG_NORM_POST) sf = stat(f);
      float gr = a.alpha;
      if (a.flags & ALG_NORM_GATE_ROW) gr *= a.flags & ALG_NORM_GATE_SIGMOID ? sigmoid(gate) : gate;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[v][j] = (f[v][j] - sf.mean) * sf.r;
        if (a.post_w) {
          cols.load(a.post_w, v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[v][j] *= w[j];
        }
        if (a.post_b) {
          cols.load(a.post_b, v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[v][j] += w[j];
        }
        if (a.scale) {
          cols.load(a.scale, v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[v][j] *= w[j];
        }
        if (a.flags & ALG_NORM_GATE_ELEMENT) {
          cols.load((const BT *)(st + pipe.at[4]), v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[v][j] *= a.flags & ALG_NORM_GATE_SIGMOID ? sigmoid(w[j]) : w[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] = fmaf(gr, f[v][j], y[v][j]);
        cols.store((XT *)a.y + row * a.ldy, v, y[v]);
      }
    }
    if (a.flags & ALG_NORM_PRE) {
      if ((a.flags & ALG_NORM_JOIN))   // (columns past the row's end hold nothing)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) y[v][j] = cols.on(v, j) ? y[v][j] : 0.f;
      const Stat sy = stat(y);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[v][j] = (y[v][j] - sy.mean) * sy.r;
        if (a.pre_w) {
          cols.load(a.pre_w, v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) y[v][j] *= w[j];
        }
        if (a.pre_b) {
          cols.load(a.pre_b, v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) y[v][j] += w[j];
        }
        cols.store((BT *)a.out + row * a.ldo, v, y[v]);
      }
    }
  });
}

template <typename XT, typename BT, bool VEC, int V>
__global__ void __launch_bounds__(512, 1) norm_backward_kernel(const NormArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  float4 *red = (float4 *)(smem + kBarBytes);
  const int g = threadIdx.x / a.T, t = threadIdx.x - g * a.T;
  const Cols<VEC> cols = {t, a.T, a.D};
  const float inv_d = 1.f / (float)a.D;
  const bool pre = a.flags & ALG_NORM_PRE, join = a.flags & ALG_NORM_JOIN, post = a.flags & ALG_NORM_POST;
  const bool sig = a.flags & ALG_NORM_GATE_SIGMOID, gate_row = a.flags & ALG_NORM_GATE_ROW, gate_el = a.flags & ALG_NORM_GATE_ELEMENT;
  float sum[kSums][V][8];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[k][v][j] = 0.f;
  int turn = 0;
  each_row<VEC, XT, BT>(a, smem, [&](int64_t row, const uint8_t *st, const RowPipe<VEC> &pipe) {
    const XT *x_row = (const XT *)(st + pipe.at[0]), *t_row = (const XT *)(st + pipe.at[1]);
    const BT *n_row = (const BT *)(st + pipe.at[2]), *f_row = (const BT *)(st + pipe.at[3]), *g_row = (const BT *)(st + pipe.at[4]);
    const float gate_1 = gate_row ? to_f32(((const BT *)a.g)[row]) : 1.f;
    // statistics of Y and F, and the means of h = dN * pre_weight and of h times the normed Y
    float mx = 0.f, mf = 0.f, mh = 0.f;
    if (a.layer) {
      float m[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float x[8], w[8];
        if (pre) {
          cols.load(x_row, v, x);
#pragma unroll
          for (int j = 0; j < 8; ++j) m[0] += x[j];
          cols.load(n_row, v, x);
          if (a.pre_w) {
            cols.load(a.pre_w, v, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= w[j];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) m[2] += x[j];
        }
        if (post) {
          cols.load(f_row, v, x);
#pragma unroll
          for (int j = 0; j < 8; ++j) m[1] += x[j];
        }
      }
      group_sum(m, red, turn, g, a.T);
      mx = m[0] * inv_d, mf = m[1] * inv_d, mh = m[2] * inv_d;
    }
    float q[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float x[8], h[8], w[8];
      if (pre) {
        cols.load(x_row, v, x, mx);
        cols.load(n_row, v, h);
        if (a.pre_w) {
          cols.load(a.pre_w, v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) h[j] *= w[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = x[j] - mx;
          q[0] = fmaf(d, d, q[0]);
          q[2] = fmaf(d, h[j], q[2]);
        }
      }
      if (post) {
        cols.load(f_row, v, x, mf);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = x[j] - mf;
          q[1] = fmaf(d, d, q[1]);
        }
      }
    }
    if (pre || post) group_sum(q, red, turn, g, a.T);
    const float rx = rsqrtf(q[0] * inv_d + a.eps), rf = post ? rsqrtf(q[1] * inv_d + a.eps) : 1.f;
    const float mhv = q[2] * inv_d * rx;
    // the row's gate and its slope
    const float gr = gate_row && sig ? sigmoid(gate_1) : gate_1, gs = sig ? gr * (1.f - gr) : 1.f;
    float e[V][8];   // gradient of V
    float m[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float d[8], x[8], h[8], w[8];
      if (a.t) {
        cols.load(t_row, v, d);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = 0.f;
      }
      if (pre) {
        cols.load(x_row, v, x, mx);
        cols.load(n_row, v, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = (x[j] - mx) * rx;
          sum[0][v][j] = fmaf(h[j], x[j], sum[0][v][j]);
          sum[1][v][j] += h[j];
        }
        if (a.pre_w) {
          cols.load(a.pre_w, v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) h[j] *= w[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = fmaf(rx, h[j] - mh - x[j] * mhv, d[j]);
      }
      cols.store((XT *)a.dr + row * a.lddr, v, d);
      if (!join) continue;
      cols.load(f_row, v, x, mf);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (x[j] - mf) * rf, d[j] *= cols.on(v, j) ? a.alpha : 0.f;
      float gate[8], slope[8];
      if (gate_el) {
        cols.load(g_row, v, gate);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (sig) gate[j] = sigmoid(gate[j]);
          slope[j] = sig ? gate[j] * (1.f - gate[j]) : 1.f;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) gate[j] = gr, slope[j] = 1.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = d[j] * gate[j];
        sum[2][v][j] = fmaf(u, x[j], sum[2][v][j]);
        sum[3][v][j] += u;
      }
      if (a.scale) {
        cols.load(a.scale, v, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] *= w[j];
      }
      // d = T * scale from here on
      if (a.post_w) {
        cols.load(a.post_w, v, w);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 1.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) e[v][j] = d[j] * gate[j] * w[j];
      if (gate_row || (gate_el && a.dg)) {
        float b[8];
        if (a.post_b) {
          cols.load(a.post_b, v, b);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) b[j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = d[j] * fmaf(x[j], w[j], b[j]);
        if (gate_el) {
#pragma unroll
          for (int j = 0; j < 8; ++j) b[j] *= slope[j];
          cols.store((BT *)a.dg + row * a.lddg, v, b);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) m[2] += b[j];
        }
      }
      if (post) {
#pragma unroll
        for (int j = 0; j < 8; ++j) m[0] += e[v][j], m[1] = fmaf(e[v][j], x[j], m[1]);
      } else if (a.df) {
        cols.store((BT *)a.df + row * a.lddf, v, e[v]);
      }
    }
    if (!join || !((post && a.df) || (gate_row && a.dg))) return;
    group_sum(m, red, turn, g, a.T);
    if (gate_row && a.dg && t == 0) from_f32(m[2] * gs, (BT *)a.dg + row);
    if (!post || !a.df) return;
    const float me = a.layer ? m[0] * inv_d : 0.f, mev = m[1] * inv_d;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float x[8];
      cols.load(f_row, v, x, mf);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = rf * (e[v][j] - me - (x[j] - mf) * rf * mev);
      cols.store((BT *)a.df + row * a.lddf, v, x);
    }
  });
  if (!a.part) return;
  // the groups' sums meet, group after group, where the rows were (a row's bytes suffice: see the launcher)
  __syncthreads();
  float *acc = (float *)(smem + kRowsAt);
  float *part = a.part + (size_t)blockIdx.x * kSums * a.D;
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    if (k < 2 ? !pre : !join) continue;
    for (int turn_g = 0; turn_g < a.G; ++turn_g) {
      if (g == turn_g) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (cols.on(v, j)) {
              const int c = cols.at(v, j);
              const float s = (turn_g ? acc[c] : 0.f) + sum[k][v][j];
              if (turn_g + 1 < a.G) acc[c] = s;
              else part[(size_t)k * a.D + c] = s;
            }
      }
      __syncthreads();
    }
  }
}

struct SumsArgs {
  int ctas, D, flags;
  float alpha;
  const float *part, *post_w, *post_b, *scale;
  float *d_post_w, *d_post_b, *d_scale, *d_pre_w, *d_pre_b;
};
// 32 columns a CTA, eight slices of the CTAs' sums.
__global__ void __launch_bounds__(256) norm_sums_kernel(const SumsArgs a) {
  __shared__ float slice[kSums][8][32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  float s[kSums] = {0.f, 0.f, 0.f, 0.f};
  if (c < a.D)
    for (int i = y; i < a.ctas; i += 8) {
      const float *p = a.part + (size_t)i * kSums * a.D + c;
      if (a.flags & ALG_NORM_PRE) s[0] += p[0], s[1] += p[a.D];
      if (a.flags & ALG_NORM_JOIN) s[2] += p[2 * (size_t)a.D], s[3] += p[3 * (size_t)a.D];
    }
#pragma unroll
  for (int k = 0; k < kSums; ++k) slice[k][y][x] = s[k];
  __syncthreads();
  if (y || c >= a.D) return;
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    s[k] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s[k] += slice[k][i][x];
  }
  const float scale = a.scale ? a.scale[c] : 1.f, w = a.post_w ? a.post_w[c] : 1.f, b = a.post_b ? a.post_b[c] : 0.f;
  if (a.d_pre_w) a.d_pre_w[c] = s[0];
  if (a.d_pre_b) a.d_pre_b[c] = s[1];
  if (a.d_post_w) a.d_post_w[c] = scale * s[2];   // (alpha is in the sums)
  if (a.d_post_b) a.d_post_b[c] = scale * s[3];
  if (a.d_scale) a.d_scale[c] = fmaf(w, s[2], b * s[3]);
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

constexpr int kSmemMax = kRowsAt + kStageBudget;

template <bool BACK, typename XT, typename BT, bool VEC, int V>
cudaError_t launch_rows(NormArgs &a, int grid, size_t smem, cudaStream_t st) {
  static OncePerDevice once;
  const void *k = BACK ? (const void *)norm_backward_kernel<XT, BT, VEC, V> : (const void *)norm_forward_kernel<XT, BT, VEC, V>;
  const cudaError_t e = once([&] { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax); });
  if (e != cudaSuccess) return e;
  void *params[] = {&a};
  return launch_pdl(k, grid, a.T * a.G, smem, st, params);
}
template <bool BACK, typename XT, typename BT>
cudaError_t launch_typed(NormArgs &a, bool vec, int grid, size_t smem, cudaStream_t st) {
  if (a.D <= 4096) return vec ? launch_rows<BACK, XT, BT, true, 1>(a, grid, smem, st) : launch_rows<BACK, XT, BT, false, 1>(a, grid, smem, st);
  return vec ? launch_rows<BACK, XT, BT, true, 2>(a, grid, smem, st) : launch_rows<BACK, XT, BT, false, 2>(a, grid, smem, st);
}

// Threads of a row, rows a CTA works on at once, rows on their way; the grid.
int shape_rows(const alg_norm_s &h, NormArgs &a, bool back, size_t *smem) {
  const int pieces = ((a.D + 7) / 8 + (a.D > 4096 ? 1 : 0)) / (a.D > 4096 ? 2 : 1);
  a.T = (pieces + 31) / 32 * 32;
  const size_t ex = elem_size(h.stream_dtype), eb = elem_size(h.dtype);
  const auto row = [&](size_t e) { return ((size_t)a.D * e + 15) / 16 * 16; };
  size_t stage = row(ex) * ((a.x ? 1 : 0) + (a.t ? 1 : 0));
  stage += row(eb) * ((a.n ? 1 : 0) + (a.f ? 1 : 0) + (a.g && (a.flags & ALG_NORM_GATE_ELEMENT) ? 1 : 0));
  const int threads = back || a.D > 4096 ? 512 : 1024;
  int groups = threads / a.T;
  if (groups > kMaxGroups) groups = kMaxGroups;
  const int64_t per_sm = (a.M + h.num_sms - 1) / h.num_sms;
  if (groups > per_sm) groups = (int)per_sm;
  while (groups > 1 && groups * stage > (size_t)kStageBudget) --groups;
  a.G = groups;
  int stages = (int)((size_t)kStageBudget / (groups * stage));
  if (stages > kMaxStages) stages = kMaxStages;
  const int64_t rows = (a.M + (int64_t)groups * h.num_sms - 1) / ((int64_t)groups * h.num_sms);
  if (stages > rows) stages = (int)rows;
  a.stages = stages;
  size_t bytes = (size_t)groups * stages * stage;
  if (back && bytes < (size_t)a.D * 4) bytes = (size_t)a.D * 4;   // the groups' sums meet there
  *smem = kRowsAt + bytes;
  const int64_t ctas = (a.M + groups - 1) / groups;
  return (int)(ctas < h.num_sms ? ctas : h.num_sms);
}

template <bool BACK>
cudaError_t launch_norm(const alg_norm_s &h, NormArgs &a, bool vec, int *grid, cudaStream_t st) {
  size_t smem = 0;
  *grid = shape_rows(h, a, BACK, &smem);
  if (h.stream_dtype == ALG_BF16)
    return h.dtype == ALG_BF16 ? launch_typed<BACK, __nv_bfloat16, __nv_bfloat16>(a, vec, *grid, smem, st)
                               : launch_typed<BACK, __nv_bfloat16, float>(a, vec, *grid, smem, st);
  return h.dtype == ALG_BF16 ? launch_typed<BACK, float, __nv_bfloat16>(a, vec, *grid, smem, st)
                             : launch_typed<BACK, float, float>(a, vec, *grid, smem, st);
}

// One matrix operand: its span, whether it is well formed, whether its rows lie on 16 bytes.
struct Operand {
  RowSpan s;
  bool ok, vec;
};
Operand operand(const void *p, int64_t ld, int64_t cols, size_t e, int64_t M) {
  if (!p) return {span(nullptr, 0, 0, 1, 0), true, true};
  return {span(p, ld, cols, e, M), ld >= cols && on_element(p, e), on_16(p, ld, e)};
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
  a.M = M, a.D = D, a.flags = h->flags, a.layer = h->kind == ALG_NORM_LAYER, a.eps = h->eps, a.alpha = alpha;
  a.x = R, a.ldx = ldr, a.f = F, a.ldf = ldf, a.g = gate, a.ldg = ldg;
  a.post_w = post_weight, a.post_b = post_bias, a.scale = scale, a.pre_w = pre_weight, a.pre_b = pre_bias;
  a.y = Y, a.ldy = ldy, a.out = N, a.ldo = ldn;
  a.status = h->d_status, a.wait_limit = kDefaultWaitLimit;
  int grid = 0;
  return launch_norm<false>(*h, a, vec, &grid, (cudaStream_t)stream) == cudaSuccess ? ALG_OK : ALG_ERR_CUDA;
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
    a.x = pre ? Y : nullptr, a.ldx = ldy;   // (Y is not needed without a norm behind it)
    a.t = dY, a.ldt = lddy;
    a.n = dN, a.ldn = lddn, a.f = F, a.ldf = ldf, a.g = gate, a.ldg = ldg;
  }
  if (!is_current(h->device)) return ALG_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  a.M = M, a.D = D, a.flags = h->flags, a.layer = h->kind == ALG_NORM_LAYER, a.eps = h->eps, a.alpha = alpha;
  a.post_w = post_weight, a.post_b = post_bias, a.scale = scale, a.pre_w = pre_weight;
  a.dr = dR, a.lddr = lddr, a.df = dF, a.lddf = lddf, a.dg = dgate, a.lddg = lddg;
  a.part = sums ? (float *)workspace : nullptr;
  a.status = h->d_status, a.wait_limit = kDefaultWaitLimit;
  int grid = 0;
  if (M > 0 && launch_norm<true>(*h, a, vec, &grid, st) != cudaSuccess) return ALG_ERR_CUDA;
  if (!sums) return ALG_OK;
  SumsArgs b = {grid, D, h->flags, alpha, a.part, post_weight, post_bias, scale, d_post_weight, d_post_bias, d_scale, d_pre_weight, d_pre_bias};
  void *params[] = {&b};
  return launch_pdl((const void *)norm_sums_kernel, (D + 31) / 32, 256, 0, st, params) == cudaSuccess ? ALG_OK : ALG_ERR_CUDA;
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
