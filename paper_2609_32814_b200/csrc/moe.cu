// Mixture of experts on up to 64 rows, in two launches.
//
// First launch: router, choice of the experts, gate and up products, silu(gate) * up * weight.  Second: down products and the
// sum over a row's experts.  Bound by HBM: every weight of a chosen expert is read once and used for all its rows.
//
// Router.  The CTAs of a thread-block cluster share the logits: each takes E / cluster experts and hands them to its peers through
// distributed shared memory.  Every cluster does that for itself (the router is read from L2), so no CTA waits for
// another cluster, and every CTA knows the choice without a launch of its own for it.
//
// Products.  A unit is 128 columns of one expert's bank (64 gate and the matching 64 up ones) or, for the down product, 128
// columns of Y over all chosen experts; its reduction is cut into chunks of 64 weight rows.  The chunks of all units in a row are
// dealt to the CTAs in equal consecutive shares, whatever the number of experts and rows.  A unit that lies in one CTA is finished there.
// The others leave their partial sums in the workspace, and whichever CTA counts itself the last of a unit adds them in CTA order (so the
// sums are the same every time) and finishes it: nobody waits.
//
// Weights come by tiled copies (64 x 64 boxes, 128-byte swizzle) through a ring of stages that one thread keeps full; eight warps
// multiply with mma.sync, weights as the 16-row operand, eight rows of X a step.  The tensor pipe has slack: at 16 KB in
// about 700 cycles a chunk needs 32 of its products per 8 rows.  A chunk's sums start at zero and are added to the unit's in
// fp32, so the length of the chains inside the tensor core does not grow with D.
#include <cfloat>
#include <cmath>
#include <new>

#include "common.cuh"
#include "rows.cuh"
#include "tc_common.cuh"

using namespace algproj;

struct alg_moe_s {
  int D = 0, F = 0, E = 0, k = 0;
  alg_moe_score_t score = ALG_MOE_SOFTMAX;
  bool renormalise = false;
  float route_scale = 1.f;
  alg_dtype_t router_dtype = ALG_BF16;
  int device = 0, num_sms = 148;
  int clusters = 0;           // of the first launch
  int *d_state = nullptr;     // status word, then the counters of both launches
  size_t state_bytes = 0;
};

namespace algproj {
namespace {

using namespace tc;

constexpr int kWarps = 8, kConsumers = kWarps * 32, kThreads = kConsumers + 32;
constexpr int kCluster = 4;
constexpr int kStages = 12;                 // at most
constexpr int kBox = 64 * 64 * 2;           // one box of weights
constexpr int kSmemLimit = 225 * 1024;
constexpr int kMaxM = ALG_MOE_MAX_M;
constexpr int kRouterRows = 4;              // rows of X at a time in the router's product

struct MoeArgs {
  int M, D, F, E, k, sigmoid, renormalise, y_f32, planes;
  float route_scale;
  const __nv_bfloat16 *X;
  int64_t ldx;
  const void *W_router;
  int router_f32, router_vec;
  const float *bias;
  int32_t *experts;
  float *weights;
  void *Y;
  int64_t ldy;
  int *route_idx;             // workspace: the choice, [M][k]
  float *route_w;
  __nv_bfloat16 *H;           // workspace: weighted hidden rows, [planes][M * k][F]
  float4 *part;               // workspace: partial sums, [CTA][2][8 warps][row tiles][32 lanes]
  int *count;                 // [CTA]: arrivals at the unit whose first contributor it is
  int *status;
  long long wait_limit;
  int stages, stage_bytes;
  int off_ring;               // the ring; in front of it what `Routes` points to
};

// The rows' choice, turned round: who takes an expert.
struct Routes {
  int *idx;        // [M * k] experts of a row, -1 for none
  float *w;        // [M * k]
  uint2 *mask;     // [E] the rows that take an expert
  int *act;        // chosen experts in ascending order
  int *first;      // [chosen + 1] their first pair
  int *n_act;
  __device__ __forceinline__ Routes(uint8_t *p, int P, int E) {
    mask = (uint2 *)p, p += (size_t)E * 8;
    idx = (int *)p, p += (size_t)P * 4;
    w = (float *)p, p += (size_t)P * 4;
    act = (int *)p, p += (size_t)E * 4;
    first = (int *)p, p += (size_t)(E + 1) * 4;
    n_act = (int *)p;
  }
  static size_t bytes(int P, int E) { return (size_t)E * 16 + (size_t)P * 8 + 8; }
};
__device__ __forceinline__ int rows_of(uint2 m) { return __popc(m.x) + __popc(m.y); }
// Rows below `row` that take the expert.
__device__ __forceinline__ int rows_below(uint2 m, int row) {
  return row < 32 ? __popc(m.x & ((1u << row) - 1u)) : __popc(m.x) + __popc(m.y & ((1u << (row - 32)) - 1u));
}
__device__ __forceinline__ bool takes(uint2 m, int row) { return (row < 32 ? m.x >> row : m.y >> (row - 32)) & 1u; }
__device__ __forceinline__ int nth_row(uint2 m, int n) {   // n < rows_of(m)
  const int lo = __popc(m.x);
  uint32_t w = n < lo ? m.x : m.y;
  for (int i = n < lo ? n : n - lo; i > 0; --i) w &= w - 1u;
  return __ffs(w) - 1 + (n < lo ? 0 : 32);
}

// From r.idx; all threads of the CTA.
__device__ void turn_round(const Routes &r, int P, int E, int k) {
  const int tid = threadIdx.x;
  for (int e = tid; e < E; e += kThreads) r.mask[e] = make_uint2(0u, 0u);
  __syncthreads();
  for (int p = tid; p < P; p += kThreads) {
    const int e = r.idx[p], m = p / k;
    if (e >= 0) atomicOr(m < 32 ? &r.mask[e].x : &r.mask[e].y, 1u << (m & 31));
  }
  __syncthreads();
  if (tid < 32) {
    int n = 0, pairs = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
      const int e = e0 + tid, c = e < E ? rows_of(r.mask[e]) : 0;
      const uint32_t used = __ballot_sync(~0u, c > 0);
      int sum = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(~0u, sum, o);
        if (tid >= o) sum += v;
      }
      const int at = n + __popc(used & ((1u << tid) - 1u));
      if (c > 0) r.act[at] = e, r.first[at] = pairs + sum - c;
      n += __popc(used);
      pairs += __shfl_sync(~0u, sum, 31);
    }
    if (tid == 0) r.first[n] = pairs, *r.n_act = n;
  }
  __syncthreads();
}

__device__ __forceinline__ void consumer_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Eight columns of the router, zero past the end.
__device__ __forceinline__ void router8(const MoeArgs &a, int k, int e, int end, float (&w)[8]) {
  if (a.router_vec) {
    if (a.router_f32) {
      Raw8<float> r;
      r.load((const float *)a.W_router + (size_t)k * a.E + e);
      r.get(w);
    } else {
      Raw8<__nv_bfloat16> r;
      r.load((const __nv_bfloat16 *)a.W_router + (size_t)k * a.E + e);
      r.get(w);
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    w[c] = 0.f;
    if (e + c < end)
      w[c] = a.router_f32 ? ((const float *)a.W_router)[(size_t)k * a.E + e + c]
                          : __bfloat162float(((const __nv_bfloat16 *)a.W_router)[(size_t)k * a.E + e + c]);
  }
}

// Logits of all rows, [M][E], in every CTA of the cluster.  Eight columns a lane, eight rows of the router a step; the lanes of
// a column group and the warps split D.
__device__ void router_logits(const MoeArgs &a, float *logits, float *red) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int per = ((a.E + kCluster - 1) / kCluster + 7) / 8 * 8;
  const int e0 = (int)cluster_rank() * per, en = max(0, min(per, a.E - e0));
  int groups = 1;
  while (groups * 8 < en) groups *= 2;
  const int slots = 32 / groups, cg = lane & (groups - 1), slot = lane / groups;
  const bool on = cg * 8 < en;
  if (warp < kWarps && en > 0) {
    for (int m0 = 0; m0 < a.M; m0 += kRouterRows) {
      float acc[kRouterRows][8];
#pragma unroll
      for (int m = 0; m < kRouterRows; ++m)
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[m][c] = 0.f;
      if (on)
        for (int k0 = (warp * slots + slot) * 8; k0 < a.D; k0 += kWarps * slots * 8) {
          float x[kRouterRows][8];
#pragma unroll
          for (int m = 0; m < kRouterRows; ++m) {
            Raw8<__nv_bfloat16> r;
            if (m0 + m < a.M) r.load(a.X + (int64_t)(m0 + m) * a.ldx + k0);
            else r.zero();
            r.get(x[m]);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float w[8];
            router8(a, k0 + i, e0 + cg * 8, e0 + en, w);
#pragma unroll
            for (int m = 0; m < kRouterRows; ++m)
#pragma unroll
              for (int c = 0; c < 8; ++c) acc[m][c] = fmaf(x[m][i], w[c], acc[m][c]);
          }
        }
      for (int o = groups; o < 32; o <<= 1)
#pragma unroll
        for (int m = 0; m < kRouterRows; ++m)
#pragma unroll
          for (int c = 0; c < 8; ++c) acc[m][c] += __shfl_xor_sync(~0u, acc[m][c], o);
      if (slot == 0 && on)
#pragma unroll
        for (int m = 0; m < kRouterRows; ++m)
#pragma unroll
          for (int c = 0; c < 8; ++c) red[(warp * kRouterRows + m) * per + cg * 8 + c] = acc[m][c];
      consumer_barrier();
      for (int i = tid; i < kRouterRows * en; i += kConsumers) {
        const int m = i / en, c = i - m * en;
        if (m0 + m < a.M) {
          float s = 0.f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) s += red[(w * kRouterRows + m) * per + c];
          const uint32_t dst = smem_u32(logits + (size_t)(m0 + m) * a.E + e0 + c);
#pragma unroll
          for (uint32_t p = 0; p < kCluster; ++p) {
            uint32_t there;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(dst), "r"(p));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(s) : "memory");
          }
        }
      }
      consumer_barrier();
    }
  }
}

// A warp chooses the experts of row m.  Without a bias the order is that of the logits, which a score that underflows or saturates
// cannot spoil.
__device__ void choose(const MoeArgs &a, const float *logits, const Routes &r, int m) {
  constexpr int kMost = ALG_MOE_MAX_EXPERTS / 32;
  const int lane = threadIdx.x & 31;
  float l[kMost], key[kMost];
  bool bad = false;
  float top = -FLT_MAX;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int e = lane + 32 * i;
    l[i] = e < a.E ? logits[(size_t)m * a.E + e] : 0.f;
    bad = bad || !isfinite(l[i]);
    if (e < a.E) top = fmaxf(top, l[i]);
  }
  bad = __any_sync(~0u, bad);
#pragma unroll
  for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
  float sum = 1.f;
  if (!a.sigmoid) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kMost; ++i)
      if (lane + 32 * i < a.E) sum += expf(l[i] - top);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  }
  auto score = [&](float x) { return a.sigmoid ? 1.f / (1.f + expf(-x)) : expf(x - top) / sum; };
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int e = lane + 32 * i;
    key[i] = -INFINITY;
    if (e < a.E) {
      key[i] = a.bias ? score(l[i]) + a.bias[e] : l[i];
      key[i] = key[i] == key[i] ? key[i] + 0.f : -INFINITY;   // (-0 is 0)
    }
  }
  int mine = -1;      // lane j keeps the j-th choice
  float w = 0.f;
  for (int j = 0; j < a.k && !bad; ++j) {
    float best = -INFINITY, at = 0.f;
    int e = 0x7FFFFFFF;
#pragma unroll
    for (int i = 0; i < kMost; ++i)
      if (key[i] > best) best = key[i], e = lane + 32 * i, at = l[i];
    const uint32_t bits = __float_as_uint(best), order = bits >> 31 ? ~bits : bits | 0x80000000u;
    const uint32_t most = __reduce_max_sync(~0u, order);
    const int win = (int)__reduce_min_sync(~0u, order == most ? (uint32_t)e : 0x7FFFFFFFu);
    if (win == 0x7FFFFFFF) break;   // nothing left to choose
    at = __shfl_sync(~0u, at, win & 31);
#pragma unroll
    for (int i = 0; i < kMost; ++i)
      if (lane + 32 * i == win) key[i] = -INFINITY;
    if (lane == j) mine = win, w = score(at);
  }
  if (a.renormalise) {
    float s = w;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    w /= fmaxf(s, 1e-20f);
  }
  w = bad ? __uint_as_float(0x7FC00000u) : w * a.route_scale;
  if (lane < a.k) {
    r.idx[m * a.k + lane] = mine;
    r.w[m * a.k + lane] = w;
  }
}

// ---- the ring ----------------------------------------------------------------------------------------------------------

struct Ring {
  uint32_t full, empty;   // shared addresses of the barriers
  uint32_t base;
  int stages, stage_bytes;
  int s = 0;
  uint32_t parity = 0;
  bool failed = false;
  __device__ __forceinline__ uint32_t stage() const { return base + s * stage_bytes; }
  __device__ __forceinline__ void next() {
    if (++s == stages) s = 0, parity ^= 1;
  }
  // After a wait that ran out nothing is right, but everybody still goes the same way to the end.
  __device__ __forceinline__ bool wait(uint32_t bar, uint32_t par, const MoeArgs &a) {
    if (mbar_try_wait(bar, par)) return true;
    if (failed) return false;
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, par))
      if (clock64() - t0 > a.wait_limit) {
        failed = true;
        atomicExch(a.status, (int)ALG_ERR_DEVICE_TIMEOUT);
        return false;
      }
    return true;
  }
  __device__ __forceinline__ bool wait_full(const MoeArgs &a) { return wait(full + 8 * s, parity, a); }
  __device__ __forceinline__ bool wait_empty(const MoeArgs &a) { return wait(empty + 8 * s, parity ^ 1, a); }
};
__device__ __forceinline__ Ring make_ring(const MoeArgs &a, uint8_t *smem, uint64_t *bars) {
  Ring r;
  r.full = smem_u32(bars), r.empty = r.full + 8 * kStages;
  r.base = smem_u32(smem + a.off_ring);
  r.stages = a.stages, r.stage_bytes = a.stage_bytes;
  return r;
}
__device__ __forceinline__ void init_ring(uint64_t *bars, int stages) {   // one thread
  const uint32_t full = smem_u32(bars), empty = full + 8 * kStages;
  for (int s = 0; s < stages; ++s) mbar_init(full + 8 * s, 1), mbar_init(empty + 8 * s, kWarps);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&w)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(b0), "r"(b1));
}
// Weights of a chunk, 16 columns of the warp by 64 rows: lanes 0-15 address rows 0-7 of the first and of the second eight
// columns, lanes 16-31 rows 8-15; `lo` and `hi`: boxes and byte columns of the two eights.
__device__ __forceinline__ void load_weights(uint32_t box, int byte_col, uint32_t (&w)[4][4]) {
  const int lane = threadIdx.x & 31, row = (lane & 7) + (lane >> 4 << 3);
  const uint32_t at = box + row * 128 + (byte_col ^ ((row & 7) << 4));
#pragma unroll
  for (int k = 0; k < 4; ++k) ldmatrix4_trans(at + k * 16 * 128, w[k]);
}

// The share of CTA c of n among `total` chunks, and whose share a chunk is in; n <= total, so that nobody's is empty (CTAs past n have none).
__device__ __forceinline__ int64_t share(int64_t total, int c, int n) { return total * c / n; }
__device__ __forceinline__ int owner(int64_t total, int64_t chunk, int n) { return (int)(((chunk + 1) * n - 1) / total); }

// The sums of a unit that several CTAs have parts of: leaves this CTA's and, in the last to come, adds all of them in CTA order.
// True in that CTA.  All consumers.
template <int NT>
__device__ bool meet_parts(const MoeArgs &a, float (&acc)[NT][4], int nt, int64_t total, int n, int per_unit, int64_t unit, int *flag) {
  const int me = blockIdx.x, tiles = (a.M + 7) / 8;
  const int c0 = owner(total, unit * per_unit, n), c1 = owner(total, (unit + 1) * per_unit - 1, n);
  if (c0 == c1) return true;
  const size_t warp_at = (size_t)(threadIdx.x >> 5) * tiles * 32 + (threadIdx.x & 31), slot = (size_t)kWarps * tiles * 32;
  auto part_of = [&](int c) {   // a CTA has at most two units it shares: the first and the last of its share
    const bool first = share(total, c, n) / per_unit == unit;
    return a.part + ((size_t)c * 2 + (first ? 0 : 1)) * slot + warp_at;
  };
  float4 *mine = part_of(me);
#pragma unroll
  for (int t = 0; t < NT; ++t)
    if (t < nt) __stcg(mine + t * 32, make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]));
  __threadfence();
  consumer_barrier();
  if (threadIdx.x == 0) {
    const bool last = atomicAdd(a.count + c0, 1) == c1 - c0;
    if (last) a.count[c0] = 0;   // as the next launch finds it
    *flag = last;
  }
  consumer_barrier();
  const bool last = *flag;
  consumer_barrier();
  if (!last) return false;
  __threadfence();
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.f;
  for (int c = c0; c <= c1; ++c) {
    const float4 *p = part_of(c);
#pragma unroll
    for (int t = 0; t < NT; ++t)
      if (t < nt) {
        const float4 v = __ldcg(p + t * 32);
        acc[t][0] += v.x, acc[t][1] += v.y, acc[t][2] += v.z, acc[t][3] += v.w;
      }
  }
  return true;
}

// ---- first launch ------------------------------------------------------------------------------------------------------

template <int NT>   // row tiles of eight: ceil(M / 8) at most
__global__ void __launch_bounds__(kThreads, 1)
moe_up_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const MoeArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ __align__(8) uint64_t bars[2 * kStages];
  __shared__ int flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, P = a.M * a.k;
  const Routes r(smem, P, a.E);
  if (tid == 0) init_ring(bars, a.stages);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  cluster_sync();   // the peers are there
  float *logits = (float *)(smem + a.off_ring), *red = logits + (size_t)a.M * a.E;
  router_logits(a, logits, red);
  cluster_sync();
  if (warp < kWarps)
    for (int m = warp; m < a.M; m += kWarps) choose(a, logits, r, m);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int p = tid; p < P; p += kThreads) {
      a.route_idx[p] = r.idx[p], a.route_w[p] = r.w[p];
      if (a.experts) a.experts[p] = r.idx[p];
      if (a.weights) a.weights[p] = r.w[p];
    }
  fence_async_smem();   // the logits' memory belongs to the copies from here on
  turn_round(r, P, a.E, a.k);

  const int strips = (a.F + 63) / 64, per_unit = (a.D + 63) / 64;
  const int64_t total = (int64_t)*r.n_act * strips * per_unit;
  const int n = (int)min((int64_t)gridDim.x, total);
  if ((int)blockIdx.x >= n) return;
  const int64_t begin = share(total, blockIdx.x, n), end = share(total, blockIdx.x + 1, n);
  Ring ring = make_ring(a, smem, bars);
  int64_t unit = begin / per_unit;
  int chunk = (int)(begin - unit * per_unit);
  int x = (int)(unit / strips), strip = (int)(unit - (int64_t)x * strips);
  if (warp == kWarps) {
    if (lane == 0)
      for (int64_t i = begin; i < end; ++i) {
        if (!ring.wait_empty(a)) break;
        const uint32_t bar = ring.full + 8 * ring.s, st = ring.stage();
        mbar_expect_tx(bar, 2 * kBox + a.M * 128);
        tma_load_3d(st, &tm_w, bar, strip * 64, chunk * 64, r.act[x]);
        tma_load_3d(st + kBox, &tm_w, bar, a.F + strip * 64, chunk * 64, r.act[x]);
        tma_load_2d(st + 2 * kBox, &tm_x, bar, chunk * 64, 0);
        ring.next();
        if (++chunk == per_unit) {
          chunk = 0;
          if (++strip == strips) strip = 0, ++x;
        }
      }
    return;
  }
  for (int64_t i = begin; i < end; ++unit) {
    const uint2 mask = r.mask[r.act[x]];
    const int rows = rows_of(mask), nt = (rows + 7) / 8;
    float acc[NT][4];
    int x_row[NT];   // the row of X this lane addresses in each tile
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.f;
      x_row[t] = t < nt ? nth_row(mask, min(t * 8 + (lane & 7), rows - 1)) : 0;
    }
    for (; chunk < per_unit && i < end; ++chunk, ++i) {
      ring.wait_full(a);
      const uint32_t st = ring.stage(), xs = st + 2 * kBox;
      uint32_t w[4][4];
      // eight gate columns and the eight up columns that go with them
      load_weights(st + ((lane >> 3) & 1) * kBox, warp * 16, w);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (t >= nt) continue;
        const uint32_t at = xs + x_row[t] * 128;
        const int sw = (x_row[t] & 7) << 4;
        uint32_t b[4], c[4];
        ldmatrix4(at + (((lane >> 3) * 16) ^ sw), b);
        ldmatrix4(at + ((64 + (lane >> 3) * 16) ^ sw), c);
        float d[4] = {0.f, 0.f, 0.f, 0.f};
        mma(d, w[0], b[0], b[1]);
        mma(d, w[1], b[2], b[3]);
        mma(d, w[2], c[0], c[1]);
        mma(d, w[3], c[2], c[3]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][e] += d[e];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(ring.empty + 8 * ring.s);
      ring.next();
    }
    if (meet_parts<NT>(a, acc, nt, total, n, per_unit, unit, &flag)) {
      const int col = strip * 64 + warp * 8 + (lane >> 2);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = t * 8 + (lane & 3) * 2 + h;
          if (row >= rows || col >= a.F) continue;
          const int m = nth_row(mask, row), e = r.act[x];
          float w = 0.f;
          for (int j = 0; j < a.k; ++j)
            if (r.idx[m * a.k + j] == e) w = r.w[m * a.k + j];
          const float gate = acc[t][h], up = acc[t][2 + h];
          float v = __fdividef(gate, 1.f + __expf(-gate)) * up * w;
          __nv_bfloat16 *dst = a.H + (size_t)(r.first[x] + row) * a.F + col;
          for (int p = 0; p < a.planes; ++p) {
            const __nv_bfloat16 b = __float2bfloat16_rn(v);
            dst[(size_t)p * P * a.F] = b;
            const float back = __bfloat162float(b);
            v = isfinite(back) ? v - back : 0.f;
          }
        }
      }
    }
    chunk = 0;
    if (++strip == strips) strip = 0, ++x;
  }
}

// ---- second launch -----------------------------------------------------------------------------------------------------

template <int NT>
__global__ void __launch_bounds__(kThreads, 1)
moe_down_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_h, const MoeArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ __align__(8) uint64_t bars[2 * kStages];
  __shared__ int flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, P = a.M * a.k;
  const Routes r(smem, P, a.E);
  if (tid == 0) init_ring(bars, a.stages);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int p = tid; p < P; p += kThreads) r.idx[p] = a.route_idx[p], r.w[p] = a.route_w[p];
  __syncthreads();
  turn_round(r, P, a.E, a.k);
  const int n_act = *r.n_act;
  const int strips = (a.D + 127) / 128, per_expert = (a.F + 63) / 64, per_unit = n_act * per_expert;
  const int tiles = (a.M + 7) / 8;
  const int64_t total = (int64_t)strips * per_unit;
  const int n = (int)min((int64_t)gridDim.x, total);
  Ring ring = make_ring(a, smem, bars);
  // what the places without an expert add to a row: nothing, or NaN
  auto rest = [&](int m) {
    float s = 0.f;
    for (int j = 0; j < a.k; ++j)
      if (r.idx[m * a.k + j] < 0) s += r.w[m * a.k + j];
    return s;
  };
  auto put = [&](int m, int c, float v) {
    if (a.y_f32) ((float *)a.Y)[(int64_t)m * a.ldy + c] = v;
    else ((__nv_bfloat16 *)a.Y)[(int64_t)m * a.ldy + c] = __float2bfloat16_rn(v);
  };
  if (total == 0) {   // nobody takes an expert
    for (int i = blockIdx.x * kThreads + tid; i < a.M * a.D; i += gridDim.x * kThreads) put(i / a.D, i % a.D, rest(i / a.D));
    return;
  }
  if ((int)blockIdx.x >= n) return;
  const int64_t begin = share(total, blockIdx.x, n), end = share(total, blockIdx.x + 1, n);
  int64_t unit = begin / per_unit;
  int at = (int)(begin - unit * per_unit), x = at / per_expert, chunk = at - x * per_expert;
  const int plane_bytes = tiles * 1024;
  if (warp == kWarps) {
    if (lane == 0)
      for (int64_t i = begin; i < end; ++i) {
        if (!ring.wait_empty(a)) break;
        const uint32_t bar = ring.full + 8 * ring.s, st = ring.stage();
        const int strip = (int)unit, p0 = r.first[x], boxes = (r.first[x + 1] - p0 + 7) / 8;
        mbar_expect_tx(bar, 2 * kBox + a.planes * boxes * 1024);
        tma_load_3d(st, &tm_w, bar, strip * 128, chunk * 64, r.act[x]);
        tma_load_3d(st + kBox, &tm_w, bar, strip * 128 + 64, chunk * 64, r.act[x]);
        for (int p = 0; p < a.planes; ++p)
          for (int b = 0; b < boxes; ++b)
            tma_load_3d(st + 2 * kBox + p * plane_bytes + b * 1024, &tm_h, bar, chunk * 64, p0 + b * 8, p);
        ring.next();
        if (++chunk == per_expert) {
          chunk = 0;
          if (++x == n_act) x = 0, ++unit;
        }
      }
    return;
  }
  for (int64_t i = begin; i < end; ++unit) {
    float acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.f;
    for (; x < n_act && i < end; ++x, chunk = 0) {
      const uint2 mask = r.mask[r.act[x]];
      for (; chunk < per_expert && i < end; ++chunk, ++i) {
        ring.wait_full(a);
        const uint32_t st = ring.stage(), hs = st + 2 * kBox;
        uint32_t w[4][4];
        load_weights(st + (warp >> 2) * kBox, (warp & 3) * 32 + ((lane >> 3) & 1) * 16, w);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint32_t here = (t < 4 ? mask.x : mask.y) >> (8 * (t & 3)) & 255u;   // rows of the tile that take the expert
          if (!here) continue;
          const int m = t * 8 + (lane & 7), row = takes(mask, m) ? rows_below(mask, m) : 0;
          float d[4] = {0.f, 0.f, 0.f, 0.f};
          for (int p = 0; p < a.planes; ++p) {
            const uint32_t h = hs + p * plane_bytes + row * 128;
            const int sw = (row & 7) << 4;
            uint32_t b[4], c[4];
            ldmatrix4(h + (((lane >> 3) * 16) ^ sw), b);
            ldmatrix4(h + ((64 + (lane >> 3) * 16) ^ sw), c);
            mma(d, w[0], b[0], b[1]);
            mma(d, w[1], b[2], b[3]);
            mma(d, w[2], c[0], c[1]);
            mma(d, w[3], c[2], c[3]);
          }
          // (the other rows' columns hold whatever the stage did)
          if (here >> (2 * (lane & 3)) & 1u) acc[t][0] += d[0], acc[t][2] += d[2];
          if (here >> (2 * (lane & 3) + 1) & 1u) acc[t][1] += d[1], acc[t][3] += d[3];
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(ring.empty + 8 * ring.s);
        ring.next();
      }
      if (chunk < per_expert) break;   // the share ends inside the expert
    }
    x = 0, chunk = 0;
    if (meet_parts<NT>(a, acc, tiles, total, n, per_unit, unit, &flag)) {
      const int col = (int)unit * 128 + warp * 16 + (lane >> 2);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int m = t * 8 + (lane & 3) * 2 + (e & 1), c = col + (e >> 1) * 8;
          if (m < a.M && c < a.D) put(m, c, acc[t][e] + rest(m));
        }
    }
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------

int row_tiles(int64_t M) { return (int)((M + 7) / 8); }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

struct MoeLayout {
  size_t idx, w, h, part, total;
};
MoeLayout moe_layout(const alg_moe_s &h, int64_t M) {
  MoeLayout L;
  const size_t P = (size_t)M * h.k;
  size_t off = 0;
  L.idx = off, off = up256(off + P * 4);
  L.w = off, off = up256(off + P * 4);
  L.h = off, off = up256(off + 3 * P * h.F * 2);
  L.part = off, off = up256(off + (size_t)h.num_sms * 2 * kWarps * row_tiles(M) * 512);
  L.total = off;
  return L;
}

using MoeKernel = void (*)(const CUtensorMap, const CUtensorMap, const MoeArgs);
MoeKernel up_kernel(int tiles) {
  return tiles <= 1 ? moe_up_kernel<1> : tiles <= 2 ? moe_up_kernel<2> : tiles <= 4 ? moe_up_kernel<4> : moe_up_kernel<8>;
}
MoeKernel down_kernel(int tiles) {
  return tiles <= 1 ? moe_down_kernel<1> : tiles <= 2 ? moe_down_kernel<2> : tiles <= 4 ? moe_down_kernel<4> : moe_down_kernel<8>;
}
cudaError_t moe_attributes() {
  static OncePerDevice once;
  return once([] {
    for (int t : {1, 2, 4, 8})
      for (MoeKernel k : {up_kernel(t), down_kernel(t)}) {
        const cudaError_t e = cudaFuncSetAttribute((const void *)k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
        if (e != cudaSuccess) return e;
      }
    return cudaSuccess;
  });
}
// Ring behind the routes: as many stages as fit.
bool fit_ring(MoeArgs &a, int stage_bytes, size_t scratch, size_t *smem) {
  a.off_ring = (int)((Routes::bytes(a.M * a.k, a.E) + 1023) / 1024 * 1024);
  a.stage_bytes = stage_bytes;
  a.stages = (kSmemLimit - 1024 - a.off_ring) / stage_bytes;
  if (a.stages > kStages) a.stages = kStages;
  size_t ring = (size_t)a.stages * stage_bytes;
  if (ring < scratch) ring = scratch;
  *smem = 1024 + a.off_ring + ring;   // (the kernels align their part to the swizzle)
  return a.stages >= 2 && *smem <= (size_t)kSmemLimit;
}

cudaError_t launch_moe(MoeKernel k, const CUtensorMap &tm_w, const CUtensorMap &tm_b, const MoeArgs &a, int grid, int cluster, size_t smem,
                       cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k, tm_w, tm_b, a);
  if (e == cudaSuccess) count_launch(1);
  return e;
}

}  // namespace
}  // namespace algproj

extern "C" {

alg_status_t alg_moe_create(alg_moe_t *out, int D, int F, int E, int top_k, alg_moe_score_t score, int renormalise, float route_scale,
                            alg_dtype_t router_dtype) {
  if (!out) return ALG_ERR_INVALID_ARG;
  *out = nullptr;
  if (D < 1 || F < 1 || E < 1 || top_k < 1 || top_k > E || (score != ALG_MOE_SOFTMAX && score != ALG_MOE_SIGMOID) || !std::isfinite(route_scale) ||
      (router_dtype != ALG_F32 && router_dtype != ALG_BF16))
    return ALG_ERR_INVALID_ARG;
  if (D % 8 || F % 8 || D > (1 << 20) || F > (1 << 20) || E > ALG_MOE_MAX_EXPERTS || top_k > ALG_MOE_MAX_TOP_K) return ALG_ERR_UNSUPPORTED_SHAPE;
  int dev = 0, sms = 0;
  alg_status_t s = kernel_device(&dev, &sms);
  if (s != ALG_OK) return s;
  if (tc_init() != cudaSuccess || moe_attributes() != cudaSuccess) return ALG_ERR_CUDA;
  alg_moe_s *h = new (std::nothrow) alg_moe_s();
  if (!h) return ALG_ERR_INVALID_ARG;
  h->D = D, h->F = F, h->E = E, h->k = top_k;
  h->score = score, h->renormalise = renormalise != 0, h->route_scale = route_scale, h->router_dtype = router_dtype;
  h->device = dev, h->num_sms = sms;
  // clusters that run at the same time with the largest shared memory a launch may ask for
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(sms / kCluster * kCluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmemLimit;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = kCluster, at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at, cfg.numAttrs = 1;
  h->state_bytes = up256((4 + 2 * (size_t)sms) * sizeof(int));
  if (cudaOccupancyMaxActiveClusters(&h->clusters, (const void *)up_kernel(8), &cfg) != cudaSuccess || h->clusters < 1 ||
      cudaMalloc(&h->d_state, h->state_bytes) != cudaSuccess || cudaMemset(h->d_state, 0, h->state_bytes) != cudaSuccess ||
      cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess) {
    if (h->d_state) cudaFree(h->d_state);
    delete h;
    return ALG_ERR_CUDA;
  }
  if (h->clusters > sms / kCluster) h->clusters = sms / kCluster;
  *out = h;
  return ALG_OK;
}

alg_status_t alg_moe_destroy(alg_moe_t h) {
  if (!h) return ALG_ERR_INVALID_ARG;
  cudaFree(h->d_state);
  delete h;
  return ALG_OK;
}

alg_status_t alg_moe_workspace_bytes(alg_moe_t h, int64_t max_M, size_t *bytes) {
  if (!h || !bytes || max_M < 0 || max_M > kMaxM) return ALG_ERR_INVALID_ARG;
  *bytes = moe_layout(*h, max_M).total;
  return ALG_OK;
}

alg_status_t alg_moe_forward(alg_moe_t h, const void *X, int64_t ldx, int64_t M, const void *W_router, const float *select_bias,
                             const void *W_gate_up, const void *W_down, void *Y, int64_t ldy, alg_dtype_t y_dtype, int32_t *experts, float *weights,
                             void *workspace, size_t workspace_bytes, void *stream) {
  if (!h || M < 0) return ALG_ERR_INVALID_ARG;
  if (M == 0) return ALG_OK;
  if (M > kMaxM) return ALG_ERR_UNSUPPORTED_SHAPE;
  if (!X || !W_router || !W_gate_up || !W_down || !Y || !workspace || (y_dtype != ALG_F32 && y_dtype != ALG_BF16)) return ALG_ERR_INVALID_ARG;
  const size_t ey = elem_size(y_dtype), er = elem_size(h->router_dtype);
  if (ldx < h->D || ldy < h->D || !on_16(X, ldx, 2) || !on_16(Y, ldy, ey) || !on_16(W_gate_up, 0, 2) || !on_16(W_down, 0, 2) ||
      !on_element(W_router, er) || !on_element(select_bias, 4) || !on_element(experts, 4) || !on_element(weights, 4) || ((uintptr_t)workspace & 255u))
    return ALG_ERR_INVALID_ARG;
  const MoeLayout L = moe_layout(*h, M);
  if (workspace_bytes < L.total) return ALG_ERR_WORKSPACE_TOO_SMALL;
  const int64_t P = M * h->k, bank = (int64_t)h->D * h->F;
  const auto flat = [](const void *p, size_t bytes) { return span(p, (int64_t)bytes, (int64_t)bytes, 1, 1); };
  const RowSpan out[4] = {span(Y, ldy, h->D, ey, M), flat(experts, P * 4), flat(weights, P * 4), flat(workspace, L.total)};
  const RowSpan in[5] = {span(X, ldx, h->D, 2, M), flat(W_router, (size_t)h->D * h->E * er), flat(select_bias, (size_t)h->E * 4),
                         flat(W_gate_up, (size_t)h->E * 2 * bank * 2), flat(W_down, (size_t)h->E * bank * 2)};
  for (int o = 0; o < 4; ++o) {
    for (const RowSpan &i : in)
      if (meet(out[o], i)) return ALG_ERR_INVALID_ARG;
    for (int p = 0; p < o; ++p)
      if (meet(out[o], out[p])) return ALG_ERR_INVALID_ARG;
  }
  if (!is_current(h->device)) return ALG_ERR_INVALID_ARG;
  char *ws = (char *)workspace;
  MoeArgs a = {};
  a.M = (int)M, a.D = h->D, a.F = h->F, a.E = h->E, a.k = h->k;
  a.sigmoid = h->score == ALG_MOE_SIGMOID, a.renormalise = h->renormalise, a.route_scale = h->route_scale;
  a.y_f32 = y_dtype == ALG_F32, a.planes = a.y_f32 ? 3 : 2;
  a.X = (const __nv_bfloat16 *)X, a.ldx = ldx;
  a.W_router = W_router, a.router_f32 = h->router_dtype == ALG_F32, a.router_vec = h->E % 8 == 0 && on_16(W_router, h->E, er);
  a.bias = select_bias, a.experts = experts, a.weights = weights;
  a.Y = Y, a.ldy = ldy;
  a.route_idx = (int *)(ws + L.idx), a.route_w = (float *)(ws + L.w);
  a.H = (__nv_bfloat16 *)(ws + L.h), a.part = (float4 *)(ws + L.part);
  a.status = h->d_state, a.wait_limit = kDefaultWaitLimit;

  const int tiles = row_tiles(M);
  CUtensorMap tm_up, tm_x, tm_down, tm_h;
  {
    const uint64_t d[3] = {(uint64_t)2 * h->F, (uint64_t)h->D, (uint64_t)h->E}, s[2] = {(uint64_t)4 * h->F, (uint64_t)4 * bank};
    const uint32_t b[3] = {64, 64, 1};
    if (make_map_nd(&tm_up, W_gate_up, 3, d, s, b, 128) != cudaSuccess) return ALG_ERR_CUDA;
    const uint64_t dd[3] = {(uint64_t)h->D, (uint64_t)h->F, (uint64_t)h->E}, sd[2] = {(uint64_t)2 * h->D, (uint64_t)2 * bank};
    if (make_map_nd(&tm_down, W_down, 3, dd, sd, b, 128) != cudaSuccess) return ALG_ERR_CUDA;
    const uint64_t dx[2] = {(uint64_t)h->D, (uint64_t)M}, sx[1] = {(uint64_t)ldx * 2};
    const uint32_t bx[2] = {64, (uint32_t)M};
    if (make_map_nd(&tm_x, X, 2, dx, sx, bx, 128) != cudaSuccess) return ALG_ERR_CUDA;
    const uint64_t dh[3] = {(uint64_t)h->F, (uint64_t)P, 3}, sh[2] = {(uint64_t)2 * h->F, (uint64_t)2 * P * h->F};
    const uint32_t bh[3] = {64, 8, 1};
    if (make_map_nd(&tm_h, a.H, 3, dh, sh, bh, 128) != cudaSuccess) return ALG_ERR_CUDA;
  }
  cudaStream_t st = (cudaStream_t)stream;
  size_t smem = 0;
  const int per = ((h->E + kCluster - 1) / kCluster + 7) / 8 * 8;
  if (!fit_ring(a, 2 * kBox + tiles * 1024, ((size_t)M * h->E + (size_t)kWarps * kRouterRows * per) * 4, &smem)) return ALG_ERR_UNSUPPORTED_SHAPE;
  a.count = h->d_state + 4;
  if (launch_moe(up_kernel(tiles), tm_up, tm_x, a, h->clusters * kCluster, kCluster, smem, st) != cudaSuccess) return ALG_ERR_CUDA;
  if (!fit_ring(a, 2 * kBox + a.planes * tiles * 1024, 0, &smem)) return ALG_ERR_UNSUPPORTED_SHAPE;
  a.count = h->d_state + 4 + h->num_sms;
  return launch_moe(down_kernel(tiles), tm_down, tm_h, a, h->num_sms, 1, smem, st) == cudaSuccess ? ALG_OK : ALG_ERR_CUDA;
}

alg_status_t alg_moe_last_status(alg_moe_t h, void *stream, alg_status_t *status) {
  if (!h || !status) return ALG_ERR_INVALID_ARG;
  int v = 0;
  if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess || cudaMemcpy(&v, h->d_state, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess)
    return ALG_ERR_CUDA;
  if (v && (cudaMemset(h->d_state, 0, h->state_bytes) != cudaSuccess || cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess)) return ALG_ERR_CUDA;
  *status = (alg_status_t)v;
  return ALG_OK;
}

}  // extern "C"
