// Mixture of experts on up to 64 rows, in two launches.
//
// First launch: router, choice of the experts, gate and up products, silu(gate) * up * weight.  Second: down products and the
// sum over a row's experts.  Bound by HBM: every weight of a chosen expert is read once and used for all its rows.
//
// Router.  The CTAs of a thread-block cluster share the logits: each reduces over an eighth of D (a quarter, for half of more than 256
// experts), adds up its peers' parts of every eighth row through distributed shared memory, chooses that row's experts and
// tells its peers.  Every cluster does that for itself (the router is read from L2), so no CTA waits for another cluster, and every CTA
// knows the choice without a launch of its own for it.  An fp32 router is taken as three bf16 terms, which hold all its bits.
//
// Products.  A unit is 128 gate and the matching 128 up columns of one expert's bank, reduced over D in chunks of 64 weight rows or, for
// the down product, 128 columns of Y over all chosen experts in chunks of 128 (32 KB either way).  The chunks of all units in a row
// are dealt to the CTAs in equal consecutive shares, whatever the number of experts and rows.  A unit that lies in one CTA is finished
// there.  The others leave their partial sums in the workspace, and whichever CTA counts itself the last of a unit adds them in CTA
// order (so the sums are the same every time) and finishes it: nobody waits.  Down sums are kept in shared memory by row of Y, so
// that a product's steps of eight rows are full of the rows that take the expert at hand (40 rows, 128 experts: 2.7 rows, one step instead of
// the 2.1 that hold them) and the parts that meet are no larger than Y.
//
// Weights come by tiled copies (boxes of 64 columns, 128-byte swizzle) through a ring of stages.  What limits such a stream is the
// thread that asks for it, about 150 cycles a copy: with 16 KB in two copies 5.5 TB/s, 32 KB in one copy 6.6 to 7.1 (gate and up
// boxes of two column blocks are one 5-D box), 8 KB rows 3.5.  So one warp asks for weights, another for the rows they
// multiply.  Eight warps multiply with mma.sync, weights as the 16-row operand, eight rows a step; a chunk's sums start at zero and are
// added to the unit's in fp32, so the length of the chains inside the tensor core does not grow with D.
//
// Measured: 40 tokens, 8 of 128 experts of 2048 x 768 206 us (1.12 GB, 5.4 TB/s), 5 tokens, 6 of 64 of 4096 x 1536 140 us (6.7 TB/s), one
// token, 8 of 128 of 2048 x 768 31 us (75.5 MB are 12 us: router, choice, the launches' border and the joins of partial sums are 20 us).
#include <cfloat>
#include <cmath>
#include <new>
#include <type_traits>

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
  long long wait_limit = kDefaultWaitLimit;
  uint32_t stall = 0;
  size_t state_bytes = 0;
};

namespace algproj {
namespace {

using namespace tc;

constexpr int kWarps = 8, kConsumers = kWarps * 32, kThreads = kConsumers + 64;   // two warps fetch
constexpr int kCluster = 8;
constexpr int kStages = 6;                  // at most
constexpr int kBox = 64 * 64 * 2;           // 64 columns of 64 rows of weights
constexpr int kChunk = 4 * kBox;            // up: [column block][gate, up][64 rows]; down: [column block][128 rows]
constexpr int kCols = 128;                  // of a unit (up: of the hidden state)
constexpr int kUpPitch = 2 * kCols + 4, kDownPitch = kCols + 4;   // floats of a row of sums in shared memory
constexpr int kAhead = 6;                   // chunks of a share of the second launch that the first asks into L2 (5 tokens, wide: 12 141.1 us, 6 139.8)
constexpr int kSmemLimit = 225 * 1024;
constexpr int kPlanes = 3;                  // bf16 terms that hold a weighted hidden value: all 24 bits of it (two, found at run time, were no faster: 24 rows 52 us against 49)
constexpr int kMaxM = ALG_MOE_MAX_M;
constexpr int kLogitCols = 256;             // experts a CTA has logits of

struct MoeArgs {
  int M, D, F, E, k, sigmoid, renormalise, y_f32;
  float route_scale;
  const void *W_router;
  int router_f32, router_copies;   // copies: the router's rows lie on 16 bytes and are bf16
  const float *bias;
  int32_t *experts;
  float *weights;
  void *Y;
  int64_t ldy;
  int *table;                 // workspace: the chosen experts, as `Chosen` lies in shared memory
  __nv_bfloat16 *H;           // workspace: weighted hidden rows, [kPlanes][M * k][ldh]
  int ldh;                    // F to the next multiple of 64
  float4 *part;               // workspace: partial sums, [CTA][2][M][256] of the first launch, [..][128] of the second
  int down_ctas, down_blocks; // of the second launch
  int blocks;                 // tensor maps of whole column blocks (one copy a chunk)
  int *count;                 // [CTA]: arrivals at the unit whose first contributor it is
  int *status;
  long long wait_limit;
  uint32_t stall;             // test aid: bytes that are expected of a chunk's rows beside their own, and never come
  int stages, stage_bytes;
  int off_sums, off_ring;     // sums by row; the ring; in front of them what `Chosen` and `Routes` point to
};

// The chosen experts in ascending order: what both launches go by.
struct Chosen {
  int *n;          // how many
  uint2 *mask;     // the rows that take them
  int *expert;
  int *first;      // [n + 1] their first pair
  float *rest;     // [M] what the places without an expert add to a row: 0, or NaN
  __device__ __forceinline__ Chosen(uint8_t *p, int most, int M) {
    n = (int *)p, p += 8;
    mask = (uint2 *)p, p += (size_t)most * 8;
    expert = (int *)p, p += (size_t)most * 4;
    first = (int *)p, p += (size_t)(most + 1) * 4;
    rest = (float *)p;
  }
  __host__ __device__ static int words(int most, int M) { return 2 + 4 * most + 1 + M; }
};
// The rows' own choice; the first launch's.
struct Routes {
  uint2 *mask;     // [E] the rows that take an expert
  int *idx;        // [M * k] experts of a row, -1 for none
  float *w;        // [M * k] their weights
  int *place;      // [E] among the chosen
  float *pair_w;   // [M * k] weights in the order of the pairs
  __device__ __forceinline__ Routes(uint8_t *p, int P, int E) {
    mask = (uint2 *)p, p += (size_t)E * 8;
    idx = (int *)p, p += (size_t)P * 4;
    w = (float *)p, p += (size_t)P * 4;
    place = (int *)p, p += (size_t)E * 4;
    pair_w = (float *)p;
  }
  static size_t bytes(int P, int E) { return (size_t)E * 12 + (size_t)P * 12; }
};
__host__ __device__ __forceinline__ int most_chosen(int P, int E) { return P < E ? P : E; }
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

__device__ __forceinline__ void consumer_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory"); }
// From r.idx, with r.mask zero; all threads of the CTA.
__device__ void turn_round(const Routes &r, const Chosen &ch, int M, int E, int k) {
  const int tid = threadIdx.x, P = M * k;
  for (int p = tid; p < P; p += kThreads) {
    const int e = r.idx[p], m = p / k;
    if (e >= 0) atomicOr(m < 32 ? &r.mask[e].x : &r.mask[e].y, 1u << (m & 31));
  }
  __syncthreads();
  if (tid < 32) {
    int n = 0, pairs = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
      const int e = e0 + tid;
      const uint2 mask = e < E ? r.mask[e] : make_uint2(0u, 0u);
      const int c = rows_of(mask);
      const uint32_t used = __ballot_sync(~0u, c > 0);
      int sum = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(~0u, sum, o);
        if (tid >= o) sum += v;
      }
      const int at = n + __popc(used & ((1u << tid) - 1u));
      if (c > 0) ch.expert[at] = e, ch.mask[at] = mask, ch.first[at] = pairs + sum - c, r.place[e] = at;
      n += __popc(used);
      pairs += __shfl_sync(~0u, sum, 31);
    }
    if (tid == 0) ch.first[n] = pairs, *ch.n = n;
  }
  __syncthreads();
}
// What only the consumers need, by them.
__device__ void weigh_pairs(const Routes &r, const Chosen &ch, int M, int k) {
  for (int p = threadIdx.x; p < M * k; p += kConsumers) {
    const int e = r.idx[p], m = p / k;
    if (e >= 0) r.pair_w[ch.first[r.place[e]] + rows_below(r.mask[e], m)] = r.w[p];
  }
  for (int m = threadIdx.x; m < M; m += kConsumers) {
    float s = 0.f;
    for (int j = 0; j < k; ++j)
      if (r.idx[m * k + j] < 0) s += r.w[m * k + j];
    ch.rest[m] = s;
  }
  consumer_barrier();
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Which part of the logits a CTA has: experts [e0, e0 + 256) over chunks [begin, end) of D.
struct LogitShare {
  int slices, e0, begin, end;
  __device__ __forceinline__ LogitShare(const MoeArgs &a) {
    const int rank = (int)cluster_rank(), chunks = (a.D + 63) / 64;
    slices = a.E > kLogitCols ? kCluster / 2 : kCluster;
    e0 = rank / slices * kLogitCols;
    const int s = rank % slices;
    begin = chunks * s / slices, end = chunks * (s + 1) / slices;
  }
};
// A chunk of a router that tiled copies cannot fetch, as they would have left it; term p of an fp32 one.  All consumers.
__device__ void fill_router(const MoeArgs &a, uint8_t *stage, int e0, int k0, int p) {
  for (int i = threadIdx.x; i < 64 * kLogitCols; i += kConsumers) {
    const int e = i & (kLogitCols - 1), k = i / kLogitCols;
    __nv_bfloat16 v = __float2bfloat16_rn(0.f);
    if (e0 + e < a.E && k0 + k < a.D) {
      const size_t at = (size_t)(k0 + k) * a.E + e0 + e;
      if (a.router_f32) {
        float rest = ((const float *)a.W_router)[at];
        v = __float2bfloat16_rn(rest);
        for (int t = 0; t < p; ++t) {
          const float back = __bfloat162float(v);
          rest = isfinite(back) ? rest - back : 0.f;
          v = __float2bfloat16_rn(rest);
        }
      } else {
        v = ((const __nv_bfloat16 *)a.W_router)[at];
      }
    }
    *(__nv_bfloat16 *)(stage + (e >> 6) * kBox + k * 128 + (((e & 63) * 2) ^ ((k & 7) << 4))) = v;
  }
}

// The logits of rows rank, rank + 8, ...: the peers' parts in their order, to sums[row / 8][E].
__device__ void gather_logits(const MoeArgs &a, const float *parts, int slices, float *sums) {
  const int rank = (int)cluster_rank();
  for (int i = threadIdx.x; i < (a.M - rank + kCluster - 1) / kCluster * a.E; i += kConsumers) {
    const int row = i / a.E, e = i - row * a.E, first = e / kLogitCols * slices;
    const uint32_t at = smem_u32(parts + (rank + kCluster * row) * kLogitCols + (e & (kLogitCols - 1)));
    float part[kCluster], sum = 0.f;
#pragma unroll
    for (int p = 0; p < kCluster; ++p) {
      uint32_t there;
      part[p] = 0.f;
      if (p < slices) {
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(first + p));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part[p]) : "r"(there));
      }
    }
#pragma unroll
    for (int p = 0; p < kCluster; ++p) sum += part[p];
    sums[i] = sum;
  }
}

// The experts of this CTA's rows (rank, rank + 8, ...: eight at most, one a warp), for all CTAs of the cluster.  An expert's place is
// the number of experts in front of it.  Without a bias the order is that of the logits, which a score that underflows or saturates
// cannot spoil.  Short loops on purpose: this code runs once a launch and costs what its instructions take to arrive.  All consumers.
__device__ void choose(const MoeArgs &a, const float *logits, uint8_t *scratch, const Routes &r) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pitch = (a.E + 3) & ~3;
  const int rank = (int)cluster_rank(), rows = (a.M - rank + kCluster - 1) / kCluster;
  float *keys = (float *)scratch, *top_of = keys + 8 * pitch, *sum_of = top_of + 8;
  int *place = (int *)(sum_of + 8);   // [8][k]
  const int m = rank + kCluster * warp;
  const float *l = logits + warp * a.E;
  auto score = [&](float x, float top, float sum) { return a.sigmoid ? 1.f / (1.f + expf(-x)) : expf(x - top) / sum; };
  bool bad = false;
  float top = -FLT_MAX, sum = 1.f;
  if (warp < rows) {
#pragma unroll 4
    for (int e = lane; e < a.E; e += 32) bad = bad || !isfinite(l[e]), top = fmaxf(top, l[e]);
    bad = __any_sync(~0u, bad);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if (!a.sigmoid && (a.bias || !a.renormalise)) {   // (else the sum cancels)
      sum = 0.f;
#pragma unroll 1
      for (int e = lane; e < a.E; e += 32) sum += expf(l[e] - top);
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    }
#pragma unroll 1
    for (int e = lane; e < pitch; e += 32) {
      float key = -INFINITY;
      if (e < a.E && !bad) key = a.bias ? score(l[e], top, sum) + a.bias[e] : l[e];
      keys[warp * pitch + e] = key == key ? key : -INFINITY;
    }
    if (lane < a.k) place[warp * a.k + lane] = -1;
  }
  consumer_barrier();
#pragma unroll 1
  for (int i = threadIdx.x; i < rows * a.E; i += kConsumers) {
    const int row = i / a.E, e = i - row * a.E;
    const float *key = keys + row * pitch, mine = key[e];
    int before = 0;
#pragma unroll 2
    for (int f = 0; f < pitch; f += 4) {
      const float4 v = *(const float4 *)(key + f);
      before += (v.x > mine || (v.x == mine && f < e)) + (v.y > mine || (v.y == mine && f + 1 < e)) + (v.z > mine || (v.z == mine && f + 2 < e)) +
                (v.w > mine || (v.w == mine && f + 3 < e));
    }
    if (before < a.k && mine > -INFINITY) place[row * a.k + before] = e;
  }
  consumer_barrier();
  if (warp >= rows) return;
  int mine = lane < a.k ? place[warp * a.k + lane] : -1;
  if (mine >= a.E) mine = -1;   // (only where the logits lie over copies that came too late: an index of nothing must not leave here)
  float w = mine >= 0 ? score(l[mine], top, sum) : 0.f;
  if (a.renormalise) {
    float s = w;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    w /= fmaxf(s, 1e-20f);
  }
  w = bad ? __uint_as_float(0x7FC00000u) : w * a.route_scale;
  if (lane < a.k) {
    const uint32_t idx_at = smem_u32(r.idx + m * a.k + lane), w_at = smem_u32(r.w + m * a.k + lane);
#pragma unroll
    for (uint32_t p = 0; p < kCluster; ++p) {
      uint32_t there;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(idx_at), "r"(p));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there), "r"(mine) : "memory");
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(w_at), "r"(p));
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there), "f"(w) : "memory");
    }
  }
}
size_t choose_bytes(int M, int E, int k) {   // logits, their sums, what `choose` works in
  const size_t rows = (M + kCluster - 1) / kCluster;
  return ((size_t)M * kLogitCols + rows * E + 3) / 4 * 16 + ((size_t)8 * ((E + 3) & ~3) + 16 + 8 * (size_t)k) * 4;
}

// ---- the ring ----------------------------------------------------------------------------------------------------------

struct Ring {
  uint32_t full, empty;   // shared addresses of the barriers
  uint32_t base;
  int stages, stage_bytes;
  int s = 0;
  uint32_t parity = 0;
  bool failed = false;
  __device__ __forceinline__ uint32_t gave_up() const { return full + 16 * kStages; }   // a word behind the barriers: some thread of the CTA did
  __device__ __forceinline__ bool stopped() const {
    uint32_t v;
    asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(v) : "r"(gave_up()) : "memory");
    return v != 0;
  }
  __device__ __forceinline__ uint32_t stage() const { return base + s * stage_bytes; }
  __device__ __forceinline__ void next() {
    if (++s == stages) s = 0, parity ^= 1;
  }
  // A wait that runs out says so in the status word.  From then on nothing is right and nothing more is asked for, but everybody still goes the
  // same way to the end, and whoever multiplies gives the copies on their way time to land before their memory is used for something else or handed on.
  __device__ __forceinline__ bool wait(uint32_t bar, uint32_t par, const MoeArgs &a) {
    if (failed) return false;
    if (mbar_try_wait(bar, par)) return true;
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, par))
      if (clock64() - t0 > a.wait_limit) {
        failed = true;
        asm volatile("st.volatile.shared.u32 [%0], 1;" ::"r"(gave_up()) : "memory");
        atomicExch(a.status, (int)ALG_ERR_DEVICE_TIMEOUT);
        return false;
      }
    return true;
  }
  __device__ __forceinline__ bool wait_full(const MoeArgs &a) { return wait(full + 8 * s, parity, a); }
  __device__ __forceinline__ bool wait_empty(const MoeArgs &a) { return wait(empty + 8 * s, parity ^ 1, a) && !stopped(); }
  __device__ __forceinline__ void let_land() const {
    if (failed)
      for (const long long t0 = clock64(); clock64() - t0 < kLandCycles;) {
      }
  }
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
  bars[2 * kStages] = 0;
  for (int s = 0; s < stages; ++s) mbar_init(full + 8 * s, 2), mbar_init(empty + 8 * s, kWarps);   // two warps fetch, eight use
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
// Weights, 16 columns of the warp by 64 rows: lanes 0-15 address rows 0-7 of the first and of the second eight
// columns, lanes 16-31 rows 8-15; `box` and `byte_col` are those of the lane's eight.
__device__ __forceinline__ void load_weights(uint32_t box, int byte_col, uint32_t (&w)[4][4]) {
  const int lane = threadIdx.x & 31, row = (lane & 7) + (lane >> 4 << 3);
  const uint32_t at = box + row * 128 + (byte_col ^ ((row & 7) << 4));
#pragma unroll
  for (int k = 0; k < 4; ++k) ldmatrix4_trans(at + k * 16 * 128, w[k]);
}

// Two tiles of sixteen columns by the eight rows a lane addresses its part of, added to acc[.][t].
template <int NT>
__device__ __forceinline__ void product(const uint32_t (&w)[2][4][4], uint32_t at, int sw, float (&acc)[2][NT][4], int t) {
  const int lane = threadIdx.x & 31;
  uint32_t b[4], c[4];
  ldmatrix4(at + (((lane >> 3) * 16) ^ sw), b);
  ldmatrix4(at + ((64 + (lane >> 3) * 16) ^ sw), c);
  float d[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
  for (int j = 0; j < 2; ++j) mma(d[j], w[j][0], b[0], b[1]);
#pragma unroll
  for (int j = 0; j < 2; ++j) mma(d[j], w[j][1], b[2], b[3]);
#pragma unroll
  for (int j = 0; j < 2; ++j) mma(d[j], w[j][2], c[0], c[1]);
#pragma unroll
  for (int j = 0; j < 2; ++j) mma(d[j], w[j][3], c[2], c[3]);
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[j][t][e] += d[j][e];
}

// CTAs that take part: at most one for each chunk, and where there are fewer units than CTAs a whole number for each unit, if that
// leaves three quarters of them: then a CTA has parts of one unit, not of two, and meets others once.
__device__ __forceinline__ int takers(int64_t units, int per_unit, int ctas) {
  if (units * per_unit < ctas) return (int)(units * per_unit);
  if (units > ctas) return ctas;
  const int even = ctas / (int)units * (int)units;
  return 4 * even >= 3 * ctas ? even : ctas;
}
// The share of CTA c of n among `total` chunks, and whose share a chunk is in; n <= total, so that nobody's is empty (CTAs past n have none).
__device__ __forceinline__ int64_t share(int64_t total, int c, int n) { return total * c / n; }
__device__ __forceinline__ int owner(int64_t total, int64_t chunk, int n) { return (int)(((chunk + 1) * n - 1) / total); }

// Where the parts of a unit lie that CTAs c0 .. c1 have parts of.  A CTA has at most two units it shares: the first of its share, and the
// last, where that is another one; all but the first contributor begin inside the unit.
struct Parts {
  int c0, c1;
  int late;         // the first contributor's is its second
  size_t slot;      // float4s of a part
  float4 *part;
  __device__ __forceinline__ Parts(const MoeArgs &a, int64_t total, int n, int per_unit, int64_t unit, int row_floats) {
    c0 = owner(total, unit * per_unit, n), c1 = owner(total, (unit + 1) * per_unit - 1, n);
    late = share(total, c0, n) / per_unit == unit ? 0 : 1;
    slot = (size_t)a.M * row_floats / 4;
    part = a.part;
  }
  __device__ __forceinline__ bool whole() const { return c0 == c1; }
  __device__ __forceinline__ float4 *of(int c) const { return part + ((size_t)c * 2 + (c == c0 ? late : 0)) * slot; }
  __device__ __forceinline__ float4 sum(int at) const {   // in CTA order
    float4 s = __ldcg(of(c0) + at);
    const float4 *p = part + at;
#pragma unroll 4
    for (int c = c0 + 1; c <= c1; ++c) {
      const float4 v = __ldcg(p + (size_t)c * 2 * slot);
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    return s;
  }
  // After this CTA's part: is it the last?  All consumers.
  __device__ __forceinline__ bool last(const MoeArgs &a, int *flag) const {
    consumer_barrier();
    if (threadIdx.x == 0) {   // (what the barrier orders before its fence, the fence orders before its count)
      __threadfence();
      const bool l = atomicAdd(a.count + c0, 1) == c1 - c0;
      if (l) a.count[c0] = 0;   // as the next launch finds it
      __threadfence();
      *flag = l;
    }
    consumer_barrier();
    return *flag;   // (nobody writes it again before the barrier of another unit)
  }
};

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2, int c3, int c4) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst), "l"(map),
               "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
               : "memory");
}

// ---- first launch ------------------------------------------------------------------------------------------------------

// The first chunks of every share of the second launch are asked into L2, so that HBM does not idle between the launches.
__device__ void ask_ahead(const CUtensorMap &tm_d, const MoeArgs &a, const Chosen &ch) {
  const int per_expert = (a.F + 127) / 128, chosen = *ch.n, per_unit = chosen * per_expert;
  const int strips = (a.D + kCols - 1) / kCols, n = takers(strips, per_unit, a.down_ctas);
  const int64_t total = (int64_t)strips * per_unit;
  for (int c = blockIdx.x; c < n; c += gridDim.x) {
    const int64_t begin = share(total, c, n), end = min(share(total, c + 1, n), begin + kAhead);
    for (int64_t i = begin; i < end; ++i) {
      const int unit = (int)(i / per_unit), at = (int)(i - (int64_t)unit * per_unit), x = at / per_expert;
      if (a.down_blocks)
        asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];" ::"l"(&tm_d), "r"(0), "r"((at - x * per_expert) * 128),
                     "r"(unit * 2), "r"(ch.expert[x]));
    }
  }
}

template <int NT>   // row tiles of eight: ceil(M / 8) at most
__global__ void __launch_bounds__(kThreads, 1)
moe_up_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_r,
              const __grid_constant__ CUtensorMap tm_d, const MoeArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ __align__(8) uint64_t bars[2 * kStages + 1];
  __shared__ int flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, P = a.M * a.k, most = most_chosen(P, a.E);
  const Chosen ch(smem, most, a.M);
  const Routes r(smem + (Chosen::words(most, a.M) * 4 + 7) / 8 * 8, P, a.E);
  if (tid == 0) {
    init_ring(bars, a.stages);
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_x) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_r) : "memory");
  }
  for (int e = tid; e < a.E; e += kThreads) r.mask[e] = make_uint2(0u, 0u);
  // the router is asked into L2 while the previous kernel still runs (L2 is where its writes would go: no stale copy)
  const size_t router = (size_t)a.D * a.E * (a.router_f32 ? 4 : 2);
  for (size_t i = ((size_t)blockIdx.x * kThreads + tid) * 128; i < router; i += (size_t)gridDim.x * kThreads * 128)
    asm volatile("prefetch.global.L2 [%0];" ::"l"((const uint8_t *)a.W_router + i));
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  Ring ring = make_ring(a, smem, bars);
  const LogitShare mine(a);
  const int tiles = (a.M + 7) / 8;
  float *logits = (float *)(smem + a.off_ring);   // [M][256], over the ring once its chunks are used
  if (warp >= kWarps) {
    if (lane == 0)
      for (int c = mine.begin; c < mine.end; ++c) {
        if (!ring.wait_empty(a)) break;
        const uint32_t bar = ring.full + 8 * ring.s, st = ring.stage();
        if (warp > kWarps) {
          mbar_expect_tx(bar, a.M * 128 + a.stall);
          tma_load_2d(st + kChunk, &tm_x, bar, c * 64, 0);
        } else if (a.router_copies) {
          const int boxes = min(4, (a.E - mine.e0 + 63) / 64);
          mbar_expect_tx(bar, boxes * kBox);
          for (int b = 0; b < boxes; ++b) tma_load_2d(st + b * kBox, &tm_r, bar, mine.e0 + b * 64, c * 64);
        } else {
          mbar_arrive(bar);
        }
        ring.next();
      }
    __syncwarp();
  } else {
    float acc[2][NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[0][t][e] = acc[1][t][e] = 0.f;
    const int box = (warp >> 1) * kBox, byte_col = (warp & 1) * 64 + ((lane >> 3) & 1) * 16;
    for (int ck = mine.begin; ck < mine.end; ++ck) {
      ring.wait_full(a);
      const uint32_t st = ring.stage(), xs = st + kChunk;
      for (int p = 0; p < (a.router_f32 ? 3 : 1); ++p) {
        if (!a.router_copies) {
          consumer_barrier();
          fill_router(a, smem + a.off_ring + ring.s * ring.stage_bytes, mine.e0, ck * 64, p);
          consumer_barrier();
        }
        uint32_t w[2][4][4];
        load_weights(st + box, byte_col, w[0]);
        load_weights(st + box, byte_col + 32, w[1]);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (t >= tiles) continue;
          const int m = min(t * 8 + (lane & 7), a.M - 1);
          product(w, xs + m * 128, (m & 7) << 4, acc, t);
        }
      }
      if (!a.router_copies) fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(ring.empty + 8 * ring.s);
      ring.next();
    }
    ring.let_land();
    consumer_barrier();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int m = t * 8 + (lane & 3) * 2 + (e & 1);
          if (m < a.M) logits[m * kLogitCols + warp * 32 + j * 16 + (lane >> 2) + (e >> 1) * 8] = acc[j][t][e];
        }
  }
  cluster_sync();   // every peer's part is there
  if (warp < kWarps) {
    float *sums = logits + a.M * kLogitCols;
    gather_logits(a, logits, mine.slices, sums);
    consumer_barrier();
    choose(a, sums, (uint8_t *)logits + (a.M * kLogitCols + (a.M + kCluster - 1) / kCluster * a.E + 3) / 4 * 16, r);
  }
  fence_async_smem();   // the logits' memory belongs to the copies from here on
  __syncwarp();
  cluster_sync();
  turn_round(r, ch, a.M, a.E, a.k);
  if (warp < kWarps) {
    weigh_pairs(r, ch, a.M, a.k);
    if (blockIdx.x == 0) {
      for (int i = tid; i < Chosen::words(most, a.M); i += kConsumers) a.table[i] = ((const int *)smem)[i];
      for (int p = tid; p < P; p += kConsumers) {
        if (a.experts) a.experts[p] = r.idx[p];
        if (a.weights) a.weights[p] = r.w[p];
      }
    }
  }

  const int strips = (a.F + kCols - 1) / kCols, per_unit = (a.D + 63) / 64;
  const int64_t units = (int64_t)*ch.n * strips, total = units * per_unit;
  const int n = takers(units, per_unit, gridDim.x);
  if ((int)blockIdx.x >= n) return;
  const int64_t begin = share(total, blockIdx.x, n), end = share(total, blockIdx.x + 1, n);
  int64_t unit = begin / per_unit;
  int chunk = (int)(begin - unit * per_unit);
  int x = (int)(unit / strips), strip = (int)(unit - (int64_t)x * strips);
  if (warp >= kWarps) {
    if (lane == 0)
      for (int64_t i = begin; i < end; ++i) {
        if (!ring.wait_empty(a)) break;
        const uint32_t bar = ring.full + 8 * ring.s, st = ring.stage();
        if (warp > kWarps) {
          mbar_expect_tx(bar, a.M * 128 + a.stall);
          tma_load_2d(st + kChunk, &tm_x, bar, chunk * 64, 0);
        } else {
          mbar_expect_tx(bar, kChunk);
          const int e = ch.expert[x];
          if (a.blocks) {
            tma_load_5d(st, &tm_w, bar, 0, chunk * 64, 0, strip * 2, e);
          } else {
            tma_load_4d(st, &tm_w, bar, strip * kCols, chunk * 64, 0, e);
            tma_load_4d(st + 2 * kBox, &tm_w, bar, strip * kCols + 64, chunk * 64, 0, e);
          }
        }
        ring.next();
        if (++chunk == per_unit) {
          chunk = 0;
          if (++strip == strips) strip = 0, ++x;
        }
      }
    if (lane == 0 && warp == kWarps) ask_ahead(tm_d, a, ch);
    return;
  }
  // a warp has sixteen gate columns and the up columns that go with them, as two tiles of eight and eight
  const int box = (warp >> 2) * 2 * kBox + ((lane >> 3) & 1) * kBox, byte_col = (warp & 3) * 32;
  float *sums = (float *)(smem + a.off_sums);   // eight rows of 128 gate and 128 up sums
  for (int64_t i = begin; i < end; ++unit) {
    const uint2 mask = ch.mask[x];
    const int rows = rows_of(mask), first = ch.first[x];
    const Parts parts(a, total, n, per_unit, unit, 2 * kCols);
    // four hidden values of a pair, from their gate and up sums
    auto finish = [&](int row, int c, float4 gate, float4 up) {
      const int col = strip * kCols + c;
      if (col >= a.ldh) return;   // (columns from F on come out as zero: their weights are)
      const float w = r.pair_w[first + row];
      // (with expf and a rounded quotient results are as far off, 4.7e-7 to 5.1e-7 of their norm: what the tensor core's sums of 64 leave)
      auto hidden = [&](float g, float u) { return __fdividef(g, 1.f + __expf(-g)) * u * w; };
      float v[4] = {hidden(gate.x, up.x), hidden(gate.y, up.y), hidden(gate.z, up.z), hidden(gate.w, up.w)};
      __nv_bfloat16 *dst = a.H + (size_t)(first + row) * a.ldh + col;
#pragma unroll
      for (int p = 0; p < kPlanes; ++p) {
        __nv_bfloat16 b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          b[e] = __float2bfloat16_rn(v[e]);
          const float back = __bfloat162float(b[e]);
          v[e] = isfinite(back) ? v[e] - back : 0.f;
        }
        *(uint2 *)(dst + (size_t)p * P * a.ldh) = *(const uint2 *)b;
      }
    };
    auto body = [&](auto tiles_of) {
      constexpr int N = decltype(tiles_of)::value;
      float acc[2][N][4];
      int x_row[N];   // the row of X this lane addresses in each tile
#pragma unroll
      for (int t = 0; t < N; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[0][t][e] = acc[1][t][e] = 0.f;
        x_row[t] = nth_row(mask, min(t * 8 + (lane & 7), rows - 1));
      }
      for (; chunk < per_unit && i < end; ++chunk, ++i) {
        ring.wait_full(a);
        const uint32_t st = ring.stage(), xs = st + kChunk;
        uint32_t w[2][4][4];
        load_weights(st + box, byte_col, w[0]);
        load_weights(st + box, byte_col + 16, w[1]);
#pragma unroll
        for (int t = 0; t < N; ++t)
          if (t * 8 < rows) product(w, xs + x_row[t] * 128, (x_row[t] & 7) << 4, acc, t);
        __syncwarp();
        if (lane == 0) mbar_arrive(ring.empty + 8 * ring.s);
        ring.next();
      }
      // eight rows at a time, four columns a thread
#pragma unroll
      for (int t = 0; t < N; ++t) {
        if (t * 8 >= rows) continue;
        consumer_barrier();
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sums[((lane & 3) * 2 + (e & 1)) * kUpPitch + (e >> 1) * kCols + warp * 16 + j * 8 + (lane >> 2)] = acc[j][t][e];
        consumer_barrier();
        const int row = t * 8 + (tid >> 5), c = (tid & 31) * 4;
        if (row >= rows) continue;
        const float4 gate = *(const float4 *)(sums + (tid >> 5) * kUpPitch + c), up = *(const float4 *)(sums + (tid >> 5) * kUpPitch + kCols + c);
        if (parts.whole()) {
          finish(row, c, gate, up);
        } else {
          float4 *mine = parts.of(blockIdx.x) + row * (2 * kCols / 4) + c / 4;
          __stcg(mine, gate), __stcg(mine + kCols / 4, up);
        }
      }
    };
    if (NT == 1 || rows <= 8) body(std::integral_constant<int, 1>());
    else if (NT == 2 || rows <= 16) body(std::integral_constant<int, NT < 2 ? NT : 2>());
    else if (NT == 4 || rows <= 32) body(std::integral_constant<int, NT < 4 ? NT : 4>());
    else body(std::integral_constant<int, NT>());
    if (!parts.whole() && parts.last(a, &flag))
      for (int e = tid; e < rows * (kCols / 4); e += kConsumers) {
        const int row = e >> 5, c = e & 31;
        finish(row, c * 4, parts.sum(row * (2 * kCols / 4) + c), parts.sum(row * (2 * kCols / 4) + kCols / 4 + c));
      }
    chunk = 0;
    if (++strip == strips) strip = 0, ++x;
  }
  ring.let_land();
}

// ---- second launch -----------------------------------------------------------------------------------------------------

template <int NT>
__global__ void __launch_bounds__(kThreads, 1)
moe_down_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_h, const MoeArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ __align__(8) uint64_t bars[2 * kStages + 1];
  __shared__ int flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, P = a.M * a.k, most = most_chosen(P, a.E);
  const Chosen ch(smem, most, a.M);
  if (tid == 0) {
    init_ring(bars, a.stages);
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_h) : "memory");
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int i = tid; i < Chosen::words(most, a.M); i += kThreads) ((int *)smem)[i] = a.table[i];
  __syncthreads();
  const int chosen = *ch.n;
  const int strips = (a.D + kCols - 1) / kCols, per_expert = (a.F + 127) / 128, per_unit = chosen * per_expert;
  const int64_t total = (int64_t)strips * per_unit;
  const int n = takers(strips, per_unit, gridDim.x);
  // eight columns' sums of a row of Y (D is a multiple of eight)
  auto put = [&](int m, int c, const float4 &u, const float4 &v) {
    if (c >= a.D) return;
    const float rest = ch.rest[m];
    const float f[8] = {u.x + rest, u.y + rest, u.z + rest, u.w + rest, v.x + rest, v.y + rest, v.z + rest, v.w + rest};
    if (a.y_f32) store8((float *)a.Y + (int64_t)m * a.ldy + c, f);
    else store8((__nv_bfloat16 *)a.Y + (int64_t)m * a.ldy + c, f);
  };
  if (total == 0) {   // nobody takes an expert
    const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = blockIdx.x * kThreads + tid; i < a.M * (a.D / 8); i += gridDim.x * kThreads) put(i / (a.D / 8), i % (a.D / 8) * 8, none, none);
    return;
  }
  if ((int)blockIdx.x >= n) return;
  const int64_t begin = share(total, blockIdx.x, n), end = share(total, blockIdx.x + 1, n);
  Ring ring = make_ring(a, smem, bars);
  int64_t unit = begin / per_unit;
  const int at = (int)(begin - unit * per_unit);
  int x = at / per_expert, chunk = at - x * per_expert;
  constexpr int group_bytes = kPlanes * 2048;   // eight hidden rows: [plane][64 columns, 64 more][8]
  if (warp >= kWarps) {
    if (lane == 0)
      for (int64_t i = begin; i < end; ++i) {
        if (!ring.wait_empty(a)) break;
        const uint32_t bar = ring.full + 8 * ring.s, st = ring.stage();
        if (warp > kWarps) {
          const int p0 = ch.first[x], groups = (ch.first[x + 1] - p0 + 7) / 8;
          mbar_expect_tx(bar, groups * group_bytes + a.stall);
          for (int g = 0; g < groups; ++g) tma_load_4d(st + kChunk + g * group_bytes, &tm_h, bar, 0, p0 + g * 8, chunk * 2, 0);
        } else {
          mbar_expect_tx(bar, kChunk);
          const int e = ch.expert[x];
          if (a.blocks) {
            tma_load_4d(st, &tm_w, bar, 0, chunk * 128, (int)unit * 2, e);
          } else {
            tma_load_3d(st, &tm_w, bar, (int)unit * kCols, chunk * 128, e);
            tma_load_3d(st + 2 * kBox, &tm_w, bar, (int)unit * kCols + 64, chunk * 128, e);
          }
        }
        ring.next();
        if (++chunk == per_expert) {
          chunk = 0;
          if (++x == chosen) x = 0, ++unit;
        }
      }
    return;
  }
  // a warp has sixteen columns
  const int box = (warp >> 2) * 2 * kBox, byte_col = (warp & 3) * 32 + ((lane >> 3) & 1) * 16;
  float *sums = (float *)(smem + a.off_sums);   // [M][128]; a warp adds to its own columns
  for (int64_t i = begin; i < end; ++unit) {
    for (int e = tid; e < a.M * kDownPitch; e += kConsumers) sums[e] = 0.f;
    consumer_barrier();
    for (; x < chosen && i < end; ++x, chunk = 0) {
      const uint2 mask = ch.mask[x];
      const int rows = rows_of(mask);
      auto body = [&](auto tiles_of) {
        constexpr int N = decltype(tiles_of)::value;
        float acc[N][4];
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][e] = 0.f;
        for (; chunk < per_expert && i < end; ++chunk, ++i) {
          ring.wait_full(a);
          const uint32_t st = ring.stage(), hs = st + kChunk + (lane & 7) * 128;
          const int sw = (lane & 7) << 4;
          uint32_t w[2][4][4];
          load_weights(st + box, byte_col, w[0]);
          load_weights(st + box + kBox, byte_col, w[1]);
#pragma unroll
          for (int t = 0; t < N; ++t) {
            if (t * 8 >= rows) continue;
            float d[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int p = 0; p < kPlanes; ++p) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t at = hs + t * group_bytes + p * 2048 + h * 1024;
                uint32_t b[4], c[4];
                ldmatrix4(at + (((lane >> 3) * 16) ^ sw), b);
                ldmatrix4(at + ((64 + (lane >> 3) * 16) ^ sw), c);
                mma(d[h], w[h][0], b[0], b[1]);
                mma(d[h], w[h][1], b[2], b[3]);
                mma(d[h], w[h][2], c[0], c[1]);
                mma(d[h], w[h][3], c[2], c[3]);
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] += d[0][e] + d[1][e];
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(ring.empty + 8 * ring.s);
          ring.next();
        }
        // to the rows that take the expert
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int row = t * 8 + (lane & 3) * 2 + h;
            if (row >= rows) continue;
            float *to = sums + nth_row(mask, row) * kDownPitch + warp * 16 + (lane >> 2);
            to[0] += acc[t][h], to[8] += acc[t][2 + h];
          }
      };
      if (NT == 1 || rows <= 8) body(std::integral_constant<int, 1>());
      else if (NT == 2 || rows <= 16) body(std::integral_constant<int, NT < 2 ? NT : 2>());
      else if (NT == 4 || rows <= 32) body(std::integral_constant<int, NT < 4 ? NT : 4>());
      else body(std::integral_constant<int, NT>());
      if (chunk < per_expert) break;   // the share ends inside the expert
    }
    x = 0, chunk = 0;
    consumer_barrier();
    const Parts parts(a, total, n, per_unit, unit, kCols);
    for (int e = tid; e < a.M * (kCols / 8); e += kConsumers) {
      const int m = e / (kCols / 8), c = e % (kCols / 8);
      const float4 u = *(const float4 *)(sums + m * kDownPitch + c * 8), v = *(const float4 *)(sums + m * kDownPitch + c * 8 + 4);
      if (parts.whole()) {
        put(m, (int)unit * kCols + c * 8, u, v);
      } else {
        float4 *mine = parts.of(blockIdx.x) + m * (kCols / 4) + c * 2;
        __stcg(mine, u), __stcg(mine + 1, v);
      }
    }
    if (!parts.whole() && parts.last(a, &flag))
      for (int e = tid; e < a.M * (kCols / 8); e += kConsumers) {
        const int m = e / (kCols / 8), c = e % (kCols / 8), at = m * (kCols / 4) + c * 2;
        put(m, (int)unit * kCols + c * 8, parts.sum(at), parts.sum(at + 1));
      }
    consumer_barrier();
  }
  ring.let_land();
}

// ---- host --------------------------------------------------------------------------------------------------------------

int row_tiles(int64_t M) { return (int)((M + 7) / 8); }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

int hidden_pitch(int F) { return (F + 63) / 64 * 64; }
struct MoeLayout {
  size_t table, h, part, total;
};
MoeLayout moe_layout(const alg_moe_s &h, int64_t M) {
  MoeLayout L;
  const size_t P = (size_t)M * h.k;
  size_t off = 0;
  L.table = off, off = up256(off + (size_t)Chosen::words(most_chosen((int)P, h.E), (int)M) * 4);
  L.h = off, off = up256(off + kPlanes * P * hidden_pitch(h.F) * 2);
  L.part = off, off = up256(off + (size_t)h.num_sms * 2 * M * 2 * kCols * sizeof(float));
  L.total = off;
  return L;
}

using UpKernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const MoeArgs);
using DownKernel = void (*)(const CUtensorMap, const CUtensorMap, const MoeArgs);
UpKernel up_kernel(int tiles) {
  return tiles <= 1 ? moe_up_kernel<1> : tiles <= 2 ? moe_up_kernel<2> : tiles <= 4 ? moe_up_kernel<4> : moe_up_kernel<8>;
}
DownKernel down_kernel(int tiles) {
  return tiles <= 1 ? moe_down_kernel<1> : tiles <= 2 ? moe_down_kernel<2> : tiles <= 4 ? moe_down_kernel<4> : moe_down_kernel<8>;
}
cudaError_t moe_attributes() {
  static OncePerDevice once;
  return once([] {
    for (int t : {1, 2, 4, 8})
      for (const void *k : {(const void *)up_kernel(t), (const void *)down_kernel(t)}) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
        if (e != cudaSuccess) return e;
      }
    return cudaSuccess;
  });
}
// Ring behind the tables: as many stages as fit.
bool fit_ring(MoeArgs &a, bool routes, size_t sums, int stage_bytes, size_t scratch, size_t *smem) {
  const int P = a.M * a.k, table = (Chosen::words(most_chosen(P, a.E), a.M) * 4 + 7) / 8 * 8;
  a.off_sums = (int)((table + (routes ? Routes::bytes(P, a.E) : 0) + 15) / 16 * 16);
  a.off_ring = (int)((a.off_sums + sums + 1023) / 1024 * 1024);
  a.stage_bytes = stage_bytes;
  a.stages = (kSmemLimit - 1024 - a.off_ring) / stage_bytes;
  if (a.stages > kStages) a.stages = kStages;
  size_t ring = (size_t)a.stages * stage_bytes;
  if (ring < scratch) ring = scratch;
  *smem = 1024 + a.off_ring + ring;   // (the kernels align their part to the swizzle)
  return a.stages >= 2 && *smem <= (size_t)kSmemLimit;
}

template <typename... Params>
cudaError_t launch_moe(void (*k)(Params...), int grid, int cluster, size_t smem, cudaStream_t st, Params... params) {
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k, params...);
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

alg_status_t alg_moe_set_option(alg_moe_t h, alg_option_t option, int64_t value) {
  return h ? wait_option(&h->wait_limit, &h->stall, option, value) : ALG_ERR_INVALID_ARG;
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
  a.y_f32 = y_dtype == ALG_F32;
  a.W_router = W_router, a.router_f32 = h->router_dtype == ALG_F32, a.router_copies = !a.router_f32 && on_16(W_router, h->E, er);
  a.bias = select_bias, a.experts = experts, a.weights = weights;
  a.Y = Y, a.ldy = ldy;
  a.table = (int *)(ws + L.table), a.H = (__nv_bfloat16 *)(ws + L.h), a.ldh = hidden_pitch(h->F), a.part = (float4 *)(ws + L.part);
  a.status = h->d_state, a.wait_limit = h->wait_limit, a.stall = h->stall;

  const int tiles = row_tiles(M);
  CUtensorMap tm_up, tm_x, tm_down, tm_h;
  const uint64_t D = h->D, F = h->F, E = h->E, H = a.ldh, up_row = 4 * F, down_row = 2 * D;
  cudaError_t e;
  if (F % 64 == 0) {   // {column of a block, row, gate / up, column block, expert}
    const uint64_t d[5] = {64, D, 2, F / 64, E}, s[4] = {up_row, 2 * F, 128, up_row * D};
    const uint32_t b[5] = {64, 64, 2, 2, 1};
    e = make_map_nd(&tm_up, W_gate_up, 5, d, s, b, 128);
  } else {             // {column, row, gate / up, expert}: what is past F reads as zero
    const uint64_t d[4] = {F, D, 2, E}, s[3] = {up_row, 2 * F, up_row * D};
    const uint32_t b[4] = {64, 64, 2, 1};
    e = make_map_nd(&tm_up, W_gate_up, 4, d, s, b, 128);
  }
  if (e != cudaSuccess) return ALG_ERR_CUDA;
  if (D % 64 == 0) {   // {column of a block, row, column block, expert}
    const uint64_t d[4] = {64, F, D / 64, E}, s[3] = {down_row, 128, down_row * F};
    const uint32_t b[4] = {64, 128, 2, 1};
    e = make_map_nd(&tm_down, W_down, 4, d, s, b, 128);
  } else {
    const uint64_t d[3] = {D, F, E}, s[2] = {down_row, down_row * F};
    const uint32_t b[3] = {64, 128, 1};
    e = make_map_nd(&tm_down, W_down, 3, d, s, b, 128);
  }
  if (e != cudaSuccess) return ALG_ERR_CUDA;
  const uint64_t dx[2] = {D, (uint64_t)M}, sx[1] = {(uint64_t)ldx * 2};
  const uint32_t bx[2] = {64, (uint32_t)M};
  const uint64_t dh[4] = {64, (uint64_t)P, H / 64, kPlanes}, sh[3] = {2 * H, 128, 2 * P * H};   // {column of a block, pair, column block, plane}
  const uint32_t bh[4] = {64, 8, 2, kPlanes};
  if (make_map_nd(&tm_x, X, 2, dx, sx, bx, 128) != cudaSuccess || make_map_nd(&tm_h, a.H, 4, dh, sh, bh, 128) != cudaSuccess) return ALG_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)stream;
  size_t smem = 0;
  CUtensorMap tm_r = tm_x;
  if (a.router_copies) {
    const uint64_t dr[2] = {E, D}, sr[1] = {2 * E};
    const uint32_t br[2] = {64, 64};
    if (make_map_nd(&tm_r, W_router, 2, dr, sr, br, 128) != cudaSuccess) return ALG_ERR_CUDA;
  }
  a.blocks = F % 64 == 0;
  a.down_ctas = h->num_sms, a.down_blocks = D % 64 == 0;
  if (!fit_ring(a, true, 8 * kUpPitch * sizeof(float), kChunk + tiles * 1024, choose_bytes(a.M, a.E, a.k), &smem)) return ALG_ERR_UNSUPPORTED_SHAPE;
  a.count = h->d_state + 4;
  if (launch_moe(up_kernel(tiles), h->clusters * kCluster, kCluster, smem, st, tm_up, tm_x, tm_r, tm_down, a) != cudaSuccess) return ALG_ERR_CUDA;
  a.blocks = D % 64 == 0;
  if (!fit_ring(a, false, (size_t)a.M * kDownPitch * sizeof(float), kChunk + kPlanes * tiles * 2048, 0, &smem)) return ALG_ERR_UNSUPPORTED_SHAPE;
  a.count = h->d_state + 4 + h->num_sms;
  return launch_moe(down_kernel(tiles), h->num_sms, 1, smem, st, tm_down, tm_h, a) == cudaSuccess ? ALG_OK : ALG_ERR_CUDA;
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
