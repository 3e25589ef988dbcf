// C-ABI entry points of a block's border, the kernels that find out their form at run time, and the second launch of the column sums.
#include <cmath>
#include <new>

#include "norm.cuh"

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

// Threads of a row, rows a CTA works on at once, rows on their way; the grid.
int shape_rows(const alg_norm_s &h, NormArgs &a, int v, bool vec, bool full, bool back, size_t *smem) {
  a.T = (a.D + 256 * v - 1) / (256 * v) * 32;
  a.stage_bytes = 0;
  for (int k = 0; k < kOps; ++k) {
    a.at[k] = a.stage_bytes;
    a.bytes[k] = (uint32_t)(a.D * elem_size(k < kN ? h.stream_dtype : h.dtype));
    if (a.op[k]) a.stage_bytes += (int)((a.bytes[k] + (vec ? 15 : 30)) / 16 * 16);   // (a row off 16 bytes brings up to 15 on either side)
  }
  const size_t stage = a.stage_bytes;
  const int kept = ((a.flags & ALG_NORM_JOIN ? 1 : 0) + (a.flags & ALG_NORM_PRE ? 1 : 0)) * (full ? 2 : 1);
  a.vectors = kept * a.T * v * 32;
  if (a.vectors > kVectorBytes) a.vectors = 0;   // (only rows of sixteen columns a thread have as many)
  const size_t budget = (size_t)kBudget - a.vectors;
  int groups = kThreads / a.T;
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

// Columns a thread has, in eights.  The sums of LayerNorm's backward pass (four a column) leave registers for eight columns; all else takes
// sixteen, which halves what a row costs each thread besides its columns (32768 x 4096 forward 274 against 265 us, gradients of 8003 x 1024 47 against 40).
int eights(bool back, bool full, int D) { return back && full && D <= kNarrow ? 1 : 2; }

template <bool BACK, typename XT, typename BT, int V>
cudaError_t launch_any(NormArgs &a, bool vec, int grid, size_t smem, cudaStream_t st) {
  constexpr int kMap = sizeof(XT) == 4 || sizeof(BT) == 4 ? kFours : kEight;
  return vec ? launch_rows<BACK, XT, BT, kMap, V, true, kAny>(a, grid, smem, st) : launch_rows<BACK, XT, BT, kScalar, V, true, kAny>(a, grid, smem, st);
}
template <bool BACK, typename XT, typename BT>
cudaError_t launch_any(NormArgs &a, int v, bool vec, int grid, size_t smem, cudaStream_t st) {
  if constexpr (BACK)
    if (v == 1) return launch_any<BACK, XT, BT, 1>(a, vec, grid, smem, st);
  return launch_any<BACK, XT, BT, 2>(a, vec, grid, smem, st);
}

// *full: LayerNorm or biases (set here; the caller asks for gradients of biases).  Kernels with their form as a constant serve bf16 F, gate and N
// on 16 bytes, with dY and all gradients in the backward pass, LayerNorm (with or without biases) or RMS norm without biases, whose
// folded vectors fit.
template <bool BACK>
cudaError_t launch_norm(const alg_norm_s &h, NormArgs &a, bool vec, bool *full, int *grid, cudaStream_t st) {
  size_t smem = 0;
  *full = *full || a.layer || a.post_b || a.pre_b;
  const int v = eights(BACK, *full, a.D);
  const bool gated = a.flags & (ALG_NORM_GATE_ROW | ALG_NORM_GATE_ELEMENT), join = a.flags & ALG_NORM_JOIN;
  bool form = vec && h.dtype == ALG_BF16 && *full == (a.layer != 0);
  if (BACK) form = form && a.op[kT] && (!join || a.out) && (!gated || a.dg) && v == (a.layer ? 1 : 2);
  if (form) {
    *grid = shape_rows(h, a, v, vec, *full, BACK, &smem);
    form = a.vectors > 0;
  }
  if (form) {
    const int gate = !gated ? kGateNone : a.flags & ALG_NORM_GATE_ROW ? kGateRow : a.flags & ALG_NORM_GATE_SIGMOID ? kGateSigmoid : kGateElement;
    const int f = (a.flags & ALG_NORM_PRE ? kFormPre : 0) | (a.flags & ALG_NORM_POST ? kFormPost : 0) | (join ? kFormJoin : 0);
    auto *launch = BACK ? (h.stream_dtype == ALG_BF16 ? launch_norm_backward_bf16 : launch_norm_backward_f32)
                        : (h.stream_dtype == ALG_BF16 ? launch_norm_forward_bf16 : launch_norm_forward_f32);
    return launch(a, f + kFormGate * gate, a.layer, *grid, smem, st);
  }
  *full = true;
  const int w = eights(BACK, true, a.D);
  *grid = shape_rows(h, a, w, vec, true, BACK, &smem);
  if (h.stream_dtype == ALG_BF16)
    return h.dtype == ALG_BF16 ? launch_any<BACK, __nv_bfloat16, __nv_bfloat16>(a, w, vec, *grid, smem, st)
                               : launch_any<BACK, __nv_bfloat16, float>(a, w, vec, *grid, smem, st);
  return h.dtype == ALG_BF16 ? launch_any<BACK, float, __nv_bfloat16>(a, w, vec, *grid, smem, st) : launch_any<BACK, float, float>(a, w, vec, *grid, smem, st);
}

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
  return launch_norm_kernel((const void *)norm_sums_kernel, (D + 31) / 32, 32 * kSlices, 0, st, params) == cudaSuccess ? ALG_OK : ALG_ERR_CUDA;
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
