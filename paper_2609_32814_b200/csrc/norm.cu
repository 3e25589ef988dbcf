// C-ABI entry points of a block's border, and the second launch of the column sums.
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
  long long wait_limit = kDefaultWaitLimit;
  uint32_t stall = 0;
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
  const auto times = [&](const float *v, float none) { return a.ctas ? a.alpha * (v ? v[c] : none) : 0.f; };   // (no rows: 0, whatever the vectors hold)
  const float scale = times(a.scale, 1.f), w = times(a.post_w, 1.f), b = times(a.post_b, 0.f);
  if (y == 0 && a.d_pre_w) a.d_pre_w[c] = r;
  if (y == 1 && a.d_pre_b) a.d_pre_b[c] = r;
  if (y == 2 && a.d_post_w) a.d_post_w[c] = scale * r;
  if (y == 2 && a.d_scale) a.d_scale[c] = fmaf(w, r, b * slice[3][0][x]);
  if (y == 3 && a.d_post_b) a.d_post_b[c] = scale * r;
}

// Places before a row's first column in its first granule, at most.
int most_off(const NormArgs &a) { return a.period > 1 || a.off ? 7 : 0; }
// Threads of a row, rows a CTA works on at once, rows on their way; the grid.
int shape_rows(const alg_norm_s &h, NormArgs &a, int v, bool full, bool back, size_t *smem) {
  a.T = (a.D + most_off(a) + 256 * v - 1) / (256 * v) * 32;
  a.stage_bytes = 0;
  for (int k = 0; k < kOps; ++k) {
    a.at[k] = a.stage_bytes;
    a.bytes[k] = (uint32_t)(a.D * elem_size(k < kN ? h.stream_dtype : h.dtype));
    if (a.op[k]) a.stage_bytes += (int)((a.bytes[k] + 30) / 16 * 16);   // (a row off 16 bytes brings up to 15 on either side)
  }
  const size_t stage = a.stage_bytes;
  a.kept = (a.flags & ALG_NORM_JOIN ? full ? 3 : 1 : 0) | (a.flags & ALG_NORM_PRE ? full && !back ? 12 : 4 : 0);
  a.vectors = __builtin_popcount(a.kept) * a.T * v * 32;
  // kept as long as a row's stage fits beside them, which only fp32 rows past 4096 columns may not (LayerNorm of 8000 x 8192 bf16, where the vectors
  // leave one stage: 140 us forward and 320 backward, from L2 at their use 496 and 845)
  if (a.vectors + stage > (size_t)kBudget) a.vectors = 0;
  const size_t budget = (size_t)kBudget - a.vectors;
  int groups = kThreads / a.T;
  if (groups > kMaxGroups) groups = kMaxGroups;
  const int64_t rows_of = (a.M + a.period - 1) / a.period, sms = h.num_sms / a.period;   // rows of a shift, CTAs for them
  const int64_t per_sm = (rows_of + sms - 1) / sms;
  if (groups > per_sm) groups = (int)per_sm;
  while (groups > 1 && 2 * groups * stage > budget) --groups;   // (a row ahead of each)
  a.G = groups;
  int stages = (int)(budget / (groups * stage));
  if (stages > kMaxStages) stages = kMaxStages;
  const int64_t rows = (rows_of + (int64_t)groups * sms - 1) / ((int64_t)groups * sms);
  if (stages > rows) stages = (int)rows;
  a.stages = stages;
  size_t bytes = (size_t)groups * stages * stage;
  if (back && bytes < (size_t)groups * a.D * 4) bytes = (size_t)groups * a.D * 4;   // the groups' sums meet there
  *smem = kRowsAt + a.vectors + bytes;
  const int64_t ctas = (rows_of + groups - 1) / groups;
  return (int)(ctas < sms ? ctas : sms) * a.period;
}

// Values that are accessed at once.
int granule(const alg_norm_s &h) { return h.stream_dtype == ALG_BF16 && h.dtype == ALG_BF16 ? 8 : 4; }
// Columns a thread has, in eights.  The sums of LayerNorm's backward pass (four a column) leave registers for eight columns; all else takes
// sixteen, which halves what a row costs each thread besides its columns (32768 x 4096 forward 274 against 265 us, gradients of 8003 x 1024 47 against 40).
int eights(bool back, bool full, const NormArgs &a) { return back && full && a.D + most_off(a) <= kNarrow ? 1 : 2; }

// *full: LayerNorm or biases (set here; the caller asks for gradients of biases).  Kernels with their form as a constant serve bf16 F, gate and N, with dY and all gradients in the backward pass, LayerNorm (with or without biases) or RMS norm without biases, whose
// folded vectors fit.  alike: the matrices lie off their granules alike; on16: they and the vectors lie on 16 bytes.
template <bool BACK>
cudaError_t launch_norm(const alg_norm_s &h, NormArgs &a, bool alike, bool on16, bool *full, int *grid, cudaStream_t st) {
  size_t smem = 0;
  *full = *full || a.layer || a.post_b || a.pre_b;
  if (a.D + most_off(a) > 2 * kNarrow) alike = false, a.off = a.ld_off = 0, a.period = 1;   // (more than the threads of a CTA hold)
  const int v = eights(BACK, *full, a);
  const bool gated = a.flags & (ALG_NORM_GATE_ROW | ALG_NORM_GATE_ELEMENT), join = a.flags & ALG_NORM_JOIN;
  bool form = alike && (a.flags & (ALG_NORM_PRE | ALG_NORM_POST)) && h.dtype == ALG_BF16 && *full == (a.layer != 0);
  if (BACK) form = form && a.op[kT] && (!join || a.out) && (!gated || a.dg) && (a.layer || v == 2);
  if (form) {
    *grid = shape_rows(h, a, v, *full, BACK, &smem);
    form = a.vectors > 0;
  }
  if (form) {
    const int gate = !gated ? kGateNone : a.flags & ALG_NORM_GATE_ROW ? kGateRow : a.flags & ALG_NORM_GATE_SIGMOID ? kGateSigmoid : kGateElement;
    const int f = (a.flags & ALG_NORM_PRE ? kFormPre : 0) | (a.flags & ALG_NORM_POST ? kFormPost : 0) | (join ? kFormJoin : 0);
    const bool bf16 = h.stream_dtype == ALG_BF16;
    if constexpr (BACK) {
      auto *launch = !a.layer ? (bf16 ? launch_norm_backward_rms_bf16 : launch_norm_backward_rms_f32)
                     : v == 1 ? (bf16 ? launch_norm_backward_layer_bf16 : launch_norm_backward_layer_f32)
                              : (bf16 ? launch_norm_backward_layer_wide_bf16 : launch_norm_backward_layer_wide_f32);
      return launch(a, f + kFormGate * gate, on16, *grid, smem, st);
    } else {
      return (bf16 ? launch_norm_forward_bf16 : launch_norm_forward_f32)(a, f + kFormGate * gate, a.layer, on16, *grid, smem, st);
    }
  }
  *full = true;
  const int w = eights(BACK, true, a);
  *grid = shape_rows(h, a, w, true, BACK, &smem);
  const bool exact = on16 && a.D % (h.stream_dtype == ALG_F32 && h.dtype == ALG_F32 ? 4 : 8) == 0;   // (copies of an exact row are not rounded up to 16 bytes)
  const int types = (h.stream_dtype == ALG_F32 ? 2 : 0) + (h.dtype == ALG_F32 ? 1 : 0);
  auto *launch = !BACK ? launch_norm_forward_any : w == 1 ? launch_norm_backward_any : launch_norm_backward_any_wide;
  return launch(a, types, alike, exact, *grid, smem, st);
}

void put_operand(NormArgs &a, int k, const void *p, int64_t ld, size_t e) { a.op[k] = (const uint8_t *)p, a.pitch[k] = (uint32_t)(ld * e); }
// One matrix operand: its span, and whether it is well formed.
struct Operand {
  RowSpan s;
  bool ok;
};
Operand operand(const void *p, int64_t ld, int64_t cols, size_t e, int64_t M) {
  if (!p) return {span(nullptr, 0, 0, 1, 0), true};
  return {span(p, ld, cols, e, M), ld >= cols && ld < kMaxLd && on_element(p, e)};
}
bool vector_ok(const float *p) { return on_element(p, 4); }
// Whether all matrices lie off their granules alike (`unit` values: eight where all are bf16, else four); how.
struct Granules {
  int unit;
  bool any = false, alike = true, on16 = true;   // on16: all rows on 16 bytes
  int off = 0, ld_off = 0;
  void add(const void *p, int64_t ld, size_t e, int64_t M) {
    if (!p) return;
    const int o = (int)((uintptr_t)p / e % unit), l = M > 1 ? (int)(ld % unit) : 0;
    on16 = on16 && on_16(p, M > 1 ? ld : 0, e);
    if (any && (o != off || l != ld_off)) alike = false;
    any = true, off = o, ld_off = l;
  }
  void tell(NormArgs &a) const {
    a.off = alike ? off : 0, a.ld_off = alike ? ld_off : 0, a.period = 1;
    while (a.period * a.ld_off % unit) a.period *= 2;
  }
};
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

alg_status_t alg_norm_set_option(alg_norm_t h, alg_option_t option, int64_t value) {
  return h ? wait_option(&h->wait_limit, &h->stall, option, value) : ALG_ERR_INVALID_ARG;
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
  for (const Operand &o : to) {
    if (!o.ok) return ALG_ERR_INVALID_ARG;
    for (const Operand &i : in)
      if (meet(o.s, i.s) && !same_rows(o.s, i.s)) return ALG_ERR_INVALID_ARG;
  }
  for (const Operand &i : in)
    if (!i.ok) return ALG_ERR_INVALID_ARG;
  if (meet(to[0].s, to[1].s)) return ALG_ERR_INVALID_ARG;
  bool on16 = true;   // the vectors
  for (const float *v : {post_weight, post_bias, scale, pre_weight, pre_bias}) {
    if (!vector_ok(v)) return ALG_ERR_INVALID_ARG;
    on16 = on16 && ((uintptr_t)v & 15u) == 0;
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
  a.status = h->d_status, a.wait_limit = h->wait_limit, a.stall = h->stall;
  Granules gr = {granule(*h)};
  gr.add(R, ldr, ex, M), gr.add(F, ldf, eb, M), gr.add(el ? gate : nullptr, ldg, eb, M), gr.add(Y, ldy, ex, M), gr.add(N, ldn, eb, M);
  gr.tell(a);
  int grid = 0;
  bool full = false;
  return launch_norm<false>(*h, a, gr.alike, on16 && gr.on16, &full, &grid, (cudaStream_t)stream) == cudaSuccess ? ALG_OK : ALG_ERR_CUDA;
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
  bool on16 = true;   // the vectors
  for (const float *v : vectors_out)
    if (!vector_ok(v)) return ALG_ERR_INVALID_ARG;
  for (const float *v : vectors_in) {
    if (!vector_ok(v)) return ALG_ERR_INVALID_ARG;
    on16 = on16 && ((uintptr_t)v & 15u) == 0;
  }
  Granules gr = {granule(*h)};
  if (sums && (!workspace || ((uintptr_t)workspace & 255u))) return ALG_ERR_INVALID_ARG;
  if (sums && workspace_bytes < sums_bytes(*h)) return ALG_ERR_WORKSPACE_TOO_SMALL;
  const RowSpan ws = sums ? span(workspace, (int64_t)sums_bytes(*h), (int64_t)sums_bytes(*h), 1, 1) : span(nullptr, 0, 0, 1, 0);
  for (int k = 0; k < 5; ++k) {   // a vector's gradient lies over nothing that is read, nor over another
    if (!vectors_out[k]) continue;
    const RowSpan out = span(vectors_out[k], D, D, 4, 1);
    if (meet(out, ws)) return ALG_ERR_INVALID_ARG;
    for (const float *v : vectors_in)
      if (v && meet(out, span(v, D, D, 4, 1))) return ALG_ERR_INVALID_ARG;
    for (int l = 0; l < k; ++l)
      if (vectors_out[l] && meet(out, span(vectors_out[l], D, D, 4, 1))) return ALG_ERR_INVALID_ARG;
  }
  NormArgs a = {};
  if (M > 0) {
    if ((pre && !Y) || !dR || pre != (dN != nullptr) || join != (F != nullptr) || (row || el) != (gate != nullptr) || (!pre && !dY)) return ALG_ERR_INVALID_ARG;
    const size_t ex = elem_size(h->stream_dtype), eb = elem_size(h->dtype);
    const Operand in[5] = {operand(Y, ldy, D, ex, M), operand(dY, lddy, D, ex, M), operand(dN, lddn, D, eb, M), operand(F, ldf, D, eb, M),
                           row ? operand(gate, 1, 1, eb, M) : operand(gate, ldg, D, eb, M)};
    const Operand to[3] = {operand(dR, lddr, D, ex, M), operand(dF, lddf, D, eb, M),
                           row ? operand(dgate, 1, 1, eb, M) : operand(dgate, lddg, D, eb, M)};
    for (int k = 0; k < 5; ++k) {
      if (!in[k].ok || meet(ws, in[k].s)) return ALG_ERR_INVALID_ARG;
      for (const float *v : vectors_out)
        if (v && meet(in[k].s, span(v, D, D, 4, 1))) return ALG_ERR_INVALID_ARG;
    }
    for (int k = 0; k < 3; ++k) {
      if (!to[k].ok || meet(ws, to[k].s)) return ALG_ERR_INVALID_ARG;
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
    gr.add(pre ? Y : nullptr, ldy, ex, M), gr.add(dY, lddy, ex, M), gr.add(dN, lddn, eb, M), gr.add(F, ldf, eb, M), gr.add(el ? gate : nullptr, ldg, eb, M);
    gr.add(dR, lddr, ex, M), gr.add(dF, lddf, eb, M), gr.add(el ? dgate : nullptr, lddg, eb, M);
    gr.tell(a);
    a.y = (uint8_t *)dR, a.pitch_y = (uint32_t)(lddr * ex), a.out = (uint8_t *)dF, a.pitch_out = (uint32_t)(lddf * eb);
    a.dg = (uint8_t *)dgate, a.pitch_dg = (uint32_t)(lddg * eb);
  }
  if (!is_current(h->device)) return ALG_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  a.M = (uint32_t)M, a.D = D, a.flags = h->flags, a.layer = h->kind == ALG_NORM_LAYER, a.eps = h->eps, a.alpha = alpha;
  a.post_w = post_weight, a.post_b = post_bias, a.scale = scale, a.pre_w = pre_weight;
  a.part = sums ? (float *)workspace : nullptr;
  a.status = h->d_status, a.wait_limit = h->wait_limit, a.stall = h->stall;
  int grid = 0;
  bool full = d_post_bias || d_pre_bias;
  if (M > 0 && launch_norm<true>(*h, a, gr.alike, on16 && gr.on16, &full, &grid, st) != cudaSuccess) return ALG_ERR_CUDA;
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
