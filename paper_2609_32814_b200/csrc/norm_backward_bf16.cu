// A block's border, backward pass, residual stream in bf16: the kernels whose form is a constant.
#include "norm.cuh"

namespace algproj {

cudaError_t launch_norm_backward_bf16(NormArgs &a, int form, bool layer, int grid, size_t smem, cudaStream_t st) {
  return layer ? launch_forms<true, __nv_bfloat16, 1, true>(a, form, grid, smem, st) : launch_forms<true, __nv_bfloat16, 2, false>(a, form, grid, smem, st);
}

}  // namespace algproj
