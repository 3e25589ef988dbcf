// A block's border, forward pass, residual stream in f32: the kernels whose form is a constant.
#include "norm.cuh"

namespace algproj {

cudaError_t launch_norm_forward_f32(NormArgs &a, int form, bool layer, bool on16, int grid, size_t smem, cudaStream_t st) {
  return layer ? launch_forms<false, float, 2, true>(a, form, on16, grid, smem, st) : launch_forms<false, float, 2, false>(a, form, on16, grid, smem, st);
}

}  // namespace algproj
