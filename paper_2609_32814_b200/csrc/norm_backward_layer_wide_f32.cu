// A block's border, backward pass, LayerNorm of rows of sixteen columns a thread, residual stream in f32: the kernels whose form is a constant.
#include "norm.cuh"

namespace algproj {

cudaError_t launch_norm_backward_layer_wide_f32(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st) {
  return launch_forms<true, float, 2, true>(a, form, on16, grid, smem, st);
}

}  // namespace algproj
