// A block's border, backward pass, RMS norm, residual stream in f32: the kernels whose form is a constant.
#include "norm.cuh"

namespace algproj {

cudaError_t launch_norm_backward_rms_f32(NormArgs &a, int form, bool on16, int grid, size_t smem, cudaStream_t st) {
  return launch_forms<true, float, 2, false>(a, form, on16, grid, smem, st);
}

}  // namespace algproj
