// A block's border, backward pass, rows of sixteen columns a thread: the kernels that find out their form at run time, for every type and alignment.
#include "norm.cuh"

namespace algproj {
namespace {

template <typename XT, typename BT>
cudaError_t launch_any(NormArgs &a, bool alike, int grid, size_t smem, cudaStream_t st) {
  constexpr int kMap = sizeof(XT) == 4 || sizeof(BT) == 4 ? kFours : kEight;
  return alike ? launch_rows<true, XT, BT, kMap, 2, true, kAny>(a, grid, smem, st) : launch_rows<true, XT, BT, kScalar, 2, true, kAny>(a, grid, smem, st);
}

}  // namespace

cudaError_t launch_norm_backward_any_wide(NormArgs &a, int types, bool alike, bool, int grid, size_t smem, cudaStream_t st) {
  switch (types) {
    case 0: return launch_any<__nv_bfloat16, __nv_bfloat16>(a, alike, grid, smem, st);
    case 1: return launch_any<__nv_bfloat16, float>(a, alike, grid, smem, st);
    case 2: return launch_any<float, __nv_bfloat16>(a, alike, grid, smem, st);
    default: return launch_any<float, float>(a, alike, grid, smem, st);
  }
}

}  // namespace algproj
