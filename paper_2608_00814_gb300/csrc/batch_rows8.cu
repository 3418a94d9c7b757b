// The CUDA-core attention kernel over 8-bit pages.
#include "batch_rows.cuh"

namespace oos {

cudaError_t launch_rows8(const BatchAttnArgs& a, int dtype, int rt, cudaStream_t st) {
  const bool vec = a.pages.d % 4 == 0 && ((uintptr_t)a.pages.k | (uintptr_t)a.pages.v) % 4 == 0;
  if (dtype == OOS_DTYPE_F32) return launch_rows<float, E4M3>(a, rt, vec, st);
  if (dtype == OOS_DTYPE_BF16) return launch_rows<__nv_bfloat16, E4M3>(a, rt, vec, st);
  return launch_rows<__half, E4M3>(a, rt, vec, st);
}

}  // namespace oos
