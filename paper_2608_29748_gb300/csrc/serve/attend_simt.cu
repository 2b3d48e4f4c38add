// Attention on the CUDA cores over caches in fp32 and bf16.
#include "attend_simt.cuh"

namespace retrace {

size_t attend_simt_partial_bytes(int head_dim) {
  const size_t DP = head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : head_dim <= 128 ? 128 : 256;
  const size_t rows = DP <= 128 ? (size_t)kMaxManyCtas * 128 : (size_t)kAttendMaxCtas * 32;
  static_assert(kMaxManyCtas * 128 >= kAttendMaxCtas * 32, "room for either kernel's parts");
  return rows * 2 * (DP + 2) * 4;
}

cudaError_t launch_attend_simt(const AttendArgs& a, cudaStream_t stream) {
  if (a.cache.dtype == RETRACE_BF16) {
    SimtParams p = simt_params(a, 2);
    return launch_typed<__nv_bfloat16, __nv_bfloat16>(p, stream);
  }
  SimtParams p = simt_params(a, 4);
  return launch_typed<float, float>(p, stream);
}

}  // namespace retrace
