// Attention on the CUDA cores over a cache in 8 bits: keys and values are turned into fp32,
// times their page's power of two (exact), on the way into shared memory.
#include "attend_simt.cuh"

namespace retrace {

cudaError_t launch_attend_simt_fp8(const AttendArgs& a, cudaStream_t stream) {
  SimtParams p = simt_params(a, 1);
  return a.dtype == RETRACE_BF16 ? launch_typed<__nv_bfloat16, __nv_fp8_e4m3>(p, stream) : launch_typed<float, __nv_fp8_e4m3>(p, stream);
}

}  // namespace retrace
