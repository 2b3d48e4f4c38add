// Joins the parts of the units that several CTAs of an attention kernel shared.
//
// With a part's maximum m_i, sum l_i and unnormalised rows o_i, and m the largest of
// the maxima: o = sum_i e^(m_i - m) o_i / sum_i e^(m_i - m) l_i.  A warp takes a row and
// keeps the loads of eight parts in flight; the rows of all units are dealt out over all
// warps.  It is a kernel of its own, launched ahead and waiting for the attention kernel
// to end, because one CTA that joins a unit by itself reads all of its parts at the rate
// of one SM: 38 parts of 128 rows of 128 took 140 us, and 2 us here.
#include <math.h>

#include "../common.cuh"
#include "serve.h"

namespace retrace {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float power(float x, float scale2) {
  if (scale2 == 0.f) return expf(x);
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * scale2));
  return y;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) attend_join_kernel(const __grid_constant__ AttendArgs a, PartShape part, int ctas) {
  __shared__ JoinUnit s_unit[kThreads];
  __shared__ int s_upto[kThreads], s_warp[kWarps];
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, D = a.cache.head_dim;
  const long long size = (long long)part.rows * (part.cols + 2);
  const int warps = gridDim.x * kWarps;
  int next = blockIdx.x * kWarps + warp;  // this warp's next row among all rows
  pdl_wait();
  int before = 0;
  for (int c0 = 0; c0 < ctas; c0 += kThreads) {
    const int c = c0 + tid;
    JoinUnit mine{};
    if (c < ctas) mine = a.units[c];
    const int rows = mine.pieces > 0 ? mine.rows : 0;
    int x = rows;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = x;
    s_unit[tid] = mine;
    __syncthreads();
    for (int w = 0; w < warp; ++w) x += s_warp[w];
    s_upto[tid] = before + x;
    __syncthreads();
    const int end = s_upto[kThreads - 1];
    for (; next < end; next += warps) {
      // the unit that holds the row: the first whose running count passes it
      int u = 0;
#pragma unroll
      for (int step = kThreads / 2; step > 0; step >>= 1)
        if (s_upto[u + step - 1] <= next) u += step;
      const JoinUnit& unit = s_unit[u];
      const int r = next - (s_upto[u] - unit.rows);
      const int slot = r < unit.first_rows ? r : part.rows / 2 + r - unit.first_rows;
      const float* first = a.partials + (long long)(c0 + u) * 2 * size;
      T* out = static_cast<T*>(a.out) + (long long)(unit.token + r / unit.group) * a.out_token +
               (unit.head + r % unit.group) * (long long)a.out_head;
      for (int col = lane * 4; col < part.cols; col += 128) {
        float top = -INFINITY, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int i0 = 0; i0 < unit.pieces; i0 += 8) {
          float2 st[8];
          float4 y[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (i0 + i >= unit.pieces) break;
            const float* from = first + ((long long)(i0 + i) * 2 + (i0 + i == 0 ? 1 : 0)) * size;
            st[i] = *reinterpret_cast<const float2*>(from + part.rows * part.cols + slot * 2);
            y[i] = *reinterpret_cast<const float4*>(from + slot * part.cols + col);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (i0 + i >= unit.pieces) break;
            if (st[i].x == -INFINITY) continue;  // the part's keys are hidden from this row
            const float up = fmaxf(top, st[i].x), f = power(top - up, part.scale2), g = power(st[i].x - up, part.scale2);
            top = up;
            sum = sum * f + st[i].y * g;
            o[0] = o[0] * f + y[i].x * g;
            o[1] = o[1] * f + y[i].y * g;
            o[2] = o[2] * f + y[i].z * g;
            o[3] = o[3] * f + y[i].w * g;
          }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (col + i < D) out[col + i] = from_f32<T>(o[i] * inv);
      }
    }
    before = end;
  }
}

}  // namespace

cudaError_t launch_attend_join(const AttendArgs& a, PartShape part, int ctas, cudaStream_t stream) {
  DeviceInfo dev;
  const cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  const dim3 grid(dev.sm_count * 2), block(kThreads);
  if (a.cache.dtype == RETRACE_BF16)
    return launch_dependent(attend_join_kernel<__nv_bfloat16>, grid, block, 0, stream, 1u, a, part, ctas);
  return launch_dependent(attend_join_kernel<float>, grid, block, 0, stream, 1u, a, part, ctas);
}

}  // namespace retrace
