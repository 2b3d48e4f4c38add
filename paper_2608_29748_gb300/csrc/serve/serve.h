// Host-side declarations of the operators around a round: the paged cache,
// attention over it, sampling.
#pragma once

#include "../internal.h"

namespace retrace {

constexpr int kMaxHeadDim = 256;

struct AppendArgs {
  const void* q;  // NULL: keys and values only
  long long q_token, q_head;
  int q_heads;
  const void* k;
  long long k_token, k_head;
  const void* v;
  long long v_token, v_head;
  const int32_t* q_start;  // NULL: T / B tokens each
  const int32_t* cache_len;
  int B, T;
  const float* rope;  // NULL: no rotation
  int rope_positions, rot, interleaved;
  retrace_kv_cache cache;
  void* q_out;
  long long qo_token, qo_head;
};
cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t stream);

// Workspace of retrace_attend: the status word (256 bytes), one ticket per CTA,
// then two partial results per CTA (a CTA's range of work begins and ends inside
// a unit at most): fp32 rows and their maximum and sum.  It does not depend on
// the batch, so one workspace serves every call of its head size.
constexpr int kAttendMaxCtas = 512;    // of the CUDA-core kernel
constexpr int kAttendMaxTcCtas = 192;  // of the tensor-core kernel
constexpr size_t kAttendTickets = 256;
constexpr size_t kAttendPartials = kAttendTickets + kAttendMaxCtas * 4;

struct AttendArgs {
  const void* q;
  long long q_token, q_head;
  int q_heads;
  const int32_t* q_start;
  const int32_t* cache_len;
  int B, T;
  float scale;
  int window, sinks, causal;
  retrace_kv_cache cache;
  void* out;
  long long out_token, out_head;
  uint32_t* status;
  uint32_t* tickets;
  float* partials;
};
cudaError_t launch_attend_simt(const AttendArgs& a, cudaStream_t stream);
size_t attend_simt_partial_bytes(int head_dim);
cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t stream);
size_t attend_tc_partial_bytes(int head_dim);
bool attend_tc_supported(const AttendArgs& a);

struct SampleArgs {
  const void* logits;
  int B, R, V;
  long long row_stride, batch_stride;
  const float* uniforms;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* tokens;
  float* probs;
};
cudaError_t launch_sample(const SampleArgs& a, retrace_dtype dtype, cudaStream_t stream);

}  // namespace retrace
