// Host-side declarations of the operators around a round: the paged cache,
// attention over it, sampling.
#pragma once

#include "../internal.h"

namespace retrace {

constexpr int kMaxHeadDim = 256;

// Lets a kernel have `bytes` of dynamic shared memory: asked of the runtime once per
// device (`done`: a bit per device, the kernel's own), not on every call.
template <typename K>
cudaError_t allow_shared(K kernel, size_t bytes, const DeviceInfo& dev, std::atomic<uint64_t>& done) {
  const uint64_t bit = 1ull << (dev.device & 63);
  if (dev.device < 64 && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

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

// Workspace of retrace_attend: the status word (256 bytes), a JoinUnit per CTA, a ticket
// per CTA (zero between calls: who takes a unit's last one clears it), then
// two partial results per CTA (a CTA's range of work begins and ends inside a unit at
// most): fp32 rows, and the maximum and sum of each.  Its size and layout do not depend on
// the batch, so one workspace serves every call of its head size.
constexpr int kAttendMaxCtas = 512;    // of the CUDA-core kernel
constexpr int kAttendMaxTcCtas = 192;  // of the tensor-core kernel

// A unit that several CTAs shared: its first rows are `part_rows` apart from the next
// ones in a part; row r is the query head head + r % group of token + r / group.
struct JoinUnit {
  int pieces;  // CTAs, from the one whose entry this is; 0: none
  int rows, first_rows;
  int token, head, group;
  int unused[2];
};
constexpr size_t kAttendUnits = 256;
constexpr size_t kAttendTickets = kAttendUnits + kAttendMaxCtas * sizeof(JoinUnit);
constexpr size_t kAttendPartials = kAttendTickets + 256 * 4;
static_assert(kAttendMaxTcCtas <= 256, "tickets");

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
  JoinUnit* units;
  uint32_t* tickets;
  float* partials;
};
// A part: `rows` rows of `cols` floats, then their (maximum, sum).
struct PartShape {
  int rows, cols;
  float scale2;  // weights are 2^(scale2 (x - maximum)); 0: e^(x - maximum)
};
cudaError_t launch_attend_join(const AttendArgs& a, PartShape part, int ctas, cudaStream_t stream);
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
