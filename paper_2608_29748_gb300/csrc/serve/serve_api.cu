// C ABI of the operators around a round (declared in include/retrace.h):
// argument checks and dispatch.
#include <stdarg.h>
#include <stdio.h>

#include "serve.h"

using namespace retrace;

namespace {

retrace_status fail(retrace_status s, const char* fmt, ...) {
  char msg[384];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof(msg), fmt, ap);
  va_end(ap);
  set_last_error(msg);
  return s;
}

retrace_status cuda_fail(cudaError_t e, const char* what) {
  return fail(RETRACE_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

bool dtype_ok(retrace_dtype t) { return t == RETRACE_BF16 || t == RETRACE_F32; }

// Query tokens, lengths and the cache, as both cache operators take them.
retrace_status check_cache(const retrace_kv_cache* c, int q_heads, int B, int T, const int32_t* q_start,
                           const int32_t* cache_len) {
  if (!c) return fail(RETRACE_ERR_INVALID_ARG, "cache is NULL");
  if (!dtype_ok(c->dtype)) return fail(RETRACE_ERR_INVALID_ARG, "unknown dtype %d", (int)c->dtype);
  if (B < 0 || T < 0 || (B == 0 && T > 0)) return fail(RETRACE_ERR_INVALID_ARG, "bad shape B=%d T=%d", B, T);
  if (T > (1 << 30)) return fail(RETRACE_ERR_UNSUPPORTED, "T=%d exceeds 2^30", T);
  if (c->kv_heads < 1 || c->head_dim < 1 || c->page_size < 1 || c->num_pages < 0 || c->max_pages < 0)
    return fail(RETRACE_ERR_INVALID_ARG, "bad cache shape: %d pages of %d slots, %d heads of %d, %d pages a sequence",
                c->num_pages, c->page_size, c->kv_heads, c->head_dim, c->max_pages);
  if (c->head_dim > kMaxHeadDim)
    return fail(RETRACE_ERR_UNSUPPORTED, "head_dim=%d exceeds %d", c->head_dim, kMaxHeadDim);
  if (q_heads < 1 || q_heads % c->kv_heads)
    return fail(RETRACE_ERR_INVALID_ARG, "q_heads=%d is no multiple of kv_heads=%d", q_heads, c->kv_heads);
  if (q_heads > 65535) return fail(RETRACE_ERR_UNSUPPORTED, "q_heads=%d exceeds 65535", q_heads);
  if (c->head_stride < 0 || c->slot_stride < 0 || c->page_stride < 0 || c->table_stride < c->max_pages)
    return fail(RETRACE_ERR_INVALID_ARG, "bad cache strides");
  if ((long long)c->max_pages * c->page_size > (1ll << 30))
    return fail(RETRACE_ERR_UNSUPPORTED, "%d pages of %d slots a sequence exceed 2^30 positions", c->max_pages, c->page_size);
  if (!q_start && B > 0 && T % B) return fail(RETRACE_ERR_INVALID_ARG, "without q_start, T=%d must be a multiple of B=%d", T, B);
  if (T == 0) return RETRACE_OK;
  if (!cache_len || !c->k || !c->v || (c->max_pages > 0 && !c->page_table))
    return fail(RETRACE_ERR_INVALID_ARG, "NULL tensor pointer");
  return RETRACE_OK;
}

}  // namespace

extern "C" {

retrace_status retrace_kv_append(const void* q, int64_t q_token_stride, int64_t q_head_stride, int q_heads,
                                 const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                                 int64_t v_token_stride, int64_t v_head_stride, const int32_t* q_start,
                                 const int32_t* cache_len, int B, int T, const float* rope, int rope_positions,
                                 int rot, int interleaved, const retrace_kv_cache* cache, void* q_out,
                                 int64_t q_out_token_stride, int64_t q_out_head_stride, cudaStream_t stream) {
  set_last_error("");
  retrace_status st = check_cache(cache, q ? q_heads : cache ? cache->kv_heads : 1, B, T, q_start, cache_len);
  if (st != RETRACE_OK) return st;
  if (rope && (rot < 0 || rot % 2 || rot > cache->head_dim || rope_positions < 0))
    return fail(RETRACE_ERR_INVALID_ARG, "rot=%d must be even and in [0, head_dim=%d], rope_positions=%d not negative", rot,
                cache->head_dim, rope_positions);
  if (q_token_stride < 0 || q_head_stride < 0 || k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 ||
      v_head_stride < 0 || q_out_token_stride < 0 || q_out_head_stride < 0)
    return fail(RETRACE_ERR_INVALID_ARG, "negative stride");
  if (T == 0) return RETRACE_OK;
  if (!k || !v || (q && !q_out)) return fail(RETRACE_ERR_INVALID_ARG, "NULL tensor pointer");
  AppendArgs a{};
  a.q = q;
  a.q_token = q_token_stride;
  a.q_head = q_head_stride;
  a.q_heads = q ? q_heads : 0;
  a.k = k;
  a.k_token = k_token_stride;
  a.k_head = k_head_stride;
  a.v = v;
  a.v_token = v_token_stride;
  a.v_head = v_head_stride;
  a.q_start = q_start;
  a.cache_len = cache_len;
  a.B = B;
  a.T = T;
  a.rope = rope;
  a.rope_positions = rope ? rope_positions : 0;
  a.rot = rope ? rot : 0;
  a.interleaved = interleaved != 0;
  a.cache = *cache;
  a.q_out = q_out;
  a.qo_token = q_out_token_stride;
  a.qo_head = q_out_head_stride;
  const cudaError_t e = launch_kv_append(a, stream);
  return e == cudaSuccess ? RETRACE_OK : cuda_fail(e, "append kernel launch");
}

size_t retrace_attend_workspace_bytes(int q_heads, int kv_heads, int head_dim, retrace_dtype dtype) {
  if (kv_heads < 1 || q_heads < 1 || q_heads % kv_heads || head_dim < 1 || head_dim > kMaxHeadDim || !dtype_ok(dtype))
    return 0;
  const size_t tc = dtype == RETRACE_BF16 ? attend_tc_partial_bytes(head_dim) : 0;
  return kAttendPartials + std::max(attend_simt_partial_bytes(head_dim), tc);
}

retrace_status retrace_attend(const void* q, int64_t q_token_stride, int64_t q_head_stride, int q_heads,
                              const int32_t* q_start, const int32_t* cache_len, int B, int T, float scale, int window,
                              int sinks, int causal, const retrace_kv_cache* cache, void* out,
                              int64_t out_token_stride, int64_t out_head_stride, void* ws, size_t ws_bytes,
                              cudaStream_t stream) {
  set_last_error("");
  retrace_status st = check_cache(cache, q_heads, B, T, q_start, cache_len);
  if (st != RETRACE_OK) return st;
  if (!(scale > -3.0e38f && scale < 3.0e38f)) return fail(RETRACE_ERR_INVALID_ARG, "scale must be finite");
  if (window < 0 || sinks < 0) return fail(RETRACE_ERR_INVALID_ARG, "window=%d and sinks=%d must not be negative", window, sinks);
  if (q_token_stride < 0 || q_head_stride < 0 || out_token_stride < 0 || out_head_stride < 0)
    return fail(RETRACE_ERR_INVALID_ARG, "negative stride");
  if (T == 0) return RETRACE_OK;
  if (!q || !out) return fail(RETRACE_ERR_INVALID_ARG, "NULL tensor pointer");
  const size_t need = retrace_attend_workspace_bytes(q_heads, cache->kv_heads, cache->head_dim, cache->dtype);
  if (!ws) return fail(RETRACE_ERR_WORKSPACE, "workspace pointer is NULL");
  if (((uintptr_t)ws & 255u) != 0) return fail(RETRACE_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (ws_bytes < need)
    return fail(RETRACE_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", ws_bytes, need);
  AttendArgs a{};
  a.q = q;
  a.q_token = q_token_stride;
  a.q_head = q_head_stride;
  a.q_heads = q_heads;
  a.q_start = q_start;
  a.cache_len = cache_len;
  a.B = B;
  a.T = T;
  a.scale = scale;
  a.window = window < (1 << 30) ? window : 0;  // no position is that far back
  a.sinks = a.window > 0 ? sinks : 0;
  a.causal = causal != 0;
  a.cache = *cache;
  a.out = out;
  a.out_token = out_token_stride;
  a.out_head = out_head_stride;
  char* w = static_cast<char*>(ws);
  a.status = reinterpret_cast<uint32_t*>(w);
  a.units = reinterpret_cast<JoinUnit*>(w + kAttendUnits);
  a.tickets = reinterpret_cast<uint32_t*>(w + kAttendTickets);
  a.partials = reinterpret_cast<float*>(w + kAttendPartials);
  const cudaError_t e = attend_tc_supported(a) ? launch_attend_tc(a, stream) : launch_attend_simt(a, stream);
  return e == cudaSuccess ? RETRACE_OK : cuda_fail(e, "attention kernel launch");
}

retrace_status retrace_sample(const void* logits, retrace_dtype dtype, int B, int R, int V, int64_t row_stride,
                              int64_t batch_stride, const float* uniforms, const float* temperature,
                              const int32_t* top_k, const float* top_p, const float* min_p, int32_t* tokens,
                              float* probs, cudaStream_t stream) {
  set_last_error("");
  if (!dtype_ok(dtype)) return fail(RETRACE_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  if (B < 0 || R < 0 || V < 1) return fail(RETRACE_ERR_INVALID_ARG, "bad shape B=%d R=%d V=%d", B, R, V);
  if ((long long)B * R > (1ll << 30)) return fail(RETRACE_ERR_UNSUPPORTED, "B*R exceeds 2^30 rows");
  if (V > (1 << 24)) return fail(RETRACE_ERR_UNSUPPORTED, "V=%d exceeds 2^24", V);
  if (row_stride < 0 || batch_stride < 0) return fail(RETRACE_ERR_INVALID_ARG, "negative stride");
  if (B == 0 || R == 0) return RETRACE_OK;
  if (!logits || !uniforms || !tokens) return fail(RETRACE_ERR_INVALID_ARG, "NULL tensor pointer");
  SampleArgs a{logits, B, R, V, row_stride, batch_stride, uniforms, temperature, top_k, top_p, min_p, tokens, probs};
  const cudaError_t e = launch_sample(a, dtype, stream);
  return e == cudaSuccess ? RETRACE_OK : cuda_fail(e, "sampling kernel launch");
}

}  // extern "C"
