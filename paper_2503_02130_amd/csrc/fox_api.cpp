// C ABI of the Forgetting Attention library: argument validation on the host,
// then kernel launches on the caller's stream.  Nothing here allocates device
// memory or synchronises.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "fox.h"
#include "fox_internal.h"

namespace {

constexpr long long kMaxElems = 1LL << 40;        // per tensor
// Workgroups per launch at 64 rows each; kernels of 1024 threads, or of fewer rows, bring
// more threads than a launch takes and are launched in parts or loop.
constexpr long long kMaxWorkgroups = 1LL << 22;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

fox_status_t check_dims(int B, int H, int L, int d) {
  if (B <= 0 || H <= 0 || L <= 0 || d <= 0) return FOX_ERR_SHAPE;
  const long long bh = (long long)B * H;
  if (bh > (1LL << 30)) return FOX_ERR_SHAPE;
  if (bh * L > (1LL << 31) - 1) return FOX_ERR_SHAPE;          // row index fits in int
  if (bh * L * d > kMaxElems) return FOX_ERR_SHAPE;
  if ((long long)L * d * 4 >= (1LL << 31)) return FOX_ERR_SHAPE;  // one head addressed in 32 bits
  if (bh * ((L + 63) / 64) > kMaxWorkgroups) return FOX_ERR_SHAPE;
  return FOX_OK;
}

fox_status_t check_dtype_d(int dtype, int d) {
  if (dtype != FOX_DTYPE_F32 && dtype != FOX_DTYPE_BF16) return FOX_ERR_UNSUPPORTED;
  if (d != 64 && d != 128) return FOX_ERR_UNSUPPORTED;
  return FOX_OK;
}

fox_status_t launch_status(hipError_t e) { return e == hipSuccess ? FOX_OK : FOX_ERR_HIP; }

fox_status_t check_projection(int dtype, int B, int L, int H, int M) {
  if (B <= 0 || L <= 0 || H <= 0 || M <= 0) return FOX_ERR_SHAPE;
  const long long n = (long long)B * L;
  if (n > (1LL << 31) - 1 || (long long)B * H * L > (1LL << 31) - 1) return FOX_ERR_SHAPE;
  if (n * M > kMaxElems) return FOX_ERR_SHAPE;
  if (dtype != FOX_DTYPE_F32 && dtype != FOX_DTYPE_BF16) return FOX_ERR_UNSUPPORTED;
  if (H > 64 || M % 8 != 0) return FOX_ERR_UNSUPPORTED;
  return FOX_OK;
}

bool valid_eps(float eps) { return isfinite(eps) && eps >= 0.0f; }

bool all_aligned16(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!aligned16(p)) return false;
  return true;
}

bool all_set(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (!p) return false;
  return true;
}

// The cache descriptor: its sizes, then its pointers.
fox_status_t check_cache(const fox_cache_t* c) {
  if (!c) return FOX_ERR_NULL;
  if (c->n_pages <= 0 || c->max_pages <= 0 || c->B <= 0 || c->H <= 0 || c->H_kv <= 0)
    return FOX_ERR_SHAPE;
  if (c->H % c->H_kv != 0) return FOX_ERR_SHAPE;
  if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1)) != 0) return FOX_ERR_SHAPE;
  if ((long long)c->max_pages * c->page > (1LL << 30)) return FOX_ERR_SHAPE;
  // every workgroup of the attention looks through the lengths
  if (c->B > (1 << 16) || (long long)c->B * c->H > (1LL << 22)) return FOX_ERR_SHAPE;
  if ((long long)c->n_pages * c->H * c->page > kMaxElems / 128) return FOX_ERR_SHAPE;
  if ((long long)c->H * c->page > (1LL << 28)) return FOX_ERR_SHAPE;  // a page of c in 32 bits
  if (c->format != FOX_CACHE_BF16 && c->format != FOX_CACHE_E4M3) return FOX_ERR_UNSUPPORTED;
  if (c->d != 64 && c->d != 128) return FOX_ERR_UNSUPPORTED;
  if (!all_set({c->k, c->v, c->c, c->page_table})) return FOX_ERR_NULL;
  if (c->format == FOX_CACHE_E4M3 && !all_set({c->k_exp, c->v_exp})) return FOX_ERR_NULL;
  if (!all_aligned16({c->k, c->v, c->c, c->page_table, c->k_exp, c->v_exp})) return FOX_ERR_ALIGN;
  return FOX_OK;
}

fox::CacheSpec cache_spec(const fox_cache_t* c) {
  return fox::CacheSpec{c->format == FOX_CACHE_E4M3, c->k, c->v, c->k_exp, c->v_exp, c->c,
                        c->page_table, c->n_pages, c->page, c->max_pages, c->B, c->H, c->H_kv,
                        c->d};
}

bool cache_dtype(int dtype) { return dtype == FOX_DTYPE_F32 || dtype == FOX_DTYPE_BF16; }

constexpr int kMaxNewTokens = 64;

// New tokens of a call.  Its largest launch has a workgroup of 256 for each of the B H n rows.
bool cache_new_ok(const fox_cache_t* c, int n) {
  return n >= 1 && n <= kMaxNewTokens && (long long)c->B * c->H * n <= (1LL << 22);
}
// Rows of a copy to or from the cache, for each head c and for each key head d / 8 threads.
bool cache_rows_ok(const fox_cache_t* c, long long rows) {
  return rows > 0 && rows * c->H <= (1LL << 31) - 1 &&
         rows * (c->H + (long long)c->H_kv * (c->d / 8)) < (1LL << 32) - 1024;
}

int cache_max_len(const fox_cache_t* c, int max_len) {
  const int cap = c->max_pages * c->page;
  return max_len <= 0 || max_len > cap ? cap : max_len;
}

fox_status_t check_packed(int B, int H, int H_kv, int N) {
  if (B <= 0 || H <= 0 || H_kv <= 0 || N <= 0 || H % H_kv != 0) return FOX_ERR_SHAPE;
  if ((long long)H * N > (1LL << 31) - 1) return FOX_ERR_SHAPE;
  if ((long long)B * H > (1LL << 21)) return FOX_ERR_SHAPE;  // a workgroup each, 1024 threads
  if ((long long)H * fox::packed_items(B, N) > kMaxWorkgroups) return FOX_ERR_SHAPE;
  return FOX_OK;
}

// The bf16 kernels hold (c_i - c_j) / scale in fp32.
bool packed_scale_ok(int dtype, float scale) {
  return dtype != FOX_DTYPE_BF16 || (isfinite(scale) && fabsf(scale) >= 0x1p-64f);
}

fox_status_t zero_rows(const fox_packed_rows_t* tensors, int n, fox::ZeroRows* x) {
  if (n < 0 || n > fox::kZeroTensors) return FOX_ERR_SHAPE;
  if (n > 0 && !tensors) return FOX_ERR_NULL;
  for (int i = 0; i < n; ++i) {
    if (!tensors[i].x) return FOX_ERR_NULL;
    if (tensors[i].heads <= 0 || tensors[i].row_bytes <= 0 || tensors[i].row_bytes % 2)
      return FOX_ERR_SHAPE;
    if (!aligned16(tensors[i].x)) return FOX_ERR_ALIGN;
    x[i] = fox::ZeroRows{tensors[i].x, tensors[i].heads, tensors[i].row_bytes};
  }
  return FOX_OK;
}

}  // namespace

extern "C" {

const char* fox_status_string(fox_status_t status) {
  switch (status) {
    case FOX_OK: return "FOX_OK";
    case FOX_ERR_NULL: return "FOX_ERR_NULL: a required pointer is NULL";
    case FOX_ERR_SHAPE: return "FOX_ERR_SHAPE: sizes must be positive and within limits";
    case FOX_ERR_UNSUPPORTED: return "FOX_ERR_UNSUPPORTED: dtype must be f32/bf16, head dim 64/128";
    case FOX_ERR_ALIGN: return "FOX_ERR_ALIGN: device pointers must be 16-byte aligned";
    case FOX_ERR_WORKSPACE: return "FOX_ERR_WORKSPACE: workspace missing or too small";
    case FOX_ERR_HIP: return "FOX_ERR_HIP: the HIP runtime reported a launch error";
    case FOX_ERR_VALUE: return "FOX_ERR_VALUE: a scalar argument is out of range (eps: finite, >= 0; scale of a "
                                "packed bf16 call: finite, at least 2^-64 in magnitude)";
    case FOX_ERR_TOO_LARGE:
      return "FOX_ERR_TOO_LARGE: the shape needs more scratch than fox_attn_decode_noalloc holds "
             "(64 MiB of split partials); use fox_attn_decode with a workspace";
    default: return "unknown fox status";
  }
}

int fox_version(void) { return 100; }

fox_status_t fox_gate_prefix(const float* gate_logit, float* log_f, float* c, int B, int H, int L,
                    hipStream_t stream) {
  if (!gate_logit || !c) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, 1);
  if (st) return st;
  if (!aligned16(gate_logit) || !aligned16(c) || (log_f && !aligned16(log_f))) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_gate_prefix(gate_logit, log_f, c, B * H, L,
                                               static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_fwd(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c, void* o,
                 float* lse, int B, int H, int L, int d, float scale, hipStream_t stream) {
  if (!q || !k || !v || !c || !o || !lse) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(c) || !aligned16(o) ||
      !aligned16(lse))
    return FOX_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == FOX_DTYPE_BF16)
    return launch_status(fox::launch_fwd_bf16(q, k, v, fox::gate_array(c), o, lse, B * H, L, d, scale, s));
  return launch_status(fox::launch_fwd_f32((const float*)q, (const float*)k, (const float*)v,
                                           fox::gate_array(c), (float*)o, lse, B * H, L, d, scale,
                                           s));
}

size_t fox_attn_bwd_workspace_bytes(fox_dtype_t dtype, int B, int H, int L, int d) {
  if (check_dims(B, H, L, d) || check_dtype_d(dtype, d)) return 0;
  return fox::bwd_workspace_bytes(B * H, L);
}

fox_status_t fox_attn_bwd(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c,
                 const void* o, const float* lse, const void* d_o, void* dq, void* dk, void* dv,
                 float* d_log_f, void* workspace, size_t workspace_bytes, int B, int H, int L,
                 int d, float scale, hipStream_t stream) {
  if (!q || !k || !v || !c || !o || !lse || !d_o || !dq || !dk || !dv || !d_log_f)
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(c) || !aligned16(o) ||
      !aligned16(lse) || !aligned16(d_o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) ||
      !aligned16(d_log_f))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::bwd_workspace_bytes(B * H, L)) return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd(dtype == FOX_DTYPE_BF16, q, k, v, c, o, lse, d_o, dq, dk,
                                       dv, d_log_f, workspace, B * H, L, d, scale,
                                       static_cast<hipStream_t>(stream)));
}

size_t fox_attn_bwd_stored_workspace_bytes(fox_dtype_t dtype, int B, int H, int L, int d) {
  if (check_dims(B, H, L, d) || check_dtype_d(dtype, d) || dtype != FOX_DTYPE_BF16) return 0;
  return fox::bwd_stored_workspace_bytes(B * H, L);
}

fox_status_t fox_attn_bwd_stored(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c,
                        const void* o, const float* lse, const void* d_o, void* dq, void* dk,
                        void* dv, float* d_log_f, void* workspace, size_t workspace_bytes, int B,
                        int H, int L, int d, float scale, hipStream_t stream) {
  if (!q || !k || !v || !c || !o || !lse || !d_o || !dq || !dk || !dv || !d_log_f)
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (dtype != FOX_DTYPE_BF16) return FOX_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(c) || !aligned16(o) ||
      !aligned16(lse) || !aligned16(d_o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) ||
      !aligned16(d_log_f))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::bwd_stored_workspace_bytes(B * H, L))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_stored(q, k, v, c, o, lse, d_o, dq, dk, dv, d_log_f,
                                              workspace, B * H, L, d, scale,
                                              static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_bwd_delta(fox_dtype_t dtype, const void* o, const void* d_o, float* delta, int B, int H,
                       int L, int d, hipStream_t stream) {
  if (!o || !d_o || !delta) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(o) || !aligned16(d_o) || !aligned16(delta)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_delta(dtype == FOX_DTYPE_BF16, o, d_o, delta, B * H, L, d,
                                             static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_bwd_dkdv(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c,
                      const float* lse, const void* d_o, const float* delta, void* dk, void* dv,
                      float* dc_k, int B, int H, int L, int d, float scale, hipStream_t stream) {
  if (!q || !k || !v || !c || !lse || !d_o || !delta || !dk || !dv || !dc_k) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(c) || !aligned16(lse) ||
      !aligned16(d_o) || !aligned16(delta) || !aligned16(dk) || !aligned16(dv) ||
      !aligned16(dc_k))
    return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_dkdv(dtype == FOX_DTYPE_BF16, q, k, v, fox::gate_array(c), lse, d_o, delta,
                                            dk, dv, dc_k, B * H, L, d, scale,
                                            static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_bwd_dq(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c,
                    const float* lse, const void* d_o, const float* delta, void* dq, float* dc_q,
                    int B, int H, int L, int d, float scale, hipStream_t stream) {
  if (!q || !k || !v || !c || !lse || !d_o || !delta || !dq || !dc_q) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(c) || !aligned16(lse) ||
      !aligned16(d_o) || !aligned16(delta) || !aligned16(dq) || !aligned16(dc_q))
    return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_dq(dtype == FOX_DTYPE_BF16, q, k, v, fox::gate_array(c), lse, d_o, delta,
                                          dq, dc_q, B * H, L, d, scale,
                                          static_cast<hipStream_t>(stream)));
}

size_t fox_attn_bwd_ds_store_bytes(fox_dtype_t dtype, int B, int H, int L, int d) {
  if (check_dims(B, H, L, d) || check_dtype_d(dtype, d) || dtype != FOX_DTYPE_BF16) return 0;
  return fox::ds_store_bytes(B * H, L);
}

fox_status_t fox_attn_bwd_dkdv_store(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                            const float* c, const float* lse, const void* d_o,
                            const float* delta, void* dk, void* dv, float* dc_k, void* ds_store,
                            size_t ds_store_bytes, int B, int H, int L, int d, float scale,
                            hipStream_t stream) {
  if (!q || !k || !v || !c || !lse || !d_o || !delta || !dk || !dv || !dc_k) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (dtype != FOX_DTYPE_BF16) return FOX_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(c) || !aligned16(lse) ||
      !aligned16(d_o) || !aligned16(delta) || !aligned16(dk) || !aligned16(dv) ||
      !aligned16(dc_k))
    return FOX_ERR_ALIGN;
  if (!ds_store || ds_store_bytes < fox::ds_store_bytes(B * H, L)) return FOX_ERR_WORKSPACE;
  if (!aligned16(ds_store)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_dkdv_store(q, k, v, fox::gate_array(c), lse, d_o, delta,
                                                  dk, dv, dc_k, ds_store, nullptr, B * H, L, d,
                                                  scale, static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_bwd_dq_stored(fox_dtype_t dtype, const void* k, const void* ds_store, size_t ds_store_bytes,
                           void* dq, float* dc_q, int B, int H, int L, int d, float scale,
                           hipStream_t stream) {
  if (!k || !dq || !dc_q) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (dtype != FOX_DTYPE_BF16) return FOX_ERR_UNSUPPORTED;
  if (!aligned16(k) || !aligned16(dq) || !aligned16(dc_q)) return FOX_ERR_ALIGN;
  if (!ds_store || ds_store_bytes < fox::ds_store_bytes(B * H, L)) return FOX_ERR_WORKSPACE;
  if (!aligned16(ds_store)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_dq_stored(k, ds_store, nullptr, dq, dc_q, B * H, L, d,
                                                 scale, static_cast<hipStream_t>(stream)));
}

fox_status_t fox_dlogf_from_dc(const float* dc_q, const float* dc_k, float* d_log_f, int B, int H, int L,
                      hipStream_t stream) {
  if (!dc_q || !dc_k || !d_log_f) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, 1);
  if (st) return st;
  if (!aligned16(dc_q) || !aligned16(dc_k) || !aligned16(d_log_f)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_reverse_scan_sum(dc_q, dc_k, d_log_f, B * H, L,
                                                    static_cast<hipStream_t>(stream)));
}

fox_status_t fox_dlogit_from_dc(const float* dc_q, const float* dc_k, const float* gate_logit,
                       float* d_log_f, float* d_logit, int B, int H, int L, hipStream_t stream) {
  if (!dc_q || !dc_k || !gate_logit || !d_logit) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, 1);
  if (st) return st;
  if (!aligned16(dc_q) || !aligned16(dc_k) || !aligned16(gate_logit) || !aligned16(d_logit) ||
      (d_log_f && !aligned16(d_log_f)))
    return FOX_ERR_ALIGN;
  return launch_status(fox::launch_reverse_scan_gate(dc_q, dc_k, gate_logit, d_log_f, d_logit,
                                                     B * H, L, static_cast<hipStream_t>(stream)));
}

size_t fox_attn_decode_workspace_bytes(fox_dtype_t dtype, int B, int H, int T, int d) {
  if (check_dims(B, H, T, d) || check_dtype_d(dtype, d)) return 0;
  return fox::decode_workspace_bytes(dtype == FOX_DTYPE_BF16, B * H, T, d);
}

fox_status_t fox_attn_decode(fox_dtype_t dtype, const void* q, const void* k_cache, const void* v_cache,
                    float* c_cache, const float* gate_logit_new, void* o, float* lse,
                    void* workspace, size_t workspace_bytes, int B, int H, int T, int d,
                    float scale, hipStream_t stream) {
  if (!q || !k_cache || !v_cache || !c_cache || !gate_logit_new || !o || !lse)
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, T, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(c_cache) ||
      !aligned16(gate_logit_new) || !aligned16(o) || !aligned16(lse))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::decode_min_workspace_bytes(B * H, T, d))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_decode(dtype == FOX_DTYPE_BF16, q, k_cache, v_cache, c_cache,
                                          gate_logit_new, o, lse, workspace, workspace_bytes,
                                          B * H, T, d, scale,
                                          static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_decode_noalloc(fox_dtype_t dtype, const void* q, const void* k_cache,
                                     const void* v_cache, float* c_cache,
                                     const float* gate_logit_new, void* o, float* lse, int B,
                                     int H, int T, int d, float scale, hipStream_t stream) {
  if (!q || !k_cache || !v_cache || !c_cache || !gate_logit_new || !o || !lse)
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, T, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(c_cache) ||
      !aligned16(gate_logit_new) || !aligned16(o) || !aligned16(lse))
    return FOX_ERR_ALIGN;
  if (fox::decode_min_workspace_bytes(B * H, T, d) > fox::kDecodeScratchBytes)
    return FOX_ERR_TOO_LARGE;
  return launch_status(fox::launch_decode_noalloc(dtype == FOX_DTYPE_BF16, q, k_cache, v_cache,
                                                  c_cache, gate_logit_new, o, lse, B * H, T, d,
                                                  scale, stream));
}

// ------------------------------------------------------- gate-aware skipping
fox_status_t fox_row_norm_max(fox_dtype_t dtype, const void* x, float* out, int B, int H, int L, int d,
                     hipStream_t stream) {
  if (!x || !out) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(x) || !aligned16(out)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_row_norm_max(dtype == FOX_DTYPE_BF16, x, out, B * H, L, d,
                                                static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_fwd_skip(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c,
                      const float* q_norm_max, const float* k_norm_max, void* o, float* lse,
                      int B, int H, int L, int d, float scale, hipStream_t stream) {
  if (!q || !k || !v || !c || !q_norm_max || !k_norm_max || !o || !lse) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(c) ||
      !aligned16(q_norm_max) || !aligned16(k_norm_max) || !aligned16(o) || !aligned16(lse))
    return FOX_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == FOX_DTYPE_BF16)
    return launch_status(fox::launch_fwd_bf16(q, k, v, fox::gate_array(c), o, lse, B * H, L, d,
                                              scale, s, q_norm_max, k_norm_max));
  return launch_status(fox::launch_fwd_f32((const float*)q, (const float*)k, (const float*)v,
                                           fox::gate_array(c), (float*)o, lse, B * H, L, d, scale,
                                           s));
}

fox_status_t fox_attn_bwd_skip(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c,
                      const void* o, const float* lse, const void* d_o, const float* q_norm_max,
                      const float* k_norm_max, void* dq, void* dk, void* dv, float* d_log_f,
                      void* workspace, size_t workspace_bytes, int B, int H, int L, int d,
                      float scale, hipStream_t stream) {
  if (!q || !k || !v || !c || !o || !lse || !d_o || !q_norm_max || !k_norm_max || !dq || !dk ||
      !dv || !d_log_f)
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(c) || !aligned16(o) ||
      !aligned16(lse) || !aligned16(d_o) || !aligned16(q_norm_max) || !aligned16(k_norm_max) ||
      !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned16(d_log_f))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::bwd_workspace_bytes(B * H, L)) return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  const bool bf = dtype == FOX_DTYPE_BF16;
  return launch_status(fox::launch_bwd(bf, q, k, v, c, o, lse, d_o, dq, dk, dv, d_log_f,
                                       workspace, B * H, L, d, scale,
                                       static_cast<hipStream_t>(stream), bf ? q_norm_max : nullptr,
                                       bf ? k_norm_max : nullptr));
}

fox_status_t fox_attn_bwd_skip_stored(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                             const float* c, const void* o, const float* lse, const void* d_o,
                             const float* q_norm_max, const float* k_norm_max, void* dq, void* dk,
                             void* dv, float* d_log_f, void* workspace, size_t workspace_bytes,
                             int B, int H, int L, int d, float scale, hipStream_t stream) {
  if (!all_set({q, k, v, c, o, lse, d_o, q_norm_max, k_norm_max, dq, dk, dv, d_log_f}))
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (dtype != FOX_DTYPE_BF16) return FOX_ERR_UNSUPPORTED;
  if (!all_aligned16({q, k, v, c, o, lse, d_o, q_norm_max, k_norm_max, dq, dk, dv, d_log_f}))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::bwd_stored_workspace_bytes(B * H, L))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_stored(q, k, v, c, o, lse, d_o, dq, dk, dv, d_log_f,
                                              workspace, B * H, L, d, scale,
                                              static_cast<hipStream_t>(stream), q_norm_max,
                                              k_norm_max));
}

fox_status_t fox_attn_decode_skip(fox_dtype_t dtype, const void* q, const void* k_cache, const void* v_cache,
                         float* c_cache, const float* gate_logit_new, const float* k_norm_max,
                         void* o, float* lse, void* workspace, size_t workspace_bytes, int B,
                         int H, int T, int d, float scale, hipStream_t stream) {
  if (!q || !k_cache || !v_cache || !c_cache || !gate_logit_new || !k_norm_max || !o || !lse)
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, T, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(c_cache) ||
      !aligned16(gate_logit_new) || !aligned16(k_norm_max) || !aligned16(o) || !aligned16(lse))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::decode_min_workspace_bytes(B * H, T, d))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_decode_skip(dtype == FOX_DTYPE_BF16, q, k_cache, v_cache,
                                               c_cache, gate_logit_new, k_norm_max, o, lse,
                                               workspace, workspace_bytes, B * H, T, d, scale,
                                               static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------- fixed gates
fox_status_t fox_fixed_gate_init(float* gate_bias, int H, float t_min, float t_max) {
  if (!gate_bias) return FOX_ERR_NULL;
  if (H <= 0 || !(t_min > 0.0f) || !(t_max >= t_min) || !isfinite(t_max)) return FOX_ERR_SHAPE;
  for (int h = 0; h < H; ++h) {
    const double frac = H > 1 ? (double)h / (double)(H - 1) : 0.0;
    const double T = exp(log((double)t_min) + (log((double)t_max) - log((double)t_min)) * frac);
    // sigmoid(b) = exp(-1/T)  <=>  b = log(e^{-1/T} / (1 - e^{-1/T}))
    gate_bias[h] = (float)(-1.0 / T - log(-expm1(-1.0 / T)));
  }
  return FOX_OK;
}

fox_status_t fox_attn_fwd_fixed_gate(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                            const float* gate_bias, void* o, float* lse, int B, int H, int L, int d,
                            float scale, hipStream_t stream) {
  if (!q || !k || !v || !gate_bias || !o || !lse) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(gate_bias) || !aligned16(o) ||
      !aligned16(lse))
    return FOX_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const fox::GateSpec g = fox::gate_fixed(gate_bias, H);
  if (dtype == FOX_DTYPE_BF16)
    return launch_status(fox::launch_fwd_bf16(q, k, v, g, o, lse, B * H, L, d, scale, s));
  return launch_status(fox::launch_fwd_f32((const float*)q, (const float*)k, (const float*)v, g,
                                           (float*)o, lse, B * H, L, d, scale, s));
}

size_t fox_attn_bwd_fixed_gate_workspace_bytes(fox_dtype_t dtype, int B, int H, int L, int d) {
  if (check_dims(B, H, L, d) || check_dtype_d(dtype, d)) return 0;
  return fox::bwd_fixed_workspace_bytes(B * H, L);
}

fox_status_t fox_attn_bwd_fixed_gate(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                            const float* gate_bias, const void* o, const float* lse,
                            const void* d_o, void* dq, void* dk, void* dv, float* d_gate_bias,
                            void* workspace, size_t workspace_bytes, int B, int H, int L, int d,
                            float scale, hipStream_t stream) {
  if (!q || !k || !v || !gate_bias || !o || !lse || !d_o || !dq || !dk || !dv)
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(gate_bias) || !aligned16(o) ||
      !aligned16(lse) || !aligned16(d_o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) ||
      (d_gate_bias && !aligned16(d_gate_bias)))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::bwd_fixed_workspace_bytes(B * H, L))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_fixed(dtype == FOX_DTYPE_BF16, q, k, v, gate_bias, H, o,
                                             lse, d_o, dq, dk, dv, d_gate_bias, workspace, B * H,
                                             L, d, scale, static_cast<hipStream_t>(stream)));
}

size_t fox_attn_bwd_fixed_gate_stored_workspace_bytes(fox_dtype_t dtype, int B, int H, int L, int d) {
  if (check_dims(B, H, L, d) || check_dtype_d(dtype, d) || dtype != FOX_DTYPE_BF16) return 0;
  return fox::bwd_fixed_stored_workspace_bytes(B * H, L);
}

// fox_attn_bwd_fixed_gate_stored and its skipping twin (norms non-NULL)
static fox_status_t bwd_fixed_stored(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                            const float* gate_bias, const void* o, const float* lse,
                            const void* d_o, const float* q_norm_max, const float* k_norm_max,
                            void* dq, void* dk, void* dv, float* d_gate_bias, void* workspace,
                            size_t workspace_bytes, int B, int H, int L, int d, float scale,
                            hipStream_t stream) {
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (dtype != FOX_DTYPE_BF16) return FOX_ERR_UNSUPPORTED;
  if (!all_aligned16({q, k, v, gate_bias, o, lse, d_o, dq, dk, dv}) ||
      (q_norm_max && !all_aligned16({q_norm_max, k_norm_max})) ||
      (d_gate_bias && !aligned16(d_gate_bias)))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::bwd_fixed_stored_workspace_bytes(B * H, L))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_fixed_stored(q, k, v, gate_bias, H, o, lse, d_o, dq, dk,
                                                    dv, d_gate_bias, workspace, B * H, L, d,
                                                    scale, static_cast<hipStream_t>(stream),
                                                    q_norm_max, k_norm_max));
}

fox_status_t fox_attn_bwd_fixed_gate_stored(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                                   const float* gate_bias, const void* o, const float* lse,
                                   const void* d_o, void* dq, void* dk, void* dv,
                                   float* d_gate_bias, void* workspace, size_t workspace_bytes,
                                   int B, int H, int L, int d, float scale, hipStream_t stream) {
  if (!all_set({q, k, v, gate_bias, o, lse, d_o, dq, dk, dv})) return FOX_ERR_NULL;
  return bwd_fixed_stored(dtype, q, k, v, gate_bias, o, lse, d_o, nullptr, nullptr, dq, dk, dv,
                          d_gate_bias, workspace, workspace_bytes, B, H, L, d, scale, stream);
}

fox_status_t fox_attn_bwd_fixed_gate_skip_stored(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                                        const float* gate_bias, const void* o, const float* lse,
                                        const void* d_o, const float* q_norm_max,
                                        const float* k_norm_max, void* dq, void* dk, void* dv,
                                        float* d_gate_bias, void* workspace,
                                        size_t workspace_bytes, int B, int H, int L, int d,
                                        float scale, hipStream_t stream) {
  if (!all_set({q, k, v, gate_bias, o, lse, d_o, q_norm_max, k_norm_max, dq, dk, dv}))
    return FOX_ERR_NULL;
  return bwd_fixed_stored(dtype, q, k, v, gate_bias, o, lse, d_o, q_norm_max, k_norm_max, dq, dk,
                          dv, d_gate_bias, workspace, workspace_bytes, B, H, L, d, scale, stream);
}

fox_status_t fox_attn_decode_fixed_gate(fox_dtype_t dtype, const void* q, const void* k_cache,
                               const void* v_cache, const float* gate_bias, void* o, float* lse,
                               void* workspace, size_t workspace_bytes, int B, int H, int T, int d,
                               float scale, hipStream_t stream) {
  if (!q || !k_cache || !v_cache || !gate_bias || !o || !lse) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, T, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(gate_bias) ||
      !aligned16(o) || !aligned16(lse))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::decode_min_workspace_bytes(B * H, T, d))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_decode_fixed(dtype == FOX_DTYPE_BF16, q, k_cache, v_cache,
                                                gate_bias, H, o, lse, workspace, workspace_bytes,
                                                B * H, T, d, scale, static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_fwd_fixed_gate_skip(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                                 const float* gate_bias, const float* q_norm_max,
                                 const float* k_norm_max, void* o, float* lse, int B, int H, int L,
                                 int d, float scale, hipStream_t stream) {
  if (!all_set({q, k, v, gate_bias, q_norm_max, k_norm_max, o, lse})) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!all_aligned16({q, k, v, gate_bias, q_norm_max, k_norm_max, o, lse})) return FOX_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const fox::GateSpec g = fox::gate_fixed(gate_bias, H);
  if (dtype == FOX_DTYPE_BF16)
    return launch_status(
        fox::launch_fwd_bf16(q, k, v, g, o, lse, B * H, L, d, scale, s, q_norm_max, k_norm_max));
  return launch_status(fox::launch_fwd_f32((const float*)q, (const float*)k, (const float*)v, g,
                                           (float*)o, lse, B * H, L, d, scale, s));
}

fox_status_t fox_attn_bwd_fixed_gate_skip(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                                 const float* gate_bias, const void* o, const float* lse,
                                 const void* d_o, const float* q_norm_max,
                                 const float* k_norm_max, void* dq, void* dk, void* dv,
                                 float* d_gate_bias, void* workspace, size_t workspace_bytes,
                                 int B, int H, int L, int d, float scale, hipStream_t stream) {
  if (!all_set({q, k, v, gate_bias, o, lse, d_o, q_norm_max, k_norm_max, dq, dk, dv}))
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!all_aligned16({q, k, v, gate_bias, o, lse, d_o, q_norm_max, k_norm_max, dq, dk, dv}) ||
      (d_gate_bias && !aligned16(d_gate_bias)))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::bwd_fixed_workspace_bytes(B * H, L))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  const bool bf = dtype == FOX_DTYPE_BF16;
  return launch_status(fox::launch_bwd_fixed(bf, q, k, v, gate_bias, H, o, lse, d_o, dq, dk, dv,
                                             d_gate_bias, workspace, B * H, L, d, scale,
                                             static_cast<hipStream_t>(stream),
                                             bf ? q_norm_max : nullptr, bf ? k_norm_max : nullptr));
}

fox_status_t fox_attn_decode_fixed_gate_skip(fox_dtype_t dtype, const void* q, const void* k_cache,
                                    const void* v_cache, const float* gate_bias,
                                    const float* k_norm_max, void* o, float* lse, void* workspace,
                                    size_t workspace_bytes, int B, int H, int T, int d,
                                    float scale, hipStream_t stream) {
  if (!all_set({q, k_cache, v_cache, gate_bias, k_norm_max, o, lse})) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, T, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!all_aligned16({q, k_cache, v_cache, gate_bias, k_norm_max, o, lse})) return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::decode_min_workspace_bytes(B * H, T, d))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_decode_fixed(dtype == FOX_DTYPE_BF16, q, k_cache, v_cache,
                                                gate_bias, H, o, lse, workspace, workspace_bytes,
                                                B * H, T, d, scale, static_cast<hipStream_t>(stream),
                                                k_norm_max));
}

// ---------------------------------------------------------------------------
// FoX (Pro) prologue and epilogue
// ---------------------------------------------------------------------------
fox_status_t fox_pro_prologue(fox_dtype_t dtype, const void* q_raw, const void* k_raw, const void* v_raw,
                     const float* k_shift_logit, const float* v_shift_logit,
                     const float* q_norm_weight, const float* k_norm_weight, float eps, void* q,
                     void* k, void* v, int B, int H, int L, int d, hipStream_t stream) {
  if (!all_set({q_raw, k_raw, v_raw, k_shift_logit, v_shift_logit, q_norm_weight, k_norm_weight,
                q, k, v}))
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!valid_eps(eps)) return FOX_ERR_VALUE;
  if (!all_aligned16({q_raw, k_raw, v_raw, k_shift_logit, v_shift_logit, q_norm_weight,
                      k_norm_weight, q, k, v}))
    return FOX_ERR_ALIGN;
  return launch_status(fox::launch_pro_prologue(
      dtype == FOX_DTYPE_BF16, q_raw, k_raw, v_raw, k_shift_logit, v_shift_logit, q_norm_weight,
      k_norm_weight, eps, q, k, v, H, B * H, L, d, static_cast<hipStream_t>(stream)));
}

size_t fox_pro_prologue_bwd_workspace_bytes(fox_dtype_t dtype, int B, int H, int L, int d) {
  if (check_dims(B, H, L, d) || check_dtype_d(dtype, d)) return 0;
  return fox::pro_prologue_bwd_workspace_bytes(B * H, L, d);
}

fox_status_t fox_pro_prologue_bwd(fox_dtype_t dtype, const void* q_raw, const void* k_raw, const void* v_raw,
                         const float* k_shift_logit, const float* v_shift_logit,
                         const float* q_norm_weight, const float* k_norm_weight, float eps,
                         const void* dq, const void* dk, const void* dv, void* dq_raw,
                         void* dk_raw, void* dv_raw, float* dk_shift_logit,
                         float* dv_shift_logit, float* dq_norm_weight, float* dk_norm_weight,
                         void* workspace, size_t workspace_bytes, int B, int H, int L, int d,
                         hipStream_t stream) {
  if (!all_set({q_raw, k_raw, v_raw, k_shift_logit, v_shift_logit, q_norm_weight, k_norm_weight,
                dq, dk, dv, dq_raw, dk_raw, dv_raw, dk_shift_logit, dv_shift_logit,
                dq_norm_weight, dk_norm_weight}))
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!valid_eps(eps)) return FOX_ERR_VALUE;
  if (!all_aligned16({q_raw, k_raw, v_raw, k_shift_logit, v_shift_logit, q_norm_weight,
                      k_norm_weight, dq, dk, dv, dq_raw, dk_raw, dv_raw, dk_shift_logit,
                      dv_shift_logit, dq_norm_weight, dk_norm_weight}))
    return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::pro_prologue_bwd_workspace_bytes(B * H, L, d))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_pro_prologue_bwd(
      dtype == FOX_DTYPE_BF16, q_raw, k_raw, v_raw, k_shift_logit, v_shift_logit, q_norm_weight,
      k_norm_weight, eps, dq, dk, dv, dq_raw, dk_raw, dv_raw, dk_shift_logit, dv_shift_logit,
      dq_norm_weight, dk_norm_weight, workspace, H, B * H, L, d,
      static_cast<hipStream_t>(stream)));
}

fox_status_t fox_pro_output_gate(fox_dtype_t dtype, const void* o, const void* g_logit,
                        const float* o_norm_weight, float eps, void* y, int B, int H, int L,
                        int d, hipStream_t stream) {
  if (!all_set({o, g_logit, o_norm_weight, y})) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!valid_eps(eps)) return FOX_ERR_VALUE;
  if (!all_aligned16({o, g_logit, o_norm_weight, y})) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_out_gate(dtype == FOX_DTYPE_BF16, o, g_logit, o_norm_weight,
                                            eps, y, H, B * H, L, d,
                                            static_cast<hipStream_t>(stream)));
}

fox_status_t fox_attn_fwd_pro(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c,
                     const void* g_logit, const float* o_norm_weight, float eps, void* o,
                     float* lse, void* y, int B, int H, int L, int d, float scale, hipStream_t stream) {
  if (!all_set({q, k, v, c, g_logit, o_norm_weight, o, lse, y})) return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!valid_eps(eps)) return FOX_ERR_VALUE;
  if (!all_aligned16({q, k, v, c, g_logit, o_norm_weight, o, lse, y})) return FOX_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == FOX_DTYPE_BF16)
    return launch_status(fox::launch_fwd_bf16_out_gate(q, k, v, c, o, lse, g_logit,
                                                       o_norm_weight, eps, y, H, B * H, L, d,
                                                       scale, s));
  hipError_t e = fox::launch_fwd_f32((const float*)q, (const float*)k, (const float*)v,
                                     fox::gate_array(c), (float*)o, lse, B * H, L, d, scale, s);
  if (e == hipSuccess)
    e = fox::launch_out_gate(false, o, g_logit, o_norm_weight, eps, y, H, B * H, L, d, s);
  return launch_status(e);
}

size_t fox_attn_bwd_pro_workspace_bytes(fox_dtype_t dtype, int B, int H, int L, int d) {
  if (check_dims(B, H, L, d) || check_dtype_d(dtype, d)) return 0;
  return fox::bwd_pro_workspace_bytes(dtype == FOX_DTYPE_BF16, B * H, L, d);
}

// fox_attn_bwd_pro and fox_attn_bwd_pro_stored: the same checks, the attention
// backward recomputing or keeping dS.
static fox_status_t attn_bwd_pro(bool keep_ds, fox_dtype_t dtype, const void* q, const void* k, const void* v,
                        const float* c, const void* o, const float* lse, const void* g_logit,
                        const float* o_norm_weight, float eps, const void* dy, void* dq,
                        void* dk, void* dv, float* d_log_f, void* dg_logit, float* do_norm_weight,
                        void* workspace, size_t workspace_bytes, int B, int H, int L, int d,
                        float scale, hipStream_t stream) {
  if (!all_set({q, k, v, c, o, lse, g_logit, o_norm_weight, dy, dq, dk, dv, d_log_f, dg_logit,
                do_norm_weight}))
    return FOX_ERR_NULL;
  fox_status_t st = check_dims(B, H, L, d);
  if (st) return st;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!valid_eps(eps)) return FOX_ERR_VALUE;
  if (!all_aligned16({q, k, v, c, o, lse, g_logit, o_norm_weight, dy, dq, dk, dv, d_log_f,
                      dg_logit, do_norm_weight}))
    return FOX_ERR_ALIGN;
  const bool bf = dtype == FOX_DTYPE_BF16;
  if (keep_ds && !bf) return FOX_ERR_UNSUPPORTED;
  const size_t need = keep_ds ? fox::bwd_pro_stored_workspace_bytes(B * H, L, d)
                              : fox::bwd_pro_workspace_bytes(bf, B * H, L, d);
  if (!workspace || workspace_bytes < need) return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_bwd_pro(bf, q, k, v, c, o, lse, g_logit, o_norm_weight, eps,
                                           dy, dq, dk, dv, d_log_f, dg_logit, do_norm_weight,
                                           workspace, H, B * H, L, d, scale,
                                           static_cast<hipStream_t>(stream), keep_ds));
}

fox_status_t fox_attn_bwd_pro(fox_dtype_t dtype, const void* q, const void* k, const void* v, const float* c,
                     const void* o, const float* lse, const void* g_logit,
                     const float* o_norm_weight, float eps, const void* dy, void* dq, void* dk,
                     void* dv, float* d_log_f, void* dg_logit, float* do_norm_weight,
                     void* workspace, size_t workspace_bytes, int B, int H, int L, int d,
                     float scale, hipStream_t stream) {
  return attn_bwd_pro(false, dtype, q, k, v, c, o, lse, g_logit, o_norm_weight, eps, dy, dq, dk,
                      dv, d_log_f, dg_logit, do_norm_weight, workspace, workspace_bytes, B, H, L,
                      d, scale, stream);
}

size_t fox_attn_bwd_pro_stored_workspace_bytes(fox_dtype_t dtype, int B, int H, int L, int d) {
  if (check_dims(B, H, L, d) || check_dtype_d(dtype, d) || dtype != FOX_DTYPE_BF16) return 0;
  return fox::bwd_pro_stored_workspace_bytes(B * H, L, d);
}

fox_status_t fox_attn_bwd_pro_stored(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                            const float* c, const void* o, const float* lse, const void* g_logit,
                            const float* o_norm_weight, float eps, const void* dy, void* dq,
                            void* dk, void* dv, float* d_log_f, void* dg_logit,
                            float* do_norm_weight, void* workspace, size_t workspace_bytes, int B,
                            int H, int L, int d, float scale, hipStream_t stream) {
  return attn_bwd_pro(true, dtype, q, k, v, c, o, lse, g_logit, o_norm_weight, eps, dy, dq, dk,
                      dv, d_log_f, dg_logit, do_norm_weight, workspace, workspace_bytes, B, H, L,
                      d, scale, stream);
}

fox_status_t fox_gate_projection(fox_dtype_t dtype, const void* x, const float* w_f, const float* b_f,
                        float* gate_logit, int B, int L, int H, int M, hipStream_t stream) {
  if (!all_set({x, w_f, gate_logit})) return FOX_ERR_NULL;
  fox_status_t st = check_projection(dtype, B, L, H, M);
  if (st) return st;
  if (!all_aligned16({x, w_f, gate_logit})) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_gate_proj_fwd(dtype == FOX_DTYPE_BF16, x, w_f, b_f, gate_logit,
                                                 B * L, L, H, M,
                                                 static_cast<hipStream_t>(stream)));
}

size_t fox_gate_projection_bwd_workspace_bytes(fox_dtype_t dtype, int B, int L, int H, int M) {
  if (check_projection(dtype, B, L, H, M)) return 0;
  return fox::gate_proj_bwd_workspace_bytes(B * L, H, M);
}

fox_status_t fox_gate_projection_bwd(fox_dtype_t dtype, const void* x, const float* w_f, const float* d_logit,
                            void* dx, float* dw_f, float* db_f, void* workspace,
                            size_t workspace_bytes, int B, int L, int H, int M, hipStream_t stream) {
  if (!all_set({x, w_f, d_logit, dw_f})) return FOX_ERR_NULL;
  fox_status_t st = check_projection(dtype, B, L, H, M);
  if (st) return st;
  if (!all_aligned16({x, w_f, d_logit, dw_f}) || (dx && !aligned16(dx))) return FOX_ERR_ALIGN;
  if (!workspace || workspace_bytes < fox::gate_proj_bwd_workspace_bytes(B * L, H, M))
    return FOX_ERR_WORKSPACE;
  if (!aligned16(workspace)) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_gate_proj_bwd(dtype == FOX_DTYPE_BF16, x, w_f, d_logit, dx,
                                                 dw_f, db_f, workspace, B, L, H, M,
                                                 static_cast<hipStream_t>(stream)));
}

fox_status_t fox_cache_append(const fox_cache_t* cache, fox_dtype_t dtype, const void* k, const void* v,
                     const float* gate_logit, const int* seq_len, const int* parent,
                     const int* n_new, int n, hipStream_t stream) {
  fox_status_t st = check_cache(cache);
  if (st) return st;
  if (!all_set({k, v, gate_logit, seq_len})) return FOX_ERR_NULL;
  if (!cache_new_ok(cache, n)) return FOX_ERR_SHAPE;
  if (!cache_dtype(dtype)) return FOX_ERR_UNSUPPORTED;
  if (!all_aligned16({k, v, gate_logit, seq_len, parent, n_new})) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_cache_append(cache_spec(cache), dtype == FOX_DTYPE_BF16, k, v,
                                                gate_logit, seq_len, parent, n_new, n, stream));
}

fox_status_t fox_cache_append_packed(const fox_cache_t* cache, fox_dtype_t dtype, const void* k,
                            const void* v, const float* c, const int* cu_seqlens,
                            const int* seq_len, int N, hipStream_t stream) {
  fox_status_t st = check_cache(cache);
  if (st) return st;
  if (!all_set({k, v, c, cu_seqlens})) return FOX_ERR_NULL;
  if (!cache_rows_ok(cache, N)) return FOX_ERR_SHAPE;
  if (!cache_dtype(dtype)) return FOX_ERR_UNSUPPORTED;
  if (!all_aligned16({k, v, c, cu_seqlens, seq_len})) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_cache_append_packed(cache_spec(cache), dtype == FOX_DTYPE_BF16,
                                                       k, v, c, cu_seqlens, seq_len, N, stream));
}

fox_status_t fox_cache_keep(const fox_cache_t* cache, const int* seq_len, const int* index,
                   const int* n_keep, int n, hipStream_t stream) {
  fox_status_t st = check_cache(cache);
  if (st) return st;
  if (!all_set({seq_len, index, n_keep})) return FOX_ERR_NULL;
  if (n < 1 || n > kMaxNewTokens) return FOX_ERR_SHAPE;
  if (!all_aligned16({seq_len, index, n_keep})) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_cache_keep(cache_spec(cache), seq_len, index, n_keep, n, stream));
}

fox_status_t fox_cache_read(const fox_cache_t* cache, fox_dtype_t dtype, const int* start,
                   const int* seq_len, void* k, void* v, float* c, int T, int zero_others,
                   hipStream_t stream) {
  fox_status_t st = check_cache(cache);
  if (st) return st;
  if (!all_set({seq_len, k, v})) return FOX_ERR_NULL;
  if (!cache_rows_ok(cache, (long long)T * cache->B)) return FOX_ERR_SHAPE;
  if (!cache_dtype(dtype)) return FOX_ERR_UNSUPPORTED;
  if (!all_aligned16({start, seq_len, k, v, c})) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_cache_read(cache_spec(cache), dtype == FOX_DTYPE_BF16, start,
                                              seq_len, k, v, c, T, zero_others != 0, stream));
}

size_t fox_attn_cache_workspace_bytes(const fox_cache_t* cache, int n, int max_len) {
  if (check_cache(cache) || !cache_new_ok(cache, n)) return 0;
  return fox::attn_cache_workspace_bytes(cache_spec(cache), n, cache_max_len(cache, max_len));
}

fox_status_t fox_attn_cache(const fox_cache_t* cache, const void* q, const int* seq_len,
                   const int* parent, const int* n_new, void* o, float* lse, void* workspace,
                   size_t workspace_bytes, int n, int max_len, float scale, hipStream_t stream) {
  fox_status_t st = check_cache(cache);
  if (st) return st;
  if (!all_set({q, seq_len, o, lse})) return FOX_ERR_NULL;
  if (!cache_new_ok(cache, n)) return FOX_ERR_SHAPE;
  if (!all_aligned16({q, seq_len, parent, n_new, o, lse, workspace})) return FOX_ERR_ALIGN;
  const fox::CacheSpec s = cache_spec(cache);
  const int len = cache_max_len(cache, max_len);
  const size_t need = fox::attn_cache_workspace_bytes(s, n, len);
  if (need && (!workspace || workspace_bytes < need)) return FOX_ERR_WORKSPACE;
  return launch_status(fox::launch_attn_cache(s, q, seq_len, parent, n_new, o, lse, workspace, n,
                                              len, scale, stream));
}

size_t fox_packed_plan_bytes(int B, int N) {
  return check_packed(B, 1, 1, N) ? 0 : (size_t)fox::packed_items(B, N) * 16;
}

fox_status_t fox_packed_plan(const int* cu_seqlens, int B, int N, void* plan, size_t plan_bytes,
                    const fox_packed_rows_t* tensors, int n, hipStream_t stream) {
  if (!cu_seqlens || !plan) return FOX_ERR_NULL;
  fox_status_t st = check_packed(B, 1, 1, N);
  if (st) return st;
  if (!all_aligned16({cu_seqlens, plan})) return FOX_ERR_ALIGN;
  if (plan_bytes < fox_packed_plan_bytes(B, N)) return FOX_ERR_WORKSPACE;
  fox::ZeroRows x[fox::kZeroTensors];
  st = zero_rows(tensors, n, x);
  if (st) return st;
  return launch_status(fox::launch_packed_plan(cu_seqlens, B, N, plan, x, n, stream));
}

fox_status_t fox_gate_prefix_packed(fox_dtype_t gate_dtype, const void* gate_logit,
                           const int* cu_seqlens, float* c, int B, int H, int N,
                           hipStream_t stream) {
  if (!all_set({gate_logit, cu_seqlens, c})) return FOX_ERR_NULL;
  fox_status_t st = check_packed(B, H, H, N);
  if (st) return st;
  if (!cache_dtype(gate_dtype)) return FOX_ERR_UNSUPPORTED;
  if (!all_aligned16({gate_logit, cu_seqlens, c})) return FOX_ERR_ALIGN;
  return launch_status(fox::launch_packed_prefix(gate_dtype == FOX_DTYPE_BF16, gate_logit,
                                                 cu_seqlens, c, B, H, N, nullptr, nullptr, 0,
                                                 stream));
}

fox_status_t fox_packed_start(fox_dtype_t gate_dtype, const void* gate_logit, const int* cu_seqlens,
                     float* c, int B, int H, int N, void* plan, size_t plan_bytes,
                     const fox_packed_rows_t* tensors, int n, hipStream_t stream) {
  if (!all_set({gate_logit, cu_seqlens, c, plan})) return FOX_ERR_NULL;
  fox_status_t st = check_packed(B, H, H, N);
  if (st) return st;
  if (!cache_dtype(gate_dtype)) return FOX_ERR_UNSUPPORTED;
  if (!all_aligned16({gate_logit, cu_seqlens, c, plan})) return FOX_ERR_ALIGN;
  if (plan_bytes < fox_packed_plan_bytes(B, N)) return FOX_ERR_WORKSPACE;
  fox::ZeroRows x[fox::kZeroTensors];
  st = zero_rows(tensors, n, x);
  if (st) return st;
  return launch_status(fox::launch_packed_prefix(gate_dtype == FOX_DTYPE_BF16, gate_logit,
                                                 cu_seqlens, c, B, H, N, plan, x, n, stream));
}

fox_status_t fox_attn_fwd_packed(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                        const float* c, const void* plan, void* o, void* o_lo, float* lse, int B, int H,
                        int H_kv, int N, int d, int max_len, float scale, hipStream_t stream) {
  if (!all_set({q, k, v, c, plan, o, lse})) return FOX_ERR_NULL;
  fox_status_t st = check_packed(B, H, H_kv, N);
  if (st) return st;
  if (d <= 0 || (long long)N * d * 4 >= (1LL << 31)) return FOX_ERR_SHAPE;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (o_lo && dtype != FOX_DTYPE_BF16) return FOX_ERR_UNSUPPORTED;
  if (!packed_scale_ok(dtype, scale)) return FOX_ERR_VALUE;
  if (!all_aligned16({q, k, v, c, plan, o, o_lo, lse})) return FOX_ERR_ALIGN;
  const int len = max_len <= 0 || max_len > N ? N : max_len;
  if (dtype == FOX_DTYPE_BF16)
    return launch_status(fox::launch_packed_fwd(q, k, v, c, o, o_lo, lse, plan, B, H, H_kv, N, d, len,
                                                scale, stream));
  return launch_status(fox::launch_packed_fwd_f32((const float*)q, (const float*)k,
                                                  (const float*)v, c, (float*)o, lse, plan, B, H,
                                                  H_kv, N, d, scale, stream));
}

size_t fox_attn_bwd_packed_workspace_bytes(fox_dtype_t dtype, int H, int H_kv, int N, int d,
                                           int max_len) {
  if (check_packed(1, H, H_kv, N) || check_dtype_d(dtype, d)) return 0;
  const int len = max_len <= 0 || max_len > N ? N : max_len;
  const int splits = fox::packed_head_split(dtype == FOX_DTYPE_BF16, H, H_kv, N, d, len);
  const size_t row = ((size_t)H * N + 3) & ~(size_t)3;  // delta, dc_q, dc_k
  return (3 * row + (splits > 1 ? (size_t)splits * 2 * H_kv * N * d : 0)) * sizeof(float);
}

fox_status_t fox_attn_bwd_packed(fox_dtype_t dtype, const void* q, const void* k, const void* v,
                        const float* c, const void* o, const void* o_lo, const float* lse,
                        const void* d_o, fox_dtype_t gate_dtype, const void* gate_logit, const int* cu_seqlens,
                        const void* plan, void* dq, void* dk, void* dv, void* d_logit,
                        float* d_log_f, int zero_behind, void* workspace,
                        size_t workspace_bytes, int B, int H, int H_kv, int N, int d,
                        int max_len, float scale, hipStream_t stream) {
  if (!all_set({q, k, v, c, o, lse, d_o, gate_logit, cu_seqlens, plan, dq, dk, dv, d_logit}))
    return FOX_ERR_NULL;
  fox_status_t st = check_packed(B, H, H_kv, N);
  if (st) return st;
  if (d <= 0 || (long long)N * d * 4 >= (1LL << 31)) return FOX_ERR_SHAPE;
  st = check_dtype_d(dtype, d);
  if (st) return st;
  if (!cache_dtype(gate_dtype) || (o_lo && dtype != FOX_DTYPE_BF16)) return FOX_ERR_UNSUPPORTED;
  if (!packed_scale_ok(dtype, scale)) return FOX_ERR_VALUE;
  if (!all_aligned16({q, k, v, c, o, o_lo, lse, d_o, gate_logit, cu_seqlens, plan, dq, dk, dv, d_logit,
                      d_log_f, workspace}))
    return FOX_ERR_ALIGN;
  if (!workspace ||
      workspace_bytes < fox_attn_bwd_packed_workspace_bytes(dtype, H, H_kv, N, d, max_len))
    return FOX_ERR_WORKSPACE;
  const int len = max_len <= 0 || max_len > N ? N : max_len;
  // delta, dc_q, dc_k, each on a 16-byte boundary
  const size_t row = ((size_t)H * N + 3) & ~(size_t)3;
  float* delta = static_cast<float*>(workspace);
  float *dcq = delta + row, *dck = dcq + row, *part = dck + row;
  hipError_t e;
  if (dtype == FOX_DTYPE_BF16)
    e = fox::launch_packed_bwd(q, k, v, c, o, o_lo, lse, d_o, dq, dk, dv, delta, dck, part, plan,
                               B, H, H_kv, N, d, len, scale, stream);
  else
    e = fox::launch_packed_bwd_f32((const float*)q, (const float*)k, (const float*)v, c,
                                   (const float*)o, lse, (const float*)d_o, (float*)dq, (float*)dk,
                                   (float*)dv, delta, dcq, dck, part, plan, B, H, H_kv, N, d,
                                   len, scale, stream);
  const int esz = dtype == FOX_DTYPE_BF16 ? 2 : 4;
  const fox::ZeroRows zeros[] = {{dq, H, d * esz},
                                 {dk, H_kv, d * esz},
                                 {dv, H_kv, d * esz},
                                 {d_logit, H, gate_dtype == FOX_DTYPE_BF16 ? 2 : 4},
                                 {d_log_f, H, 4}};
  const bool bf = dtype == FOX_DTYPE_BF16;
  const fox::HeadSum sum{part, dk, dv, bf, fox::packed_head_split(bf, H, H_kv, N, d, len), H_kv, d};
  if (e == hipSuccess)
    e = fox::launch_packed_gate_grad(gate_dtype == FOX_DTYPE_BF16,
                                     dtype == FOX_DTYPE_BF16 ? nullptr : dcq, dck, gate_logit,
                                     cu_seqlens, d_log_f, d_logit, B, H, N, sum, zeros,
                                     !zero_behind ? 0 : d_log_f ? 5 : 4, stream);
  return launch_status(e);
}

fox_status_t fox_packed_zero_behind(const fox_packed_rows_t* tensors, int n, const int* cu_seqlens,
                           int B, int N, hipStream_t stream) {
  if (!cu_seqlens) return FOX_ERR_NULL;
  if (n < 1 || B <= 0 || N <= 0) return FOX_ERR_SHAPE;
  fox::ZeroRows x[fox::kZeroTensors];
  fox_status_t st = zero_rows(tensors, n, x);
  if (st) return st;
  return launch_status(fox::launch_packed_zero(x, n, cu_seqlens, B, N, stream));
}

}  // extern "C"
