// C ABI of the paged cache's operators: argument validation, workspace layout
// and launches. Host code only.
#include <math.h>
#include <stdio.h>

#include "abi.h"
#include "cache.h"
#include "fp2.h"
#include "rotary_rows.h"

namespace {

using fp2::CacheProblem;

constexpr int kMaxLen = fp2::kMaxBlocks * fp2::kBlock;   // 1M tokens
constexpr int kMaxBatch = 65536;

template <class... A>
fp2_status_t fail(fp2_status_t st, const char* fmt, A... a) {
  char buf[256];
  snprintf(buf, sizeof(buf), fmt, a...);
  return fp2::set_error(st, buf);
}
fp2_status_t fail(fp2_status_t st, const char* msg) { return fp2::set_error(st, msg); }
fp2_status_t ok() { return fp2::set_error(FP2_OK, ""); }

// Whether n elements at a share memory with m at b.
template <class T>
bool overlap(const T* a, int64_t n, const T* b, int64_t m) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + (uint64_t)m * sizeof(T) && y < x + (uint64_t)n * sizeof(T);
}

bool aligned(const void* x, uintptr_t n) { return ((uintptr_t)x & (n - 1)) == 0; }

// cross: the new tokens are queries of other sequences, so they have a bound of their own, and no window.
fp2_status_t check_params(const fp2_cache_params_t* p, bool cross = false) {
  if (!p) return fail(FP2_EINVAL, "params is null");
  if (p->batch < 0) return fail(FP2_EINVAL, "batch %d < 0", p->batch);
  if (p->batch > kMaxBatch) return fail(FP2_EUNSUPPORTED, "batch %d > %d", p->batch, kMaxBatch);
  if (p->num_kv_heads < 1) return fail(FP2_EINVAL, "num_kv_heads %d < 1", p->num_kv_heads);
  if (p->num_kv_heads > 1024) return fail(FP2_EUNSUPPORTED, "num_kv_heads %d > 1024", p->num_kv_heads);
  if (p->num_q_heads < 1 || p->num_q_heads % p->num_kv_heads)
    return fail(FP2_EINVAL, "num_q_heads %d is not a positive multiple of num_kv_heads %d",
                p->num_q_heads, p->num_kv_heads);
  const int g = p->num_q_heads / p->num_kv_heads;
  if (g != 1 && g != 2 && g != 4 && g != 8)
    return fail(FP2_EUNSUPPORTED, "group size %d not in {1, 2, 4, 8}", g);
  if (p->head_dim <= 0) return fail(FP2_EINVAL, "head_dim %d <= 0", p->head_dim);
  if (p->head_dim != fp2::kHeadDim) return fail(FP2_EUNSUPPORTED, "head_dim %d != 128", p->head_dim);
  if (p->page_size < 1) return fail(FP2_EINVAL, "page_size %d < 1", p->page_size);
  if (p->max_kv_len < 0) return fail(FP2_EINVAL, "max_kv_len %d < 0", p->max_kv_len);
  if (p->max_kv_len > kMaxLen) return fail(FP2_EUNSUPPORTED, "max_kv_len %d > %d", p->max_kv_len, kMaxLen);
  if (cross) {
    if (p->max_seq_len < 0) return fail(FP2_EINVAL, "max_seq_len %d < 0", p->max_seq_len);
    if (p->max_seq_len > kMaxLen) return fail(FP2_EUNSUPPORTED, "max_seq_len %d > %d", p->max_seq_len, kMaxLen);
    if (p->window_tokens != 0 || p->sink_tokens != 0)
      return fail(FP2_EINVAL, "window_tokens and sink_tokens must be 0: every query sees all keys");
  } else if (p->max_seq_len < 0 || p->max_seq_len > p->max_kv_len)
    return fail(FP2_EINVAL, "max_seq_len %d outside [0, max_kv_len = %d]", p->max_seq_len, p->max_kv_len);
  const int pages = (int)(((int64_t)p->max_kv_len + p->page_size - 1) / p->page_size);
  if (p->max_pages_per_seq < pages)
    return fail(FP2_EINVAL, "max_pages_per_seq %d < ceil(max_kv_len / page_size) = %d",
                p->max_pages_per_seq, pages);
  if (p->dtype != FP2_BF16 && p->dtype != FP2_FP8_E4M3) return fail(FP2_EINVAL, "dtype %d unknown", p->dtype);
  if ((int64_t)p->batch * (p->max_kv_len + 4096ll) > 1ll << 35)   // tiles of 32 keys are counted in 31 bits
    return fail(FP2_EUNSUPPORTED, "batch %d x max_kv_len %d > 2^35 - 4096 batch", p->batch, p->max_kv_len);
  const int sb = p->scale_tokens;
  if (sb != 0) {
    if (p->dtype != FP2_FP8_E4M3) return fail(FP2_EINVAL, "scale_tokens %d with a bf16 cache", sb);
    if (sb < 0) return fail(FP2_EINVAL, "scale_tokens %d < 0", sb);
    if (sb != 16 && sb != 32 && sb != 64 && sb != 128)
      return fail(FP2_EUNSUPPORTED, "scale_tokens %d not in {16, 32, 64, 128}", sb);
    if (p->page_size % sb)
      return fail(FP2_EINVAL, "page_size %d is not a multiple of scale_tokens %d", p->page_size, sb);
  }
  if (p->sink_tokens < 0 || p->window_tokens < 0)
    return fail(FP2_EINVAL, "sink_tokens and window_tokens must be >= 0");
  if (p->kv_splits < 0 || p->kv_splits > 32)
    return fail(FP2_EINVAL, "kv_splits %d not in [0, 32]", p->kv_splits);
  if (!isfinite(p->softmax_scale)) return fail(FP2_EINVAL, "softmax_scale is not finite");
  return FP2_OK;
}

fp2_status_t check_cu(const int32_t* cu, int batch, int bound, const char* name) {
  if (cu[0] != 0) return fail(FP2_EINVAL, "%s[0] = %d != 0", name, cu[0]);
  for (int b = 0; b < batch; ++b) {
    const int64_t len = (int64_t)cu[b + 1] - cu[b];
    if (len < 0) return fail(FP2_EINVAL, "%s decreases at %d", name, b);
    if (len > bound)
      return fail(FP2_EINVAL, "%s: sequence %d has length %lld > its bound %d", name, b, (long long)len, bound);
  }
  return FP2_OK;
}

fp2_status_t check_lengths(const fp2_cache_params_t* p, const int32_t* cu, const int32_t* cu_host,
                           const int32_t* cuk, const int32_t* cuk_host, bool need_cu, bool cross = false) {
  if ((need_cu && !cu) || !cuk) return fail(FP2_EINVAL, "cu_seqlens or cu_seqlens_k is null");
  fp2_status_t st;
  if (cu_host && (st = check_cu(cu_host, p->batch, p->max_seq_len, "cu_seqlens"))) return st;
  if (cuk_host && (st = check_cu(cuk_host, p->batch, p->max_kv_len, "cu_seqlens_k"))) return st;
  if (cu_host && cuk_host && !cross)
    for (int b = 0; b < p->batch; ++b)
      if (cuk_host[b + 1] - cuk_host[b] < cu_host[b + 1] - cu_host[b])
        return fail(FP2_EINVAL, "sequence %d: fewer cached than new tokens", b);
  return FP2_OK;
}

fp2_status_t check_cache(const fp2_cache_params_t* p, const fp2_kv_cache_t* c, const int32_t* table,
                         bool need_v) {
  if (!c) return fail(FP2_EINVAL, "cache is null");
  if (!c->k || (need_v && !c->v)) return fail(FP2_EINVAL, "cache: k or v is null");
  if (!aligned(c->k, 16) || !aligned(c->v, 16))
    return fail(FP2_EINVAL, "cache: k and v must be 16-byte aligned");
  if (!table) return fail(FP2_EINVAL, "block_table is null");
  if (p->dtype == FP2_FP8_E4M3) {
    const bool block = p->scale_tokens > 0;
    const void* ks = block ? (const void*)c->k_block_scale : (const void*)c->k_head_scale;
    const void* vs = block ? (const void*)c->v_block_scale : (const void*)c->v_head_scale;
    if (!ks || (need_v && !vs))
      return fail(FP2_EINVAL, "cache: the %s scales of the codes are null", block ? "block" : "head");
  }
  return FP2_OK;
}

CacheProblem make_problem(const fp2_cache_params_t* p, const void* q, const int32_t* cu,
                          const int32_t* cuk, const fp2_kv_cache_t* c, const int32_t* table) {
  CacheProblem r{};
  r.q = (const uint16_t*)q;
  r.cu = cu;
  r.cuk = cuk;
  if (c) {
    r.k = (uint8_t*)c->k;
    r.v = (uint8_t*)c->v;
    r.k_head = c->k_head_scale;
    r.v_head = c->v_head_scale;
    r.k_block = c->k_block_scale;
    r.v_block = c->v_block_scale;
  }
  const int pg = p->page_size;
  r.pm.table = table;
  r.pm.stride = p->max_pages_per_seq;
  r.pm.page = pg;
  r.pm.shift = (pg & (pg - 1)) ? -1 : __builtin_ctz(pg);
  r.batch = p->batch;
  r.hq = p->num_q_heads;
  r.hkv = p->num_kv_heads;
  r.g = p->num_q_heads / p->num_kv_heads;
  r.form = p->dtype == FP2_BF16 ? fp2::kCacheBf16 : p->scale_tokens ? fp2::kCacheBlock : fp2::kCacheHead;
  r.sb_shift = p->scale_tokens ? __builtin_ctz(p->scale_tokens) : 0;
  const bool all = p->window_tokens == 0 || p->window_tokens >= p->max_kv_len;
  r.window = all ? fp2::kNoWindow : p->window_tokens;
  r.sink = all ? 0 : p->sink_tokens < p->max_kv_len ? p->sink_tokens : p->max_kv_len;
  r.max_new = p->max_seq_len;
  r.max_kv = p->max_kv_len;
  r.splits = p->kv_splits;
  const double scale = p->softmax_scale > 0.f ? (double)p->softmax_scale : 1.0 / sqrt((double)fp2::kHeadDim);
  r.scale_log2 = (float)(scale * 1.4426950408889634074);
  return r;
}

bool few_rows(const CacheProblem& r) { return (int64_t)r.max_new * r.g <= fp2::kFewRows; }

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Bytes that the attention needs, and the offsets of the maxima and of the
// sequences' parts behind the partial outputs.
size_t attend_bytes(const CacheProblem& r, size_t* ml, size_t* at, bool cross = false) {
  int64_t slots = 0;
  int rows = 0;
  const bool few = few_rows(r);
  if (r.batch > 0 && r.max_new > 0) {
    if (few) fp2::cache_decode_partials(r, &slots, &rows);
    else if (cross) fp2::cache_cross_partials(r, &slots, &rows);
    else fp2::cache_extend_partials(r, &slots, &rows);
  }
  *ml = (size_t)slots * rows * fp2::kHeadDim * sizeof(float);   // a multiple of 256
  *at = *ml + align256((size_t)slots * rows * 2 * sizeof(float));
  if (!slots || r.splits) return *at;
  return *at + (few ? align256((size_t)r.batch * 2 * sizeof(int32_t)) : cross ? (size_t)fp2::kCrossCuts * 16 : 0);
}

size_t weights_bytes(const CacheProblem& r) {
  return r.batch > 0 ? align256((size_t)fp2::cache_weights_partials(r) * sizeof(float)) : 0;
}

// The attentions' queries and outputs.
fp2_status_t check_attention(const fp2_cache_params_t* params, const void* q, const void* out, const float* lse,
                             const int32_t* cu_seqlens_host) {
  if (!q || !out) return fail(FP2_EINVAL, "q or out is null");
  if (!aligned(q, 16) || !aligned(out, 16)) return fail(FP2_EINVAL, "q and out must be 16-byte aligned");
  if (q == out) return fail(FP2_EINVAL, "out must not be q");
  if (cu_seqlens_host) {   // then the rows that are read and written are known
    const int64_t heads = (int64_t)cu_seqlens_host[params->batch] * params->num_q_heads;
    const int64_t row = 2 * fp2::kHeadDim * heads, sums = sizeof(float) * heads;
    const char *qb = (const char*)q, *ob = (const char*)out, *lb = (const char*)lse;
    if (overlap(qb, row, ob, row)) return fail(FP2_EINVAL, "out must not overlap q");
    if (lse && (overlap(qb, row, lb, sums) || overlap(ob, row, lb, sums)))
      return fail(FP2_EINVAL, "lse must not overlap q or out");
  }
  return FP2_OK;
}

fp2_status_t check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return FP2_OK;
  if (!ws) return fail(FP2_EWORKSPACE, "workspace is null (need %zu bytes)", need);
  if (!aligned(ws, 256)) return fail(FP2_EWORKSPACE, "workspace is not 256-byte aligned");
  if (bytes < need) return fail(FP2_EWORKSPACE, "workspace has %zu bytes, need %zu", bytes, need);
  return FP2_OK;
}

fp2_status_t hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  if (e == hipErrorInvalidValue) return fail(FP2_EUNSUPPORTED, "%s: more threads than a launch takes (2^32 - 1)", what);
  return fail(FP2_EHIP, "%s: %s", what, hipGetErrorString(e));
}

// Bytes from the first row's start to the last row's end.
struct Extent {
  const char* at;
  int64_t stride, width, rows;     // in bytes, but for the rows
};
// Whether rows that are written meet rows of another tensor. Rows of one stride may lie between each
// other's (parts of one matrix).
bool rows_meet(const Extent& a, const Extent& b) {
  if (a.rows == 0 || b.rows == 0) return false;
  const char *ae = a.at + (a.rows - 1) * a.stride + a.width, *be = b.at + (b.rows - 1) * b.stride + b.width;
  if (a.at >= be || b.at >= ae) return false;
  if (a.stride != b.stride || a.stride == 0) return true;
  const int64_t off = ((b.at - a.at) % a.stride + a.stride) % a.stride;
  return off < a.width || off + b.width > a.stride;
}

fp2_status_t check_rotary(const fp2_rotary_t* r) {
  if (!r) return fail(FP2_EINVAL, "rotary is null");
  if (r->dim < 2 || r->dim > fp2::kHeadDim || r->dim % 2)
    return fail(FP2_EINVAL, "rotary: dim %d is not even and in [2, 128]", r->dim);
  if (r->interleaved != 0 && r->interleaved != 1)
    return fail(FP2_EINVAL, "rotary: interleaved %d is not 0 or 1", r->interleaved);
  if (!r->turns) return fail(FP2_EINVAL, "rotary: turns is null");
  if (!aligned(r->turns, 8)) return fail(FP2_EINVAL, "rotary: turns must be 8-byte aligned");
  if (!(r->scale > 0.f) || !isfinite(r->scale) || !isfinite(1.f / r->scale))
    return fail(FP2_EINVAL, "rotary: scale must be positive and finite, and its inverse too");
  return FP2_OK;
}

fp2::Rotary make_rotary(const fp2_rotary_t* r, bool inverse, bool scaled) {
  if (!r) return fp2::make_rotary(nullptr, 2, false, 1.0);
  return fp2::make_rotary(r->turns, r->dim, inverse, !scaled ? 1.0 : inverse ? 1.0 / r->scale : (double)r->scale);
}

fp2_status_t check_strided(const char* name, const void* x, int64_t stride, int width) {
  if (!x) return fail(FP2_EINVAL, "%s is null", name);
  if (!aligned(x, 16) || stride % 8) return fail(FP2_EINVAL, "%s must have 16-byte aligned rows", name);
  if (stride < width) return fail(FP2_EINVAL, "%s: a stride of %lld for rows of %d", name, (long long)stride, width);
  return FP2_OK;
}

constexpr int64_t kMaxRows = 1ll << 31;      // tokens of a call

// Rows that are turned; `tokens` < 0: not known on the host.
fp2_status_t check_rows(const char* name, const fp2_rotary_rows_t* x, int64_t tokens) {
  if (x->heads < 1 || x->heads > 8192) return fail(FP2_EINVAL, "%s: heads %d not in [1, 8192]", name, x->heads);
  const int width = x->heads * fp2::kHeadDim;
  fp2_status_t st;
  if (tokens != 0 && ((st = check_strided(name, x->x, x->x_stride, width)) ||
                      (st = check_strided(name, x->out, x->out_stride, width))))
    return st;
  if (x->out_dtype != FP2_BF16 && x->out_dtype != FP2_FP8_E4M3)
    return fail(FP2_EINVAL, "%s: out_dtype %d unknown", name, x->out_dtype);
  if (x->out_dtype == FP2_FP8_E4M3) {
    if (!x->out_scale) return fail(FP2_EINVAL, "%s: out_scale of the codes is null", name);
    if (x->out_stride % 16) return fail(FP2_EINVAL, "%s must have 16-byte aligned rows", name);
  }
  return FP2_OK;
}

Extent in_of(const fp2_rotary_rows_t* x, int64_t tokens) {
  return Extent{(const char*)x->x, 2 * x->x_stride, 2ll * x->heads * fp2::kHeadDim, tokens};
}
Extent out_of(const fp2_rotary_rows_t* x, int64_t tokens) {
  const int e = x->out_dtype == FP2_BF16 ? 2 : 1;
  return Extent{(const char*)x->out, e * x->out_stride, (int64_t)e * x->heads * fp2::kHeadDim, tokens};
}
bool in_place(const fp2_rotary_rows_t* x) {
  return x->x == x->out && x->x_stride == x->out_stride && x->out_dtype == FP2_BF16;
}

fp2::RotaryRows make_rows(const fp2_rotary_rows_t* x) {
  if (!x) return fp2::RotaryRows{};
  return fp2::RotaryRows{(const uint16_t*)x->x, x->x_stride, (uint8_t*)x->out, x->out_stride,
                         x->out_dtype == FP2_FP8_E4M3 ? x->out_scale : nullptr, x->heads};
}

}  // namespace

extern "C" {

size_t fp2_cache_workspace_bytes(const fp2_cache_params_t* params) {
  if (check_params(params) != FP2_OK) return 0;
  const CacheProblem r = make_problem(params, nullptr, nullptr, nullptr, nullptr, nullptr);
  size_t ml, at;
  const size_t a = attend_bytes(r, &ml, &at), w = weights_bytes(r);
  return a > w ? a : w;
}

fp2_status_t fp2_cache_append(const fp2_cache_params_t* params, const void* k_new,
                              const void* v_new, const int32_t* cu_seqlens,
                              const int32_t* cu_seqlens_host, const int32_t* cu_seqlens_k,
                              const int32_t* cu_seqlens_k_host, const fp2_kv_cache_t* cache,
                              const int32_t* block_table, void* stream) {
  fp2_status_t st = check_params(params);
  if (st != FP2_OK) return st;
  if (params->batch == 0 || params->max_seq_len == 0) return ok();
  if ((st = check_lengths(params, cu_seqlens, cu_seqlens_host, cu_seqlens_k, cu_seqlens_k_host, true)))
    return st;
  if ((st = check_cache(params, cache, block_table, true))) return st;
  if (!k_new || !v_new) return fail(FP2_EINVAL, "k_new or v_new is null");
  if (!aligned(k_new, 16) || !aligned(v_new, 16))
    return fail(FP2_EINVAL, "k_new and v_new must be 16-byte aligned");
  const CacheProblem r = make_problem(params, nullptr, cu_seqlens, cu_seqlens_k, cache, block_table);
  return hip_status(fp2::launch_cache_append(r, (const uint16_t*)k_new, (const uint16_t*)v_new,
                                             (hipStream_t)stream),
                    "fp2_cache_append launch");
}

fp2_status_t fp2_cache_attend(const fp2_cache_params_t* params, const void* q,
                              const int32_t* cu_seqlens, const int32_t* cu_seqlens_host,
                              const int32_t* cu_seqlens_k, const int32_t* cu_seqlens_k_host,
                              const fp2_kv_cache_t* cache, const int32_t* block_table, void* out,
                              float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  fp2_status_t st = check_params(params);
  if (st != FP2_OK) return st;
  if (params->batch == 0 || params->max_seq_len == 0) return ok();
  if ((st = check_lengths(params, cu_seqlens, cu_seqlens_host, cu_seqlens_k, cu_seqlens_k_host, true)))
    return st;
  if ((st = check_cache(params, cache, block_table, true))) return st;
  if ((st = check_attention(params, q, out, lse, cu_seqlens_host))) return st;
  const CacheProblem r = make_problem(params, q, cu_seqlens, cu_seqlens_k, cache, block_table);
  size_t ml, at;
  if ((st = check_workspace(workspace, workspace_bytes, attend_bytes(r, &ml, &at)))) return st;
  const fp2::CachePartials part{(float*)workspace, (float*)((char*)workspace + ml),
                                (int32_t*)((char*)workspace + at)};
  const hipError_t e =
      few_rows(r) ? fp2::launch_cache_decode(r, part, (uint16_t*)out, lse, (hipStream_t)stream)
                  : fp2::launch_cache_extend(r, part, (uint16_t*)out, lse, (hipStream_t)stream);
  return hip_status(e, "fp2_cache_attend launch");
}

fp2_status_t fp2_cache_weights(const fp2_cache_params_t* params, const void* q, const float* lse,
                               const int32_t* cu_seqlens, const int32_t* cu_seqlens_host,
                               const int32_t* cu_seqlens_k, const int32_t* cu_seqlens_k_host,
                               const fp2_kv_cache_t* cache, const int32_t* block_table,
                               const float* weights_in, float* weights, int64_t weights_stride,
                               void* workspace, size_t workspace_bytes, void* stream) {
  fp2_status_t st = check_params(params);
  if (st != FP2_OK) return st;
  if (params->batch == 0 || params->max_kv_len == 0) return ok();
  if ((st = check_lengths(params, cu_seqlens, cu_seqlens_host, cu_seqlens_k, cu_seqlens_k_host, true)))
    return st;
  if ((st = check_cache(params, cache, block_table, false))) return st;
  if ((params->max_seq_len > 0 && (!q || !lse)) || !weights)
    return fail(FP2_EINVAL, "q, lse or weights is null");
  if (!aligned(q, 16)) return fail(FP2_EINVAL, "q must be 16-byte aligned");
  if (weights_stride < params->max_kv_len)
    return fail(FP2_EINVAL, "weights_stride %lld < max_kv_len %d", (long long)weights_stride,
                params->max_kv_len);
  const int64_t entries = (int64_t)params->batch * params->num_kv_heads * weights_stride;
  if (weights_in && weights_in != weights && overlap<float>(weights_in, entries, weights, entries))
    return fail(FP2_EINVAL, "weights overlaps weights_in without being the same");
  const CacheProblem r = make_problem(params, q, cu_seqlens, cu_seqlens_k, cache, block_table);
  if ((st = check_workspace(workspace, workspace_bytes, weights_bytes(r)))) return st;
  return hip_status(fp2::launch_cache_weights(r, lse, weights_in, weights, weights_stride,
                                              (float*)workspace, (hipStream_t)stream),
                    "fp2_cache_weights launch");
}

fp2_status_t fp2_cache_evict(const fp2_cache_params_t* params, const fp2_kv_cache_t* cache,
                             const int32_t* cu_seqlens_k, const int32_t* cu_seqlens_k_host,
                             const int32_t* block_table, const int32_t* target_table,
                             int32_t target_pages, int32_t budget, int32_t recent_tokens,
                             const float* weights, float* weights_out, int64_t weights_stride,
                             int32_t* kept, int32_t* cu_seqlens_k_out, void* stream) {
  fp2_status_t st = check_params(params);
  if (st != FP2_OK) return st;
  if (budget < 1) return fail(FP2_EINVAL, "budget %d < 1", budget);
  if (budget > kMaxLen) return fail(FP2_EUNSUPPORTED, "budget %d > %d", budget, kMaxLen);
  if (recent_tokens < 0) return fail(FP2_EINVAL, "recent_tokens %d < 0", recent_tokens);
  if ((int64_t)params->sink_tokens + recent_tokens > budget)
    return fail(FP2_EINVAL, "sink_tokens %d + recent_tokens %d > budget %d", params->sink_tokens,
                recent_tokens, budget);
  if (params->batch == 0 || params->max_kv_len == 0) return ok();
  if ((st = check_lengths(params, nullptr, nullptr, cu_seqlens_k, cu_seqlens_k_host, false))) return st;
  if ((st = check_cache(params, cache, block_table, true))) return st;
  if (!target_table) return fail(FP2_EINVAL, "target_table is null");
  const int stay = budget < params->max_kv_len ? budget : params->max_kv_len;
  const int pages = (int)(((int64_t)stay + params->page_size - 1) / params->page_size);
  if (target_pages < pages)
    return fail(FP2_EINVAL, "target_pages %d < %d for %d tokens", target_pages, pages, stay);
  if (!weights || !weights_out || !kept || !cu_seqlens_k_out)
    return fail(FP2_EINVAL, "weights, weights_out, kept or cu_seqlens_k_out is null");
  if (weights_stride < params->max_kv_len)
    return fail(FP2_EINVAL, "weights_stride %lld < max_kv_len %d", (long long)weights_stride,
                params->max_kv_len);
  const int64_t entries = (int64_t)params->batch * params->num_kv_heads * weights_stride;
  if (overlap<float>(weights, entries, weights_out, entries))
    return fail(FP2_EINVAL, "weights_out must not overlap weights");
  if (overlap<int32_t>(cu_seqlens_k, params->batch + 1, cu_seqlens_k_out, params->batch + 1))
    return fail(FP2_EINVAL, "cu_seqlens_k_out must not overlap cu_seqlens_k");
  CacheProblem r = make_problem(params, nullptr, nullptr, cu_seqlens_k, cache, block_table);
  r.sink = params->sink_tokens;
  fp2::PageMap to = r.pm;
  to.table = target_table;
  to.stride = target_pages;
  return hip_status(fp2::launch_cache_evict(r, to, budget, recent_tokens, weights, weights_stride,
                                            weights_out, weights_stride, kept, cu_seqlens_k_out,
                                            (hipStream_t)stream),
                    "fp2_cache_evict launch");
}

fp2_status_t fp2_rotary(const fp2_rotary_t* rotary, int64_t tokens, const int32_t* positions, int32_t inverse,
                        const fp2_rotary_rows_t* q, const fp2_rotary_rows_t* k, void* stream) {
  fp2_status_t st = check_rotary(rotary);
  if (st != FP2_OK) return st;
  if (tokens < 0) return fail(FP2_EINVAL, "tokens %lld < 0", (long long)tokens);
  if (tokens >= kMaxRows) return fail(FP2_EUNSUPPORTED, "tokens %lld >= 2^31", (long long)tokens);
  if (inverse != 0 && inverse != 1) return fail(FP2_EINVAL, "inverse %d is not 0 or 1", inverse);
  if (!q) return fail(FP2_EINVAL, "q is null");
  if ((st = check_rows("q", q, tokens)) || (k && (st = check_rows("k", k, tokens)))) return st;
  if (tokens == 0) return ok();
  if (!positions) return fail(FP2_EINVAL, "positions is null");
  const Extent pos{(const char*)positions, 4, 4, tokens};
  if (rows_meet(out_of(q, tokens), pos) || (k && rows_meet(out_of(k, tokens), pos)))
    return fail(FP2_EINVAL, "an output overlaps positions");
  if (!in_place(q) && rows_meet(out_of(q, tokens), in_of(q, tokens)))
    return fail(FP2_EINVAL, "q: out overlaps x without being the same");
  if (k) {
    if (!in_place(k) && rows_meet(out_of(k, tokens), in_of(k, tokens)))
      return fail(FP2_EINVAL, "k: out overlaps x without being the same");
    if (rows_meet(out_of(q, tokens), in_of(k, tokens)) || rows_meet(out_of(k, tokens), in_of(q, tokens)) ||
        rows_meet(out_of(q, tokens), out_of(k, tokens)))
      return fail(FP2_EINVAL, "q and k: an output overlaps the other's rows");
  }
  return hip_status(fp2::launch_rotary(make_rotary(rotary, inverse, true), rotary->interleaved, tokens, positions,
                                       make_rows(q), make_rows(k), (hipStream_t)stream),
                    "fp2_rotary launch");
}

fp2_status_t fp2_cache_append_rotary(const fp2_cache_params_t* params, const fp2_rotary_t* rotary,
                                     const fp2_rotary_rows_t* q, const void* k_new, int64_t k_stride,
                                     const void* v_new, int64_t v_stride, const int32_t* positions,
                                     const int32_t* cu_seqlens, const int32_t* cu_seqlens_host,
                                     const int32_t* cu_seqlens_k, const int32_t* cu_seqlens_k_host,
                                     const fp2_kv_cache_t* cache, const int32_t* block_table, void* stream) {
  fp2_status_t st = check_params(params);
  if (st != FP2_OK) return st;
  if ((st = check_rotary(rotary))) return st;
  if (params->batch == 0 || params->max_seq_len == 0) return ok();
  if ((st = check_lengths(params, cu_seqlens, cu_seqlens_host, cu_seqlens_k, cu_seqlens_k_host, true)))
    return st;
  if ((st = check_cache(params, cache, block_table, true))) return st;
  const int width = params->num_kv_heads * fp2::kHeadDim;
  if ((st = check_strided("k_new", k_new, k_stride, width)) || (st = check_strided("v_new", v_new, v_stride, width)))
    return st;
  if (q) {
    if ((st = check_rows("q", q, -1))) return st;
    if (q->heads != params->num_q_heads)
      return fail(FP2_EINVAL, "q has %d heads, params %d", q->heads, params->num_q_heads);
    if (cu_seqlens_host) {   // then the rows that are read and written are known
      const int64_t n = cu_seqlens_host[params->batch];
      const Extent o = out_of(q, n), ks{(const char*)k_new, 2 * k_stride, 2ll * width, n},
                   vs{(const char*)v_new, 2 * v_stride, 2ll * width, n}, pos{(const char*)positions, 4, 4, positions ? n : 0};
      if (!in_place(q) && rows_meet(o, in_of(q, n))) return fail(FP2_EINVAL, "q: out overlaps x without being the same");
      if (rows_meet(o, ks) || rows_meet(o, vs) || rows_meet(o, pos))
        return fail(FP2_EINVAL, "q: out overlaps k_new, v_new or positions");
    }
  }
  const CacheProblem r = make_problem(params, nullptr, cu_seqlens, cu_seqlens_k, cache, block_table);
  return hip_status(fp2::launch_cache_append_rotary(r, make_rotary(rotary, false, true), rotary->interleaved, make_rows(q),
                                                    (const uint16_t*)k_new, k_stride, (const uint16_t*)v_new, v_stride,
                                                    positions, (hipStream_t)stream),
                    "fp2_cache_append_rotary launch");
}

fp2_status_t fp2_cache_read(const fp2_cache_params_t* params, const fp2_rotary_t* rotary, const int32_t* positions,
                            const int32_t* cu_seqlens, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens_k,
                            const int32_t* cu_seqlens_k_host, const fp2_kv_cache_t* cache, const int32_t* block_table,
                            void* k_out, void* v_out, void* stream) {
  fp2_status_t st = check_params(params);
  if (st != FP2_OK) return st;
  if (rotary && (st = check_rotary(rotary))) return st;
  if (!rotary && positions) return fail(FP2_EINVAL, "positions without rotary");
  if (params->batch == 0 || params->max_seq_len == 0) return ok();
  if ((st = check_lengths(params, cu_seqlens, cu_seqlens_host, cu_seqlens_k, cu_seqlens_k_host, true)))
    return st;
  if (!k_out && !v_out) return fail(FP2_EINVAL, "k_out and v_out are null");
  if ((st = check_cache(params, cache, block_table, v_out != nullptr))) return st;
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return fail(FP2_EINVAL, "k_out and v_out must be 16-byte aligned");
  if (cu_seqlens_host) {   // then the rows that are written are known
    const int64_t rows = cu_seqlens_host[params->batch], n = 2 * rows * params->num_kv_heads * fp2::kHeadDim;
    const char *ko = (const char*)k_out, *vo = (const char*)v_out, *pos = (const char*)positions;
    if (ko && vo && overlap(ko, n, vo, n)) return fail(FP2_EINVAL, "k_out overlaps v_out");
    if (pos && ((ko && overlap(ko, n, pos, 4 * rows)) || (vo && overlap(vo, n, pos, 4 * rows))))
      return fail(FP2_EINVAL, "an output overlaps positions");
  }
  const CacheProblem r = make_problem(params, nullptr, cu_seqlens, cu_seqlens_k, cache, block_table);
  return hip_status(fp2::launch_cache_read(r, make_rotary(rotary, true, true), rotary && rotary->interleaved, positions,
                                           (uint16_t*)k_out, (uint16_t*)v_out, (hipStream_t)stream),
                    "fp2_cache_read launch");
}

fp2_status_t fp2_cache_move(const fp2_cache_params_t* params, const fp2_rotary_t* rotary, const int32_t* moves,
                            int64_t batch_stride, int64_t head_stride, int64_t token_stride,
                            const int32_t* cu_seqlens_k, const int32_t* cu_seqlens_k_host, const fp2_kv_cache_t* cache,
                            const int32_t* block_table, const int32_t* target_table, int32_t target_pages, void* stream) {
  fp2_status_t st = check_params(params);
  if (st != FP2_OK) return st;
  if (rotary && (st = check_rotary(rotary))) return st;
  if (!rotary && moves) return fail(FP2_EINVAL, "moves without rotary");
  if (!rotary && !target_table) return fail(FP2_EINVAL, "neither rotary nor target_table: nothing to move");
  if (batch_stride < 0 || head_stride < 0 || token_stride < 0) return fail(FP2_EINVAL, "a stride of moves is negative");
  if (params->batch == 0 || params->max_kv_len == 0) return ok();
  if (rotary && !moves) return fail(FP2_EINVAL, "moves is null");
  if ((st = check_lengths(params, nullptr, nullptr, cu_seqlens_k, cu_seqlens_k_host, false))) return st;
  if ((st = check_cache(params, cache, block_table, target_table != nullptr))) return st;
  CacheProblem r = make_problem(params, nullptr, nullptr, cu_seqlens_k, cache, block_table);
  fp2::PageMap to = r.pm;
  to.table = target_table;
  to.stride = target_pages;
  if (target_table) {
    const int pages = (int)(((int64_t)params->max_kv_len + params->page_size - 1) / params->page_size);
    if (target_table == block_table) return fail(FP2_EINVAL, "target_table is block_table (null moves in place)");
    if (target_pages < pages)
      return fail(FP2_EINVAL, "target_pages %d < %d for %d tokens", target_pages, pages, params->max_kv_len);
  }
  return hip_status(fp2::launch_cache_move(r, make_rotary(rotary, false, false), rotary && rotary->interleaved,
                                           fp2::Moves{moves, batch_stride, head_stride, token_stride}, to,
                                           (hipStream_t)stream),
                    "fp2_cache_move launch");
}

size_t fp2_cache_cross_workspace_bytes(const fp2_cache_params_t* params) {
  if (check_params(params, true) != FP2_OK) return 0;
  const CacheProblem r = make_problem(params, nullptr, nullptr, nullptr, nullptr, nullptr);
  size_t ml, at;
  return attend_bytes(r, &ml, &at, true);
}

fp2_status_t fp2_cache_cross(const fp2_cache_params_t* params, const void* q, const int32_t* cu_seqlens,
                             const int32_t* cu_seqlens_host, const int32_t* cu_seqlens_k,
                             const int32_t* cu_seqlens_k_host, const fp2_kv_cache_t* cache, const int32_t* block_table,
                             void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  fp2_status_t st = check_params(params, true);
  if (st != FP2_OK) return st;
  if (params->batch == 0 || params->max_seq_len == 0) return ok();
  if ((st = check_lengths(params, cu_seqlens, cu_seqlens_host, cu_seqlens_k, cu_seqlens_k_host, true, true)))
    return st;
  // (without keys there is no cache to read)
  if (params->max_kv_len > 0 && (st = check_cache(params, cache, block_table, true))) return st;
  if ((st = check_attention(params, q, out, lse, cu_seqlens_host))) return st;
  const CacheProblem r = make_problem(params, q, cu_seqlens, cu_seqlens_k, cache, block_table);
  size_t ml, at;
  if ((st = check_workspace(workspace, workspace_bytes, attend_bytes(r, &ml, &at, true)))) return st;
  const fp2::CachePartials part{(float*)workspace, (float*)((char*)workspace + ml),
                                (int32_t*)((char*)workspace + at)};
  const hipError_t e =
      few_rows(r) ? fp2::launch_cache_decode(r, part, (uint16_t*)out, lse, (hipStream_t)stream, true)
                  : fp2::launch_cache_cross(r, part, (uint16_t*)out, lse, (hipStream_t)stream);
  return hip_status(e, "fp2_cache_cross launch");
}

}  // extern "C"
