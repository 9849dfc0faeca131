// Host side of the operators on a caller's own tensors: argument checks, the
// rotary frequencies, and the calls' translation for the launchers.
#include "operators.h"

#include <math.h>

#include "wino.h"

using namespace wino;

namespace {

// A launch holds fewer than 2^32 threads: 64 per rotary token, of which four
// make a workgroup; 256 per 32 rows of attention, one row tile more per
// sequence and KV head.
constexpr int64_t kMaxTokens = ((int64_t)1 << 26) - 4;
constexpr int64_t kMaxRows = (int64_t)1 << 28;
constexpr int64_t kMaxSeqHeads = (int64_t)1 << 22;
// 16 rows of keys or values are within 2^31 bytes of each other
constexpr int64_t kMaxKvStride = (int64_t)1 << 26;

bool dtype_ok(int32_t d) { return d == WINO_ACT_BF16 || d == WINO_ACT_FP16; }
bool head_dim_ok(int32_t hd) { return hd == 64 || hd == 128; }

// strides and alignment the kernels' 16-byte accesses need
wino_status check_heads(const wino_heads* x, int64_t n_tokens, int32_t n_heads, int32_t hd, bool output) {
  if (!x || !x->data) return WINO_ERR_INVALID_ARG;
  if (x->token_stride < 0 || x->head_stride < 0) return WINO_ERR_UNSUPPORTED;
  if (x->token_stride % 8 || x->head_stride % 8 || reinterpret_cast<uintptr_t>(x->data) % 16)
    return WINO_ERR_UNSUPPORTED;
  if (output && ((n_tokens > 1 && x->token_stride < hd) || (n_heads > 1 && x->head_stride < hd)))
    return WINO_ERR_SHAPE;
  return WINO_OK;
}

Heads heads(const wino_heads* x) {
  return Heads{static_cast<uint16_t*>(x->data), x->token_stride, x->head_stride};
}

int page_shift(int32_t page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}

wino_status check_cache(const wino_kv_cache* c, bool written) {
  if (!c || !c->k || !c->v) return WINO_ERR_INVALID_ARG;
  if (!dtype_ok(c->dtype)) return WINO_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->n_kv_heads < 1) return WINO_ERR_SHAPE;
  if (!head_dim_ok(c->head_dim)) return WINO_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return WINO_ERR_UNSUPPORTED;
  if (c->page_stride < 0 || c->page_stride % 8 || c->token_stride >= kMaxKvStride) return WINO_ERR_UNSUPPORTED;
  wino_heads rows{c->k, c->token_stride, c->head_stride};
  wino_status s = check_heads(&rows, c->page_size, c->n_kv_heads, c->head_dim, written);
  if (s != WINO_OK) return s;
  if (reinterpret_cast<uintptr_t>(c->v) % 16) return WINO_ERR_UNSUPPORTED;
  if (written && c->n_pages > 1 && c->page_stride < c->head_dim) return WINO_ERR_SHAPE;
  return WINO_OK;
}

wino_status check_rope(const wino_rope_params* p, int64_t n_tokens, int32_t n_heads, const double* freq,
                       const int32_t* pos) {
  if (!p || !freq || !pos) return WINO_ERR_INVALID_ARG;
  if (!dtype_ok(p->dtype) || !isfinite(p->magnitude)) return WINO_ERR_INVALID_ARG;
  if (p->layout != WINO_ROPE_HALF && p->layout != WINO_ROPE_INTERLEAVED) return WINO_ERR_INVALID_ARG;
  if (!head_dim_ok(p->head_dim)) return WINO_ERR_UNSUPPORTED;
  if (p->rotary_dim < 1 || p->rotary_dim > p->head_dim) return WINO_ERR_SHAPE;
  if (p->rotary_dim % 16) return WINO_ERR_UNSUPPORTED;
  if (n_tokens < 0 || n_tokens > kMaxTokens || n_heads < 1 || n_heads > 65535) return WINO_ERR_SHAPE;
  return WINO_OK;
}

RopeCall rope_call(const wino_rope_params* p, int64_t n_tokens, int32_t n_heads, const double* freq,
                   const int32_t* pos, const wino_heads* x, const wino_heads* out) {
  RopeCall c{};
  c.hd = p->head_dim; c.rot = p->rotary_dim; c.interleaved = p->layout == WINO_ROPE_INTERLEAVED;
  c.f16 = p->dtype == WINO_ACT_FP16;
  c.sign = p->inverse ? -1.f : 1.f; c.magnitude = p->magnitude;
  c.n_tokens = n_tokens; c.freq = freq; c.pos = pos;
  c.nq = n_heads; c.q = heads(x); c.qo = heads(out);
  return c;
}

wino_status check_attn(const wino_attn_params* p) {
  if (!p || !dtype_ok(p->dtype)) return WINO_ERR_INVALID_ARG;
  if (p->mask != WINO_MASK_FULL && p->mask != WINO_MASK_CAUSAL && p->mask != WINO_MASK_SHADOW)
    return WINO_ERR_INVALID_ARG;
  if (!(p->scale >= 1e-6f && p->scale <= 1e6f)) return WINO_ERR_INVALID_ARG;
  if (p->n_heads < 1 || p->n_kv_heads < 1 || p->n_heads % p->n_kv_heads || p->n_heads > 65535)
    return WINO_ERR_SHAPE;
  if (p->mask == WINO_MASK_SHADOW && (p->block_len < 1 || p->block_len > (1 << 20))) return WINO_ERR_SHAPE;
  if (!head_dim_ok(p->head_dim)) return WINO_ERR_UNSUPPORTED;
  return WINO_OK;
}

wino_status check_sizes(const wino_attn_params* p, int32_t batch, int32_t total_q, int32_t max_kv) {
  if (batch < 1 || batch > 65535 || total_q < 0 || max_kv < 0 || max_kv > (1 << 30)) return WINO_ERR_SHAPE;
  if ((int64_t)total_q * p->n_heads > kMaxRows || (int64_t)batch * p->n_kv_heads > kMaxSeqHeads)
    return WINO_ERR_SHAPE;
  return WINO_OK;
}

AttnCall attn_call(const wino_attn_params* p, int32_t batch, int32_t total_q, int32_t max_kv) {
  AttnCall c{};
  c.hq = p->n_heads; c.hk = p->n_kv_heads; c.hd = p->head_dim; c.f16 = p->dtype == WINO_ACT_FP16;
  c.mask = p->mask; c.block_len = p->mask == WINO_MASK_SHADOW ? p->block_len : 0; c.scale = p->scale;
  c.batch = batch; c.total_q = total_q; c.max_kv = max_kv;
  return c;
}

// what both attention calls check and take over alike
wino_status prepare_attn(const wino_attn_params* p, AttnCall& c, const int32_t* cu_q, const int32_t* cur_start,
                         const wino_heads* q, const wino_heads* out, float* lse, void* ws, size_t ws_bytes) {
  if (!cu_q || (p->mask == WINO_MASK_SHADOW && !cur_start)) return WINO_ERR_INVALID_ARG;
  wino_status s = check_heads(q, c.total_q, p->n_heads, p->head_dim, false);
  if (s == WINO_OK) s = check_heads(out, c.total_q, p->n_heads, p->head_dim, true);
  if (s != WINO_OK) return s;
  if (attention_splits(c)) {
    const size_t need = attention_workspace(c);
    if (!ws) return WINO_ERR_INVALID_ARG;
    if (ws_bytes < need) return WINO_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(ws) % 16) return WINO_ERR_UNSUPPORTED;
  }
  c.cu_q = cu_q; c.cur_start = p->mask == WINO_MASK_SHADOW ? cur_start : nullptr;
  c.q = heads(q); c.o = heads(out); c.lse = lse; c.ws = ws;
  return WINO_OK;
}

wino_status launched(hipError_t e) { return e == hipSuccess ? WINO_OK : WINO_ERR_HIP; }

}  // namespace

extern "C" {

wino_status wino_rope_frequencies(const wino_rope_config* c, double* h_freq, float* h_magnitude) {
  if (!c || !h_freq || !h_magnitude) return WINO_ERR_INVALID_ARG;
  if (c->scaling < WINO_ROPE_SCALE_NONE || c->scaling > WINO_ROPE_SCALE_PARTS) return WINO_ERR_INVALID_ARG;
  if (!isfinite(c->theta) || c->theta <= 1) return WINO_ERR_INVALID_ARG;
  const bool scaled = c->scaling != WINO_ROPE_SCALE_NONE;
  if (scaled && (!isfinite(c->factor) || c->factor < 1)) return WINO_ERR_INVALID_ARG;
  if (c->rotary_dim < 2 || c->rotary_dim % 2 || c->rotary_dim > 65536) return WINO_ERR_SHAPE;
  if (c->scaling == WINO_ROPE_SCALE_BASE && c->rotary_dim == 2) return WINO_ERR_SHAPE;
  if (c->scaling == WINO_ROPE_SCALE_PARTS &&
      (!(c->orig_len > 0) || !isfinite(c->orig_len) || !isfinite(c->turns_fast) || !isfinite(c->turns_slow) ||
       c->turns_fast <= c->turns_slow))
    return WINO_ERR_INVALID_ARG;
  const double r = c->rotary_dim, two_pi = 6.283185307179586476925286766559;
  double theta = c->theta;
  if (c->scaling == WINO_ROPE_SCALE_BASE) theta *= pow(c->factor, r / (r - 2));
  if (!isfinite(theta)) return WINO_ERR_INVALID_ARG;
  for (int j = 0; j < c->rotary_dim / 2; ++j) {
    double f = pow(theta, -2.0 * j / r);
    if (c->scaling == WINO_ROPE_SCALE_LINEAR) f /= c->factor;
    if (c->scaling == WINO_ROPE_SCALE_PARTS) {
      const double turns = c->orig_len * f / two_pi;
      const double keep = fmin(fmax((turns - c->turns_slow) / (c->turns_fast - c->turns_slow), 0.0), 1.0);
      f = f * keep + f / c->factor * (1 - keep);
    }
    h_freq[j] = f;
  }
  *h_magnitude = c->scaling == WINO_ROPE_SCALE_PARTS ? (float)(0.1 * log(c->factor) + 1.0) : 1.f;
  return WINO_OK;
}

wino_status wino_rope(const wino_rope_params* p, int64_t n_tokens, int32_t n_heads, const double* d_freq,
                      const int32_t* d_pos, const wino_heads* x, const wino_heads* out, void* stream) {
  wino_status s = check_rope(p, n_tokens, n_heads, d_freq, d_pos);
  if (s == WINO_OK) s = check_heads(x, n_tokens, n_heads, p->head_dim, false);
  if (s == WINO_OK) s = check_heads(out, n_tokens, n_heads, p->head_dim, true);
  if (s != WINO_OK || n_tokens == 0) return s;
  return launched(launch_rope(rope_call(p, n_tokens, n_heads, d_freq, d_pos, x, out),
                              static_cast<hipStream_t>(stream)));
}

wino_status wino_rope_append(const wino_rope_params* p, const wino_kv_cache* cache, int64_t n_tokens,
                             int32_t n_heads, const double* d_freq, const int32_t* d_pos, const int64_t* d_slot,
                             const wino_heads* q, const wino_heads* k, const wino_heads* v,
                             const wino_heads* q_out, void* stream) {
  wino_status s = check_rope(p, n_tokens, n_heads, d_freq, d_pos);
  if (s != WINO_OK) return s;
  if (p->inverse || !d_slot) return WINO_ERR_INVALID_ARG;
  s = check_cache(cache, true);
  if (s != WINO_OK) return s;
  if (cache->dtype != p->dtype) return WINO_ERR_INVALID_ARG;
  if (cache->head_dim != p->head_dim || cache->n_kv_heads > 65535) return WINO_ERR_SHAPE;
  s = check_heads(q, n_tokens, n_heads, p->head_dim, false);
  if (s == WINO_OK) s = check_heads(q_out, n_tokens, n_heads, p->head_dim, true);
  if (s == WINO_OK) s = check_heads(k, n_tokens, cache->n_kv_heads, p->head_dim, false);
  if (s == WINO_OK) s = check_heads(v, n_tokens, cache->n_kv_heads, p->head_dim, false);
  if (s != WINO_OK || n_tokens == 0) return s;
  RopeCall c = rope_call(p, n_tokens, n_heads, d_freq, d_pos, q, q_out);
  c.nk = cache->n_kv_heads; c.k = heads(k); c.v = heads(v); c.slot = d_slot;
  c.ck = static_cast<uint16_t*>(cache->k); c.cv = static_cast<uint16_t*>(cache->v);
  c.page_stride = cache->page_stride; c.token_stride = cache->token_stride; c.head_stride = cache->head_stride;
  c.page_shift = page_shift(cache->page_size);
  c.n_slots = (int64_t)cache->n_pages << c.page_shift;
  return launched(launch_rope(c, static_cast<hipStream_t>(stream)));
}

size_t wino_attention_workspace_bytes(const wino_attn_params* p, int32_t batch, int32_t total_q,
                                      int32_t max_kv_len) {
  if (check_attn(p) != WINO_OK || check_sizes(p, batch, total_q, max_kv_len) != WINO_OK) return 0;
  return attention_workspace(attn_call(p, batch, total_q, max_kv_len));
}

wino_status wino_paged_attention(const wino_attn_params* p, const wino_kv_cache* cache, int32_t batch,
                                 int32_t total_q, int32_t max_kv_len, const int32_t* d_cu_q,
                                 const int32_t* d_kv_len, const int32_t* d_page_table, int64_t table_stride,
                                 int32_t table_width, const int32_t* d_cur_start, const wino_heads* q,
                                 const wino_heads* out, float* d_lse, void* d_workspace,
                                 size_t workspace_bytes, void* stream) {
  wino_status s = check_attn(p);
  if (s == WINO_OK) s = check_cache(cache, false);
  if (s == WINO_OK) s = check_sizes(p, batch, total_q, max_kv_len);
  if (s != WINO_OK) return s;
  if (!d_kv_len || !d_page_table || cache->dtype != p->dtype) return WINO_ERR_INVALID_ARG;
  if (cache->n_kv_heads != p->n_kv_heads || cache->head_dim != p->head_dim) return WINO_ERR_SHAPE;
  if (table_width < 0 || table_stride < 0 || (batch > 1 && table_stride < table_width)) return WINO_ERR_SHAPE;
  if (max_kv_len > (int64_t)table_width * cache->page_size) return WINO_ERR_SHAPE;
  AttnCall c = attn_call(p, batch, total_q, max_kv_len);
  s = prepare_attn(p, c, d_cu_q, d_cur_start, q, out, d_lse, d_workspace, workspace_bytes);
  if (s != WINO_OK || total_q == 0) return s;
  c.paged = 1;
  c.kv_len = d_kv_len; c.table = d_page_table; c.table_stride = table_stride;
  c.page_shift = page_shift(cache->page_size); c.n_pages = cache->n_pages;
  c.k = static_cast<const uint16_t*>(cache->k); c.v = static_cast<const uint16_t*>(cache->v);
  c.k_ts = c.v_ts = cache->token_stride; c.k_hs = c.v_hs = cache->head_stride;
  c.page_stride = cache->page_stride;
  return launched(launch_seq_attention(c, static_cast<hipStream_t>(stream)));
}

wino_status wino_packed_attention(const wino_attn_params* p, int32_t batch, int32_t total_q, int32_t total_k,
                                  int32_t max_kv_len, const int32_t* d_cu_q, const int32_t* d_cu_k,
                                  const int32_t* d_cur_start, const wino_heads* q, const wino_heads* k,
                                  const wino_heads* v, const wino_heads* out, float* d_lse, void* d_workspace,
                                  size_t workspace_bytes, void* stream) {
  wino_status s = check_attn(p);
  if (s == WINO_OK) s = check_sizes(p, batch, total_q, max_kv_len);
  if (s != WINO_OK) return s;
  if (!d_cu_k) return WINO_ERR_INVALID_ARG;
  if (total_k < 0) return WINO_ERR_SHAPE;
  s = check_heads(k, total_k, p->n_kv_heads, p->head_dim, false);
  if (s == WINO_OK) s = check_heads(v, total_k, p->n_kv_heads, p->head_dim, false);
  if (s != WINO_OK) return s;
  if (k->token_stride >= kMaxKvStride || v->token_stride >= kMaxKvStride) return WINO_ERR_UNSUPPORTED;
  AttnCall c = attn_call(p, batch, total_q, max_kv_len);
  s = prepare_attn(p, c, d_cu_q, d_cur_start, q, out, d_lse, d_workspace, workspace_bytes);
  if (s != WINO_OK || total_q == 0) return s;
  c.cu_k = d_cu_k; c.total_k = total_k;
  const Heads hk = heads(k), hv = heads(v);
  c.k = hk.p; c.v = hv.p; c.k_ts = hk.ts; c.k_hs = hk.hs; c.v_ts = hv.ts; c.v_hs = hv.hs;
  return launched(launch_seq_attention(c, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
