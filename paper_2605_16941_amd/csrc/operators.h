// Launch interface of the operators on a caller's own tensors (k_rope.hip,
// k_seq_attn.hip); the host checks are in operators.cpp.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace wino {

// Rows of heads: element e of head h of row t at p[t * ts + h * hs + e].
struct Heads {
  uint16_t* p;
  int64_t ts, hs;
};

struct RopeCall {
  int hd, rot, interleaved, f16;
  float sign, magnitude;  // sign -1: inverse
  int64_t n_tokens;
  const double* freq;  // [rot / 2] radians per position
  const int32_t* pos;  // [n_tokens]
  int nq;
  Heads q, qo;
  // cache write (nk = 0: none)
  int nk;
  Heads k, v;
  const int64_t* slot;
  uint16_t *ck, *cv;
  int64_t page_stride, token_stride, head_stride;
  int64_t n_slots;
  int page_shift;
};
hipError_t launch_rope(const RopeCall& c, hipStream_t st);

struct AttnCall {
  int hq, hk, hd, f16, mask, block_len;
  float scale;
  int batch, total_q, max_kv;
  const int32_t* cu_q;
  const int32_t* cur_start;
  Heads q, o;
  float* lse;
  // keys and values: rows of sequence b from cu_k[b] on, or (paged) pages
  int paged;
  const int32_t* cu_k;
  int total_k;
  const int32_t* kv_len;
  const int32_t* table;
  int64_t table_stride;
  int page_shift, n_pages;
  const uint16_t *k, *v;
  int64_t k_ts, k_hs, v_ts, v_hs;  // token and head strides
  int64_t page_stride;
  void* ws;
};
size_t attention_workspace(const AttnCall& c);  // for these sizes and all smaller ones
bool attention_splits(const AttnCall& c);       // whether this call uses it
hipError_t launch_seq_attention(const AttnCall& c, hipStream_t st);

}  // namespace wino
