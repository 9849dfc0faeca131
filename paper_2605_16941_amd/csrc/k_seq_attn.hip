// Attention of packed query rows over the keys of their sequence, which lie
// in the pages of a cache or in rows of their own (grouped KV heads; full,
// causal and WINO shadow masks).
//
// A wave owns one (row, head): each lane scores one key of 64, the wave keeps
// the running maximum and sum of the softmax, and adds p_j v_j with the head's
// values spread over its lanes.  Keys the row does not see are not read.
#include "common.h"
#include "operators.h"

namespace wino {
namespace {

// last sequence b with cu[b] <= t
__device__ __forceinline__ int seq_of(const int32_t* cu, int batch, int t) {
  int lo = 0, hi = batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <int HD, class A>
__global__ __launch_bounds__(256) void seq_attn_kernel(AttnCall c) {
  constexpr int E = HD / 64;
  const int lane = threadIdx.x & 63;
  const int h = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int t = blockIdx.x;
  if (h >= c.hq || t < c.cu_q[0] || t >= c.cu_q[c.batch]) return;
  const int b = seq_of(c.cu_q, c.batch, t);
  const int q0 = c.cu_q[b], nq = c.cu_q[b + 1] - q0, i = t - q0;
  int k0 = 0, nkv;
  if (c.paged) {
    nkv = c.kv_len[b];
  } else {
    k0 = min(max(c.cu_k[b], 0), c.total_k);
    nkv = min(c.cu_k[b + 1], c.total_k) - k0;
  }
  nkv = min(max(nkv, 0), c.max_kv);
  int end = nkv, skip = -1;
  if (c.mask == 1) end = min(end, nkv - nq + i + 1);
  if (c.mask == 2) {
    const int s = i - (nq - c.block_len);
    if (s < 0) end = nkv - c.block_len;
    else skip = c.cur_start[b] + s;
  }
  const uint16_t* q = c.q.p + t * c.q.ts + h * c.q.hs;
  const int hk = h / (c.hq / c.hk);
  const float sc = c.scale * 1.4426950408889634f;
  float m = kNegBig, l = 0.f, o[E] = {};
  for (int j0 = 0; j0 < end; j0 += 64) {
    const int j = j0 + lane;
    bool ok = j < end && j != skip;
    int64_t ko = 0, vo = 0;
    if (ok && c.paged) {
      const int page = c.table[b * c.table_stride + (j >> c.page_shift)];
      ok = page >= 0 && page < c.n_pages;
      ko = vo = (int64_t)page * c.page_stride + (j & ((1 << c.page_shift) - 1)) * c.k_ts;
    } else if (ok) {
      ko = (int64_t)(k0 + j) * c.k_ts;
      vo = (int64_t)(k0 + j) * c.v_ts;
    }
    float s = kNegBig;
    if (ok) {
      s = 0.f;
      for (int e = 0; e < HD; ++e) s += A::val(q[e]) * A::val(c.k[ko + hk * c.k_hs + e]);
      s *= sc;
    }
    const float mn = fmaxf(m, valu_max(s));
    const float al = exp2f(m - mn), p = ok ? exp2f(s - mn) : 0.f;
    l = l * al + valu_sum(p);
    m = mn;
    for (int e = 0; e < E; ++e) o[e] *= al;
    for (int n = 0; n < 64; ++n) {
      if (!__shfl(ok, n)) continue;
      const float pn = __shfl(p, n);
      const int64_t v = __shfl(vo, n);
      for (int e = 0; e < E; ++e) o[e] += pn * A::val(c.v[v + hk * c.v_hs + lane * E + e]);
    }
  }
  uint16_t* out = c.o.p + t * c.o.ts + h * c.o.hs;
  for (int e = 0; e < E; ++e) out[lane * E + e] = A::cvt(l > 0.f || l != l ? o[e] / l : 0.f);
  if (c.lse && lane == 0)
    c.lse[(int64_t)t * c.hq + h] = l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace

size_t attention_workspace(const AttnCall&) { return 0; }

hipError_t launch_seq_attention(const AttnCall& c, hipStream_t st) {
  const dim3 grid(c.total_q, (c.hq + 3) / 4);
  if (c.f16) {
    if (c.hd == 128) seq_attn_kernel<128, ActF16><<<grid, 256, 0, st>>>(c);
    else seq_attn_kernel<64, ActF16><<<grid, 256, 0, st>>>(c);
  } else {
    if (c.hd == 128) seq_attn_kernel<128, ActBf16><<<grid, 256, 0, st>>>(c);
    else seq_attn_kernel<64, ActBf16><<<grid, 256, 0, st>>>(c);
  }
  return hipGetLastError();
}

}  // namespace wino
