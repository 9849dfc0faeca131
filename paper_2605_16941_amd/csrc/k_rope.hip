// Rotary positions on rows of heads, and the write of rotated keys and of
// values into a paged cache.
//
// A unit is 16 values of one head: for the half layout 8 of the first half of
// the rotated part and their 8 partners, for the interleaved one 16
// neighbours, in both the 8 pairs 8u..8u+7 (rotary_dim is a multiple of 16),
// and past the rotated part 16 values that are copied.  A thread reads its
// unit whole before it writes it, so a row may be rotated in place.
//
// A wave works on one token, alone or, where tokens are few, beside others that
// take shares of its head rows: its lanes first compute the token's cosines and
// sines, one pair each, and share them through LDS; then hd/16 lanes per head
// walk the wave's head rows.  The angle is taken in 64 bits and reduced to a
// fraction of a turn before the fp32 sine and cosine, so that position 2^20
// is as exact as position 0.  Bound by memory: 4 bytes per value.
#include "common.h"
#include "operators.h"

namespace wino {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int HD, bool INTER, bool STREAM, class A>
__global__ __launch_bounds__(256) void rope_kernel(RopeCall c, int rows, int per_wave) {
  constexpr int U = HD / 16, HPW = 64 / U;
  __shared__ float2 cs[4][HD / 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * 4 + wave;
  const bool live = t < c.n_tokens;
  if (live && lane < c.rot / 2) {
    const double turn = (double)c.pos[t] * c.freq[lane] * 0.15915494309189533576888;
    float s, co;
    sincospif(2.f * (float)(turn - rint(turn)), &s, &co);
    cs[wave][lane] = make_float2(co * c.magnitude, s * c.magnitude * c.sign);
  }
  __syncthreads();
  if (!live) return;
  const int u = lane % U;
  const bool turns = u < c.rot / 16;
  float2 w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = turns ? cs[wave][u * 8 + i] : make_float2(1.f, 0.f);
  // element offsets of the unit's two 16-byte halves
  const int oa = !turns || INTER ? u * 16 : u * 8;
  const int ob = !turns || INTER ? u * 16 + 8 : c.rot / 2 + u * 8;
  const int64_t slot = c.nk ? c.slot[t] : -1;
  const bool writes = slot >= 0 && slot < c.n_slots;
  const int64_t row_off = writes ? (slot >> c.page_shift) * c.page_stride +
                                       (slot & ((1 << c.page_shift) - 1)) * c.token_stride
                                 : 0;
  // one head row's unit: from src to dst, turned or copied
  auto unit = [&](const uint16_t* src, uint16_t* dst, bool rotate, auto stream) {
    const int a = rotate ? oa : u * 16, b = rotate ? ob : u * 16 + 8;
    uint4 xa = *reinterpret_cast<const uint4*>(src + a), xb = *reinterpret_cast<const uint4*>(src + b);
    if (rotate) {
      uint32_t va[4] = {xa.x, xa.y, xa.z, xa.w}, vb[4] = {xb.x, xb.y, xb.z, xb.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a0 = A::val(va[i] & 0xFFFF), a1 = A::val(va[i] >> 16);
        const float b0 = A::val(vb[i] & 0xFFFF), b1 = A::val(vb[i] >> 16);
        if (INTER) {  // words of the first half hold pairs 0..3, of the second 4..7
          va[i] = A::pack2(a0 * w[i].x - a1 * w[i].y, a1 * w[i].x + a0 * w[i].y);
          vb[i] = A::pack2(b0 * w[4 + i].x - b1 * w[4 + i].y, b1 * w[4 + i].x + b0 * w[4 + i].y);
        } else {
          const float2 w0 = w[2 * i], w1 = w[2 * i + 1];
          va[i] = A::pack2(a0 * w0.x - b0 * w0.y, a1 * w1.x - b1 * w1.y);
          vb[i] = A::pack2(b0 * w0.x + a0 * w0.y, b1 * w1.x + a1 * w1.y);
        }
      }
      xa = make_uint4(va[0], va[1], va[2], va[3]);
      xb = make_uint4(vb[0], vb[1], vb[2], vb[3]);
    }
    if (decltype(stream)::value) {
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, xa), reinterpret_cast<u32x4*>(dst + a));
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, xb), reinterpret_cast<u32x4*>(dst + b));
    } else {
      *reinterpret_cast<uint4*>(dst + a) = xa;
      *reinterpret_cast<uint4*>(dst + b) = xb;
    }
  };
  std::bool_constant<STREAM> stream;
  std::false_type keep;
  const int r1 = min(rows, (int)(blockIdx.y + 1) * per_wave);
  int r = blockIdx.y * per_wave + lane / U;
  for (; r < min(c.nq, r1); r += HPW) unit(c.q.p + t * c.q.ts + r * c.q.hs, c.qo.p + t * c.qo.ts + r * c.qo.hs, turns, stream);
  if (!writes) return;
  for (; r < r1; r += HPW) {
    const bool val = r >= c.nq + c.nk;
    const int h = r - c.nq - (val ? c.nk : 0);
    unit(val ? c.v.p + t * c.v.ts + h * c.v.hs : c.k.p + t * c.k.ts + h * c.k.hs,
         (val ? c.cv : c.ck) + row_off + h * c.head_stride, turns && !val, keep);
  }
}

template <int HD, class A>
hipError_t launch_hd(const RopeCall& c, hipStream_t st) {
  // A wave per token where that makes 2048 waves (two per SIMD), else several
  // that share its head rows: 64 tokens of 96 rows
  // of 128 values take 2.9 us, with a wave per token 6.4.
  constexpr int HPW = 64 / (HD / 16);
  const int rows = c.nq + 2 * c.nk, steps = (rows + HPW - 1) / HPW;
  const int64_t want = (2047 + c.n_tokens) / c.n_tokens;
  const int waves = (int)(want < steps ? want : steps);
  const int per_wave = (steps + waves - 1) / waves * HPW;
  const dim3 grid((unsigned)((c.n_tokens + 3) / 4), (unsigned)((rows + per_wave - 1) / per_wave));
  // Large outputs are written past the caches (8448 x 32 x 128: 31.6 -> 24.3 us,
  // 5.7 TB/s; 49 MB of queries beside their keys 35.1 -> 30.8), smaller ones
  // and the cache's rows, which attention reads next, are not (25 MB of queries
  // 13.3 us, past the caches 15.0).
  const bool stream = c.n_tokens * c.nq * HD * 2 > (40 << 20);
  if (c.interleaved) {
    if (stream) rope_kernel<HD, true, true, A><<<grid, 256, 0, st>>>(c, rows, per_wave);
    else rope_kernel<HD, true, false, A><<<grid, 256, 0, st>>>(c, rows, per_wave);
  } else {
    if (stream) rope_kernel<HD, false, true, A><<<grid, 256, 0, st>>>(c, rows, per_wave);
    else rope_kernel<HD, false, false, A><<<grid, 256, 0, st>>>(c, rows, per_wave);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeCall& c, hipStream_t st) {
  if (c.f16) return c.hd == 128 ? launch_hd<128, ActF16>(c, st) : launch_hd<64, ActF16>(c, st);
  return c.hd == 128 ? launch_hd<128, ActBf16>(c, st) : launch_hd<64, ActBf16>(c, st);
}

}  // namespace wino
