// Attention of packed query rows over the keys of their sequence, which lie
// in the pages of a cache or in rows of their own (grouped KV heads; full,
// causal and WINO shadow masks).
//
// Rows.  The G = n_heads / n_kv_heads query heads that share a KV head are
// rows of one matrix: row r of a sequence and KV head is token r / G, head
// r % G of the group.  A workgroup of four waves owns 32*QW such rows and a
// chunk of the keys; KW = 4 / QW waves share 32 rows and split each tile's
// keys.  Long prompts take QW = 4 (every wave its own rows, K and V read from
// LDS by all four); single tokens and blocks take QW = 1 or 2, so that the few
// rows there are do not leave three waves idle while the keys stream in.
//
// Each wave computes S^T = K Q^T (32x32x16 MFMA), so a lane holds 16 keys per
// 32-key block of ONE row and the softmax's running maximum and sum stay in
// the lane (and its partner 32 apart); the same registers, rounded to the
// type, are the B operand of O^T = V^T P^T.  One pass over the keys: O and the
// sum are rescaled when the maximum moves.
//
// K and V tiles go global -> LDS by LDS-DMA, double-buffered, 16-byte chunks
// XOR-swizzled.  V lies in the cache as it was written, one token per row; its
// transposed operand comes out of LDS through the transposing read
// (ds_read_b64_tr_b16: 16 lanes read a 4-key x 16-value block and each gets
// the 4 keys of one value), whose keys 4g..4g+3 and 8+4g..8+4g+3 are the ones
// the score registers hold, so nothing is permuted.
//
// Unseen keys.  A tile that some row does not see whole is an edge tile: its
// scores go through the mask, rows of V that no row of the workgroup sees are
// cleared in LDS (what lies behind a sequence in its last page may be
// anything), and so are infinities and NaN in the others, as 0 * inf would
// reach the rows that do not see them.  If there were any, the rows that do
// see them get them after the output is written (repair).
#include "common.h"
#include "operators.h"

namespace wino {
namespace {

constexpr int kThreads = 256;

struct AttnPlan {
  int tiles;   // row tiles over all sequences (an upper bound: the rest exit)
  int splits;  // key chunks per row tile
  int chunk;   // keys per chunk, a multiple of 128
  float* part_o;   // [splits][total_q * hq][hd] unnormalised
  float2* part_ml; // [splits][total_q * hq] (maximum, sum)
};

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// First row tile of sequence b: every sequence gets the tiles its rows can
// touch in a common grid of R rows plus one, which is enough for its own
// ceil(rows / R) and needs no table.  shift = log2(R).
__device__ __forceinline__ int tile_start(const AttnCall& c, int G, int shift, int b) {
  return ((clampi(c.cu_q[b], 0, c.total_q) * G) >> shift) + b;
}

// The last of `batch` sequences for which starts(b) holds (it holds for a
// leading run of them, or for none: 0); 64 lanes probe at once.
template <class F>
__device__ __forceinline__ int last_seq(int batch, F starts) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = batch;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int at = lane * step;
    const bool yes = at < n && starts(lo + at);
    const int cnt = max(__popcll(__ballot(yes)), 1);
    lo += (cnt - 1) * step;
    n = min(step, n - (cnt - 1) * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

struct Seq {
  int q0, nq, k0, nkv;
};
__device__ __forceinline__ Seq seq_of(const AttnCall& c, int b) {
  Seq s;
  s.q0 = clampi(c.cu_q[b], 0, c.total_q);
  s.nq = clampi(c.cu_q[b + 1], s.q0, c.total_q) - s.q0;
  if (c.paged) {
    s.k0 = 0;
    s.nkv = c.kv_len[b];
  } else {
    s.k0 = clampi(c.cu_k[b], 0, c.total_k);
    s.nkv = clampi(c.cu_k[b + 1], s.k0, c.total_k) - s.k0;
  }
  s.nkv = clampi(s.nkv, 0, c.max_kv);
  return s;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

// 4 keys x 16 values from row-major LDS: lane i of 16 passes the address of 4
// values of key i / 4 and gets value i of the 4 keys.
__device__ __forceinline__ uint2 read_tr(const uint16_t* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) s16x4*)p));
}

// ln sum exp from the maximum (raw scores) and the sum of powers of two
__device__ __forceinline__ float log_sum(float m, float l, float scale_log2) {
  return l == 0.f ? -INFINITY : (m * scale_log2 + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// 0xFFFF in each 16-bit half that is infinite or NaN (exponent all ones)
template <class A>
__device__ __forceinline__ uint32_t nonfinite(uint32_t w) {
  const uint32_t top = A::kF16 ? (w & 0x7C007C00u) + 0x04000400u : (w & 0x7F807F80u) + 0x00800080u;
  return ((top & 0x80008000u) >> 15) * 0xFFFFu;
}

template <int HD, int QW, bool PAGED, class A>
__global__ __launch_bounds__(kThreads, QW == 4 ? 2 : 1) void seq_attn_kernel(AttnCall c, AttnPlan pl) {
  constexpr int KW = 4 / QW;
  constexpr int KB2 = KW == 1 ? 2 : (KW == 2 ? 2 : 1);  // 32-key blocks per wave and tile
  constexpr int BKV = 32 * KB2 * KW;                    // keys per tile: 64, 128, 128
  constexpr int RSHIFT = QW == 1 ? 5 : (QW == 2 ? 6 : 7);
  constexpr int FE = HD / 32, KS = HD / 16, KCH = HD / 8;
  constexpr int KROWS = 1024 / (2 * HD);     // rows per 1 KB copy
  constexpr int RW = BKV / 4;                // rows each wave copies
  constexpr int INS = RW / KROWS;            // copies per wave and operand
  constexpr int NGW = RW / 16, NG = BKV / 16;  // 16-row groups per wave, per tile
  constexpr int GINS = INS / NGW;            // copies per group
  constexpr int KTILE = BKV * HD, STAGE = 2 * KTILE;
  constexpr int OROW = HD + 4;               // floats per row of the waves' merge
  static_assert(KW == 1 || 128 * OROW * 4 <= 2 * STAGE * 2, "merge buffer");
  __shared__ __attribute__((aligned(1024))) uint16_t smem[2 * STAGE];
  __shared__ float2 sml[KW > 1 ? 4 : 1][32];

  const int G = c.hq / c.hk;
  // KV heads spread over the XCDs so that the row tiles of a head meet in one
  // L2: whole heads per XCD where they divide evenly (contiguous ranges),
  // else heads fastest, which leaves every XCD the same mix of short and long
  // causal tiles.  Causal tiles run from the last (longest) to the first.
  const int per_head = pl.tiles * pl.splits;
  int head, idx;
  if ((c.hk & 7) == 0) {
    const int lin = xcd_remap(blockIdx.x, per_head * c.hk);
    head = lin / per_head;
    idx = lin - head * per_head;
  } else {
    head = blockIdx.x % c.hk;
    idx = blockIdx.x / c.hk;
  }
  const int split = idx / pl.tiles;
  const int tile = pl.tiles - 1 - (idx - split * pl.tiles);
  const int b = last_seq(c.batch, [&](int x) { return tile_start(c, G, RSHIFT, x) <= tile; });
  const Seq sq = seq_of(c, b);
  const int n_rows = sq.nq * G;
  const int row0 = (tile - tile_start(c, G, RSHIFT, b)) << RSHIFT;
  if (row0 < 0 || row0 >= n_rows) return;
  const int kbeg = split * pl.chunk;
  if (split && kbeg >= sq.nkv) return;

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, grp = lane >> 5;
  const int qw = wave / KW, kw = wave % KW;
  const int nkv = sq.nkv;

  // what the tile's rows see: keys below kend for some row, below kmin for all
  const int i_first = row0 / G, i_last = (min(row0 + 32 * QW, n_rows) - 1) / G;
  const int n_plain = sq.nq - c.block_len;  // rows before the shadow rows
  int kend = nkv, kmin = nkv, ex0 = 0, ex1 = 0, cur = 0;
  if (c.mask == 1) {
    kend = min(nkv, nkv - sq.nq + i_last + 1);
    kmin = nkv - sq.nq + i_first + 1;
  } else if (c.mask == 2) {
    cur = c.cur_start[b];
    if (i_first < n_plain) kmin = nkv - c.block_len;
    if (i_last < n_plain) kend = kmin;
    else {
      ex0 = cur;
      ex1 = (int)min((int64_t)cur + c.block_len, (int64_t)0x7FFFFFFF);
    }
  }
  const int64_t row_base = (int64_t)sq.q0 * c.hq + (int64_t)head * G;  // of (token 0, head 0 of the group)
  const bool split_out = pl.splits > 1 && nkv > pl.chunk;
  if (split && kbeg >= kend) {  // a chunk of the sequence that this tile does not see
    for (int r = row0 + tid; r < min(row0 + 32 * QW, n_rows); r += kThreads) {
      const int64_t g = row_base + (int64_t)(r / G) * c.hq + r % G;
      pl.part_ml[(int64_t)split * c.total_q * c.hq + g] = make_float2(kNegBig, 0.f);
    }
    return;
  }
  const int kstop = min(kend, kbeg + pl.chunk);
  const int ntile = kstop > kbeg ? (kstop - kbeg + BKV - 1) / BKV : 0;

  // this lane's row
  const int r_lane = row0 + qw * 32 + (lane & 31);
  const bool rvalid = r_lane < n_rows;
  const int r_use = min(r_lane, n_rows - 1);
  const int tok = r_use / G, hg = r_use - tok * G;
  int klim = nkv, excl = -1;
  if (c.mask == 1) klim = min(nkv, nkv - sq.nq + tok + 1);
  if (c.mask == 2) {
    if (tok < n_plain) klim = nkv - c.block_len;
    else excl = (int)min((int64_t)cur + (tok - n_plain), (int64_t)0x7FFFFFFF);
  }
  const bool wave_live = row0 + qw * 32 < n_rows;

  typename A::v8 qf[KS];
  {
    const uint16_t* qr = c.q.p + (int64_t)(sq.q0 + tok) * c.q.ts + (int64_t)(head * G + hg) * c.q.hs;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = A::frag(*reinterpret_cast<const uint4*>(qr + ks * 16 + grp * 8));
  }

  // ---- copies.  Every 16-row group has a uniform base address and fixed
  // per-lane offsets (row within the group, swizzled chunk).
  const uint16_t* kbase = c.k + (int64_t)head * c.k_hs + (PAGED ? 0 : (int64_t)sq.k0 * c.k_ts);
  const uint16_t* vbase = c.v + (int64_t)head * c.v_hs + (PAGED ? 0 : (int64_t)sq.k0 * c.v_ts);
  const int32_t* trow = PAGED ? c.table + (int64_t)b * c.table_stride : nullptr;
  const int last_page = PAGED ? max((nkv - 1) >> c.page_shift, 0) : 0;
  const int pmask = PAGED ? (1 << c.page_shift) - 1 : 0;
  int rin[GINS];         // row within the group
  int kch[INS], vch[INS];  // swizzled source chunk (elements)
#pragma unroll
  for (int i = 0; i < GINS; ++i) rin[i] = i * KROWS + lane / KCH;
#pragma unroll
  for (int i = 0; i < INS; ++i) {
    const int r = wave * RW + i * KROWS + lane / KCH, pos = lane % KCH;
    kch[i] = (pos ^ (KCH == 16 ? (r & 15) : ((r ^ (r >> 3)) & 7))) * 8;
    vch[i] = (pos ^ (KCH == 16 ? (r & 3) * 4 : ((r >> 1) & 1) * 4)) * 8;
  }
  int64_t koff[GINS], voff[GINS];
#pragma unroll
  for (int i = 0; i < GINS; ++i) {
    koff[i] = rin[i] * c.k_ts;
    voff[i] = rin[i] * c.v_ts;
  }
  // ids of a tile's pages, one 16-key group per lane
  auto load_ids = [&](int t) {
    const int key = kbeg + t * BKV + (lane & (NG - 1)) * 16;
    return PAGED ? trow[min(key >> c.page_shift, last_page)] : 0;
  };
  auto issue = [&](int t, int stage, int ids) {
    const int kv0 = kbeg + t * BKV;
    uint16_t* sK = smem + stage * STAGE + wave * RW * HD;
    uint16_t* sV = sK + KTILE;
#pragma unroll
    for (int gg = 0; gg < NGW; ++gg) {
      const int key = kv0 + (wave * NGW + gg) * 16;
      const uint16_t *kg, *vg;
      if (PAGED) {
        const int id = __builtin_amdgcn_readlane(ids, wave * NGW + gg);
        const int64_t off = (int64_t)((uint32_t)id < (uint32_t)c.n_pages ? id : 0) * c.page_stride +
                            (int64_t)(key & pmask) * c.k_ts;
        kg = kbase + off;
        vg = vbase + off;
      } else {
        // keys past the sequence are copies of its last one
        const int k = min(key, nkv - 1);
        kg = kbase + (int64_t)k * c.k_ts;
        vg = vbase + (int64_t)k * c.v_ts;
      }
      const bool tail = !PAGED && key + 16 > nkv;
#pragma unroll
      for (int i = 0; i < GINS; ++i) {
        const int n = gg * GINS + i;
        int64_t ko = koff[i], vo = voff[i];
        if (tail) {
          const int r = max(min(rin[i], nkv - 1 - key), 0);
          ko = r * c.k_ts;
          vo = r * c.v_ts;
        }
        dma16(kg + ko + kch[n] - (n & 3) * 512, sK + (n & ~3) * 512, n & 3);
        dma16(vg + vo + vch[n] - (n & 3) * 512, sV + (n & ~3) * 512, n & 3);
      }
    }
  };

  f32x16 oacc[FE];
#pragma unroll
  for (int fe = 0; fe < FE; ++fe)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[fe][i] = 0.f;
  float mrun = kNegBig, lrun = 0.f;
  int found = 0;  // infinities or NaN cleared from edge tiles
  const float scale_log2 = c.scale * 1.4426950408889634f;
  const float rescale_gap = 8.f / scale_log2;

  // fragment addresses
  const int kr = lane & 31;
  const int li = lane & 15;                       // lane within the transposing read
  const int vrow = grp * 4 + (li >> 2);           // its key, relative to the step
  const int vcol = ((lane >> 4) & 1) * 2 + ((li & 3) >> 1);  // its 16-byte chunk within 32 values
  const int vsub = (li & 1) * 4;

  int ids = 0;
  uint32_t bad = 0, bad_next = 0;
  auto bad_of = [&](int v) {
    return PAGED ? (uint32_t)__ballot((uint32_t)v >= (uint32_t)c.n_pages) & ((1u << NG) - 1) : 0u;
  };
  if (ntile > 0) {
    ids = load_ids(0);
    bad_next = bad_of(ids);
    issue(0, 0, ids);
    ids = load_ids(1);
  }
  for (int t = 0; t < ntile; ++t) {
    const int kv0 = kbeg + t * BKV, stage = t & 1;
    const uint16_t* sK = smem + stage * STAGE;
    uint16_t* sVw = smem + stage * STAGE + KTILE;
    bad = bad_next;
    const bool edge = kv0 + BKV > kmin || bad || (kv0 < ex1 && kv0 + BKV > ex0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (edge) {
      // this wave's rows of V: cleared where no row sees them or not finite
#pragma unroll
      for (int i = 0; i < INS; ++i) {
        const int r = wave * RW + i * KROWS + lane / KCH;
        uint4* p = reinterpret_cast<uint4*>(sVw + wave * RW * HD + i * 512 + lane * 8);
        if (kv0 + r >= kend || ((bad >> (r >> 4)) & 1)) {
          *p = make_uint4(0, 0, 0, 0);
        } else {
          const uint4 w = *p;
          const uint4 m = make_uint4(nonfinite<A>(w.x), nonfinite<A>(w.y), nonfinite<A>(w.z), nonfinite<A>(w.w));
          if (m.x | m.y | m.z | m.w) {
            found = 1;
            *p = make_uint4(w.x & ~m.x, w.y & ~m.y, w.z & ~m.z, w.w & ~m.w);
          }
        }
      }
    }
    __syncthreads();
    if (t + 1 < ntile) {
      bad_next = bad_of(ids);
      issue(t + 1, stage ^ 1, ids);
      if (PAGED) ids = load_ids(t + 2);
    }
    if (!wave_live) continue;
    const uint16_t* sV = sVw;

    auto kfrag = [&](int ks, int kb2) {
      const int r = (kw * KB2 + kb2) * 32 + kr;
      const int swz = KCH == 16 ? (r & 15) : ((r ^ (r >> 3)) & 7);
      return A::frag(*reinterpret_cast<const uint4*>(sK + r * HD + ((ks * 2 + grp) ^ swz) * 8));
    };
    // values fe*32 .. +31 (A operand rows) of the 16 keys of step ks4
    auto vfrag = [&](int ks4, int fe) {
      const int r0 = kw * KB2 * 32 + ks4 * 16 + vrow;
      const int ch = fe * 4 + vcol;
      const int swz = KCH == 16 ? (r0 & 3) * 4 : ((r0 >> 1) & 1) * 4;  // the same 8 rows on
      const uint16_t* p = sV + r0 * HD + (ch ^ swz) * 8 + vsub;
      const uint2 lo = read_tr(p), hi = read_tr(p + 8 * HD);
      return A::frag(make_uint4(lo.x, lo.y, hi.x, hi.y));
    };
    f32x16 s[KB2];
#pragma unroll
    for (int kb2 = 0; kb2 < KB2; ++kb2)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb2][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kb2 = 0; kb2 < KB2; ++kb2) s[kb2] = A::mma(kfrag(ks, kb2), qf[ks], s[kb2]);

    const int key0 = kv0 + kw * KB2 * 32 + 4 * grp;  // key of register i: key0 + 32 kb2 + 8 (i/4) + i%4
    auto seen = [&](int kb2, int i) {
      const int key = key0 + kb2 * 32 + 8 * (i >> 2) + (i & 3);
      return key < klim && key != excl && !((bad >> ((kw * KB2 + kb2) * 2 + (i >> 3))) & 1);
    };
    if (edge) {
#pragma unroll
      for (int kb2 = 0; kb2 < KB2; ++kb2)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb2][i] = seen(kb2, i) ? s[kb2][i] : kNegBig;
    }
    float tmax = kNegBig;
#pragma unroll
    for (int kb2 = 0; kb2 < KB2; ++kb2)
#pragma unroll
      for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, s[kb2][i]);
    tmax = max_xor32(tmax);
    // The reference maximum moves, and O and the sum are rescaled, only when a
    // score exceeds it by more than 8 in the exponent of two: probabilities
    // stay below 2^8 and the rescale is rare after the first tile.
    const bool resc = tmax > mrun + rescale_gap;
    if (__any(resc)) {
      const float mnew = resc ? tmax : mrun;
      const float alpha = __builtin_amdgcn_exp2f((mrun - mnew) * scale_log2);
      lrun *= alpha;
      mrun = mnew;
#pragma unroll
      for (int fe = 0; fe < FE; ++fe)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[fe][i] *= alpha;
    }
    const float mc = mrun == kNegBig ? 0.f : mrun * scale_log2;
    float psum = 0.f;
#pragma unroll
    for (int kb2 = 0; kb2 < KB2; ++kb2)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[kb2][i], scale_log2, -mc));
        s[kb2][i] = p;
        psum += p;
      }
    lrun += psum;

    auto pfrag = [&](int ks4) {
      const int base = 8 * (ks4 & 1);
      const f32x16& x = s[ks4 >> 1];
      return A::frag(make_uint4(A::pack2(x[base], x[base + 1]), A::pack2(x[base + 2], x[base + 3]),
                                A::pack2(x[base + 4], x[base + 5]), A::pack2(x[base + 6], x[base + 7])));
    };
#pragma unroll
    for (int ks4 = 0; ks4 < KB2 * 2; ++ks4) {
      const typename A::v8 pf = pfrag(ks4);
#pragma unroll
      for (int fe = 0; fe < FE; ++fe) oacc[fe] = A::mma(vfrag(ks4, fe), pf, oacc[fe]);
    }
  }
  lrun = sum_xor32(lrun);

  const int64_t part0 = (int64_t)split * c.total_q * c.hq;
  if (KW == 1) {
    const int64_t orow = row_base + (int64_t)tok * c.hq + hg;
    if (rvalid && split_out) {
      float* dst = pl.part_o + (part0 + orow) * HD;
#pragma unroll
      for (int fe = 0; fe < FE; ++fe)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4*>(dst + fe * 32 + mfma_row(i, lane)) =
              make_float4(oacc[fe][i], oacc[fe][i + 1], oacc[fe][i + 2], oacc[fe][i + 3]);
      if (grp == 0) pl.part_ml[part0 + orow] = make_float2(mrun, lrun);
    } else if (rvalid) {
      const float inv = lrun == 0.f ? 0.f : 1.f / lrun;
      uint16_t* dst = c.o.p + (int64_t)(sq.q0 + tok) * c.o.ts + (int64_t)(head * G + hg) * c.o.hs;
#pragma unroll
      for (int fe = 0; fe < FE; ++fe)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<uint2*>(dst + fe * 32 + mfma_row(i, lane)) =
              make_uint2(A::pack2(oacc[fe][i] * inv, oacc[fe][i + 1] * inv),
                         A::pack2(oacc[fe][i + 2] * inv, oacc[fe][i + 3] * inv));
      if (c.lse && grp == 0) c.lse[orow] = log_sum(mrun, lrun, scale_log2);
    }
  } else {
    // the KW waves of a row block meet in LDS
    __syncthreads();  // every wave is done with the last tile
    float* ob = reinterpret_cast<float*>(smem);
    {
      float* dst = ob + (wave * 32 + (lane & 31)) * OROW;
#pragma unroll
      for (int fe = 0; fe < FE; ++fe)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4*>(dst + fe * 32 + mfma_row(i, lane)) =
              make_float4(oacc[fe][i], oacc[fe][i + 1], oacc[fe][i + 2], oacc[fe][i + 3]);
      if (grp == 0) sml[KW > 1 ? wave : 0][lane & 31] = make_float2(mrun, lrun);
    }
    __syncthreads();
    constexpr int TPR = kThreads / (32 * QW);  // threads per row
    constexpr int EPT = HD / TPR;              // values per thread
    const int rl = tid / TPR, e0 = (tid % TPR) * EPT;
    const int r = row0 + rl;
    if (r < n_rows) {
      float M = kNegBig, L = 0.f, wgt[KW];
#pragma unroll
      for (int w = 0; w < KW; ++w) M = fmaxf(M, sml[(rl >> 5) * KW + w][rl & 31].x);
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float2 ml = sml[(rl >> 5) * KW + w][rl & 31];
        wgt[w] = __builtin_amdgcn_exp2f((ml.x - M) * scale_log2);
        L += wgt[w] * ml.y;
      }
      const int tk = r / G, hh = r - tk * G;
      const int64_t orow = row_base + (int64_t)tk * c.hq + hh;
      const float inv = split_out ? 1.f : (L == 0.f ? 0.f : 1.f / L);
      float* po = pl.part_o + (part0 + orow) * HD + e0;
      uint16_t* oo = c.o.p + (int64_t)(sq.q0 + tk) * c.o.ts + (int64_t)(head * G + hh) * c.o.hs + e0;
#pragma unroll
      for (int e = 0; e < EPT; e += 4) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          const float4 x =
              *reinterpret_cast<const float4*>(ob + (((rl >> 5) * KW + w) * 32 + (rl & 31)) * OROW + e0 + e);
          a.x += wgt[w] * x.x; a.y += wgt[w] * x.y; a.z += wgt[w] * x.z; a.w += wgt[w] * x.w;
        }
        if (split_out) *reinterpret_cast<float4*>(po + e) = a;
        else
          *reinterpret_cast<uint2*>(oo + e) =
              make_uint2(A::pack2(a.x * inv, a.y * inv), A::pack2(a.z * inv, a.w * inv));
      }
      if (e0 == 0) {
        if (split_out) pl.part_ml[part0 + orow] = make_float2(M, L);
        else if (c.lse) c.lse[orow] = log_sum(M, L, scale_log2);
      }
    }
  }

  // ---- repair: the cleared infinities and NaN, added for the rows that see
  // their keys (one thread per value and row, in the order of the keys)
  if (!__syncthreads_or(found)) return;
  __syncthreads();  // the output is in memory
  for (int t = 0; t < ntile; ++t) {
    const int kv0 = kbeg + t * BKV;
    const uint32_t tb = bad_of(load_ids(t));
    if (!(kv0 + BKV > kmin || tb || (kv0 < ex1 && kv0 + BKV > ex0))) continue;
    for (int j = 0; j < BKV && kv0 + j < kend; ++j) {
      if ((tb >> (j >> 4)) & 1) continue;
      const int key = kv0 + j, e = tid % HD;
      const int64_t at = PAGED ? (int64_t)trow[key >> c.page_shift] * c.page_stride + (int64_t)(key & pmask) * c.v_ts
                               : (int64_t)key * c.v_ts;
      const uint16_t v = vbase[at + e];
      if (!nonfinite<A>(v)) continue;
      for (int r = row0 + tid / HD; r < min(row0 + 32 * QW, n_rows); r += kThreads / HD) {
        const int tk = r / G, hh = r - tk * G;
        int lim = nkv, ex = -1;
        if (c.mask == 1) lim = min(nkv, nkv - sq.nq + tk + 1);
        if (c.mask == 2) {
          if (tk < n_plain) lim = nkv - c.block_len;
          else ex = (int)min((int64_t)cur + (tk - n_plain), (int64_t)0x7FFFFFFF);
        }
        if (key >= lim || key == ex) continue;
        if (split_out) {
          pl.part_o[(part0 + row_base + (int64_t)tk * c.hq + hh) * HD + e] += A::val(v);
        } else {
          uint16_t* o = c.o.p + (int64_t)(sq.q0 + tk) * c.o.ts + (int64_t)(head * G + hh) * c.o.hs + e;
          *o = A::cvt(A::val(*o) + A::val(v));
        }
      }
    }
  }
}

// Joins the chunks of a row: a wave per (token, head), in the chunks' order.
template <int HD, class A>
__global__ __launch_bounds__(kThreads) void seq_attn_merge_kernel(AttnCall c, AttnPlan pl) {
  constexpr int E = HD / 64;
  const int lane = threadIdx.x & 63;
  const int64_t rows = (int64_t)c.total_q * c.hq;
  const int64_t g = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (g >= rows) return;
  const int t = (int)(g / c.hq), h = (int)(g - (int64_t)t * c.hq);
  if (t < c.cu_q[0] || t >= c.cu_q[c.batch]) return;
  const int b = last_seq(c.batch, [&](int x) { return c.cu_q[x] <= t; });
  const Seq sq = seq_of(c, b);
  const int n = (sq.nkv + pl.chunk - 1) / pl.chunk;
  if (n <= 1) return;  // the row's one chunk wrote the output
  const float scale_log2 = c.scale * 1.4426950408889634f;
  float M = kNegBig;
  for (int s = lane; s < n; s += 64) M = fmaxf(M, pl.part_ml[s * rows + g].x);
  M = valu_max(M);
  float L = 0.f, o[E] = {};
  for (int s = 0; s < n; ++s) {
    const float2 ml = pl.part_ml[s * rows + g];
    if (ml.y == 0.f) continue;  // a chunk the row's tile does not see, or the row does not
    const float w = __builtin_amdgcn_exp2f((ml.x - M) * scale_log2);
    L += w * ml.y;
    const float* p = pl.part_o + (s * rows + g) * HD + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += w * p[e];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  uint16_t* dst = c.o.p + (int64_t)t * c.o.ts + (int64_t)h * c.o.hs + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = A::cvt(o[e] * inv);
  if (c.lse && lane == 0)
    c.lse[g] = log_sum(M, L, scale_log2);
}

struct Choice {
  int qw, splits, chunk, tiles;
};

Choice choose(const AttnCall& c) {
  Choice x;
  const int64_t rows = (int64_t)c.total_q * (c.hq / c.hk);
  const int64_t per_seq = rows / c.batch;
  x.qw = per_seq <= 32 ? 1 : (per_seq <= 64 ? 2 : 4);
  const int R = 32 * x.qw;
  x.tiles = (int)(rows / R) + c.batch;
  const int64_t units = ((rows + R - 1) / R > c.batch ? (rows + R - 1) / R : c.batch) * c.hk;
  const int64_t slots = 512;
  int64_t want = units >= slots ? 1 : (slots + units - 1) / units;
  int64_t chunk = (c.max_kv + want - 1) / want;
  if (chunk < 512) chunk = 512;
  chunk = (chunk + 127) / 128 * 128;
  x.chunk = (int)chunk;
  x.splits = (int)((c.max_kv + chunk - 1) / chunk);
  if (x.splits < 1) x.splits = 1;
  return x;
}

template <int HD, class A>
hipError_t launch_hd(const AttnCall& c, hipStream_t st) {
  const Choice x = choose(c);
  AttnPlan pl{x.tiles, x.splits, x.chunk, nullptr, nullptr};
  const int64_t rows = (int64_t)c.total_q * c.hq;
  if (x.splits > 1) {
    pl.part_o = static_cast<float*>(c.ws);
    pl.part_ml = reinterpret_cast<float2*>(pl.part_o + x.splits * rows * HD);
  }
  const int64_t wgs = (int64_t)x.tiles * x.splits * c.hk;
  const unsigned grid = (unsigned)wgs;
  if (c.paged) {
    if (x.qw == 1) seq_attn_kernel<HD, 1, true, A><<<grid, kThreads, 0, st>>>(c, pl);
    else if (x.qw == 2) seq_attn_kernel<HD, 2, true, A><<<grid, kThreads, 0, st>>>(c, pl);
    else seq_attn_kernel<HD, 4, true, A><<<grid, kThreads, 0, st>>>(c, pl);
  } else {
    if (x.qw == 1) seq_attn_kernel<HD, 1, false, A><<<grid, kThreads, 0, st>>>(c, pl);
    else if (x.qw == 2) seq_attn_kernel<HD, 2, false, A><<<grid, kThreads, 0, st>>>(c, pl);
    else seq_attn_kernel<HD, 4, false, A><<<grid, kThreads, 0, st>>>(c, pl);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || x.splits == 1) return e;
  seq_attn_merge_kernel<HD, A><<<(unsigned)((rows + 3) / 4), kThreads, 0, st>>>(c, pl);
  return hipGetLastError();
}

}  // namespace

size_t attention_workspace(const AttnCall& c) {
  const Choice x = choose(c);
  return x.splits > 1 ? (size_t)x.splits * c.total_q * c.hq * (c.hd + 2) * 4 : 0;
}

hipError_t launch_seq_attention(const AttnCall& c, hipStream_t st) {
  if (c.f16) return c.hd == 128 ? launch_hd<128, ActF16>(c, st) : launch_hd<64, ActF16>(c, st);
  return c.hd == 128 ? launch_hd<128, ActBf16>(c, st) : launch_hd<64, ActBf16>(c, st);
}

}  // namespace wino
