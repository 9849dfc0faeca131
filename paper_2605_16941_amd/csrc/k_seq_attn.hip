// Attention of packed query rows over the keys of their sequence, which lie
// in the pages of a cache or in rows of their own (grouped KV heads; full,
// causal and WINO shadow masks).
//
// Rows.  The G = n_heads / n_kv_heads query heads that share a KV head are
// rows of one matrix: row r of a sequence and KV head is token r / G, head
// r % G of the group.  A workgroup owns 32*QW such rows and a chunk of the
// keys, 64 of them at a time.  Long prompts take QW = 4: four waves, each its
// own rows, K and V read from LDS by all four.  Blocks take QW = 2 and single
// tokens QW = 1: KW = 2 waves share 32 rows and split each tile's keys, so that
// the few rows there are do not leave waves idle while the keys stream in; they
// join in LDS at the end.
//
// What bounds it, measured: few rows by memory (single tokens of 64 sequences
// over 8192 keys each, 8 KV heads of 128: 383 us, 5.6 TB/s of keys and values),
// many rows by the matrix cores and the power they take (8192 x 8192, 32 heads of
// 128: 977 us, 1125 TFLOP/s), short sequences by the time until a workgroup's
// first tile (16 sequences of 64 rows, each over 544 keys, 32 KV heads: 41.5 us;
// over 300 to 544 keys 35.8).
//
// Each wave computes S^T = K Q^T (32x32x16 MFMA), so a lane holds 16 keys per
// 32-key block of ONE row and the softmax's running maximum and sum stay in
// the lane (and its partner 32 apart); the same registers, rounded to the
// type, are the B operand of O^T = V^T P^T.  One pass over the keys: O and the
// sum are rescaled when the maximum moves.  The weights are rounded to the type
// there (half a step of each; the sum takes them unrounded), as the products
// with V have 16-bit operands: errors against 64 bits are 2.1-2.3e-3 (bf16) and
// 2.1-2.9e-4 (fp16) in the 2-norm, of which the output's own rounding is 1.7e-3
// and 2.0e-4.  Weights in two parts would double these products.
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
#include <math.h>

#include "operators.h"

namespace wino {
namespace {

constexpr int kThreads = 256;  // of the merge kernel

struct AttnPlan {
  int splits;       // most key chunks a sequence can have
  int chunk_shift;  // log2 of the keys per chunk, at least 8
  float* part_o;   // [splits][total_q * hq][hd] unnormalised
  float2* part_ml; // [splits][total_q * hq] (maximum, sum; a sum below zero: part_o is not written)
};

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

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

// The units of work of a KV head are (sequence, key chunk, row tile), numbered
// sequence by sequence.  Each workgroup finds its own by a scan over the
// sequences' counts: a grid of the host's upper bound then has its idle
// workgroups at the end.  (With idle ones between, every other workgroup say,
// half of the shader engines, which take workgroups in turn, got no work.)
struct Unit {
  Seq seq;
  int b, rem;  // sequence, unit within it (negative: none)
};
// Inclusive sum over the lanes: within rows of 16 by DPP row shifts, then the
// rows' totals by row broadcasts (lane 15 to the next row, lane 31 to the upper
// half).
__device__ __forceinline__ int scan_incl(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);  // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);  // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);  // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15 into rows 1, 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31 into rows 2, 3
  return v;
}
// count(s): units of a sequence.  find(total) is called once the total is
// known and returns the unit to look for, or a negative number for none.
template <class Count, class Find>
__device__ __forceinline__ Unit find_unit(const AttnCall& c, Count count, Find find) {
  const int lane = threadIdx.x & 63;
  const int strip = (c.batch + 63) >> 6;  // consecutive sequences per lane
  int v = 0;
  Seq mine{};
#pragma unroll 4
  for (int j = 0; j < strip; ++j) {
    const int b = lane * strip + j;
    mine = seq_of(c, min(b, c.batch - 1));
    const int n = count(mine);
    v += b < c.batch ? n : 0;
  }
  int incl = scan_incl(v);
  Unit u;
  u.rem = find(__builtin_amdgcn_readlane(incl, 63));
  if (u.rem < 0) return u;
  int at = min(__popcll(__ballot(incl <= u.rem)), 63);  // the lane that holds it
  if (at) u.rem -= __builtin_amdgcn_readlane(incl, at - 1);
  u.b = min(at * strip, c.batch - 1);
  if (strip > 1) {
    for (int lo = u.b, end = min(lo + strip, c.batch); lo < end; lo += 64) {
      mine = seq_of(c, min(lo + lane, c.batch - 1));
      incl = scan_incl(lo + lane < end ? count(mine) : 0);
      at = __popcll(__ballot(incl <= u.rem));
      u.b = min(lo + min(at, 63), c.batch - 1);
      if (at < 64) {
        if (at) u.rem -= __builtin_amdgcn_readlane(incl, at - 1);
        break;
      }
      u.rem -= __builtin_amdgcn_readlane(incl, 63);
    }
    at = min(at, 63);
  }
  u.seq.q0 = __builtin_amdgcn_readlane(mine.q0, at);
  u.seq.nq = __builtin_amdgcn_readlane(mine.nq, at);
  u.seq.k0 = __builtin_amdgcn_readlane(mine.k0, at);
  u.seq.nkv = __builtin_amdgcn_readlane(mine.nkv, at);
  return u;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 4 keys x 16 values from row-major LDS: lane i of 16 passes the address of 4
// values of key i / 4 and gets value i of the 4 keys.
__device__ __forceinline__ uint2 read_tr(uint32_t lds) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) s16x4*)(uintptr_t)lds));
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

// LDS-DMA of N x 64 x 16 bytes: lane l's 16 bytes at base + off[j] go to byte
// lds + 1024 j + 16 l.  Written out, with the waits for it (vmcnt, in the
// kernel), because the compiler otherwise waits for every copy in flight
// before the next transposing read, which it takes for a write to LDS.  The
// instruction's offset counts for both addresses; off[j] already has
// 1024 (N - 1 - j) added and base 1024 (N - 1) subtracted.  m0 is a reserved
// register: the compiler keeps nothing in it, and does not let it be named as
// overwritten.  s_nop 4: a scalar
// that the vector unit wrote (readfirstlane) may be read by a memory
// instruction five wait states later, which the compiler does not see to here.
template <int N>
__device__ __forceinline__ void copy_lds(uint32_t lds, const char* base, const uint32_t* off) {
  if (N == 4) {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 4\n\t"
        "global_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:%6\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:%7\n\tglobal_load_lds_dwordx4 %4, %5 offset:%8" ::"s"(lds),
        "v"(off[0]), "v"(off[1]), "v"(off[N > 2 ? 2 : 0]), "v"(off[N > 2 ? 3 : 0]), "s"(base), "n"(1024), "n"(2 * 1024),
        "n"(3 * 1024)
        : "memory");
  } else {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 4\n\t"
        "global_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024" ::"s"(lds),
        "v"(off[0]), "v"(off[1]), "s"(base)
        : "memory");
  }
}

// Waves per SIMD the registers are kept for: 64-wide heads over packed keys fit
// a third workgroup (8192 causal rows 324 -> 302 us, 24 prompts of up to 700
// rows 36.6 -> 33.5); with the page addresses that spills (295 -> 307 us).
constexpr int attn_threads(int qw) { return qw == 1 ? 128 : 256; }
constexpr int attn_waves(int hd, int qw, bool paged) {
  return hd == 64 && qw == 4 && !paged ? 3 : 2;
}
// Bytes of LDS for the tiles: two stages of K and V, or the waves' outputs if
// those are larger.  32 rows: sequences of one tile need one stage, and twice
// as many workgroups then fit a CU (54 sequences of 11 keys, 32 KV heads:
// 16 us, with two stages 26).
constexpr int attn_lds(int hd, int qw, int stages) {
  const int nw = attn_threads(qw) / 64, tiles = stages * 2 * 64 * hd * 2, outputs = qw < 4 ? nw * 32 * (hd + 4) * 4 : 0;
  return tiles > outputs ? tiles : outputs;
}

template <int HD, int QW, bool PAGED, class A>
__global__ __launch_bounds__(attn_threads(QW), attn_waves(HD, QW, PAGED)) void seq_attn_kernel(AttnCall c, AttnPlan pl) {
  constexpr int NT = attn_threads(QW), NW = NT / 64;
  constexpr int KW = NW / QW;
  constexpr int KB2 = KW == 1 ? 2 : 1;  // 32-key blocks per wave and tile
  constexpr int BKV = 32 * KB2 * KW;    // keys per tile: 64
  constexpr int RSHIFT = QW == 1 ? 5 : (QW == 2 ? 6 : 7);
  constexpr int FE = HD / 32, KS = HD / 16, KCH = HD / 8;
  constexpr int KROWS = 1024 / (2 * HD);     // rows per 1 KB copy
  constexpr int RW = BKV / NW;               // rows each wave copies
  constexpr int INS = RW / KROWS;            // copies per wave and operand
  constexpr int NGW = RW / 16, NG = BKV / 16;  // 16-row groups per wave, per tile
  constexpr int GINS = INS / NGW;            // copies per group
  constexpr int KTILE = BKV * HD, STAGE = 2 * KTILE;
  constexpr int OROW = HD + 4;               // floats per row of the waves' merge
  static_assert(BKV == 64, "attn_lds");
  extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];
  __shared__ float2 sml[KW > 1 ? NW : 1][32];

  const int G = c.hq / c.hk;
  // KV heads fastest: workgroups go to the 8 XCDs in turn, so where the heads
  // divide by 8 (or 8 by them) the row tiles of a head meet in one L2, and every
  // XCD gets the same mix of short and long causal tiles, which run from the
  // last (longest) to the first.  (Whole heads per XCD in contiguous ranges: the
  // same times within 1.5%.)
  int head = 0;
  const Unit unit = find_unit(
      c,
      [&](const Seq& q) {
        const int tiles = (q.nq * G + 32 * QW - 1) >> RSHIFT;
        return tiles * max((q.nkv + (1 << pl.chunk_shift) - 1) >> pl.chunk_shift, 1);
      },
      [&](int per_head) {
        const int p = blockIdx.x, idx = p / c.hk;
        head = p - idx * c.hk;
        return idx < per_head ? idx : -1;
      });
  if (unit.rem < 0) return;
  const int b = unit.b;
  const Seq sq = unit.seq;
  const int n_rows = sq.nq * G;
  const int tiles = (n_rows + 32 * QW - 1) >> RSHIFT;
  const int split = unit.rem / max(tiles, 1);
  const int row0 = (tiles - 1 - (unit.rem - split * tiles)) << RSHIFT;
  const int kbeg = split << pl.chunk_shift;
  // Offsets that do not ascend count wrongly, past 32 bits where every sequence
  // spans most rows: a unit is taken only if it is one of its sequence's, so that
  // nothing outside the tensors is touched whatever the offsets.
  if (row0 < 0 || row0 >= n_rows || split >= pl.splits || (split && kbeg >= sq.nkv)) return;

  const int tid = threadIdx.x, lane = tid & 63, grp = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
  const bool split_out = nkv > (1 << pl.chunk_shift);
  if (split && kbeg >= kend) {  // a chunk of the sequence that this tile does not see
    for (int r = row0 + tid; r < min(row0 + 32 * QW, n_rows); r += NT) {
      const int64_t g = row_base + (int64_t)(r / G) * c.hq + r % G;
      pl.part_ml[(int64_t)split * c.total_q * c.hq + g] = make_float2(kNegBig, -1.f);
    }
    return;
  }
  const int kstop = min(kend, kbeg + (1 << pl.chunk_shift));
  const int ntile = kstop > kbeg ? (kstop - kbeg + BKV - 1) / BKV : 0;

  // this lane's row: its query and what it sees
  int klim = nkv, excl = -1;
  const bool wave_live = row0 + qw * 32 < n_rows;
  const uint16_t* qr;
  {
    const int r = min(row0 + qw * 32 + (lane & 31), n_rows - 1);
    const int tok = r / G, hg = r - tok * G;
    if (c.mask == 1) klim = min(nkv, nkv - sq.nq + tok + 1);
    if (c.mask == 2) {
      if (tok < n_plain) klim = nkv - c.block_len;
      else excl = (int)min((int64_t)cur + (tok - n_plain), (int64_t)0x7FFFFFFF);
    }
    qr = c.q.p + (int64_t)(sq.q0 + tok) * c.q.ts + (int64_t)(head * G + hg) * c.q.hs + grp * 8;
  }

  // ---- copies.  Every 16-row group has a uniform base address and fixed
  // 32-bit per-lane offsets (row within the group, swizzled chunk; 16 token
  // strides are below 2^31 bytes).
  const uint16_t* kbase = c.k + (int64_t)head * c.k_hs + (PAGED ? 0 : (int64_t)sq.k0 * c.k_ts);
  const uint16_t* vbase = c.v + (int64_t)head * c.v_hs + (PAGED ? 0 : (int64_t)sq.k0 * c.v_ts);
  const int32_t* trow = PAGED ? c.table + (int64_t)b * c.table_stride : nullptr;
  const int last_page = PAGED ? max((nkv - 1) >> c.page_shift, 0) : 0;
  const int pmask = PAGED ? (1 << c.page_shift) - 1 : 0;
  uint32_t koff[INS], voff[INS];  // bytes
  auto offset = [&](int n, int row, bool val) {
    const int r = wave * RW + n * KROWS + lane / KCH, pos = lane % KCH;
    const int swz = val ? (KCH == 16 ? (r & 3) * 4 : ((r >> 1) & 1) * 4) : (KCH == 16 ? (r & 15) : ((r ^ ((r & 31) >> 3)) & 7));
    return (uint32_t)row * (uint32_t)(val ? c.v_ts : c.k_ts) * 2u + (uint32_t)(pos ^ swz) * 16u +
           (uint32_t)(GINS - 1 - n % GINS) * 1024u;
  };
#pragma unroll
  for (int n = 0; n < INS; ++n) {
    koff[n] = offset(n, (n % GINS) * KROWS + lane / KCH, false);
    voff[n] = offset(n, (n % GINS) * KROWS + lane / KCH, true);
  }
  // ids of a tile's pages, one 16-key group per lane
  auto load_ids = [&](int t) {
    const int key = kbeg + t * BKV + (lane & (NG - 1)) * 16;
    return PAGED ? trow[min(key >> c.page_shift, last_page)] : 0;
  };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)smem;
  auto issue = [&](int t, bool val, int ids) {
#pragma unroll
    for (int gg = 0; gg < NGW; ++gg) {
      const int key = kbeg + t * BKV + (wave * NGW + gg) * 16;
      const uint16_t* src = val ? vbase : kbase;
      if (PAGED) {
        const int id = __builtin_amdgcn_readlane(ids, wave * NGW + gg);
        src += (int64_t)((uint32_t)id < (uint32_t)c.n_pages ? id : 0) * c.page_stride + (int64_t)(key & pmask) * c.k_ts;
      } else {
        src += (int64_t)min(key, nkv - 1) * (val ? c.v_ts : c.k_ts);
      }
      const char* base = reinterpret_cast<const char*>(uniform_ptr(src)) - (GINS - 1) * 1024;
      const uint32_t dst =
          lds0 + 2u * ((t & 1) * STAGE + (val ? KTILE : 0) + wave * RW * HD + gg * GINS * 512);
      if (!PAGED && key + 16 > nkv) {  // rows past the sequence are copies of its last one
        uint32_t off[GINS];
#pragma unroll
        for (int i = 0; i < GINS; ++i)
          off[i] = offset(gg * GINS + i, max(min(i * KROWS + lane / KCH, nkv - 1 - key), 0), val);
        copy_lds<GINS>(__builtin_amdgcn_readfirstlane(dst), base, off);
      } else {
        copy_lds<GINS>(__builtin_amdgcn_readfirstlane(dst), base, (val ? voff : koff) + gg * GINS);
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

  // Fragment addresses (bytes): one per operand, of step and block 0.  The
  // swizzles XOR address bits that the k step (K) and the 32-value block (V)
  // occupy, so the others follow by XOR with a constant; they are formed anew
  // for every tile, which costs less than the registers that would hold them.
  const int kr = lane & 31, li = lane & 15;
  const int kswz = KCH == 16 ? (kr & 15) : ((kr ^ (kr >> 3)) & 7);
  uint32_t kaddr = lds0 + 2u * (((kw * KB2) * 32 + kr) * HD + (grp ^ kswz) * 8);
  // transposing read: lane i of 16 points at values 4 (i % 4) of key i / 4
  const int vr0 = kw * KB2 * 32 + grp * 4 + (li >> 2);
  const int vch = ((lane >> 4) & 1) * 2 + ((li & 3) >> 1);
  const int vswz = KCH == 16 ? (vr0 & 3) * 4 : ((vr0 >> 1) & 1) * 4;
  uint32_t vaddr = lds0 + 2u * (KTILE + vr0 * HD + (vch ^ vswz) * 8 + (li & 1) * 4);

  auto bad_of = [&](int v) {
    return PAGED ? (uint32_t)__ballot((uint32_t)v >= (uint32_t)c.n_pages) & ((1u << NG) - 1) : 0u;
  };
  auto kfrag = [&](int par, int ks, int kb2) {
    const uint32_t at = (kaddr ^ (uint32_t)(ks * 32)) + (uint32_t)(2 * (par * STAGE + kb2 * 32 * HD));
    const u32x4 v = *(__attribute__((address_space(3))) const u32x4*)(uintptr_t)at;
    return A::frag(make_uint4(v.x, v.y, v.z, v.w));
  };
  // values fe*32 .. +31 (A operand rows) of the 16 keys of step ks4
  auto vfrag = [&](int par, int ks4, int fe) {
    const uint32_t at = (vaddr ^ (uint32_t)(fe * 64)) + (uint32_t)(2 * (par * STAGE + ks4 * 16 * HD));
    const uint2 lo = read_tr(at), hi = read_tr(at + 2 * 8 * HD);
    return A::frag(make_uint4(lo.x, lo.y, hi.x, hi.y));
  };
  auto zero = [](f32x16 (&s)[KB2]) {
#pragma unroll
    for (int kb2 = 0; kb2 < KB2; ++kb2)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb2][i] = 0.f;
  };
  // page ids of tiles t, t + 1, t + 2
  int id0 = 0, id1 = 0, id2 = 0;

  typename A::v8 qf[KS];

  // Tile t: its scores are in s.  While their exponentials are taken, the
  // scores of tile t + 1 are computed into sn (the matrix cores and the vector
  // units work at once within the wave); then O += V^T P^T.  K(t + 1) and V(t)
  // were requested a tile ago; K(t + 2) and V(t + 1) are requested here.
  auto step = [&](int t, auto parity, auto has_next, f32x16 (&s)[KB2], f32x16 (&sn)[KB2]) {
    const int par = parity;
    constexpr bool NEXT = decltype(has_next)::value;
    const int kv0 = kbeg + t * BKV;
    const uint32_t bad = bad_of(id0);
    const bool edge = kv0 + BKV > kmin || bad || (kv0 < ex1 && kv0 + BKV > ex0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (edge) {
      // this wave's rows of V: cleared where no row sees them or not finite
#pragma unroll
      for (int i = 0; i < INS; ++i) {
        const int r = wave * RW + i * KROWS + lane / KCH;
        uint4* p = reinterpret_cast<uint4*>(smem + par * STAGE + KTILE + wave * RW * HD + i * 512 + lane * 8);
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
    if (NEXT) {
      id0 = id1;
      id1 = id2;
      if (PAGED) asm volatile("" : "+v"(id0), "+v"(id1));  // in registers before the copies start
      issue(t + 1, true, id0);
      if (t + 2 < ntile) issue(t + 2, false, id1);
      if (PAGED) id2 = load_ids(t + 3);
    }
    if (!wave_live) return;
    asm volatile("" : "+v"(kaddr), "+v"(vaddr));

    if (edge) {
      // register i of block kb2 holds key key0 + 32 kb2 + 8 (i / 4) + i % 4
      const int key0 = kv0 + kw * KB2 * 32 + 4 * grp;
      const int lim = klim - key0;
#pragma unroll
      for (int kb2 = 0; kb2 < KB2; ++kb2)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[kb2][i] = kb2 * 32 + 8 * (i >> 2) + (i & 3) < lim ? s[kb2][i] : kNegBig;
      if (bad || ex1 > ex0) {
        const int ex = (int)((uint32_t)excl - (uint32_t)key0);  // (a key that is not excluded from this row: below them all)
#pragma unroll
        for (int kb2 = 0; kb2 < KB2; ++kb2)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool out = kb2 * 32 + 8 * (i >> 2) + (i & 3) == ex || ((bad >> ((kw * KB2 + kb2) * 2 + (i >> 3))) & 1);
            s[kb2][i] = out ? kNegBig : s[kb2][i];
          }
      }
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

    // exponentials of s and scores of the next tile
    float psum = 0.f;
    uint32_t ph[KB2 * 8];
    constexpr int NE = KB2 * 16, PER = NE / KS;  // exponentials per k step
    constexpr int AHEAD = 1;  // K reads run this many steps before their MFMAs
    typename A::v8 kf[AHEAD + 1][KB2];
    if (NEXT) {
      zero(sn);
#pragma unroll
      for (int ks = 0; ks < AHEAD; ++ks)
#pragma unroll
        for (int kb2 = 0; kb2 < KB2; ++kb2) kf[ks][kb2] = kfrag(par ^ 1, ks, kb2);
      __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * KB2, 0);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (NEXT) {
        if (ks + AHEAD < KS)
#pragma unroll
          for (int kb2 = 0; kb2 < KB2; ++kb2) kf[(ks + AHEAD) % (AHEAD + 1)][kb2] = kfrag(par ^ 1, ks + AHEAD, kb2);
#pragma unroll
        for (int kb2 = 0; kb2 < KB2; ++kb2) sn[kb2] = A::mma(kf[ks % (AHEAD + 1)][kb2], qf[ks], sn[kb2]);
      }
#pragma unroll
      for (int x = 0; x < PER; x += 2) {
        const int n = ks * PER + x;
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[n >> 4][n & 15], scale_log2, -mc));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[n >> 4][(n & 15) + 1], scale_log2, -mc));
        psum += p0;
        psum += p1;
        ph[n >> 1] = A::pack2(p0, p1);
      }
      if (NEXT) {
        // pinned: two K reads, then each MFMA with its share of the vector work
        if (ks + AHEAD < KS) __builtin_amdgcn_sched_group_barrier(0x100, KB2, 0);
#pragma unroll
        for (int kb2 = 0; kb2 < KB2; ++kb2) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x400, PER / KB2, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, PER / KB2 * 5 / 2, 0);
        }
      }
    }
    lrun += psum;
    // (128-wide heads: V reads two products ahead and a raised priority among
    // the SIMD's waves, 1170 -> 1132 us at 8192 x 8192 x 32 heads; 64-wide
    // heads lose 2% to it)
    constexpr int NV = KB2 * 2 * FE, VA = HD == 128 ? 2 : 0;
    typename A::v8 vf[VA + 1];
    if (VA) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int n = 0; n < VA; ++n) vf[n] = vfrag(par, n / FE, n % FE);
      __builtin_amdgcn_sched_group_barrier(0x100, 2 * VA, 0);
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int ks4 = n / FE, fe = n % FE;
      if (n + VA < NV) {
        vf[(n + VA) % (VA + 1)] = vfrag(par, (n + VA) / FE, (n + VA) % FE);
        if (VA) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      const typename A::v8 pf = A::frag(make_uint4(ph[4 * ks4], ph[4 * ks4 + 1], ph[4 * ks4 + 2], ph[4 * ks4 + 3]));
      oacc[fe] = A::mma(vf[n % (VA + 1)], pf, oacc[fe]);
      if (VA) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    if (VA) __builtin_amdgcn_s_setprio(0);
  };

  if (ntile > 0) {
    f32x16 s0[KB2], s1[KB2];
    id0 = load_ids(0);
    id1 = load_ids(1);
    id2 = load_ids(2);
    if (PAGED) asm volatile("" : "+v"(id0), "+v"(id1), "+v"(id2));
    issue(0, false, id0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = A::frag(*reinterpret_cast<const uint4*>(qr + ks * 16));
    issue(0, true, id0);
    if (ntile > 1) issue(1, false, id1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // known to be here: else the compiler, which does not see the copies, waits
    // for the queries again inside the loop, and with that for copies in flight
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
    __syncthreads();
    zero(s0);
    if (wave_live) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int kb2 = 0; kb2 < KB2; ++kb2) s0[kb2] = A::mma(kfrag(0, ks, kb2), qf[ks], s0[kb2]);
    }
    std::integral_constant<int, 0> even;
    std::integral_constant<int, 1> odd;
    std::true_type more;
    std::false_type last;
    int t = 0;
    for (; t + 2 < ntile; t += 2) {
      step(t, even, more, s0, s1);
      step(t + 1, odd, more, s1, s0);
    }
    if (t + 1 < ntile) {
      step(t, even, more, s0, s1);
#pragma unroll
      for (int kb2 = 0; kb2 < KB2; ++kb2) s0[kb2] = s1[kb2];
      ++t;
    }
    step(t, t & 1, last, s0, s1);
  }
  lrun = sum_xor32(lrun);

  // (the row is worked out again: kept, it would cost registers in the loop)
  int row0e = row0;
  asm volatile("" : "+s"(row0e));
  const int re = row0e + qw * 32 + (lane & 31);
  const bool rvalid = re < n_rows;
  const int tok = re / G, hg = re - tok * G;
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
    constexpr int TPR = NT / (32 * QW);  // threads per row
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
      for (int r = row0 + tid / HD; r < min(row0 + 32 * QW, n_rows); r += NT / HD) {
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
  const int n = (sq.nkv + (1 << pl.chunk_shift) - 1) >> pl.chunk_shift;
  if (n <= 1) return;  // the row's one chunk wrote the output
  const float scale_log2 = c.scale * 1.4426950408889634f;
  float M = kNegBig;
  for (int s = lane; s < n; s += 64) M = fmaxf(M, pl.part_ml[s * rows + g].x);
  M = valu_max(M);
  float L = 0.f, o[E] = {};
  const float* p = pl.part_o + g * HD + lane * E;
  for (int s0 = 0; s0 < n; s0 += 64) {
    // a lane per chunk for the weights, then every lane its values of each
    const float2 ml = s0 + lane < n ? pl.part_ml[(s0 + lane) * rows + g] : make_float2(kNegBig, -1.f);
    // Only outputs that were not written are left out.  A chunk whose weight is
    // zero in fp32 still counts: NaN and infinities at keys the row sees are not
    // finite however small their weight.
    const uint64_t unwritten = __ballot(ml.y < 0.f);
    const float w = __builtin_amdgcn_exp2f((ml.x - M) * scale_log2);
    const float l = valu_sum(ml.y < 0.f ? 0.f : w * ml.y);
    L += l;
    const int m = min(64, n - s0);
    for (int s = 0; s < m; ++s) {
      const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s));
      const float* q = p + (s0 + s) * rows * HD;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float v = q[e];
        o[e] += (unwritten >> s) & 1 ? 0.f : ws * v;
      }
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  uint16_t* dst = c.o.p + (int64_t)t * c.o.ts + (int64_t)h * c.o.hs + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = A::cvt(o[e] * inv);
  if (c.lse && lane == 0)
    c.lse[g] = log_sum(M, L, scale_log2);
}

// Rows per workgroup and keys per chunk.
//
// Rows: 32, 64 or 128, by the mean rows of a sequence and KV head: a tile of
// more rows than a sequence has computes on copies, one of fewer reads the
// keys once more per tile.
//
// Chunks: splitting a sequence's keys fills the chip when workgroups are few
// and evens out sequences of different lengths, at the price of a workgroup's
// fixed time per chunk and of partial outputs written and read back.  A unit
// of n keys is taken to last fix + n * key us, key falling from `full` (every
// slot taken) to `alone`; the host knows the longest length only, so the chunk
// taken is the one with the least mean time over two guesses, all sequences of
// that length and lengths spread evenly up to it.  Times measured on 28
// problems (1-256 sequences, 1-2048 rows, 544-16000 keys, both head sizes) with
// every chunk of 2^8..2^13 keys and none: the choice is 2% behind the best of
// them in the mean and 8% at most; on 12 drawn ones 3% and 20%.  Measured both
// ways: one token of one sequence over 8192 keys, 8 KV heads of 128: 127 us
// whole, 24 in chunks of 256, which it takes (21 in 512); 4 sequences of 200-500
// rows over 3000-16000 keys, 32 heads over 4 KV heads: 424 us whole, which it
// takes, 482 in chunks of 1024 (397 in 4096: 7% that the times do not foresee).
// slots: workgroups that run at once (64-wide heads over packed keys have 768 at
// 128 rows; their times were fitted with 512).
struct UnitTimes {
  int slots;
  float fix, full, alone;
};
UnitTimes unit_times(int hd, int qw) {
  if (hd == 128) {
    if (qw == 1) return {512, 4.4f, 0.044f, 0.018f};
    if (qw == 2) return {512, 7.f, 0.055f, 0.0135f};
    return {512, 8.f, 0.0344f, 0.021f};
  }
  if (qw == 1) return {1024, 8.f, 0.0477f, 0.0125f};
  if (qw == 2) return {512, 6.f, 0.03f, 0.009f};
  return {512, 7.f, 0.021f, 0.013f};
}

// log2 of the keys of a whole sequence, of the largest and of the smallest chunk
constexpr int kWhole = 30, kLargest = 20, kSmallest = 8;
constexpr int kMostChunks = 512;

// Partial rows (a row and head of a chunk) a call may have.  It grows with every
// size, so that a workspace for a program's largest sizes serves its smaller
// calls, though those may be split where the largest are not.  64 per key and
// 2^21 hold back what the times below would choose in fewer than 1 of 1000
// problems of up to 512 sequences, 16384 rows and 131072 keys, where by the
// same times the next best is 8% behind at most.
int64_t most_partial_rows(const AttnCall& c) {
  const int64_t chunks = ((int64_t)c.max_kv + (1 << kSmallest) - 1) >> kSmallest;
  if (chunks < 2) return 0;
  const int64_t all = (int64_t)c.total_q * c.hq * (chunks < kMostChunks ? chunks : kMostChunks);
  const int64_t some = c.max_kv < (1 << 15) ? (int64_t)64 * c.max_kv : 1 << 21;
  return all < some ? all : some;
}

struct Choice {
  int qw, splits, chunk_shift;
  int64_t units;  // per KV head, at most
};

Choice choose(const AttnCall& c) {
  Choice x;
  const int64_t rows = (int64_t)c.total_q * (c.hq / c.hk);
  const int64_t per_seq = rows / c.batch;
  x.qw = per_seq <= 32 ? 1 : (per_seq <= 64 ? 2 : 4);
  const int R = 32 * x.qw;
  const int64_t tiles = (rows + R - 1) / R > c.batch ? (rows + R - 1) / R : c.batch;
  const UnitTimes u = unit_times(c.hd, x.qw);
  auto key_time = [&](float units) { return fmaxf(u.alone, u.full * fminf(1.f, units / u.slots)); };
  const float one = (float)tiles * c.hk, part = (float)c.total_q * c.hq * (c.hd + 2) * 8 / 4e6f;
  const int64_t most_partial = most_partial_rows(c);
  x.chunk_shift = kWhole;
  float best = 0.f;
  for (int cs = kLargest + 1; cs >= kSmallest; --cs) {  // the first: not split
    const bool whole = cs > kLargest;
    const int64_t chunk = (int64_t)1 << (whole ? kWhole : cs);
    const int64_t ns = c.max_kv > 0 ? (c.max_kv + chunk - 1) / chunk : 1;
    // (at most 2^22 workgroups, 2^25 rows to join)
    if (!whole && (ns < 2 || ns > kMostChunks || ns * c.total_q * c.hq > most_partial ||
                   (rows / R + c.batch) * ns * c.hk > 1 << 22 || rows * c.hk > 1 << 25))
      continue;
    const float n = (float)(chunk < c.max_kv ? chunk : c.max_kv), s = (float)ns;
    const float us = one * s, ur = one * (s + 1) / 2;
    const float even = ceilf(us / u.slots) * (u.fix + n * key_time(us));
    const float longest = u.fix + n * key_time(ur);
    const float spread = fmaxf(longest, (ur * u.fix + one * c.max_kv / 2 * u.full) / u.slots + longest / 2);
    const float join = whole ? 0.f : 8 + part * (s + (s + 1) / 2);
    const float t = even + spread + join;
    if (whole || t < 0.97f * best) {
      best = t;
      x.chunk_shift = whole ? kWhole : cs;
    }
  }
  x.splits = c.max_kv > 0 ? (int)((c.max_kv + ((int64_t)1 << x.chunk_shift) - 1) >> x.chunk_shift) : 1;
  x.units = (rows / R + c.batch) * x.splits;
  return x;
}

template <int HD, class A>
hipError_t launch_hd(const AttnCall& c, hipStream_t st) {
  const Choice x = choose(c);
  AttnPlan pl{x.splits, x.chunk_shift, nullptr, nullptr};
  const int64_t rows = (int64_t)c.total_q * c.hq;
  if (x.splits > 1) {
    pl.part_o = static_cast<float*>(c.ws);
    pl.part_ml = reinterpret_cast<float2*>(pl.part_o + x.splits * rows * HD);
  }
  const unsigned grid = (unsigned)(x.units * c.hk);
  const int lds = attn_lds(HD, x.qw, x.qw == 1 && c.max_kv <= 64 ? 1 : 2);
  const dim3 block(attn_threads(x.qw));
  if (c.paged) {
    if (x.qw == 1) seq_attn_kernel<HD, 1, true, A><<<grid, block, lds, st>>>(c, pl);
    else if (x.qw == 2) seq_attn_kernel<HD, 2, true, A><<<grid, block, lds, st>>>(c, pl);
    else seq_attn_kernel<HD, 4, true, A><<<grid, block, lds, st>>>(c, pl);
  } else {
    if (x.qw == 1) seq_attn_kernel<HD, 1, false, A><<<grid, block, lds, st>>>(c, pl);
    else if (x.qw == 2) seq_attn_kernel<HD, 2, false, A><<<grid, block, lds, st>>>(c, pl);
    else seq_attn_kernel<HD, 4, false, A><<<grid, block, lds, st>>>(c, pl);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || x.splits == 1) return e;
  seq_attn_merge_kernel<HD, A><<<(unsigned)((rows + 3) / 4), kThreads, 0, st>>>(c, pl);
  return hipGetLastError();
}

}  // namespace

size_t attention_workspace(const AttnCall& c) { return (size_t)most_partial_rows(c) * (c.hd + 2) * 4; }

bool attention_splits(const AttnCall& c) { return choose(c).splits > 1; }

hipError_t launch_seq_attention(const AttnCall& c, hipStream_t st) {
  if (c.f16) return c.hd == 128 ? launch_hd<128, ActF16>(c, st) : launch_hd<64, ActF16>(c, st);
  return c.hd == 128 ? launch_hd<128, ActBf16>(c, st) : launch_hd<64, ActBf16>(c, st);
}

}  // namespace wino
