// Block-sparse attention with a learned relative position bias by buckets
// (gfx950): S = scale Q K^T + table[head][bucket(key - query)] on the kept
// 64 x 64 blocks, softmax over the kept keys, O = P V, and its gradients, that
// of the table included.  Head dim 64, bf16 I/O, fp32 softmax and sums.
//
// The products are those of attn_kernels.hip: two waves per 64-row block, 32
// rows each, everything transposed so that a lane owns one row, 32x32x16 MFMA,
// tiles copied global -> LDS directly into swizzled rows.  What is added:
//
//  * The bias depends on key - query alone, so a 64 x 64 block needs 127 values
//    of its head, which relpos_bias_kernel has laid out by distance, in log2 units.
//    Most blocks lie in one bucket (beyond the largest distance every block
//    does): there the bias is one scalar, added in the fma that scales the score
//    (dK/dV: taken off the row's log-sum), at no cost.  For the others ("mixed") the
//    block's 128-value window goes to LDS as 128 units of 16 bytes, unit W holding
//    values W .. W + 3: a lane's four consecutive keys are then one aligned
//    ds_read_b128 whatever its row, free of bank conflicts, and the eight reads of a
//    block differ by immediates.
//  * A pair whose bucket is -1 has bias -inf: probability 0.  Blocks wholly
//    outside the attended distances, and key blocks past a sequence's length, are
//    cut off a row's block list before the loop; the running maximum starts at a
//    finite -1e30, so that a row with nothing to attend to sums to 0 (O = 0, lse =
//    -inf) without a NaN on the way.
//  * Rows and tokens past a sequence's length read as zeros by the buffers'
//    range check, whatever the memory holds there.
//  * Table gradient: sums of dS per bucket, in fp32.  A block of one bucket adds up
//    in a register per lane.  Of the others the sums along the diagonals are
//    wanted: register e of an accumulator holds one key for 16 query lanes, so two DPP
//    row shifts (left by the key's index in its 16, right by 16 minus it, zeros
//    shifted in) add it to the diagonals that end and begin in those 16 keys: two
//    VALU instructions per 64 scores and no LDS.  The diagonals then go to the
//    plan's order by bucket and a segmented scan over the wave leaves one sum per
//    bucket.  No atomics; every sum has a fixed order.
//  * Lists of very different length (a stripe's rows and columns; grouped heads; few
//    blocks of long lists) are shared by several workgroups and joined in order.
//
// Rounded to fewer bits: P before P V and P^T dO, dS before its products (bf16, the
// matrix cores' input; sums and the table gradient take them in fp32), and the
// outputs.
//
// 8 x 12 x 4096, 7 blocks per row, 3 of them mixed (without a bias, attn_kernels.hip,
// same run; boxes differ by a tenth): forward 79 (72) us, 83 on inputs that change from
// call to call; dQ with the table gradient 120 (98), three waves per SIMD where 24 KiB
// of LDS and 150 registers leave room, not four; dK/dV 127 (113), two waves.  Busy
// cycles of VALU / MFMA / LDS: forward 57 - 58 / 27 - 28 / 16 - 17 %, dQ 50 / 23 / 17 %,
// dK/dV 40 - 42 / 29 / 23 - 24 %.  No unit is full: a wave's steps S -> softmax ->
// product of a block depend on one another, and the waves that fit a SIMD do not fill
// the gaps.
// Measured and not kept: mixed scores that start at their bias in the accumulator, with
// every block on one path (forward 78 at three waves, dQ 124 - 129 against 119 - 122;
// dK/dV keeps it: 135 -> 128); a loop body per kind of block (51 - 61 registers
// spilled); one window instead of two for the forward (76 us); the lane offsets of the
// copies kept over the loop (24 registers spilled, 90 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pf_attn.h"
#include "pf_launch.h"

namespace pf {
namespace {

constexpr int WIN = 128 * 16;        // bytes of a bias window in LDS
constexpr float kFloor = -1e30f;     // running maximum before any key (log2 units)
// Running maximum from which the forward rounds a one-bucket block's scores before
// it takes the maximum off.  Below, one fma does both: the maximum is a rounded
// score, the fma's own is not, and the largest key's exponent is off zero by up to 2^-24
// of it: here 2^-12 of a probability, an eighth of its rounding to bf16; at scores of 2^31
// (where it was measured: NaN, and rows of zeros) past the exponential's range.
constexpr float kLarge = 4096.f;

// Token rows [0, n) of a head: range-checked, 16 bytes at a time.
__device__ __forceinline__ rsrc_t rows_rsrc(const bf16_t *p, int n, uint32_t row_bytes) {
  return make_rsrc(p, n > 0 ? (int64_t)(n - 1) * row_bytes + D * 2 : 0);
}

// Copies of one tile of 64 token rows by the two waves of a workgroup, as
// TileCopy of attn_kernels.hip with a row stride.  All of the address is in the
// lane offset, which the range check sees.
struct RowCopy {
  uint32_t row, chunk;  // this lane's in the first window
  int w4;
  __device__ __forceinline__ void init(int lane, int w) {
    const int x = (((lane >> 4) & 1) << 2) | (((lane >> 5) & 1) << 1);
    w4 = w * 4;
    row = (uint32_t)(w4 * 8 + (lane >> 3));
    chunk = (uint32_t)(((lane & 7) ^ x) << 4);
  }
  // off: byte offset of the tile's first row; NW windows of 8 rows.
  template <int NW = 4>
  __device__ __forceinline__ void issue(rsrc_t r, uint32_t off, uint32_t row_bytes, uint8_t *tile) const {
    // The lane offsets are formed anew each time: kept over the loop they
    // would take the registers of four waves per SIMD.
    uint32_t q = row, ch = chunk;
    asm volatile("" : "+v"(q), "+v"(ch));
    const uint32_t v = q * row_bytes + off;
    sfor<NW>([&](auto i) __attribute__((always_inline)) {
      dma16(r, tile + (w4 + i) * 1024, v + (ch ^ (i & 1) * 16) + i * 8 * row_bytes, 0);
    });
  }
};

// A window of the bias (128 values from byte offset `off` of the head's
// array) as 16-byte units; wave w copies units 64 w .. 64 w + 63.
__device__ __forceinline__ void copy_window(rsrc_t r, int off, uint8_t *win, int lane, int w) {
  dma16(r, win + w * 1024, (uint32_t)(off + (w * 64 + lane) * 4), 0);
}

// MFMA operand rows i0 + l % 32 (k as frag_r) from range-checked memory.
__device__ __forceinline__ bf16x8 frag_b(rsrc_t r, int row, uint32_t row_bytes, int ks, int lane) {
  const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(
      r, (int)((uint32_t)row * row_bytes + ks * 32 + (lane >> 5) * 16), 0, 0);
  return __builtin_bit_cast(bf16x8, v);
}

// Registers 8 p .. 8 p + 7 of accumulator dt (g = 2 dt + p): 16 columns of row
// l % 32, times scale, or zeros where !live, to dst when `store`: the halves swap
// registers so that each lane stores 16 bytes.
__device__ __forceinline__ void put_eight(bf16_t *dst, int g, f32x4 lo, f32x4 hi, float scale, bool live,
                                          bool store, int lane) {
  const uint32_t x0 = pack2(lo[0] * scale, lo[1] * scale), x1 = pack2(lo[2] * scale, lo[3] * scale);
  const uint32_t y0 = pack2(hi[0] * scale, hi[1] * scale), y1 = pack2(hi[2] * scale, hi[3] * scale);
  const auto s0 = __builtin_amdgcn_permlane32_swap(x0, y0, false, false);
  const auto s1 = __builtin_amdgcn_permlane32_swap(x1, y1, false, false);
  u32x4 v = {s0[0], s1[0], s0[1], s1[1]};
  if (!live) v = u32x4{0u, 0u, 0u, 0u};
  if (store) *(u32x4 *)(dst + g * 16 + (lane >> 5) * 8) = v;
}

// Row l % 32's 64 columns: two transposed accumulators.
__device__ __forceinline__ void put_row(bf16_t *dst, const f32x16 (&o)[2], float scale, bool live,
                                        bool store, int lane) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x16 &v = o[g >> 1];
    const int e = 8 * (g & 1);
    put_eight(dst, g, f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]},
              f32x4{v[e + 4], v[e + 5], v[e + 6], v[e + 7]}, scale, live, store, lane);
  }
}

// x of another lane by a DPP control; lanes without a source read 0.
template <int CTRL>
__device__ __forceinline__ float dpp0(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int dppi(int old, int x) {
  return __builtin_amdgcn_update_dpp(old, x, CTRL, ROWS, 0xf, false);
}
constexpr int kRowShl = 0x100, kRowShr = 0x110, kRowBcast15 = 0x142, kRowBcast31 = 0x143;

// One step of a scan over the lanes of a wave, segmented by id (equal ids lie
// next to one another): adds the source lane's sum where the ids agree.
template <int CTRL, int ROWS>
__device__ __forceinline__ void seg_step(float &sum, int id) {
  const int oid = dppi<CTRL, ROWS>(-1, id);
  const float o = __uint_as_float(dppi<CTRL, ROWS>(0, (int)__float_as_uint(sum)));
  sum += oid == id ? o : 0.f;
}
__device__ __forceinline__ void seg_scan(float &sum, int id) {
  seg_step<kRowShr + 1, 0xf>(sum, id);
  seg_step<kRowShr + 2, 0xf>(sum, id);
  seg_step<kRowShr + 4, 0xf>(sum, id);
  seg_step<kRowShr + 8, 0xf>(sum, id);
  seg_step<kRowBcast15, 0xa>(sum, id);
  seg_step<kRowBcast31, 0xc>(sum, id);
}

// What a workgroup of a launch over row blocks (a.nbh heads) works on: a part
// of block blk's list.  Blocks below nlong, the long rows or columns of a mask
// with global stripes, go first in plong parts, the others in pshort.  A block in
// several parts leaves fp32 partial results in slot `slot`, which a second launch
// joins in part order; -1: the block is this workgroup's alone.
struct Work {
  int bh, blk, part, parts, slot;
};
__device__ __forceinline__ Work find_work(const RelposArgs &a, int L) {
  Work k;
  const int lt = a.nbh * a.nlong * a.plong, m = a.ntile - a.nlong;
  if (L < lt) {
    const int u = L / a.plong;
    k = Work{u / a.nlong, u % a.nlong, L - u * a.plong, a.plong, a.plong > 1 ? L : -1};
  } else {
    const int r = L - lt, u = r / a.pshort;
    k = Work{u / m, a.nlong + u % m, r - u * a.pshort, a.pshort,
             a.pshort > 1 ? r + (a.plong > 1 ? lt : 0) : -1};
  }
  return k;
}
// The block that workgroup J of a join works on, and its first slot.
__device__ __forceinline__ Work find_join(const RelposArgs &a, int J) {
  const int lt = a.nbh * a.nlong * a.plong, nl = a.plong > 1 ? a.nbh * a.nlong : 0;
  if (J < nl) return Work{J / a.nlong, J % a.nlong, 0, a.plong, J * a.plong};
  const int u = J - nl, m = a.ntile - a.nlong;
  return Work{u / m, a.nlong + u % m, 0, a.pshort, u * a.pshort + (a.plong > 1 ? lt : 0)};
}

// Slot layouts: an accumulator pair of the two waves register-major (16 bytes
// a lane, a KiB per store), then for the forward the running maximum and sum.
constexpr int kAccFloats = kRelposAccFloats, kFwdSlot = kRelposFwdSlot;
__device__ __forceinline__ void put_acc(float *slot, const f32x16 (&o)[2], int w, int lane) {
  float *q = slot + (w * 64 + lane) * 4;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int dt = i >> 2, e = (i & 3) * 4;
    *(f32x4 *)(q + i * 512) = f32x4{o[dt][e], o[dt][e + 1], o[dt][e + 2], o[dt][e + 3]};
  }
}
// First and one past the last position of a row's block list whose column
// lies in [lo, hi] (columns ascend): counted 64 at a time, one load deep where a
// search would be a chain of them.
__device__ __forceinline__ void trim(const int32_t *col, int &p0, int &p1, int lo, int hi, int lane) {
  int below = 0, upto = 0;
  for (int i = p0; i < p1; i += 64) {
    const bool in = i + lane < p1;
    const int c = in ? col[i + lane] : 0;
    below += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && c < lo));
    upto += __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && c <= hi));
  }
  p1 = p0 + upto;
  p0 = min(p0 + below, p1);
}

// Part wk.part of the positions [p0, p1).
__device__ __forceinline__ void take_part(const Work &wk, int &p0, int &p1) {
  if (wk.parts == 1) return;
  const int per = (p1 - p0 + wk.parts - 1) / wk.parts;
  p0 = min(p1, p0 + wk.part * per);
  p1 = min(p1, p0 + per);
}

// Tokens of sequence b.
__device__ __forceinline__ int seq_len(const RelposArgs &a, int b) {
  return a.kv_len ? min(max(ld_meta(a.kv_len + b), 0), a.Skv) : a.Skv;
}

// The kernel's arguments read again here: those needed after the loop need not
// occupy scalar registers in it.
__device__ __forceinline__ const RelposArgs &late_args() {
  auto *p = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const RelposArgs *)p;
}

// Bias of a block: what the plan says about its distances (info, see
// RelposArgs) and the bias of its middle one, which is that of all of them when
// info names one bucket.
struct BlockBias {
  int info;
  float mid;
};

// Scores are taken out of the accumulators into scalars before a branch changes
// them: as vectors, the two sides' 16 registers would be joined by copies (21
// spilled registers in the forward, 73 -> 90 us).
struct Scores {
  float v[16];
  __device__ __forceinline__ void take(const f32x16 &s) {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = s[e];
  }
  // In log2 units with a mixed block's bias, v c + b; u: the lane's first unit.
  __device__ __forceinline__ void add_window(float c, const uint8_t *u) {
#pragma unroll
    for (int e4 = 0; e4 < 4; ++e4) {
      const f32x4 b = *(const f32x4 *)(u + e4 * 128);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[e4 * 4 + j] = __builtin_fmaf(v[e4 * 4 + j], c, b[j]);
    }
  }
  // Keys from `lim` on (counted from the lane's first) do not exist.
  __device__ __forceinline__ void cut(int lim) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if ((e >> 2) * 8 + (e & 3) >= lim) v[e] = -INFINITY;
  }
  // Entries 8 j .. 8 j + 7 as a bf16 K-operand.
  __device__ __forceinline__ bf16x8 pack(int j) const {
    bf16x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (__bf16)v[8 * j + e];
    return r;
  }
};

// ---------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------
// O and lse of row `row` of a sequence's Sq, the first nrow of which hold
// tokens; l: this lane's keys only.
__device__ __forceinline__ void fwd_store(const RelposArgs &a, int bh, int row, int nrow,
                                          const f32x16 (&o)[2], float m, float l, int lane) {
  l = add_xor32(l);
  const bool store = row >= 0 && row < a.Sq, live = row < nrow;
  bf16_t *O = (bf16_t *)a.Oout.p + bh / a.H * a.Oout.seq + bh % a.H * a.Oout.head + (int64_t)row * a.Oout.tok;
  put_row(O, o, l == 0.f ? 0.f : 1.f / l, live, store, lane);
  if (lane < 32 && store)
    a.lse[(int64_t)bh * a.Sq + row] = live ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

// A workgroup of two waves per 64-row block (or part of its list).
__global__ __launch_bounds__(128, 4) void relpos_fwd_kernel(RelposArgs a) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  uint8_t *const ks = stage_buf<0, TILE>(), *const vs = stage_buf<1, TILE>();
  uint8_t *const w0 = stage_buf<2, WIN>(), *const w1 = stage_buf<3, WIN>();

  const Work wk = find_work(a, xcd_remap(blockIdx.x, gridDim.x));
  const int bh = wk.bh, b = bh / a.H, h = bh % a.H, hk = h / a.G;
  const int len = seq_len(a, b);
  const int start = a.q_start ? min(max(ld_meta(a.q_start + b), 0), a.seq) : 0;
  const int qb = (start >> 6) + wk.blk;
  // Row index of this lane's query, and the rows that hold tokens.
  const int row = qb * BQ + w * 32 + (lane & 31) - start;
  const int nrow = min(max(len - start, 0), a.Sq);
  if (qb * BQ - start >= a.Sq) return;  // a tile past the last row

  const bf16_t *Q = (const bf16_t *)a.Q.p + b * a.Q.seq + h * a.Q.head;
  const bf16_t *K = (const bf16_t *)a.K.p + b * a.K.seq + hk * a.K.head;
  const bf16_t *V = (const bf16_t *)a.V.p + b * a.V.seq + hk * a.V.head;
  const float *bias = a.bias + (int64_t)h * a.bias_ld;
  const uint32_t qrb = (uint32_t)(a.Q.tok * 2), krb = (uint32_t)(a.K.tok * 2), vrb = (uint32_t)(a.V.tok * 2);
  const rsrc_t rq = rows_rsrc(Q, nrow, qrb), rk = rows_rsrc(K, len, krb), rv = rows_rsrc(V, len, vrb);
  const rsrc_t rb = make_rsrc(bias, (int64_t)a.seq * 8);
  const float c = a.scale * kLog2e;

  int p0 = 0, p1 = 0;
  if (nrow > qb * BQ - start && qb < a.nb) {
    p0 = ld_meta(a.row_ptr + qb);
    p1 = ld_meta(a.row_ptr + qb + 1);
    trim(a.col_idx, p0, p1, qb + a.omin, min(qb + a.omax, (len + BQ - 1) / BQ - 1), lane);
    take_part(wk, p0, p1);
  }
  f32x16 o[2];
#pragma unroll
  for (int e = 0; e < 16; ++e) o[0][e] = o[1][e] = 0.f;
  float m_run = kFloor, l_run = 0.f;  // l_run: this lane's keys only
  bool large = false;  // some row's m_run is beyond kLarge

  if (p0 < p1) {
    RowCopy cp;
    cp.init(lane, w);
    auto block_bias = [&](int col) __attribute__((always_inline)) {
      const int d = col - qb;
      return BlockBias{ld_meta(a.info + d + a.nb - 1), ld_meta(bias + d * BQ + a.seq)};
    };
    auto issue_k = [&](int col, uint8_t *win) __attribute__((always_inline)) {
      cp.issue(rk, (uint32_t)(col * BQ) * krb, krb, ks);
      copy_window(rb, ((col - qb) * BQ + a.seq - BQ) * 4, win, lane, w);
    };
    int ccur = ld_meta(a.col_idx + p0);
    issue_k(ccur, w0);
    bf16x8 qf[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) qf[i] = frag_b(rq, row, qrb, i, lane);
    BlockBias bb = block_bias(ccur);
    // The next block, one iteration ahead (the last one again at the end: its
    // copies land and are not read).
    int cn = ld_meta(a.col_idx + min(p0 + 1, p1 - 1));

    // Unit of this lane's first key in the window: key - query + 64.
    const int unit = 64 + (lane >> 5) * 4 - (w * 32 + (lane & 31));
    Scores s[2];
    auto step = [&](int p, const uint8_t *win, uint8_t *wnext) __attribute__((always_inline)) {
      wait_vm<0>();  // this wave's K and window have landed,
      barrier();     // every wave's have, and the last block's V is read
      cp.issue(rv, (uint32_t)(ccur * BQ) * vrb, vrb, vs);
      const BlockBias bn = block_bias(cn);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        f32x16 acc;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = MFMA32(frag_r(ks, kt * 32, i, lane), qf[i], acc);
        s[kt].take(acc);
      }
      wait_vm<4>();  // (no wait: the four V copies may be in flight)
      barrier();     // every wave has read K
      issue_k(cn, wnext);
      // Scores in log2 units: s cm + ca.
      float cm = c, ca = bb.mid;
      if (bb.info >= kRelposMixed) {
        s[0].add_window(c, win + unit * 16);
        s[1].add_window(c, win + unit * 16 + 512);
        cm = 1.f;
        ca = 0.f;
      }
      const int left = len - ccur * BQ;  // keys from the block's first on
      if (left < BQ) {
        s[0].cut(left - (lane >> 5) * 4);
        s[1].cut(left - (lane >> 5) * 4 - 32);
      }
      float bmax = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) bmax = fmaxf(bmax, s[kt].v[e]);
      // The reference m_run (the same in both lanes of a query) moves only when
      // some lane's maximum grew by more than 8 (log2 units): until then the
      // probabilities stay below 2^8.
      const float bm = __builtin_fmaf(bmax, cm, ca);
      if (__builtin_amdgcn_ballot_w64(bm > m_run + 8.0f)) {
        const float m_cand = fmaxf(m_run, max_xor32(bm));
        const float alpha = fast_exp2(m_run - m_cand);
        m_run = m_cand;
        large = __builtin_amdgcn_ballot_w64(fabsf(m_run) > kLarge && m_run > kFloor) != 0;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
      }
      // Beyond kLarge the scores are rounded before the maximum is taken off, as
      // the maximum was.
      if (large && bb.info < kRelposMixed) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[kt].v[e] = __builtin_fmaf(s[kt].v[e], cm, ca);
        cm = 1.f;
        ca = 0.f;
      }
      const float off = ca - m_run;
      float rs = 0.f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = fast_exp2(__builtin_fmaf(s[kt].v[e], cm, off));
          s[kt].v[e] = x;
          rs += x;
        }
      l_run += rs;
      ccur = cn;
      bb = bn;
      cn = ld_meta(a.col_idx + min(p + 2, p1 - 1));
      wait_vm<5>();  // V has landed; the next K and window stay in flight
      barrier();
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x8 pb = s[kt].pack(j);
#pragma unroll
          for (int dt = 0; dt < 2; ++dt)
            o[dt] = MFMA32(frag_t(vs, kt * 32 + j * 16, dt * 32, lane), pb, o[dt]);
        }
    };
    // Two windows in turn: a block's is read after the next one's copy has begun.
    for (int p = p0; p < p1; p += 2) {
      step(p, w0, w1);
      if (p + 1 < p1) step(p + 1, w1, w0);
    }
    wait_vm<0>();  // no copy outlives the workgroup
  }

  const RelposArgs &z = late_args();
  if (wk.slot >= 0) {
    float *slot = z.slots + (int64_t)wk.slot * kFwdSlot;
    put_acc(slot, o, w, lane);
    slot[kAccFloats + w * 128 + lane] = m_run;
    slot[kAccFloats + w * 128 + 64 + lane] = l_run;
    return;
  }
  fwd_store(z, bh, row, nrow, o, m_run, l_run, lane);
}

// Join of the forward's parts in order, online: four workgroups per block, eight
// accumulator registers each.
__global__ __launch_bounds__(128) void relpos_fwd_join_kernel(RelposArgs a) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, g = blockIdx.x & 3;
  const Work wk = find_join(a, blockIdx.x >> 2);
  const int b = wk.bh / a.H, h = wk.bh % a.H;
  const int start = a.q_start ? min(max(ld_meta(a.q_start + b), 0), a.seq) : 0;
  const int first = ((start >> 6) + wk.blk) * BQ - start;
  if (first >= a.Sq) return;  // no part has written
  const int row = first + w * 32 + (lane & 31);
  const float *slot = a.slots + (int64_t)wk.slot * kFwdSlot;
  const float *ml = slot + kAccFloats + w * 128 + lane, *acc = slot + g * 1024 + (w * 64 + lane) * 4;
  float m = kFloor, l = 0.f;
  f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll 4
  for (int p = 0; p < wk.parts; ++p) {
    const int64_t at = (int64_t)p * kFwdSlot;
    const float mp = ml[at], lp = ml[at + 64];
    const f32x4 u = *(const f32x4 *)(acc + at), v = *(const f32x4 *)(acc + at + 512);
    const float mn = fmaxf(m, mp), x = fast_exp2(m - mn), y = fast_exp2(mp - mn);
    l = l * x + lp * y;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo[j] = lo[j] * x + u[j] * y;
      hi[j] = hi[j] * x + v[j] * y;
    }
    m = mn;
  }
  l = add_xor32(l);
  const bool store = row >= 0 && row < a.Sq, live = row < min(max(seq_len(a, b) - start, 0), a.Sq);
  bf16_t *O = (bf16_t *)a.Oout.p + b * a.Oout.seq + h * a.Oout.head + (int64_t)row * a.Oout.tok;
  put_eight(O, g, lo, hi, l == 0.f ? 0.f : 1.f / l, live, store, lane);
  if (g == 0 && lane < 32 && store)
    a.lse[(int64_t)wk.bh * a.Sq + row] = live ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

// ---------------------------------------------------------------------------
// Forward of one query row per sequence (decoding one token)
// ---------------------------------------------------------------------------
// The G query heads of a key/value head are the rows of one tile (G <= 32), so
// keys and values are read once.  A wave works alone, without barriers, on part of
// a (sequence, key/value head)'s block list, with tiles of its own; four of them
// share a workgroup.  The rows differ in head and agree in position: each lane
// reads its head's bias of its keys from memory (256 bytes a head and block).
// 16 sequences of up to 4096 keys, 16 query on 4 key/value heads: 12.4 us (40 MB, 3.3
// TB/s) and 4.1 for the join; on the kernel above, a wave's 64 rows nearly empty and
// every key read four times, 67 us.  Bound by the latency of a wave's four blocks.
__global__ __launch_bounds__(256, 2) void relpos_decode_kernel(RelposArgs a) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  uint8_t *const ks = stage_buf<0, 4 * TILE>() + w * TILE, *const vs = stage_buf<1, 4 * TILE>() + w * TILE;
  const int u = xcd_remap(blockIdx.x, gridDim.x) * 4 + w;
  if (u >= a.nbh * a.pshort) return;
  const int bhk = u / a.pshort, part = u - bhk * a.pshort;
  const int b = bhk / a.Hkv, hk = bhk % a.Hkv;
  const int len = seq_len(a, b);
  const int pos = a.q_start ? min(max(ld_meta(a.q_start + b), 0), a.seq) : 0, qb = pos >> 6;
  const int r = lane & 31, h = hk * a.G + r;
  const bool live = pos < len, mine = r < a.G;

  const bf16_t *K = (const bf16_t *)a.K.p + b * a.K.seq + hk * a.K.head;
  const bf16_t *V = (const bf16_t *)a.V.p + b * a.V.seq + hk * a.V.head;
  const uint32_t krb = (uint32_t)(a.K.tok * 2), vrb = (uint32_t)(a.V.tok * 2);
  const rsrc_t rk = rows_rsrc(K, len, krb), rv = rows_rsrc(V, len, vrb);
  const float c = a.scale * kLog2e;
  int p0 = 0, p1 = 0;
  if (live && qb < a.nb) {
    p0 = ld_meta(a.row_ptr + qb);
    p1 = ld_meta(a.row_ptr + qb + 1);
    trim(a.col_idx, p0, p1, qb + a.omin, min(qb + a.omax, (len + BQ - 1) / BQ - 1), lane);
    take_part(Work{0, 0, part, a.pshort, 0}, p0, p1);
  }
  f32x16 o[2];
#pragma unroll
  for (int e = 0; e < 16; ++e) o[0][e] = o[1][e] = 0.f;
  float m_run = kFloor, l_run = 0.f;
  if (p0 < p1) {
    RowCopy cp;
    cp.init(lane, 0);
    // Bias of this lane's head (rows past G read 0), from key 0's distance on.
    const rsrc_t rb = make_rsrc(a.bias + (int64_t)hk * a.G * a.bias_ld, (int64_t)a.G * a.bias_ld * 4);
    const uint32_t boff =
        (uint32_t)r * (uint32_t)(a.bias_ld * 4) + (uint32_t)(a.seq - pos + (lane >> 5) * 4) * 4u;
    int col = ld_meta(a.col_idx + p0);
    cp.issue<8>(rk, (uint32_t)(col * BQ) * krb, krb, ks);
    bf16x8 qf[4];
    const bf16_t *Q = (const bf16_t *)a.Q.p + b * a.Q.seq + h * a.Q.head;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (mine) v = *(const u32x4 *)(Q + i * 16 + (lane >> 5) * 8);
      qf[i] = __builtin_bit_cast(bf16x8, v);
    }
    u32x4 bv[8];
    auto load_bias = [&](int cb) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        bv[i] = __builtin_amdgcn_raw_buffer_load_b128(
            rb, mine ? (int)(boff + (uint32_t)(cb * BQ + i * 8) * 4u) : 0x7ffffff0, 0, 0);
    };
    load_bias(col);
    cp.issue<8>(rv, (uint32_t)(col * BQ) * vrb, vrb, vs);
    for (int p = p0; p < p1; ++p) {
      const int cn = ld_meta(a.col_idx + min(p + 1, p1 - 1));
      // The waits count the copies alone: eight newer ones, whatever the
      // order of the loads to registers among them.
      wait_vm<8>();  // K has landed; V may be in flight
      f32x16 s[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kt][e] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[kt] = MFMA32(frag_r(ks, kt * 32, i, lane), qf[i], s[kt]);
      }
      wait_vm<63>();  // (K's reads have returned)
      cp.issue<8>(rk, (uint32_t)(cn * BQ) * krb, krb, ks);
      const int lim = len - col * BQ - (lane >> 5) * 4;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint32_t bits = bv[kt * 4 + (e >> 2)][e & 3];
          s[kt][e] = __builtin_fmaf(s[kt][e], c, __uint_as_float(bits));
          if (kt * 32 + (e >> 2) * 8 + (e & 3) >= lim) s[kt][e] = -INFINITY;
        }
      float bmax = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) bmax = fmaxf(bmax, s[kt][e]);
      if (__builtin_amdgcn_ballot_w64(bmax > m_run + 8.0f)) {
        const float m_cand = fmaxf(m_run, max_xor32(bmax));
        const float alpha = fast_exp2(m_run - m_cand);
        m_run = m_cand;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
      }
      float rs = 0.f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = fast_exp2(s[kt][e] - m_run);
          s[kt][e] = x;
          rs += x;
        }
      l_run += rs;
      wait_vm<8>();  // V has landed; the next K stays in flight
      load_bias(cn);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x8 pb = pack_k(s[kt], j);
#pragma unroll
          for (int dt = 0; dt < 2; ++dt)
            o[dt] = MFMA32(frag_t(vs, kt * 32 + j * 16, dt * 32, lane), pb, o[dt]);
        }
      wait_vm<63>();  // (V's reads have returned)
      cp.issue<8>(rv, (uint32_t)(cn * BQ) * vrb, vrb, vs);
      col = cn;
    }
    wait_vm<0>();  // no copy outlives the wave
  }
  if (a.pshort > 1) {
    if (!mine) return;
    float *slot = a.slots + (int64_t)u * kRelposDecodeSlot;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int dt = i >> 2, e = (i & 3) * 4;
      *(f32x4 *)(slot + i * 256 + lane * 4) = f32x4{o[dt][e], o[dt][e + 1], o[dt][e + 2], o[dt][e + 3]};
    }
    slot[2048 + lane] = m_run;
    slot[2112 + lane] = l_run;
    return;
  }
  l_run = add_xor32(l_run);
  put_row((bf16_t *)a.Oout.p + b * a.Oout.seq + h * a.Oout.head, o, l_run == 0.f ? 0.f : 1.f / l_run,
          live, mine, lane);
  if (lane < 32 && mine)
    a.lse[(int64_t)b * a.H + h] = live ? (m_run + __log2f(l_run)) * kLn2 : -INFINITY;
}

// Join of the decode kernel's parts, a workgroup per (sequence, query head):
// 16 threads across the row's columns, four each, 16 threads down the parts; each
// runs through its parts online, then the 16 are added through LDS in order.
__global__ __launch_bounds__(256) void relpos_decode_join_kernel(RelposArgs a) {
  __shared__ float mx[16], red[16][16 * 5];
  const int cg = threadIdx.x & 15, q = threadIdx.x >> 4;
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H, hk = h / a.G, r = h - hk * a.G;
  // Columns 4 cg ..: accumulator group i of lane r (+ 32 for the odd fours).
  const int i = (cg >> 3) * 4 + ((cg & 7) >> 1), lane = r + (cg & 1) * 32;
  const float *slot = a.slots + ((int64_t)b * a.Hkv + hk) * a.pshort * kRelposDecodeSlot;
  float m = kFloor, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int p = q; p < a.pshort; p += 16) {
    const float *s = slot + (int64_t)p * kRelposDecodeSlot;
    const float mp = s[2048 + r], lp = s[2112 + r] + s[2112 + 32 + r];
    const f32x4 v = *(const f32x4 *)(s + i * 256 + lane * 4);
    const float mn = fmaxf(m, mp), x = fast_exp2(m - mn), y = fast_exp2(mp - mn);
    l = l * x + lp * y;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = o[j] * x + v[j] * y;
    m = mn;
  }
  if (cg == 0) mx[q] = m;
  __syncthreads();
  float top = mx[0];
#pragma unroll
  for (int k = 1; k < 16; ++k) top = fmaxf(top, mx[k]);
  const float x = fast_exp2(m - top);
  float *mine = &red[q][cg * 5];
#pragma unroll
  for (int j = 0; j < 4; ++j) mine[j] = o[j] * x;
  mine[4] = l * x;
  __syncthreads();
  if (q) return;
  float s[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 16; ++k)
#pragma unroll
    for (int j = 0; j < 5; ++j) s[j] += red[k][cg * 5 + j];
  const float inv = s[4] == 0.f ? 0.f : 1.f / s[4];
  bf16_t *O = (bf16_t *)a.Oout.p + b * a.Oout.seq + h * a.Oout.head + cg * 4;
  *(u32x2 *)O = u32x2{pack2(s[0] * inv, s[1] * inv), pack2(s[2] * inv, s[3] * inv)};
  if (cg == 0) a.lse[blockIdx.x] = (top + __log2f(s[4])) * kLn2;
}

// ---------------------------------------------------------------------------
// Backward, pass 1: delta, dQ, and the table gradient's sums of this block row
// ---------------------------------------------------------------------------
constexpr int DPITCH = 136;  // floats per diagonal row (units 1 .. 132 are written)

__global__ __launch_bounds__(128, 3) void relpos_bwd_dq_kernel(RelposArgs a) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  uint8_t *const ks = stage_buf<0, TILE>(), *const vs = stage_buf<1, TILE>();
  uint8_t *const win = stage_buf<2, WIN>();
  // Per wave: the diagonals of a block by lane row (16 queries, one half of the
  // keys), zero where a row has none; sums per bucket.
  __shared__ float diag[2][4 * DPITCH];
  __shared__ float bsum[2][kRelposMaxBuckets];

  const int L = xcd_remap(blockIdx.x, gridDim.x);
  const Work wk = find_work(a, L);
  const int bh = wk.bh, qb = wk.blk, b = bh / a.H, h = bh % a.H, hk = h / a.G;
  const int len = seq_len(a, b);
  const int row = qb * BQ + w * 32 + (lane & 31);

  const bf16_t *Q = (const bf16_t *)a.Q.p + b * a.Q.seq + h * a.Q.head;
  const bf16_t *K = (const bf16_t *)a.K.p + b * a.K.seq + hk * a.K.head;
  const bf16_t *V = (const bf16_t *)a.V.p + b * a.V.seq + hk * a.V.head;
  const bf16_t *O = (const bf16_t *)a.O.p + b * a.O.seq + h * a.O.head;
  const bf16_t *dO = (const bf16_t *)a.dO.p + b * a.dO.seq + h * a.dO.head;
  const float *bias = a.bias + (int64_t)h * a.bias_ld;
  const uint32_t qrb = (uint32_t)(a.Q.tok * 2), krb = (uint32_t)(a.K.tok * 2), vrb = (uint32_t)(a.V.tok * 2);
  const uint32_t orb = (uint32_t)(a.O.tok * 2), grb = (uint32_t)(a.dO.tok * 2);
  const rsrc_t rq = rows_rsrc(Q, len, qrb), rk = rows_rsrc(K, len, krb), rv = rows_rsrc(V, len, vrb);
  const rsrc_t ro = rows_rsrc(O, len, orb), rg = rows_rsrc(dO, len, grb);
  const rsrc_t rb = make_rsrc(bias, (int64_t)a.seq * 8);
  const float c = a.scale * kLog2e;

  for (int i = lane; i < 4 * DPITCH; i += 64) diag[w][i] = 0.f;
  for (int i = lane; i < a.nbucket; i += 64) bsum[w][i] = 0.f;

  int p0 = 0, p1 = 0;
  if (len > qb * BQ) {
    p0 = ld_meta(a.row_ptr + qb);
    p1 = ld_meta(a.row_ptr + qb + 1);
    trim(a.col_idx, p0, p1, qb + a.omin, min(qb + a.omax, (len + BQ - 1) / BQ - 1), lane);
    take_part(wk, p0, p1);
  }
  f32x16 dq[2];
#pragma unroll
  for (int e = 0; e < 16; ++e) dq[0][e] = dq[1][e] = 0.f;

  // delta = rowsum(dO o O); rows past the length read zeros.
  bf16x8 qf[4], gf[4];
  float delta = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    qf[i] = frag_b(rq, row, qrb, i, lane);
    gf[i] = frag_b(rg, row, grb, i, lane);
    const bf16x8 of = frag_b(ro, row, orb, i, lane);
#pragma unroll
    for (int e = 0; e < 8; ++e) delta += (float)of[e] * (float)gf[i][e];
  }
  delta = add_xor32(delta);
  const bool live = row < len, store = row < a.Sq;
  if (lane < 32 && store && wk.part == 0) a.delta[(int64_t)bh * a.Sq + row] = delta;
  // Rows without a token or without a key: probability 0 everywhere.
  const float lse = live ? a.lse_in[(int64_t)bh * a.Sq + row] : -INFINITY;
  const float lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;

  if (p0 < p1) {
    RowCopy cp;
    cp.init(lane, w);
    auto block_bias = [&](int col) __attribute__((always_inline)) {
      const int d = col - qb;
      return BlockBias{ld_meta(a.info + d + a.nb - 1), ld_meta(bias + d * BQ + a.seq)};
    };
    auto issue_k = [&](int col) __attribute__((always_inline)) {
      cp.issue(rk, (uint32_t)(col * BQ) * krb, krb, ks);
      copy_window(rb, ((col - qb) * BQ + a.seq - BQ) * 4, win, lane, w);
    };
    int ccur = ld_meta(a.col_idx + p0);
    cp.issue(rv, (uint32_t)(ccur * BQ) * vrb, vrb, vs);
    issue_k(ccur);
    BlockBias bb = block_bias(ccur);
    int cn = ld_meta(a.col_idx + min(p0 + 1, p1 - 1));
    const int unit = 64 + (lane >> 5) * 4 - (w * 32 + (lane & 31));
    // First diagonal unit of this lane: key - query + 64 at key 0 of its half,
    // query its row's first less lane % 16 (see the shifts below).
    float *const dg = &diag[w][(lane >> 4) * DPITCH + 64 + (lane >> 5) * 4 - (lane & 15) -
                               16 * ((lane >> 4) & 1) - 32 * w];

    int ucur = -1;       // bucket that usum belongs to
    float usum = 0.f;
    auto flush = [&]() __attribute__((always_inline)) {
      if (ucur >= 0) {
        seg_scan(usum, 0);
        if (lane == 63) bsum[w][ucur] += usum;
      }
      usum = 0.f;
    };

    Scores s;
    f32x16 dp;
    for (int p = p0; p < p1; ++p) {
      wait_vm<0>();  // this wave's copies of the block have landed,
      barrier();     // every wave's have
      const bool mixed = bb.info >= kRelposMixed;
      // Order by bucket of a mixed block's distances, two per lane.
      const uint32_t ord = mixed ? a.order[(int64_t)(bb.info - kRelposMixed) * 64 + lane] : 0u;
      if (!mixed && bb.info != ucur) {
        flush();
        ucur = bb.info;
      }
      const BlockBias bn = block_bias(cn);
      const float cm = mixed ? 1.f : c, ca = (mixed ? 0.f : bb.mid) - lse2;
      const int left = len - ccur * BQ;  // keys from the block's first on
      float dsum[5] = {};
      auto scores = [&](int kt) __attribute__((always_inline)) {
        f32x16 acc;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = dp[e] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc = MFMA32(frag_r(ks, kt * 32, i, lane), qf[i], acc);
          dp = MFMA32(frag_r(vs, kt * 32, i, lane), gf[i], dp);
        }
        s.take(acc);
      };
      auto grads = [&](auto kt_) __attribute__((always_inline)) {
        constexpr int kt = decltype(kt_)::value;
        if (mixed) s.add_window(c, win + (unit + kt * 32) * 16);
        if (left < BQ) s.cut(left - (lane >> 5) * 4 - kt * 32);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float pr = fast_exp2(__builtin_fmaf(s.v[e], cm, ca));
          s.v[e] = pr * (dp[e] - delta);  // dS^T
        }
        if (mixed) {
          // Key 16 a + j + 4 (l / 32) of this half, query lane x of its 16:
          // diagonal 16 a - x from lane x + j, 16 (a + 1) - x from x + j - 16.
          sfor<16>([&](auto ee) __attribute__((always_inline)) {
            constexpr int e = decltype(ee)::value;
            constexpr int j = ((e >> 2) & 1) * 8 + (e & 3), m = kt * 2 + (e >> 3);
            if constexpr (j == 0) {
              dsum[m] += s.v[e];
            } else {
              dsum[m] += dpp0<kRowShl + j>(s.v[e]);
              dsum[m + 1] += dpp0<kRowShr + 16 - j>(s.v[e]);
            }
          });
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) usum += s.v[e];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x8 d = s.pack(j);
#pragma unroll
          for (int dt = 0; dt < 2; ++dt)
            dq[dt] = MFMA32(frag_t(ks, kt * 32 + j * 16, dt * 32, lane), d, dq[dt]);
        }
      };
      scores(0);
      grads(std::integral_constant<int, 0>{});
      scores(1);
      wait_vm<0>();
      barrier();  // every wave has read V
      cp.issue(rv, (uint32_t)(cn * BQ) * vrb, vrb, vs);
      grads(std::integral_constant<int, 1>{});
      if (mixed) {
#pragma unroll
        for (int m = 0; m < 5; ++m) dg[16 * m] = dsum[m];
        const int o0 = ord & 127, o1 = (ord >> 8) & 127, i0 = (ord >> 16) & 255, i1 = ord >> 24;
        const float *dd = diag[w];
        float v0 = 0.f, v1 = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          v0 += dd[r * DPITCH + o0];
          v1 += dd[r * DPITCH + o1];
        }
        // Two sorted distances per lane.  A lane whose two lie in different
        // buckets closes the first one's segment with its v0.
        float sum = i0 == i1 ? v0 + v1 : v1;
        seg_scan(sum, i1);
        // Sum of the lanes before, if their last bucket is this lane's first.
        const int pid = dppi<0x138, 0xf>(-1, i1);  // wave_shr:1
        const float prev = __uint_as_float(dppi<0x138, 0xf>(0, (int)__float_as_uint(sum)));
        const int nid = dppi<0x130, 0xf>(-1, i0);  // wave_shl:1
        if (i0 != i1) bsum[w][i0] += v0 + (pid == i0 ? prev : 0.f);
        if (nid != i1) bsum[w][i1] += sum;
      }
      ccur = cn;
      bb = bn;
      cn = ld_meta(a.col_idx + min(p + 2, p1 - 1));
      wait_vm<4>();
      barrier();  // every wave has read K and the window
      issue_k(ccur);
    }
    flush();
    wait_vm<0>();  // no copy outlives the workgroup
  }
  const RelposArgs &z = late_args();
  if (wk.slot >= 0) put_acc(z.slots + (int64_t)wk.slot * kAccFloats, dq, w, lane);
  else
    put_row((bf16_t *)z.dQ.p + b * z.dQ.seq + h * z.dQ.head + (int64_t)row * z.dQ.tok, dq, z.scale, live,
            store, lane);
  __syncthreads();
  float *P = z.partials + (int64_t)L * z.nbucket;
  for (int i = threadIdx.x; i < z.nbucket; i += 128) P[i] = bsum[0][i] + bsum[1][i];
}

// ---------------------------------------------------------------------------
// Backward, pass 2: dK and dV (a key block of one key/value head; its G query
// heads and their kept query blocks one after another)
// ---------------------------------------------------------------------------
// dtable[h][c]: the dQ launch's partials, one row of nbucket sums per workgroup,
// added over sequences, block rows and parts in a fixed order: a head's rows are
// tab_nl consecutive ones per sequence among the long blocks', then tab_ns among the
// others'.  A workgroup takes kRelposTabCols buckets of a head, eight threads a bucket.
__device__ __forceinline__ void table_sums(const RelposArgs &a, int t, float *red) {
  constexpr int C = kRelposTabCols, PARTS = 128 / C;
  const int nb = a.nbucket, nc = (nb + C - 1) / C, h = t / nc;
  if (h >= a.H) return;
  const int cc = threadIdx.x % C, part = threadIdx.x / C, c = t % nc * C + cc;
  float s = 0.f;
  auto add = [&](const float *p, int n) {  // n rows per sequence
    const int total = a.B * n;
#pragma unroll 8
    for (int i = part; i < total; i += PARTS) {
      const int b = i / n, r = i - b * n;
      s += p[(((int64_t)b * a.H + h) * n + r) * nb];
    }
  };
  if (c < nb) {
    add(a.partials + c, a.tab_nl);
    add(a.partials + (int64_t)a.B * a.H * a.tab_nl * nb + c, a.tab_ns);
  }
  red[threadIdx.x] = s;
  __syncthreads();
  if (part || c >= nb) return;
#pragma unroll
  for (int p = 1; p < PARTS; ++p) s += red[p * C + cc];
  a.dtable[(int64_t)h * nb + c] = s;
}

__global__ __launch_bounds__(128, 2) void relpos_bwd_dkv_kernel(RelposArgs a) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  uint8_t *const qs0 = stage_buf<0, TILE>(), *const gs0 = stage_buf<1, TILE>();
  uint8_t *const qs1 = stage_buf<2, TILE>(), *const gs1 = stage_buf<3, TILE>();
  uint8_t *const w0 = stage_buf<4, WIN>(), *const w1 = stage_buf<5, WIN>();
  // Row terms of the 64 queries: lse (log2 units, less the bias of a block of one
  // bucket), then -delta.
  __shared__ __attribute__((aligned(16))) float rt0[2 * BQ], rt1[2 * BQ];

  // The first workgroups add up the table gradient, beside the others' work (in a
  // launch of its own: 4 x 16 x 1511 both passes 65.3 -> 62.5 us without it).
  if ((int)blockIdx.x < a.tab_wg) {
    table_sums(a, blockIdx.x, rt0);
    return;
  }
  const Work wk = find_work(a, xcd_remap(blockIdx.x - a.tab_wg, gridDim.x - a.tab_wg));
  const int kb = wk.blk, b = wk.bh / a.Hkv, hk = wk.bh % a.Hkv;
  const int len = seq_len(a, b);
  const int key = kb * BQ + w * 32 + (lane & 31);

  const bf16_t *K = (const bf16_t *)a.K.p + b * a.K.seq + hk * a.K.head;
  const bf16_t *V = (const bf16_t *)a.V.p + b * a.V.seq + hk * a.V.head;
  const uint32_t qrb = (uint32_t)(a.Q.tok * 2), krb = (uint32_t)(a.K.tok * 2), vrb = (uint32_t)(a.V.tok * 2);
  const uint32_t grb = (uint32_t)(a.dO.tok * 2);
  const float c = a.scale * kLog2e, inv_c = 1.f / c;

  int p0 = 0, p1 = 0;
  if (len > kb * BQ) {
    p0 = ld_meta(a.col_ptr + kb);
    p1 = ld_meta(a.col_ptr + kb + 1);
    trim(a.row_idx, p0, p1, kb - a.omax, min(kb - a.omin, (len + BQ - 1) / BQ - 1), lane);
  }
  f32x16 dk[2], dv[2];
#pragma unroll
  for (int e = 0; e < 16; ++e) dk[0][e] = dk[1][e] = dv[0][e] = dv[1][e] = 0.f;

  // This part of the column's items: (query head of the group, position).
  int i0 = 0, i1 = (p1 - p0) * a.G;
  take_part(wk, i0, i1);
  if (i0 < i1) {
    const rsrc_t rk = rows_rsrc(K, len, krb), rv = rows_rsrc(V, len, vrb);
    RowCopy cp;
    cp.init(lane, w);
    bf16x8 kf[4], vf[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      kf[i] = frag_b(rk, key, krb, i, lane);
      vf[i] = frag_b(rv, key, vrb, i, lane);
    }
    struct Item {
      int g, p;
    };
    auto next = [&](Item it) __attribute__((always_inline)) {
      return it.p + 1 < p1 ? Item{it.g, it.p + 1} : Item{it.g + 1, p0};
    };
    float rt = 0.f;  // row term of the block in flight (wave 0: lse, wave 1: delta)
    BlockBias bf{0, 0.f};  // the bias of the block in flight
    auto issue = [&](Item it, uint8_t *qt, uint8_t *gt, uint8_t *win) __attribute__((always_inline)) {
      const int h = hk * a.G + it.g, qb = ld_meta(a.row_idx + it.p);
      const bf16_t *Q = (const bf16_t *)a.Q.p + b * a.Q.seq + h * a.Q.head;
      const bf16_t *dO = (const bf16_t *)a.dO.p + b * a.dO.seq + h * a.dO.head;
      cp.issue(rows_rsrc(Q, len, qrb), (uint32_t)(qb * BQ) * qrb, qrb, qt);
      cp.issue(rows_rsrc(dO, len, grb), (uint32_t)(qb * BQ) * grb, grb, gt);
      // The head's bias by descending distance: by query - key.
      const float *rev = a.bias + (int64_t)h * a.bias_ld + 2 * (int64_t)a.seq;
      copy_window(make_rsrc(rev, (int64_t)a.seq * 8), ((qb - kb) * BQ + a.seq - BQ) * 4, win, lane, w);
      bf = BlockBias{ld_meta(a.info + (kb - qb) + a.nb - 1), ld_meta(rev + (qb - kb) * BQ + a.seq)};
      const int q = qb * BQ + lane;
      const float *src = (w == 0 ? a.lse_in : a.delta) + (int64_t)(b * a.H + h) * a.Sq;
      rt = q < len ? src[q] : (w == 0 ? -INFINITY : 0.f);
    };
    const int unit = 64 + (lane >> 5) * 4 - (w * 32 + (lane & 31));
    auto step = [&](bool more, Item nx, uint8_t *qt, uint8_t *gt, const uint8_t *wc, float (&rc)[2 * BQ],
                    uint8_t *qn, uint8_t *gn, uint8_t *wn) __attribute__((always_inline)) {
      wait_vm<0>();
      // The stage's row terms were last read two blocks ago, before the
      // previous barrier.
      const bool mixed = bf.info >= kRelposMixed;
      rc[w * BQ + lane] = w ? -rt : rt == -INFINITY ? INFINITY : rt * kLog2e - (mixed ? 0.f : bf.mid);
      wait_vm<0>();
      barrier();
      if (more) issue(nx, qn, gn, wn);
      const float *lsep = &rc[(lane >> 5) * 4], *delp = lsep + BQ;
#pragma unroll
      for (int qq = 0; qq < 2; ++qq) {
        // S[query][key], dP[query][key] of 32 queries x this wave's 32 keys; dP
        // starts at -delta.
        f32x16 s, dp;
        // A mixed block's scores start at their bias, in units of the unscaled
        // score: what follows is the same for every block.
        if (mixed) {
#pragma unroll
          for (int e4 = 0; e4 < 4; ++e4) {
            const f32x4 bv = *(const f32x4 *)(wc + (unit + qq * 32 + e4 * 8) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[e4 * 4 + j] = bv[j] * inv_c;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e] = 0.f;
        }
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const f32x4 de = *(const f32x4 *)(delp + qq * 32 + e4 * 8);
#pragma unroll
          for (int j = 0; j < 4; ++j) dp[e4 * 4 + j] = de[j];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s = MFMA32(frag_r(qt, qq * 32, i, lane), kf[i], s);
          dp = MFMA32(frag_r(gt, qq * 32, i, lane), vf[i], dp);
        }
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const f32x4 ls = *(const f32x4 *)(lsep + qq * 32 + e4 * 8);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int e = e4 * 4 + j;
            const float pr = fast_exp2(__builtin_fmaf(s[e], c, -ls[j]));
            s[e] = pr;
            dp[e] = pr * dp[e];  // dS
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x8 pb = pack_k(s, j), sb = pack_k(dp, j);
#pragma unroll
          for (int dt = 0; dt < 2; ++dt) {
            dv[dt] = MFMA32(frag_t(gt, qq * 32 + j * 16, dt * 32, lane), pb, dv[dt]);
            dk[dt] = MFMA32(frag_t(qt, qq * 32 + j * 16, dt * 32, lane), sb, dk[dt]);
          }
        }
      }
    };
    Item it{i0 / (p1 - p0), p0 + i0 % (p1 - p0)};
    issue(it, qs0, gs0, w0);
    for (int i = i0; i < i1; i += 2) {
      it = next(it);
      step(i + 1 < i1, it, qs0, gs0, w0, rt0, qs1, gs1, w1);
      if (i + 1 < i1) {
        it = next(it);
        step(i + 2 < i1, it, qs1, gs1, w1, rt1, qs0, gs0, w0);
      }
    }
  }
  if (wk.slot >= 0) {
    float *slot = a.slots + (int64_t)wk.slot * (2 * kAccFloats);
    put_acc(slot, dk, w, lane);
    put_acc(slot + kAccFloats, dv, w, lane);
    return;
  }
  const bool live = key < len, store = key < a.Skv;
  put_row((bf16_t *)a.dK.p + b * a.dK.seq + hk * a.dK.head + (int64_t)key * a.dK.tok, dk, a.scale, live,
          store, lane);
  put_row((bf16_t *)a.dV.p + b * a.dV.seq + hk * a.dV.head + (int64_t)key * a.dV.tok, dv, 1.f, live, store,
          lane);
}

// Sums of the parts' dQ (KV false) or dK and dV, in part order: four workgroups
// per block and tensor, eight accumulator registers each.
template <bool KV>
__global__ __launch_bounds__(128) void relpos_bwd_join_kernel(RelposArgs a) {
  constexpr int GROUPS = KV ? 8 : 4, SLOT = (KV ? 2 : 1) * kAccFloats;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const Work wk = find_join(a, blockIdx.x / GROUPS);
  const int kv = blockIdx.x % GROUPS / 4, g = blockIdx.x % 4;
  const int heads = KV ? a.Hkv : a.H, b = wk.bh / heads, h = wk.bh % heads;
  const int row = wk.blk * BQ + w * 32 + (lane & 31);
  const bool live = row < seq_len(a, b), store = row < a.Sq;
  const float *slot = a.slots + (int64_t)wk.slot * SLOT + kv * kAccFloats + g * 1024 + (w * 64 + lane) * 4;
  f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll 4
  for (int p = 0; p < wk.parts; ++p) {
    lo += *(const f32x4 *)(slot + (int64_t)p * SLOT);
    hi += *(const f32x4 *)(slot + (int64_t)p * SLOT + 512);
  }
  const RowViewOut &t = !KV ? a.dQ : kv == 0 ? a.dK : a.dV;
  const float scale = KV && kv == 1 ? 1.f : a.scale;
  bf16_t *dst = (bf16_t *)t.p + b * t.seq + h * t.head + (int64_t)row * t.tok;
  put_eight(dst, g, lo, hi, scale, live, store, lane);
}

// ---------------------------------------------------------------------------
// The bias by distance
// ---------------------------------------------------------------------------
// out[h][d + seq] = log2(e) table[h][bucket(d)], -inf where the bucket is -1; then
// the same by descending distance, out[h][2 seq + f] = out[h][2 seq - f] (distance
// seq - f).  Entry 0 of either (distance -seq, seq) is never used: -inf.
__global__ __launch_bounds__(256) void relpos_bias_kernel(RelposBiasArgs a) {
  const int e = blockIdx.x * 256 + threadIdx.x, h = blockIdx.y;
  if (e >= 2 * a.seq) return;
  const int id = a.bucket[e];
  const float v = id < 0 ? -INFINITY : a.table[(int64_t)h * a.nbucket + id] * kLog2e;
  float *o = a.out + (int64_t)h * 4 * a.seq;
  o[e] = v;
  o[2 * (int64_t)a.seq + (e ? 2 * a.seq - e : 0)] = v;
}

}  // namespace

namespace {
int64_t parts_grid(const RelposArgs &a) {
  return (int64_t)a.nbh * ((int64_t)a.nlong * a.plong + (int64_t)(a.ntile - a.nlong) * a.pshort);
}
int64_t join_grid(const RelposArgs &a) {
  return (int64_t)a.nbh * ((a.plong > 1 ? a.nlong : 0) + (a.pshort > 1 ? a.ntile - a.nlong : 0));
}
template <typename F>
hipError_t go(F kernel, int64_t grid, const RelposArgs &a, hipStream_t s) {
  if (grid <= 0 || grid > 0x7fffffff) return hipErrorInvalidValue;
  launch_kernel(kernel, dim3((unsigned)grid), dim3(128), s, a);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_relpos_fwd(const RelposArgs &a, hipStream_t s) {
  return go(relpos_fwd_kernel, parts_grid(a), a, s);
}
hipError_t launch_relpos_fwd_join(const RelposArgs &a, hipStream_t s) {
  return go(relpos_fwd_join_kernel, 4 * join_grid(a), a, s);
}
hipError_t launch_relpos_decode(const RelposArgs &a, hipStream_t s) {
  const int64_t units = (int64_t)a.nbh * a.pshort, grid = (units + 3) / 4;
  if (units <= 0 || units > 0x7fffffff || a.G > kRelposDecodeRows) return hipErrorInvalidValue;
  launch_kernel(relpos_decode_kernel, dim3((unsigned)grid), dim3(256), s, a);
  return hipGetLastError();
}
hipError_t launch_relpos_decode_join(const RelposArgs &a, hipStream_t s) {
  launch_kernel(relpos_decode_join_kernel, dim3((unsigned)(a.B * a.H)), dim3(256), s, a);
  return hipGetLastError();
}
hipError_t launch_relpos_bwd_dq(const RelposArgs &a, hipStream_t s) {
  return go(relpos_bwd_dq_kernel, parts_grid(a), a, s);
}
hipError_t launch_relpos_bwd_dkv(const RelposArgs &a, hipStream_t s) {
  return go(relpos_bwd_dkv_kernel, a.tab_wg + parts_grid(a), a, s);
}
hipError_t launch_relpos_bwd_join(bool kv, const RelposArgs &a, hipStream_t s) {
  return kv ? go(relpos_bwd_join_kernel<true>, 8 * join_grid(a), a, s)
            : go(relpos_bwd_join_kernel<false>, 4 * join_grid(a), a, s);
}

hipError_t launch_relpos_bias(const RelposBiasArgs &a, int H, hipStream_t s) {
  launch_kernel(relpos_bias_kernel, dim3((unsigned)((2 * (int64_t)a.seq + 255) / 256), (unsigned)H),
                dim3(256), s, a);
  return hipGetLastError();
}

}  // namespace pf
