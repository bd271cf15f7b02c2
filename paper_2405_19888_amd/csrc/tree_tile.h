// The tree-decode query tile on MFMA (gfx950): up to 128 (fp32 caches: 64) columns
// against ranges of paged key sequences.
//
// A column is one (drafted row, query head) pair; the columns of a tile read the same
// cache head, so with grouped queries a key fetched once serves G heads of every row.
// Per 16-token block
//   S^T  = K Q^T    (tokens x columns)      v_mfma_f32_16x16x32_{f16,bf16} / 16x16x4f32
//   O^T += V^T P^T  (D x columns)
// with an online softmax in fp32 whose reference moves only when a column's logits
// exceed it by more than 2^8 (as the prefill tile's), so most blocks need no
// cross-lane maximum.  Probabilities are rounded to the cache's type for the product
// (16-bit caches: the matrix cores take both factors in one type, and high and low halves
// would double the second product), and the output is divided by the sum of the rounded
// ones, so a dominant weight's rounding cancels; the lse keeps the sum of the unrounded ones.
// Against 64 bits the output is off by 1.3 to 1.4 times its own rounding (fp16 2.9e-4 for
// 2.1e-4, bf16 2.3e-3 for 1.7e-3 of its norm).
//
// Keys and values pass through LDS in 16 KiB stages (8 of each: 32 tokens of 128
// 16-bit elements) by direct-to-LDS loads into a ring of three, two stages ahead.
// Column sets of 16 go round the waves (set w + 4 c to wave w), so a tile of up to 64
// columns gives each wave one set.
//
// Bound by the matrix cores and the softmax beside them: three workgroups of a CU take
// 1.28 us for a 32-token stage of 128 columns each (1.25 PFLOP/s; a large bf16 product
// reaches 1.12), one alone 0.74.  What a piece costs beside its stages, 17 us (queries
// and masks after the row lists, the first stages, the masked ones, the partial results,
// instructions fetched for the first time), bounds the short ones.  The 16-bit instances for
// heads of 128 keep three waves a SIMD by spilling: k_tree_partials 31 vector and 147 scalar
// registers, k_tree_decode 2 and 49, stored and loaded outside the stage loops, once a piece.
//
// Mask: drafted tokens follow the cached ones, from own position `base` on.  The
// bits of the tokens a column sees are kept per 32-token word counted from base
// rounded down to 32 (bits below base set, bits past the last token clear), so a
// pair of blocks takes one word per column and needs no other test.
//
// A drafted token's value that is no finite number must not reach the columns that
// do not see it, though its probability there is 0 (0 * NaN).  Stages that hold
// drafted tokens are scanned: such elements are cleared in LDS, and added afterwards,
// element by element, to the columns that see them.
#pragma once

#include <cfloat>

#include "prefill_tile.h"
#include "tree_args.h"

namespace parrot {

namespace tree_detail {

using namespace prefix_detail;

template <int DT> constexpr int kSets = DT == kF32 ? kTreeSets32 : kTreeSets16;
template <int DT> constexpr int kCols = 64 * kSets<DT>;
constexpr int kRing3 = 3;
constexpr int kMaskWords = (kTreeRows + 31 + 31) / 32;      // a request's rows from any alignment

template <int DT>
struct Lds {
  char ring[kRing3][kStageBytes];
  unsigned mask[kMaskWords][kCols<DT>];   // visible drafted tokens of each column
  int tbl[kTreeSpan];                     // block ids of the current span, clamped
  int rows[kCols<DT> + 2];                // q rows that hold the tile's columns
  int held[kCols<DT> + 1];                // prefix tiles: their numbers among rows with prefixes
  unsigned bad[kRing3][4];                // tokens of a stage with cleared values, a bit each
};
// three workgroups of a CU share its 160 KiB, handed out in pieces of 1280 bytes
static_assert(sizeof(Lds<kF16>) <= 42 * 1280, "three workgroups per CU");

// Swizzle of a stage's rows (see the two tiles this follows).
template <int DT, int D>
PARROT_DEV int swizzle(int t) {
  if constexpr (DT == kF32) return swz(t);
  else return swz_wide<D * 2 / 16>(t);
}

PARROT_DEV bool any_nonfinite16(const u32x4& v, unsigned expo) {   // expo: the type's exponent mask
  bool bad = false;
  const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad = bad || (w[i] & expo) == expo || ((w[i] >> 16) & expo) == expo;
  return bad;
}
// the 16 bytes with every element that is no finite number cleared; true if any was
template <int DT>
PARROT_DEV bool clear_nonfinite(u32x4& v) {
  unsigned w[4] = {v.x, v.y, v.z, v.w};
  bool bad = false;
  if constexpr (DT == kF32) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((w[i] & 0x7F800000u) == 0x7F800000u) { w[i] = 0u; bad = true; }
  } else {
    constexpr unsigned expo = DT == kF16 ? 0x7C00u : 0x7F80u;
    if (!any_nonfinite16(v, expo)) return false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((w[i] & expo) == expo) w[i] &= 0xFFFF0000u;
      if (((w[i] >> 16) & expo) == expo) w[i] &= 0x0000FFFFu;
    }
    bad = true;
  }
  v = u32x4{w[0], w[1], w[2], w[3]};
  return bad;
}

template <int DT>
PARROT_DEV float elem_at(const char* p) {
  if constexpr (DT == kF32) return *reinterpret_cast<const float*>(p);
  else if constexpr (DT == kF16) return (float)*reinterpret_cast<const _Float16*>(p);
  else return __uint_as_float((unsigned)*reinterpret_cast<const unsigned short*>(p) << 16);
}

}  // namespace tree_detail

// One key range of a tile.
struct TreeRange {
  const void* pk; const void* pv;   // pools
  const int* tbl;                   // block table row of the sequence
  int npool;                        // blocks in the pools
  int t0, t1;                       // tokens [t0, t1), t0 a multiple of 32
  int mask0;                        // first token of mask word 0 (a multiple of 32); tokens
                                    // from there on go by the mask.  t1 or more: no mask
  int base, end;                    // masked ranges: the drafted tokens are [base, end)
  bool once = false;                // tiles: no other tile reads these keys
};

// A wave's columns: NS sets of 16 with their queries, softmax statistics and output, in
// registers.
template <int DT, int D, int NS>
struct TreeState {
  static constexpr int EB = Elem<DT>::kBytes;
  static constexpr int ROW_B = D * EB;
  static constexpr int GRAN = ROW_B / 16;                    // 16-byte granules per row
  static constexpr int BLK_B = kBlock * ROW_B;               // one block of one head
  static constexpr int DT16 = D / 16;
  static constexpr int KS = DT == kF32 ? D / 4 : D / 32;     // MFMA k-steps over D
  static constexpr float kLazy = 8.f;

  int lane, H, h;
  int set0, stride;                   // set c is set set0 + stride c of the columns
  float scale, inv_scale;
  unsigned qsign;
  u32x4 qf[NS][DT == kF32 ? 1 : KS];
  float qs[NS][DT == kF32 ? KS : 1];
  float mref[NS], thr[NS], lsum[NS], lsr[NS];
  f32x4 o[NS][DT16];

  PARROT_DEV TreeState(int heads, int head, float scale_log2, int first, int step)
      : H(heads), h(head), set0(first), stride(step) {
    lane = threadIdx.x & 63;
    // a negative scale flips the sign of q (exact); a zero scale is taken as 1e-30
    scale = fmaxf(fabsf(scale_log2), 1e-30f);
    inv_scale = 1.f / scale;
    qsign = scale_log2 < 0.f ? (DT == kF32 ? 0x80000000u : 0x80008000u) : 0u;
  }
  // the column that this lane holds in set c
  PARROT_DEV int column(int c) const { return (set0 + stride * c) * 16 + (lane & 15); }

  // Loads the queries of `ncols` columns; qrow(col) is the column's row of q in units
  // of heads (row * HQ + query head).  Lane group g of 16 holds, of k-step ks, the
  // elements 32 ks + 8 g .. + 7 (16-bit), or 4 ks + g (fp32; CHUNKS: 4 g + ks % 4 of
  // 16-element piece ks / 4, as keys come from 16-byte loads).
  template <bool CHUNKS, class F>
  PARROT_DEV void load_queries(const void* q, int ncols, F qrow) {
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      const int col = column(c);
      const bool ok = col < ncols;
      const char* src = (const char*)q + (size_t)(ok ? qrow(col) : 0) * ROW_B;
      if constexpr (DT == kF32) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int e = CHUNKS ? 16 * (ks >> 2) + 4 * (lane >> 4) + (ks & 3) : 4 * ks + (lane >> 4);
          qs[c][ks] = ok ? reinterpret_cast<const float*>(src)[e] : 0.f;
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          qf[c][ks] = ok ? ld16(src + (32 * ks + 8 * (lane >> 4)) * 2) : u32x4{0u, 0u, 0u, 0u};
        }
      }
      mref[c] = -FLT_MAX; thr[c] = -INFINITY; lsum[c] = 0.f; lsr[c] = 0.f;
#pragma unroll
      for (int i = 0; i < DT16; ++i) o[c][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (qsign) {                        // (a rare branch: it waits for the loads)
#pragma unroll
      for (int c = 0; c < NS; ++c)
        if constexpr (DT == kF32) {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) qs[c][ks] = -qs[c][ks];
        } else {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) qf[c][ks] ^= u32x4{qsign, qsign, qsign, qsign};
        }
    }
  }

  // NX logits a lane: x[i] is token tok0 + 16 (i / 4) + 4 (lane / 16) + i % 4.  mask: those whose
  // bit of `vis` (from tok0 on) is clear become -inf.  softmax: x becomes the
  // probabilities, set c's state moves on.
  template <int NX>
  PARROT_DEV void mask(float* x, unsigned vis) const {
    const unsigned mine = vis >> (4 * (lane >> 4));
#pragma unroll
    for (int i = 0; i < NX; ++i) x[i] = (mine >> ((i >> 2) * 16 + (i & 3))) & 1u ? x[i] : -INFINITY;
  }
  template <int NX>
  PARROT_DEV void softmax(float* x, int c) {
    // (grouped as v_max3 takes them)
    float lm = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    if constexpr (NX == 8)
      lm = fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), fmaxf(fmaxf(x[3], x[4]), x[5])), fmaxf(x[6], x[7]));
    if (__builtin_amdgcn_ballot_w64(lm > thr[c]) != 0) {
      const float mn = fmaxf(mref[c], max_xor32(max_xor16(lm)) * scale);
      const float alpha = fast_exp2(mref[c] - mn);
      lsum[c] *= alpha;
      lsr[c] *= alpha;
#pragma unroll
      for (int i = 0; i < DT16; ++i) o[c][i] *= alpha;
      mref[c] = mn;
      thr[c] = (mn + kLazy) * inv_scale;
    }
#pragma unroll
    for (int i = 0; i < NX; ++i) x[i] = fast_exp2(__builtin_fmaf(x[i], scale, -mref[c]));
    if constexpr (NX == 8) lsum[c] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    else lsum[c] += (x[0] + x[1]) + (x[2] + x[3]);
  }

  // Adds the cleared elements of the values (see the head of this file) of the tokens in
  // `bad` to set c: p are the lane's probabilities, vis its column's bits, value_row(t)
  // the memory of token t's value.
  template <int NX, class F>
  PARROT_DEV void add_cleared(const float* p, int c, unsigned vis, unsigned bad, F value_row) {
    while (bad) {                                            // wave-uniform
      const int t = __ffs((int)bad) - 1;
      bad &= bad - 1;
      float mine = 0.f;                                      // held by lane group (t % 16) / 4
#pragma unroll
      for (int i = 0; i < NX; ++i)
        if (i == (t >> 4) * 4 + (t & 3)) mine = p[i];
      const float pt = __shfl(mine, (lane & 15) + 16 * ((t & 15) >> 2));
      const char* row = value_row(t);
#pragma unroll
      for (int dt = 0; dt < DT16; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = tree_detail::elem_at<DT>(row + (dt * 16 + 4 * (lane >> 4) + i) * EB);
          if (!(fabsf(v) <= FLT_MAX) && ((vis >> t) & 1u)) o[c][dt][i] = __builtin_fmaf(pt, v, o[c][dt][i]);
        }
    }
  }

  // The columns' result: f(c, col, weight sum for the output, base-2 lse, weight sum)
  // per set; the lane holds elements dt * 16 + 4 (lane / 16) .. + 3 of its column.
  template <class F>
  PARROT_DEV void finish(F f) {
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      const float lt = sum_xor32(sum_xor16(lsum[c]));
      const float lw = DT == kF32 ? lt : sum_xor32(sum_xor16(lsr[c]));
      f(c, column(c), lw, mref[c] + fast_log2(lt), lt);
    }
  }
};

// One wave's part of a tile.  Waves of one workgroup may run parts of different NS side
// by side: every part makes the same loads and barriers.
template <int DT, int D, int NS>
struct TreeTile : TreeState<DT, D, NS> {
  using Base = TreeState<DT, D, NS>;
  using Base::lane; using Base::H; using Base::h; using Base::qf; using Base::qs; using Base::o; using Base::lsr;
  using Base::column;
  static constexpr int ROW_B = Base::ROW_B, GRAN = Base::GRAN, BLK_B = Base::BLK_B, DT16 = Base::DT16, KS = Base::KS;
  static constexpr int STAGE_BLK = prefix_detail::kTensorStage / BLK_B;
  static constexpr int PER_WAVE = prefix_detail::kStageChunks / 4;
  using L = tree_detail::Lds<DT>;

  L& lds;
  int wave;
  bool act;                           // wave-uniform: the wave has columns
  // 16-bit caches: LDS byte addresses of this lane's K fragment (k-step ks) and V^T
  // fragment (d tile dt) in block 0 of ring buffer 0; buffers and blocks add constants.
  // Opaque, so that one register holds each and a read is one instruction.
  unsigned ka[DT == kF32 ? 1 : KS], va[DT == kF32 ? 1 : DT16];

  PARROT_DEV TreeTile(L& l, int heads, int head, float scale_log2, int ncols)
      : Base(heads, head, scale_log2, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), 4), lds(l) {
    wave = this->set0;
    act = wave * 16 < ncols;
    if constexpr (DT != kF32) {
      const unsigned base = lds_addr(&lds.ring[0][0]);
      const int krow = lane & 15, vrow = 4 * (lane >> 4) + ((lane & 15) >> 2);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        ka[ks] = base + krow * ROW_B + (((4 * ks + (lane >> 4)) ^ tree_detail::swizzle<DT, D>(krow)) << 4);
        asm volatile("" : "+v"(ka[ks]));
      }
#pragma unroll
      for (int dt = 0; dt < DT16; ++dt) {
        va[dt] = base + prefix_detail::kTensorStage + vrow * ROW_B + 8 * (lane & 1) +
                 (((2 * dt + ((lane & 3) >> 1)) ^ tree_detail::swizzle<DT, D>(vrow)) << 4);
        asm volatile("" : "+v"(va[dt]));
      }
    }
  }

  // memory of the value of token tok of the range
  PARROT_DEV const char* value_row(const TreeRange& rg, int span0, int tok) const {
    const int blk = lds.tbl[tok / kBlock - span0];
    return (const char*)rg.pv + (((size_t)blk * H + h) * kBlock + tok % kBlock) * ROW_B;
  }

  // S^T of one block for set c; kb: the block's K in LDS
  PARROT_DEV f32x4 scores32(const char* kb, int c) const {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    const int row = lane & 15;
    const char* krow = kb + row * ROW_B + 4 * (lane >> 4);
    // (eight reads, then their products: left alone, the compiler waits for each read where
    // registers are short, and a stage takes 1.4 times as long)
#pragma unroll
    for (int k0 = 0; k0 < KS; k0 += 8) {
      float kv[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        kv[i] = *reinterpret_cast<const float*>(krow + (((k0 + i) ^ tree_detail::swizzle<DT, D>(row)) << 4));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 8; ++i) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[i], qs[c][k0 + i], s, 0, 0, 0);
    }
    return s;
  }

  // One pair of blocks (32 tokens from tok0) of a stage, 16-bit caches; `at` is the byte
  // offset of the pair in the ring (a constant but for masked stages).  K fragments
  // are read ahead of their products and V^T fragments two d tiles per wait; one at a
  // time, the LDS round trips took twice the time of the products.
  template <bool MASKED>
  PARROT_DEV void pair(const TreeRange& rg, int span0, int at, int tok0, unsigned bad) {
    using namespace prefix_detail;
    f32x4 s[NS][2];
#pragma unroll
    for (int c = 0; c < NS; ++c) s[c][0] = s[c][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    {
      u32x4 kf[2][KS];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[b][ks] = lds_read16(ka[ks], at + b * BLK_B);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int c = 0; c < NS; ++c) s[c][b] = Mfma<DT>::qk(kf[b][ks], qf[c][ks], s[c][b]);
    }
    unsigned pw[NS][4];
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = s[c][0][i]; x[4 + i] = s[c][1][i]; }
      unsigned vis = 0xFFFFFFFFu;
      if constexpr (MASKED) {
        if (tok0 >= rg.mask0) vis = lds.mask[(tok0 - rg.mask0) >> 5][column(c)];
        else if (rg.t1 - tok0 < 32) vis = (1u << (rg.t1 - tok0)) - 1u;
        this->template mask<8>(x, vis);
      }
      this->template softmax<8>(x, c);
      if constexpr (MASKED) {
        if (bad) this->template add_cleared<8>(x, c, vis, bad, [&](int t) { return value_row(rg, span0, tok0 + t); });
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pw[c][i] = pack2<DT>(x[2 * i], x[2 * i + 1]);
        lsr[c] = add_pair<DT>(pw[c][i], lsr[c]);
      }
    }
    static_assert(DT16 % 2 == 0, "d tiles are read in pairs");
#pragma unroll
    for (int dt = 0; dt < DT16; dt += 2) {
      unsigned long long v[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        v[u][0] = lds_read_tr<DT>(va[dt + u], at);
        v[u][1] = lds_read_tr<DT>(va[dt + u], at + BLK_B);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < NS; ++c) {
          const unsigned long long b0 = pw[c][0] | ((unsigned long long)pw[c][1] << 32);
          const unsigned long long b1 = pw[c][2] | ((unsigned long long)pw[c][3] << 32);
          o[c][dt + u] = Mfma<DT>::pv2(v[u][0], v[u][1], b0, b1, o[c][dt + u]);
        }
    }
  }

  // One block (16 tokens from tok0) of a stage; fp32 caches.
  template <bool MASKED>
  PARROT_DEV void block32(const TreeRange& rg, int span0, int buf, int bl, int tok0, unsigned bad) {
    const char* kb = lds.ring[buf] + bl * BLK_B;
    const char* vb = kb + prefix_detail::kTensorStage;
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      const f32x4 s = scores32(kb, c);
      float x[4] = {s[0], s[1], s[2], s[3]};
      if constexpr (MASKED) {
        unsigned vis = 0xFFFFu;
        if (tok0 >= rg.mask0) vis = (lds.mask[(tok0 - rg.mask0) >> 5][column(c)] >> (tok0 & 16)) & 0xFFFFu;
        else if (rg.t1 - tok0 < 16) vis = (1u << (rg.t1 - tok0)) - 1u;
        this->template mask<4>(x, vis);
        this->template softmax<4>(x, c);
        if (bad) this->template add_cleared<4>(x, c, vis, bad, [&](int t) { return value_row(rg, span0, tok0 + t); });
      } else {
        this->template softmax<4>(x, c);
      }
      // O^T[d][col] += V^T[d][t] P^T[t][col] with k index kk <-> token 4 kk + kt
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        const int row = 4 * (lane >> 4) + kt;
        const char* vrow = vb + row * ROW_B + 4 * (lane & 3);
        float v[DT16];
#pragma unroll
        for (int dt = 0; dt < DT16; ++dt)
          v[dt] = *reinterpret_cast<const float*>(
              vrow + (((4 * dt + ((lane & 15) >> 2)) ^ tree_detail::swizzle<DT, D>(row)) << 4));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int dt = 0; dt < DT16; ++dt) o[c][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[dt], x[kt], o[c][dt], 0, 0, 0);
      }
    }
  }

  // The range's tokens: every wave of the workgroup calls it, whether it has columns
  // or not (all of them load and synchronise).
  // first() runs once the first block ids are requested.
  template <class F>
  PARROT_DEV void run(const TreeRange& rg, F first) {
    using namespace prefix_detail;
    for (int t = rg.t0; t < rg.t1; t += kTreeSpan * kBlock) {
      const int b0 = t / kBlock;
      const int nb = (min(rg.t1, t + kTreeSpan * kBlock) - t + kBlock - 1) / kBlock;
      const int id = (int)threadIdx.x < nb ? rg.tbl[b0 + threadIdx.x] : 0;
      if (t == rg.t0) first();
      lds_sync();                                            // the LDS of what ran before is free
      if ((int)threadIdx.x < nb) lds.tbl[threadIdx.x] = clampi(id, 0, rg.npool - 1);
      lds_sync();
      span(rg, b0, nb);
    }
  }

  PARROT_DEV void span(const TreeRange& rg, int b0, int nb) {
    using namespace prefix_detail;
    const int tid = threadIdx.x;
    const size_t blk_stride = (size_t)H * BLK_B;
    const int nstages = (nb + STAGE_BLK - 1) / STAGE_BLK, last = nstages - 1;
    // Direct-to-LDS loads: wave w issues the 1 KiB chunks w, w + 4, ... of a stage;
    // lane l fills bytes [16 l, 16 l + 16) of its chunk from the granule that the
    // swizzle puts there.
    int c_bl[PER_WAVE];
    unsigned c_src[PER_WAVE];
    bool c_v[PER_WAVE];
#pragma unroll
    for (int j = 0; j < PER_WAVE; ++j) {
      const int q = wave + j * 4;
      const int off = (q % (kStageChunks / 2)) * 1024 + lane * 16;
      c_v[j] = q >= kStageChunks / 2;
      c_bl[j] = off / BLK_B;
      const int t = (off % BLK_B) / ROW_B, pos = (off % ROW_B) / 16;
      c_src[j] = (unsigned)(h * BLK_B + t * ROW_B + ((pos ^ tree_detail::swizzle<DT, D>(t)) << 4));
    }
    int tb[PER_WAVE];
    auto table = [&](int st) {
#pragma unroll
      for (int j = 0; j < PER_WAVE; ++j) tb[j] = lds.tbl[min(st * STAGE_BLK + c_bl[j], nb - 1)];   // past the end: re-read
    };
    auto issue_as = [&](int buf, auto once_c) {
#pragma unroll
      for (int j = 0; j < PER_WAVE; ++j) {
        const unsigned blk = min((unsigned)__builtin_amdgcn_readfirstlane(tb[j]), (unsigned)(rg.npool - 1));
        const char* base = (const char*)(c_v[j] ? rg.pv : rg.pk) + (size_t)blk * blk_stride;
        const unsigned to = lds_addr(&lds.ring[buf][(wave + j * 4) * 1024]);
        if constexpr (decltype(once_c)::value) lds_dma16_sbase_stream(base, c_src[j], to);
        else lds_dma16_sbase(base, c_src[j], to);
      }
    };
    auto issue = [&](int buf) {
      if (rg.once) issue_as(buf, std::true_type{});
      else issue_as(buf, std::false_type{});
    };
    table(0);
    issue(0);
    table(min(1, last));
    issue(1);
    table(min(2, last));
    // the compiler tracks the query loads but not the direct-to-LDS ones: it waits for
    // the queries here, once, and not inside the loop
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      if constexpr (DT == kF32) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : : "v"(qs[c][ks]));
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : : "v"(qf[c][ks]));
      }
    }
    wait_vmcnt<0>();
    // stages that every column sees whole come first
    const int full = max(0, min(rg.t1, rg.mask0) - b0 * kBlock) / (STAGE_BLK * kBlock);
    const int plain = min(full, nstages);
    // `bufc` carries the ring buffer as a constant: every LDS address of the stage is a
    // lane constant plus an immediate offset
    auto step = [&](int st, auto bufc) {
      constexpr int buf = decltype(bufc)::value;
      wait_vmcnt<PER_WAVE>();            // this stage's loads are the oldest two rounds'
      lds_sync();
      issue((buf + 2) % 3);
      table(min(st + 3, last));
      if (!act) return;
      const int tok_st = (b0 + st * STAGE_BLK) * kBlock;
      if constexpr (DT == kF32) {
#pragma unroll 1
        for (int bl = 0; bl < STAGE_BLK; ++bl) block32<false>(rg, b0, buf, bl, tok_st + bl * kBlock, 0u);
      } else {
#pragma unroll
        for (int bl = 0; bl < STAGE_BLK; bl += 2)
          pair<false>(rg, b0, buf * kStageBytes + bl * BLK_B, tok_st + bl * kBlock, 0u);
      }
    };
    for (int st = 0; st < plain; st += 3) {
      step(st, std::integral_constant<int, 0>{});
      if (st + 1 < plain) step(st + 1, std::integral_constant<int, 1>{});
      if (st + 2 < plain) step(st + 2, std::integral_constant<int, 2>{});
    }
#pragma unroll 1
    for (int st = plain, buf = plain % 3; st < nstages; ++st) {
      wait_vmcnt<PER_WAVE>();
      lds_sync();
      const int tok_st = (b0 + st * STAGE_BLK) * kBlock;
      // rows past the range end are cleared (0 * NaN), and the values of drafted tokens
      // that are no finite numbers, with a bit for their token
      if (tid < 4) lds.bad[buf][tid] = 0u;
      lds_sync();
      const int stop = min(rg.t1, rg.end);
#pragma unroll 1
      for (int i = tid; i < kTensorStage / 16; i += 256) {
        const int row = i / GRAN, tok = tok_st + row;
        if (tok >= rg.base) {
          u32x4* at = reinterpret_cast<u32x4*>(lds.ring[buf] + kTensorStage + i * 16);
          u32x4 v = u32x4{0u, 0u, 0u, 0u};
          bool write = tok >= stop;
          if (!write) {
            v = *at;
            write = tree_detail::clear_nonfinite<DT>(v);
            if (write) atomicOr(&lds.bad[buf][row >> 5], 1u << (row & 31));
          }
          if (write) *at = v;
        }
      }
      lds_sync();
      const int next = buf == 0 ? 2 : buf - 1;               // (st + 2) % 3
      issue(next);
      table(min(st + 3, last));
      if (act) {
#pragma unroll 1
        for (int bl = 0; bl < STAGE_BLK; bl += DT == kF32 ? 1 : 2) {
          const int tok0 = tok_st + bl * kBlock;
          if (tok0 >= rg.t1) break;
          const unsigned bad = __builtin_amdgcn_readfirstlane(lds.bad[buf][bl >> 1]);
          if constexpr (DT == kF32) block32<true>(rg, b0, buf, bl, tok0, bad >> (16 * (bl & 1)) & 0xFFFFu);
          else pair<true>(rg, b0, buf * kStageBytes + bl * BLK_B, tok0, bad);
        }
      }
      buf = buf == 2 ? 0 : buf + 1;
    }
    wait_vmcnt<0>();                     // the re-read stages issued by the last iterations
  }
};

}  // namespace parrot
