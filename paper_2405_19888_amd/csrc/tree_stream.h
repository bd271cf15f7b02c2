// A wave that streams key ranges of one cache head by itself, for up to 32 columns
// (tree_tile.h has the columns' mathematics and the mask).
//
// With few columns a key range is bound by memory, and what the shared tile costs is
// latency: barriers per stage, three of four waves without columns, a set-up per piece
// for a whole workgroup.  Here every wave has a range of its own and nothing to wait
// for but its loads: 8 KiB of K (as the QK operand wants it, 64 contiguous bytes of
// 16 token rows an instruction) and 8 KiB of V (contiguous) come into registers one step
// ahead; V goes through 8 KiB of the wave's own LDS, swizzled, to be read transposed.
// Four waves a CU keep 64 KiB in flight.  Bound by memory (32 heads of 128 in bfloat16):
// 8 requests of 16 rows on 9600 tokens, 1.26 GB, take 211 us with the join (6.0 TB/s; a plain read 7.06), of 32 rows
// 222, eight waves a CU 235 and 240, a shared tile 246 and more; 96 requests of 16 rows
// on 800 tokens 222 (185 at that rate: queries, masks and first keys of each piece have
// nothing to hide behind).  All waits are the compiler's.
#pragma once

#include "tree_tile.h"

namespace parrot {

constexpr int kStreamLds = 8192;          // bytes of LDS per wave
constexpr int kStreamCols = 32;           // columns of a wave, at most

template <int DT, int D, int NS>
struct TreeStream : TreeState<DT, D, NS> {
  using Base = TreeState<DT, D, NS>;
  using Base::lane; using Base::H; using Base::h; using Base::qf; using Base::qs; using Base::o; using Base::lsr;
  using Base::column;
  static constexpr int ROW_B = Base::ROW_B, GRAN = Base::GRAN, BLK_B = Base::BLK_B, DT16 = Base::DT16, KS = Base::KS;
  static constexpr int NBLK = kStreamLds / BLK_B;            // blocks per step
  static constexpr int TOK = NBLK * kBlock;                  // tokens per step
  static constexpr int NL = 8;                               // loads of each tensor per step
  static constexpr int KL = NL / NBLK;                       // K loads per block
  static constexpr int LPT = 64 / (1024 / ROW_B);            // lanes per token of a V load
  static_assert(NL * 1024 == kStreamLds && NBLK >= 1, "a step is eight loads of each tensor");

  char* lds;
  unsigned va[DT == kF32 ? 1 : DT16];
  unsigned mlo[NS], mhi[NS];              // the columns' mask words

  PARROT_DEV TreeStream(char* wave_lds, int heads, int head, float scale_log2)
      : Base(heads, head, scale_log2, 0, 1), lds(wave_lds) {
    if constexpr (DT != kF32) {
      const int vrow = 4 * (lane >> 4) + ((lane & 15) >> 2);
#pragma unroll
      for (int dt = 0; dt < DT16; ++dt) {
        va[dt] = lds_addr(lds) + vrow * ROW_B + 8 * (lane & 1) +
                 (((2 * dt + ((lane & 3) >> 1)) ^ tree_detail::swizzle<DT, D>(vrow)) << 4);
        asm volatile("" : "+v"(va[dt]));
      }
    }
#pragma unroll
    for (int c = 0; c < NS; ++c) mlo[c] = mhi[c] = 0u;
  }

  // The mask words of the request's drafted rows (at most 32).  Lane j holds row j's bits
  // and the ancestor they reach; taking over that ancestor's bits and reach doubles it.
  PARROT_DEV void build_masks(const int* tree, const RowSpan& rw, int base, int G) {
    const bool mine = lane < rw.count;
    int up = -1;
    if (mine) {
      up = tree ? tree[rw.first + lane] : lane - 1;
      if (up < -1 || up >= lane) up = -1;
    }
    unsigned bits = mine && lane < 32 ? 1u << lane : 0u;
    for (int reach = 1; reach < rw.count; reach <<= 1) {
      const int from = up < 0 ? lane : up;
      const unsigned theirs = (unsigned)__shfl((int)bits, from);
      const int further = __shfl(up, from);
      if (up >= 0) { bits |= theirs; up = further; }
    }
    const int shift = base & 31;
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      const int j = min(column(c) / G, kWave - 1);
      const unsigned b = (unsigned)__shfl((int)bits, j);     // (0 past the request's rows)
      mlo[c] = (b << shift) | ((1u << shift) - 1u);
      mhi[c] = shift ? b >> (32 - shift) : 0u;
    }
  }

  PARROT_DEV void run(const TreeRange& rg) {
    const int b0 = rg.t0 / kBlock;
    const int nb = (rg.t1 - rg.t0 + kBlock - 1) / kBlock;
    if (nb <= 0) return;
    const int steps = (nb + NBLK - 1) / NBLK;
    const size_t blk_stride = (size_t)H * BLK_B;
    const int plain = min(rg.t1, rg.mask0);                  // keys before it need no mask
    int id[NBLK], cur[NBLK];
    auto ids = [&](int st) {                                 // past the end: the last block again, unused
#pragma unroll
      for (int b = 0; b < NBLK; ++b) id[b] = ld_uniform(rg.tbl + b0 + min(st * NBLK + b, nb - 1));
    };
    u32x4 kr[NL], vr[NL];
    const int koff = (lane & 15) * ROW_B + (lane >> 4) * 16;
    auto issue = [&]() {
#pragma unroll
      for (int b = 0; b < NBLK; ++b) {
        cur[b] = (int)min((unsigned)id[b], (unsigned)(rg.npool - 1));
        const size_t off = (size_t)cur[b] * blk_stride + (size_t)h * BLK_B;
        const char* kp = (const char*)rg.pk + off + koff;
        const char* vp = (const char*)rg.pv + off + lane * 16;
#pragma unroll
        for (int l = 0; l < KL; ++l) kr[b * KL + l] = ld16(kp + l * 64);
#pragma unroll
        for (int l = 0; l < KL; ++l) vr[b * KL + l] = ld16_stream(vp + l * 1024);
      }
    };
    ids(0);
    issue();
    ids(min(1, steps - 1));
#pragma unroll 1
    for (int st = 0; st < steps; ++st) {
      const int tok0 = (b0 + st * NBLK) * kBlock;
      const bool masked = tok0 + TOK > plain;
      // S^T of the step's blocks
      f32x4 s[NS][NBLK];
#pragma unroll
      for (int c = 0; c < NS; ++c)
#pragma unroll
        for (int b = 0; b < NBLK; ++b) s[c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int l = 0; l < KL; ++l)
#pragma unroll
        for (int b = 0; b < NBLK; ++b)
#pragma unroll
          for (int c = 0; c < NS; ++c) {
            if constexpr (DT == kF32) {
              float k[4];
              Elem<DT>::to_f32(kr[b * KL + l], k);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                s[c][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], qs[c][4 * l + e], s[c][b], 0, 0, 0);
            } else {
              s[c][b] = prefix_detail::Mfma<DT>::qk(kr[b * KL + l], qf[c][l], s[c][b]);
            }
          }
      // values past the range, and drafted ones that are no finite numbers, are cleared
      unsigned long long bad = 0;                            // a bit per token of the step
      if (masked) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int tok = tok0 + (i * 1024 + lane * 16) / ROW_B;
          bool cleared = false;
          if (tok >= min(rg.t1, rg.end)) vr[i] = u32x4{0u, 0u, 0u, 0u};
          else if (tok >= rg.base) cleared = tree_detail::clear_nonfinite<DT>(vr[i]);
          const unsigned long long lanes = __ballot(cleared);
          if (lanes)
#pragma unroll
            for (int k = 0; k < 64 / LPT; ++k)
              if ((lanes >> (k * LPT)) & ((1ull << LPT) - 1ull)) bad |= 1ull << (i * (64 / LPT) + k);
        }
      }
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int off = i * 1024 + lane * 16, t = (off % BLK_B) / ROW_B, pos = (off % ROW_B) / 16;
        *reinterpret_cast<u32x4*>(lds + off - pos * 16 + ((pos ^ tree_detail::swizzle<DT, D>(t)) << 4)) = vr[i];
      }
      int was[NBLK];
#pragma unroll
      for (int b = 0; b < NBLK; ++b) was[b] = cur[b];
      // (the next step's loads take this step's registers: not before they are free)
      __builtin_amdgcn_sched_barrier(0);
      if (st + 1 < steps) {
        issue();
        ids(min(st + 2, steps - 1));
      }
      auto value_row = [&](int t) {
        int blk = was[0];
#pragma unroll
        for (int b = 1; b < NBLK; ++b)
          if ((t >> 4) == b) blk = was[b];
        return (const char*)rg.pv + (((size_t)blk * H + h) * kBlock + (t & 15)) * ROW_B;
      };
      if constexpr (DT == kF32) {
#pragma unroll
        for (int b = 0; b < NBLK; ++b) {
          const int tokb = tok0 + b * kBlock;
          if (tokb >= rg.t1) break;
#pragma unroll
          for (int c = 0; c < NS; ++c) {
            float x[4] = {s[c][b][0], s[c][b][1], s[c][b][2], s[c][b][3]};
            unsigned vis = 0xFFFFu;
            if (masked) {
              vis = visible(rg, tokb & ~31, c) >> (tokb & 16) & 0xFFFFu;
              this->template mask<4>(x, vis);
            }
            this->template softmax<4>(x, c);
            const unsigned gone = (unsigned)(bad >> (b * kBlock)) & 0xFFFFu;
            if (gone) this->template add_cleared<4>(x, c, vis, gone, [&](int t) { return value_row(b * kBlock + t); });
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
              const int row = 4 * (lane >> 4) + kt;
              const char* vrow = lds + b * BLK_B + row * ROW_B + 4 * (lane & 3);
#pragma unroll
              for (int dt = 0; dt < DT16; ++dt) {
                const float v = *reinterpret_cast<const float*>(
                    vrow + (((4 * dt + ((lane & 15) >> 2)) ^ tree_detail::swizzle<DT, D>(row)) << 4));
                o[c][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, x[kt], o[c][dt], 0, 0, 0);
              }
            }
          }
        }
      } else {
#pragma unroll
        for (int b = 0; b < NBLK; b += 2) {
          const int tokp = tok0 + b * kBlock;
          if (tokp >= rg.t1) break;
          unsigned pw[NS][4];
#pragma unroll
          for (int c = 0; c < NS; ++c) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = s[c][b][i]; x[4 + i] = s[c][b + 1][i]; }
            unsigned vis = 0xFFFFFFFFu;
            if (masked) {
              vis = visible(rg, tokp, c);
              this->template mask<8>(x, vis);
            }
            this->template softmax<8>(x, c);
            const unsigned gone = (unsigned)(bad >> (b * kBlock));
            if (gone) this->template add_cleared<8>(x, c, vis, gone, [&](int t) { return value_row(b * kBlock + t); });
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              pw[c][i] = pack2<DT>(x[2 * i], x[2 * i + 1]);
              lsr[c] = add_pair<DT>(pw[c][i], lsr[c]);
            }
          }
#pragma unroll
          for (int dt = 0; dt < DT16; dt += 2) {
            unsigned long long v[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              v[u][0] = lds_read_tr<DT>(va[dt + u], b * BLK_B);
              v[u][1] = lds_read_tr<DT>(va[dt + u], (b + 1) * BLK_B);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int c = 0; c < NS; ++c) {
                const unsigned long long p0 = pw[c][0] | ((unsigned long long)pw[c][1] << 32);
                const unsigned long long p1 = pw[c][2] | ((unsigned long long)pw[c][3] << 32);
                o[c][dt + u] = prefix_detail::Mfma<DT>::pv2(v[u][0], v[u][1], p0, p1, o[c][dt + u]);
              }
          }
        }
      }
    }
  }

 private:
  // bits of the 32 tokens from tok (a multiple of 32) that column c sees
  PARROT_DEV unsigned visible(const TreeRange& rg, int tok, int c) const {
    if (tok >= rg.mask0) return tok == rg.mask0 ? mlo[c] : mhi[c];
    return rg.t1 - tok < 32 ? (1u << (rg.t1 - tok)) - 1u : 0xFFFFFFFFu;
  }
};

}  // namespace parrot
