// Arguments of the tree-decode kernels, shared by the kernels and the host code.
#pragma once

#include "draft_args.h"

namespace parrot {

// Columns of a tree tile: (row, query head) pairs that read one cache head.  Four
// waves with sets of 16 columns each.
constexpr int kTreeSets16 = 2;           // 16-bit caches: 128 columns
constexpr int kTreeSets32 = 1;           // fp32 caches: 64 columns
constexpr int tree_cols(int dtype) { return 64 * (dtype == kF32 ? kTreeSets32 : kTreeSets16); }
constexpr int kTreeSpan = 128;           // key blocks whose ids are held at a time

struct TreeArgs {
  const void* q;                         // [T][HQ][D]
  const void* pk; const void* pv;
  const void* sk; const void* sv;
  const int* ptab; const int* plen; const int* stab; const int* slen; const int* gid;
  const int* parents;                    // nested groups (NULL: flat)
  const int* qoff;                       // [R + 1]
  const int* tree;                       // drafted rows' parents (NULL: chains)
  void* out; float* lse;                 // [T][HQ][D] dtype, [T][HQ]
  int T, R, H, G, NG, depth;             // G query heads per cache head
  int pstride, sstride, max_p, max_s, max_q, npblk, nsblk;
  int tiles;                             // column tiles per request
  float scale_log2;

  // Split plan only.  Partial results: outputs o_part [slot][D] (normalised) and log-sum-exps
  // lse_part [slot] (base 2).  The first [held][HQ][seg_pre] slots are the prefixes': for each
  // row of a request that has any, counted in request order (`held` bounds them), entry
  // l * seg_p + c is chunk c of the prefix at level l of the request's chain (0: outermost).
  // From own0 on, [H][pieces][piece_cols] are the own tokens': tile t of request r, cut by run
  // u, is piece u + r * tiles + t.  Along the cost each next piece takes the next run or the
  // next tile, so no two share a number, and their bytes go with the runs and the tiles,
  // not with the rows times the pieces a row may have.
  float* o_part; float* lse_part;
  size_t own0;
  int held, pieces, piece_cols;
  int* desc;                             // [T][kTreeDesc]: what the join needs of each row
  int seg, seg_p, seg_pre;               // seg: partial results of a row, at most
  int cp;                                // prefix chunk tokens
  int tiles_p;                           // column tiles per group
  int sets;                              // 0: own tokens by tiles, else by waves of that many column sets
  int own_wgs;                           // workgroups of the own tokens
  int runs;                              // runs of the own tokens' cost: a workgroup each (by waves: a wave)
                                         // per cache head
  int min_run;                           // least cost of a run
  int n_pre;                             // prefix workgroups
  int first;                             // of them before those of the own tokens: all or none
};

// Row descriptor: cost of the first unit of the row's first column tile, cost between
// tiles, units, run length, prefix chunks of the chain's levels (outermost first, 16
// bits each, two ints), the row within its request, its request and (bit 0) whether that has
// prefixes, the row's number among those that have.
constexpr int kTreeDesc = 12;

// The partial results of a row: its prefix chunks, outermost level first (lo, hi: their
// counts, as the descriptor holds them), then `own` pieces of its own tokens.  Index i is
// entry slot(i): below seg_pre of the row's prefix slots, from there on its pieces.  Counts are clamped so that any descriptor (that of a row
// which no request holds was never written) stays inside them.
struct TreeSlots {
  int b1, b2, b3, b4, n, seg_p, seg_pre;
  __host__ __device__ int slot(int i) const {
    int sl = seg_pre + (i - b4);
    sl = i < b4 ? 3 * seg_p + (i - b3) : sl;
    sl = i < b3 ? 2 * seg_p + (i - b2) : sl;
    sl = i < b2 ? seg_p + (i - b1) : sl;
    return i < b1 ? i : sl;
  }
};
__host__ __device__ inline TreeSlots tree_slots(unsigned lo, unsigned hi, int own, int seg_p, int seg_pre, int seg) {
  auto least = [](int x, int y) { return x < y ? x : y; };
  auto chunks = [&](unsigned count, int level) {               // (the row has slots for seg_pre / seg_p levels)
    return least((int)count, least(seg_p, seg_pre - level * seg_p < 0 ? 0 : seg_pre - level * seg_p));
  };
  TreeSlots s;
  s.b1 = chunks(lo & 0xFFFFu, 0);
  s.b2 = s.b1 + chunks(lo >> 16, 1);
  s.b3 = s.b2 + chunks(hi & 0xFFFFu, 2);
  s.b4 = s.b3 + chunks(hi >> 16, 3);
  s.n = s.b4 + least(own < 0 ? 0 : own, seg - seg_pre);
  s.seg_p = seg_p;
  s.seg_pre = seg_pre;
  return s;
}

// Own tokens are streamed in units of kTreeUnit tokens; a column tile of a request costs
// its units and kTreeSetup more.
constexpr int kTreeSetup = 2;
constexpr int tree_unit(int dtype, int D) { return dtype != kF32 && D == 64 ? 64 : 32; }

// One workgroup per request, cache head and column tile, output written by it: a tile,
// or (small: at most 16 columns, rows of tree_small_rows) waves that share the keys.
constexpr bool tree_small_rows(int dtype, int D) { return D * (dtype == kF32 ? 4 : 2) >= 256; }
hipError_t launch_tree(const TreeArgs& a, bool small, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
// Partial results of prefixes and own tokens, and their combination.
hipError_t launch_tree_partials(const TreeArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
hipError_t launch_tree_join(const TreeArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);

}  // namespace parrot
