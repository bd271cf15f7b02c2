// Attention for trees of drafted tokens over the paged cache (see tree_tile.h for the
// tile and its mathematics).
//
// One workgroup per (request, cache head, column tile) goes through the prefixes of the
// request's group chain and its own tokens and writes the output.
#include "tree_tile.h"

namespace parrot {

// The visible drafted tokens of the tile's columns into lds.mask.  Row j sees itself
// and what its parent sees: each thread holds one row's bits and the ancestor they
// reach, and takes over that ancestor's bits and reach, so the reach doubles at each
// of at most seven steps.  Uses the ring, which is free until the first range runs.
template <int DT, int D>
PARROT_DEV void build_masks(const TreeArgs& a, tree_detail::Lds<DT>& lds, const RowSpan& rw, int base,
                            int col0, int ncols) {
  constexpr int NW = kTreeRows / 32;
  struct Scratch { unsigned bits[kTreeRows][NW]; int up[kTreeRows]; };
  static_assert(sizeof(Scratch) <= sizeof(lds.ring), "scratch fits the ring");
  Scratch& sc = *reinterpret_cast<Scratch*>(&lds.ring[0][0]);
  const int tid = threadIdx.x;
  const bool mine = tid < rw.count;
  unsigned bits[NW];
#pragma unroll
  for (int w = 0; w < NW; ++w) bits[w] = mine && (tid >> 5) == w ? 1u << (tid & 31) : 0u;
  int up = -1;
  if (mine) {
    up = a.tree ? a.tree[rw.first + tid] : tid - 1;
    if (up < -1 || up >= tid) up = -1;
  }
  auto publish = [&] {
    if (mine) {
#pragma unroll
      for (int w = 0; w < NW; ++w) sc.bits[tid][w] = bits[w];
      sc.up[tid] = up;
    }
    __syncthreads();
  };
  for (int reach = 1; reach < rw.count; reach <<= 1) {
    publish();
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < NW; ++w) bits[w] |= sc.bits[up][w];
      up = sc.up[up];
    }
    __syncthreads();
  }
  publish();
  if (tid < tree_detail::kCols<DT>) {
    const int j = (col0 + tid) / a.G;
    const int shift = base & 31;
    unsigned below = (1u << shift) - 1u;                    // cached tokens of word 0
#pragma unroll
    for (int w = 0; w <= NW; ++w) {
      const unsigned b = w < NW && tid < ncols ? sc.bits[j][w < NW ? w : 0] : 0u;
      lds.mask[w][tid] = (b << shift) | below;
      below = shift ? b >> (32 - shift) : 0u;
    }
  }
  static_assert(NW + 1 == tree_detail::kMaskWords, "rows shifted by up to 31 bits");
}

// The output rows of a tile that saw its columns' whole contexts.
template <int DT, int D, int NS, class F>
PARROT_DEV void write_output(const TreeArgs& a, TreeTile<DT, D, NS>& tile, int ncols, F row_of) {
  tile.finish([&](int c, int col, float lw, float lse2, float) {
    if (col >= ncols) return;
    const size_t at = row_of(col);
    const float inv = 1.f / lw;            // (0 only where every logit is -inf: the result is NaN)
    char* dst = (char*)a.out + (at * D + 4 * (tile.lane >> 4)) * Elem<DT>::kBytes;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      const f32x4 v = tile.o[c][dt] * inv;
      if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(dst + dt * 64) = v;
      else store4<DT>(dst + dt * 32, v);
    }
    if (tile.lane < 16) a.lse[at] = lse2 * kLn2;
  });
}

template <int DT, int D, int NS>
PARROT_DEV void tree_item(const TreeArgs& a, tree_detail::Lds<DT>& lds, int r, int h, const RowSpan& rw, int S,
                          int col0, int ncols) {
  const int base = S - rw.count;
  const int HQ = a.H * a.G;
  TreeTile<DT, D, NS> tile(lds, a.H, h, a.scale_log2);
  auto row_of = [&](int col) {                              // in units of heads
    const int x = col0 + col;
    return (size_t)(rw.first + x / a.G) * HQ + h * a.G + x % a.G;
  };
  tile.load_queries(a.q, ncols, row_of);

  int g = ld_uniform(a.gid + r);
  for (int l = 0;; ++l) {                                   // the chain's prefixes, then the own tokens
    const bool pre = l < a.depth && g >= 0 && g < a.NG;
    const int P = pre ? clampi(ld_uniform(a.plen + g), 0, a.max_p) : 0;
    TreeRange rg;
    rg.pk = pre ? a.pk : a.sk;
    rg.pv = pre ? a.pv : a.sv;
    rg.tbl = pre ? a.ptab + (long)g * a.pstride : a.stab + (long)r * a.sstride;
    rg.npool = pre ? a.npblk : a.nsblk;
    rg.t0 = 0;
    rg.t1 = pre ? P : S;
    rg.mask0 = pre ? 0x40000000 : base & ~31;
    rg.base = pre ? P : base;
    rg.end = rg.t1;
    tile.run(rg);
    if (!pre) break;
    g = a.parents ? ld_uniform(a.parents + g) : -1;
  }

  write_output<DT, D, NS>(a, tile, ncols, row_of);
}

template <int DT, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3, 3)))
void k_tree_decode(TreeArgs a) {
  constexpr int COLS = tree_detail::kCols<DT>;
  __shared__ __attribute__((aligned(1024))) tree_detail::Lds<DT> lds;
  // a sequence's column tiles read the same keys: they are 8 workgroups apart, on one XCD
  const int idx = (int)(blockIdx.x / (8 * a.tiles)) * 8 + (int)(blockIdx.x % 8);
  const int col0 = (int)(blockIdx.x / 8 % a.tiles) * COLS;
  if (idx >= a.R * a.H) return;
  const int r = idx / a.H, h = idx % a.H;
  const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
  const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
  const int ncols = min(COLS, rw.count * a.G - col0);
  if (ncols <= 0) return;
  build_masks<DT, D>(a, lds, rw, S - rw.count, col0, ncols);
  // the waves' parts: two sets where the wave's second one has columns
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (tree_detail::kSets<DT> == 2 && (wave + 4) * 16 < ncols)
    tree_item<DT, D, tree_detail::kSets<DT>>(a, lds, r, h, rw, S, col0, ncols);
  else
    tree_item<DT, D, 1>(a, lds, r, h, rw, S, col0, ncols);
}

// ------------------------------------------------------------------ split plan
// Two kinds of workgroups of one launch write partial results, the join combines them.
//
//  own role, workgroups [0, runs * H): the own tokens of all requests, laid end to end
//    by (request, column tile, unit of tokens), cut into `runs` equal runs; a workgroup
//    streams one run of one cache head.  Nothing depends on how ragged the contexts
//    are, and the heads of a run read a block's heads together.  Where runs cut a
//    sequence, each piece gets a partial result.
//  prefix role: the rows of all requests that read a group's prefix, stacked in request
//    order, a column tile of them against one chunk of the prefix, so that the
//    prefix is streamed once per tile and not once per request.

struct OwnCost { int S, count, first, tiles, units; };   // units per tile, setup excluded
template <int DT, int D>
PARROT_DEV OwnCost own_cost(const TreeArgs& a, int r) {
  OwnCost c;
  c.S = clampi(a.slen[r], 0, a.max_s);
  const int begin = a.qoff[r], end = a.qoff[r + 1];
  c.first = clampi(begin, 0, a.T);
  const int cap = min(min(c.S, a.max_q), a.T - c.first);
  const long n = (long)end - begin;
  c.count = (int)(n < 0 ? 0 : n > cap ? cap : n);
  c.tiles = (c.count * a.G + tree_detail::kCols<DT> - 1) / tree_detail::kCols<DT>;
  c.units = (c.S + tree_unit(DT, D) - 1) / tree_unit(DT, D);
  return c;
}

// Inclusive sum over the workgroup's 256 threads; *total is the whole sum.
PARROT_DEV int scan256(int x, int* lds4, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int v = __shfl_up(x, d);
    if (lane >= d) x += v;
  }
  __syncthreads();
  if (lane == kWave - 1) lds4[wave] = x;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += lds4[w];
    sum += lds4[w];
  }
  *total = sum;
  return x + before;
}

// A tile's partial results: slot `slot` of the columns' rows.
template <int DT, int D, int NS, class F>
PARROT_DEV void write_partial(const TreeArgs& a, TreeTile<DT, D, NS>& tile, int ncols, int slot, F row_of) {
  tile.finish([&](int c, int col, float lw, float lse2, float lt) {
    if (col >= ncols) return;
    const size_t at = row_of(col) * (size_t)a.seg + slot;
    const float inv = lw == 0.f ? 0.f : 1.f / lw;           // a piece may hold no key the row sees
    float* dst = a.o_part + at * D + 4 * (tile.lane >> 4);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(dst + dt * 16) = tile.o[c][dt] * inv;
    if (tile.lane < 16) a.lse_part[at] = lt == 0.f ? -INFINITY : lse2;
  });
}

template <int DT, int D, int NS>
PARROT_DEV void own_piece(const TreeArgs& a, tree_detail::Lds<DT>& lds, int r, int h, const RowSpan& rw, int S,
                          int col0, int ncols, int t0, int t1, int slot, bool whole) {
  const int HQ = a.H * a.G, base = S - rw.count;
  TreeTile<DT, D, NS> tile(lds, a.H, h, a.scale_log2);
  auto row_of = [&](int col) {
    const int x = col0 + col;
    return (size_t)(rw.first + x / a.G) * HQ + h * a.G + x % a.G;
  };
  tile.load_queries(a.q, ncols, row_of);
  TreeRange rg;
  rg.pk = a.sk; rg.pv = a.sv; rg.tbl = a.stab + (long)r * a.sstride; rg.npool = a.nsblk;
  rg.t0 = t0; rg.t1 = t1; rg.mask0 = base & ~31; rg.base = base; rg.end = S;
  tile.run(rg);
  if (whole) write_output<DT, D, NS>(a, tile, ncols, row_of);
  else write_partial<DT, D, NS>(a, tile, ncols, slot, row_of);
}

template <int DT, int D>
PARROT_DEV void tree_own_role(const TreeArgs& a, tree_detail::Lds<DT>& lds, int wg) {
  constexpr int COLS = tree_detail::kCols<DT>, UNIT = tree_unit(DT, D);
  const int tid = threadIdx.x;
  const int run = wg / a.H, h = wg % a.H;
  int* scratch = reinterpret_cast<int*>(lds.tbl);
  // the whole cost, then where this run begins
  int total = 0;
  for (int b = 0; b < a.R; b += 256) {
    int cost = 0, sum;
    if (b + tid < a.R) {
      const OwnCost c = own_cost<DT, D>(a, b + tid);
      cost = c.tiles * (c.units + kTreeSetup);
    }
    scan256(cost, scratch, &sum);
    total += sum;
  }
  const int q = max(a.min_run, (total + a.runs - 1) / a.runs);
  const int u0 = run * q, u1 = min(total, u0 + q);
  const bool writes = wg == 0;                    // this workgroup leaves the starts for the join
  if (u0 >= total && !writes) return;
  int r = -1, start = 0, before = 0;
  for (int b = 0; b < a.R && (r < 0 || writes); b += 256) {
    int cost = 0, sum;
    if (b + tid < a.R) {
      const OwnCost c = own_cost<DT, D>(a, b + tid);
      cost = c.tiles * (c.units + kTreeSetup);
    }
    const int incl = before + scan256(cost, scratch, &sum);
    if (writes && b + tid < a.R) a.starts[b + tid] = incl - cost;
    if (cost > 0 && incl - cost <= u0 && u0 < incl) { scratch[8] = b + tid; scratch[9] = incl - cost; }
    __syncthreads();
    if (r < 0 && u0 >= before && u0 < before + sum) { r = scratch[8]; start = scratch[9]; }
    before += sum;
  }
  if (writes && tid == 0) { a.starts[a.R] = total; a.starts[a.R + 1] = q; }
  if (r < 0 || u0 >= total) return;
  r = __builtin_amdgcn_readfirstlane(r);
  start = __builtin_amdgcn_readfirstlane(start);

  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (; r < a.R && start < u1; ++r) {
    const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
    const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
    const int tiles = (rw.count * a.G + COLS - 1) / COLS, units = (S + UNIT - 1) / UNIT;
    const int g = ld_uniform(a.gid + r);
    const bool prefixed = a.seg_p > 0 && g >= 0 && g < a.NG;
    for (int t = 0; t < tiles; ++t, start += units + kTreeSetup) {
      const int s0 = start + kTreeSetup;          // cost of the first unit
      const int st0 = max(u0 - s0, 0), st1 = min(u1 - s0, units);
      if (st1 <= st0) continue;
      const int piece = run - s0 / q;
      const bool whole = !prefixed && st0 == 0 && st1 == units;
      const int col0 = t * COLS, ncols = min(COLS, rw.count * a.G - col0);
      const int t0 = st0 * UNIT, t1 = min(S, st1 * UNIT);
      __syncthreads();                            // the ring is free
      if (t1 > ((S - rw.count) & ~31)) build_masks<DT, D>(a, lds, rw, S - rw.count, col0, ncols);
      if (tree_detail::kSets<DT> == 2 && (wave + 4) * 16 < ncols)
        own_piece<DT, D, tree_detail::kSets<DT>>(a, lds, r, h, rw, S, col0, ncols, t0, t1, a.seg_pre + piece, whole);
      else
        own_piece<DT, D, 1>(a, lds, r, h, rw, S, col0, ncols, t0, t1, a.seg_pre + piece, whole);
    }
  }
}

template <int DT, int D, int NS>
PARROT_DEV void prefix_piece(const TreeArgs& a, tree_detail::Lds<DT>& lds, int g, int h, int P, int t0, int t1,
                             int col0, int row0, int ncols, int slot) {
  const int* rows = reinterpret_cast<const int*>(&lds.mask[0][0]);
  const int HQ = a.H * a.G;
  TreeTile<DT, D, NS> tile(lds, a.H, h, a.scale_log2);
  auto row_of = [&](int col) {
    const int x = col0 + col;
    return (size_t)rows[x / a.G - row0] * HQ + h * a.G + x % a.G;
  };
  tile.load_queries(a.q, ncols, row_of);
  TreeRange rg;
  rg.pk = a.pk; rg.pv = a.pv; rg.tbl = a.ptab + (long)g * a.pstride; rg.npool = a.npblk;
  rg.t0 = t0; rg.t1 = t1; rg.mask0 = 0x40000000; rg.base = t1; rg.end = t1;
  tile.run(rg);
  write_partial<DT, D, NS>(a, tile, ncols, slot, row_of);
}

template <int DT, int D>
PARROT_DEV void tree_prefix_role(const TreeArgs& a, tree_detail::Lds<DT>& lds, int wg) {
  constexpr int COLS = tree_detail::kCols<DT>;
  // (group, chunk, head) items; their column tiles are 8 workgroups apart, on one XCD
  const int tile = wg / 8 % a.tiles_p;
  int idx = wg / (8 * a.tiles_p) * 8 + wg % 8;
  if (idx >= a.NG * a.seg_p * a.H) return;
  const int h = idx % a.H; idx /= a.H;
  const int c = idx % a.seg_p, g = idx / a.seg_p;
  const int P = clampi(ld_uniform(a.plen + g), 0, a.max_p);
  const int t0 = c * a.cp;
  if (t0 >= P) return;
  const int t1 = min(P, t0 + a.cp);
  int lvl = 0;                                            // ancestors of g (< depth)
  if (a.parents)
    for (int x = ld_uniform(a.parents + g); x >= 0 && x < a.NG && lvl < a.depth - 1; x = ld_uniform(a.parents + x)) ++lvl;
  // rows [row0, row0 + COLS] of the stacked list hold this tile's columns
  const int col0 = tile * COLS, row0 = col0 / a.G;
  int* rows = reinterpret_cast<int*>(&lds.mask[0][0]);
  constexpr int MOST = COLS + 1;
  static_assert(sizeof(lds.mask) >= (MOST + 1) * sizeof(int), "the row list fits the mask");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (wave == 0) {
    int base = 0;
    for (int b = 0; b < a.R && base < row0 + MOST; b += kWave) {
      const int r = b + lane;
      bool reads = false;
      OwnCost oc;
      oc.count = 0; oc.first = 0;
      if (r < a.R) {
        int x = a.gid[r];
        oc = own_cost<DT, D>(a, r);
        for (int d = 0; d < a.depth && x >= 0 && x < a.NG; ++d) {
          if (x == g) { reads = true; break; }
          x = a.parents ? a.parents[x] : -1;
        }
      }
      const int n = reads ? oc.count : 0;
      int incl = n;
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) {
        const int v = __shfl_up(incl, d);
        if (lane >= d) incl += v;
      }
      const int first = base + incl - n;
      for (int x = max(first, row0), e = min(first + n, row0 + MOST); x < e; ++x) rows[x - row0] = oc.first + x - first;
      base += __shfl(incl, kWave - 1);
    }
    if (lane == 0) rows[MOST] = base;
  }
  __syncthreads();
  const int ncols = min(COLS, rows[MOST] * a.G - col0);
  if (ncols <= 0) return;
  if (tree_detail::kSets<DT> == 2 && (wave + 4) * 16 < ncols)
    prefix_piece<DT, D, tree_detail::kSets<DT>>(a, lds, g, h, P, t0, t1, col0, row0, ncols, lvl * a.seg_p + c);
  else
    prefix_piece<DT, D, 1>(a, lds, g, h, P, t0, t1, col0, row0, ncols, lvl * a.seg_p + c);
}

template <int DT, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3, 3)))
void k_tree_partials(TreeArgs a) {
  __shared__ __attribute__((aligned(1024))) tree_detail::Lds<DT> lds;
  const int own = a.runs * a.H;
  if ((int)blockIdx.x < own) tree_own_role<DT, D>(a, lds, blockIdx.x);
  else tree_prefix_role<DT, D>(a, lds, blockIdx.x - own);
}

// Join: a workgroup per row combines the partial results of its query heads.  With
// base-2 log-sum-exps l_i and normalised outputs o_i of disjoint key sets,
// l = log2 sum 2^{l_i}, o = sum 2^{l_i - l} o_i.  A wave takes a head at a time; lane i
// holds the weight of partial i.
template <int DT, int D>
__global__ __launch_bounds__(256) void k_tree_join(TreeArgs a) {
  using E = Elem<DT>;
  constexpr int EPL = D / kWave;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x;
  const int r = __builtin_amdgcn_readfirstlane(request_of_row(a.qoff, a.R, t, lane));
  if (r < 0) return;
  const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
  const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
  if (t < rw.first || t >= rw.first + rw.count) return;   // padding
  const int q = ld_uniform(a.starts + a.R + 1), start = ld_uniform(a.starts + r);
  const int units = (S + tree_unit(DT, D) - 1) / tree_unit(DT, D);
  // the chunks of the chain's levels, outermost first
  int np[kMaxDepth] = {0, 0, 0, 0}, len[kMaxDepth];
  int nlev = 0;
  const int gid = ld_uniform(a.gid + r);
  const bool prefixed = a.seg_p > 0 && gid >= 0 && gid < a.NG;
  for (int g = gid; a.seg_p > 0 && g >= 0 && g < a.NG && nlev < a.depth;
       g = a.parents ? ld_uniform(a.parents + g) : -1)
    len[nlev++] = min((clampi(ld_uniform(a.plen + g), 0, a.max_p) + a.cp - 1) / a.cp, a.seg_p);
#pragma unroll
  for (int l = 0; l < kMaxDepth; ++l)
#pragma unroll
    for (int x = 0; x < kMaxDepth; ++x)
      if (x == nlev - 1 - l) np[l] = len[x];
  const int b1 = np[0], b2 = b1 + np[1], b3 = b2 + np[2], b4 = b3 + np[3];
  const int HQ = a.H * a.G;
  for (int hq = wave; hq < HQ; hq += 4) {
    const int col = (t - rw.first) * a.G + hq % a.G;
    const int s0 = start + col / tree_detail::kCols<DT> * (units + kTreeSetup) + kTreeSetup;
    const int pieces = (s0 + units - 1) / q - s0 / q + 1;
    if (!prefixed && pieces == 1) continue;               // written by the piece itself
    const int n = b4 + pieces;
    auto slot_of = [&](int i) {
      int sl = a.seg_pre + (i - b4);
      sl = i < b4 ? 3 * a.seg_p + (i - b3) : sl;
      sl = i < b3 ? 2 * a.seg_p + (i - b2) : sl;
      sl = i < b2 ? a.seg_p + (i - b1) : sl;
      return i < b1 ? i : sl;
    };
    const size_t at = (size_t)t * HQ + hq;
    const float* lsep = a.lse_part + at * a.seg;
    const float* op = a.o_part + at * a.seg * D;
    float mx = -INFINITY;
    for (int i = lane; i < n; i += kWave) mx = fmaxf(mx, lsep[slot_of(i)]);
    mx = fmaxf(mx, dpp_f<kDppXor1>(mx));
    mx = fmaxf(mx, dpp_f<kDppXor2>(mx));
    mx = fmaxf(mx, dpp_f<kDppHalfMirror>(mx));
    mx = fmaxf(mx, dpp_f<kDppMirror>(mx));
    mx = max_xor32(max_xor16(mx));
    float tot = 0.f, acc[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[e] = 0.f;
    for (int b = 0; b < n; b += kWave) {
      // (no guard on mx: logits that are all -inf give NaN)
      const float w = b + lane < n ? fast_exp2(lsep[slot_of(b + lane)] - mx) : 0.f;
      tot += w;
      const int m = min(kWave, n - b);
      for (int i = 0; i < m; ++i) {
        const float wi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), i));
        const float* src = op + (size_t)slot_of(b + i) * D + lane * EPL;
#pragma unroll
        for (int e = 0; e < EPL; ++e) acc[e] = __builtin_fmaf(wi, src[e], acc[e]);
      }
    }
    tot = group_sum<64>(tot);
    const float inv = 1.f / tot;
    char* dst = (char*)a.out + (at * D + lane * EPL) * E::kBytes;
#pragma unroll
    for (int e = 0; e < EPL; ++e) E::store1(dst + e * E::kBytes, acc[e] * inv);
    if (lane == 0) a.lse[at] = (mx + fast_log2(tot)) * kLn2;
  }
}

template <int DT, int D>
static hipError_t launch_tree_t(const TreeArgs& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const long groups = ((long)a.R * a.H + 7) / 8;
  hipExtLaunchKernelGGL((k_tree_decode<DT, D>), dim3((unsigned)(groups * 8 * a.tiles)), dim3(256), 0, s, e0, e1, 0, a);
  return hipGetLastError();
}

hipError_t launch_tree(const TreeArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (a.T < 1 || a.R < 1 || a.H < 1 || a.G < 1 || a.max_q < 1 || a.max_q > kTreeRows || a.tiles < 1 ||
      (long)a.tiles * tree_cols(dtype) < (long)a.max_q * a.G || a.sstride < 1 || a.nsblk < 1 ||
      ((long)a.R * a.H + 7) / 8 * 8 * a.tiles > 0x7fffffffL || (a.NG > 0 && (a.npblk < 1 || a.pstride < 1)))
    return hipErrorInvalidValue;
  switch (dtype * 1000 + D) {
    case kF32 * 1000 + 64: return launch_tree_t<kF32, 64>(a, s, e0, e1);
    case kF32 * 1000 + 128: return launch_tree_t<kF32, 128>(a, s, e0, e1);
    case kF16 * 1000 + 64: return launch_tree_t<kF16, 64>(a, s, e0, e1);
    case kF16 * 1000 + 128: return launch_tree_t<kF16, 128>(a, s, e0, e1);
    case kBF16 * 1000 + 64: return launch_tree_t<kBF16, 64>(a, s, e0, e1);
    case kBF16 * 1000 + 128: return launch_tree_t<kBF16, 128>(a, s, e0, e1);
  }
  return hipErrorInvalidValue;
}

template <int DT, int D>
static void launch_partials_t(const TreeArgs& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const dim3 grid((unsigned)((long)a.runs * a.H + a.n_pre));
  hipExtLaunchKernelGGL((k_tree_partials<DT, D>), grid, dim3(256), 0, s, e0, e1, 0, a);
}
template <int DT, int D>
static void launch_join_t(const TreeArgs& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  hipExtLaunchKernelGGL((k_tree_join<DT, D>), dim3((unsigned)a.T), dim3(256), 0, s, e0, e1, 0, a);
}

#define PARROT_TREE_LAUNCH(NAME)                                              \
  switch (dtype * 1000 + D) {                                                 \
    case kF32 * 1000 + 64: NAME<kF32, 64>(a, s, e0, e1); break;               \
    case kF32 * 1000 + 128: NAME<kF32, 128>(a, s, e0, e1); break;             \
    case kF16 * 1000 + 64: NAME<kF16, 64>(a, s, e0, e1); break;               \
    case kF16 * 1000 + 128: NAME<kF16, 128>(a, s, e0, e1); break;             \
    case kBF16 * 1000 + 64: NAME<kBF16, 64>(a, s, e0, e1); break;             \
    case kBF16 * 1000 + 128: NAME<kBF16, 128>(a, s, e0, e1); break;           \
    default: return hipErrorInvalidValue;                                     \
  }                                                                           \
  return hipGetLastError()

hipError_t launch_tree_partials(const TreeArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const long pre = a.n_pre > 0 ? ((long)a.NG * a.seg_p * a.H + 7) / 8 * 8 * a.tiles_p : 0;
  if (a.T < 1 || a.R < 1 || a.H < 1 || a.G < 1 || a.max_q < 1 || a.max_q > kTreeRows || a.sstride < 1 ||
      a.nsblk < 1 || a.runs < 1 || a.min_run < 1 || !a.o_part || !a.lse_part || !a.starts || a.n_pre != pre ||
      (a.n_pre > 0 && (a.npblk < 1 || a.pstride < 1 || a.cp < 64 || a.cp % 64 != 0 || a.depth < 1)) ||
      (long)a.runs * a.H + a.n_pre > 0x7fffffffL || a.depth > kMaxDepth)
    return hipErrorInvalidValue;
  PARROT_TREE_LAUNCH(launch_partials_t);
}

hipError_t launch_tree_join(const TreeArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  PARROT_TREE_LAUNCH(launch_join_t);
}

}  // namespace parrot
