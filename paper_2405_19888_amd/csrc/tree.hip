// Attention for trees of drafted tokens over the paged cache (see tree_tile.h for the
// tile and its mathematics).
//
// k_tree_decode: a workgroup per (request, cache head, column tile) goes through the
// prefixes of the request's group chain and its own tokens and writes the output.
// k_tree_small: the same for at most 16 columns, by waves that share the keys.
// k_tree_partials, k_tree_join: the split plan, pieces of prefixes and of own tokens, and
// their combination.
#include "tree_stream.h"

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

// The output rows of a tile that saw its columns' whole contexts.  Every row sees itself, so a
// weight sum of 0 means that each logit is -inf: output and log-sum-exp are NaN then, as the
// join gives them (-inf is left to contexts without keys, which no row has).
template <int DT, int D, int NS, class F>
PARROT_DEV void write_output(const TreeArgs& a, TreeState<DT, D, NS>& tile, int ncols, F row_of) {
  tile.finish([&](int c, int col, float lw, float lse2, float lt) {
    if (col >= ncols) return;
    const size_t at = row_of(col);
    const float inv = 1.f / lw;
    char* dst = (char*)a.out + (at * D + 4 * (tile.lane >> 4)) * Elem<DT>::kBytes;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      const f32x4 v = tile.o[c][dt] * inv;
      if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(dst + dt * 64) = v;
      else store4<DT>(dst + dt * 32, v);
    }
    if (tile.lane < 16) a.lse[at] = lt == 0.f ? __builtin_nanf("") : lse2 * kLn2;
  });
}

template <int DT, int D, int NS>
PARROT_DEV void tree_item(const TreeArgs& a, tree_detail::Lds<DT>& lds, int r, int h, const RowSpan& rw, int S,
                          int col0, int ncols) {
  const int base = S - rw.count;
  const int HQ = a.H * a.G;
  TreeTile<DT, D, NS> tile(lds, a.H, h, a.scale_log2, ncols);
  auto row_of = [&](int col) {                              // in units of heads
    const int x = col0 + col;
    return (size_t)(rw.first + x / a.G) * HQ + h * a.G + x % a.G;
  };
  tile.template load_queries<false>(a.q, ncols, row_of);

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
    tile.run(rg, [] {});
    if (!pre) break;
    g = a.parents ? ld_uniform(a.parents + g) : -1;
  }

  if (tile.act) write_output<DT, D, NS>(a, tile, ncols, row_of);
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

// The first slot of an own piece: its columns follow.
PARROT_DEV size_t piece_slot(const TreeArgs& a, int h, int piece) {
  return a.own0 + ((size_t)h * a.pieces + piece) * a.piece_cols;
}

// A tile's partial results, each column's at slot slot_of(col).
template <int DT, int D, int NS, class F>
PARROT_DEV void write_partial(const TreeArgs& a, TreeState<DT, D, NS>& tile, int ncols, F slot_of) {
  tile.finish([&](int c, int col, float lw, float lse2, float lt) {
    if (col >= ncols) return;
    const size_t at = slot_of(col);
    const float inv = lw == 0.f ? 0.f : 1.f / lw;           // a piece may hold no key the row sees
    float* dst = a.o_part + at * D + 4 * (tile.lane >> 4);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(dst + dt * 16) = tile.o[c][dt] * inv;
    if (tile.lane < 16) a.lse_part[at] = lt == 0.f ? -INFINITY : lse2;
  });
}

// One tile against one key range: columns col0 .. col0 + ncols of the sequence whose rows
// from row0 on are in lds.rows.  slot: the chunk's entry of each row (own: the piece's
// number); < 0: the columns' whole context, the output.
struct TreePiece { TreeRange rg; int h, col0, ncols, row0, slot; };

template <int DT, int D, int NS>
PARROT_DEV void tree_piece(const TreeArgs& a, tree_detail::Lds<DT>& lds, const TreePiece& pc, bool own) {
  TreeTile<DT, D, NS> tile(lds, a.H, pc.h, a.scale_log2, pc.ncols);
  auto row_of = [&](int col) {                              // in units of heads
    const int x = pc.col0 + col, row = x / a.G;
    return (size_t)lds.rows[row - pc.row0] * (a.H * a.G) + pc.h * a.G + (x - row * a.G);
  };
  tile.run(pc.rg, [&] { tile.template load_queries<false>(a.q, pc.ncols, row_of); });
  if (!tile.act) return;
  if (pc.slot < 0) write_output<DT, D, NS>(a, tile, pc.ncols, row_of);
  else if (own) write_partial<DT, D, NS>(a, tile, pc.ncols, [&](int col) { return piece_slot(a, pc.h, pc.slot) + col; });
  else write_partial<DT, D, NS>(a, tile, pc.ncols, [&](int col) {
    const int x = pc.col0 + col, row = x / a.G;
    return ((size_t)lds.held[row - pc.row0] * (a.H * a.G) + pc.h * a.G + (x - row * a.G)) * a.seg_pre + pc.slot;
  });
}

// The run of an own-role wave (tiles: of all waves of its workgroup), and where it stands.
// pad: 0, or the run length q to a multiple of which a tile's cost is taken up where its
// request has several.
struct OwnRun { int u0, u1, q, pad, r, start, tile; };
PARROT_DEV int tile_cost(int units, int tiles, int pad) {
  const int cost = units + kTreeSetup;
  return tiles > 1 && pad > 0 ? (cost + pad - 1) / pad * pad : cost;
}

// Whether request r has prefixes that the prefix role reads.
PARROT_DEV bool has_prefixes(const TreeArgs& a, int gid) { return a.seg_p > 0 && gid >= 0 && gid < a.NG; }

// What the join needs of the rows of request r, whose cost starts at `start` and whose rows
// are numbers held0, held0 + 1 .. of those with prefixes.
template <int DT, int D>
PARROT_DEV void write_desc(const TreeArgs& a, int r, const OwnCost& c, int start, int held0, int q, int pad) {
  int len[kMaxDepth], nlev = 0;
  const int gid = a.gid[r];
  const bool prefixed = has_prefixes(a, gid);
  for (int g = gid; a.seg_p > 0 && g >= 0 && g < a.NG && nlev < a.depth; g = a.parents ? a.parents[g] : -1) {
    const int n = min((clampi(a.plen[g], 0, a.max_p) + a.cp - 1) / a.cp, a.seg_p);
#pragma unroll
    for (int l = 0; l < kMaxDepth; ++l)
      if (l == nlev) len[l] = n;
    ++nlev;
  }
  unsigned lo = 0, hi = 0;                                  // outermost level first
#pragma unroll
  for (int l = 0; l < kMaxDepth; ++l)
    if (l < nlev) {
      const int at = nlev - 1 - l;
      if (at < 2) lo |= (unsigned)len[l] << (16 * at);
      else hi |= (unsigned)len[l] << (16 * (at - 2));
    }
  for (int j = 0; j < c.count; ++j) {
    int4* d = reinterpret_cast<int4*>(a.desc + (size_t)(c.first + j) * kTreeDesc);
    d[0] = int4{start + kTreeSetup, tile_cost(c.units, c.tiles, pad), c.units, q};
    d[1] = int4{(int)lo, (int)hi, j, 2 * r + (prefixed ? 1 : 0)};
    d[2] = int4{held0 + j, 0, 0, 0};
  }
}

// The tiles of a request read the same keys: with their costs taken up to a multiple of the
// run length, they are cut at the same tokens, the workgroups that read a token do it
// at about the same time, and it comes from memory once (6 requests of 96 .. 256 columns
// on 9000 .. 33000 tokens, 8 heads of 128 in fp16: 156 us, 180 without, at that step).  That costs each such tile half a run of
// idle workgroups, so it is done where they are at most a quarter of the runs.

// Finds the runs run_of(wave) of the cost (each wave gets its own); false for a wave whose
// run is empty.  The first kDescWgs workgroups also write the row descriptors, a share
// of the requests each.  Every wave of the workgroup calls it.
constexpr int kDescWgs = 16;
template <int DT, int D, class F>
PARROT_DEV bool find_run(const TreeArgs& a, int* scratch, int wg, F run_of, OwnRun* o) {
  const int tid = threadIdx.x;
  OwnCost c;
  int pad = 0;
  auto cost_of = [&](int r) {
    if (r >= a.R) return 0;
    c = own_cost<DT, D>(a, r);
    return c.tiles * tile_cost(c.units, c.tiles, pad);
  };
  int total = 0, shared = 0, cost = 0, incl = 0;  // shared: tiles of requests that have several
  auto sum_up = [&] {
    total = 0;
    for (int b = 0; b < a.R; b += 256) {
      int sum;
      cost = cost_of(b + tid);
      incl = scan256(cost, scratch, &sum);
      total += sum;
      if (a.tiles > 1 && pad == 0) {
        scan256(cost > 0 && c.tiles > 1 ? c.tiles : 0, scratch, &sum);
        shared += sum;
      }
    }
  };
  sum_up();
  int q = max(a.min_run, (total + a.runs - 1) / a.runs);
  if (shared > 0 && shared <= a.runs / 4) {       // (at most `shared` runs more than the cost fills)
    pad = q = max(a.min_run, (total + a.runs - shared - 1) / (a.runs - shared));
    sum_up();
  }
  if (tid < 4) scratch[8 + 2 * tid] = -1;
  __syncthreads();
  const bool writes = wg < kDescWgs;
  bool all = false;                               // every wave's run was found or is empty
  for (int b = 0, before = 0, held = 0; b < a.R && (!all || writes); b += 256) {
    int sum = total;
    if (a.R > 256) {                              // (few requests: the first pass stands)
      cost = cost_of(b + tid);
      incl = before + scan256(cost, scratch, &sum);
    }
    if (writes) {
      int rows = 0, held0 = 0;
      if (a.seg_p > 0) {                          // rows with prefixes before the request's
        int here;
        rows = b + tid < a.R && has_prefixes(a, a.gid[b + tid]) ? c.count : 0;
        held0 = held + scan256(rows, scratch, &here) - rows;
        held += here;
      }
      if (b + tid < a.R && cost > 0 && tid % min(kDescWgs, a.own_wgs) == wg)
        write_desc<DT, D>(a, b + tid, c, incl - cost, held0, q, pad);
    }
    all = true;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int u0 = run_of(w) * q;
      if (incl - cost <= u0 && u0 < incl) { scratch[8 + 2 * w] = b + tid; scratch[9 + 2 * w] = incl - cost; }
      all = all && (u0 >= total || u0 < before + sum);
    }
    before += sum;
  }
  __syncthreads();
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  o->q = q;
  o->pad = pad;
  o->u0 = run_of(wave) * q;
  o->u1 = min(total, o->u0 + q);
  o->r = __builtin_amdgcn_readfirstlane(scratch[8 + 2 * wave]);
  o->start = __builtin_amdgcn_readfirstlane(scratch[9 + 2 * wave]);
  o->tile = 0;
  return o->r >= 0 && o->u0 < total;
}

// The next piece of an own run; false when the run is done.
template <int DT, int D>
PARROT_DEV bool next_own(const TreeArgs& a, tree_detail::Lds<DT>& lds, int run, OwnRun* o, TreePiece* pc) {
  constexpr int COLS = tree_detail::kCols<DT>, UNIT = tree_unit(DT, D);
  while (o->r < a.R && o->start < o->u1) {
    const int S = clampi(ld_uniform(a.slen + o->r), 0, a.max_s);
    const int g = ld_uniform(a.gid + o->r);
    const RowSpan rw = row_span(a.qoff, o->r, a.T, min(S, a.max_q));
    const int tiles = (rw.count * a.G + COLS - 1) / COLS, units = (S + UNIT - 1) / UNIT;
    if (o->tile >= tiles) { ++o->r; o->tile = 0; continue; }
    const int s0 = o->start + kTreeSetup;         // cost of the first unit
    const int st0 = max(o->u0 - s0, 0), st1 = min(o->u1 - s0, units);
    const int r = o->r, t = o->tile++;
    o->start += tile_cost(units, tiles, o->pad);
    if (st1 <= st0) continue;
    const bool prefixed = a.seg_p > 0 && g >= 0 && g < a.NG;
    const int base = S - rw.count;
    pc->rg.pk = a.sk; pc->rg.pv = a.sv; pc->rg.tbl = a.stab + (long)r * a.sstride; pc->rg.npool = a.nsblk;
    pc->rg.t0 = st0 * UNIT; pc->rg.t1 = min(S, st1 * UNIT);
    pc->rg.mask0 = base & ~31; pc->rg.base = base; pc->rg.end = S;
    pc->rg.once = tiles == 1;
    pc->col0 = t * COLS;
    pc->ncols = min(COLS, rw.count * a.G - pc->col0);
    pc->row0 = pc->col0 / a.G;
    pc->slot = !prefixed && st0 == 0 && st1 == units ? -1 : run + r * a.tiles + t;
    __syncthreads();                              // the last piece is done with the LDS
    if (threadIdx.x < COLS) lds.rows[threadIdx.x] = min(rw.first + pc->row0 + (int)threadIdx.x, a.T - 1);
    if (pc->rg.t1 > pc->rg.mask0) build_masks<DT, D>(a, lds, rw, base, pc->col0, pc->ncols);
    __syncthreads();
    return true;
  }
  return false;
}

// The piece of prefix workgroup wg; false if there is none.
template <int DT, int D>
PARROT_DEV bool prefix_piece(const TreeArgs& a, tree_detail::Lds<DT>& lds, int wg, TreePiece* pc) {
  constexpr int COLS = tree_detail::kCols<DT>;
  // (group, chunk, head) items; their column tiles are 8 workgroups apart, on one XCD
  const int tile = wg / 8 % a.tiles_p;
  int idx = wg / (8 * a.tiles_p) * 8 + wg % 8;
  if (idx >= a.NG * a.seg_p * a.H) return false;
  pc->h = idx % a.H; idx /= a.H;
  const int c = idx % a.seg_p, g = idx / a.seg_p;
  const int P = clampi(ld_uniform(a.plen + g), 0, a.max_p);
  const int t0 = c * a.cp;
  if (t0 >= P) return false;
  int lvl = 0;                                            // ancestors of g (< depth)
  if (a.parents)
    for (int x = ld_uniform(a.parents + g); x >= 0 && x < a.NG && lvl < a.depth - 1; x = ld_uniform(a.parents + x)) ++lvl;
  // rows [row0, row0 + COLS] of the stacked list hold this tile's columns
  pc->col0 = tile * COLS;
  pc->row0 = pc->col0 / a.G;
  constexpr int MOST = COLS + 1;
  const int row0 = pc->row0;
  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x;
    int base = 0, held = 0;                               // rows of the list, rows with prefixes
    for (int b = 0; b < a.R && base < row0 + MOST; b += kWave) {
      const int r = b + lane;
      bool reads = false, any = false;
      OwnCost oc;
      oc.count = 0; oc.first = 0;
      if (r < a.R) {
        int x = a.gid[r];
        oc = own_cost<DT, D>(a, r);
        any = has_prefixes(a, x);
        for (int d = 0; d < a.depth && x >= 0 && x < a.NG; ++d) {
          if (x == g) { reads = true; break; }
          x = a.parents ? a.parents[x] : -1;
        }
      }
      const int n = reads ? oc.count : 0, m = any ? oc.count : 0;
      int incl = n, among = m;
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) {
        const int v = __shfl_up(incl, d), u = __shfl_up(among, d);
        if (lane >= d) { incl += v; among += u; }
      }
      const int first = base + incl - n, held0 = held + among - m;
      for (int x = max(first, row0), e = min(first + n, row0 + MOST); x < e; ++x) {
        lds.rows[x - row0] = oc.first + x - first;
        lds.held[x - row0] = clampi(held0 + x - first, 0, a.held - 1);
      }
      base += __shfl(incl, kWave - 1);
      held += __shfl(among, kWave - 1);
    }
    if (lane == 0) lds.rows[MOST] = base;
  }
  __syncthreads();
  pc->ncols = __builtin_amdgcn_readfirstlane(min(COLS, lds.rows[MOST] * a.G - pc->col0));
  if (pc->ncols <= 0) return false;
  pc->rg.pk = a.pk; pc->rg.pv = a.pv; pc->rg.tbl = a.ptab + (long)g * a.pstride; pc->rg.npool = a.npblk;
  pc->rg.t0 = t0; pc->rg.t1 = min(P, t0 + a.cp);
  pc->rg.mask0 = 0x40000000; pc->rg.base = pc->rg.end = pc->rg.t1;
  pc->slot = lvl * a.seg_p + c;
  return true;
}

// Own role by waves (requests of at most kStreamCols columns): wave w of workgroup wg
// streams run (4 wg + w) / H of cache head (4 wg + w) % H, so the waves of a workgroup
// read adjacent heads of the same blocks.  No barrier once the runs are found.
template <int DT, int D, int NS>
PARROT_DEV void stream_role(const TreeArgs& a, char* lds, int wg) {
  constexpr int UNIT = tree_unit(DT, D);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int run = (4 * wg + wave) / a.H, h = (4 * wg + wave) % a.H, HQ = a.H * a.G;
  OwnRun o;
  if (!find_run<DT, D>(a, reinterpret_cast<int*>(lds), wg, [&](int w) { return (4 * wg + w) / a.H; }, &o)) {
    __syncthreads();                              // (the others wait below)
    return;
  }
  __syncthreads();                                // the scratch becomes value rows
  TreeStream<DT, D, NS> st(lds + wave * kStreamLds, a.H, h, a.scale_log2);
  for (int start = o.start; o.r < a.R && start < o.u1; ++o.r) {
    const int r = o.r;
    const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
    const int g = ld_uniform(a.gid + r);
    const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
    if (rw.count == 0) continue;
    const int units = (S + UNIT - 1) / UNIT, s0 = start + kTreeSetup;
    const int st0 = max(o.u0 - s0, 0), st1 = min(o.u1 - s0, units);
    start += units + kTreeSetup;
    if (st1 <= st0) continue;
    const bool prefixed = a.seg_p > 0 && g >= 0 && g < a.NG;
    const int base = S - rw.count, ncols = min(rw.count * a.G, 16 * NS);
    TreeRange rg;
    rg.pk = a.sk; rg.pv = a.sv; rg.tbl = a.stab + (long)r * a.sstride; rg.npool = a.nsblk;
    rg.t0 = st0 * UNIT; rg.t1 = min(S, st1 * UNIT);
    rg.mask0 = base & ~31; rg.base = base; rg.end = S;
    auto row_of = [&](int col) {
      const int row = col / a.G;
      return (size_t)(rw.first + row) * HQ + h * a.G + (col - row * a.G);
    };
    st.template load_queries<true>(a.q, ncols, row_of);
    if (rg.t1 > rg.mask0) st.build_masks(a.tree, rw, base, a.G);
    st.run(rg);
    if (!prefixed && st0 == 0 && st1 == units) write_output<DT, D, NS>(a, st, ncols, row_of);
    else write_partial<DT, D, NS>(a, st, ncols, [&](int col) { return piece_slot(a, h, run + r) + col; });
  }
}

// SETS 0: own tokens by tiles, else by waves of that many column sets.
template <int DT, int D, int SETS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SETS > 0 ? 2 : 3)))
void k_tree_partials(TreeArgs a) {
  __shared__ __attribute__((aligned(1024))) tree_detail::Lds<DT> lds;
  static_assert(sizeof(lds) >= 4 * kStreamLds, "the waves' value rows fit");
  // (all prefix workgroups, a.first of them, come before those of the own tokens, or none)
  const int at = (int)blockIdx.x - a.first;
  const bool own = at >= 0 && at < a.own_wgs;
  const int wg = own ? at : at < 0 ? (int)blockIdx.x : at - a.own_wgs;
  if constexpr (SETS > 0) {
    if (own) {
      stream_role<DT, D, SETS>(a, &lds.ring[0][0], wg);
      return;
    }
  }
  const int run = wg / a.H, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  OwnRun o;
  TreePiece pc;
  bool more;
  if (SETS == 0 && own) {
    pc.h = wg % a.H;
    more = find_run<DT, D>(a, lds.tbl, wg, [&](int) { return run; }, &o) && next_own<DT, D>(a, lds, run, &o, &pc);
  } else {
    more = prefix_piece<DT, D>(a, lds, wg, &pc);
  }
  while (more) {                                          // one place for both roles' tiles
    if (tree_detail::kSets<DT> == 2 && (wave + 4) * 16 < pc.ncols)
      tree_piece<DT, D, tree_detail::kSets<DT>>(a, lds, pc, SETS == 0 && own);
    else
      tree_piece<DT, D, 1>(a, lds, pc, SETS == 0 && own);
    more = SETS == 0 && own && next_own<DT, D>(a, lds, run, &o, &pc);
  }
}

// One launch for a small call of at most 16 columns: kSmallWaves waves share the keys of
// one request and cache head (the chain's prefixes, then the own tokens: a contiguous
// share of their units each) and meet in LDS.  Bound by latency, 2.4 us a step of 16 KiB
// (fp32: 4): one request of 4 rows on 300, 2000 tokens takes 9.6, 26.8 us at 32 16-bit
// heads of 128 (the tile: 11.6, 41), at fp32 17.8 us on 300 (32).  Rows of 128 bytes, 64
// tokens a step, leave most waves idle: the tile takes them (8 requests of 4 rows on 1000
// tokens, 32 heads of 64: 17.6 us, 27 here), and 17 to 32 columns, whose waves meet for longer than they
// read (32 requests of 20 rows on 300 tokens, 32 heads of 128: 42.6 us, 55.8 here).
constexpr int kSmallWaves = 8;
template <int DT, int D>
__global__ __launch_bounds__(kSmallWaves * 64) void k_tree_small(TreeArgs a) {
  using E = Elem<DT>;
  constexpr int UNIT = tree_unit(DT, D), NW = kSmallWaves, COLS = 16, STRIDE = D + 4;   // (rows off the same banks)
  constexpr int O_B = NW * COLS * STRIDE * 4;
  __shared__ __attribute__((aligned(1024))) char lds[O_B > NW * kStreamLds ? O_B : NW * kStreamLds];
  __shared__ float s_m[NW][COLS], s_t[NW][COLS], s_w[NW][COLS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x / a.H, h = blockIdx.x % a.H, HQ = a.H * a.G;
  const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
  int g = ld_uniform(a.gid + r);
  const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
  const int ncols = min(rw.count * a.G, COLS), base = S - rw.count;
  if (ncols == 0) return;
  TreeStream<DT, D, 1> st(lds + wave * kStreamLds, a.H, h, a.scale_log2);
  auto row_of = [&](int col) {
    const int row = col / a.G;
    return (size_t)(rw.first + row) * HQ + h * a.G + (col - row * a.G);
  };
  st.template load_queries<true>(a.q, ncols, row_of);
  st.build_masks(a.tree, rw, base, a.G);
  // lengths of the chain's prefixes, innermost first, then the own tokens
  int grp[kMaxDepth], len[kMaxDepth + 1], total = 0;
#pragma unroll
  for (int l = 0; l < kMaxDepth; ++l) {
    grp[l] = 0; len[l] = 0;
    if (l < a.depth && g >= 0 && g < a.NG) {
      grp[l] = g;
      len[l] = clampi(ld_uniform(a.plen + g), 0, a.max_p);
      g = a.parents ? ld_uniform(a.parents + g) : -1;
    } else {
      g = -1;
    }
    total += (len[l] + UNIT - 1) / UNIT;
  }
  len[kMaxDepth] = S;
  total += (S + UNIT - 1) / UNIT;
  const int u0 = total * wave / NW, u1 = total * (wave + 1) / NW;
  int at = 0;
#pragma unroll 1
  for (int l = 0; l <= kMaxDepth; ++l) {
    int n = len[kMaxDepth], gl = 0;
#pragma unroll
    for (int x = 0; x < kMaxDepth; ++x)
      if (x == l) { n = len[x]; gl = grp[x]; }
    const bool pre = l < kMaxDepth;
    const int units = (n + UNIT - 1) / UNIT;
    TreeRange rg;
    rg.pk = pre ? a.pk : a.sk;
    rg.pv = pre ? a.pv : a.sv;
    rg.tbl = pre ? a.ptab + (long)gl * a.pstride : a.stab + (long)r * a.sstride;
    rg.npool = pre ? a.npblk : a.nsblk;
    rg.t0 = max(u0 - at, 0) * UNIT;
    rg.t1 = min(n, (u1 - at) * UNIT);
    rg.mask0 = pre ? 0x40000000 : base & ~31;
    rg.base = pre ? rg.t1 : base;
    rg.end = pre ? rg.t1 : S;
    at += units;
    if (rg.t0 < rg.t1) st.run(rg);
  }
  // the waves' results meet in LDS
  __syncthreads();
  float* so = reinterpret_cast<float*>(lds);
  st.finish([&](int c, int col, float lw, float, float lt) {
    float* dst = so + ((size_t)wave * COLS + col) * STRIDE + 4 * (st.lane >> 4);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) *reinterpret_cast<f32x4*>(dst + dt * 16) = st.o[c][dt];
    if (st.lane < 16) { s_m[wave][col] = st.mref[c]; s_t[wave][col] = lt; s_w[wave][col] = lw; }
  });
  __syncthreads();
  constexpr int EPT = 4;                                  // elements per thread
  for (int x = threadIdx.x; x < ncols * (D / EPT); x += NW * 64) {
    const int col = x / (D / EPT), d = x % (D / EPT) * EPT;
    float mx = s_m[0][col];
#pragma unroll
    for (int w = 1; w < NW; ++w) mx = fmaxf(mx, s_m[w][col]);
    float tot = 0.f, wsum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = fast_exp2(s_m[w][col] - mx);
      tot = __builtin_fmaf(f, s_t[w][col], tot);
      wsum = __builtin_fmaf(f, s_w[w][col], wsum);
      acc += f * *reinterpret_cast<const f32x4*>(so + ((size_t)w * COLS + col) * STRIDE + d);
    }
    const size_t row = row_of(col);
    char* dst = (char*)a.out + (row * D + d) * E::kBytes;
    const f32x4 v = acc * (1.f / wsum);
    if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(dst) = v;
    else store4<DT>(dst, v);
    if (d == 0) a.lse[row] = tot == 0.f ? __builtin_nanf("") : (mx + fast_log2(tot)) * kLn2;   // (as write_output)
  }
}

// Join of the partial results of a row's query heads.  With base-2 log-sum-exps l_i and
// normalised outputs o_i of disjoint key sets, l = log2 sum 2^{l_i}, o = sum 2^{l_i - l} o_i.
// D / 4 lanes hold a head (16 bytes a lane), so a wave takes two or four heads of a
// row; lane i of them holds the weight of partial i.  Bound by the round trips of
// descriptor, log-sum-exps and outputs, and by the partial results' bytes.
template <int DT, int D>
__global__ __launch_bounds__(256) void k_tree_join(TreeArgs a) {
  constexpr int GW = D / 4, HPW = kWave / GW;             // lanes per head, heads per wave
  constexpr int U = 4;                                    // partial results loaded together
  const int lane = threadIdx.x & 63;
  const int HQ = a.H * a.G;
  const unsigned per_row = (HQ + HPW - 1) / HPW;          // (T * HQ is below 2^31)
  const unsigned w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = (int)(w / per_row);
  if (t >= a.T) return;
  const int hq = (int)(w - t * per_row) * HPW + lane / GW, i0 = lane % GW;
  const int* d = a.desc + (size_t)t * kTreeDesc;
  const int first = ld_uniform(d), between = ld_uniform(d + 1), units = ld_uniform(d + 2), q = max(1, ld_uniform(d + 3));
  const unsigned lo = (unsigned)ld_uniform(d + 4), hi = (unsigned)ld_uniform(d + 5);
  const int j = ld_uniform(d + 6), of = ld_uniform(d + 7), prefixed = of & 1;
  const int held = clampi(ld_uniform(d + 8), 0, max(a.held - 1, 0));
  if (t >= ld_uniform(a.qoff + a.R)) return;              // padding (its descriptor holds nothing)
  const int x = j * a.G + hq % a.G, tile = x / tree_detail::kCols<DT>;
  const int s0 = first + tile * between;
  const int pieces = (s0 + units - 1) / q - s0 / q + 1;
  const bool live = hq < HQ && !(prefixed == 0 && pieces == 1);   // one piece: it wrote the output
  // the row's first own piece and its column there (clamped as the slots are)
  const int piece = clampi(s0 / q + (of >> 1) * a.tiles + tile, 0, a.pieces - 1);
  const int col = clampi(x - tile * tree_detail::kCols<DT>, 0, a.piece_cols - 1);
  const TreeSlots slots = tree_slots(lo, hi, min(pieces, a.pieces - piece), a.seg_p, a.seg_pre, a.seg);
  const int n = live ? slots.n : 0;
  int most = n;
#pragma unroll
  for (int m = GW; m < kWave; m <<= 1) most = max(most, __shfl_xor(most, m));
  most = __builtin_amdgcn_readfirstlane(most);
  const size_t at = (size_t)t * HQ + min(hq, HQ - 1);
  const size_t pre = ((size_t)held * HQ + min(hq, HQ - 1)) * a.seg_pre, own = piece_slot(a, min(hq, HQ - 1) / a.G, piece) + col;
  const float* l_pre = a.lse_part + pre;
  const float* l_own = a.lse_part + own;
  const float* o_pre = a.o_part + pre * D + i0 * 4;
  const float* o_own = a.o_part + own * D + i0 * 4;
  auto lse_of = [&](int i) {                              // of partial i
    const int sl = slots.slot(i);
    return sl < a.seg_pre ? l_pre[sl] : l_own[(sl - a.seg_pre) * a.piece_cols];
  };
  auto out_of = [&](int i) {
    const int sl = slots.slot(i);
    return sl < a.seg_pre ? o_pre + sl * D : o_own + (sl - a.seg_pre) * a.piece_cols * D;
  };
  // the lane's first log-sum-exp, and the first outputs beside it
  const float l0 = i0 < n ? lse_of(i0) : -INFINITY;
  f32x4 v[U];
  auto load = [&](int i) {                                // partials i .. i + U - 1, those that exist
#pragma unroll
    for (int u = 0; u < U; ++u) {
      v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (i + u < n) v[u] = *reinterpret_cast<const f32x4*>(out_of(i + u));
    }
  };
  load(0);
  float mx = l0;
#pragma unroll 1
  for (int i = i0 + GW; i < n; i += GW) mx = fmaxf(mx, lse_of(i));
  mx = fmaxf(mx, dpp_f<kDppXor1>(mx));
  mx = fmaxf(mx, dpp_f<kDppXor2>(mx));
  mx = fmaxf(mx, dpp_f<kDppHalfMirror>(mx));
  mx = fmaxf(mx, dpp_f<kDppMirror>(mx));
  if constexpr (GW == 32) mx = max_xor16(mx);
  float tot = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int b = 0; b < most; b += GW) {
    // (no guard on mx: logits that are all -inf give NaN)
    const float wl = b == 0 ? l0 : b + i0 < n ? lse_of(b + i0) : -INFINITY;
    const float wt = b + i0 < n ? fast_exp2(wl - mx) : 0.f;
    tot += wt;
    const int end = min(GW, most - b);
#pragma unroll 1
    for (int i = 0; i < end; i += U) {
      if (b + i > 0) load(b + i);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float wi = __shfl(wt, (lane & ~(GW - 1)) + min(i + u, GW - 1));
        acc += (b + i + u < n ? wi : 0.f) * v[u];
      }
    }
  }
  tot = group_sum<GW>(tot);
  if (!live) return;
  char* dst = (char*)a.out + (at * D + i0 * 4) * Elem<DT>::kBytes;
  const f32x4 res = acc * (1.f / tot);
  if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(dst) = res;
  else store4<DT>(dst, res);
  if (i0 == 0) a.lse[at] = (mx + fast_log2(tot)) * kLn2;
}

template <int DT, int D>
static void launch_tree_t(const TreeArgs& a, bool small, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if constexpr (tree_small_rows(DT, D)) {
    if (small) {
      hipExtLaunchKernelGGL((k_tree_small<DT, D>), dim3((unsigned)((long)a.R * a.H)), dim3(kSmallWaves * 64), 0, s, e0, e1, 0, a);
      return;
    }
  }
  const long groups = ((long)a.R * a.H + 7) / 8;
  hipExtLaunchKernelGGL((k_tree_decode<DT, D>), dim3((unsigned)(groups * 8 * a.tiles)), dim3(256), 0, s, e0, e1, 0, a);
}
template <int DT, int D>
static void launch_partials_t(const TreeArgs& a, int, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const dim3 grid((unsigned)((long)a.own_wgs + a.n_pre));
  if (a.sets == 0) hipExtLaunchKernelGGL((k_tree_partials<DT, D, 0>), grid, dim3(256), 0, s, e0, e1, 0, a);
  else if (a.sets == 1) hipExtLaunchKernelGGL((k_tree_partials<DT, D, 1>), grid, dim3(256), 0, s, e0, e1, 0, a);
  else if constexpr (DT != kF32) hipExtLaunchKernelGGL((k_tree_partials<DT, D, 2>), grid, dim3(256), 0, s, e0, e1, 0, a);
}
template <int DT, int D>
static void launch_join_t(const TreeArgs& a, int, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const int hpw = kWave / (D / 4), per_row = (a.H * a.G + hpw - 1) / hpw;
  hipExtLaunchKernelGGL((k_tree_join<DT, D>), dim3((unsigned)(((long)a.T * per_row + 3) / 4)), dim3(256), 0, s, e0, e1, 0, a);
}

#define PARROT_TREE_LAUNCH(NAME, X)                                       \
  switch (dtype * 1000 + D) {                                                 \
    case kF32 * 1000 + 64: NAME<kF32, 64>(a, X, s, e0, e1); break;        \
    case kF32 * 1000 + 128: NAME<kF32, 128>(a, X, s, e0, e1); break;      \
    case kF16 * 1000 + 64: NAME<kF16, 64>(a, X, s, e0, e1); break;        \
    case kF16 * 1000 + 128: NAME<kF16, 128>(a, X, s, e0, e1); break;      \
    case kBF16 * 1000 + 64: NAME<kBF16, 64>(a, X, s, e0, e1); break;      \
    case kBF16 * 1000 + 128: NAME<kBF16, 128>(a, X, s, e0, e1); break;    \
    default: return hipErrorInvalidValue;                                     \
  }                                                                           \
  return hipGetLastError()

// What every launch needs; sets > 0 promises that a request's columns fit them.
static bool tree_args_ok(const TreeArgs& a) {
  return a.T >= 1 && a.R >= 1 && a.H >= 1 && a.G >= 1 && a.max_q >= 1 && a.max_q <= kTreeRows && a.sstride >= 1 &&
         a.nsblk >= 1 && a.depth <= kMaxDepth && (a.NG == 0 || (a.npblk >= 1 && a.pstride >= 1)) && a.sets >= 0 &&
         a.sets <= 2 && (a.sets == 0 || (long)a.max_q * a.G <= 16 * a.sets);
}

hipError_t launch_tree(const TreeArgs& a, bool small, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (!tree_args_ok(a) || a.tiles < 1 || (long)a.tiles * tree_cols(dtype) < (long)a.max_q * a.G ||
      ((long)a.R * a.H + 7) / 8 * 8 * a.tiles * kSmallWaves * 64 > 0xffffffffL ||
      (small && (a.sets != 1 || !tree_small_rows(dtype, D))))
    return hipErrorInvalidValue;
  PARROT_TREE_LAUNCH(launch_tree_t, small);
}

hipError_t launch_tree_partials(const TreeArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const long pre = a.n_pre > 0 ? ((long)a.NG * a.seg_p * a.H + 7) / 8 * 8 * a.tiles_p : 0;
  if (!tree_args_ok(a) || (a.sets == 2 && dtype == kF32) || a.runs < 1 || a.min_run < 1 || a.own_wgs < 1 ||
      (long)a.own_wgs * (a.sets ? 4 : 1) < (long)a.runs * a.H || !a.o_part || !a.lse_part || !a.desc || a.n_pre != pre ||
      a.pieces < a.runs + a.R * (long)a.tiles || a.piece_cols < (a.sets ? 16 * a.sets : tree_cols(dtype)) || a.own0 != (size_t)a.held * a.H * a.G * a.seg_pre || (a.n_pre > 0 && a.held < 1) || (a.first != 0 && a.first != a.n_pre) ||
      (a.n_pre > 0 && (a.cp < 64 || a.cp % 64 != 0 || a.depth < 1)) || ((long)a.own_wgs + a.n_pre) * 256 > 0xffffffffL)
    return hipErrorInvalidValue;
  PARROT_TREE_LAUNCH(launch_partials_t, 0);
}

hipError_t launch_tree_join(const TreeArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (!tree_args_ok(a) || !a.o_part || !a.lse_part || !a.desc || a.seg < 1 || a.pieces < 1 || a.piece_cols < 1) return hipErrorInvalidValue;
  PARROT_TREE_LAUNCH(launch_join_t, 0);
}

}  // namespace parrot
