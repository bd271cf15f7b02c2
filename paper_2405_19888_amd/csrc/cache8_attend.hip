// Attention over a cache held in 8 bits (cache8_args.h has the format, cache8_tile.h the
// wave's mathematics): plan, partial results and join, or one launch for small calls.
//
// What a step has to read is laid end to end as a list of costs: column tiles of the groups'
// prefixes (the rows of all requests below a group, stacked, so that a prefix is read once per tile
// and not once per request), and column tiles of the requests' own tokens.  A tile costs its units
// of 32 keys and kPieceSetup.  The list is cut into equal runs, a wave of each cache head takes
// one, and where a run ends inside a tile, the pieces are joined.  Nothing depends on how
// ragged the contexts are.  Sequences of many columns have a list of their own, of wide tiles, whose
// runs workgroups take; both lists share the device by their costs.
//
// The list depends on lengths and groups alone, so one plan serves every layer of a step.
#include "cache8_tile.h"

namespace parrot {

// ---------------------------------------------------------------------- plan
// Inclusive sum over the wave: within rows of 16 lanes, then the rows before.
PARROT_DEV int scan_wave(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast 31 into rows 2 and 3
  return x;
}
// Inclusive sum over the workgroup's 1024 threads; *total is the whole sum.
PARROT_DEV int scan1024(int x, int* lds, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = scan_wave(x);
  __syncthreads();
  if (lane == kWave - 1) lds[wave] = x;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const int s = lds[w];
    before += w < wave ? s : 0;
    sum += s;
  }
  *total = sum;
  return x + before;
}

// The rows of request r, and its own tokens.
struct Own8 { int first, count, keys; };
PARROT_DEV Own8 own_rows(const Step8& a, int r) {
  Own8 o;
  o.keys = clampi(a.slen[r], 0, a.max_s);
  const int begin = a.qoff[r], end = a.qoff[r + 1];
  o.first = clampi(begin, 0, a.T);
  const int cap = min(min(o.keys, a.max_q), a.T - o.first);
  const long n = (long)end - begin;
  o.count = (int)(n < 0 ? 0 : n > cap ? cap : n);
  return o;
}

// Rows of each of the wave's requests that read groups, by level of the chain: the wave's rows of each
// group, and each request's place among them.
PARROT_DEV void walk_groups(const Plan8Args& a, const int* req, int* pos, int* count) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, NG = a.st.NG;
  const int r0 = (int)((long)a.st.R * wave / kPlanWaves), r1 = (int)((long)a.st.R * (wave + 1) / kPlanWaves);
  int* mine = count + (long)wave * NG;
  for (int b = r0; b < r1; b += kWave) {
    const int r = b + lane;
    int n = 0, grp = -1, place[kMaxDepth] = {};
    if (r < r1) {
      n = req[(long)r * kReqInts + kReqCount];
      grp = req[(long)r * kReqInts + kReqReads];
    }
#pragma unroll
    for (int l = 0; l < kMaxDepth; ++l) {
      const bool on = n > 0 && grp >= 0;                // (no levels below the call's)
      unsigned long long todo = __ballot(on);
      while (todo) {
        const int leader = __ffsll(todo) - 1;
        const int gl = __builtin_amdgcn_readlane(grp, leader);
        const bool same = on && grp == gl;
        const int incl = scan_wave(same ? n : 0);
        const int base = mine[gl];
        if (same) place[l] = base + incl - n;
        if (lane == leader) mine[gl] = base + __builtin_amdgcn_readlane(incl, kWave - 1);
        todo &= ~__ballot(same);
        __threadfence_block();                          // (a wave's own writes come back in order)
      }
      grp = on && l + 1 < kMaxDepth ? req[(long)r * kReqInts + kReqChain + 2 * (l + 1)] : -1;
    }
    if (r < r1) *reinterpret_cast<int4*>(pos + (long)r * kMaxDepth) = int4{place[0], place[1], place[2], place[3]};
  }
}
static_assert(kMaxDepth == 4, "a request's places are one store");
// The planning wave that counted request r (plans hold fewer than 2^26 requests).
PARROT_DEV int wave_of(int r, int R) { return (int)(((unsigned)r * kPlanWaves + kPlanWaves - 1) / (unsigned)R); }

// One workgroup: a few round trips and scans for a usual batch, 1024 requests, groups or entries a
// round.  What it looks up again and again is in LDS where it fits.
constexpr int kPlanReqs = 1024, kPlanCounts = 4096, kPlanSeqs = 2048;
// Tiles of a sequence of n columns: wide or narrow ones.
PARROT_DEV int2 tiles_of(const Plan8Args& a, long n) {
  return n > a.wide_from ? int2{(int)((n + a.wide_cols - 1) / a.wide_cols), 0} : int2{0, (int)((n + a.cols - 1) / a.cols)};
}
__global__ __launch_bounds__(1024) void k_cache8_plan(Plan8Args a) {
  __shared__ int lds[kPlanWaves + 2];
  __shared__ __attribute__((aligned(16))) int l_req[kPlanReqs * kReqInts];
  __shared__ int l_count[kPlanCounts], l_seq[2 * kPlanSeqs], l_cost[kPlanSeqs], l_slot[kPlanSeqs];
  const int tid = threadIdx.x;
  const Step8& st = a.st;
  int* ent = a.plan + a.at.entry;
  int* rows = a.plan + a.at.row;
  int* list = a.plan + a.at.list;
  int* pos = a.plan + a.at.pos;
  const int nseq = st.NG + st.R;
  int* const g_req = a.plan + a.at.req;
  int* req = st.R <= kPlanReqs ? l_req : g_req;
  int* count = (long)(kPlanWaves + 1) * st.NG + 1 <= kPlanCounts ? l_count : a.plan + a.at.count;
  // first entries of each sequence: wide ones, and narrow ones counted from the first of them
  int* seq = nseq < kPlanSeqs ? l_seq : a.plan + a.at.seq;
  int* seqn = seq + nseq;
  int* off = count + (long)kPlanWaves * st.NG;          // first place of each group's rows

  // the requests
  for (int r = tid; r < st.R; r += 1024) {
    const Own8 o = own_rows(st, r);
    int v[kReqInts] = {o.first, o.count, o.keys, -1, -1, 0, -1, 0, -1, 0, -1, 0};
    int grp = st.gid[r];
    const bool chained = (long)o.count * st.G >= a.wide_cols;
#pragma unroll
    for (int l = 0; l < kMaxDepth; ++l)
      if (l < st.depth && grp >= 0 && grp < st.NG) {
        v[kReqChain + 2 * l] = grp;
        v[kReqChain + 2 * l + 1] = clampi(st.plen[grp], 0, st.max_p);
        if (l == 0 && !chained) v[kReqReads] = grp;
        grp = st.parents ? st.parents[grp] : -1;
      } else {
        grp = -1;
      }
    // (the attention reads the requests from the plan)
#pragma unroll
    for (int i = 0; i < kReqInts; i += 4) {
      *reinterpret_cast<int4*>(g_req + (long)r * kReqInts + i) = int4{v[i], v[i + 1], v[i + 2], v[i + 3]};
      if (req != g_req) *reinterpret_cast<int4*>(req + r * kReqInts + i) = int4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    }
    const int2 tiles = tiles_of(a, (long)o.count * st.G);
    seq[st.NG + r] = tiles.x;
    seqn[st.NG + r] = tiles.y;
  }
  if (tid == 0) lds[kPlanWaves] = 0;                    // rows to join
  for (long i = tid; i < (long)kPlanWaves * st.NG; i += 1024) count[i] = 0;
  __syncthreads();
  // rows of each group, and each request's place among them
  if (st.depth > 0) {
    walk_groups(a, req, pos, count);
    __syncthreads();
    int before = 0;
    for (int b = 0; b < st.NG; b += 1024) {
      const int g = b + tid;
      int n = 0;
      if (g < st.NG)
        for (int w = 0; w < kPlanWaves; ++w) {          // counts become places
          const int x = count[(long)w * st.NG + g];
          count[(long)w * st.NG + g] = n;
          n += x;
        }
      int sum;
      const int incl = scan1024(n, lds, &sum);
      if (g < st.NG) {
        off[g] = before + incl - n;
        const int2 tiles = tiles_of(a, clampi(st.plen[g], 0, st.max_p) > 0 ? (long)n * st.G : 0);
        seq[g] = tiles.x;
        seqn[g] = tiles.y;
      }
      before += sum;
    }
    if (tid == 0) off[st.NG] = before;
    __syncthreads();
  }
  // tiles become first entries
  int wide = 0, narrow = 0;
  for (int b = 0; b < nseq; b += 1024) {
    const int i = b + tid;
    const int n = i < nseq ? seq[i] : 0, m = i < nseq ? seqn[i] : 0;
    int sum = 0, summ;
    int incl = 0;
    if (a.wide_from < 0x7fffffff) incl = scan1024(n, lds, &sum);
    const int inclm = scan1024(m, lds, &summ);
    if (i < nseq) {
      seq[i] = wide + incl - n;
      seqn[i] = narrow + inclm - m;
    }
    wide += sum;
    narrow += summ;
  }
  const int entries = min(wide + narrow, a.max_entries);
  int* cost = entries <= kPlanSeqs ? l_cost : a.plan + a.at.cost;
  __syncthreads();

  // the entries, and where each starts in the cost
  int total = 0;
  int e_cost = 0, e_units = 0, e_cols = 0;              // of the thread's entry, if there is one round of them
  bool e_parts = false;
  for (int b = 0; b < entries; b += 1024) {
    const int e = b + tid;
    int c = 0, v[kEntryInts] = {};
    if (e < entries) {
      const bool w = e < wide;
      const int* first = w ? seq : seqn;
      const int cols = w ? a.wide_cols : a.cols, at = w ? e : e - wide;
      int lo = 0, hi = nseq;                            // the last sequence that starts at or before e
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= at) lo = mid; else hi = mid;
      }
      v[kEntCol0] = (at - first[lo]) * cols;
      if (lo < st.NG) {
        const int n = off[lo + 1] - off[lo];
        v[kEntSeq] = ~lo;
        v[kEntCols] = (int)min((long)cols, (long)n * st.G - v[kEntCol0]);
        v[kEntKeys] = v[kEntBase] = clampi(st.plen[lo], 0, st.max_p);
        v[kEntFirst] = off[lo];
        v[kEntUnits] = (v[kEntKeys] + kUnit - 1) / kUnit;
      } else {
        const int* o = req + (long)(lo - st.NG) * kReqInts;
        v[kEntSeq] = lo - st.NG;
        v[kEntCols] = (int)min((long)cols, (long)o[kReqCount] * st.G - v[kEntCol0]);
        const int from = o[kReqKeys] - o[kReqCount];    // row j sees own tokens 0 .. from + j
        v[kEntKeys] = from + (v[kEntCol0] + v[kEntCols] - 1) / st.G + 1;
        v[kEntBase] = from;
        v[kEntFirst] = o[kReqFirst];
        v[kEntUnits] = (v[kEntKeys] + kUnit - 1) / kUnit;
        if (o[kReqReads] < 0 && o[kReqChain] >= 0) {
          v[kEntChained] = 1;
          for (int l = 0; l < kMaxDepth; ++l) v[kEntUnits] += (o[kReqChain + 2 * l + 1] + kUnit - 1) / kUnit;
        }
      }
      c = v[kEntUnits] + kPieceSetup;
    }
    int sum;
    const int incl = scan1024(c, lds, &sum);
    if (e < entries) {
      v[kEntCost] = total + incl - c;
      cost[e] = v[kEntCost];
      e_cost = v[kEntCost];
      e_units = v[kEntUnits];
      e_cols = v[kEntCols];
      e_parts = v[kEntSeq] < 0 || req[(long)v[kEntSeq] * kReqInts + kReqReads] >= 0;
      int4* to = reinterpret_cast<int4*>(ent + (long)e * kEntryInts);
      to[0] = int4{v[0], v[1], v[2], v[3]};
      to[1] = int4{v[4], v[5], v[6], v[7]};
      to[2] = int4{v[8], v[9], v[10], v[11]};
    }
    total += sum;
  }
  __syncthreads();
  // a cache head's workgroups are shared by the two costs: a wide unit comes out of LDS and keeps a
  // workgroup half as long as a narrow one, which streams, keeps a wave (288 requests, 256 of them
  // below 8 prefixes, us for the plan and two layers: 237; as 0.3 of it 294, as long 253)
  const int wcost = wide == 0 ? 0 : wide < entries ? cost[wide] : total;
  const int wwgs = wide == 0 ? 0 : wide == entries ? a.wgs
                 : clampi((int)((2L * a.wgs * wcost + ((long)wcost + total) / 2) / ((long)wcost + total)), 1, a.wgs - 1);
  const int nruns = 4 * (a.wgs - wwgs);
  const int qw = wwgs == 0 ? 1 : max(a.min_run, (int)(((long)wcost + wwgs - 1) / wwgs));
  const int q = nruns == 0 ? 1 : max(a.min_run, (int)(((long)total - wcost + nruns - 1) / nruns));
  // the first entry of each run: the wide role's, then the narrow one's
  for (int run = tid; run < wwgs + nruns; run += 1024) {
    const bool w = run < wwgs;
    const long c0 = w ? (long)run * qw : wcost + (long)(run - wwgs) * q;
    if (c0 >= (w ? wcost : total)) continue;
    int lo = w ? 0 : wide, hi = w ? wide : entries;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cost[mid] <= c0) lo = mid; else hi = mid;
    }
    a.plan[a.at.run + run] = lo;
  }
  // pieces, and the slots of their partial results
  int slots = 0;
  for (int b = 0; b < entries; b += 1024) {
    const int e = b + tid;
    int n = 0, pieces = 0;
    int* v = ent + (long)e * kEntryInts;
    if (e < entries) {                                  // (its own entries)
      if (entries > 1024) {
        e_cost = v[kEntCost];
        e_units = v[kEntUnits];
        e_cols = v[kEntCols];
        e_parts = v[kEntSeq] < 0 || req[(long)v[kEntSeq] * kReqInts + kReqReads] >= 0;
      }
      const int s0 = e_cost + kPieceSetup - (e < wide ? 0 : wcost), len = e < wide ? qw : q;
      pieces = (s0 + e_units - 1) / len - s0 / len + 1;
      n = pieces == 1 && !e_parts ? 0 : pieces * e_cols;
    }
    int sum;
    const int incl = scan1024(n, lds, &sum);
    if (e < entries) {
      const int slot = n == 0 ? -1 : slots + incl - n;
      v[kEntSlot] = slot;
      v[kEntPieces] = pieces;
      if (e < kPlanSeqs) l_slot[e] = slot;
    }
    slots += sum;
  }
  const int* const e_slot = entries <= kPlanSeqs ? l_slot : ent + kEntSlot;
  const int e_step = entries <= kPlanSeqs ? 1 : kEntryInts;
  __syncthreads();
  // the groups' row lists, what the join needs of each row, and the rows that it takes
  const int used = clampi(st.qoff[st.R], 0, st.T);
  for (int t = tid; t < used; t += 1024) {
    int lo = 0, hi = st.R;                              // the last request that starts at or before t
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (req[(long)mid * kReqInts + kReqFirst] <= t) lo = mid; else hi = mid;
    }
    const int* o = req + (long)lo * kReqInts;
    const int j = t - o[kReqFirst];
    if (j < 0 || j >= o[kReqCount]) continue;           // no request holds it
    int v[kRowInts] = {};
    const bool w = (long)o[kReqCount] * st.G > a.wide_from;
    const int first = w ? seq[st.NG + lo] : wide + seqn[st.NG + lo], cols = w ? a.wide_cols : a.cols;
    v[kRowToken] = t;
    v[kRowEntry] = first;
    v[kRowPlace] = j;
    if (o[kReqReads] >= 0)
#pragma unroll
      for (int l = 0; l < kMaxDepth; ++l) {
        const int grp = o[kReqChain + 2 * l];
        if (grp >= 0) {
          const int at = count[(long)wave_of(lo, st.R) * st.NG + grp] + pos[(long)lo * kMaxDepth + l] + j;
          v[kRowGroup + 2 * l + 1] = -1;
          if (o[kReqChain + 2 * l + 1] > 0) {           // (a prefix without tokens has no entries)
            v[kRowGroup + 2 * l] = (long)(off[grp + 1] - off[grp]) * st.G > a.wide_from ? seq[grp] : wide + seqn[grp];
            v[kRowGroup + 2 * l + 1] = at;
            v[kRowLevels] = l + 1;
          }
          list[min((long)off[grp] + at, (long)st.T * st.depth - 1)] = t;
        }
      }
    // (the row's columns are in one or more of its request's tiles)
    bool parts = false;
    for (int e = first + (int)((long)j * st.G / cols); e <= first + (int)(((long)j * st.G + st.G - 1) / cols) && e < entries; ++e)
      parts = parts || e_slot[(long)e * e_step] >= 0;
    if (parts) {                                        // (their order is of no matter: each is joined by itself)
      int4* d = reinterpret_cast<int4*>(rows + (long)min(atomicAdd(&lds[kPlanWaves], 1), st.T - 1) * kRowInts);
      d[0] = int4{v[0], v[1], v[2], v[3]};
      d[1] = int4{v[4], v[5], v[6], v[7]};
      d[2] = int4{v[8], v[9], v[10], v[11]};
    }
  }
  __syncthreads();
  if (tid == 0) {
    *reinterpret_cast<int4*>(a.plan) = int4{entries, wide, lds[kPlanWaves], wcost};
    *reinterpret_cast<int4*>(a.plan + 4) = int4{total, wwgs, qw, q};
  }
}

// ----------------------------------------------------------- partial results
// Keys of one sequence of a call: a request's own tokens, or a group's prefix.
PARROT_DEV Range8 range_of(const Attend8Args& a, bool own, int seq, int keys, int u0, int u1) {
  Range8 rg;
  const Pool8 pool = own ? a.own : a.pre;
  rg.pool.k = alone(pool.k);
  rg.pool.v = alone(pool.v);
  rg.pool.scales = alone(pool.scales);
  rg.tbl = alone(own ? a.stab + (long)seq * a.sstride : a.ptab + (long)seq * a.pstride);
  rg.npool = alone(own ? a.nsblk : a.npblk);
  rg.u0 = u0;
  rg.u1 = u1;
  rg.end = rg.plain = keys;
  return rg;
}

// Output of a column that saw its whole context.  Every row sees itself: no weights mean that each
// logit is -inf.
template <int DT, int D, int NS>
PARROT_DEV void write_column(const Attend8Args& a, const Tile8<DT, D, NS>& tile, int c, long at, float inv, float lse2) {
  const int g = tile.lane >> 4;
  char* dst = (char*)a.out + (at * D + 16 * g) * Elem<DT>::kBytes;
  const float f = lse2 == -INFINITY ? __builtin_nanf("") : inv;
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = tile.four(c, x, i) * f;
      char* to = dst + (64 * x + 4 * i) * Elem<DT>::kBytes;
      if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(to) = v;
      else *reinterpret_cast<uint2*>(to) = uint2{Wide8<DT>::pack(v[0], v[1]), Wide8<DT>::pack(v[2], v[3])};
    }
  if (g == 0) a.lse[at] = lse2 == -INFINITY ? __builtin_nanf("") : lse2 * kLn2;
}

// An entry as the kernel reads it: wave-uniform, every index clamped to what it may address.
struct Entry { int seq, col0, cols, cost, units, slot, keys, base, first, chained; };
PARROT_DEV Entry load_entry(const Attend8Args& a, int e) {
  const int* p = a.plan + a.at.entry + (long)e * kEntryInts;
  Entry v;
  v.seq = ld_uniform(p + kEntSeq);
  v.seq = v.seq >= 0 ? min(v.seq, a.R - 1) : max(v.seq, -max(a.NG, 1));
  v.col0 = max(ld_uniform(p + kEntCol0), 0);
  v.cols = clampi(ld_uniform(p + kEntCols), 0, max(16 * a.sets, a.wide));
  v.cost = ld_uniform(p + kEntCost);
  v.keys = clampi(ld_uniform(p + kEntKeys), 0, v.seq >= 0 ? a.max_s : a.max_p);
  v.units = max(ld_uniform(p + kEntUnits), 0);
  v.slot = ld_uniform(p + kEntSlot);
  v.base = ld_uniform(p + kEntBase);
  v.first = max(ld_uniform(p + kEntFirst), 0);
  v.chained = ld_uniform(p + kEntChained);
  return v;
}

// Units [u0, u1) of an entry, piece number `piece`.  WIDE: a workgroup's waves take 16 * NS columns
// of it each.
template <int DT, int D, int NS, bool WIDE>
PARROT_DEV void attend_piece(const Attend8Args& a, const Entry& e, int h, int u0, int u1, int piece, char* ring) {
  const int HQ = a.H * a.G;
  const bool own = e.seq >= 0;
  const int first_col = WIDE ? (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 16 * NS : 0;
  Tile8<DT, D, NS> tile(a.H, h);
  int at[NS], sees[NS];                                 // the columns' places in [T][HQ], or -1, and own keys
#pragma unroll
  for (int c = 0; c < NS; ++c) {
    const int col = first_col + tile.column(c);
    const int x = e.col0 + col, j = x / a.G;
    at[c] = -1;
    if (col < e.cols) {
      int row = e.first + j;
      if (!own) row = a.plan[a.at.list + min((long)row, (long)a.T * max(a.depth, 1) - 1)];
      at[c] = clampi(row, 0, a.T - 1) * HQ + h * a.G + (x - j * a.G);
    }
    sees[c] = min(e.keys, e.base + j + 1);
  }
  tile.load_queries(a.q, a.flip != 0, [&](int c) { return (long)at[c]; });
  const int cols = min(e.cols - first_col, 16 * NS);    // (below 1: a wave that loads for the others)
  // own keys that every column of the wave sees, and that any does
  const int plain = min(e.keys, e.base + (e.col0 + first_col) / a.G + 1);
  const int most = min(e.keys, e.base + (e.col0 + first_col + cols - 1) / a.G + 1);
  // the chain's prefixes where they come first, then the entry's own keys
  const int* chain = a.plan + a.at.req + (long)(own ? e.seq : 0) * kReqInts + kReqChain;
  int from = 0;                                         // units before the range
#pragma unroll 1
  for (int l = own && e.chained ? 0 : kMaxDepth; l <= kMaxDepth; ++l) {
    const bool pre = l < kMaxDepth;
    const int grp = pre ? clampi(ld_uniform(chain + 2 * l), 0, max(a.NG - 1, 0)) : 0;
    const int keys = pre ? clampi(ld_uniform(chain + 2 * l + 1), 0, a.NG > 0 ? a.max_p : 0) : e.keys;
    const int units = (keys + kUnit - 1) / kUnit;
    const int b = max(u0 - from, 0), f = min(u1 - from, units);
    from += units;
    if (b >= f) continue;
    Range8 rg = range_of(a, own && !pre, pre ? grp : own ? e.seq : ~e.seq, keys, b, f);
    if (own && !pre) rg.plain = plain;
#pragma unroll
    for (int c = 0; c < NS; ++c) tile.lim[c] = own && !pre ? sees[c] : keys;
    if constexpr (WIDE) tile.run_shared(rg, alone(a.scale_log2), ring, cols < 1 ? 0 : own && !pre ? most : keys);
    // (one set alone takes streaming loads; a narrow tile of two sets is its keys' only reader too: 64 requests of
    // eight rows of four query heads on 3000 tokens 108 us with cached loads, 94 with streaming ones)
    else tile.template run<NS == 1>(rg, alone(a.scale_log2));
  }

  const int g = tile.lane >> 4;
  const long slot = e.slot + (long)piece * e.cols;
  const bool direct = e.slot < 0;
  if (!direct && slot + e.cols > a.slots) return;
  tile.finish([&](int c, int col, float inv, float lse2) {
    if (at[c] < 0) return;
    if (direct) {
      write_column(a, tile, c, at[c], inv, lse2);
    } else {
      const long sl = (long)h * a.slots + slot + first_col + col;
      float* dst = a.o_part + sl * D + 16 * g;
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(dst + 64 * x + 4 * i) = tile.four(c, x, i) * inv;
      if (g == 0) a.lse_part[sl] = lse2;
    }
  });
}

// A run of a cost list: entries from `first` on, costs [c0, c1) after `base`.
template <class F>
PARROT_DEV void walk_run(const Attend8Args& a, int first, int end, long base, long c0, long c1, int q, int run, F piece) {
  Entry next = load_entry(a, clampi(first, 0, a.max_entries - 1));
#pragma unroll 1
  for (int e = max(first, 0); e < end; ++e) {
    const Entry v = next;
    const long s0 = v.cost - base + kPieceSetup;
    if (s0 - kPieceSetup >= c1) break;
    next = load_entry(a, min(e + 1, a.max_entries - 1));  // (on its way while this one is worked on)
    const int u0 = (int)max(c0 - s0, 0L), u1 = (int)min(c1 - s0, (long)v.units);
    if (u0 >= u1 || v.cols == 0) continue;
    piece(v, u0, u1, run - (int)(s0 / q));
  }
}

// SETS: column sets of narrow tiles, at most.  WIDE: wide tiles too.
template <int DT, int D, int SETS, bool WIDE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void k_cache8_attend(Attend8Args a) {
  constexpr int WSETS = DT == kF32 ? 1 : 2;
  __shared__ __attribute__((aligned(16))) char ring[WIDE ? Tile8<DT, D, WSETS>::RING * Tile8<DT, D, WSETS>::UNIT_B : 16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int entries = clampi(ld_uniform(a.plan + kHeadEntries), 0, a.max_entries);
  const int wcost = ld_uniform(a.plan + kHeadWideCost), total = ld_uniform(a.plan + kHeadCost);
  const int wwgs = WIDE ? clampi(ld_uniform(a.plan + kHeadWideWgs), 0, a.wgs) : 0;
  if constexpr (WIDE) {
    if ((int)blockIdx.x < wwgs * a.H) {                 // neighbouring runs of a head on one XCD
      const int h = blockIdx.x % a.H, run = blockIdx.x / a.H;
      const int q = max(ld_uniform(a.plan + kHeadWideRun), 1), end = clampi(ld_uniform(a.plan + kHeadWide), 0, entries);
      const long c0 = (long)run * q, c1 = min((long)wcost, c0 + q);
      if (c0 >= wcost) return;
      walk_run(a, ld_uniform(a.plan + a.at.run + run), end, 0, c0, c1, q, run, [&](const Entry& v, int u0, int u1, int piece) {
        attend_piece<DT, D, WSETS, true>(a, v, h, u0, u1, piece, ring);
      });
      return;
    }
  }
  // neighbouring heads of the same blocks
  const int w = ((int)blockIdx.x - wwgs * a.H) * 4 + wave;
  const int h = w % a.H, run = w / a.H;
  const int q = max(ld_uniform(a.plan + kHeadRun), 1);
  const long c0 = (long)run * q, c1 = min((long)total - wcost, c0 + q);
  if (c0 >= (long)total - wcost || run >= 4 * (a.wgs - wwgs)) return;
  walk_run(a, ld_uniform(a.plan + a.at.run + wwgs + run), entries, wcost, c0, c1, q, run,
           [&](const Entry& v, int u0, int u1, int piece) {
    if (SETS > 1 && v.cols > 16) attend_piece<DT, D, SETS, false>(a, v, h, u0, u1, piece, ring);
    else attend_piece<DT, D, 1, false>(a, v, h, u0, u1, piece, ring);
  });
}

// ---------------------------------------------------------------- one launch
// A workgroup per (request, cache head, column tile): its waves share the units of the whole
// context (the chain's prefixes, then the own tokens) and meet in LDS.  For small calls, which
// are bound by latency: no plan, no partial results, one launch.
template <int DT, int D, int NW>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(DT == kF32 ? 2 : 3)))
void k_cache8_direct(Attend8Args a) {
  constexpr int NS = 1, COLS = 16 * NS, STRIDE = D + 4;                   // (rows off the same banks)
  __shared__ __attribute__((aligned(16))) float s_o[NW][COLS][STRIDE];
  __shared__ float s_m[NW][COLS], s_t[NW][COLS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile_no = blockIdx.x % a.tiles, rest = blockIdx.x / a.tiles;
  const int h = rest % a.H, r = rest / a.H, HQ = a.H * a.G;
  const Step8& st = a.st;
  const int S = clampi(ld_uniform(st.slen + r), 0, a.max_s);
  int grp = a.NG > 0 ? ld_uniform(st.gid + r) : -1;
  const RowSpan rw = row_span(st.qoff, r, a.T, min(S, st.max_q));
  const int col0 = tile_no * COLS, ncols = min(COLS, rw.count * a.G - col0);
  if (ncols <= 0) return;
  const int base = S - rw.count;
  const int keys = base + (col0 + ncols - 1) / a.G + 1;   // own tokens that the tile sees
  Tile8<DT, D, NS> tile(a.H, h);
  auto row_of = [&](int col) {
    const int x = col0 + col, j = x / a.G;
    return (long)(rw.first + j) * HQ + h * a.G + (x - j * a.G);
  };
  tile.load_queries(a.q, a.flip != 0, [&](int c) { return tile.column(c) < ncols ? row_of(tile.column(c)) : -1L; });
  // lengths of the chain's prefixes, innermost first
  int id[kMaxDepth], len[kMaxDepth], total = (keys + kUnit - 1) / kUnit;
#pragma unroll
  for (int l = 0; l < kMaxDepth; ++l) {
    const bool on = l < st.depth && grp >= 0 && grp < a.NG;
    id[l] = on ? grp : 0;
    len[l] = on ? clampi(ld_uniform(st.plen + id[l]), 0, a.max_p) : 0;
    grp = on && st.parents ? ld_uniform(st.parents + id[l]) : -1;
    total += (len[l] + kUnit - 1) / kUnit;
  }
  const int u0 = (int)((long)total * wave / NW), u1 = (int)((long)total * (wave + 1) / NW);
  int from = 0;
#pragma unroll 1
  for (int l = 0; l <= kMaxDepth; ++l) {
    int n = keys, gl = r;
#pragma unroll
    for (int x = 0; x < kMaxDepth; ++x)
      if (x == l) { n = len[x]; gl = id[x]; }
    const bool own = l == kMaxDepth;
    const int units = (n + kUnit - 1) / kUnit;
    const int b = max(u0 - from, 0), f = min(u1 - from, units);
    from += units;
    if (b >= f) continue;
    Range8 rg = range_of(a, own, gl, n, b, f);
    if (own) rg.plain = min(n, base + col0 / a.G + 1);
#pragma unroll
    for (int c = 0; c < NS; ++c) tile.lim[c] = own ? min(keys, base + (col0 + tile.column(c)) / a.G + 1) : n;
    tile.template run<false>(rg, alone(a.scale_log2));
  }
  // the waves' results meet in LDS: normalised outputs and log-sum-exps
  tile.finish([&](int c, int col, float inv, float lse2) {
    const int g = tile.lane >> 4;
#pragma unroll
    for (int x = 0; x < D / 64; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(&s_o[wave][col][64 * x + 16 * g + 4 * i]) = tile.four(c, x, i) * inv;
    if (g == 0) s_t[wave][col] = lse2;
  });
  __syncthreads();
  for (int col = threadIdx.x; col < COLS; col += NW * 64) {     // weights of the waves, and the sum
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) mx = fmaxf(mx, s_t[w][col]);
    float sum = 0.f, wt[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      wt[w] = s_t[w][col] == -INFINITY ? 0.f : fast_exp2(s_t[w][col] - mx);
      sum += wt[w];
    }
#pragma unroll
    for (int w = 0; w < NW; ++w) s_m[w][col] = wt[w] / sum;       // (no weights at all: NaN)
    if (col < ncols) a.lse[row_of(col)] = sum == 0.f ? __builtin_nanf("") : (mx + fast_log2(sum)) * kLn2;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < ncols * (D / 4); x += NW * 64) {
    const int col = x / (D / 4), d = x % (D / 4) * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) acc += s_m[w][col] * *reinterpret_cast<const f32x4*>(&s_o[w][col][d]);
    char* dst = (char*)a.out + (row_of(col) * D + d) * Elem<DT>::kBytes;
    if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(dst) = acc;
    else *reinterpret_cast<uint2*>(dst) = uint2{Wide8<DT>::pack(acc[0], acc[1]), Wide8<DT>::pack(acc[2], acc[3])};
  }
}

// ---------------------------------------------------------------------- join
// With base-2 log-sum-exps l_i and normalised outputs o_i of disjoint keys, l = log2 sum 2^l_i
// and o = sum 2^(l_i - l) o_i.  D / 4 lanes hold a query head (16 bytes a lane); GROUPS of them
// share a head's partial results where few heads have many, and meet in LDS.
template <int DT, int D, int GROUPS>
__global__ __launch_bounds__(256) void k_cache8_join(Attend8Args a) {
  constexpr int GW = D / 4, HEADS = 256 / (GW * GROUPS);    // query heads of a workgroup
  constexpr bool MEET = GROUPS > 1;
  __shared__ float s_m[MEET ? GROUPS : 1][HEADS], s_l[MEET ? GROUPS : 1][HEADS];
  __shared__ f32x4 s_o[MEET ? GROUPS : 1][HEADS][GW];
  const int HQ = a.H * a.G, parts = (HQ + HEADS - 1) / HEADS;
  const int wide = ld_uniform(a.plan + kHeadWide);
  const int i0 = threadIdx.x % GW, sub = threadIdx.x / GW, mine = sub % HEADS, grp = sub / HEADS;
  const long work = (long)clampi(ld_uniform(a.plan + kHeadJoins), 0, a.T) * parts;
  for (long w = blockIdx.x; w < work; w += gridDim.x) {
    const int* d = a.plan + a.at.row + (w / parts) * kRowInts;
    const int t = clampi(ld_uniform(d + kRowToken), 0, a.T - 1);
    const int hq = (int)(w % parts) * HEADS + mine;
    const bool live = hq < HQ;
    const int h = min(hq, HQ - 1) / a.G, gq = min(hq, HQ - 1) % a.G;
    const int levels = clampi(ld_uniform(d + kRowLevels), 0, kMaxDepth);
    // own tokens, then the chain's prefixes: slots, columns, pieces and the row's column of each
    int slot[1 + kMaxDepth], nc[1 + kMaxDepth], n[1 + kMaxDepth], col[1 + kMaxDepth];
#pragma unroll
    for (int s = 0; s <= kMaxDepth; ++s) {
      n[s] = 0;
      if (s <= levels) {
        const int place = ld_uniform(d + (s ? kRowGroup + 2 * s - 1 : (int)kRowPlace)), x = place * a.G + gq;
        const int e0 = ld_uniform(d + (s ? kRowGroup + 2 * s - 2 : (int)kRowEntry));
        const int cols = e0 < wide ? max(a.wide, 1) : 16 * a.sets;
        const int* v = a.plan + a.at.entry + (long)clampi(e0 + x / cols, 0, a.max_entries - 1) * kEntryInts;
        slot[s] = v[kEntSlot];
        nc[s] = v[kEntCols];
        n[s] = place < 0 ? 0 : min(v[kEntPieces], 4 * a.wgs);   // (a piece per run at most)
        col[s] = x % cols;
      }
    }
    const bool direct = slot[0] < 0;                    // the piece wrote the output
    float m = -INFINITY, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s <= kMaxDepth; ++s) {
      if (s > levels) break;
      const int pieces = direct ? 0 : n[s];
#pragma unroll 1
      for (int i = grp; i < pieces; i += 4 * GROUPS) {
        float lp[4];
        f32x4 op[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int k = i + u * GROUPS;
          const long at = slot[s] + (long)k * nc[s] + col[s];
          const bool on = k < pieces && at >= 0 && at < a.slots;
          const long sl = (long)h * a.slots + (on ? at : 0);
          lp[u] = -INFINITY;
          if (on) {
            lp[u] = a.lse_part[sl];
            op[u] = *reinterpret_cast<const f32x4*>(a.o_part + sl * D + 4 * i0);
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (lp[u] == -INFINITY) continue;             // no key the row sees
          const float mn = fmaxf(m, lp[u]);
          const float f = fast_exp2(m - mn), wt = fast_exp2(lp[u] - mn);
          // (a logit that is no number, or +inf, makes the sums NaN)
          m = lp[u] != lp[u] ? lp[u] : mn;
          l = l * f + wt;
          acc = acc * f + op[u] * wt;
        }
      }
    }
    if constexpr (MEET) {
      __syncthreads();                                  // (the last row's results have been read)
      s_m[grp][mine] = m;
      s_l[grp][mine] = l;
      s_o[grp][mine][i0] = acc;
      __syncthreads();
      if (grp == 0) {
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) m = fmaxf(m, s_m[k][mine]);
        l = 0.f;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
          const float mk = s_m[k][mine];
          const float wt = mk == -INFINITY ? 0.f : fast_exp2(mk - m);
          l += wt * s_l[k][mine];
          acc += wt * s_o[k][mine][i0];
        }
      }
    }
    if (grp != 0 || !live || direct) continue;
    // (no weights at all: every logit is -inf, as the one piece gives it)
    const float inv = l == 0.f ? __builtin_nanf("") : 1.f / l;
    const f32x4 res = l == 0.f ? f32x4{inv, inv, inv, inv} : acc * inv;
    const size_t at = (size_t)t * HQ + hq;
    char* dst = (char*)a.out + (at * D + 4 * i0) * Elem<DT>::kBytes;
    if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(dst) = res;
    else *reinterpret_cast<uint2*>(dst) = uint2{Wide8<DT>::pack(res[0], res[1]), Wide8<DT>::pack(res[2], res[3])};
    if (i0 == 0) a.lse[at] = l == 0.f ? __builtin_nanf("") : (m + fast_log2(l)) * kLn2;
  }
}

// ------------------------------------------------------------------ launches
hipError_t launch_plan8(const Plan8Args& a, hipStream_t s) {
  if (a.st.T < 1 || a.st.R < 1 || a.st.G < 1 || a.cols < 16 || a.wide_cols < 1 || a.wide_from < 1 || a.wgs < 2 || a.min_run < 1 ||
      a.max_entries < 1 || a.st.depth < 0 || a.st.depth > kMaxDepth || (a.st.NG > 0) != (a.st.depth > 0))
    return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_cache8_plan, dim3(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}

template <int DT, int D>
static hipError_t launch_attend_t(const Attend8Args& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  constexpr int MOST = DT == kF32 ? 1 : 2;
  const long wgs = (long)a.wgs * a.H;
  if (wgs * 256 > 0xffffffffL || a.sets > MOST || (a.wide != 0 && a.wide != wide_cols(DT))) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wgs), wg(256);
  if (a.wide) hipExtLaunchKernelGGL((k_cache8_attend<DT, D, MOST, true>), grid, wg, 0, s, e0, e1, 0, a);
  else if (a.sets == 1) hipExtLaunchKernelGGL((k_cache8_attend<DT, D, 1, false>), grid, wg, 0, s, e0, e1, 0, a);
  else if constexpr (MOST > 1) hipExtLaunchKernelGGL((k_cache8_attend<DT, D, 2, false>), grid, wg, 0, s, e0, e1, 0, a);
  return hipGetLastError();
}
template <int DT, int D>
static hipError_t launch_direct_t(const Attend8Args& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const long wgs = (long)a.R * a.H * a.tiles;
  if (a.tiles < 1 || wgs * 512 > 0xffffffffL) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wgs);
  if (a.waves == 8) hipExtLaunchKernelGGL((k_cache8_direct<DT, D, 8>), grid, dim3(512), 0, s, e0, e1, 0, a);
  else hipExtLaunchKernelGGL((k_cache8_direct<DT, D, 4>), grid, dim3(256), 0, s, e0, e1, 0, a);
  return hipGetLastError();
}
constexpr int kJoinWgs = 2048;           // workgroups of a join: eight a CU
template <int DT, int D>
static hipError_t launch_join_t(const Attend8Args& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  constexpr int MANY = 256 / (D / 4) / 2;
  const long heads = (long)a.T * a.H * a.G;
  if (heads / 2 <= kJoinWgs) {                          // few heads, whose partial results may be many
    hipExtLaunchKernelGGL((k_cache8_join<DT, D, MANY>), dim3((unsigned)((heads + 1) / 2 + a.T)), dim3(256), 0, s, e0, e1, 0, a);
  } else {
    const long wgs = heads / (256 / (D / 4)) + a.T;
    hipExtLaunchKernelGGL((k_cache8_join<DT, D, 1>), dim3((unsigned)(wgs < kJoinWgs ? wgs : kJoinWgs)), dim3(256), 0, s, e0, e1, 0, a);
  }
  return hipGetLastError();
}

#define PARROT_CACHE8_LAUNCH(NAME)                                        \
  switch (dtype * 1000 + D) {                                             \
    case kF32 * 1000 + 64: return NAME<kF32, 64>(a, s, e0, e1);           \
    case kF32 * 1000 + 128: return NAME<kF32, 128>(a, s, e0, e1);         \
    case kF16 * 1000 + 64: return NAME<kF16, 64>(a, s, e0, e1);           \
    case kF16 * 1000 + 128: return NAME<kF16, 128>(a, s, e0, e1);         \
    case kBF16 * 1000 + 64: return NAME<kBF16, 64>(a, s, e0, e1);         \
    case kBF16 * 1000 + 128: return NAME<kBF16, 128>(a, s, e0, e1);       \
  }                                                                       \
  return hipErrorInvalidValue

static bool attend_ok(const Attend8Args& a) {
  return a.T >= 1 && a.R >= 1 && a.H >= 1 && a.G >= 1 && a.sstride >= 1 && a.nsblk >= 1 &&
         (a.NG == 0 || (a.npblk >= 1 && a.pstride >= 1)) && (a.sets == 1 || a.sets == 2);
}
static bool parts_ok(const Attend8Args& a) {
  return attend_ok(a) && a.wgs >= 2 && a.max_entries >= 1 && a.plan && a.o_part && a.lse_part && a.slots >= 1;
}
hipError_t launch_attend8(const Attend8Args& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (!parts_ok(a)) return hipErrorInvalidValue;
  PARROT_CACHE8_LAUNCH(launch_attend_t);
}
hipError_t launch_join8(const Attend8Args& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (!parts_ok(a)) return hipErrorInvalidValue;
  PARROT_CACHE8_LAUNCH(launch_join_t);
}
hipError_t launch_direct8(const Attend8Args& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const Step8& st = a.st;
  if (!attend_ok(a) || !st.qoff || !st.slen || (a.NG > 0 && (!st.gid || !st.plen)) || st.depth > kMaxDepth ||
      (long)a.tiles * 16 < (long)st.max_q * a.G)
    return hipErrorInvalidValue;
  PARROT_CACHE8_LAUNCH(launch_direct_t);
}

}  // namespace parrot
