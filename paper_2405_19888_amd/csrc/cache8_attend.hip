// Attention over a cache held in 8 bits (cache8_args.h has the format, cache8_tile.h the
// wave's mathematics): plan, partial results, join.
//
// What a step has to read is laid end to end as one list of costs: column tiles of the groups'
// prefixes (the rows of all requests below a group, stacked, so that a prefix is read once per tile
// and not once per request), then column tiles of the requests' own tokens.  A tile costs its units
// of 32 keys and kPieceSetup.  The list is cut into equal runs, a wave of each cache head takes
// one, and where a run ends inside a tile, the pieces are joined.  Nothing depends on how
// ragged the contexts are, and no wave waits for another.
//
// The list depends on lengths and groups alone, so one plan serves every layer of a step.
#include "cache8_tile.h"

namespace parrot {

// ---------------------------------------------------------------------- plan
// Inclusive sum over the workgroup's 1024 threads; *total is the whole sum.
PARROT_DEV int scan1024(int x, int* lds, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int v = __shfl_up(x, d);
    if (lane >= d) x += v;
  }
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
PARROT_DEV Own8 own_rows(const Plan8Args& a, int r) {
  Own8 o;
  o.keys = clampi(a.slen[r], 0, a.max_s);
  const int begin = a.qoff[r], end = a.qoff[r + 1];
  o.first = clampi(begin, 0, a.T);
  const int cap = min(min(o.keys, a.max_q), a.T - o.first);
  const long n = (long)end - begin;
  o.count = (int)(n < 0 ? 0 : n > cap ? cap : n);
  return o;
}

// Rows of each of the wave's requests that read groups, by level of the chain: counts of the
// wave's rows per group (assign false), or each request's place in the group's list.
PARROT_DEV void walk_groups(const Plan8Args& a, int* count, bool assign) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r0 = (int)((long)a.R * wave / kPlanWaves), r1 = (int)((long)a.R * (wave + 1) / kPlanWaves);
  int* mine = count + (long)wave * a.NG;
  int* pos = a.plan + a.at.pos;
  for (int b = r0; b < r1; b += kWave) {
    const int r = b + lane;
    int n = 0, grp = -1;
    if (r < r1) {
      n = own_rows(a, r).count;
      grp = a.gid[r];
    }
    for (int l = 0; l < a.depth; ++l) {
      const bool on = n > 0 && grp >= 0 && grp < a.NG;
      unsigned long long todo = __ballot(on);
      if (!todo) break;
      while (todo) {
        const int leader = __ffsll(todo) - 1;
        const int gl = __shfl(grp, leader);
        const bool same = on && grp == gl;
        const unsigned long long all = __ballot(same);
        int incl = same ? n : 0;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
          const int x = __shfl_up(incl, d);
          if (lane >= d) incl += x;
        }
        const int base = mine[gl];
        if (assign && same) pos[(long)r * kMaxDepth + l] = base + incl - n;
        const int sum = __shfl(incl, kWave - 1);
        if (lane == leader) mine[gl] = base + sum;
        todo &= ~all;
        // (a wave's own writes come back in order)
        __threadfence_block();
      }
      grp = on && a.parents ? a.parents[grp] : -1;
    }
  }
}

// One workgroup: a few round trips and scans for a usual batch, 1024 requests, groups or entries a round.
__global__ __launch_bounds__(1024) void k_cache8_plan(Plan8Args a) {
  __shared__ int lds[kPlanWaves];
  const int tid = threadIdx.x;
  int* head = a.plan;
  int* cost = a.plan + a.at.cost;
  int* ent = a.plan + a.at.entry;
  int* rows = a.plan + a.at.row;
  int* list = a.plan + a.at.list;
  int* seq = a.plan + a.at.seq;
  int* count = a.plan + a.at.count;
  int* off = count + (long)kPlanWaves * a.NG;           // first place of each group's rows
  const int* pos = a.plan + a.at.pos;

  // rows of each group, and each request's place among them
  if (a.depth > 0) {
    for (long i = tid; i < (long)kPlanWaves * a.NG; i += 1024) count[i] = 0;
    __syncthreads();
    walk_groups(a, count, false);
    __syncthreads();
    int before = 0;
    for (int b = 0; b < a.NG; b += 1024) {
      const int g = b + tid;
      int n = 0;
      if (g < a.NG)
        for (int w = 0; w < kPlanWaves; ++w) {          // counts become places
          const int x = count[(long)w * a.NG + g];
          count[(long)w * a.NG + g] = n;
          n += x;
        }
      int sum;
      const int incl = scan1024(n, lds, &sum);
      if (g < a.NG) {
        off[g] = before + incl - n;
        // tiles of the group
        seq[g] = clampi(a.plen[g], 0, a.max_p) > 0 ? (int)(((long)n * a.G + a.cols - 1) / a.cols) : 0;
      }
      before += sum;
    }
    if (tid == 0) off[a.NG] = before;
    __syncthreads();
    walk_groups(a, count, true);
  }
  for (int r = tid; r < a.R; r += 1024)
    seq[a.NG + r] = (int)(((long)own_rows(a, r).count * a.G + a.cols - 1) / a.cols);
  __syncthreads();
  // tiles become first entries
  const int nseq = a.NG + a.R;
  int entries = 0;
  for (int b = 0; b < nseq; b += 1024) {
    const int i = b + tid;
    const int n = i < nseq ? seq[i] : 0;
    int sum;
    const int incl = scan1024(n, lds, &sum);
    if (i < nseq) seq[i] = entries + incl - n;
    entries += sum;
  }
  entries = min(entries, a.max_entries);
  __syncthreads();

  // the entries, and where each starts in the cost
  int total = 0;
  for (int b = 0; b < entries; b += 1024) {
    const int e = b + tid;
    int c = 0, v[kEntryInts] = {};
    if (e < entries) {
      int lo = 0, hi = nseq;                            // the last sequence that starts at or before e
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (seq[mid] <= e) lo = mid; else hi = mid;
      }
      const int tile = e - seq[lo];
      v[kEntCol0] = tile * a.cols;
      if (lo < a.NG) {
        const int n = off[lo + 1] - off[lo];
        v[kEntSeq] = ~lo;
        v[kEntCols] = (int)min((long)a.cols, (long)n * a.G - v[kEntCol0]);
        v[kEntKeys] = v[kEntBase] = clampi(a.plen[lo], 0, a.max_p);
        v[kEntFirst] = off[lo];
      } else {
        const Own8 o = own_rows(a, lo - a.NG);
        v[kEntSeq] = lo - a.NG;
        v[kEntCols] = (int)min((long)a.cols, (long)o.count * a.G - v[kEntCol0]);
        const int from = o.keys - o.count;              // row j sees own tokens 0 .. from + j
        v[kEntKeys] = from + (v[kEntCol0] + v[kEntCols] - 1) / a.G + 1;
        v[kEntBase] = from;
        v[kEntFirst] = o.first;
      }
      v[kEntUnits] = (v[kEntKeys] + kUnit - 1) / kUnit;
      c = v[kEntUnits] + kPieceSetup;
    }
    int sum;
    const int incl = scan1024(c, lds, &sum);
    if (e < entries) {
      v[kEntCost] = total + incl - c;
      cost[e] = v[kEntCost];
      int4* to = reinterpret_cast<int4*>(ent + (long)e * kEntryInts);
      to[0] = int4{v[0], v[1], v[2], v[3]};
      to[1] = int4{v[4], v[5], v[6], v[7]};
      to[2] = int4{v[8], v[9], v[10], v[11]};
    }
    total += sum;
  }
  const int q = max(a.min_run, (int)(((long)total + a.runs - 1) / a.runs));
  // pieces, and the slots of their partial results
  int slots = 0;
  for (int b = 0; b < entries; b += 1024) {
    const int e = b + tid;
    int n = 0, pieces = 0;
    int* v = ent + (long)e * kEntryInts;
    if (e < entries) {                                  // (its own entries)
      const int s0 = v[kEntCost] + kPieceSetup;
      pieces = (s0 + v[kEntUnits] - 1) / q - s0 / q + 1;
      const int r = v[kEntSeq], grp = r >= 0 ? a.gid[r] : 0;
      const bool alone = r >= 0 && !(a.depth > 0 && grp >= 0 && grp < a.NG);
      n = alone && pieces == 1 ? 0 : pieces * v[kEntCols];
    }
    int sum;
    const int incl = scan1024(n, lds, &sum);
    if (e < entries) {
      v[kEntSlot] = n == 0 ? -1 : slots + incl - n;
      v[kEntPieces] = pieces;
    }
    slots += sum;
  }
  if (tid == 0) {
    head[0] = entries;
    head[1] = q;
    head[2] = total;
    head[3] = slots;
  }
  // the groups' row lists, and what the join needs of each row
  const int used = clampi(a.qoff[a.R], 0, a.T);
  for (int t = tid; t < a.T; t += 1024) {
    if (t >= used) { rows[(long)t * kRowInts + kRowLevels] = -1; continue; }        // padding
    int lo = 0, hi = a.R;                               // the last request that starts at or before t
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.qoff[mid] <= t) lo = mid; else hi = mid;
    }
    const Own8 o = own_rows(a, lo);
    const int j = t - o.first;
    int* d = rows + (long)t * kRowInts;
    if (j < 0 || j >= o.count) { d[kRowLevels] = -1; continue; }     // no request holds it
    d[kRowEntry] = seq[a.NG + lo];
    d[kRowPlace] = j;
    int levels = 0;
    int grp = a.gid[lo];
    for (int l = 0; l < a.depth && grp >= 0 && grp < a.NG; ++l) {
      const int at = pos[(long)lo * kMaxDepth + l] + j;
      if (clampi(a.plen[grp], 0, a.max_p) > 0) {
        d[kRowGroup + 2 * levels] = seq[grp];
        d[kRowGroup + 2 * levels + 1] = at;
        ++levels;
      }
      list[min((long)off[grp] + at, (long)a.T * a.depth - 1)] = t;
      grp = a.parents ? a.parents[grp] : -1;
    }
    d[kRowLevels] = levels;
  }
}

// ----------------------------------------------------------- partial results
// An entry as the kernels read it: wave-uniform, every index clamped to what it may address.
struct Entry { int seq, col0, cols, cost, units, slot, keys, base, first; };
PARROT_DEV Entry load_entry(const Attend8Args& a, int e) {
  const int* p = a.plan + a.at.entry + (long)e * kEntryInts;
  Entry v;
  v.seq = ld_uniform(p + kEntSeq);
  v.seq = v.seq >= 0 ? min(v.seq, a.R - 1) : max(v.seq, -max(a.NG, 1));
  v.col0 = max(ld_uniform(p + kEntCol0), 0);
  v.cols = clampi(ld_uniform(p + kEntCols), 0, 16 * a.sets);
  v.cost = ld_uniform(p + kEntCost);
  v.keys = clampi(ld_uniform(p + kEntKeys), 0, v.seq >= 0 ? a.max_s : a.max_p);
  v.units = clampi(ld_uniform(p + kEntUnits), 0, (v.keys + kUnit - 1) / kUnit);
  v.slot = ld_uniform(p + kEntSlot);
  v.base = ld_uniform(p + kEntBase);
  v.first = max(ld_uniform(p + kEntFirst), 0);
  return v;
}

// Units [u0, u1) of an entry, piece number `piece`.
template <int DT, int D, int NS>
PARROT_DEV void attend_piece(const Attend8Args& a, const Entry& e, int h, int u0, int u1, int piece) {
  const int HQ = a.H * a.G;
  Tile8<DT, D, NS> tile(a.H, h);
  int at[NS];                                           // the columns' places in [T][HQ], or -1
#pragma unroll
  for (int c = 0; c < NS; ++c) {
    const int col = tile.column(c);
    const int x = e.col0 + col, j = x / a.G;
    at[c] = -1;
    if (col < e.cols) {
      int row = e.first + j;
      if (e.seq < 0) row = a.plan[a.at.list + min((long)row, (long)a.T * max(a.depth, 1) - 1)];
      at[c] = clampi(row, 0, a.T - 1) * HQ + h * a.G + (x - j * a.G);
    }
    tile.lim[c] = e.seq < 0 ? e.keys : min(e.keys, e.base + j + 1);
  }
  tile.load_queries(a.q, a.flip != 0, [&](int c) { return (long)at[c]; });
  Range8 rg;
  const bool own = e.seq >= 0;
  rg.pool = own ? a.own : a.pre;
  rg.tbl = own ? a.stab + (long)e.seq * a.sstride : a.ptab + (long)~e.seq * a.pstride;
  rg.npool = own ? a.nsblk : a.npblk;
  rg.u0 = u0;
  rg.u1 = u1;
  rg.end = e.keys;
  rg.plain = own ? min(e.keys, e.base + e.col0 / a.G + 1) : e.keys;
  tile.run(rg, a.scale_log2);

  const int g = tile.lane >> 4;
  const long slot = e.slot + (long)piece * e.cols;
  const bool direct = e.slot < 0;
  if (!direct && slot + e.cols > a.slots) return;
  tile.finish([&](int c, int col, float inv, float lse2) {
    if (at[c] < 0) return;
    if (direct) {
      char* dst = (char*)a.out + ((long)at[c] * D + 16 * g) * Elem<DT>::kBytes;
      // (every row sees itself: no weights mean that each logit is -inf)
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
      if (g == 0) a.lse[at[c]] = lse2 == -INFINITY ? __builtin_nanf("") : lse2 * kLn2;
    } else {
      const long sl = (long)h * a.slots + slot + col;
      float* dst = a.o_part + sl * D + 16 * g;
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(dst + 64 * x + 4 * i) = tile.four(c, x, i) * inv;
      if (g == 0) a.lse_part[sl] = lse2;
    }
  });
}

template <int DT, int D, int SETS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(SETS > 2 || (DT == kF32 && SETS > 1) ? 1 : 2)))
void k_cache8_attend(Attend8Args a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  int run, h;
  if (a.wide) {                                         // neighbouring tiles of one head, on one XCD
    h = blockIdx.x % a.H;
    run = (int)(blockIdx.x / a.H) * 4 + wave;
  } else {                                              // neighbouring heads of the same blocks
    const int w = blockIdx.x * 4 + wave;
    h = w % a.H;
    run = w / a.H;
  }
  if (run >= a.runs) return;
  const int entries = clampi(ld_uniform(a.plan), 0, a.max_entries);
  const int q = max(ld_uniform(a.plan + 1), 1), total = ld_uniform(a.plan + 2);
  const long c0 = (long)run * q, c1 = min((long)total, c0 + q);
  if (c0 >= total || entries == 0) return;
  // the last entry that starts at or before the run, a factor of 64 a round trip
  const int* cost = a.plan + a.at.cost;
  int e = 0;
  for (int n = entries; n > 1;) {
    const int step = (n + kWave - 1) / kWave;
    const int at = lane * step;
    const int k = __popcll(__ballot(at < n && cost[e + min(at, n - 1)] <= c0));
    e += max(k - 1, 0) * step;
    n = min(step, n - max(k - 1, 0) * step);
    if (step == 1) break;
  }
  e = __builtin_amdgcn_readfirstlane(e);
#pragma unroll 1
  for (; e < entries; ++e) {
    const Entry v = load_entry(a, e);
    if (v.cost >= c1) break;
    const long s0 = (long)v.cost + kPieceSetup;
    const int u0 = (int)max(c0 - s0, 0L), u1 = (int)min(c1 - s0, (long)v.units);
    if (u0 >= u1 || v.cols == 0) continue;
    const int piece = run - (int)(s0 / q);
    if (SETS > 2 && v.cols > 32) attend_piece<DT, D, SETS>(a, v, h, u0, u1, piece);
    else if (SETS > 1 && v.cols > 16) attend_piece<DT, D, SETS < 2 ? SETS : 2>(a, v, h, u0, u1, piece);
    else attend_piece<DT, D, 1>(a, v, h, u0, u1, piece);
  }
}

// ---------------------------------------------------------------------- join
// With base-2 log-sum-exps l_i and normalised outputs o_i of disjoint keys, l = log2 sum 2^l_i
// and o = sum 2^(l_i - l) o_i.  A workgroup per row and HPW query heads: D / 4 lanes a head (16
// bytes a lane), the workgroup's other lane groups take every GROUPS-th partial result.
template <int DT, int D, int HPW>
__global__ __launch_bounds__(256) void k_cache8_join(Attend8Args a) {
  constexpr int GW = D / 4, GROUPS = 256 / (GW * HPW);
  __shared__ float s_m[GROUPS][HPW], s_l[GROUPS][HPW];
  __shared__ f32x4 s_o[GROUPS][HPW][GW];
  const int HQ = a.H * a.G, parts = (HQ + HPW - 1) / HPW;
  const int t = blockIdx.x / parts, i0 = threadIdx.x % GW, sub = threadIdx.x / GW;
  const int mine = sub % HPW, grp = sub / HPW;
  const int hq = (int)(blockIdx.x % parts) * HPW + mine;
  const int* d = a.plan + a.at.row + (long)t * kRowInts;
  const int levels = ld_uniform(d + kRowLevels);
  if (levels < 0) return;
  const bool live = hq < HQ;
  const int h = min(hq, HQ - 1) / a.G, gq = min(hq, HQ - 1) % a.G, cols = 16 * a.sets;
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  bool direct = false;
#pragma unroll 1
  for (int s = -1; s < min(levels, a.depth); ++s) {     // own tokens, then the chain's prefixes
    const int x = (s < 0 ? ld_uniform(d + kRowPlace) : ld_uniform(d + kRowGroup + 2 * s + 1)) * a.G + gq;
    const int e = (s < 0 ? ld_uniform(d + kRowEntry) : ld_uniform(d + kRowGroup + 2 * s)) + x / cols;
    const int* v = a.plan + a.at.entry + (long)clampi(e, 0, a.max_entries - 1) * kEntryInts;
    const int slot = v[kEntSlot], nc = v[kEntCols], n = min(v[kEntPieces], a.runs);   // (a piece per run at most)
    if (slot < 0) { direct = true; continue; }          // the piece wrote the output
    const int col = x % cols;
#pragma unroll 1
    for (int i = grp; i < n; i += 4 * GROUPS) {
      float lp[4];
      f32x4 op[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int k = i + u * GROUPS;
        const long at = slot + (long)k * nc + col;
        const bool on = k < n && at >= 0 && at < a.slots;
        const long sl = (long)h * a.slots + (on ? at : 0);
        lp[u] = on ? a.lse_part[sl] : -INFINITY;
        op[u] = on ? *reinterpret_cast<const f32x4*>(a.o_part + sl * D + 4 * i0) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (lp[u] == -INFINITY) continue;               // no key the row sees
        const float mn = fmaxf(m, lp[u]);
        const float f = fast_exp2(m - mn), w = fast_exp2(lp[u] - mn);
        // (a logit that is no number, or +inf, makes the sums NaN)
        m = lp[u] != lp[u] ? lp[u] : mn;
        l = l * f + w;
        acc = acc * f + op[u] * w;
      }
    }
  }
  s_m[grp][mine] = m;
  s_l[grp][mine] = l;
  s_o[grp][mine][i0] = acc;
  __syncthreads();
  if (grp != 0 || !live || direct) return;
  float mx = s_m[0][mine];
#pragma unroll
  for (int k = 1; k < GROUPS; ++k) mx = fmaxf(mx, s_m[k][mine]);
  float sum = 0.f;
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < GROUPS; ++k) {
    const float mk = s_m[k][mine];
    const float w = mk == -INFINITY ? 0.f : fast_exp2(mk - mx);
    sum += w * s_l[k][mine];
    acc += w * s_o[k][mine][i0];
  }
  // (no weights at all: every logit is -inf, as the one piece gives it)
  const float inv = 1.f / sum;
  const f32x4 res = sum == 0.f ? f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")} : acc * inv;
  const size_t at = (size_t)t * HQ + hq;
  char* dst = (char*)a.out + (at * D + 4 * i0) * Elem<DT>::kBytes;
  if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(dst) = res;
  else *reinterpret_cast<uint2*>(dst) = uint2{Wide8<DT>::pack(res[0], res[1]), Wide8<DT>::pack(res[2], res[3])};
  if (i0 == 0) a.lse[at] = sum == 0.f ? __builtin_nanf("") : (mx + fast_log2(sum)) * kLn2;
}

// ------------------------------------------------------------------ launches
hipError_t launch_plan8(const Plan8Args& a, hipStream_t s) {
  if (a.T < 1 || a.R < 1 || a.G < 1 || a.cols < 16 || a.runs < 1 || a.min_run < 1 || a.max_entries < 1 ||
      a.depth < 0 || a.depth > kMaxDepth || (a.NG > 0) != (a.depth > 0))
    return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_cache8_plan, dim3(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}

template <int DT, int D>
static hipError_t launch_attend_t(const Attend8Args& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const long waves = (long)a.runs * a.H;
  const long wgs = a.wide ? (a.runs + 3L) / 4 * a.H : (waves + 3) / 4;
  if (wgs * 256 > 0xffffffffL) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wgs);
  if (a.sets == 1) hipExtLaunchKernelGGL((k_cache8_attend<DT, D, 1>), grid, dim3(256), 0, s, e0, e1, 0, a);
  else if (a.sets == 2) hipExtLaunchKernelGGL((k_cache8_attend<DT, D, 2>), grid, dim3(256), 0, s, e0, e1, 0, a);
  else if constexpr (DT != kF32) hipExtLaunchKernelGGL((k_cache8_attend<DT, D, 4>), grid, dim3(256), 0, s, e0, e1, 0, a);
  return hipGetLastError();
}
constexpr int kJoinHeads = 2;            // query heads of a join workgroup
template <int DT, int D>
static hipError_t launch_join_t(const Attend8Args& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const long parts = ((long)a.H * a.G + kJoinHeads - 1) / kJoinHeads;
  if (parts * a.T * 256 > 0xffffffffL) return hipErrorInvalidValue;
  hipExtLaunchKernelGGL((k_cache8_join<DT, D, kJoinHeads>), dim3((unsigned)(parts * a.T)), dim3(256), 0, s, e0, e1, 0, a);
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

static bool attend_ok(const Attend8Args& a, int dtype) {
  return a.T >= 1 && a.R >= 1 && a.H >= 1 && a.G >= 1 && a.runs >= 1 && a.max_entries >= 1 && a.sstride >= 1 &&
         a.nsblk >= 1 && (a.NG == 0 || (a.npblk >= 1 && a.pstride >= 1)) && a.o_part && a.lse_part && a.slots >= 1 &&
         (a.sets == 1 || a.sets == 2 || (a.sets == 4 && dtype != kF32));
}
hipError_t launch_attend8(const Attend8Args& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (!attend_ok(a, dtype)) return hipErrorInvalidValue;
  PARROT_CACHE8_LAUNCH(launch_attend_t);
}
hipError_t launch_join8(const Attend8Args& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (!attend_ok(a, dtype)) return hipErrorInvalidValue;
  PARROT_CACHE8_LAUNCH(launch_join_t);
}

}  // namespace parrot
