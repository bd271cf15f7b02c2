// C ABI of caches held in 8 bits: fill of new rows, plan and attention; and copies of cache blocks.
// Argument checks, sizing and launches; host scalars only.
#include <algorithm>
#include <cmath>

#include "cache8_args.h"
#include "host.h"

using parrot::set_error;

namespace {

#define PARROT_TRY(x) do { parrot_status _s = (x); if (_s != PARROT_OK) return _s; } while (0)

long ceil_div(long a, long b) { return (a + b - 1) / b; }
hipEvent_t ev(void* p) { return reinterpret_cast<hipEvent_t>(p); }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

parrot_status bad(const char* fmt, long a = 0, long b = 0) {
  return set_error(PARROT_ERR_INVALID_ARGUMENT, fmt, a, b);
}

parrot_status launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return set_error(PARROT_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
  return set_error(PARROT_OK, "");
}

parrot_status check_pool(const parrot_cache8* c, const char* name) {
  if (!c) return set_error(PARROT_ERR_INVALID_ARGUMENT, "%s is NULL", name);
  char k[32], v[32], s[32];
  snprintf(k, sizeof k, "%s->k", name);
  snprintf(v, sizeof v, "%s->v", name);
  snprintf(s, sizeof s, "%s->scales", name);
  const parrot::PtrCheck need[] = {{c->k, k, 16}, {c->v, v, 16}, {c->scales, s, 4}};
  return parrot::check_pointers(need);
}
parrot::Pool8 pool(const parrot_cache8* c) { return {c->k, c->v, c->scales}; }

// ----------------------------------------------------------------- attention
struct Plan8 {
  int depth;                       // levels of prefixes that the plan has room for
  bool direct;                     // one launch without a plan
  int tiles, waves;                // its column tiles per request, waves of a workgroup
  int sets, cols, wgs, min_run;    // column sets and columns of a narrow tile, workgroups of a cache head
  int wide;                        // columns of a wide tile, 0 where the call has none
  int max_entries;
  long slots;
  parrot::Plan8Layout at;
  size_t plan_bytes, o_bytes, lse_bytes;
};

// Overrides the rule below for tests and tuning (per thread, set through
// parrot_test_cache8_path): 0 one launch of eight waves a workgroup, 2 of four, 1 plan, partial
// results and join.
thread_local int g_path = -1;

constexpr int kMinRun = 6;         // cost of a run at least: four units and a tile's setup

// One launch or plan, partial results and join, by estimates of both in microseconds a layer (the
// plan's own 9 us spread over four), lengths taken as 0.7 of their bounds.
//  * one launch: 7 us, 1.5 more per round of workgroups (three of four waves a CU), and the largest of a
//    workgroup's latency (1.15 us per unit of 32 keys of a wave, 1.55 in fp32), its bytes (own keys at
//    5.5 TB/s; what other tiles or requests read again, from the caches, at 12) and its products at
//    400 TFLOP/s;
//  * plan: 16 us, its bytes at 6.4 TB/s, its products at 600 TFLOP/s.
// Four waves a workgroup where there are more of them than CUs, or few keys for eight.
// Measured, bfloat16, 128-element heads, one launch (eight waves, four) and plan, us a layer of four: one request
// on 4000 tokens, 8 cache heads of four query heads 24, 31, 20; 8 on 1500 12.7, 14.9, 20; 32 cache heads of
// one: 8 requests on 1500 19.6, 22.5, 24; 64 on 300 51, 31, 32; 64 on 1500 107, 100, 96; 16 requests of
// 8 heads on one prefix of 2000 17.4, 20.7, 24.8.
struct OneLaunch { bool taken; int waves; };
OneLaunch one_launch(const parrot_problem* p, const parrot_tree_rows* rows, int depth, long tiles, long cus) {
  const double mean = 0.7, R = p->num_requests, H = p->num_heads, kv = 2.0 * p->head_dim * H;
  const double pre = p->num_groups > 0 ? (double)depth * p->max_prefix_len : 0, longest = p->max_suffix_len + pre;
  const bool f32 = p->dtype == PARROT_DTYPE_F32;
  const double wgs = R * H * tiles;
  const int waves = wgs > cus || longest <= 16 * parrot::kUnit ? 4 : 8;
  const double flops = 4.0 * rows->num_query_rows * rows->num_query_heads * p->head_dim * mean * longest;
  const double own = R * mean * p->max_suffix_len * kv;
  const double latency = longest / (parrot::kUnit * waves) * (f32 ? 1.55 : 1.15);
  const double one = 7 + 1.5 * wgs / (3 * cus) +
                     std::max({latency, own / 5.5e6 + ((tiles - 1) * own + R * tiles * mean * pre * kv) / 12e6, flops / 4e8});
  const double shared = std::min(R, (double)p->num_groups) * mean * pre * kv;
  const double plan = 16 + std::max((own + shared) / 6.4e6, flops / 6e8);
  return {one < plan, waves};
}

parrot_status check_attend(const parrot_problem* p, const parrot_tree_rows* rows, Plan8* pl) {
  PARROT_TRY(parrot::check_problem_fields(p));
  if (!rows) return bad("rows is NULL");
  *pl = Plan8{};
  const long T = rows->num_query_rows, R = p->num_requests, H = p->num_heads, NG = p->num_groups;
  if (T < 0) return bad("num_query_rows %ld < 0", T);
  if (T == 0) return PARROT_OK;
  if (R == 0) return bad("num_query_rows %ld > 0 with no requests", T);
  if (rows->max_query_rows < 1 || rows->max_query_rows > p->max_suffix_len)
    return bad("max_query_rows %ld not in [1, max_suffix_len = %ld]", rows->max_query_rows, p->max_suffix_len);
  if (rows->num_query_heads < 1 || rows->num_query_heads % H != 0)
    return bad("num_query_heads %ld is not a multiple of num_heads %ld", rows->num_query_heads, H);
  if (NG > 0 && (rows->max_group_rows < 0 || rows->max_group_rows > T))
    return bad("max_group_rows %ld not in [0, num_query_rows]", rows->max_group_rows);
  if (T * rows->num_query_heads > 0x7fffffffL)
    return set_error(PARROT_ERR_UNSUPPORTED, "num_query_rows * num_query_heads > 2^31 - 1");
  const long G = rows->num_query_heads / H, cus = parrot::device_cus();
  const bool f32 = p->dtype == PARROT_DTYPE_F32;
  pl->depth = NG > 0 ? std::max(1, (int)p->max_prefix_depth) : 0;
  const long most = G * std::max((long)rows->max_query_rows, NG > 0 ? (long)rows->max_group_rows : 0L);
  const int dt = (int)p->dtype;
  pl->sets = most <= 16 || f32 ? 1 : 2;
  pl->cols = 16 * pl->sets;
  pl->wide = most > parrot::wide_from(dt) ? parrot::wide_cols(dt) : 0;
  // two workgroups a CU (three of a cache of 64-element heads whose calls have 16 columns at most: 64
  // requests on 3000 tokens 43 us, 48 with two; 128-element heads 75 and 73)
  const auto wgs_of = [&](int sets, bool wide) {
    return std::max(2L, cus * (p->head_dim == 64 && sets == 1 && !wide ? 3 : 2) / H);
  };
  pl->wgs = (int)wgs_of(pl->sets, pl->wide != 0);
  pl->min_run = kMinRun;
  // column tiles: those that columns fill, and one more for each sequence (sizes as for the
  // narrowest tiles and the most slots of calls of fewer columns, so that they never decrease)
  const long tiles = (1 + pl->depth) * T * G / 16 + R + NG;
  const long units = ceil_div(p->max_suffix_len, parrot::kUnit) +
                     (NG > 0 ? pl->depth * ceil_div(p->max_prefix_len, parrot::kUnit) : 0);
  long spread = 4 * wgs_of(1, false) * 16;
  if (pl->sets > 1) spread = std::max(spread, 4 * wgs_of(2, false) * 32);
  if (pl->wide) spread = std::max(spread, std::max(4L * pl->wgs * pl->cols, (long)pl->wgs * pl->wide));
  pl->slots = (1 + pl->depth) * T * G + spread;
  const double ints = (double)tiles * (1 + parrot::kEntryInts) + (double)T * (parrot::kRowInts + pl->depth) + 4.0 * wgs_of(1, false) +
                      (NG + R) * (2.0 + parrot::kMaxDepth + parrot::kReqInts) + (parrot::kPlanWaves + 1.0) * NG;
  if (((1.0 + pl->depth) * T * G / pl->cols + R + NG) * (units + parrot::kPieceSetup) > 1.5e9 || pl->slots > 0x7fffffffL || ints > 1.0e9 ||
      R + NG > 0x3fffffffL || pl->wgs * H * 256 > 0xffffffffL)
    return set_error(PARROT_ERR_UNSUPPORTED, "attention over 8 bits: %ld rows in %ld column tiles of %ld units", T, tiles, units);
  pl->max_entries = (int)tiles;
  auto& at = pl->at;
  long n = parrot::kPlanHead;
  auto take = [&n](long ints) { const long first = n; n = (n + ints + 3) & ~3L; return first; };
  at.cost = take(tiles);
  at.entry = take(tiles * parrot::kEntryInts);
  at.run = take(4 * wgs_of(1, false));
  at.row = take(T * parrot::kRowInts);
  at.list = take(T * std::max(pl->depth, 1));
  at.seq = take(2 * (NG + R) + 1);
  at.req = take(R * parrot::kReqInts);
  at.pos = take(R * parrot::kMaxDepth);
  at.count = take((parrot::kPlanWaves + 1) * NG + 1);
  at.total = n;
  pl->plan_bytes = align256((size_t)n * sizeof(int32_t));
  pl->o_bytes = align256((size_t)H * pl->slots * p->head_dim * sizeof(float));
  pl->lse_bytes = align256((size_t)H * pl->slots * sizeof(float));
  pl->tiles = (int)ceil_div(rows->max_query_rows * G, 16);
  const bool fits = R * H * pl->tiles <= 1L << 22;
  const OneLaunch one = one_launch(p, rows, pl->depth, pl->tiles, cus);
  pl->waves = g_path >= 0 ? (g_path == 2 ? 4 : 8) : one.waves;
  pl->direct = fits && (g_path >= 0 ? g_path != 1 : one.taken);
  return PARROT_OK;
}

// The int arrays of a step: checks, and as the kernels take them.
parrot_status step_arrays(const parrot_problem* p, const parrot_tree_rows* rows, const Plan8& pl, const int32_t* query_offsets,
                          const int32_t* prefix_lens, const int32_t* prefix_parents, const int32_t* suffix_lens,
                          const int32_t* group_ids, parrot::Step8* st) {
  const parrot::PtrCheck need[] = {{query_offsets, "query_offsets", 4}, {suffix_lens, "suffix_lens", 4},
                                   {group_ids, "group_ids", 4}};
  PARROT_TRY(parrot::check_pointers(need));
  if (p->num_groups > 0) {
    const parrot::PtrCheck pre[] = {{prefix_lens, "prefix_lens", 4}};
    PARROT_TRY(parrot::check_pointers(pre));
    if (prefix_parents && reinterpret_cast<uintptr_t>(prefix_parents) % 4)
      return bad("prefix_parents is not 4-byte aligned");
  }
  st->qoff = query_offsets; st->plen = prefix_lens; st->slen = suffix_lens; st->gid = group_ids;
  st->parents = p->num_groups > 0 ? prefix_parents : nullptr;
  st->T = rows->num_query_rows; st->R = p->num_requests; st->NG = p->num_groups;
  st->G = rows->num_query_heads / p->num_heads;
  st->depth = st->parents ? pl.depth : std::min(pl.depth, 1);
  st->max_p = p->num_groups > 0 ? p->max_prefix_len : 0;
  st->max_s = p->max_suffix_len; st->max_q = rows->max_query_rows;
  return PARROT_OK;
}

parrot_status record_none(const parrot_trace& tr, hipStream_t s) {
  for (void* e : {tr.merge_start, tr.merge_stop})
    if (e && hipEventRecord(ev(e), s) != hipSuccess) return set_error(PARROT_ERR_HIP, "hipEventRecord failed");
  return set_error(PARROT_OK, "");
}

}  // namespace

extern "C" {

parrot_status parrot_cache8_fill(
    const parrot_problem* p, const parrot_fill_rows* rows, const parrot_rotary* rotary, const void* q, const void* k,
    const void* v, const void* q_norm, const void* k_norm, const int32_t* positions, const int32_t* query_offsets,
    const int32_t* suffix_block_tables, const int32_t* suffix_lens, void* q_out, const parrot_cache8* suffix, void* stream,
    const parrot_trace* trace) {
  PARROT_TRY(parrot::check_fill(p, rows));
  if (rows->num_query_rows == 0) return set_error(PARROT_OK, "");
  parrot::Fill8Args a{};
  int partner;
  PARROT_TRY(parrot::fill_args(p, rows, rotary, q, k, v, q_norm, k_norm, positions, query_offsets, suffix_block_tables,
                               suffix_lens, q_out, &a.f, &partner));
  PARROT_TRY(check_pool(suffix, "suffix"));
  if (suffix->k == suffix->v) return bad("suffix->k and suffix->v are the same pool");
  a.f.sk = suffix->k; a.f.sv = suffix->v; a.scales = suffix->scales;
  const long elt = p->dtype == PARROT_DTYPE_F32 ? 4 : 2;
  const long units = rows->max_query_rows == 1 ? p->num_requests : rows->num_query_rows / 16 + 2L * p->num_requests;
  if (rows->max_query_rows == 1) {         // a lane group per head
    parrot::fill_slabs(&a.f, 4096 / (p->head_dim * elt), p->num_requests);
  } else {
    // a wave or half of one per head; four workgroups a CU are there at once, and the units' heads
    // go over as many as leave the last round fullest (470 units of 96 heads in bfloat16: two a unit 89 us,
    // three 104, one 131, nine 96)
    const long step = p->head_dim * elt == 128 ? 8 : 4, steps = ceil_div(a.f.HQ + 2L * a.f.H, step);
    const long busy = ceil_div(rows->num_query_rows, 16) + p->num_requests, room = 4L * parrot::device_cus();
    long best = 1;
    double least = 1e30;
    for (long n = 1; n <= std::min(steps, 24L); ++n) {
      const double t = (double)ceil_div(busy * n, room) * ceil_div(steps, n) + 0.1 * n;
      if (t < least) { least = t; best = n; }
    }
    a.f.slab_heads = (int)(ceil_div(steps, best) * step);
    a.f.slabs = (int)ceil_div(a.f.HQ + 2L * a.f.H, a.f.slab_heads);
  }
  if (units * a.f.slabs * 256 > 0xffffffffL)
    return set_error(PARROT_ERR_UNSUPPORTED, "fill needs %ld workgroups", units * a.f.slabs);
  a.units = (int)units;
  return launched(parrot::launch_fill8(a, partner, (int)p->dtype, p->head_dim, reinterpret_cast<hipStream_t>(stream),
                                       trace ? ev(trace->partials_start) : nullptr,
                                       trace ? ev(trace->partials_stop) : nullptr),
                  "8-bit fill kernel");
}

size_t parrot_cache8_plan_bytes(const parrot_problem* p, const parrot_tree_rows* rows) {
  Plan8 pl;
  if (check_attend(p, rows, &pl) != PARROT_OK) return (size_t)-1;
  set_error(PARROT_OK, "");
  return pl.plan_bytes;
}

size_t parrot_cache8_workspace_bytes(const parrot_problem* p, const parrot_tree_rows* rows) {
  Plan8 pl;
  if (check_attend(p, rows, &pl) != PARROT_OK) return (size_t)-1;
  set_error(PARROT_OK, "");
  return pl.o_bytes + pl.lse_bytes;
}

parrot_status parrot_cache8_plan(
    const parrot_problem* p, const parrot_tree_rows* rows, const int32_t* query_offsets, const int32_t* prefix_lens,
    const int32_t* prefix_parents, const int32_t* suffix_lens, const int32_t* group_ids, void* plan, size_t plan_bytes,
    void* stream) {
  Plan8 pl;
  PARROT_TRY(check_attend(p, rows, &pl));
  if (rows->num_query_rows == 0) return set_error(PARROT_OK, "");
  parrot::Plan8Args a{};
  PARROT_TRY(step_arrays(p, rows, pl, query_offsets, prefix_lens, prefix_parents, suffix_lens, group_ids, &a.st));
  const parrot::PtrCheck need[] = {{plan, "plan", 256}};
  PARROT_TRY(parrot::check_pointers(need));
  if (plan_bytes < pl.plan_bytes)
    return set_error(PARROT_ERR_WORKSPACE_TOO_SMALL, "plan is %zu bytes, need %zu", plan_bytes, pl.plan_bytes);
  if (pl.direct) return set_error(PARROT_OK, "");
  a.plan = reinterpret_cast<int*>(plan);
  a.at = pl.at;
  a.cols = pl.cols;
  a.wide_cols = parrot::wide_cols((int)p->dtype);
  a.wide_from = pl.wide ? parrot::wide_from((int)p->dtype) : 0x7fffffff;
  a.wgs = pl.wgs; a.min_run = pl.min_run;
  a.max_entries = pl.max_entries;
  return launched(parrot::launch_plan8(a, reinterpret_cast<hipStream_t>(stream)), "plan kernel");
}

parrot_status parrot_cache8_attention(
    const parrot_problem* p, const parrot_tree_rows* rows, const void* q, const int32_t* query_offsets,
    const parrot_cache8* prefix, const parrot_cache8* suffix, const int32_t* prefix_block_tables, const int32_t* prefix_lens,
    const int32_t* prefix_parents, const int32_t* suffix_block_tables, const int32_t* suffix_lens, const int32_t* group_ids,
    const void* plan, size_t plan_bytes, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream,
    const parrot_trace* trace) {
  Plan8 pl;
  PARROT_TRY(check_attend(p, rows, &pl));
  if (rows->num_query_rows == 0) return set_error(PARROT_OK, "");
  parrot::Attend8Args a{};
  PARROT_TRY(step_arrays(p, rows, pl, query_offsets, prefix_lens, prefix_parents, suffix_lens, group_ids, &a.st));
  const parrot::PtrCheck need[] = {{q, "q", 16}, {suffix_block_tables, "suffix_block_tables", 4}, {plan, "plan", 256},
                                   {out, "out", 16}, {lse, "lse", 4}, {workspace, "workspace", 256}};
  PARROT_TRY(parrot::check_pointers(need));
  PARROT_TRY(check_pool(suffix, "suffix"));
  if (p->num_groups > 0) {
    PARROT_TRY(check_pool(prefix, "prefix"));
    const parrot::PtrCheck pre[] = {{prefix_block_tables, "prefix_block_tables", 4}};
    PARROT_TRY(parrot::check_pointers(pre));
  }
  if (q == out) return bad("out is q");
  if (plan_bytes < pl.plan_bytes)
    return set_error(PARROT_ERR_WORKSPACE_TOO_SMALL, "plan is %zu bytes, need %zu", plan_bytes, pl.plan_bytes);
  if (workspace_bytes < pl.o_bytes + pl.lse_bytes)
    return set_error(PARROT_ERR_WORKSPACE_TOO_SMALL, "workspace is %zu bytes, need %zu", workspace_bytes, pl.o_bytes + pl.lse_bytes);
  a.q = q; a.out = out; a.lse = lse;
  a.own = pool(suffix);
  if (p->num_groups > 0) a.pre = pool(prefix);
  a.ptab = prefix_block_tables; a.stab = suffix_block_tables;
  a.plan = reinterpret_cast<const int*>(plan);
  a.at = pl.at;
  a.o_part = reinterpret_cast<float*>(workspace);
  a.lse_part = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + pl.o_bytes);
  a.slots = pl.slots;
  a.T = rows->num_query_rows; a.R = p->num_requests; a.H = p->num_heads; a.NG = p->num_groups;
  a.G = a.st.G; a.depth = pl.depth;
  a.pstride = p->prefix_table_stride; a.sstride = p->suffix_table_stride;
  a.max_p = a.st.max_p; a.max_s = p->max_suffix_len;
  a.npblk = p->num_groups > 0 ? p->num_prefix_blocks : 1; a.nsblk = p->num_suffix_blocks;
  a.wgs = pl.wgs; a.sets = pl.sets; a.wide = pl.wide; a.max_entries = pl.max_entries; a.tiles = pl.tiles; a.waves = pl.waves;
  a.flip = p->sm_scale < 0.f;
  a.scale_log2 = std::fabs(p->sm_scale) * parrot::kLog2e;
  const parrot_trace none = {nullptr, nullptr, nullptr, nullptr};
  const parrot_trace& tr = trace ? *trace : none;
  const int dt = (int)p->dtype, D = p->head_dim;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (pl.direct) {
    PARROT_TRY(launched(parrot::launch_direct8(a, dt, D, s, ev(tr.partials_start), ev(tr.partials_stop)), "8-bit attention kernel"));
    return record_none(tr, s);
  }
  PARROT_TRY(launched(parrot::launch_attend8(a, dt, D, s, ev(tr.partials_start), ev(tr.partials_stop)), "8-bit attention kernel"));
  return launched(parrot::launch_join8(a, dt, D, s, ev(tr.merge_start), ev(tr.merge_stop)), "8-bit join kernel");
}

// Test hooks (not in parrot_attn.h): the path of this thread's calls (see g_path; -1 gives the
// choice back), and the one these arguments take (-1: invalid).
void parrot_test_cache8_path(int path) { g_path = path >= 0 && path <= 2 ? path : -1; }
int parrot_test_cache8_planned(const parrot_problem* p, const parrot_tree_rows* rows) {
  Plan8 pl;
  return check_attend(p, rows, &pl) == PARROT_OK ? !pl.direct : -1;
}

parrot_status parrot_validate_cache8_inputs(
    const parrot_problem* p, const parrot_tree_rows* rows, const int32_t* query_offsets,
    const int32_t* prefix_block_tables, const int32_t* prefix_lens, const int32_t* prefix_parents,
    const int32_t* suffix_block_tables, const int32_t* suffix_lens, const int32_t* group_ids, int32_t* scratch,
    void* stream) {
  Plan8 pl;
  PARROT_TRY(check_attend(p, rows, &pl));
  if (rows->num_query_rows == 0) return set_error(PARROT_OK, "");
  const parrot_prefill_rows as_prefill = {rows->num_query_rows, rows->max_query_rows, rows->max_group_rows};
  const parrot::ValidateTree tree = {nullptr};
  return parrot::validate_inputs(p, prefix_block_tables, prefix_lens, prefix_parents, suffix_block_tables,
                                 suffix_lens, group_ids, scratch, stream, &as_prefill, query_offsets, &tree);
}

// -------------------------------------------------------------------- blocks
parrot_status parrot_copy_blocks(const parrot_block_pool* pools, int32_t num_pools, int32_t num_blocks, const int32_t* src,
                                 const int32_t* dst, int32_t num_copies, void* stream, const parrot_trace* trace) {
  if (num_pools < 0) return bad("num_pools %ld < 0", num_pools);
  if (num_copies < 0) return bad("num_copies %ld < 0", num_copies);
  if (num_blocks < 1) return bad("num_blocks %ld < 1", num_blocks);
  if (num_pools > 0 && !pools) return bad("pools is NULL");
  if (num_pools == 0 || num_copies == 0) return set_error(PARROT_OK, "");
  const parrot::PtrCheck need[] = {{src, "src", 4}, {dst, "dst", 4}};
  PARROT_TRY(parrot::check_pointers(need));
  if (src == dst) return bad("src and dst are the same array");
  for (int32_t i = 0; i < num_pools; ++i) {
    const parrot_block_pool& x = pools[i];
    if (!x.base) return bad("pool %ld is NULL", i);
    if (x.block_bytes < 2 || x.block_bytes % 2 != 0 || x.block_bytes > (1LL << 31))
      return bad("block_bytes of pool %ld is not even and in [2, 2^31]", i);
    if (reinterpret_cast<uintptr_t>(x.base) % (x.block_bytes % 16 ? 2 : 16)) return bad("pool %ld is not aligned", i);
  }
  // (a launch's arguments hold kCopyPools pools)
  int32_t done = 0;
  while (done < num_pools) {
    parrot::CopyArgs a{};
    a.src = src; a.dst = dst; a.blocks = num_blocks;
    const int32_t first = done;
    for (; done < num_pools && done - first < parrot::kCopyPools; ++done) {
      a.base[done - first] = pools[done].base;
      a.bytes[done - first] = (unsigned)pools[done].block_bytes;
    }
    a.pools = done - first;
    // a launch holds less than 2^32 threads
    long most = 0;
    for (int i = 0; i < a.pools; ++i) most = std::max(most, (long)a.bytes[i]);
    const long each = ceil_div(most, 16384) * a.pools * 256, at_once = std::max(1L, 0xf0000000L / each);
    if (each > 0xf0000000L) return set_error(PARROT_ERR_UNSUPPORTED, "blocks of %ld bytes", most);
    for (long i = 0; i < num_copies; i += at_once) {
      a.n = (int)std::min(at_once, num_copies - i);
      a.src = src + i; a.dst = dst + i;
      PARROT_TRY(launched(parrot::launch_copy_blocks(a, reinterpret_cast<hipStream_t>(stream),
                                                     trace && first == 0 && i == 0 ? ev(trace->partials_start) : nullptr,
                                                     trace && done == num_pools && i + at_once >= num_copies
                                                         ? ev(trace->partials_stop) : nullptr),
                          "copy kernel"));
    }
  }
  return set_error(PARROT_OK, "");
}

}  // extern "C"
