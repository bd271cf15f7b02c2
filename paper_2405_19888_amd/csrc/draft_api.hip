// C ABI of a drafting step: rotary embeddings (host), fill of new rows, tree decode,
// accept and commit.  Argument checks, sizing and launches; host scalars only.
#include <algorithm>
#include <cmath>

#include "draft_args.h"
#include "host.h"
#include "tree_args.h"

using parrot::set_error;

namespace {

#define PARROT_TRY(x) do { parrot_status _s = (x); if (_s != PARROT_OK) return _s; } while (0)

long ceil_div(long a, long b) { return (a + b - 1) / b; }
hipEvent_t ev(void* p) { return reinterpret_cast<hipEvent_t>(p); }

parrot_status bad(const char* fmt, long a = 0, long b = 0) {
  return set_error(PARROT_ERR_INVALID_ARGUMENT, fmt, a, b);
}

parrot_status launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return set_error(PARROT_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
  return set_error(PARROT_OK, "");
}

static_assert(PARROT_ROTARY_MAX_PAIRS == parrot::kRotaryPairs && PARROT_MAX_TREE_ROWS == parrot::kTreeRows,
              "header and kernels agree");

constexpr long double kTwoPi = 6.283185307179586476925286766559005768L;

parrot_status check_rotary(int32_t rotary_dim, int32_t interleaved) {
  if (rotary_dim < 2 || rotary_dim > 2 * PARROT_ROTARY_MAX_PAIRS || rotary_dim % 2 != 0)
    return bad("rotary_dim %ld is not even and in [2, %ld]", rotary_dim, 2 * PARROT_ROTARY_MAX_PAIRS);
  if (interleaved != 0 && interleaved != 1) return bad("interleaved %ld is not 0 or 1", interleaved);
  return PARROT_OK;
}

// Frequencies are computed with the 64 bits that x86-64's long double has: what a fraction of a turn is off
// by comes n times at position n, and those of a double (2^-53 of it) are off by 2^-25 turns at
// the last position.
parrot_status store_rotary(parrot_rotary* rotary, int32_t rotary_dim, int32_t interleaved,
                           const long double* radians, double amplitude) {
  if (!((float)amplitude > 0.f) || !std::isfinite((float)amplitude)) return bad("amplitude is not positive and finite in fp32");
  parrot_rotary out{};
  out.rotary_dim = rotary_dim;
  out.interleaved = interleaved;
  out.amplitude = (float)amplitude;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    const long double turns = radians[i] / kTwoPi;
    if (!(turns >= 0.0L && turns < 1.0L)) return bad("frequency %ld is not in [0, 2 pi)", i);
    // the nearest multiple of 2^-64 (it fits: turns < 1 is at most 1 - 2^-64)
    out.turns[i] = (uint64_t)std::round(std::ldexp(turns, 64));
  }
  *rotary = out;
  return set_error(PARROT_OK, "");
}

}  // namespace

// -------------------------------------------------------------------- rotary
extern "C" {

parrot_status parrot_rotary_from_frequencies(parrot_rotary* rotary, int32_t rotary_dim,
                                             int32_t interleaved, const double* radians,
                                             double amplitude) {
  if (!rotary || !radians) return bad(rotary ? "radians is NULL" : "rotary is NULL");
  PARROT_TRY(check_rotary(rotary_dim, interleaved));
  long double wide[PARROT_ROTARY_MAX_PAIRS];
  std::copy(radians, radians + rotary_dim / 2, wide);
  return store_rotary(rotary, rotary_dim, interleaved, wide, amplitude);
}

parrot_status parrot_rotary_init(parrot_rotary* rotary, const parrot_rotary_config* c) {
  if (!rotary || !c) return bad(rotary ? "config is NULL" : "rotary is NULL");
  PARROT_TRY(check_rotary(c->rotary_dim, c->interleaved));
  if (!(c->base > 1.0) || !std::isfinite(c->base)) return bad("base is not finite and above 1");
  if (c->scaling < PARROT_ROTARY_SCALE_NONE || c->scaling > PARROT_ROTARY_SCALE_WAVELENGTH)
    return set_error(PARROT_ERR_UNSUPPORTED, "rotary scaling %d", (int)c->scaling);
  const bool yarn = c->scaling == PARROT_ROTARY_SCALE_YARN, blended = yarn || c->scaling == PARROT_ROTARY_SCALE_WAVELENGTH;
  const double s = c->scaling == PARROT_ROTARY_SCALE_NONE ? 1.0 : c->factor;
  if (!(s >= 1.0) || !std::isfinite(s)) return bad("factor is not finite and at least 1");
  double low = c->low, high = c->high;
  if (blended) {
    if (!(c->original_length >= 1.0) || !std::isfinite(c->original_length))
      return bad("original_length is not finite and at least 1");
    if (low == 0.0 && high == 0.0) { low = 1.0; high = yarn ? 32.0 : 4.0; }
    if (!(low > 0.0) || !(high > low) || !std::isfinite(high)) return bad("low and high are not 0 < low < high");
  }
  if (c->scaling == PARROT_ROTARY_SCALE_NTK && c->rotary_dim < 4) return bad("NTK scaling needs rotary_dim >= 4");
  if (!(c->amplitude >= 0.0)) return bad("amplitude is negative");
  const long double rd = c->rotary_dim;
  const long double base = c->scaling == PARROT_ROTARY_SCALE_NTK ? c->base * std::pow((long double)s, rd / (rd - 2)) : c->base;
  // YaRN: the pairs that turn `high` and `low` times in the trained length, rounded
  // outwards, bound the blend
  double first = 0.0, last = 0.0;
  if (yarn) {
    auto pair_of = [&](double turns) {
      return c->rotary_dim * std::log(c->original_length / (turns * (double)kTwoPi)) / (2.0 * std::log(c->base));
    };
    first = std::max(std::floor(pair_of(high)), 0.0);
    last = std::min(std::ceil(pair_of(low)), c->rotary_dim - 1.0);
  }
  const auto share = [](long double x) { return std::min(1.0L, std::max(0.0L, x)); };
  long double radians[PARROT_ROTARY_MAX_PAIRS];
  for (int i = 0; i < c->rotary_dim / 2; ++i) {
    const long double f = std::pow(base, -2 * i / rd);
    long double keep = 1;                                    // share of the unscaled frequency
    if (c->scaling == PARROT_ROTARY_SCALE_LINEAR) keep = 0;
    if (yarn) keep = 1 - share((i - first) / std::max((long double)(last - first), 1e-3L));
    if (c->scaling == PARROT_ROTARY_SCALE_WAVELENGTH)
      keep = share((c->original_length * f / kTwoPi - low) / (high - low));
    radians[i] = c->scaling == PARROT_ROTARY_SCALE_NTK ? f : f * keep + f / s * (1 - keep);
  }
  const double amplitude = c->amplitude > 0.0 ? c->amplitude : yarn ? 0.1 * std::log(s) + 1.0 : 1.0;
  return store_rotary(rotary, c->rotary_dim, c->interleaved, radians, amplitude);
}

}  // extern "C"

// ---------------------------------------------------------------------- fill
namespace {

parrot_status check_fill_rows(const parrot_problem* p, const parrot_fill_rows* rows) {
  PARROT_TRY(parrot::check_problem_fields(p));
  if (!rows) return bad("rows is NULL");
  if (rows->num_query_rows < 0) return bad("num_query_rows %ld < 0", rows->num_query_rows);
  if (rows->num_query_rows == 0) return PARROT_OK;
  if (p->num_requests == 0) return bad("num_query_rows %ld > 0 with no requests", rows->num_query_rows);
  if (rows->max_query_rows < 1 || rows->max_query_rows > p->max_suffix_len)
    return bad("max_query_rows %ld not in [1, max_suffix_len = %ld]", rows->max_query_rows, p->max_suffix_len);
  if (!(rows->norm_eps >= 0.f) || !std::isfinite(rows->norm_eps)) return bad("norm_eps is not finite and >= 0");
  return PARROT_OK;
}

}  // namespace

extern "C" parrot_status parrot_rotary_fill(
    const parrot_problem* p, const parrot_fill_rows* rows, const parrot_rotary* rotary, const void* q,
    const void* k, const void* v, const void* q_norm, const void* k_norm, const int32_t* positions,
    const int32_t* query_offsets, const int32_t* suffix_block_tables, const int32_t* suffix_lens,
    void* q_out, void* suffix_k, void* suffix_v, void* stream, const parrot_trace* trace) {
  PARROT_TRY(check_fill_rows(p, rows));
  if (rows->num_query_rows == 0) return set_error(PARROT_OK, "");
  if ((q == nullptr) != (q_out == nullptr)) return bad(q ? "q_out is NULL and q is not" : "q is NULL and q_out is not");
  const parrot::PtrCheck need[] = {
      {k, "k", 16}, {v, "v", 16}, {query_offsets, "query_offsets", 4},
      {suffix_block_tables, "suffix_block_tables", 4}, {suffix_lens, "suffix_lens", 4},
      {suffix_k, "suffix_k", 16}, {suffix_v, "suffix_v", 16}};
  PARROT_TRY(parrot::check_pointers(need));
  const long T = rows->num_query_rows, D = p->head_dim, H = p->num_heads;
  const long elt = p->dtype == PARROT_DTYPE_F32 ? 4 : 2;
  const long HQ = q ? rows->num_query_heads : 0;
  if (q) {
    if (HQ < 1) return bad("num_query_heads %ld < 1", HQ);
    const parrot::PtrCheck qs[] = {{q, "q", 16}, {q_out, "q_out", 16}};
    PARROT_TRY(parrot::check_pointers(qs));
  }
  for (const parrot::PtrCheck& c : {parrot::PtrCheck{q_norm, "q_norm", 16}, parrot::PtrCheck{k_norm, "k_norm", 16}})
    if (c.ptr) {
      const parrot::PtrCheck one[] = {c};
      PARROT_TRY(parrot::check_pointers(one));
    }
  struct { const char* name; int64_t stride; long width; } strides[] = {
      {"q_stride", rows->q_stride, HQ * D}, {"k_stride", rows->k_stride, H * D}, {"v_stride", rows->v_stride, H * D}};
  for (auto& s : strides) {
    if (s.width == 0) continue;
    if (s.stride < s.width || s.stride > (1LL << 40))
      return set_error(PARROT_ERR_INVALID_ARGUMENT, "%s %lld not in [%ld, 2^40]", s.name, (long long)s.stride, s.width);
    if (s.stride * elt % 16 != 0)
      return set_error(PARROT_ERR_INVALID_ARGUMENT, "%s %lld is not a multiple of 16 bytes", s.name, (long long)s.stride);
  }
  if (q && q == q_out && rows->q_stride != HQ * D)
    return bad("q_out = q needs q_stride %ld = num_query_heads * head_dim", (long)rows->q_stride);
  if (q && HQ > 0x7fffffffL / 128) return set_error(PARROT_ERR_UNSUPPORTED, "num_query_heads %ld", HQ);
  if (rotary) {
    PARROT_TRY(check_rotary(rotary->rotary_dim, rotary->interleaved));
    if (rotary->rotary_dim > D) return bad("rotary_dim %ld > head_dim %ld", rotary->rotary_dim, D);
    const parrot::PtrCheck pos[] = {{positions, "positions", 4}};
    PARROT_TRY(parrot::check_pointers(pos));
  }

  parrot::FillArgs a{};
  a.q = q; a.k = k; a.v = v;
  a.q_stride = rows->q_stride * elt; a.k_stride = rows->k_stride * elt; a.v_stride = rows->v_stride * elt;
  a.q_norm = q ? q_norm : nullptr; a.k_norm = k_norm;
  a.positions = positions; a.qoff = query_offsets; a.stab = suffix_block_tables; a.slen = suffix_lens;
  a.q_out = q_out; a.sk = suffix_k; a.sv = suffix_v;
  a.T = (int)T; a.R = p->num_requests; a.HQ = (int)HQ; a.H = (int)H;
  a.sstride = p->suffix_table_stride; a.max_s = p->max_suffix_len; a.max_q = rows->max_query_rows;
  a.nsblk = p->num_suffix_blocks;
  a.eps = rows->norm_eps; a.amplitude = 1.f;
  int partner = parrot::kRotaryNone;
  if (rotary) {
    a.rd = rotary->rotary_dim;
    a.amplitude = rotary->amplitude;
    std::copy(rotary->turns, rotary->turns + PARROT_ROTARY_MAX_PAIRS, a.turns);
    const int per_lane = 16 / (int)elt;
    partner = rotary->interleaved ? parrot::kRotaryInterleaved
              : a.rd / 2 % per_lane == 0 ? parrot::kRotaryHalfVector : parrot::kRotaryHalfScalar;
  }
  // a row's heads over several workgroups where rows alone do not fill the device
  const long heads = HQ + 2 * H, step = 4096 / (D * elt);
  const long slabs = std::max(1L, std::min(ceil_div(heads, step), ceil_div(4L * parrot::device_cus(), T)));
  a.slab_heads = (int)(ceil_div(ceil_div(heads, slabs), step) * step);
  a.slabs = (int)ceil_div(heads, a.slab_heads);
  if (T * a.slabs > 0x7fffffffL) return set_error(PARROT_ERR_UNSUPPORTED, "fill needs %ld workgroups", T * a.slabs);
  return launched(parrot::launch_fill(a, partner, (int)p->dtype, (int)D, reinterpret_cast<hipStream_t>(stream),
                                      trace ? ev(trace->partials_start) : nullptr,
                                      trace ? ev(trace->partials_stop) : nullptr),
                  "fill kernel");
}

// --------------------------------------------------------------- tree decode
namespace {

struct TreePlan {
  int depth, max_depth, tiles;   // levels of a chain: this call's, at most
  bool split;                    // partial results and join, else one launch
  bool small;                    // the one launch: waves that share the keys, else a tile
  int cp, tiles_p, seg_p, seg_pre, seg, sets, own_wgs, runs, min_run;
  long n_pre;
  bool pre_first;                // prefix workgroups before the own tokens'
  long held;                     // rows with prefixes, at most
  int pieces, piece_cols;        // of a cache head's own tokens, columns of each
  size_t own0, slots;            // first slot of the own tokens' partial results, slots in all
  size_t o_bytes, lse_bytes;
  size_t used_bytes;             // of workspace, by this call
  size_t total_bytes;            // what no call of at most these sizes exceeds
};

// Overrides the estimate below for tests and tuning (per thread, set through
// parrot_test_tree_path): 0 one launch, 1 partial results and join.
thread_local int g_tree_path = -1;

constexpr int kTreeMinRun = 10;      // cost of a run at least: 8 units and a tile's setup
constexpr int kTreeChunkMax = 2560, kTreeChunkMin = 256;   // prefix chunks are halved while above the second
constexpr int kTreeChunkLeast = 160;
constexpr double kTreeSplitLeast = 22;   // microseconds of a split call, at least

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// How own tokens are cut for requests of at most `cols` columns: by waves of `sets` column
// sets, else (0) by tiles.
struct OwnRole { int sets, wgs, runs, tiles, piece_cols; };
OwnRole own_role(int dtype, long H, long cols, long cus) {
  const bool f32 = dtype == PARROT_DTYPE_F32;
  OwnRole o;
  o.sets = cols <= 16 ? 1 : cols <= 32 && !f32 ? 2 : 0;
  o.tiles = (int)ceil_div(cols, parrot::tree_cols(dtype));
  const long per_wg = o.sets ? 4 : 1;
  o.wgs = (int)std::max((o.sets ? 1 : o.tiles > 1 || f32 ? 3 : 2) * cus, ceil_div(H, per_wg));
  o.runs = (int)(o.wgs * per_wg / H);
  o.piece_cols = o.sets ? 16 * o.sets : parrot::tree_cols(dtype);
  return o;
}

// Slots of the prefixes' partial results that no call of at most these sizes exceeds: each
// of `held` rows has one per query head, level and chunk.  Chunks are halved only while their
// workgroups, one per cache head, chunk and column tile, are fewer than 3/2 a CU, so after that
// there are less than 3 a CU, of tree_cols slots at most per level: those tiles hold every row
// that has prefixes.
double prefix_slot_bound(const parrot_problem* p, const parrot_tree_rows* rows, long held, int levels, long cus) {
  if (levels == 0 || held == 0) return 0;
  const double each = (double)held * rows->num_query_heads * levels;
  return std::min(each * ceil_div(p->max_prefix_len, kTreeChunkLeast),
                  std::max(each * ceil_div(p->max_prefix_len, kTreeChunkMax), 3.0 * cus * parrot::tree_cols(p->dtype) * levels));
}

// The row counts of a tree call (or of accept and commit, which have no heads).
parrot_status check_tree_counts(int32_t requests, const parrot_tree_rows* rows) {
  if (!rows) return bad("rows is NULL");
  const long T = rows->num_query_rows;
  if (T < 0) return bad("num_query_rows %ld < 0", T);
  if (T == 0) return PARROT_OK;
  if (requests == 0) return bad("num_query_rows %ld > 0 with no requests", T);
  if (rows->max_query_rows < 1 || rows->max_query_rows > PARROT_MAX_TREE_ROWS)
    return bad("max_query_rows %ld not in [1, %ld]", rows->max_query_rows, PARROT_MAX_TREE_ROWS);
  return PARROT_OK;
}

// Whether the split plan is the faster one, by estimates of both times in microseconds.
// Lengths are bounds: the mean is taken as 0.7 of them, the longest as the bound.
//  * one launch: 8 us and 4 more per round of workgroups (three a CU), and the largest of
//    a workgroup's latency (0.55 us a 16 KiB stage with one column set a wave, 0.75 with
//    two, 1.4 with fp32; waves that share the keys 2.4 for 8 steps of 16 KiB, fp32 4), the
//    bytes (own tokens at 5.6 TB/s, the prefixes that every request reads again at 12
//    from the caches) and the products at 750 TFLOP/s (fp32 100).
//  * split plan: by tiles 14 us (fp32 36) and 8 per piece of a workgroup, by waves 12 us and
//    3 per piece of a wave but 22 at least, 8 for prefixes; the own tokens once per
//    column tile at 6.0 TB/s (by waves 6.4) or their products (fp32: those of whole tiles),
//    the prefixes' products, and the partial results, written and read, at 4.7 TB/s;
//    kTreeSplitLeast at least.
// The first grows with every size, and the second has a least value: `never` is set where no
// call of at most these sizes splits.
// Measured, one launch and split, bfloat16 heads of 128: a request of 64 rows on 300, 2000,
// 8000 tokens and 32 heads 15 and 20, 47 and 24, 155 and 46 us; 32 requests of 64 rows,
// four query heads on each of 8, on 300, 4000 tokens 29 and 72, 181 and 284; 32 requests of
// 8 rows on 100 own tokens and one prefix of 300, 4000 tokens and 32 heads 33 and 31, 162 and
// 58; 128 requests of 4 rows on 1000 tokens and 8 heads 103 and 95.
bool tree_splits(const parrot_problem* p, const parrot_tree_rows* rows, const TreePlan& pl, long cus, bool* never) {
  const double mean = 0.7, R = p->num_requests, H = p->num_heads, HQ = rows->num_query_heads, D = p->head_dim;
  const double T = rows->num_query_rows, eb = p->dtype == PARROT_DTYPE_F32 ? 4 : 2, kv = 2 * D * eb * H;
  const bool f32 = p->dtype == PARROT_DTYPE_F32;
  const double own = p->max_suffix_len, pre = p->num_groups > 0 ? (double)pl.max_depth * p->max_prefix_len : 0;
  const double flops_own = 4 * D * T * HQ * mean * own, flops_pre = 4 * D * T * HQ * mean * pre;
  const double rate = f32 ? 1e8 : 7.5e8, qo = 2 * T * HQ * D * eb;
  double one;
  const double stage = 16384 / (2 * D * eb), mem = (R * mean * own * kv + qo) / 5.6e6 + R * mean * pre * kv / 12e6;
  if (pl.small) {
    one = 8 + std::max((own + pre) / (8 * stage) * (f32 ? 4 : 2.4), mem);
  } else {
    const double items = R * H * pl.tiles, rounds = std::ceil(items / (3 * cus));
    const double lat = f32 ? 1.4 : rows->max_query_rows * HQ / H <= 64 ? 0.55 : 0.75;
    one = 8 + 4 * rounds + std::max({rounds * (own + pre) / stage * lat, mem, (flops_own + flops_pre) / rate});
  }
  const double cuts = std::min(pl.runs / (R * pl.tiles), own / parrot::tree_unit(p->dtype, p->head_dim) / pl.min_run);
  const double pieces = pre > 0 ? 1 + cuts + pl.max_depth * std::ceil(mean * p->max_prefix_len / pl.cp)
                                : cuts < 1 ? 2 * cuts : 1 + cuts;
  const double rest = flops_pre / rate + T * HQ * D * 8 * pieces / 4.7e6 + (pre > 0 ? 8 : 0);
  double split;
  if (pl.sets) {
    const double waves = std::max((R * mean * own * kv + qo) / 6.4e6, flops_own / rate);
    split = std::max(kTreeSplitLeast, 12 + 3 * std::ceil(R * H / (4 * cus)) + waves + rest);
  } else {
    const double cols = rows->max_query_rows * HQ / H, fill = f32 ? pl.tiles * parrot::tree_cols(p->dtype) / cols : 1;
    split = (f32 ? 36 : 14) + 8 * std::ceil(R * H * pl.tiles / pl.own_wgs) +
            std::max((pl.tiles * R * mean * own * kv + qo) / 6e6, flops_own * fill / rate) + rest;
  }
  *never = one <= kTreeSplitLeast;
  return std::max(split, kTreeSplitLeast) < one;
}

parrot_status check_tree(const parrot_problem* p, const parrot_tree_rows* rows, bool nested, TreePlan* pl) {
  PARROT_TRY(parrot::check_problem_fields(p));
  PARROT_TRY(check_tree_counts(p->num_requests, rows));
  *pl = TreePlan{};
  const long T = rows->num_query_rows;
  if (T == 0) return PARROT_OK;
  if (rows->max_query_rows > p->max_suffix_len)
    return bad("max_query_rows %ld > max_suffix_len %ld", rows->max_query_rows, p->max_suffix_len);
  if (rows->num_query_heads < 1 || rows->num_query_heads % p->num_heads != 0)
    return bad("num_query_heads %ld is not a multiple of num_heads %ld", rows->num_query_heads, p->num_heads);
  if (p->num_groups > 0 && (rows->max_group_rows < 0 || rows->max_group_rows > T))
    return bad("max_group_rows %ld not in [0, num_query_rows]", rows->max_group_rows);
  if (T * rows->num_query_heads > 0x7fffffffL)
    return set_error(PARROT_ERR_UNSUPPORTED, "num_query_rows * num_query_heads > 2^31 - 1");
  const long G = rows->num_query_heads / p->num_heads;
  // (the plan is that of nested calls for flat ones too, so that one workspace serves both)
  pl->max_depth = p->num_groups > 0 ? std::max(1, (int)p->max_prefix_depth) : 0;
  pl->depth = nested ? pl->max_depth : std::min(pl->max_depth, 1);
  pl->tiles = (int)ceil_div(rows->max_query_rows * G, parrot::tree_cols(p->dtype));
  const long H = p->num_heads, R = p->num_requests, cus = parrot::device_cus(), cols = parrot::tree_cols(p->dtype);
  if (ceil_div(R * H, 8) * 8 * pl->tiles > 0x7fffffffL)
    return set_error(PARROT_ERR_UNSUPPORTED, "tree decode needs too many workgroups");
  // The split plan (figures here and below: 32 heads of 128 in bfloat16 but where it says
  // fp32, no other tokens, a query head for each).  Prefix chunks are as long as their workgroups still fill the device
  // (a chunk more costs a tile 64 KB of partial results, written and read: 48 requests of 48 rows,
  // eight on each of six prefixes of 2304 tokens, take 156 us in one chunk; at an earlier step 179 in one,
  // 199 in two, 237 in five),
  // but not so long that the last ones run alone (8 requests of 48 rows on one of 8192 tokens: 126
  // us in chunks of 4096, 98 of 2048, 111 of 1024).  A group has at most tiles_p tiles, all
  // of them together a tile each beyond what their rows fill.
  const long mg = p->num_groups > 0 ? rows->max_group_rows : 0;
  pl->tiles_p = (int)ceil_div(mg * G, cols);
  pl->cp = kTreeChunkMax;
  if (pl->tiles_p > 0) {
    const long tiles = std::min(p->num_groups * (long)pl->tiles_p, ceil_div(T * pl->max_depth * G, cols) + p->num_groups);
    while (pl->cp > kTreeChunkMin && tiles * H * ceil_div(p->max_prefix_len, pl->cp) < cus * 3 / 2) pl->cp /= 2;
    const long chunks = std::max(1L, ceil_div(p->max_prefix_len, pl->cp));       // of equal length
    pl->cp = (int)(std::max(1L, ceil_div(p->max_prefix_len, chunks * 64)) * 64);
    pl->seg_p = (int)ceil_div(p->max_prefix_len, pl->cp);
    pl->n_pre = ceil_div((long)p->num_groups * pl->seg_p * H, 8) * 8 * pl->tiles_p;
  }
  if (pl->seg_p > 0xffff) return set_error(PARROT_ERR_UNSUPPORTED, "tree decode: %ld prefix chunks", (long)pl->seg_p);
  pl->seg_pre = pl->max_depth * pl->seg_p;
  // Own tokens: requests of at most 32 columns go by waves, each with a run of its own.
  // Four waves a CU read fastest (8 requests of 16 rows on 9600 tokens: 217 us, 235 with
  // eight, 246 with twelve; with three 212, but 96 requests on 800 tokens 237 for 228).
  // Tiles: two workgroups per CU (8 requests of 64 and 128 rows on 9600 tokens: 239 and 257
  // us; 216 and 280 with one, 261 and 279 with three), three where a request may have several
  // tiles and the products bound it, and for fp32 (32 requests of 20 rows on 4000 tokens: 1411
  // us with two, 1107 with three; one launch, which such calls take, 845).
  const long most_cols = rows->max_query_rows * G;
  // (fp32 caches with two column sets spill: 32 requests of 20 rows on 1000 tokens 440 us, by
  // tiles 295).
  const OwnRole own = own_role((int)p->dtype, H, most_cols, cus);
  pl->sets = own.sets;
  pl->small = pl->sets == 1 && parrot::tree_small_rows(p->dtype, p->head_dim) && R * H <= cus;
  pl->own_wgs = own.wgs;
  pl->runs = own.runs;
  pl->piece_cols = own.piece_cols;
  pl->min_run = kTreeMinRun;
  const long units = ceil_div(p->max_suffix_len, parrot::tree_unit(p->dtype, p->head_dim));
  // the longer items start first, so that the short ones fill up (those
  // on six prefixes of 2304 tokens: 167 us, 182 with the own tokens first, at that step)
  pl->pre_first = (double)R * pl->tiles * units / pl->runs < (double)pl->cp / parrot::tree_unit(p->dtype, p->head_dim);
  const long seg = pl->seg_pre + std::min(ceil_div(units, pl->min_run) + 1, (long)pl->runs);
  const double cost = (double)R * pl->tiles * (units + parrot::kTreeSetup);
  // slots of the own tokens, by this call's columns and by fewer
  const auto own_slots = [&](const OwnRole& o) { return (double)H * (o.runs + (double)R * o.tiles) * o.piece_cols; };
  double own_most = own_slots(own);
  for (const long c : {16L, 32L, cols})
    if (c < most_cols) own_most = std::max(own_most, own_slots(own_role((int)p->dtype, H, c, cus)));
  pl->held = pl->seg_pre > 0 ? std::min(T, p->num_groups * mg) : 0;
  const double pre_slots = (double)pl->held * rows->num_query_heads * pl->seg_pre, pre_most = prefix_slot_bound(p, rows, pl->held, pl->max_depth, cus);
  if ((pl->own_wgs + pl->n_pre) * 256 > 0xffffffffL || ceil_div(R * H, 8) * 8 * pl->tiles * 512 > 0xffffffffL || cost > 1.5e9 || (own_most + std::max(pre_slots, pre_most)) * p->head_dim > 1e18)
    return set_error(PARROT_ERR_UNSUPPORTED, "tree decode: %.3g units of own tokens", cost);
  pl->seg = (int)seg;
  pl->pieces = (int)(pl->runs + R * pl->tiles);
  pl->own0 = (size_t)pre_slots;
  pl->slots = pl->own0 + (size_t)own_slots(own);
  bool never = false;
  pl->split = tree_splits(p, rows, *pl, cus, &never);
  if (g_tree_path >= 0) { pl->split = g_tree_path == 1; never = !pl->split; }
  const auto bytes = [&](size_t slots) {
    return align256(slots * p->head_dim * sizeof(float)) + align256(slots * sizeof(float)) + align256((size_t)T * parrot::kTreeDesc * sizeof(int32_t));
  };
  pl->o_bytes = align256(pl->slots * p->head_dim * sizeof(float));
  pl->lse_bytes = align256(pl->slots * sizeof(float));
  pl->total_bytes = never ? 256 : bytes((size_t)own_most + (size_t)pre_most);
  pl->used_bytes = pl->split ? bytes(pl->slots) : 0;
  if (pl->used_bytes > pl->total_bytes)
    return set_error(PARROT_ERR_UNSUPPORTED, "tree decode: the plan needs %zu bytes of %zu", pl->used_bytes, pl->total_bytes);
  return PARROT_OK;
}

parrot_status record_none(const parrot_trace& tr, hipStream_t s) {
  for (void* e : {tr.merge_start, tr.merge_stop})
    if (e && hipEventRecord(ev(e), s) != hipSuccess) return set_error(PARROT_ERR_HIP, "hipEventRecord failed");
  return set_error(PARROT_OK, "");
}

}  // namespace

extern "C" {

size_t parrot_tree_workspace_bytes(const parrot_problem* p, const parrot_tree_rows* rows) {
  TreePlan pl;
  if (check_tree(p, rows, true, &pl) != PARROT_OK) return (size_t)-1;
  set_error(PARROT_OK, "");
  return pl.total_bytes;
}

parrot_status parrot_shared_prefix_tree_decode(
    const parrot_problem* p, const parrot_tree_rows* rows, const void* q, const int32_t* query_offsets,
    const int32_t* tree_parents, const void* prefix_k, const void* prefix_v, const void* suffix_k,
    const void* suffix_v, const int32_t* prefix_block_tables, const int32_t* prefix_lens,
    const int32_t* prefix_parents, const int32_t* suffix_block_tables, const int32_t* suffix_lens,
    const int32_t* group_ids, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream,
    const parrot_trace* trace) {
  TreePlan pl;
  PARROT_TRY(check_tree(p, rows, prefix_parents != nullptr, &pl));
  if (rows->num_query_rows == 0) return set_error(PARROT_OK, "");
  const parrot::PtrCheck need[] = {
      {q, "q", 16}, {query_offsets, "query_offsets", 4}, {suffix_k, "suffix_k", 16}, {suffix_v, "suffix_v", 16},
      {suffix_block_tables, "suffix_block_tables", 4}, {suffix_lens, "suffix_lens", 4}, {group_ids, "group_ids", 4},
      {out, "out", 16}, {lse, "lse", 4}, {workspace, "workspace", 256}};
  PARROT_TRY(parrot::check_pointers(need));
  if (tree_parents && reinterpret_cast<uintptr_t>(tree_parents) % 4) return bad("tree_parents is not 4-byte aligned");
  if (p->num_groups > 0) {
    const parrot::PtrCheck pre[] = {{prefix_k, "prefix_k", 16}, {prefix_v, "prefix_v", 16},
                                    {prefix_block_tables, "prefix_block_tables", 4}, {prefix_lens, "prefix_lens", 4}};
    PARROT_TRY(parrot::check_pointers(pre));
    if (prefix_parents && reinterpret_cast<uintptr_t>(prefix_parents) % 4)
      return bad("prefix_parents is not 4-byte aligned");
  }
  if (workspace_bytes < pl.total_bytes)
    return set_error(PARROT_ERR_WORKSPACE_TOO_SMALL, "workspace is %zu bytes, need %zu", workspace_bytes, pl.total_bytes);

  parrot::TreeArgs a{};
  a.q = q; a.pk = prefix_k; a.pv = prefix_v; a.sk = suffix_k; a.sv = suffix_v;
  a.ptab = prefix_block_tables; a.plen = prefix_lens; a.stab = suffix_block_tables; a.slen = suffix_lens;
  a.gid = group_ids; a.parents = p->num_groups > 0 ? prefix_parents : nullptr;
  a.qoff = query_offsets; a.tree = tree_parents;
  a.out = out; a.lse = lse;
  a.T = rows->num_query_rows; a.R = p->num_requests; a.H = p->num_heads;
  a.G = rows->num_query_heads / p->num_heads; a.NG = p->num_groups; a.depth = pl.depth;
  a.pstride = p->prefix_table_stride; a.sstride = p->suffix_table_stride;
  a.max_p = p->max_prefix_len; a.max_s = p->max_suffix_len; a.max_q = rows->max_query_rows;
  a.npblk = p->num_groups > 0 ? p->num_prefix_blocks : 1; a.nsblk = p->num_suffix_blocks;
  a.tiles = pl.tiles;
  a.scale_log2 = p->sm_scale * parrot::kLog2e;
  a.cp = pl.cp; a.tiles_p = pl.tiles_p; a.seg = pl.seg; a.seg_p = pl.seg_p; a.seg_pre = pl.seg_pre;
  a.sets = pl.sets; a.own_wgs = pl.own_wgs; a.runs = pl.runs; a.min_run = pl.min_run; a.n_pre = (int)pl.n_pre;
  a.first = pl.pre_first ? a.n_pre : 0;
  a.o_part = reinterpret_cast<float*>(workspace);
  a.lse_part = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + pl.o_bytes);
  a.desc = reinterpret_cast<int*>(reinterpret_cast<char*>(workspace) + pl.o_bytes + pl.lse_bytes);
  a.own0 = pl.own0; a.held = (int)pl.held; a.pieces = pl.pieces; a.piece_cols = pl.piece_cols;
  const parrot_trace none = {nullptr, nullptr, nullptr, nullptr};
  const parrot_trace& tr = trace ? *trace : none;
  const int dt = (int)p->dtype, D = p->head_dim;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (!pl.split) {
    PARROT_TRY(launched(parrot::launch_tree(a, pl.small, dt, D, s, ev(tr.partials_start), ev(tr.partials_stop)), "tree kernel"));
    return record_none(tr, s);
  }
  PARROT_TRY(launched(parrot::launch_tree_partials(a, dt, D, s, ev(tr.partials_start), ev(tr.partials_stop)),
                      "tree partials kernel"));
  return launched(parrot::launch_tree_join(a, dt, D, s, ev(tr.merge_start), ev(tr.merge_stop)), "tree join kernel");
}

parrot_status parrot_validate_tree_inputs(
    const parrot_problem* p, const parrot_tree_rows* rows, const int32_t* query_offsets,
    const int32_t* tree_parents, const int32_t* prefix_block_tables, const int32_t* prefix_lens,
    const int32_t* prefix_parents, const int32_t* suffix_block_tables, const int32_t* suffix_lens,
    const int32_t* group_ids, int32_t* scratch, void* stream) {
  TreePlan pl;
  PARROT_TRY(check_tree(p, rows, prefix_parents != nullptr, &pl));
  if (rows->num_query_rows == 0) return set_error(PARROT_OK, "");
  const parrot_prefill_rows as_prefill = {rows->num_query_rows, rows->max_query_rows, rows->max_group_rows};
  const parrot::ValidateTree tree = {tree_parents};
  return parrot::validate_inputs(p, prefix_block_tables, prefix_lens, prefix_parents, suffix_block_tables,
                                 suffix_lens, group_ids, scratch, stream, &as_prefill, query_offsets, &tree);
}

// Test hooks (not in parrot_attn.h): the path of this thread's tree calls (see
// g_tree_path; -1 gives the choice back), the path these arguments take (-1: invalid), and
// their kernel: one launch by a tile (0) or by waves that share the keys (1), partial results
// by tiles (2) or by waves of one or two column sets (3, 4).
void parrot_test_tree_path(int path) { g_tree_path = path == 0 || path == 1 ? path : -1; }
int parrot_test_tree_split(const parrot_problem* p, const parrot_tree_rows* rows, int nested) {
  TreePlan pl;
  return check_tree(p, rows, nested != 0, &pl) == PARROT_OK ? pl.split : -1;
}
int parrot_test_tree_kernel(const parrot_problem* p, const parrot_tree_rows* rows, int nested) {
  TreePlan pl;
  if (check_tree(p, rows, nested != 0, &pl) != PARROT_OK) return -1;
  return pl.split ? 2 + pl.sets : pl.small ? 1 : 0;
}
// Bytes of workspace that the plan of these arguments writes.
size_t parrot_test_tree_used_bytes(const parrot_problem* p, const parrot_tree_rows* rows, int nested) {
  TreePlan pl;
  return check_tree(p, rows, nested != 0, &pl) == PARROT_OK ? pl.used_bytes : (size_t)-1;
}
// The slots that the join reads for a row's descriptor into out[0 .. most): how many.
int parrot_test_tree_slots(uint32_t lo, uint32_t hi, int own, int seg_p, int seg_pre, int seg, int* out, int most) {
  const parrot::TreeSlots s = parrot::tree_slots(lo, hi, own, seg_p, seg_pre, seg);
  for (int i = 0; i < s.n && i < most; ++i) out[i] = s.slot(i);
  return s.n;
}

// --------------------------------------------------------- accept and commit
parrot_status parrot_tree_accept(
    int32_t num_requests, const parrot_tree_rows* rows, const int32_t* query_offsets, const int32_t* tree_parents,
    const int32_t* draft_tokens, const int32_t* target_tokens, const int32_t* root_tokens, int32_t* accept_rows,
    int32_t* accept_lens, int32_t* next_tokens, void* stream, const parrot_trace* trace) {
  if (num_requests < 0) return bad("num_requests %ld < 0", num_requests);
  PARROT_TRY(check_tree_counts(num_requests, rows));
  if (num_requests == 0) return set_error(PARROT_OK, "");
  const parrot::PtrCheck need[] = {{query_offsets, "query_offsets", 4}, {root_tokens, "root_tokens", 4},
                                   {accept_lens, "accept_lens", 4}, {next_tokens, "next_tokens", 4}};
  PARROT_TRY(parrot::check_pointers(need));
  if (rows->num_query_rows > 0) {
    const parrot::PtrCheck more[] = {{draft_tokens, "draft_tokens", 4}, {target_tokens, "target_tokens", 4},
                                     {accept_rows, "accept_rows", 4}};
    PARROT_TRY(parrot::check_pointers(more));
    if (tree_parents && reinterpret_cast<uintptr_t>(tree_parents) % 4) return bad("tree_parents is not 4-byte aligned");
  }
  const void* outs[] = {accept_rows, accept_lens, next_tokens};
  const void* ins[] = {query_offsets, tree_parents, draft_tokens, target_tokens, root_tokens};
  for (const void* o : outs)
    for (const void* i : ins)
      if (o && o == i) return bad("an output array is also an input");
  parrot::AcceptArgs a{};
  a.qoff = query_offsets; a.parents = tree_parents; a.draft = draft_tokens; a.target = target_tokens;
  a.root = root_tokens; a.rows = accept_rows; a.lens = accept_lens; a.next = next_tokens;
  a.R = num_requests; a.T = rows->num_query_rows; a.max_q = rows->num_query_rows > 0 ? rows->max_query_rows : 0;
  return launched(parrot::launch_accept(a, reinterpret_cast<hipStream_t>(stream),
                                        trace ? ev(trace->partials_start) : nullptr,
                                        trace ? ev(trace->partials_stop) : nullptr),
                  "accept kernel");
}

parrot_status parrot_tree_commit(
    const parrot_problem* p, const parrot_tree_rows* rows, const int32_t* query_offsets, const int32_t* accept_rows,
    const int32_t* accept_lens, const int32_t* suffix_block_tables, const int32_t* suffix_lens, void* suffix_k,
    void* suffix_v, int32_t* committed_lens, void* stream, const parrot_trace* trace) {
  PARROT_TRY(parrot::check_problem_fields(p));
  PARROT_TRY(check_tree_counts(p->num_requests, rows));
  if (p->num_requests == 0) return set_error(PARROT_OK, "");
  if (rows->num_query_rows > 0 && rows->max_query_rows > p->max_suffix_len)
    return bad("max_query_rows %ld > max_suffix_len %ld", rows->max_query_rows, p->max_suffix_len);
  const parrot::PtrCheck need[] = {{query_offsets, "query_offsets", 4}, {accept_lens, "accept_lens", 4},
                                   {suffix_block_tables, "suffix_block_tables", 4}, {suffix_lens, "suffix_lens", 4},
                                   {suffix_k, "suffix_k", 16}, {suffix_v, "suffix_v", 16},
                                   {committed_lens, "committed_lens", 4}};
  PARROT_TRY(parrot::check_pointers(need));
  if (rows->num_query_rows > 0) {
    const parrot::PtrCheck more[] = {{accept_rows, "accept_rows", 4}};
    PARROT_TRY(parrot::check_pointers(more));
  }
  if (committed_lens == suffix_lens || committed_lens == accept_lens || committed_lens == accept_rows ||
      committed_lens == query_offsets)
    return bad("committed_lens is also an input");
  if (suffix_k == suffix_v) return bad("suffix_k and suffix_v are the same pool");
  if ((long)p->num_suffix_blocks * p->block_size > 0x7fffffffL || (long)p->num_requests * ceil_div(p->num_heads, 8) > 0x7fffffffL)
    return set_error(PARROT_ERR_UNSUPPORTED, "commit: num_suffix_blocks %d or num_requests %d too large",
                     p->num_suffix_blocks, p->num_requests);
  parrot::CommitArgs a{};
  a.qoff = query_offsets; a.rows = accept_rows; a.lens = accept_lens;
  a.stab = suffix_block_tables; a.slen = suffix_lens;
  a.sk = suffix_k; a.sv = suffix_v; a.committed = committed_lens;
  a.R = p->num_requests; a.T = rows->num_query_rows; a.H = p->num_heads;
  a.sstride = p->suffix_table_stride; a.max_s = p->max_suffix_len;
  a.max_q = rows->num_query_rows > 0 ? rows->max_query_rows : 0; a.nsblk = p->num_suffix_blocks;
  return launched(parrot::launch_commit(a, (int)p->dtype, p->head_dim, reinterpret_cast<hipStream_t>(stream),
                                        trace ? ev(trace->partials_start) : nullptr,
                                        trace ? ev(trace->partials_stop) : nullptr),
                  "commit kernel");
}

}  // extern "C"
