// Arguments of the kernels of a cache held in 8 bits, shared by the kernels and the host
// code, and the format itself.
//
// A block-head is 16 tokens of one head of one block: 16 * D codes (e4m3) of keys and as many of
// values, and a byte each for their scales: b stands for 2^(b - 127), and a value is its code
// times that.  Keys are row-major, [16][D].  Values are [D / 64][4][16][4][4]: token
// 4 g + t, element 64 x + 4 c + d at [x][g][c][d][t].
#pragma once

#include "draft_args.h"

namespace parrot {

constexpr int kBlockTokens = 16;
constexpr int kUnit = 32;                // tokens of a unit: two blocks, one k step of the PV product

struct Pool8 { const void* k; const void* v; const void* scales; };

struct Fill8Args {
  FillArgs f;                            // sk, sv: the code pools
  void* scales;                          // [nsblk][H][2]
  int units;                             // (request, block) pairs, at most
};
hipError_t launch_fill8(const Fill8Args& a, int partner, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);

// Where a plan holds what, in ints from its start.  Entries are the column tiles of sequences:
// the groups first (their columns are the rows of all requests that read the group's prefix, times
// the query heads of a cache head), then the requests (their own rows' columns), in order.
// Sequences of more than wide_from columns have tiles of wide_cols columns, which a workgroup's four
// waves take together; their entries come before the others', whose tiles a wave takes alone.  A
// request with a wide tile's columns of its own goes through its group chain by itself, in one
// piece with its own tokens, and is no reader of the groups.
struct Plan8Layout {
  long cost, entry, run, row, list, seq, req, pos, count, total;
};
constexpr int kPlanHead = 16;            // ints of the head, see Head8
constexpr int kEntryInts = 12;
constexpr int kRowInts = 12;
constexpr int kReqInts = 12;
constexpr int kPlanWaves = 16;           // waves of the planning workgroup
constexpr int kPieceSetup = 2;           // cost of a tile beside its units

// Columns of a wide tile, and columns above which a sequence has wide tiles: what one narrow tile
// holds.  bfloat16, 8 cache heads of 128 elements, four query heads on each, us for the plan and a layer with
// wide tiles and with several narrow ones: four prompts of 400 rows on 8000 tokens 282 and 445, 64 requests of ten
// rows on 3000 118 and 178, ten rows on one prefix of 16000 39 and 44; four of 400 rows on 1000 in
// float32 109 and 196.
constexpr int wide_cols(int dtype) { return dtype == kF32 ? 64 : 128; }
constexpr int wide_from(int dtype) { return wide_cols(dtype) / 4; }

// The head: entries, wide ones among them, rows to join, cost of the wide entries, cost of all, a
// cache head's workgroups of the wide role, run lengths of wide and narrow roles.
enum Head8 { kHeadEntries, kHeadWide, kHeadJoins, kHeadWideCost, kHeadCost, kHeadWideWgs, kHeadWideRun, kHeadRun };
// An entry: sequence (request r, or ~g for group), its columns [col0, col0 + ncols), cost at which it
// starts, units, first slot of its partial results (-1: it writes the output), pieces, own keys (of a
// group: its prefix's), keys that every column sees, first row (group: first place in the row
// list), whether the chain's prefixes come first.
enum Entry8 { kEntSeq, kEntCol0, kEntCols, kEntCost, kEntUnits, kEntSlot, kEntPieces, kEntKeys, kEntBase, kEntFirst, kEntChained };
// A row that is joined, in no order: its token, entry of its request's first tile, its place in the
// request, levels of prefixes, then for each level the entry of the group's first tile and the row's
// place in the group's list (-1: a prefix without tokens).
enum Row8 { kRowToken, kRowEntry, kRowPlace, kRowLevels, kRowGroup };
// A request: first row, rows, own tokens, its group where it reads groups' results (-1), then
// its chain's groups and their tokens, innermost first.
enum Req8 { kReqFirst, kReqCount, kReqKeys, kReqReads, kReqChain };

// The int arrays of a step.
struct Step8 {
  const int* qoff; const int* plen; const int* parents; const int* slen; const int* gid;
  int T, R, NG, G, depth, max_p, max_s, max_q;   // depth: levels of this call's chains
};
struct Plan8Args {
  Step8 st;
  int* plan;
  Plan8Layout at;
  int cols;                              // columns of a narrow tile
  int wide_cols, wide_from;              // of a wide tile; columns above which a sequence has wide ones
  int wgs, min_run;                      // workgroups of a cache head; cost of a run at least
  int max_entries;
};
hipError_t launch_plan8(const Plan8Args& a, hipStream_t s);

struct Attend8Args {
  const void* q;                         // [T][HQ][D]
  Pool8 pre, own;
  const int* ptab; const int* stab;
  const int* plan;
  Plan8Layout at;
  Step8 st;                              // the one launch without a plan
  void* out; float* lse;                 // [T][HQ][D] dtype, [T][HQ]
  float* o_part; float* lse_part;        // [H][slots][D] normalised, [H][slots] base 2
  long slots;
  int T, R, H, G, NG, depth;             // depth: levels that the plan has room for
  int pstride, sstride, max_p, max_s, npblk, nsblk;
  int wgs, max_entries;                  // workgroups of a cache head
  int sets, wide;                        // column sets of a narrow tile, columns of a wide one (0: the call has none)
  int tiles, waves;                      // one launch: column tiles of a request, waves of a workgroup (4 or 8)
  int flip;                              // sm_scale < 0: queries change sign
  float scale_log2;                      // |sm_scale| log2(e)
};
hipError_t launch_attend8(const Attend8Args& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
hipError_t launch_join8(const Attend8Args& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);
// One launch, without a plan: a workgroup per request, cache head and column tile.
hipError_t launch_direct8(const Attend8Args& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);

// A copy of blocks of several pools, each with its block's bytes (a multiple of 2).
constexpr int kCopyPools = 128;          // pools of one launch
struct CopyArgs {
  void* base[kCopyPools];
  unsigned bytes[kCopyPools];
  const int* src; const int* dst;
  int n, pools, blocks;
};
hipError_t launch_copy_blocks(const CopyArgs& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);

}  // namespace parrot
