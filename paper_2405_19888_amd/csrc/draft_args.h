// Arguments of the kernels of a drafting step (fill of new rows, accept, commit),
// shared by the kernels and the host code.
#pragma once

#include "common.h"

namespace parrot {

constexpr int kRotaryPairs = 64;         // rotated pairs of a head (PARROT_ROTARY_MAX_PAIRS)
constexpr int kTreeRows = 128;           // drafted rows of a request (PARROT_MAX_TREE_ROWS)

// How a lane of the fill gets the element each of its own is paired with.
enum RotaryPartner {
  kRotaryNone = 0,       // no rotation
  kRotaryInterleaved,    // in the lane's own 16 bytes
  kRotaryHalfVector,     // 16 aligned bytes elsewhere in the head
  kRotaryHalfScalar      // unaligned: element by element
};

struct FillArgs {
  const void* q; const void* k; const void* v;   // q NULL: keys and values only
  long q_stride, k_stride, v_stride;             // bytes between rows
  const void* q_norm; const void* k_norm;        // [D] dtype or NULL
  const int* positions;
  const int* qoff; const int* stab; const int* slen;
  void* q_out; void* sk; void* sv;
  int T, R, HQ, H;                               // HQ = 0 when q is NULL
  int sstride, max_s, max_q, nsblk;
  int slabs, slab_heads;                         // workgroups per row, heads (q, k, v) of each
  int rd;                                        // rotated elements
  float eps, amplitude;
  unsigned long long turns[kRotaryPairs];
};
hipError_t launch_fill(const FillArgs& a, int partner, int dtype, int D, hipStream_t s, hipEvent_t e0,
                       hipEvent_t e1);

struct AcceptArgs {
  const int* qoff; const int* parents;           // parents NULL: chains
  const int* draft; const int* target; const int* root;
  int* rows; int* lens; int* next;
  int R, T, max_q;
};
hipError_t launch_accept(const AcceptArgs& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1);

struct CommitArgs {
  const int* qoff; const int* rows; const int* lens;
  const int* stab; const int* slen;
  void* sk; void* sv;
  int* committed;
  int R, T, H, sstride, max_s, max_q, nsblk;
};
hipError_t launch_commit(const CommitArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1);

#if defined(__HIPCC__)
// The request of row t: the last one whose first row is at or before it, or -1.
// The lanes of a wave test every step-th request, then the requests of that step: a
// round trip per factor of 64.
PARROT_DEV int request_of_row(const int* qoff, int R, int t, int lane) {
  int r = -1;
  for (int base = 0, n = R; n > 0;) {
    const int step = (n + kWave - 1) / kWave;
    const int at = lane * step;
    const int k = __popcll(__ballot(at < n && qoff[base + min(at, n - 1)] <= t));
    if (k == 0 || step == 1) { r = base + k - 1; break; }
    base += (k - 1) * step;
    n = min(step, n - (k - 1) * step);
  }
  return r;
}

// Rows of request r (wave-uniform), clamped so that every row index stays in [0, T) and
// the request has at most `most` of them.
struct RowSpan { int first, count; };
PARROT_DEV RowSpan row_span(const int* qoff, int r, int T, int most) {
  const int begin = ld_uniform(qoff + r), end = ld_uniform(qoff + r + 1);
  const int first = clampi(begin, 0, T);
  const long n = (long)end - begin;
  const int cap = min(most, T - first);
  return {first, (int)(n < 0 ? 0 : n > cap ? cap : n)};
}
#endif

}  // namespace parrot
