// After a tree of drafted tokens was verified: which of them a greedy model agrees
// with (accept), and the move of their keys and values into cache order (commit).
//
// Both are bound by latency: a launch and a few dependent round trips; commit moves
// 4 * D * H * elt bytes per token that is not in place already.
#include "draft_args.h"

namespace parrot {

// Accept: one wave per request, up to two rows per lane.  A step of the walk is a
// vote over the rows whose parent is the row reached last and whose token is the
// one wanted; the lowest such row is the next.  Rows come after their parents, so
// the row index grows at every step and the walk ends.
__global__ __launch_bounds__(64) void k_tree_accept(AcceptArgs a) {
  constexpr int NR = kTreeRows / kWave;
  const int lane = threadIdx.x;
  const int r = blockIdx.x;
  int want = ld_uniform(a.root + r);
  const RowSpan rw = row_span(a.qoff, r, a.T, a.max_q);
  int parent[NR], draft[NR], target[NR], taken[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const int j = lane + k * kWave;
    const bool in = j < rw.count;
    const int t = rw.first + (in ? j : 0);
    parent[k] = !in ? -2 : a.parents ? a.parents[t] : j - 1;
    draft[k] = in ? a.draft[t] : 0;
    target[k] = in ? a.target[t] : 0;
    taken[k] = -1;
  }
  int at = -1, len = 0;
  for (;;) {
    int next = -1;
#pragma unroll
    for (int k = NR - 1; k >= 0; --k) {
      const int j = lane + k * kWave;
      const unsigned long long fit = __ballot(parent[k] == at && draft[k] == want && j > at);
      if (fit) next = k * kWave + __ffsll((long long)fit) - 1;
    }
    if (next < 0) break;
    at = next;
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      if (next / kWave == k) want = __builtin_amdgcn_readlane(target[k], next % kWave);
      if (len == lane + k * kWave) taken[k] = next;
    }
    ++len;
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const int j = lane + k * kWave;
    if (j < rw.count) a.rows[rw.first + j] = taken[k];
  }
  if (lane == 0) {
    a.lens[r] = len;
    a.next[r] = want;
  }
}

hipError_t launch_accept(const AcceptArgs& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (a.R < 1 || a.T < 0 || a.max_q < 0 || a.max_q > kTreeRows) return hipErrorInvalidValue;
  hipExtLaunchKernelGGL(k_tree_accept, dim3((unsigned)a.R), dim3(64), 0, s, e0, e1, 0, a);
  return hipGetLastError();
}

// Commit: a workgroup per (request, 8 heads of K and of V).  The moved row of slot i
// is a_i >= i, so taking the slots in order, a batch at a time, with all reads of a
// batch before its writes, never reads a slot that was written already: later
// batches read slots a_j >= j behind all written ones.
template <int DT, int D>
__global__ __launch_bounds__(256) void k_tree_commit(CommitArgs a) {
  constexpr int ROW_B = D * Elem<DT>::kBytes;
  constexpr int LPH = ROW_B / 16;                 // lanes per piece (one token, head and tensor)
  constexpr int PPS = 256 / LPH;                  // pieces per workgroup and step
  constexpr int BATCH = 4;                        // steps whose reads are in flight together
  __shared__ int s_from[kTreeRows];               // byte offsets would pass 32 bits: block * 16 + slot
  __shared__ int s_to[kTreeRows];
  __shared__ int s_n;
  const int slabs = (a.H + 7) / 8;
  const int r = blockIdx.x / slabs, slab = blockIdx.x % slabs;
  const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
  const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
  const int m = clampi(ld_uniform(a.lens + r), 0, rw.count);
  const int cached = S - rw.count;
  if (slab == 0 && threadIdx.x == 0) a.committed[r] = cached + m;
  // the moves, in slot order without those in place: two rows per lane of wave 0
  if (threadIdx.x < kWave) {
    int n = 0;
    for (int b = 0; b < m; b += kWave) {
      const int i = b + threadIdx.x;
      int from = 0, to = 0;
      bool moves = false;
      if (i < m) {
        const int row = clampi(a.rows[rw.first + i], i, rw.count - 1);
        moves = row != i;
        const int p = cached + row, d = cached + i;
        from = clampi(a.stab[(long)r * a.sstride + p / kBlock], 0, a.nsblk - 1) * kBlock + p % kBlock;
        to = clampi(a.stab[(long)r * a.sstride + d / kBlock], 0, a.nsblk - 1) * kBlock + d % kBlock;
      }
      const unsigned long long mask = __ballot(moves);
      const int at = n + __popcll(mask & ((1ull << threadIdx.x) - 1ull));
      if (moves) { s_from[at] = from; s_to[at] = to; }
      n += __popcll(mask);
    }
    if (threadIdx.x == 0) s_n = n;
  }
  __syncthreads();
  const int heads = min(8, a.H - slab * 8);
  const int per = 2 * heads;                      // pieces per token: K and V of the heads
  const int total = s_n * per;
  const int sub = threadIdx.x % LPH;
  const auto place = [&](int tok, int piece) {    // address of a piece
    const int h = slab * 8 + piece % heads;
    const size_t off = (((size_t)(tok / kBlock) * a.H + h) * kBlock + tok % kBlock) * ROW_B + sub * 16;
    return (char*)(piece < heads ? a.sk : a.sv) + off;
  };
  for (int x0 = 0; x0 < total; x0 += BATCH * PPS) {
    u32x4 v[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int x = x0 + b * PPS + threadIdx.x / LPH;
      v[b] = u32x4{0u, 0u, 0u, 0u};
      if (x < total) v[b] = ld16(place(s_from[x / per], x % per));
    }
    // every wave's reads have arrived before any wave writes
#pragma unroll
    for (int b = 0; b < BATCH; ++b) asm volatile("" : : "v"(v[b]));
    __syncthreads();
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int x = x0 + b * PPS + threadIdx.x / LPH;
      if (x < total) *reinterpret_cast<u32x4*>(place(s_to[x / per], x % per)) = v[b];
    }
  }
}

template <int DT, int D>
static hipError_t launch_commit_t(const CommitArgs& a, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const dim3 grid((unsigned)((long)a.R * ((a.H + 7) / 8)));
  hipExtLaunchKernelGGL((k_tree_commit<DT, D>), grid, dim3(256), 0, s, e0, e1, 0, a);
  return hipGetLastError();
}

hipError_t launch_commit(const CommitArgs& a, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  if (a.R < 1 || a.T < 0 || a.H < 1 || a.max_q < 0 || a.max_q > kTreeRows ||
      (a.max_q > 0 && a.sstride < 1) || a.nsblk < 1 || (long)a.nsblk * kBlock > 0x7fffffffL || (long)a.R * ((a.H + 7) / 8) > 0x7fffffffL)
    return hipErrorInvalidValue;
  switch (dtype * 1000 + D) {
    case kF32 * 1000 + 64: return launch_commit_t<kF32, 64>(a, s, e0, e1);
    case kF32 * 1000 + 128: return launch_commit_t<kF32, 128>(a, s, e0, e1);
    case kF16 * 1000 + 64: return launch_commit_t<kF16, 64>(a, s, e0, e1);
    case kF16 * 1000 + 128: return launch_commit_t<kF16, 128>(a, s, e0, e1);
    case kBF16 * 1000 + 64: return launch_commit_t<kBF16, 64>(a, s, e0, e1);
    case kBF16 * 1000 + 128: return launch_commit_t<kBF16, 128>(a, s, e0, e1);
  }
  return hipErrorInvalidValue;
}

}  // namespace parrot
