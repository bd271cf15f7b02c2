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

template <int DT, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void k_tree_decode(TreeArgs a) {
  constexpr int COLS = tree_detail::kCols<DT>;
  __shared__ __attribute__((aligned(1024))) tree_detail::Lds<DT> lds;
  // a sequence's column tiles read the same keys: they are 8 workgroups apart, on one XCD
  const int idx = (int)(blockIdx.x / (8 * a.tiles)) * 8 + (int)(blockIdx.x % 8);
  const int col0 = (int)(blockIdx.x / 8 % a.tiles) * COLS;
  if (idx >= a.R * a.H) return;
  const int r = idx / a.H, h = idx % a.H;
  const int S = clampi(a.slen[r], 0, a.max_s);
  const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
  const int ncols = min(COLS, rw.count * a.G - col0);
  if (ncols <= 0) return;
  const int base = S - rw.count;
  const int HQ = a.H * a.G;

  TreeTile<DT, D> tile(lds, a.H, h, a.scale_log2);
  auto row_of = [&](int col) {                              // in units of heads
    const int x = col0 + col;
    return (size_t)(rw.first + x / a.G) * HQ + h * a.G + x % a.G;
  };
  tile.load_queries(a.q, ncols, row_of);
  build_masks<DT, D>(a, lds, rw, base, col0, ncols);

  int g = a.gid[r];
  for (int l = 0; l < a.depth && g >= 0 && g < a.NG; ++l) {
    const int P = clampi(a.plen[g], 0, a.max_p);
    tile.run(TreeRange{a.pk, a.pv, a.ptab + (long)g * a.pstride, a.npblk, 0, P, 0x40000000, P, P});
    g = a.parents ? a.parents[g] : -1;
  }
  tile.run(TreeRange{a.sk, a.sv, a.stab + (long)r * a.sstride, a.nsblk, 0, S, base & ~31, base, S});

  tile.finish([&](int c, int col, float lw, float lse2, float) {
    if (col >= ncols) return;
    const size_t at = row_of(col);
    const int d0 = 4 * (tile.lane >> 4);
    const float inv = 1.f / lw;            // (0 only where every logit is -inf: the result is NaN)
    char* dst = (char*)a.out + (at * D + d0) * Elem<DT>::kBytes;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      const f32x4 v = tile.o[c][dt] * inv;
      if constexpr (DT == kF32) *reinterpret_cast<f32x4*>(dst + dt * 64) = v;
      else store4<DT>(dst + dt * 32, v);
    }
    if (tile.lane < 16) a.lse[at] = lse2 * kLn2;
  });
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

}  // namespace parrot
