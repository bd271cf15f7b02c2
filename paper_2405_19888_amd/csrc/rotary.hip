// Fill of new rows: per-head RMS norm of queries and keys, rotation to their
// positions, queries to q_out, keys and values into the paged cache, in one pass.
//
// Per head x of a query or key row, with g the norm's weight (or 1) and c_e, s_e
// the amplitude times cosine and sine of the angle of element e's pair,
//   y_e = (x_e g_e c_e -/+ x_p g_p s_e) / sqrt(mean(x^2) + eps),  p the pair's other element
// in fp32, rounded once.  Everything is read once and written once (but for halves whose
// partners no 16 bytes line up with, below), so the call is bound by memory: 7500 rows of 96 16-bit heads of 128, normalised and rotated in halves,
// 369 MB, take 73 us (5.1 TB/s; a large copy reaches 4.7, without the 256 MB cache
// that holds part of what was just written); fp32, 738 MB, 147 us.
//
// Angles: position n turns pair i by n f_i.  In fp32 that product is off by 0.006
// radians at n = 100000, so f_i / (2 pi) comes as a 64-bit binary fraction of a turn:
// the integer product n * turns_i wraps modulo a turn by itself and its top 32 bits
// are the angle to 2^-32 turns.  Two bits choose the quadrant; the rest, at most an
// eighth of a turn, goes through the Taylor series of sine and cosine up to x^9 and
// x^10 (truncation below 2e-9).
//
// Layout: 16 bytes of one head per lane, D * elt / 16 lanes a head, so a workgroup
// takes 8 to 32 heads a step; it owns one row, or a slab of a row's heads when rows are
// few.  A row's cache slot takes about four dependent round trips (request, length,
// table entry): one wave finds it, another one turns the pairs, once per row, and the
// first two steps' data are requested before.  Partners in other lanes come by a
// lane exchange after the norm, so a lane keeps 16 factors, and eight waves fit a SIMD.
// (Before, a lane turned its own pairs and kept the products with both norms' weights: its
// registers left five waves a SIMD, and those rows took 113 us, 139 with three steps ahead
// and four waves; 1500 rows of 48 heads 14.7 and 17.9 us for 11.0.  Two rows a
// workgroup: as long, and 12.3 us.)
//
// kRotaryHalfScalar (half layout, RD / 2 no multiple of a lane's 16 bytes: RD = 20, 50): a lane
// reads each partner, and its weight, again from the caches, 2 or 4 bytes at a time: the rows
// above take 197 us with RD = 20 and 175 with RD = 50, 78 with 128; 1500 rows of 48 heads 27
// for 12.
#include "draft_args.h"

namespace parrot {

// cosine and sine of 2 pi * phase / 2^32
PARROT_DEV void cos_sin_turns(unsigned phase, float* c, float* s) {
  const unsigned quad = (phase + 0x20000000u) >> 30;             // nearest quarter turn
  const int rest = (int)(phase - (quad << 30));                  // [-2^29, 2^29)
  const float x = (float)rest * 1.4629180792671596e-9f;          // 2 pi / 2^32
  const float z = x * x;
  float sn = 2.7557319e-6f;                                      // 1/9!
  sn = __builtin_fmaf(sn, z, -1.9841270e-4f);
  sn = __builtin_fmaf(sn, z, 8.3333333e-3f);
  sn = __builtin_fmaf(sn, z, -1.6666667e-1f);
  sn = __builtin_fmaf(sn * z, x, x);
  float cs = -2.7557319e-7f;                                     // -1/10!
  cs = __builtin_fmaf(cs, z, 2.4801587e-5f);
  cs = __builtin_fmaf(cs, z, -1.3888889e-3f);
  cs = __builtin_fmaf(cs, z, 4.1666667e-2f);
  cs = __builtin_fmaf(cs, z, -0.5f);
  cs = __builtin_fmaf(cs, z, 1.0f);
  const float a = (quad & 1) ? sn : cs, b = (quad & 1) ? cs : sn;
  *c = ((quad + 1) & 2) ? -a : a;                                // quadrants 1, 2: cosine negative
  *s = (quad & 2) ? -b : b;                                      // quadrants 2, 3: sine negative
}

template <int DT>
PARROT_DEV float load_elem(const char* p) {
  if constexpr (DT == kF32) return *reinterpret_cast<const float*>(p);
  else if constexpr (DT == kF16) return (float)*reinterpret_cast<const _Float16*>(p);
  else return __uint_as_float((unsigned)*reinterpret_cast<const unsigned short*>(p) << 16);
}

template <int DT>
PARROT_DEV u32x4 pack16(const float* f) {
  if constexpr (DT == kF32) {
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  } else if constexpr (DT == kF16) {
    f16x8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (_Float16)f[i];
    return __builtin_bit_cast(u32x4, h);
  } else {
    bf16x8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (__bf16)f[i];
    return __builtin_bit_cast(u32x4, h);
  }
}

constexpr int kAhead = 2;                     // steps requested ahead

template <int DT, int D, int PARTNER>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(PARTNER == kRotaryHalfScalar ? 4 : 8)))
void k_rotary_fill(FillArgs a) {
  using E = Elem<DT>;
  constexpr int EB = E::kBytes, EPL = E::kPerLoad;
  constexpr int LPH = D * EB / 16;            // lanes per head
  constexpr int HPS = 256 / LPH;              // heads per workgroup and step
  __shared__ float turn_c[kRotaryPairs], turn_s[kRotaryPairs];
  __shared__ long row_slot;                   // -1: padding
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x / a.slabs, slab = blockIdx.x % a.slabs;
  const int sub = threadIdx.x % LPH;
  const int e0 = sub * EPL;                   // the lane's first element
  const int half = a.rd >> 1;

  // a step is HPS heads of the slab, 16 bytes of one per lane
  const int heads = a.HQ + 2 * a.H;
  const int begin = slab * a.slab_heads, end = min(begin + a.slab_heads, heads);
  const int steps = (end - begin + HPS - 1) / HPS;
  const int x0h = begin + (int)threadIdx.x / LPH;
  auto source = [&](int x) {                  // (past the slab: its last head, unused)
    x = min(x, end - 1);
    const int h = x < a.HQ ? x : x < a.HQ + a.H ? x - a.HQ : x - a.HQ - a.H;
    const char* row = x < a.HQ ? (const char*)a.q + t * a.q_stride
                    : x < a.HQ + a.H ? (const char*)a.k + t * a.k_stride : (const char*)a.v + t * a.v_stride;
    return row + (size_t)h * (D * EB);
  };
  u32x4 raw[kAhead];
  auto request = [&](int st, u32x4& to) {
    if (st < steps) to = ld16(source(x0h + st * HPS) + sub * 16);
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) request(i, raw[i]);

  // wave 0: the row's cache slot; wave 1: the cosines and sines of its pairs
  if (PARTNER != kRotaryNone && wave == 1 && lane < half) {
    float c, s;
    cos_sin_turns((unsigned)((a.turns[lane] * (unsigned long long)(long long)a.positions[t]) >> 32), &c, &s);
    turn_c[lane] = c * a.amplitude;
    turn_s[lane] = s * a.amplitude;
  }
  if (wave == 0) {
    long slot = -1;
    const int r = __builtin_amdgcn_readfirstlane(request_of_row(a.qoff, a.R, t, lane));
    if (r >= 0) {
      const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
      const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
      if (t >= rw.first && t < rw.first + rw.count) {
        const int own = S - rw.count + (t - rw.first);
        const int blk = clampi(ld_uniform(a.stab + (long)r * a.sstride + own / kBlock), 0, a.nsblk - 1);
        slot = ((long)blk * a.H * kBlock + own % kBlock) * (D * EB);          // head 0
      }
    }
    if (lane == 0) row_slot = slot;
  }
  const u32x4 zero = {0u, 0u, 0u, 0u};
  const u32x4 wq = a.q_norm ? ld16((const char*)a.q_norm + e0 * EB) : zero;
  const u32x4 wk = a.k_norm ? ld16((const char*)a.k_norm + e0 * EB) : zero;
  // bit i: the lane's element i turns
  const unsigned turns = PARTNER == kRotaryNone || e0 >= a.rd ? 0u : a.rd - e0 >= EPL ? (1u << EPL) - 1u : (1u << (a.rd - e0)) - 1u;
  const int far = !turns ? 0 : e0 >= half ? -half : half;
  const int partner = lane + far / EPL;       // (half layout: the lane that holds the partners)
  __syncthreads();

  const long slot = row_slot;
  if (slot < 0) return;                     // padding
  // cosine and signed sine of the lane's elements
  float c[EPL], s[EPL];
  if constexpr (PARTNER != kRotaryNone) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = e0 + i;
      const int pair = PARTNER == kRotaryInterleaved ? e >> 1 : e < half ? e : e - half;
      const bool second = PARTNER == kRotaryInterleaved ? (e & 1) : e >= half;
      const bool on = (turns >> i) & 1u;
      c[i] = on ? turn_c[on ? pair : 0] : 1.f;
      s[i] = on ? turn_s[on ? pair : 0] : 0.f;
      s[i] = second ? s[i] : -s[i];
    }
  }
#pragma unroll 1
  for (int st = 0; st < steps; ++st) {
    const u32x4 cur = raw[0];
#pragma unroll
    for (int i = 0; i + 1 < kAhead; ++i) raw[i] = raw[i + 1];
    request(st + kAhead, raw[kAhead - 1]);
    const int x = x0h + st * HPS;
    const bool live = x < end;
    const int kind = x < a.HQ ? 0 : x < a.HQ + a.H ? 1 : 2;                 // query, key, value
    const int h = kind == 0 ? x : kind == 1 ? x - a.HQ : x - a.HQ - a.H;
    u32x4 res = cur;                                                        // values are copied
    if (__builtin_amdgcn_ballot_w64(kind < 2 && live)) {                    // (lanes of a head are of one kind)
      float n[EPL];
      E::to_f32(cur, n);
      const bool norm = kind == 0 ? a.q_norm != nullptr : a.k_norm != nullptr;
      float rs = 1.f, w[EPL];
      if (a.q_norm || a.k_norm) {                   // uniform: all lanes take part in the sums
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) ss = __builtin_fmaf(n[i], n[i], ss);
        ss = group_sum<LPH>(ss);
        rs = 1.f / sqrtf(ss * (1.f / D) + a.eps);
        E::to_f32(kind == 0 ? wq : wk, w);
#pragma unroll
        for (int i = 0; i < EPL; ++i) n[i] = norm ? n[i] * rs * w[i] : n[i];
      }
      float y[EPL];
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        y[i] = n[i];
        float far_n = 0.f;                          // the partner
        if constexpr (PARTNER == kRotaryInterleaved) far_n = n[i ^ 1];
        if constexpr (PARTNER == kRotaryHalfVector) far_n = __shfl(n[i], partner);
        if constexpr (PARTNER == kRotaryHalfScalar) {
          const int at = ((turns >> i) & 1u) ? (e0 + i >= half ? e0 + i - half : e0 + i + half) : e0 + i;
          far_n = load_elem<DT>(source(x) + at * EB);
          if (norm) far_n = far_n * rs * load_elem<DT>((const char*)(kind == 0 ? a.q_norm : a.k_norm) + at * EB);
        }
        // (a selection: 0 times an infinite partner is no zero)
        if constexpr (PARTNER != kRotaryNone)
          y[i] = ((turns >> i) & 1u) ? __builtin_fmaf(far_n, s[i], n[i] * c[i]) : n[i];
      }
      if (kind < 2) res = pack16<DT>(y);
    }
    char* dst = kind == 0 ? (char*)a.q_out + ((size_t)t * a.HQ + h) * (D * EB)
                          : (char*)(kind == 1 ? a.sk : a.sv) + slot + (size_t)h * (kBlock * D * EB);
    if (live) *reinterpret_cast<u32x4*>(dst + sub * 16) = res;
  }
}

template <int DT, int D>
static hipError_t launch_fill_t(const FillArgs& a, int partner, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const dim3 grid((unsigned)((long)a.T * a.slabs)), wg(256);
  switch (partner) {
    case kRotaryNone: hipExtLaunchKernelGGL((k_rotary_fill<DT, D, kRotaryNone>), grid, wg, 0, s, e0, e1, 0, a); break;
    case kRotaryInterleaved:
      hipExtLaunchKernelGGL((k_rotary_fill<DT, D, kRotaryInterleaved>), grid, wg, 0, s, e0, e1, 0, a);
      break;
    case kRotaryHalfVector:
      hipExtLaunchKernelGGL((k_rotary_fill<DT, D, kRotaryHalfVector>), grid, wg, 0, s, e0, e1, 0, a);
      break;
    default: hipExtLaunchKernelGGL((k_rotary_fill<DT, D, kRotaryHalfScalar>), grid, wg, 0, s, e0, e1, 0, a);
  }
  return hipGetLastError();
}

hipError_t launch_fill(const FillArgs& a, int partner, int dtype, int D, hipStream_t s, hipEvent_t e0,
                       hipEvent_t e1) {
  if (a.T < 1 || a.R < 1 || a.H < 1 || a.HQ < 0 || a.slabs < 1 || a.sstride < 1 || a.nsblk < 1 ||
      (long)a.slabs * a.slab_heads < a.HQ + 2L * a.H || (long)a.T * a.slabs > 0x7fffffffL || a.rd > D || a.rd > 2 * kRotaryPairs ||
      (partner != kRotaryNone && !a.positions))
    return hipErrorInvalidValue;
  switch (dtype * 1000 + D) {
    case kF32 * 1000 + 64: return launch_fill_t<kF32, 64>(a, partner, s, e0, e1);
    case kF32 * 1000 + 128: return launch_fill_t<kF32, 128>(a, partner, s, e0, e1);
    case kF16 * 1000 + 64: return launch_fill_t<kF16, 64>(a, partner, s, e0, e1);
    case kF16 * 1000 + 128: return launch_fill_t<kF16, 128>(a, partner, s, e0, e1);
    case kBF16 * 1000 + 64: return launch_fill_t<kBF16, 64>(a, partner, s, e0, e1);
    case kBF16 * 1000 + 128: return launch_fill_t<kBF16, 128>(a, partner, s, e0, e1);
  }
  return hipErrorInvalidValue;
}

}  // namespace parrot
