// Fill of new rows: per-head RMS norm of queries and keys, rotation to their
// positions, queries to q_out, keys and values into the paged cache, in one pass.
//
// Per head x of a query or key row, with g the norm's weight (or 1) and c_e, s_e
// the amplitude times cosine and sine of the angle of element e's pair,
//   y_e = (x_e g_e c_e -/+ x_p g_p s_e) / sqrt(mean(x^2) + eps),  p the pair's other element
// in fp32, rounded once.  Everything is read once and written once, so the call is
// bound by memory; the cosines and sines of a row serve all of its heads and stay
// in registers with the weights multiplied in (c g and s g of the lane's elements).
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
// few.  A row's cache slot (request, length, table entry) takes about four
// dependent round trips; the row's data are requested beside them.
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

template <int DT, int D, int PARTNER>
__global__ __launch_bounds__(256) void k_rotary_fill(FillArgs a) {
  using E = Elem<DT>;
  constexpr int EB = E::kBytes, EPL = E::kPerLoad;
  constexpr int LPH = D * EB / 16;            // lanes per head
  constexpr int HPS = 256 / LPH;              // heads per workgroup and step
  const int lane = threadIdx.x & 63;
  const int t = blockIdx.x / a.slabs, slab = blockIdx.x % a.slabs;
  const int sub = threadIdx.x % LPH;
  const int e0 = sub * EPL;                   // the lane's first element
  const int half = a.rd >> 1;

  // the row's cache slot
  const int r = __builtin_amdgcn_readfirstlane(request_of_row(a.qoff, a.R, t, lane));
  if (r < 0) return;
  const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
  const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
  if (t < rw.first || t >= rw.first + rw.count) return;      // padding
  const int own = S - rw.count + (t - rw.first);
  const int blk = clampi(ld_uniform(a.stab + (long)r * a.sstride + own / kBlock), 0, a.nsblk - 1);
  const size_t slot = ((size_t)blk * a.H * kBlock + own % kBlock) * (D * EB);   // head 0

  // c[i], s[i]: factors of the lane's element i and of its partner, for queries
  // and for keys (the norm's weights multiplied in)
  float cq[EPL], ck[EPL], sq[EPL], sk[EPL];
  bool turns[EPL];
  int other[EPL];                             // the partner's element
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    cq[i] = ck[i] = 1.f; sq[i] = sk[i] = 0.f;
    turns[i] = false;
    other[i] = e0 + i;
  }
  if constexpr (PARTNER != kRotaryNone) {
    const long long pos = a.positions[t];
    float cs = 1.f, sn = 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = e0 + i;
      turns[i] = e < a.rd;
      const int pair = PARTNER == kRotaryInterleaved ? e >> 1 : e < half ? e : e - half;
      const bool second = PARTNER == kRotaryInterleaved ? (e & 1) : e >= half;
      if (PARTNER != kRotaryInterleaved || !(i & 1)) {
        const unsigned long long w = a.turns[turns[i] ? pair : 0] * (unsigned long long)pos;
        cos_sin_turns((unsigned)(w >> 32), &cs, &sn);
        cs *= a.amplitude; sn *= a.amplitude;
      }
      if (turns[i]) {
        cq[i] = ck[i] = cs;
        sq[i] = sk[i] = second ? sn : -sn;
        other[i] = PARTNER == kRotaryInterleaved ? (e ^ 1) : second ? e - half : e + half;
      }
    }
  }
  if (a.q_norm) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      cq[i] *= load_elem<DT>((const char*)a.q_norm + (e0 + i) * EB);
      if (PARTNER != kRotaryNone) sq[i] *= load_elem<DT>((const char*)a.q_norm + other[i] * EB);
    }
  }
  if (a.k_norm) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      ck[i] *= load_elem<DT>((const char*)a.k_norm + (e0 + i) * EB);
      if (PARTNER != kRotaryNone) sk[i] *= load_elem<DT>((const char*)a.k_norm + other[i] * EB);
    }
  }

  const int heads = a.HQ + 2 * a.H;
  const int end = min((slab + 1) * a.slab_heads, heads);
  for (int hb = slab * a.slab_heads; hb < end; hb += HPS) {
    const int x = hb + threadIdx.x / LPH;
    const bool live = x < end;
    const int kind = !live ? 2 : x < a.HQ ? 0 : x < a.HQ + a.H ? 1 : 2;       // query, key, value
    const int h = !live ? 0 : kind == 0 ? x : kind == 1 ? x - a.HQ : x - a.HQ - a.H;
    const char* src = kind == 0 ? (const char*)a.q + t * a.q_stride
                    : kind == 1 ? (const char*)a.k + t * a.k_stride : (const char*)a.v + t * a.v_stride;
    src += (size_t)h * (D * EB);
    const u32x4 raw = ld16(src + sub * 16);
    float x0[EPL], x1[EPL];
    E::to_f32(raw, x0);
    if constexpr (PARTNER == kRotaryInterleaved) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) x1[i] = x0[i ^ 1];
    } else if constexpr (PARTNER == kRotaryHalfVector) {
      E::to_f32(ld16(src + other[0] * EB), x1);      // rd / 2 is a multiple of EPL
    } else if constexpr (PARTNER == kRotaryHalfScalar) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) x1[i] = load_elem<DT>(src + other[i] * EB);
    }
    float rs = 1.f;
    if (a.q_norm || a.k_norm) {                       // uniform: all lanes take part in the sums
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) ss = __builtin_fmaf(x0[i], x0[i], ss);
      ss = group_sum<LPH>(ss);
      if (kind == 0 ? a.q_norm != nullptr : a.k_norm != nullptr) rs = 1.f / sqrtf(ss * (1.f / D) + a.eps);
    }
    u32x4 res = raw;                                  // values are copied
    if (kind < 2) {
      float y[EPL];
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        y[i] = x0[i] * (kind == 0 ? cq[i] : ck[i]);
        // (a selection: 0 times an infinite partner is no zero)
        if constexpr (PARTNER != kRotaryNone)
          y[i] = turns[i] ? __builtin_fmaf(x1[i], kind == 0 ? sq[i] : sk[i], y[i]) : y[i];
        y[i] *= rs;
      }
      res = pack16<DT>(y);
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
      (long)a.slabs * a.slab_heads < a.HQ + 2L * a.H || (long)a.T * a.slabs > 0x7fffffffL || a.rd > D ||
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
