// Fill of new rows into a cache held in 8 bits: per-head RMS norm of queries and keys and their
// rotation, as the 16-bit fill has them (rotary.hip), then queries to q_out, and keys and values
// as codes with a scale for each block and head (cache8_args.h).
//
// Per block and head, with y the new rows in fp32 (in 64 bits where each request has one) and a their
// largest finite |y|:
//   need = the least power of two with a / need <= 448, the largest code,
//   s    = need if the rows hold the block's first slot, else max(old scale, need),
//   code = y / s rounded to nearest even (NaN for what is no finite number).
// Scales are powers of two, so y / s is exact and the only rounding is the code's; tokens that the
// block held before are brought to a raised scale by the same rule, which keeps their
// bits unless they fall below 2^-6 s.
//
// A workgroup takes the rows of one request that go to one block (a unit), for a slab of the
// heads: 16 bytes of a row's head per lane.  A block-head's rows are in registers until their scale is
// known and are written once: keys 8 bytes a lane and row, values 16 bytes for four tokens of four
// elements.  Cosines and sines are computed once a unit and come from LDS by element.
#include "cache8_args.h"
#include "rotary_math.h"

namespace parrot {

// Maximum over aligned groups of N lanes.
template <int N>
PARROT_DEV float group_max(float x) {
  x = fmaxf(x, dpp_f<kDppXor1>(x));
  x = fmaxf(x, dpp_f<kDppXor2>(x));
  x = fmaxf(x, dpp_f<kDppHalfMirror>(x));
  if constexpr (N >= 16) x = fmaxf(x, dpp_f<kDppMirror>(x));
  if constexpr (N >= 32) x = max_xor16(x);
  if constexpr (N >= 64) x = max_xor32(x);
  return x;
}

// The value of the lane N / 2 further on in aligned groups of N lanes.
template <int N>
PARROT_DEV float other_half(float x) {
  if constexpr (N == 8) return dpp_f<0x1B>(dpp_f<kDppHalfMirror>(x));      // 7 - i, then i ^ 3
  else if constexpr (N == 16) return dpp_f<0x128>(x);                      // rotated by 8
  else return __shfl_xor(x, N / 2);
}

// The scale byte that `most` needs: 448 is 1.75 * 2^8.
PARROT_DEV int need_byte(float most) {
  const unsigned u = __float_as_uint(most);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return most > 0.f ? max(e, 1) : 0;
}

// Four codes of x / 2^(byte - 127).
PARROT_DEV unsigned encode4(const float* x, int byte) {
  float y[4];
  unsigned bad = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool fine = __builtin_fabsf(x[i]) <= 3.402823466e38f;
    y[i] = fine ? __builtin_amdgcn_ldexpf(x[i], 127 - byte) : 0.f;
    bad |= fine ? 0u : 0x7Fu << (8 * i);
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return (unsigned)w | bad;
}

// Four codes of finite x, inv = 2^(127 - byte).
PARROT_DEV unsigned encode4_fine(const float* x, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, w, true);
  return (unsigned)w;
}

// Four codes brought from a scale byte to a larger one.
PARROT_DEV unsigned recode4(unsigned w, int from, int to) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  float y[4] = {a[0], a[1], b[0], b[1]};
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_ldexpf(y[i], from - to);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
  const unsigned nan = ((((w & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u) * 255u;
  return ((unsigned)r & ~nan) | (w & nan);
}

// The unit (a request's rows that go to one block) of a workgroup.
struct Unit8 { int phi, n, row, id; };                     // slots [phi, phi + n) of block id take rows from `row` on
// ONE: each request has a row at most, and the units are the requests.  Else a request of Q rows
// has at most Q / 16 + 2 units, and those of request r start at qoff[r] / 16 + 2 r.
template <bool ONE>
PARROT_DEV bool find_unit(const FillArgs& a, int u, Unit8* o) {
  const int lane = threadIdx.x & 63;
  int r = u, part = 0;
  if constexpr (!ONE) {
    r = -1;
    for (int base = 0, n = a.R; n > 0;) {
      const int step = (n + kWave - 1) / kWave;
      const int at = lane * step, i = base + min(at, n - 1);
      const int k = __popcll(__ballot(at < n && clampi(a.qoff[i], 0, a.T) / 16 + 2 * i <= u));
      if (k == 0 || step == 1) { r = base + k - 1; break; }
      base += (k - 1) * step;
      n = min(step, n - (k - 1) * step);
    }
    r = __builtin_amdgcn_readfirstlane(r);
    if (r < 0) return false;
    part = u - (clampi(ld_uniform(a.qoff + r), 0, a.T) / 16 + 2 * r);
  }
  const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
  const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
  const int from = S - rw.count;                           // own position of the first row
  const int blk = from / kBlockTokens + part;              // the unit's block of the request
  const int p0 = max(from, blk * kBlockTokens), p1 = min(S, (blk + 1) * kBlockTokens);
  if (p0 >= p1) return false;
  o->phi = p0 % kBlockTokens;
  o->n = p1 - p0;
  o->row = rw.first + (p0 - from);
  o->id = clampi(ld_uniform(a.stab + (long)r * a.sstride + blk), 0, a.nsblk - 1);
  return true;
}

// Head x of a row: 0 query, 1 key, 2 value.
struct Head8Of { int kind, h; const char* src; long stride; const char* weight; };
PARROT_DEV Head8Of head_of(const FillArgs& a, int x, int head_bytes) {
  Head8Of o;
  o.kind = x < a.HQ ? 0 : x < a.HQ + a.H ? 1 : 2;
  o.h = o.kind == 0 ? x : o.kind == 1 ? x - a.HQ : x - a.HQ - a.H;
  o.src = (o.kind == 0 ? (const char*)a.q : o.kind == 1 ? (const char*)a.k : (const char*)a.v) + (size_t)o.h * head_bytes;
  o.stride = o.kind == 0 ? a.q_stride : o.kind == 1 ? a.k_stride : a.v_stride;
  o.weight = (const char*)(o.kind == 0 ? a.q_norm : o.kind == 1 ? a.k_norm : nullptr);
  return o;
}

// The double counterparts of what a row's sum, root and partners take.
template <int CTRL>
PARROT_DEV double dpp_d(double x) {
  const auto v = __builtin_bit_cast(uint2, x);
  return __builtin_bit_cast(double, uint2{(unsigned)__builtin_amdgcn_mov_dpp((int)v.x, CTRL, 0xF, 0xF, true),
                                          (unsigned)__builtin_amdgcn_mov_dpp((int)v.y, CTRL, 0xF, 0xF, true)});
}
template <int N>
PARROT_DEV double group_sum(double x) {
  x += dpp_d<kDppXor1>(x);
  x += dpp_d<kDppXor2>(x);
  x += dpp_d<kDppHalfMirror>(x);
  if constexpr (N >= 16) x += dpp_d<kDppMirror>(x);
  if constexpr (N >= 32) x += __shfl_xor(x, 16);
  return x;
}
template <int N>
PARROT_DEV double other_half(double x) {
  if constexpr (N == 8) return dpp_d<0x1B>(dpp_d<kDppHalfMirror>(x));
  else if constexpr (N == 16) return dpp_d<0x128>(x);
  else return __shfl_xor(x, N / 2);
}
PARROT_DEV float fused(float x, float y, float z) { return __builtin_fmaf(x, y, z); }
PARROT_DEV double fused(double x, double y, double z) { return __builtin_fma(x, y, z); }
// (one step behind the instruction's estimate, where x r^2 is a number)
PARROT_DEV float reciprocal_root(float x) {
  const float r = __builtin_amdgcn_rsqf(x);
  return x > 1e-37f && x < 1e37f ? fused(0.5f * r, fused(-x * r, r, 1.f), r) : r;
}
PARROT_DEV double reciprocal_root(double x) {
  const double r = __builtin_amdgcn_rsq(x);
  return x > 1e-300 && x < 1e300 ? fused(0.5 * r, fused(-x * r, r, 1.), r) : r;
}
PARROT_DEV float narrowed(float x, bool) { return x; }
// odd: rounded to odd, so that a further rounding to few bits gives what one rounding would.
PARROT_DEV float narrowed(double x, bool odd) {
  const float f = (float)x;
  const double back = f;
  if (!odd || back == x || !(__builtin_fabsf(f) <= 3.402823466e38f)) return f;
  return __uint_as_float((__float_as_uint(f) - (__builtin_fabs(back) > __builtin_fabs(x) ? 1u : 0u)) | 1u);
}

// One row of a head in a group of LPH lanes: out (16 bytes of it as floats) normalised and rotated, in R.
// turn_c and turn_s hold cosine and signed sine (times the amplitude) of the row's elements.  src: the
// row, for partners that no 16 bytes line up with.
template <int DT, int D, int PARTNER, class R>
PARROT_DEV void turn_row(const FillArgs& a, const Head8Of& hd, const float* w, const R* turn_c, const R* turn_s,
                         const char* src, float* out) {
  constexpr int EPL = Elem<DT>::kPerLoad, LPH = D / EPL;
  const int lane = threadIdx.x & 63, e0 = lane % LPH * EPL, half = a.rd >> 1;
  R rs = 1, y[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) y[e] = out[e];
  if (hd.weight) {
    R ss = 0;
#pragma unroll
    for (int e = 0; e < EPL; ++e) ss = fused(y[e], y[e], ss);
    ss = group_sum<LPH>(ss);
    rs = reciprocal_root(ss * (R(1) / D) + a.eps);
#pragma unroll
    for (int e = 0; e < EPL; ++e) y[e] = y[e] * rs * w[e];
  }
  if constexpr (PARTNER != kRotaryNone) {
    R z[EPL];
    const bool all = a.rd == D;
    if constexpr (PARTNER == kRotaryInterleaved) {
#pragma unroll
      for (int e = 0; e < EPL; ++e) z[e] = y[e ^ 1];
    } else if constexpr (PARTNER == kRotaryHalfVector) {
      if (all) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) z[e] = other_half<LPH>(y[e]);
      } else {
        const int far = e0 >= a.rd ? 0 : e0 >= half ? -half : half;
#pragma unroll
        for (int e = 0; e < EPL; ++e) z[e] = __shfl(y[e], lane + far / EPL);
      }
    } else {
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const int at = e0 + e < a.rd ? (e0 + e >= half ? e0 + e - half : e0 + e + half) : e0 + e;
        z[e] = load_elem<DT>(src + at * Elem<DT>::kBytes);
        if (hd.weight) z[e] = z[e] * rs * load_elem<DT>(hd.weight + at * Elem<DT>::kBytes);
      }
    }
    constexpr int QUAD = 16 / sizeof(R);
    typedef R vec __attribute__((ext_vector_type(QUAD)));
    R c[EPL], s[EPL];
#pragma unroll
    for (int e = 0; e < EPL; e += QUAD) {
      const vec cv = *reinterpret_cast<const vec*>(turn_c + e0 + e), sv = *reinterpret_cast<const vec*>(turn_s + e0 + e);
#pragma unroll
      for (int i = 0; i < QUAD; ++i) { c[e + i] = cv[i]; s[e + i] = sv[i]; }
    }
    // (a selection where some pass: 0 times an infinite partner is no zero)
#pragma unroll
    for (int e = 0; e < EPL; ++e) y[e] = all || e0 + e < a.rd ? fused(z[e], s[e], y[e] * c[e]) : y[e];
  }
#pragma unroll
  for (int e = 0; e < EPL; ++e) out[e] = narrowed(y[e], DT != kF32 || hd.kind == 1);
}

// A unit's table of turns, rows lo .. hi of it (row i of the unit is row_of(i)).
template <int D, int PARTNER, class R, class F>
PARROT_DEV void turn_table(const FillArgs& a, R (*turn_c)[D], R (*turn_s)[D], int lo, int hi, F row_of) {
  const int half = a.rd >> 1;
  if constexpr (PARTNER != kRotaryNone) {
    for (int x = threadIdx.x + lo * half; x < hi * half; x += 256) {
      const int i = x / half, p = x - i * half;
      double c, s;                                         // (rounded once, to R)
      cos_sin_turns(a.turns[p] * (unsigned long long)(long long)a.positions[row_of(i)], &c, &s);
      c *= a.amplitude;
      s *= a.amplitude;
      const int one = PARTNER == kRotaryInterleaved ? 2 * p : p, two = PARTNER == kRotaryInterleaved ? one + 1 : p + half;
      turn_c[i][one] = turn_c[i][two] = (R)c;
      turn_s[i][one] = (R)-s;
      turn_s[i][two] = (R)s;
    }
    __syncthreads();
  }
}

// One row a request: a lane group per head.  Bound by the launch and the round trips of length,
// block and scale: 7 requests, 32 heads of 128 in float16, 4.7 us; 256 requests of 48 heads, normalised,
// 5.1 (in fp32 0.4 less, and one key in a million gets the code beside the nearest).  So where no scale grows; where
// some do, as in most steps, tokens that a raised block held are brought to the new scale one after the
// other, up to 15 round trips more: 10.7 and 15.0 us.
template <int DT, int D, int PARTNER>
__global__ __launch_bounds__(256) void k_cache8_fill_tokens(FillArgs a, unsigned char* scales) {
  using E = Elem<DT>;
  constexpr int EB = E::kBytes, EPL = E::kPerLoad, LPH = D / EPL;
  constexpr int HPS = 256 / LPH;              // heads per workgroup and step
  __shared__ __attribute__((aligned(16))) double turn_c[1][D], turn_s[1][D];
  Unit8 un;
  if (!find_unit<true>(a, blockIdx.x / a.slabs, &un)) return;
  turn_table<D, PARTNER>(a, turn_c, turn_s, 0, 1, [&](int) { return un.row; });
  const int phi = un.phi, slab = blockIdx.x % a.slabs;
  const int sub = threadIdx.x % LPH, e0 = sub * EPL;
  const int begin = slab * a.slab_heads, end = min(begin + a.slab_heads, a.HQ + 2 * a.H);
#pragma unroll 1
  for (int x = begin + (int)threadIdx.x / LPH; x < end; x += HPS) {
    const Head8Of hd = head_of(a, x, D * EB);
    const char* src = hd.src + un.row * hd.stride;
    const u32x4 raw = ld16(src + sub * 16);
    const size_t bh = (size_t)un.id * a.H + hd.h;
    unsigned char* scale = scales + bh * 2 + (hd.kind == 2);
    const int old = hd.kind > 0 && phi > 0 ? *scale : 0;
    float w[EPL], y[EPL];
    if (hd.weight) E::to_f32(ld16(hd.weight + e0 * EB), w);
    E::to_f32(raw, y);
    // (64 bits, so that a key's code is that of the formula's value; so few rows have the time)
    if (hd.kind < 2) turn_row<DT, D, PARTNER>(a, hd, w, turn_c[0], turn_s[0], src, y);
    if (hd.kind == 0) {
      *reinterpret_cast<u32x4*>((char*)a.q_out + ((size_t)un.row * a.HQ + hd.h) * (D * EB) + sub * 16) = pack16<DT>(y);
      continue;
    }
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      const float m = __builtin_fabsf(y[e]);
      most = m <= 3.402823466e38f ? fmaxf(most, m) : most;
    }
    most = group_max<LPH>(most);
    const int now = max(old, need_byte(most));
    const bool raised = phi > 0 && now > old;
    if (sub == 0) *scale = (unsigned char)now;
    char* dst = (char*)(hd.kind == 1 ? a.sk : a.sv) + bh * (kBlockTokens * D);
    if (hd.kind == 1) {
      char* mine = dst + e0;
      if (raised)
        for (int t = 0; t < phi; ++t) {
#pragma unroll
          for (int e = 0; e < EPL; e += 4) {
            unsigned* p = reinterpret_cast<unsigned*>(mine + t * D + e);
            *p = recode4(*p, old, now);
          }
        }
      char* to = mine + phi * D;
      if constexpr (EPL == 8) *reinterpret_cast<uint2*>(to) = uint2{encode4(y, now), encode4(y + 4, now)};
      else *reinterpret_cast<unsigned*>(to) = encode4(y, now);
    } else {
      // four tokens of the lane's elements, four of them at a time, are 16 bytes
      char* mine = dst + e0 / 64 * 1024 + e0 % 64 / 4 * 16;
      if (raised)
        for (int g = 0; g < phi / 4; ++g) {
#pragma unroll
          for (int e = 0; e < EPL; e += 4) {
            u32x4* p = reinterpret_cast<u32x4*>(mine + g * 256 + e * 4);
            const u32x4 v = *p;
            *p = u32x4{recode4(v.x, old, now), recode4(v.y, old, now), recode4(v.z, old, now), recode4(v.w, old, now)};
          }
        }
      const int g = phi / 4, t = phi & 3;
      const unsigned before = (1u << (8 * t)) - 1u, here = 0xFFu << (8 * t);
#pragma unroll
      for (int e = 0; e < EPL; e += 4) {
        u32x4* p = reinterpret_cast<u32x4*>(mine + g * 256 + e * 4);
        u32x4 v = *p;
        const unsigned code = encode4(y + e, now);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const unsigned was = raised && t > 0 ? (recode4(v[d], old, now) & before) | (v[d] & ~before) : v[d];
          v[d] = (was & ~here) | ((code >> (8 * d) & 0xFFu) << (8 * t));
        }
        *p = v;
      }
    }
  }
}

// Any rows: a wave, or half of one, per head of a block, GROUPS lane groups of it, each with RPG of the
// block's 16 slots, so that values' four tokens lie in one lane and a block-head's largest element is
// a wave's maximum.  Bound by memory: see the figures at the launch.
template <int DT, int D, int PARTNER>
__global__ __launch_bounds__(256)
void k_cache8_fill(FillArgs a, unsigned char* scales) {
  using E = Elem<DT>;
  constexpr int EB = E::kBytes, EPL = E::kPerLoad, LPH = D / EPL;
  constexpr int GROUPS = LPH == 32 ? 2 : 4, RPG = kBlockTokens / GROUPS;
  constexpr int LH = LPH * GROUPS, HPS = 256 / LH;         // lanes of a head, heads per workgroup and step
  static_assert(LH <= kWave && RPG % 4 == 0, "a head's rows are in one wave, a value's four tokens in one lane");
  __shared__ __attribute__((aligned(16))) float turn_c[kBlockTokens][D], turn_s[kBlockTokens][D];
  Unit8 un;
  if (!find_unit<false>(a, blockIdx.x / a.slabs, &un)) return;
  const int phi = un.phi, end_slot = phi + un.n, slab = blockIdx.x % a.slabs;
  auto row_of = [&](int slot) { return un.row + slot - phi; };
  turn_table<D, PARTNER>(a, turn_c, turn_s, phi, end_slot, row_of);
  const int sub = threadIdx.x % LPH, e0 = sub * EPL;
  const int slot0 = threadIdx.x / LPH % GROUPS * RPG;      // the lane's slots
  const int begin = slab * a.slab_heads, end = min(begin + a.slab_heads, a.HQ + 2 * a.H);
#pragma unroll 1
  for (int x = begin + (int)threadIdx.x / LH; x < end; x += HPS) {
    const Head8Of hd = head_of(a, x, D * EB);
    u32x4 raw[RPG];
#pragma unroll
    for (int j = 0; j < RPG; ++j) {
      raw[j] = u32x4{0u, 0u, 0u, 0u};
      if (slot0 + j >= phi && slot0 + j < end_slot) raw[j] = ld16_stream(hd.src + row_of(slot0 + j) * hd.stride + sub * 16);
    }
    const size_t bh = (size_t)un.id * a.H + hd.h;
    unsigned char* scale = scales + bh * 2 + (hd.kind == 2);
    const int old = hd.kind > 0 && phi > 0 ? *scale : 0;
    float w[EPL];
    if (hd.weight) E::to_f32(ld16(hd.weight + e0 * EB), w);
    float y[RPG][EPL];
    float most = 0.f, none = 0.f;                          // none: 0 where all are finite
#pragma unroll
    for (int j = 0; j < RPG; ++j) {
      E::to_f32(raw[j], y[j]);
      // (lane groups go together: the exchanges are among a row's lanes)
      if (hd.kind < 2 && slot0 + j >= phi && slot0 + j < end_slot)
        turn_row<DT, D, PARTNER>(a, hd, w, turn_c[slot0 + j], turn_s[slot0 + j],
                                 hd.src + row_of(slot0 + j) * hd.stride, y[j]);
      if (hd.kind == 0) {
        if (slot0 + j >= phi && slot0 + j < end_slot)
          *reinterpret_cast<u32x4*>((char*)a.q_out + ((size_t)row_of(slot0 + j) * a.HQ + hd.h) * (D * EB) + sub * 16) = pack16<DT>(y[j]);
      } else {
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          most = fmaxf(most, __builtin_fabsf(y[j][e]));
          none = __builtin_fmaf(y[j][e], 0.f, none);
        }
      }
    }
    if (hd.kind == 0) continue;
    const bool fine = __ballot(!(none == 0.f)) == 0;       // (of the whole wave: one way for all)
    if (!fine) {
      most = 0.f;
#pragma unroll
      for (int j = 0; j < RPG; ++j)
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const float m = __builtin_fabsf(y[j][e]);
          most = m <= 3.402823466e38f ? fmaxf(most, m) : most;
        }
    }
    most = group_max<LH>(most);
    const int now = max(old, need_byte(most));
    const float inv = __uint_as_float(now >= 254 ? 0x00400000u : (unsigned)(254 - now) << 23);
    const bool raised = phi > 0 && now > old;
    if (threadIdx.x % LH == 0) *scale = (unsigned char)now;
    char* dst = (char*)(hd.kind == 1 ? a.sk : a.sv) + bh * (kBlockTokens * D);
    auto encode = [&](const float* z) { return fine ? encode4_fine(z, inv) : encode4(z, now); };
    if (hd.kind == 1) {
#pragma unroll
      for (int j = 0; j < RPG; ++j) {
        const int slot = slot0 + j;
        char* to = dst + slot * D + e0;
        if (slot >= phi && slot < end_slot) {
          if constexpr (EPL == 8) *reinterpret_cast<uint2*>(to) = uint2{encode(y[j]), encode(y[j] + 4)};
          else *reinterpret_cast<unsigned*>(to) = encode(y[j]);
        } else if (raised && slot < phi) {
#pragma unroll
          for (int e = 0; e < EPL; e += 4) {
            unsigned* p = reinterpret_cast<unsigned*>(to + e);
            *p = recode4(*p, old, now);
          }
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < RPG; k += 4) {
        const int t0 = slot0 + k;                          // four slots: those from before, new ones, those that stay
        const int kept = clampi(phi - t0, 0, 4), filled = clampi(end_slot - t0, 0, 4);
        if (filled == 0 || (kept == 4 && !raised)) continue;
        const unsigned before = kept < 4 ? (1u << (8 * kept)) - 1u : ~0u, behind = filled < 4 ? ~0u << (8 * filled) : 0u;
#pragma unroll
        for (int e = 0; e < EPL; e += 4) {
          u32x4* p = reinterpret_cast<u32x4*>(dst + e0 / 64 * 1024 + t0 / 4 * 256 + (e0 % 64 + e) / 4 * 16);
          u32x4 v = {0u, 0u, 0u, 0u};
          if (before | behind) v = *p;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const float col[4] = {y[k][e + d], y[k + 1][e + d], y[k + 2][e + d], y[k + 3][e + d]};
            const unsigned was = v[d], held = raised && kept > 0 ? recode4(was, old, now) : was;
            v[d] = (held & before) | (was & behind) | encode(col);          // (slots without a new row give 0)
          }
          *p = v;
        }
      }
    }
  }
}

#define PARROT_FILL8(PARTNER)                                                                                             \
  if (a.f.max_q == 1) hipExtLaunchKernelGGL((k_cache8_fill_tokens<DT, D, PARTNER>), grid, wg, 0, s, e0, e1, 0, a.f, sc); \
  else hipExtLaunchKernelGGL((k_cache8_fill<DT, D, PARTNER>), grid, wg, 0, s, e0, e1, 0, a.f, sc);                       \
  break
template <int DT, int D>
static hipError_t launch_fill8_t(const Fill8Args& a, int partner, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const dim3 grid((unsigned)((long)a.units * a.f.slabs)), wg(256);
  unsigned char* sc = (unsigned char*)a.scales;
  switch (partner) {
    case kRotaryNone: PARROT_FILL8(kRotaryNone);
    case kRotaryInterleaved: PARROT_FILL8(kRotaryInterleaved);
    case kRotaryHalfVector: PARROT_FILL8(kRotaryHalfVector);
    default: PARROT_FILL8(kRotaryHalfScalar);
  }
  return hipGetLastError();
}

hipError_t launch_fill8(const Fill8Args& a, int partner, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const FillArgs& f = a.f;
  if (f.T < 1 || f.R < 1 || f.H < 1 || f.HQ < 0 || f.slabs < 1 || f.sstride < 1 || f.nsblk < 1 || f.max_q < 1 || !a.scales ||
      (long)f.slabs * f.slab_heads < f.HQ + 2L * f.H || (long)a.units * f.slabs > 0x7fffffffL || f.rd > D ||
      f.rd > 2 * kRotaryPairs || (partner != kRotaryNone && !f.positions) ||
      a.units < (f.max_q == 1 ? (long)f.R : f.T / 16 + 2L * f.R))
    return hipErrorInvalidValue;
  switch (dtype * 1000 + D) {
    case kF32 * 1000 + 64: return launch_fill8_t<kF32, 64>(a, partner, s, e0, e1);
    case kF32 * 1000 + 128: return launch_fill8_t<kF32, 128>(a, partner, s, e0, e1);
    case kF16 * 1000 + 64: return launch_fill8_t<kF16, 64>(a, partner, s, e0, e1);
    case kF16 * 1000 + 128: return launch_fill8_t<kF16, 128>(a, partner, s, e0, e1);
    case kBF16 * 1000 + 64: return launch_fill8_t<kBF16, 64>(a, partner, s, e0, e1);
    case kBF16 * 1000 + 128: return launch_fill8_t<kBF16, 128>(a, partner, s, e0, e1);
  }
  return hipErrorInvalidValue;
}

}  // namespace parrot
