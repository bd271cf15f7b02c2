// Fill of new rows into a cache held in 8 bits: per-head RMS norm of queries and keys and their
// rotation, as the 16-bit fill has them (rotary.hip), then queries to q_out, and keys and values
// as codes with a scale for each block and head (cache8_args.h).
//
// Per block and head, with y the new rows in fp32 and a their largest finite |y|:
//   need = the least power of two with a / need <= 448, the largest code,
//   s    = need if the rows hold the block's first slot, else max(old scale, need),
//   code = y / s rounded to nearest even (NaN for what is no finite number).
// Scales are powers of two, so y / s is exact and the only rounding is the code's; tokens that the
// block held before are brought to a raised scale by the same rule, which keeps their
// bits unless they fall below 2^-6 s.
//
// A workgroup takes the rows of one request that go to one block (a unit), for a slab of the
// heads: 16 bytes of a row's head per lane, so that one lane group holds a head's rows of the whole
// block in registers, finds their scale and writes them once.  Keys are written 8 bytes a lane
// and row, values 16 bytes for four tokens of four elements.
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
  return x;
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

// ROWS 1: a row per request, whose unit is its request; 16: any rows.
template <int DT, int D, int PARTNER, int ROWS>
__global__ __launch_bounds__(256) void k_cache8_fill(FillArgs a, unsigned char* scales) {
  using E = Elem<DT>;
  constexpr int EB = E::kBytes, EPL = E::kPerLoad;
  constexpr int LPH = D * EB / 16;            // lanes per head
  constexpr int HPS = 256 / LPH;              // heads per workgroup and step
  __shared__ float turn_c[ROWS][kRotaryPairs], turn_s[ROWS][kRotaryPairs];
  const int lane = threadIdx.x & 63;
  const int u = blockIdx.x / a.slabs, slab = blockIdx.x % a.slabs;

  // the unit's request: a request of Q rows has at most Q / 16 + 2 units, and those of request r
  // start at qoff[r] / 16 + 2 r
  int r = u, part = 0;
  if constexpr (ROWS > 1) {
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
    if (r < 0) return;
    part = u - (clampi(ld_uniform(a.qoff + r), 0, a.T) / 16 + 2 * r);
  }
  const int S = clampi(ld_uniform(a.slen + r), 0, a.max_s);
  const RowSpan rw = row_span(a.qoff, r, a.T, min(S, a.max_q));
  const int from = S - rw.count;                           // own position of the first row
  const int blk0 = from / kBlockTokens + part;             // the unit's block of the request
  const int p0 = max(from, blk0 * kBlockTokens), p1 = min(S, (blk0 + 1) * kBlockTokens);
  if (p0 >= p1) return;
  const int phi = p0 % kBlockTokens, n = p1 - p0;          // slots [phi, phi + n)
  const int t0 = rw.first + (p0 - from);                   // the unit's first row
  const int id = clampi(ld_uniform(a.stab + (long)r * a.sstride + blk0), 0, a.nsblk - 1);

  // registers are indexed by slot (ROWS 16) or hold the one row
  const int lo = ROWS > 1 ? phi : 0, hi = lo + n;
  auto row_of = [&](int i) { return t0 + i - lo; };
  const int half = a.rd >> 1;
  if constexpr (PARTNER != kRotaryNone) {
    for (int x = threadIdx.x; x < ROWS * half; x += 256) {
      const int i = x / half, p = x - i * half;
      if (i < lo || i >= hi) continue;
      float c, s;
      cos_sin_turns((unsigned)((a.turns[p] * (unsigned long long)(long long)a.positions[row_of(i)]) >> 32), &c, &s);
      turn_c[i][p] = c * a.amplitude;
      turn_s[i][p] = s * a.amplitude;
    }
    __syncthreads();
  }

  const int sub = threadIdx.x % LPH;
  const int e0 = sub * EPL;                                // the lane's first element
  const unsigned turns = PARTNER == kRotaryNone || e0 >= a.rd ? 0u : a.rd - e0 >= EPL ? (1u << EPL) - 1u : (1u << (a.rd - e0)) - 1u;
  const int far = !turns ? 0 : e0 >= half ? -half : half;
  const int partner = lane + far / EPL;                    // (half layout: the lane that holds the partners)
  const int heads = a.HQ + 2 * a.H;
  const int begin = slab * a.slab_heads, end = min(begin + a.slab_heads, heads);
#pragma unroll 1
  for (int x = begin + (int)threadIdx.x / LPH; x < end; x += HPS) {
    const int kind = x < a.HQ ? 0 : x < a.HQ + a.H ? 1 : 2;                 // query, key, value
    const int h = kind == 0 ? x : kind == 1 ? x - a.HQ : x - a.HQ - a.H;
    const char* src = kind == 0 ? (const char*)a.q : kind == 1 ? (const char*)a.k : (const char*)a.v;
    const long stride = kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride;
    src += (size_t)h * (D * EB);
    u32x4 raw[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (i >= lo && i < hi) raw[i] = ld16(src + row_of(i) * stride + sub * 16);
    const char* weight = (const char*)(kind == 0 ? a.q_norm : kind == 1 ? a.k_norm : nullptr);
    float w[EPL];
    if (weight) E::to_f32(ld16(weight + e0 * EB), w);
    // the row's elements, normalised and rotated
    auto row = [&](int i, float* y) {
      E::to_f32(raw[i], y);
      if (kind == 2) return;
      float rs = 1.f;
      if (weight) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) ss = __builtin_fmaf(y[e], y[e], ss);
        ss = group_sum<LPH>(ss);
        rs = 1.f / sqrtf(ss * (1.f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < EPL; ++e) y[e] = y[e] * rs * w[e];
      }
      if constexpr (PARTNER != kRotaryNone) {
        float z[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          if constexpr (PARTNER == kRotaryInterleaved) z[e] = y[e ^ 1];
          if constexpr (PARTNER == kRotaryHalfVector) z[e] = __shfl(y[e], partner);
          if constexpr (PARTNER == kRotaryHalfScalar) {
            const int at = ((turns >> e) & 1u) ? (e0 + e >= half ? e0 + e - half : e0 + e + half) : e0 + e;
            z[e] = load_elem<DT>(src + row_of(i) * stride + at * EB);
            if (weight) z[e] = z[e] * rs * load_elem<DT>(weight + at * EB);
          }
        }
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const int at = e0 + e;
          const int pair = PARTNER == kRotaryInterleaved ? at >> 1 : at < half ? at : at - half;
          const bool second = PARTNER == kRotaryInterleaved ? (at & 1) : at >= half;
          const bool on = (turns >> e) & 1u;
          const float c = turn_c[i][on ? pair : 0], s = turn_s[i][on ? pair : 0];
          // (a selection: 0 times an infinite partner is no zero)
          y[e] = on ? __builtin_fmaf(z[e], second ? s : -s, y[e] * c) : y[e];
        }
      }
    };
    if (kind == 0) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
        if (i >= lo && i < hi) {
          float y[EPL];
          row(i, y);
          *reinterpret_cast<u32x4*>((char*)a.q_out + ((size_t)row_of(i) * a.HQ + h) * (D * EB) + sub * 16) = pack16<DT>(y);
        }
      continue;
    }
    const size_t bh = (size_t)id * a.H + h;
    unsigned char* scale = scales + bh * 2 + (kind - 1);
    const int old = phi > 0 ? *scale : 0;
    char* dst = (char*)(kind == 1 ? a.sk : a.sv) + bh * (kBlockTokens * D);
    float y[ROWS][EPL];
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
#pragma unroll
      for (int e = 0; e < EPL; ++e) y[i][e] = 0.f;
      if (i >= lo && i < hi) {
        row(i, y[i]);
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const float m = __builtin_fabsf(y[i][e]);
          most = m <= 3.402823466e38f ? fmaxf(most, m) : most;
        }
      }
    }
    most = group_max<LPH>(most);
    const int now = max(old, need_byte(most));
    const bool raised = phi > 0 && now > old;
    if (sub == 0) *scale = (unsigned char)now;
    if (kind == 1) {
      char* mine = dst + e0;
      if (raised)
        for (int t = 0; t < phi; ++t) {
#pragma unroll
          for (int e = 0; e < EPL; e += 4) {
            unsigned* p = reinterpret_cast<unsigned*>(mine + t * D + e);
            *p = recode4(*p, old, now);
          }
        }
#pragma unroll
      for (int i = 0; i < ROWS; ++i)
        if (i >= lo && i < hi) {
          char* to = mine + (ROWS > 1 ? i : phi) * D;
          if constexpr (EPL == 8) *reinterpret_cast<uint2*>(to) = uint2{encode4(y[i], now), encode4(y[i] + 4, now)};
          else *reinterpret_cast<unsigned*>(to) = encode4(y[i], now);
        }
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
#pragma unroll
      for (int gi = 0; gi < (ROWS > 1 ? 4 : 1); ++gi) {
        const int g = ROWS > 1 ? gi : phi / 4;
        if (ROWS > 1 && (4 * g + 4 <= phi || 4 * g >= phi + n)) continue;
        // the group's slots: first those from before, then new rows, then those that stay as they were
        const int kept = max(phi - 4 * g, 0), filled = min(phi + n - 4 * g, 4);
        const unsigned before = (1u << (8 * kept)) - 1u;
        const unsigned behind = filled < 4 ? ~0u << (8 * filled) : 0u;
#pragma unroll
        for (int e = 0; e < EPL; e += 4) {
          u32x4* p = reinterpret_cast<u32x4*>(mine + g * 256 + e * 4);
          u32x4 v = {0u, 0u, 0u, 0u};
          if (before | behind) {
            v = *p;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              const unsigned was = v[d];
              v[d] = ((raised && kept > 0 ? recode4(was, old, now) : was) & before) | (was & behind);
            }
          }
          if constexpr (ROWS > 1) {
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              const float col[4] = {y[4 * gi][e + d], y[4 * gi + 1][e + d], y[4 * gi + 2][e + d], y[4 * gi + 3][e + d]};
              v[d] |= encode4(col, now);                   // (slots without a new row give 0)
            }
          } else {
            const unsigned code = encode4(y[0] + e, now);
#pragma unroll
            for (int d = 0; d < 4; ++d) v[d] |= (code >> (8 * d) & 0xFFu) << (8 * (phi & 3));
          }
          *p = v;
        }
      }
    }
  }
}

template <int DT, int D, int ROWS>
static hipError_t launch_fill8_t(const Fill8Args& a, int partner, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const dim3 grid((unsigned)((long)a.units * a.f.slabs)), wg(256);
  switch (partner) {
    case kRotaryNone: hipExtLaunchKernelGGL((k_cache8_fill<DT, D, kRotaryNone, ROWS>), grid, wg, 0, s, e0, e1, 0, a.f, (unsigned char*)a.scales); break;
    case kRotaryInterleaved:
      hipExtLaunchKernelGGL((k_cache8_fill<DT, D, kRotaryInterleaved, ROWS>), grid, wg, 0, s, e0, e1, 0, a.f, (unsigned char*)a.scales);
      break;
    case kRotaryHalfVector:
      hipExtLaunchKernelGGL((k_cache8_fill<DT, D, kRotaryHalfVector, ROWS>), grid, wg, 0, s, e0, e1, 0, a.f, (unsigned char*)a.scales);
      break;
    default: hipExtLaunchKernelGGL((k_cache8_fill<DT, D, kRotaryHalfScalar, ROWS>), grid, wg, 0, s, e0, e1, 0, a.f, (unsigned char*)a.scales);
  }
  return hipGetLastError();
}

template <int DT, int D>
static hipError_t launch_fill8_r(const Fill8Args& a, int partner, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  return a.f.max_q == 1 ? launch_fill8_t<DT, D, 1>(a, partner, s, e0, e1) : launch_fill8_t<DT, D, 16>(a, partner, s, e0, e1);
}

hipError_t launch_fill8(const Fill8Args& a, int partner, int dtype, int D, hipStream_t s, hipEvent_t e0, hipEvent_t e1) {
  const FillArgs& f = a.f;
  if (f.T < 1 || f.R < 1 || f.H < 1 || f.HQ < 0 || f.slabs < 1 || f.sstride < 1 || f.nsblk < 1 || f.max_q < 1 || !a.scales ||
      (long)f.slabs * f.slab_heads < f.HQ + 2L * f.H || (long)a.units * f.slabs > 0x7fffffffL || f.rd > D ||
      f.rd > 2 * kRotaryPairs || (partner != kRotaryNone && !f.positions) ||
      a.units < (f.max_q == 1 ? (long)f.R : f.T / 16 + 2L * f.R))
    return hipErrorInvalidValue;
  switch (dtype * 1000 + D) {
    case kF32 * 1000 + 64: return launch_fill8_r<kF32, 64>(a, partner, s, e0, e1);
    case kF32 * 1000 + 128: return launch_fill8_r<kF32, 128>(a, partner, s, e0, e1);
    case kF16 * 1000 + 64: return launch_fill8_r<kF16, 64>(a, partner, s, e0, e1);
    case kF16 * 1000 + 128: return launch_fill8_r<kF16, 128>(a, partner, s, e0, e1);
    case kBF16 * 1000 + 64: return launch_fill8_r<kBF16, 64>(a, partner, s, e0, e1);
    case kBF16 * 1000 + 128: return launch_fill8_r<kBF16, 128>(a, partner, s, e0, e1);
  }
  return hipErrorInvalidValue;
}

}  // namespace parrot
