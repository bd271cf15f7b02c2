// A wave's attention over a range of keys held in 8 bits, for up to 16 * NS columns.
//
// A column is a (row, query head) pair that reads the wave's cache head.  Per unit of 32
// tokens (two blocks), with c_b the block's key scale times sm_scale log2(e):
//   S^T = K Q^T        (tokens x columns) on the matrix cores, codes widened to the queries' type
//   p   = 2^(c_b s - m), m a reference no more than 11 below the column's largest logit
//   O^T += V^T P       (elements x columns), values widened and scaled by their block's 2^e
// Widening is exact (a code has four significant bits), so the operands are the values the
// cache stands for; the only roundings are those of P and of the fp32 sums.
//
// No lane exchange: a lane's S^T values (tokens 4 g .. 4 g + 3 of a block for
// g = lane / 16, column lane % 16) are the PV operand's k group g, and the layout of the
// values holds the same four tokens side by side (cache8_args.h).  A wave whose columns are all
// that read its keys (run) needs nothing but its own loads, 16 bytes a lane: 8 KiB on their way, the
// next keys as soon as the last ones have been multiplied, the next values behind the last
// products.  Waves that share keys (run_shared) take them from a ring in LDS.
//
// Bounds: 16 columns read memory (64 requests on 3000 tokens, 393 MB in 64 us: 6.1 TB/s of the 7.1 that
// plain reads reach).  Wide tiles are bound by issue: of a unit's 1430 cycles for 32 columns of 128
// elements (four prompts of 400 rows on 8000 tokens, 760 TFLOP/s), the matrix products are 710, widening 370,
// the exponentials and sums of 1024 weights 400 (by each instruction's own rate; products and the rest
// overlap in part, between two waves of a SIMD).  Narrow tiles of 17 to 32 columns wait for memory (3.9 TB/s):
// their registers leave two waves a SIMD and one unit ahead.
//
// Types: bfloat16 and float16 round P once, and the output is divided by the sum of the rounded
// weights (a dominant weight's rounding cancels).  float32 queries and weights are cut into
// three bfloat16 parts, which hold all 24 bits: three products for one, at 16 times the rate of
// the fp32 ones.  float16 does not hold every scale: values are taken relative to a power of two that
// is raised as blocks need it, in the columns that see them alone; they are exact down to 2^-15 of
// it, and smaller blocks are multiplied by themselves, while the sums are scaled up.
#pragma once

#include "cache8_args.h"

namespace parrot {

template <int DT> struct Wide8;
template <> struct Wide8<kF16> {
  typedef f16x8 v8;
  PARROT_DEV static unsigned two(unsigned w, float s, bool hi) {
    return __builtin_bit_cast(unsigned, hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, true)
                                           : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, false));
  }
  PARROT_DEV static f32x4 mma(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  PARROT_DEV static unsigned pack(float x, float y) { return __builtin_bit_cast(unsigned, f16x2{(_Float16)x, (_Float16)y}); }
};
struct WideBf16 {
  typedef bf16x8 v8;
  PARROT_DEV static unsigned two(unsigned w, float s, bool hi) {
    return __builtin_bit_cast(unsigned, hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
                                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
  }
  PARROT_DEV static f32x4 mma(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
  }
  PARROT_DEV static unsigned pack(float x, float y) { return __builtin_bit_cast(unsigned, bf16x2{(__bf16)x, (__bf16)y}); }
};
template <> struct Wide8<kBF16> : WideBf16 {};
template <> struct Wide8<kF32> : WideBf16 {};

// The high 16 bits of two floats, the first in the low half.
PARROT_DEV unsigned high_halves(float x, float y) {
  return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}
PARROT_DEV float high_part(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

// One range of keys for the columns of one tile.
struct Range8 {
  Pool8 pool;
  const int* tbl;
  int npool;                             // blocks of the pool
  int u0, u1;                            // units
  int end;                               // keys; from here on slots hold anything
  int plain;                             // keys before it are seen by every column
};

// A wave-uniform value in scalar registers of its own.  Kernel arguments come sixteen registers a
// load, and a loop that uses one of them keeps (or spills, lane by lane) all sixteen.
template <class V>
PARROT_DEV V alone(V v) {
  asm("" : "+s"(v));
  return v;
}

template <int DT, int D, int NS>
struct Tile8 {
  using W = Wide8<DT>;
  static constexpr int X = D / 64;                    // 16-byte loads of each tensor, per block and lane
  // (units on their way: 8 KiB; 16 KiB changes nothing, 64 requests on 3000 tokens 72 us both ways)
  static constexpr int NU = 2 / X;
  static constexpr int PARTS = DT == kF32 ? 3 : 1;
  static constexpr int BLK_B = kBlockTokens * D;
  static constexpr float kMostSum = 2048.f;           // of a lane's eight weights
  static constexpr float kNoKey = -3.0e38f;           // a reference that every finite logit moves

  int lane, h, H;
  u32x4 qf[NS][PARTS][2 * X];
  f32x4 o[NS][4 * X];
  float mref[NS], lt[NS];
  f32x4 lw[NS];                                       // the rounded weights' sum, four times
  int lim[NS];                                        // keys the lane's column sees
  // float16: o is in units of 2^(cexp - 127); columns that see the unit at hand have vexp
  int vexp, cexp[NS];

  PARROT_DEV Tile8(int heads, int head) : lane(threadIdx.x & 63), h(head), H(alone(heads)) {
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      mref[c] = kNoKey; lt[c] = 0.f; lw[c] = f32x4{0.f, 0.f, 0.f, 0.f}; lim[c] = cexp[c] = 0;
#pragma unroll
      for (int t = 0; t < 4 * X; ++t) o[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    vexp = 0;
  }
  PARROT_DEV int column(int c) const { return 16 * c + (lane & 15); }

  // Queries of the tile's columns; at(c) is the column's place in [T][HQ], or -1.
  template <class F>
  PARROT_DEV void load_queries(const void* q, bool flip, F at) {
    const int g = lane >> 4;
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      const long row = at(c);
      const char* src = (const char*)q + (row < 0 ? 0 : row) * (D * Elem<DT>::kBytes);
      const bool on = row >= 0;
#pragma unroll
      for (int s = 0; s < 2 * X; ++s) {
        const int d = (s >> 1) * 64 + g * 16 + (s & 1) * 8;
        if constexpr (DT == kF32) {
          u32x4 lo = ld16(src + d * 4), hi = ld16(src + d * 4 + 16);
          const unsigned w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
          unsigned p[3][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x = on ? __uint_as_float(w[2 * i]) : 0.f, y = on ? __uint_as_float(w[2 * i + 1]) : 0.f;
            x = flip ? -x : x;
            y = flip ? -y : y;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
              p[k][i] = high_halves(x, y);
              x -= high_part(x);
              y -= high_part(y);
            }
          }
#pragma unroll
          for (int k = 0; k < 3; ++k) qf[c][k][s] = u32x4{p[k][0], p[k][1], p[k][2], p[k][3]};
        } else {
          u32x4 v = ld16(src + d * 2);
          const unsigned f = flip ? 0x80008000u : 0u;
          qf[c][0][s] = on ? u32x4{v.x ^ f, v.y ^ f, v.z ^ f, v.w ^ f} : u32x4{0u, 0u, 0u, 0u};
        }
      }
    }
  }

  PARROT_DEV void scale_outputs(float f, int c) {
#pragma unroll
    for (int t = 0; t < 4 * X; ++t) o[c][t] *= f;
  }
  // float16: the columns that see token tok (or all) change their unit to 2^(to - 127).
  PARROT_DEV void raise_unit(int to, bool all, int tok) {
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      const bool sees = all || tok < lim[c];
      if (__builtin_expect(vexp > 0 && to != vexp, false)) scale_outputs(sees ? ldexpf(1.f, cexp[c] - to) : 1.f, c);
      cexp[c] = sees ? to : cexp[c];
    }
    vexp = to;
  }

  // ONCE: no other tile reads the keys, and streaming loads take them (438 MB of 64 requests in
  // bfloat16, four query heads on each of 8: 72 us, 82 with cached loads; as a flag at run time the
  // compiler makes one load of the two).
  template <bool ONCE>
  PARROT_DEV void run(const Range8& rg, float scale_log2) {
    const int g = lane >> 4;
    const int last = max((rg.end - 1) / kBlockTokens, 0);
    // keys: row lane % 16, 16 bytes at 16 g of each 64; values: 16 bytes a lane
    const unsigned koff = (lane & 15) * D + g * 16, voff = lane * 16;
    u32x4 kr[NU][2][X], vr[NU][2][X];
    unsigned sc[NU][2];                               // a block's scale bytes: keys, values
    size_t bh[2];                                     // block-heads of the next unit to request
    auto find = [&](int u) {                          // (past the end: the last block)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int id = (int)min((unsigned)ld_uniform(rg.tbl + min(2 * u + b, last)), (unsigned)(rg.npool - 1));
        bh[b] = (size_t)id * H + h;
      }
    };
    auto request = [&](const void* pool, unsigned off, unsigned step, u32x4 (&to)[2][X]) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const char* p = (const char*)pool + bh[b] * BLK_B + off;
#pragma unroll
        for (int x = 0; x < X; ++x) to[b][x] = ONCE ? ld16_stream(p + x * step) : ld16(p + x * step);
      }
    };
    auto scales = [&](unsigned (&to)[2]) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const unsigned word = (unsigned)ld_uniform((const int*)((const char*)rg.pool.scales + ((bh[b] * 2) & ~(size_t)3)));
        to[b] = (bh[b] & 1 ? word >> 16 : word) & 0xFFFFu;
      }
    };
    find(rg.u0);
#pragma unroll
    for (int n = 0; n < NU; ++n)
      if (rg.u0 + n < rg.u1) {
        request(rg.pool.k, koff, 64, kr[n]);
        request(rg.pool.v, voff, 1024, vr[n]);
        scales(sc[n]);
        find(rg.u0 + n + 1);
      }
#pragma unroll 1
    for (int ub = rg.u0; ub < rg.u1; ub += NU) {
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        const int u = ub + n;
        if (u >= rg.u1) break;
        const bool more = u + NU < rg.u1;
        unsigned next[2] = {0, 0};
        // (the next loads take this unit's registers: not before they are free)
        unit(rg, u * kUnit, kr[n], vr[n], sc[n], scale_log2, [&] {
          __builtin_amdgcn_sched_barrier(0);
          if (more) {
            request(rg.pool.k, koff, 64, kr[n]);
            scales(next);
          }
        });
        __builtin_amdgcn_sched_barrier(0);
        if (more) {
          request(rg.pool.v, voff, 1024, vr[n]);
          sc[n][0] = next[0];
          sc[n][1] = next[1];
          find(u + NU + 1);
        }
      }
    }
  }

  // The same range for four waves of a workgroup, each with columns of its own: the keys' and
  // values' bytes come into a ring in LDS, three units ahead, once for all of them (a wave alone reads
  // them again from the L2, one unit ahead, for its columns).  `keys`: the wave's columns see no further; below 1:
  // it has no columns and loads for the others.  Rows of keys are swizzled, granule j of 16 bytes
  // of row r at j ^ f(r), on the global side of the loads, so that the 16 rows of a read lie in
  // different banks.
  static constexpr int RING = 4;                      // units
  static constexpr int UNIT_B = 4 * BLK_B;
  PARROT_DEV void run_shared(const Range8& rg, float scale_log2, char* ring, int keys) {
    constexpr int PER_WAVE = X;                       // loads of a wave and unit
    const int g = lane >> 4, r = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int last = max((rg.end - 1) / kBlockTokens, 0);
    const int blk = X == 2 ? wave >> 1 : wave & 1;    // the block of a unit that the wave loads from
    const unsigned ksrc = X == 2 ? (lane >> 3) * 128 + (((lane & 7) ^ (lane >> 3)) << 4)
                                 : (lane >> 2) * 64 + (((lane & 3) ^ (lane >> 4 & 3)) << 4);
    const unsigned vsrc = lane * 16;
    const unsigned f = X == 2 ? r & 7 : r >> 2 & 3;
    const unsigned to = lds_addr(ring) + wave * 1024;
    auto id_of = [&](int u, int b) {                  // (past the end: the last block)
      return (int)min((unsigned)ld_uniform(rg.tbl + min(2 * u + b, last)), (unsigned)(rg.npool - 1));
    };
    auto issue = [&](int id, unsigned buf) {
      const size_t off = ((size_t)id * H + h) * BLK_B;
      if constexpr (X == 2) {
        const size_t half = off + (wave & 1) * 1024;
        lds_dma16_sbase((const char*)rg.pool.k + half, ksrc, to + buf);
        lds_dma16_sbase((const char*)rg.pool.v + half, vsrc, to + buf + 2 * BLK_B);
      } else {
        lds_dma16_sbase((const char*)(wave < 2 ? rg.pool.k : rg.pool.v) + off, wave < 2 ? ksrc : vsrc, to + buf);
      }
    };
    auto scale_of = [&](int id) {
      const size_t bh = (size_t)id * H + h;
      const unsigned word = (unsigned)ld_uniform((const int*)((const char*)rg.pool.scales + ((bh * 2) & ~(size_t)3)));
      return (bh & 1 ? word >> 16 : word) & 0xFFFFu;
    };
    wait_vmcnt<0>();                                  // (queries)
    lds_sync();                                       // the ring of the range before has been read
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) issue(id_of(min(rg.u0 + i, rg.u1 - 1), blk), i * UNIT_B);
    int next_id = id_of(min(rg.u0 + RING - 1, rg.u1 - 1), blk);
    unsigned sc[2] = {scale_of(id_of(rg.u0, 0)), scale_of(id_of(rg.u0, 1))};
    int id1[2] = {id_of(rg.u0 + 1, 0), id_of(rg.u0 + 1, 1)};
    unsigned buf = 0;
    u32x4 kr[2][X], vr[2][X];
    auto keys_at = [&](unsigned at) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int x = 0; x < X; ++x)
          kr[b][x] = *reinterpret_cast<const u32x4*>(ring + at + b * BLK_B + r * D + (((x * 4 + g) ^ f) << 4));
    };
    wait_vmcnt<(RING - 2) * PER_WAVE>();
    lds_sync();
    keys_at(0);
#pragma unroll 1
    for (int u = rg.u0; u < rg.u1; ++u) {
      wait_vmcnt<(RING - 3) * PER_WAVE>();            // the next unit's loads are the oldest
      lds_sync();                                     // ... of every wave, and the last unit has been read
      issue(next_id, (buf + (RING - 1) * UNIT_B) % (RING * UNIT_B));
      next_id = id_of(min(u + RING, rg.u1 - 1), blk);
      const unsigned ahead[2] = {scale_of(id1[0]), scale_of(id1[1])};
      id1[0] = id_of(u + 2, 0);
      id1[1] = id_of(u + 2, 1);
      const unsigned after = (buf + UNIT_B) % (RING * UNIT_B);
      if (u * kUnit < keys) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int x = 0; x < X; ++x) vr[b][x] = *reinterpret_cast<const u32x4*>(ring + buf + (2 + b) * BLK_B + x * 1024 + lane * 16);
        unit(rg, u * kUnit, kr, vr, sc, scale_log2, [&] {
          __builtin_amdgcn_sched_barrier(0);
          keys_at(after);
        });
      }
      sc[0] = ahead[0];
      sc[1] = ahead[1];
      buf = after;
    }
    wait_vmcnt<0>();                                  // the last unit's loads, repeated by the last rounds
  }

  // Output of column c and its log-sum-exp: f(c, column, factor of o, log2 of the sum, rounded sum).
  template <class F>
  PARROT_DEV void finish(F f) {
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      const float t = sum_xor32(sum_xor16(lt[c]));
      float w = t;
      if constexpr (DT != kF32) w = lw[c][0];
      float inv = w == 0.f ? 0.f : 1.f / w;
      if constexpr (DT == kF16) inv *= cexp[c] > 0 ? __uint_as_float((unsigned)cexp[c] << 23) : 1.f;
      f(c, column(c), inv, t == 0.f ? -INFINITY : mref[c] + fast_log2(t));
    }
  }
  // Elements 64 x + 16 (lane / 16) + 4 i .. + 3 of column c.
  PARROT_DEV f32x4 four(int c, int x, int i) const {
    return f32x4{o[c][4 * x][i], o[c][4 * x + 1][i], o[c][4 * x + 2][i], o[c][4 * x + 3][i]};
  }

 private:
  // keys_read(): the unit's keys have been read.  The products go ahead of the other wave's softmax
  // (four prompts of 400 rows on 8000 tokens 314 us a layer, 341 without, before the steps below).
  template <class F>
  PARROT_DEV void unit(const Range8& rg, int tok0, u32x4 (&k)[2][X], u32x4 (&v)[2][X], unsigned (&sc)[2], float scale_log2,
                       F keys_read) {
    const int g = lane >> 4;
    f32x4 s[NS][2];
#pragma unroll
    for (int c = 0; c < NS; ++c) s[c][0] = s[c][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int st = 0; st < 2 * X; ++st)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const unsigned w0 = k[b][st >> 1][2 * (st & 1)], w1 = k[b][st >> 1][2 * (st & 1) + 1];
        const u32x4 kf = {W::two(w0, 1.f, false), W::two(w0, 1.f, true), W::two(w1, 1.f, false), W::two(w1, 1.f, true)};
#pragma unroll
        for (int c = 0; c < NS; ++c)
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p) s[c][b] = W::mma(kf, qf[c][p][st], s[c][b]);
      }
    __builtin_amdgcn_s_setprio(0);
    keys_read();
    const bool masked = tok0 + kUnit > rg.plain;
    bool bad = false;                                  // a value that some columns see may be no finite number
    if (masked) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int left = rg.end - (tok0 + 16 * b + 4 * g);
        const unsigned keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
        unsigned any = 0;
#pragma unroll
        for (int x = 0; x < X; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const unsigned w = v[b][x][i] & keep;
            v[b][x][i] = w;
            any |= (w & 0x7F7F7F7Fu) + 0x01010101u;
          }
        bad = bad || (any & 0x80808080u) != 0 || (DT != kF16 && alone(sc[b]) >= kLeastOver << 8);
      }
      bad = __ballot(bad) != 0;
    }
    float cb[2], vs[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      cb[b] = __uint_as_float((sc[b] & 0xFFu) << 23) * scale_log2;
      vs[b] = __uint_as_float((sc[b] >> 8) << 23);
    }
    // float16: the blocks go one after the other where one lies more than 2^15 below the unit (448 * 2^7 is a
    // float16: so far above it a block may lie), or where some columns see the first alone and the second
    // needs another unit; a column's bits depend on the blocks that it sees
    bool apart = false;
    int last = 0;                                      // the unit behind the second block
    if constexpr (DT == kF16) {
      const int e0 = sc[0] >> 8, e1 = sc[1] >> 8;
      if (__builtin_expect(vexp == 0 || (unsigned)(e0 - vexp + 15) > 22u || (unsigned)(e1 - vexp + 15) > 22u, false)) {
        const int first = e0 > vexp + 7 || vexp == 0 ? e0 : vexp;
        last = e1 > first + 7 || first == 0 ? e1 : first;
        apart = (masked && last != first && first > 0) || (e0 > 0 && e0 < last - 15) || (e1 > 0 && e1 < last - 15);
        raise_unit(apart ? first : last, !masked, tok0);
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) vs[b] = __uint_as_float((unsigned)(127 + max((b ? e1 : e0) - vexp, -15)) << 23);
    }
    // weights against the references at hand; their sums tell where one is more than 2^8 (a first
    // key's is infinite), and no maximum is taken until then.  A column's reference is raised by its own
    // sums alone, so that no row's bits depend on another row.
    float w[NS][8], sum[NS];
    bool raise = false;
#pragma unroll
    for (int c = 0; c < NS; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[c][i] = __builtin_fmaf(s[c][i >> 2][i & 3], cb[i >> 2], -mref[c]);
      if (masked) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          w[c][i] = tok0 + 16 * (i >> 2) + 4 * g + (i & 3) < lim[c] ? w[c][i] : -INFINITY;
      }
      sum[c] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[c] += w[c][i] = fast_exp2(w[c][i]);
      raise = raise || sum[c] > kMostSum;
    }
    // (one branch for all sets: 64 requests of 16 rows on 3000 tokens 130 us a layer, 137 with one for each)
    if (__ballot(raise)) {
      const int tok1 = alone(tok0);                    // (or the masks above are kept in scalar registers)
#pragma unroll
      for (int c = 0; c < NS; ++c) {
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          mx = fmaxf(mx, !masked || tok1 + 16 * (i >> 2) + 4 * g + (i & 3) < lim[c] ? s[c][i >> 2][i & 3] * cb[i >> 2] : -INFINITY);
        const float m = max_xor32(max_xor16(sum[c])) > kMostSum ? fmaxf(mref[c], max_xor32(max_xor16(mx))) : mref[c];
        const float f = fast_exp2(mref[c] - m);
        mref[c] = m;
        lt[c] *= f;
        lw[c] *= f;
        scale_outputs(f, c);
        sum[c] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = __builtin_fmaf(s[c][i >> 2][i & 3], cb[i >> 2], -m);
          w[c][i] = fast_exp2(!masked || tok1 + 16 * (i >> 2) + 4 * g + (i & 3) < lim[c] ? y : -INFINITY);
          sum[c] += w[c][i];
        }
      }
    }
    const unsigned two = W::pack(1.f, 1.f);
    const u32x4 ones = {two, two, two, two};
    unsigned pw[NS][PARTS][4];
#pragma unroll
    for (int c = 0; c < NS; ++c) {
      const float (&x)[8] = w[c];
      lt[c] += sum[c];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (DT == kF32) {
          float y0 = x[2 * i], y1 = x[2 * i + 1];
#pragma unroll
          for (int p = 0; p < 3; ++p) {
            pw[c][p][i] = high_halves(y0, y1);
            y0 -= high_part(y0);
            y1 -= high_part(y1);
          }
        } else {
          pw[c][0][i] = W::pack(x[2 * i], x[2 * i + 1]);
        }
      }
      // (the matrix cores have time for the sum: as dot products 64 requests of 16 rows take 129 us a layer, 113 so)
      if constexpr (DT != kF32) lw[c] = W::mma(ones, u32x4{pw[c][0][0], pw[c][0][1], pw[c][0][2], pw[c][0][3]}, lw[c]);
    }
    if (bad) mark_bad(v, sc, x_seen(tok0));
    // (twice where the float16 blocks go one after the other: 2^-126 makes zeros of the other block's codes)
#pragma unroll 1
    for (int part = apart ? 0 : 1;; ++part) {
      int up = 0;
      if constexpr (DT == kF16)
        if (__builtin_expect(apart, false)) {
          if (part) raise_unit(last, !masked, tok0 + kBlockTokens);
          const int e = (part ? sc[1] : sc[0]) >> 8, rel = e - vexp;
          up = e > 0 ? clampi(-15 - rel, 0, 60) : 0;     // (sums are below 2^58: scaled by as much they are floats)
          const float in = __uint_as_float((unsigned)(127 + max(rel + up, -126)) << 23), zero = __uint_as_float(1u << 23);
          vs[0] = part ? zero : in;
          vs[1] = part ? in : zero;
          if (__builtin_expect(up > 0, false))
#pragma unroll
            for (int c = 0; c < NS; ++c) scale_outputs(__uint_as_float((unsigned)(127 + up) << 23), c);
        }
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int x = 0; x < X; ++x)
#pragma unroll
        for (int dd = 0; dd < 4; ++dd) {
          const unsigned w0 = v[0][x][dd], w1 = v[1][x][dd];
          const u32x4 vf = {W::two(w0, vs[0], false), W::two(w0, vs[0], true), W::two(w1, vs[1], false), W::two(w1, vs[1], true)};
#pragma unroll
          for (int c = 0; c < NS; ++c)
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p)
              o[c][4 * x + dd] = W::mma(vf, u32x4{pw[c][p][0], pw[c][p][1], pw[c][p][2], pw[c][p][3]}, o[c][4 * x + dd]);
        }
      __builtin_amdgcn_s_setprio(0);
      if (__builtin_expect(up > 0, false))
#pragma unroll
        for (int c = 0; c < NS; ++c) scale_outputs(__uint_as_float((unsigned)(127 - up) << 23), c);
      if (__builtin_expect(part, 1)) break;
    }
  }

  // 1 where the lane's column sees the token of its P operand, as that operand.
  struct Seen { u32x4 w[NS]; };
  PARROT_DEV Seen x_seen(int tok0) const {
    Seen r;
    const int g = lane >> 4;
#pragma unroll
    for (int c = 0; c < NS; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = tok0 + 16 * (i >> 1) + 4 * g + 2 * (i & 1);
        r.w[c][i] = W::pack(t < lim[c] ? 1.f : 0.f, t + 1 < lim[c] ? 1.f : 0.f);
      }
    return r;
  }
  // What carries into the high bit of the bytes of codes that are no finite numbers: NaN (127) and, where
  // values keep a block's scale of byte kLeastOver or more, the codes from (262 - byte) 8 on: 2^128 and more.
  static constexpr unsigned kLeastOver = 247;
  PARROT_DEV static unsigned over(unsigned byte) {
    return (DT == kF16 || byte < kLeastOver ? 1u : 8u * byte - 1968u) * 0x01010101u;
  }
  // Values that are no finite numbers, in a unit that not all columns see whole: they make NaN of the
  // element in the columns that see their token, and are cleared for the others.
  PARROT_DEV void mark_bad(u32x4 (&v)[2][X], const unsigned (&sc)[2], const Seen& seen) {
    const unsigned up[2] = {over(sc[0] >> 8), over(sc[1] >> 8)};
#pragma unroll
    for (int x = 0; x < X; ++x)
#pragma unroll
      for (int dd = 0; dd < 4; ++dd) {
        u32x4 one;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const unsigned w = v[b][x][dd];
          const unsigned nan = (((w & 0x7F7F7F7Fu) + up[b]) >> 7) & 0x01010101u;             // 1 in such bytes
          v[b][x][dd] = w & ~(nan * 255u);
          const unsigned code = nan * 0x38u;                                               // 1.0 in e4m3
          one[2 * b] = W::two(code, 1.f, false);
          one[2 * b + 1] = W::two(code, 1.f, true);
        }
#pragma unroll
        for (int c = 0; c < NS; ++c) {
          const f32x4 n = W::mma(one, seen.w[c], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int i = 0; i < 4; ++i)                  // (n counts: all bits set where it is not 0)
            o[c][4 * x + dd][i] = __int_as_float(__float_as_int(o[c][4 * x + dd][i]) | ((0 - __float_as_int(n[i])) >> 31));
        }
      }
  }
};

}  // namespace parrot
