// Device pieces of the fills of new rows (16-bit and fp32 caches, and 8-bit ones): angles,
// and elements in and out of 16 bytes.
#pragma once

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

// The same of 2 pi * phase / 2^64, to 2^-45.
PARROT_DEV void cos_sin_turns(unsigned long long phase, double* c, double* s) {
  const unsigned quad = (unsigned)((phase + 0x2000000000000000ull) >> 62);
  const double x = (double)(long long)(phase - ((unsigned long long)quad << 62)) * 3.4061215800304850e-19;   // 2 pi / 2^64
  const double z = x * x;
  double sn = 1.6059043836821613e-10;                            // 1/13!
  sn = __builtin_fma(sn, z, -2.5052108385441720e-8);
  sn = __builtin_fma(sn, z, 2.7557319223985893e-6);
  sn = __builtin_fma(sn, z, -1.9841269841269841e-4);
  sn = __builtin_fma(sn, z, 8.3333333333333333e-3);
  sn = __builtin_fma(sn, z, -1.6666666666666667e-1);
  sn = __builtin_fma(sn * z, x, x);
  double cs = -1.1470745597729725e-11;                           // -1/14!
  cs = __builtin_fma(cs, z, 2.0876756987868099e-9);
  cs = __builtin_fma(cs, z, -2.7557319223985891e-7);
  cs = __builtin_fma(cs, z, 2.4801587301587302e-5);
  cs = __builtin_fma(cs, z, -1.3888888888888889e-3);
  cs = __builtin_fma(cs, z, 4.1666666666666667e-2);
  cs = __builtin_fma(cs, z, -0.5);
  cs = __builtin_fma(cs, z, 1.0);
  const double a = (quad & 1) ? sn : cs, b = (quad & 1) ? cs : sn;
  *c = ((quad + 1) & 2) ? -a : a;
  *s = (quad & 2) ? -b : b;
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

}  // namespace parrot
