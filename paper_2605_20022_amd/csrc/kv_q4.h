// The 4-bit KV cache: layout and conversions shared by its kernels (internal; flexdraft.h has the format).
#pragma once
#include "fd_common.h"

namespace fd {

struct Q4Cache {
  unsigned char* k_codes; unsigned char* k_scales; unsigned char* v_codes; bf16_t* v_scales;
  long long sp, sh;         // blocks between pages and heads; a block is page_size tokens of a head
};

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

// Number of a token in the order of the arrays, 64 bits: its codes are at D/2 times it, and so on.
__device__ __forceinline__ long long q4_token(const Q4Cache& c, int page, int head, int page_size, int slot) {
  return ((long long)page * c.sp + (long long)head * c.sh) * page_size + slot;
}

// The eight codes of a word as bf16 pairs, times a power of two: exact.
__device__ __forceinline__ u32x4 q4_to_bf16(unsigned w, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  r[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  r[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  r[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return r;
}
__device__ __forceinline__ void q4_to_f32(unsigned w, float scale, float (&x)[8]) {
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    f32x2 v;
    switch (b) {            // the byte is part of the instruction
      case 0: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0); break;
      case 1: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1); break;
      case 2: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2); break;
      default: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3); break;
    }
    x[2 * b] = v[0]; x[2 * b + 1] = v[1];
  }
}
// Eight values already divided by their scale, to nearest, ties to the even code; |x| <= 6 but for the rounding of the scale, beyond that 6.
__device__ __forceinline__ unsigned f32_to_q4(const float (&x)[8]) {
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], 1.f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], 1.f, 3);
  return w;
}

// e + 127 of the smallest 2^e >= 2^-126 with top <= 6 * 2^e: with top = m 2^x, 1 <= m < 2, that is x - 2 up to m = 1.5, else x - 1.
__device__ __forceinline__ int q4_key_exponent(float top) {
  const unsigned u = __float_as_uint(top);
  const int b = (int)(u >> 23) - 2 + ((u & 0x7fffffu) > 0x400000u ? 1 : 0);
  return b < 1 ? 1 : b;
}
__device__ __forceinline__ float q4_key_scale(unsigned byte) { return __uint_as_float(byte << 23); }      // byte 255: infinity, which the conversion takes as NaN

}  // namespace fd
