// Internal: what the kernels over 8-bit pages share.
#ifndef LORC_Q8_H_
#define LORC_Q8_H_

#include "lorc_device.h"

namespace lorc {

// Of the softmax reference (see lorc_decode_q8.hip): a value scale counts as at least 2^kLeastExp, and the largest weight times scale is 2^kTopExp.
constexpr int kLeastExp = -40, kTopExp = 15;
// A weight times scale, below the largest fp16.  (It is at most 2^kTopExp but where fp32 rounds the reference by a unit: scores of 2^24 and more.)
__device__ __forceinline__ float below_f16_max(float w) { return __builtin_amdgcn_fmed3f(w, 0.f, 65504.f); }

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 half2_t;

__device__ __forceinline__ float pow2_of(uint32_t byte) { return __uint_as_float(byte << 23); }  // 2^(byte - 127)

// eight codes (two words) times a power of two, as fp16 or as bf16
__device__ __forceinline__ f16x8 codes_f16(u32x2 v, float scale = 1.f) {
  u32x4 r;
  const half2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v[0], scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v[0], scale, true);
  const half2_t c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v[1], scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)v[1], scale, true);
  r[0] = __builtin_bit_cast(uint32_t, a);
  r[1] = __builtin_bit_cast(uint32_t, b);
  r[2] = __builtin_bit_cast(uint32_t, c);
  r[3] = __builtin_bit_cast(uint32_t, d);
  return __builtin_bit_cast(f16x8, r);
}
__device__ __forceinline__ u32x4 codes_bf16(u32x2 v, float scale) {
  u32x4 r;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v[0], scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v[0], scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v[1], scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)v[1], scale, true);
  r[0] = __builtin_bit_cast(uint32_t, a);
  r[1] = __builtin_bit_cast(uint32_t, b);
  r[2] = __builtin_bit_cast(uint32_t, c);
  r[3] = __builtin_bit_cast(uint32_t, d);
  return r;
}
// the first n of eight bytes
__device__ __forceinline__ u32x2 keep_bytes(u32x2 v, int n) {
  n = n < 0 ? 0 : (n > 8 ? 8 : n);
  const uint64_t m = n == 8 ? ~0ull : (1ull << (8 * n)) - 1ull;
  return u32x2{v[0] & (uint32_t)m, v[1] & (uint32_t)(m >> 32)};
}

// Four values that are at most 448 in magnitude as e4m3 codes: rounded (hi), and what that leaves rounded (lo).
__device__ __forceinline__ void code_pair(float a, float b, float c, float d, int& hi, int& lo) {
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, hi, true);
  const auto h01 = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), h23 = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(a - h01[0], b - h01[1], 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(c - h23[0], d - h23[1], lo, true);
}

// exponent byte (exponent + 127) of the least power of two of which 448 is at least the magnitude with the bf16 bits `a` (no sign):
// 448 = 1.75 x 2^8; not below 1 (2^-126)
__device__ __forceinline__ int scale_byte(uint32_t a) {
  const int e = (int)(a >> 7) - 8 + ((a & 0x7f) > 0x60 ? 1 : 0);
  return e < 1 ? 1 : e;
}
__device__ __forceinline__ float inverse_scale(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
// magnitude bits of a bf16, 0 where it is inf or NaN
__device__ __forceinline__ uint32_t magnitude(uint32_t half) {
  const uint32_t a = half & 0x7fffu;
  return a < 0x7f80u ? a : 0u;
}

// A copy of 256 bytes global -> LDS, four per lane (see dma_1k).
__device__ __forceinline__ void dma_256(u32x4 rsrc, uint32_t lds_off, uint32_t lane4, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :
               : "s"(lds_off), "v"(lane4), "s"(rsrc), "s"(soff)
               : "memory");
}
// A value that is the same in every lane, in a scalar register whatever the compiler believes about it.
__device__ __forceinline__ uint32_t uniform_u32(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

}  // namespace lorc
#endif  // LORC_Q8_H_
