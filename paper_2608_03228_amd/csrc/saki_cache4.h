// The 4-bit form of the paged cache, on the device.
//
// Bytes of one (block, head): codes of 64 tokens, two dims a byte, the even one
// in the low half.  A key's 64 bytes are contiguous: a lane's 16 are one group
// of 32 dims with one scale, which the matrix instruction sums over.  Values
// stand as [token / 4][dim / 8][token % 4][4 bytes]: a lane's 16 are 8 dims of 4
// consecutive tokens, as the transposed operand wants them, so that no load is
// narrower than 16 bytes and one byte permute a pair of elements transposes.
// Scales are E8M0 bytes [2 (keys, values)][64 tokens][4 groups]: a byte shifted
// into the exponent's place is the scale operand of the conversions, and 255
// makes them NaN.
#pragma once

#include "saki_cache.h"

namespace {

constexpr int kCodes4 = kTile * kHeadDim / 2;  // bytes of one (block, head), keys or values
constexpr int kGroup4 = 32;                    // dims that share a scale
constexpr int kGroups4 = kHeadDim / kGroup4;
constexpr int kScales4 = 2 * kTile * kGroups4;  // bytes of one (block, head)

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// The scale's byte for a group whose largest |x| has these bits: the least s =
// 2^e with |x| <= 7 s, 7 = 0.875 * 2^3.  An element of (6 s, 7 s] becomes 6 s, no
// further from it than half a step of the codes' last binade.  (6 s as the limit
// leaves 6% more squared error on Gaussian groups, 13% more on Laplacian ones.)
// e is at least -100 and at most 120, above which elements saturate; a group
// with an element that is not finite is NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int e = (int)(top >> 23) - 126 - ((top & 0x7fffffu) <= 0x600000u ? 3 : 2);
  return (uint32_t)(min(max(e, -100), 120) + 127);
}

// Eight floats over the scale as codes: nearest, ties to the even code.
__device__ __forceinline__ uint32_t encode8(const float* x, float s) {
  uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
}

// Two codes (byte B of four) times their scale: exact in bf16 (2 significant bits).
template <int B>
__device__ __forceinline__ uint32_t decode2(uint32_t c, float s) {
  const bf16x2_t v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, B);
  uint32_t r;
  __builtin_memcpy(&r, &v, 4);
  return r;
}
// Eight codes times their scale.
__device__ __forceinline__ void decode8(uint32_t c, float s, uint32_t* pairs) {
  pairs[0] = decode2<0>(c, s), pairs[1] = decode2<1>(c, s);
  pairs[2] = decode2<2>(c, s), pairs[3] = decode2<3>(c, s);
}
__device__ __forceinline__ void decode8(uint32_t c, float s, float* x) {
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0);
  const f32x2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
  const f32x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2);
  const f32x2_t e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
  x[4] = d[0], x[5] = d[1], x[6] = e[0], x[7] = e[1];
}

// Tables are read by scalar loads: a wait for a vector load would wait for the tiles that are on their way
// too.
typedef __attribute__((address_space(4))) int const_int;

// Where 8 dims (8 m ..) of a block's token lie: bytes from the block's codes.
__device__ __forceinline__ int code_at(int which, int token, int m) {
  return which ? token / 4 * 256 + m * 16 + token % 4 * 4 : token * (kHeadDim / 2) + m * 4;
}

// Blocks and heads of a cache: row numbers (64 tokens a block) fit an int.
int check_cache4(const void* k, const void* v, const void* scales, int n_blocks, int H_kv) {
  if (n_blocks < 0 || H_kv <= 0) return SAKI_ERR_ARG;
  if ((long long)n_blocks * H_kv > INT_MAX / kTile || H_kv > 32767) return SAKI_ERR_UNSUPPORTED;
  if (n_blocks > 0 && (!k || !v || !scales || !aligned(k, 16) || !aligned(v, 16) || !aligned(scales, 16)))
    return SAKI_ERR_ARG;
  return SAKI_OK;
}

}  // namespace
