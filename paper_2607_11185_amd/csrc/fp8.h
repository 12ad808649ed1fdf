// Tensors in 8-bit floating point (e4m3: 4 exponent and 3 mantissa bits, largest
// number 448, no infinities), with one power of two for each block of 128 columns
// of a row, or of 128 rows x 128 columns: value = number(code) 2^s, s least with
// max|x| <= 448 2^s and s >= -127, over the finite values of the block, stored as the
// byte s + 127.  Infinities and NaN are kept as NaN codes, each by itself, so that one
// of them spoils its own row and column of a product and not its block.  A power of
// two makes division and product exact: a code is the one rounding of x 2^-s (half a
// step is 2^-4 of the number, 2^-10 2^s below 2^-6 2^s), and the matrix cores take the
// bytes as they are.
// Layout, as the matrix product reads it: rows of codes are filled up with zero codes
// to 16 bytes; the bytes of one block of columns lie side by side, filled up to 16.
#pragma once

#include "common.h"

namespace seg {
namespace fp8 {

constexpr int BLOCK = 128;
constexpr int LAST = 247;  // the byte of fp32's largest numbers: 256 steps are 2^128, numbers stop at 240

inline long ld_code(long cols) { return (cols + 15) / 16 * 16; }
inline long blocks_of(long n) { return (n + BLOCK - 1) / BLOCK; }
inline long ld_exp(long rows, int block_rows) { return ((rows + block_rows - 1) / block_rows + 15) / 16 * 16; }
inline size_t code_bytes(long rows, long cols) { return (size_t)rows * ld_code(cols); }
inline size_t exp_bytes(long rows, long cols, int block_rows) {
  return (size_t)blocks_of(cols) * ld_exp(rows, block_rows);
}

// refuses arrays that are missing, misaligned or of another kind of block
inline void check(const seg_fp8 *p, const char *what) {
  SEG_CHECK(p, SEG_ERR_ARG, "%s: the struct of the 8-bit arrays is NULL", what);
  SEG_CHECK(p->block_rows == 1 || p->block_rows == BLOCK, SEG_ERR_UNSUPPORTED,
            "%s: blocks of %d rows, not of 1 or 128", what, p->block_rows);
  SEG_CHECK(p->code && p->exp, SEG_ERR_ARG, "%s: an 8-bit array is NULL", what);
  SEG_CHECK(reinterpret_cast<uintptr_t>(p->code) % 16 == 0 && reinterpret_cast<uintptr_t>(p->exp) % 16 == 0,
            SEG_ERR_UNSUPPORTED, "%s: an 8-bit array is not on a 16-byte boundary", what);
}

// Magnitudes of finite numbers compare as their bits do; infinities and NaN count as 0.
__device__ __forceinline__ unsigned mag(float x) {
  const unsigned a = __builtin_bit_cast(unsigned, x) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}

// byte of a block whose largest magnitude has the bits a: with a = 1.f 2^(e - 127), 448 2^s
// = 1.75 2^(s + 8), so s + 127 is e - 8, or e - 7 where 1.f is above 1.75
__device__ __forceinline__ int exp_byte(unsigned a) {
  const int b = (int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
  return b < 0 ? 0 : b;
}
// 2^-s (byte at most 247)
__device__ __forceinline__ float inv_scale(int byte) {
  return __builtin_bit_cast(float, (unsigned)(254 - byte) << 23);
}
// 2^s (2^-127 is a subnormal number); NaN for the byte 255, which packing does not write
__device__ __forceinline__ float scale(int byte) {
  const unsigned b = byte == 0 ? 1u << 22 : (unsigned)byte << 23;
  return __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : b);
}

// Codes of eight values, lowest byte first: the conversion rounds to nearest, ties to
// even, subnormal numbers among them, and makes NaN codes of infinities and NaN.
__device__ __forceinline__ uint2 codes8(float (&v)[8], int byte) {
  const float inv = inv_scale(byte);
  if (byte >= LAST) {  // finite values stay finite: below 256 steps
    const float top = 240.f * 0x1p120f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (mag(v[j])) v[j] = fminf(fmaxf(v[j], -top), top);
  }
  int a = 0, b = 0;
  a = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, a, false);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, a, true);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, b, false);
  b = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, b, true);
  return make_uint2((unsigned)a, (unsigned)b);
}

// The largest of a over aligned groups of 16 lanes, by lane permutations inside the
// vector unit: lanes 1 0 3 2 and 2 3 0 1 of a quad, lane 7 - i of eight, 8 lanes on.
__device__ __forceinline__ unsigned max16(unsigned a) {
  a = max(a, (unsigned)__builtin_amdgcn_mov_dpp((int)a, 0xb1, 0xf, 0xf, true));
  a = max(a, (unsigned)__builtin_amdgcn_mov_dpp((int)a, 0x4e, 0xf, 0xf, true));
  a = max(a, (unsigned)__builtin_amdgcn_mov_dpp((int)a, 0x141, 0xf, 0xf, true));
  return max(a, (unsigned)__builtin_amdgcn_mov_dpp((int)a, 0x128, 0xf, 0xf, true));
}

}  // namespace fp8
}  // namespace seg
