// Activations in 8 bits: signed codes in blocks of 32 consecutive columns of a
// row (the last block of a row may be shorter), with one power of two a block:
// value = code 2^s, s least with max|x| <= 127 2^s and s >= -127, stored as the
// byte s + 127 (255: the block holds an infinity or a NaN, and reads as NaN; in
// the last one that fp32 reaches, codes stop at 63 and finite values stay finite).
// A power of two makes division and product exact, so the only rounding is that
// of x 2^-s to the nearest integer (ties to even), and a value has at most 8
// significant bits: bf16 holds it exactly, and so do the matrix products that
// read it.
#pragma once

#include "common.h"

namespace seg {
namespace act8 {

constexpr int BLOCK = 32;
constexpr int LAST = 249;  // the byte of fp32's largest numbers: 64 steps are 2^128, codes stop at 63
constexpr int NOT_FINITE = 255;

inline long blocks_of(long cols) { return (cols + BLOCK - 1) / BLOCK; }

// refuses what one launch of seg_act_pack or seg_act_unpack does not hold
void check_launch(long rows, long cols, seg_dtype dt);
// seg_act_pack and seg_act_unpack, timed under `name` (NULL: not)
void pack(int64_t rows, int32_t cols, seg_dtype dt, const void *x, int64_t ldx, const seg_act8 *out,
          const char *name, hipStream_t st);
void unpack(int64_t rows, int32_t cols, seg_dtype dt, const seg_act8 *in, void *x, int64_t ldx,
            const char *name, hipStream_t st);

// Magnitudes compare as their bits do, infinities and NaN above all numbers.
__device__ __forceinline__ unsigned mag(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }

// exponent byte of a block whose largest magnitude has the bits a: with a =
// 1.f 2^(e - 127), 127 2^s = 1.984375 2^(s + 6), so s + 127 is e - 6, or e - 5
// where 1.f is above 1.984375
__device__ __forceinline__ int exp_byte(unsigned a) {
  if (a >= 0x7f800000u) return NOT_FINITE;
  const int b = (int)(a >> 23) - 6 + ((a & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return b < 0 ? 0 : b;
}

// 2^-s of a finite block (byte at most 249)
__device__ __forceinline__ float inv_scale(int byte) {
  return __builtin_bit_cast(float, (unsigned)(254 - byte) << 23);
}

// 2^s (2^-127 is a subnormal number), NaN for a block that is not finite
__device__ __forceinline__ float scale(int byte) {
  const unsigned b = byte == 0 ? 1u << 22 : (unsigned)byte << 23;
  return __builtin_bit_cast(float, byte == NOT_FINITE ? 0x7fc00000u : b);
}

// Values as the codes hold them in the rare blocks of byte >= LAST: below 64 steps, or
// zeros where the block is not finite (whose 2^-s then is 0 too).
template <int N>
__device__ __forceinline__ float rare(float (&v)[N], int byte) {
  if (byte == NOT_FINITE) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = 0.f;
    return 0.f;
  }
  const float top = 63.f * 0x1p122f;
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = fminf(fmaxf(v[j], -top), top);
  return inv_scale(byte);
}

// codes of four values, lowest byte first; inv = 2^-s.  x 2^-s + 1.5 2^23 rounds to
// the nearest integer, ties to even, in one operation (the product is exact), and
// holds that integer in its low bits.
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d, float inv) {
  const float magic = 0x1.8p23f;
  const unsigned i = __builtin_bit_cast(unsigned, fmaf(a, inv, magic)), j = __builtin_bit_cast(unsigned, fmaf(b, inv, magic));
  const unsigned k = __builtin_bit_cast(unsigned, fmaf(c, inv, magic)), l = __builtin_bit_cast(unsigned, fmaf(d, inv, magic));
  // the low bytes side by side
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(l, k, 0x0c0c0400u), __builtin_amdgcn_perm(j, i, 0x0c0c0400u),
                               0x05040100u);
}

// codes of the N values (a multiple of 4) that a lane has of a block
template <int N>
__device__ __forceinline__ void codes(float (&v)[N], int byte, unsigned (&c)[N / 4]) {
  float inv = inv_scale(byte);
  if (byte >= LAST) inv = rare(v, byte);
#pragma unroll
  for (int q = 0; q < N / 4; ++q) c[q] = codes4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], inv);
}

// value j of four codes
__device__ __forceinline__ float value(unsigned codes, int j, float scale) {
  return (float)((int)(codes << (24 - 8 * j)) >> 24) * scale;
}

// The largest of a over aligned groups of 4 and of 8 lanes, by lane permutations inside
// the vector unit (a general exchange goes through LDS).
template <int CTRL>
__device__ __forceinline__ unsigned max_dpp(unsigned a) {
  return max(a, (unsigned)__builtin_amdgcn_mov_dpp((int)a, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ unsigned max4(unsigned a) {
  return max_dpp<0x4e>(max_dpp<0xb1>(a));  // lanes 1 0 3 2, then 2 3 0 1 of a quad
}
__device__ __forceinline__ unsigned max8(unsigned a) {
  return max_dpp<0x141>(max4(a));  // lane 7 - i of a group of 8
}

// The largest of a over lanes 16 and 32 apart (the four that share a row of a product's
// result).
__device__ __forceinline__ unsigned max_groups(unsigned a) {
  const auto p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  a = max(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  return max(q[0], q[1]);
}

// Eight codes of a chunk of columns, their block's scale with them.
__device__ __forceinline__ void values8(const unsigned (&w)[2], float sc, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = value(w[j / 4], j & 3, sc);
}

}  // namespace act8
}  // namespace seg
