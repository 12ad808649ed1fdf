// What the losses on the vocabulary projection share: the logits' product with the
// statistics of its softmax, dz from the logits, and the loss's sum.
#pragma once

#include <algorithm>

#include "common.h"
#include "gemm.h"

namespace seg {
namespace {

using gemm::EpiOut;
using gemm::ST;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// A part of a softmax's sum as it is kept: NaN without a maximum gets one, so that it reaches
// the whole.
__device__ __forceinline__ float2 part_of(float mx2, float sm) {
  return make_float2(sm != sm && mx2 == -INFINITY ? 0.f : mx2, sm);
}

// Epilogue of the logits GEMM (M = vocab, N = rows): writes zT, captures the
// target logit (TARGET) and the per-(row, vocab tile) max / sum-exp partials.
template <bool TARGET>
struct EpiLogits {
  float *zt;        // [M][ldz] fp32, or NULL (a forward-only call needs the statistics alone)
  long ldz;
  float2 *stats;    // [ceil(M/128) slabs][N]: (max, sum exp(z - max)) in log2 units
  int nrows;        // N
  const int32_t *target;  // [N]
  float *ztgt;      // [N]
  float scale;
  // zT is larger than the 256 MB last-level cache: its stores go past the
  // caches (a smaller one's stay, for the pass over it that follows: 1,024 x
  // 32,000, 46 us with them in the cache, 52 without)
  bool stream;
  static constexpr bool kSwap = false;
  // A lane holds 32 of the 128 vocabulary rows of one column n (three other
  // lanes the rest), so maximum, exponentials and sum mostly stay in the lane;
  // a wave covers one 128-row slab.  Only the slab that the vocabulary ends in
  // tests its rows, and only waves that hold a target look for it.  The
  // exponents come from the logits as they are stored, scaled and rounded first:
  // scale * log2(e) as one rounded factor moved every exponent of a row the same
  // way, up to 6e-8 of the logit (log-probs up to 1.7 times further off).
  template <int NI, int NJ>
  __device__ __forceinline__ void operator()(const f32x4 (&acc)[NI][NJ],
                                             const gemm::Tile &t) const {
    static_assert(NI == 8, "logits epilogue expects 128-row wave tiles");
    const int slab_row = t.m0 + t.wr;
    if (slab_row >= t.M) return;
    if (zt) {
      // 16 rows x 64 columns at a time through the wave's LDS: column c of row
      // r in place c ^ 16 (r / 4), stored 16 bytes a lane, 256 to a row (4
      // bytes a lane, 64 to a row: 7.3 ms for 7,680 rows x 3,584 x 151,936; so
      // 6.8, past the caches 6.6)
      float *w = reinterpret_cast<float *>(t.lds);
      const int lane = t.grp * 16 + t.col, n = t.n0 + t.wc + t.col * 4;
      float *zp = zt + (long)slab_row * ldz + n;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            w[(4 * t.grp + r) * 64 + ((16 * j + t.col) ^ (16 * t.grp))] = acc[i][j][r] * scale;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int rr = p * 4 + t.grp, row = 16 * i + rr;
          const f32x4 v = *reinterpret_cast<const f32x4 *>(w + rr * 64 + ((4 * t.col) ^ (16 * p)));
          if (n < ldz && slab_row + row < t.M) {
            f32x4 *d = reinterpret_cast<f32x4 *>(zp + (long)row * ldz);
            if (stream) __builtin_nontemporal_store(v, d);
            else *d = v;
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
    if (slab_row + 128 <= t.M) slab<true>(acc, t, slab_row);
    else slab<false>(acc, t, slab_row);
  }
  template <bool WHOLE, int NI, int NJ>
  __device__ __forceinline__ void slab(const f32x4 (&acc)[NI][NJ], const gemm::Tile &t,
                                       int slab_row) const {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int n = t.n0 + t.wc + j * 16 + t.col;
      const bool nok = n < t.N;
      // the lane's rows are base + k, k = 16 i + r
      const int base = slab_row + 4 * t.grp, left = t.M - base;
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int k = 16 * i + r;
          const float z = acc[i][j][r] * scale;
          if (WHOLE || k < left) mx = fmaxf(mx, z);
        }
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mx2 = mx * LOG2E;
      float sm = 0.f;
      if (mx != -INFINITY) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (WHOLE || 16 * i + r < left)
              sm += __builtin_amdgcn_exp2f(fmaf(acc[i][j][r] * scale, LOG2E, -mx2));
      } else if constexpr (!TARGET) {  // -inf and NaN alone
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if ((WHOLE || 16 * i + r < left) && acc[i][j][r] != acc[i][j][r]) sm = acc[i][j][r];
      }
      sm += __shfl_xor(sm, 16, 64);
      sm += __shfl_xor(sm, 32, 64);
      if (t.grp == 0 && nok)
        stats[(long)(slab_row / 128) * nrows + n] = TARGET ? make_float2(mx2, sm) : part_of(mx2, sm);
      if constexpr (TARGET) {
        const int at = (nok ? target[n] : -1) - base;  // the target as a k of the lane
        const bool mine = at >= 0 && at < min(116, left) && !(at & 12);
        if (__any(mine)) {
#pragma unroll
          for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (mine && at == 16 * i + r) ztgt[n] = acc[i][j][r] * scale;
        }
      }
    }
  }
};

// A part of a softmax's sum: the largest exponent (log2 units) and the sum below it
// (an all -inf part, or no part yet, adds nothing).
__device__ __forceinline__ float2 meet(float2 a, float2 p) {
  const float m2 = fmaxf(a.x, p.x);
  return make_float2(m2, (a.x == -INFINITY ? 0.f : a.y * exp2f(a.x - m2)) + (p.x == -INFINITY ? 0.f : p.y * exp2f(p.x - m2)));
}

// loss_sum = loss_scale * sum(loss_tok), fixed-order reduction by one block of
// 256 threads.
__device__ __forceinline__ void loss_sum_block(const float *__restrict__ loss_tok, int rows,
                                               float scale, float *__restrict__ out) {
  __shared__ double red[256];
  const int t = threadIdx.x;
  double s = 0.0;
#pragma unroll 8
  for (int i = t; i < rows; i += 256) s += (double)loss_tok[i];
  red[t] = s;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (t < o) red[t] += red[t + o];
    __syncthreads();
  }
  if (t == 0) *out = (float)(red[0] * (double)scale);
}

__global__ void __launch_bounds__(256) k_loss_sum(const float *__restrict__ loss_tok, int rows,
                                                  float scale, float *__restrict__ out) {
  loss_sum_block(loss_tok, rows, scale, out);
}

// dzT = g[r] * (onehot(target[r]) - exp(z - lse[r])), or (without TARGET) g[r] *
// exp(z - lse[r]), from zT [V][Rp] to bf16 [V][Rp], zero in the padded columns and,
// without TARGET, where g is zero.  Bound by HBM (6 bytes an element):
// a thread keeps lse, g and target of its 8 columns in registers and walks
// down the vocabulary rows of its block with 16-byte accesses.  One more row of
// the grid's blocks has its first block form loss_sum.
constexpr int DZ_COLS = 256;  // of a block of 256 threads

// Vocabulary rows per block: about 1,024 blocks, and no longer ones than
// hide the loads of lse, g and target (7,680 rows x 151,936: 1.86 ms with 32
// rows, 1.34 with 64, 1.31 with 256; 1,024 x 32,000: 70 us with 24, 45 with
// 64).
inline int dz_rows(int V, int Rp) {
  const long r = (long)V * ((Rp + DZ_COLS - 1) / DZ_COLS) / 1024 / 8 * 8;
  return (int)std::min<long>(128, std::max<long>(8, r));
}

template <bool TARGET>
__global__ void __launch_bounds__(256) k_dz(const float *__restrict__ zt, int V, int R, int Rp, int vrows,
                                            const float *__restrict__ lse,
                                            const float *__restrict__ g,
                                            const int32_t *__restrict__ target,
                                            unsigned short *__restrict__ dzt,
                                            const float *__restrict__ loss_tok, float loss_scale,
                                            float *__restrict__ loss_sum) {
  if (blockIdx.y == gridDim.y - 1) {
    if (blockIdx.x == 0) loss_sum_block(loss_tok, R, loss_scale, loss_sum);
    return;
  }
  const int r0 = blockIdx.x * DZ_COLS + (threadIdx.x & 31) * 8;
  if (r0 >= Rp) return;  // Rp is a multiple of 32
  float l[8], gr[8];
  int tg[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool ok = r0 + j < R;
    l[j] = ok ? lse[r0 + j] : 0.f;
    gr[j] = ok ? g[r0 + j] : 0.f;
    tg[j] = TARGET && ok ? target[r0 + j] : -1;
  }
  const int v1 = min(V, (int)(blockIdx.y + 1) * vrows);
#pragma unroll 4
  for (int v = blockIdx.y * vrows + (threadIdx.x >> 5); v < v1; v += 8) {
    const f32x4 *src = reinterpret_cast<const f32x4 *>(zt + (long)v * Rp + r0);
    const f32x4 a = src[0], b = src[1];
    u16x8 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float z = j < 4 ? a[j] : b[j - 4];
      // (x log2(e) rounded once in front of the hardware exponential is 16
      // times further from e^x at x = -12 and no faster at 7,680 rows x 151,936:
      // 1.30 against 1.31 ms; 49 against 51 us at 1,024 x 32,000)
      const float p = expf(z - l[j]);
      if constexpr (TARGET) o[j] = r0 + j < R ? f2bf_bits(gr[j] * ((v == tg[j] ? 1.f : 0.f) - p)) : 0;
      else o[j] = gr[j] == 0.f ? 0 : f2bf_bits(gr[j] * p);
    }
    *reinterpret_cast<u16x8 *>(dzt + (long)v * Rp + r0) = o;
  }
}

// 8 elements as bf16, with 16-byte accesses where `vec`
template <class TI>
__device__ __forceinline__ u16x8 load8(const TI *p, bool vec) {
  u16x8 r;
  if (vec && sizeof(TI) == 2) return *reinterpret_cast<const u16x8 *>(p);
  if (vec) {
    const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r[j] = f2bf_bits(a[j]);
      r[4 + j] = f2bf_bits(b[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = load_bf(p, j);
  }
  return r;
}

}  // namespace
}  // namespace seg
