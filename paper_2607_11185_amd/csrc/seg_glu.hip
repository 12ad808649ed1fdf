// Gated feed-forward block silu(x Wg^T) * (x Wu^T) with its backward.
//
// Forward: one GEMM launch for both projections; its epilogue forms the product
// from the fp32 accumulators (one rounding, of m), and can keep the gate and up
// values for the backward, in bf16 or in 8 bits with a power of two per 32
// features (act8.h).  Backward: one streaming pass turns the kept values and dm
// into dg and du, and two GEMM launches give dx = dg Wg + du Wu (one sum over
// both contractions) and both weight gradients.
#include <algorithm>
#include <cmath>

#include "act8.h"
#include "common.h"
#include "gemm.h"
#include "glu.h"

namespace seg {
namespace {

using gemm::EpiOut;
using gemm::ST;

constexpr int MAX_DIM = 1 << 20;  // GEMM rows are addressed with 32-bit offsets
constexpr long MAX_SUMS = 64L << 20;  // fp32 partial sums of a launch at most (256 MB)

// s = 1 / (1 + exp(-g)): the reciprocal and one step towards 1 / x, which has the bits of
// the division 1.f / x at every float x in [1, 2^126) (found on this card by trying them
// all, which no test repeats); the fixup makes inf 0 and keeps NaN.  Beyond (g < -87.3) 1 / x
// is a subnormal number, which the reciprocal does not give: there, for all N together as
// it is rare, the division itself.  Against divisions throughout: 8192 x 3584 x 2 x 18944 with
// kept values read back 1779 -> 1760 us, 1500 x 2048 x 2 x 5504 82.4 -> 81.1 (without the rare
// branch, and zeros beyond, 1757 and 81.1).
template <int N>
__device__ __forceinline__ void sigmoids(const float (&g)[N], float (&s)[N]) {
  float x[N], top = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    x[j] = 1.f + __expf(-g[j]);
    top = fmaxf(top, x[j]);
    const float r = __builtin_amdgcn_rcpf(x[j]);
    s[j] = __builtin_amdgcn_div_fixupf(fmaf(fmaf(-x[j], r, 1.f), r, r), x[j], 1.f);
  }
  if (top >= 0x1p126f) {
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = 1.f / x[j];
  }
}

enum Keep { NONE, BF16, CODES };

// Epilogue of the GEMM over pairs of gate and up blocks (gemm.h, kPair): columns
// 0..31 of a wave tile hold the gate, 32..63 the up values of the same 32
// features.  m [rows][I] bf16 and the kept values leave through the wave's LDS, 32
// rows x 32 features at a time, so that a lane stores 8 features of a row.  A
// wave tile's 32 features are one block of the 8-bit format: the four lanes
// that share a row find its largest magnitudes with two exchanges.
template <Keep KEEP>
struct EpiGlu {
  static constexpr bool kSwap = true, kPair = true;
  const unsigned short *second;  // up projection
  int features;                  // I
  unsigned short *m;
  glu::Kept k;
  template <int NI, int NJ>
  __device__ __forceinline__ void operator()(const f32x4 (&acc)[NI][NJ], const gemm::Tile &t) const {
    static_assert(NJ == 4, "64-column wave tiles");
    if (t.n0 + t.wc >= t.N) return;
    const int lane = t.grp * 16 + t.col, q = lane & 3;
    const int f0 = (t.n0 + t.wc) / 2, f = f0 + q * 8;  // the wave tile's features, the lane's when storing
    const long I = features;
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    // bf16 [3 outputs][32 rows][8 chunks of 4 features] (2 KB each), chunk c of
    // row r in slot c ^ (r & 6): pairs of chunks stay together.  Codes [2][32
    // rows][8 dwords of 4 features] behind m's 2 KB, swizzled the same way.
    gemm::u32x2 *w = reinterpret_cast<gemm::u32x2 *>(t.lds);
    unsigned *wc = reinterpret_cast<unsigned *>(t.lds + 2048);
#pragma unroll
    for (int bm = 0; bm < NI / 2; ++bm) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x4 *g = &acc[bm * 2 + i][0], *u = &acc[bm * 2 + i][2];
        unsigned cg[2], cu[2];
        if constexpr (KEEP == CODES) {
          unsigned tg = 0, tu = 0;
          float vg[8], vu[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            vg[j] = g[j / 4][j & 3];
            vu[j] = u[j / 4][j & 3];
            tg = max(tg, act8::mag(vg[j]));
            tu = max(tu, act8::mag(vu[j]));
          }
          const int eg = act8::exp_byte(act8::max_groups(tg)), eu = act8::exp_byte(act8::max_groups(tu));
          act8::codes(vg, eg, cg);
          act8::codes(vu, eu, cu);
          const int row = t.m0 + t.wr + bm * 32 + i * 16 + t.col;
          const long at = (long)row * ((I + act8::BLOCK - 1) / act8::BLOCK) + f0 / act8::BLOCK;
          if (row < t.M && t.grp == 0) k.g8.exp[at] = (uint8_t)eg;
          if (row < t.M && t.grp == 1) k.u8.exp[at] = (uint8_t)eu;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x4 gv = g[j], uv = u[j];
          const float ga[4] = {gv[0], gv[1], gv[2], gv[3]};
          float sg[4], mv[4];
          sigmoids(ga, sg);
#pragma unroll
          for (int r = 0; r < 4; ++r) mv[r] = gv[r] * sg[r] * uv[r];
          const int at = (i * 16 + t.col) * 8 + ((j * 4 + t.grp) ^ (t.col & 6));
          w[at] = gemm::u32x2{gemm::pack2(mv[0], mv[1]), gemm::pack2(mv[2], mv[3])};
          if constexpr (KEEP == BF16) {
            w[256 + at] = gemm::u32x2{gemm::pack2(gv[0], gv[1]), gemm::pack2(gv[2], gv[3])};
            w[512 + at] = gemm::u32x2{gemm::pack2(uv[0], uv[1]), gemm::pack2(uv[2], uv[3])};
          }
          if constexpr (KEEP == CODES) {
            wc[at] = cg[j];
            wc[256 + at] = cu[j];
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
      if (f < I) {  // I is a multiple of 8
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const int r = p * 16 + (lane >> 2), row = t.m0 + t.wr + bm * 32 + r;
          const int at = r * 8 + ((2 * q) ^ (r & 6));
          if (row < t.M) {
            const long off = (long)row * I + f;
            *reinterpret_cast<u32x4 *>(m + off) = *reinterpret_cast<const u32x4 *>(w + at);
            if constexpr (KEEP == BF16) {
              *reinterpret_cast<u32x4 *>(k.g16 + off) = *reinterpret_cast<const u32x4 *>(w + 256 + at);
              *reinterpret_cast<u32x4 *>(k.u16 + off) = *reinterpret_cast<const u32x4 *>(w + 512 + at);
            }
            if constexpr (KEEP == CODES) {
              *reinterpret_cast<gemm::u32x2 *>(k.g8.code + off) = *reinterpret_cast<const gemm::u32x2 *>(wc + at);
              *reinterpret_cast<gemm::u32x2 *>(k.u8.code + off) =
                  *reinterpret_cast<const gemm::u32x2 *>(wc + 256 + at);
            }
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// The epilogue's work on a rest's tiles from their partial sums: 16 blocks a tile,
// 8 features of a row a thread, four lanes a block of 32 features.
template <Keep KEEP>
__global__ void __launch_bounds__(256) k_finish_glu(const gemm::RestTiles<1> t, const EpiGlu<KEEP> ep) {
  const int local = blockIdx.x / 16, chunk = (blockIdx.x % 16) * 256 + threadIdx.x;
  int mt, nt;
  gemm::tile_of(t.t0 + local, (t.M[0] + 255) / 256, (t.N[0] + gemm::BN - 1) / gemm::BN, mt, nt);
  const int r = chunk / 16, c = chunk % 16, col = c / 4 * 64 + c % 4 * 8;  // the gate's columns in the tile
  const int row = mt * 256 + r, f = nt * (gemm::BN / 2) + c * 8;
  const long I = ep.features;
  const bool in = row < t.M[0] && f < I;
  float g[8], u[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] = u[j] = 0.f;
  if (in) {
    t.sum8(local, r, col, g);
    t.sum8(local, r, col + 32, u);
  }
  int eg = 0, eu = 0;
  if constexpr (KEEP == CODES) {
    unsigned tg = 0, tu = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      tg = max(tg, act8::mag(g[j]));
      tu = max(tu, act8::mag(u[j]));
    }
    eg = act8::exp_byte(act8::max4(tg));
    eu = act8::exp_byte(act8::max4(tu));
  }
  if (!in) return;
  const long off = (long)row * I + f;
  u16x8 m;
  float sg[8];
  sigmoids(g, sg);
#pragma unroll
  for (int j = 0; j < 8; ++j) m[j] = f2bf_bits(g[j] * sg[j] * u[j]);
  *reinterpret_cast<u16x8 *>(ep.m + off) = m;
  if constexpr (KEEP == BF16) {
    u16x8 a, b;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      a[j] = f2bf_bits(g[j]);
      b[j] = f2bf_bits(u[j]);
    }
    *reinterpret_cast<u16x8 *>(ep.k.g16 + off) = a;
    *reinterpret_cast<u16x8 *>(ep.k.u16 + off) = b;
  }
  if constexpr (KEEP == CODES) {
    const long at = (long)row * ((I + act8::BLOCK - 1) / act8::BLOCK) + f / act8::BLOCK;
    if (c % 4 == 0) {
      ep.k.g8.exp[at] = (uint8_t)eg;
      ep.k.u8.exp[at] = (uint8_t)eu;
    }
    unsigned cg[2], cu[2];
    act8::codes(g, eg, cg);
    act8::codes(u, eu, cu);
    *reinterpret_cast<uint2 *>(ep.k.g8.code + off) = make_uint2(cg[0], cg[1]);
    *reinterpret_cast<uint2 *>(ep.k.u8.code + off) = make_uint2(cu[0], cu[1]);
  }
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// x and weights of a forward for few rows.
struct RowsArgs {
  const unsigned short *x, *wg, *wu;
  long ldx;
  int rows, hidden;
};

// Features of a block of the kernels for few rows: one block of the 8-bit format.
constexpr int FEATURES = act8::BLOCK;
constexpr int FEW = 2;      // rows that k_glu_few takes at most
constexpr int ROWS = 64;    // and k_glu_rows
constexpr int PARTS = 4;    // of K, k_glu_few; each four waves
constexpr unsigned FEW_LDS = 64u << 10;

// The forward for a handful of rows (at most T), where the weights' bytes are all
// the work.  Measured, plain reads reach 6.7 TB/s when a load takes whole 128-byte
// lines past the caches (__builtin_nontemporal_load), 6.0 through them, and 5.0 past
// them in the half lines of a matrix product's operand layout.  So no matrix product: a
// load takes 64 k of 8 features, a lane 8 k of one, and multiplies them with its k of
// every row of x, which lies in LDS as all waves need it.  A block takes 32 features;
// four waves of it 8 of them each, and four such groups a quarter of K each.  The
// eight lanes of a feature add up by exchange, the quarters in LDS, in order.
// 3,584 x 2 x 18,944, 1 / 2 / 4 rows: 46.7 / 47.1 / 49.0 us (5.8 / 5.8 / 5.5 TB/s;
// k_glu_rows takes 47.1 / 47.1 / 47.3); 2,048 x 2 x 5,504: 10.9 / 11.3 / 11.5 (11.7);
// 896 x 2 x 4,864: 6.0 / 6.0 / 7.1 (6.4).  With K in halves 47 us and 15.5.
template <int T, Keep KEEP>
__global__ void __launch_bounds__(256 * PARTS) k_glu_few(const RowsArgs a, const EpiGlu<KEEP> ep) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float sums[PARTS][2][T][FEATURES];  // part of K, gate or up, row, feature
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int H = a.hidden, I = ep.features, f0 = blockIdx.x * FEATURES;
  const int steps = (H + 63) / 64, per = (steps + PARTS - 1) / PARTS;  // of a part
  bf16x8 *xs = reinterpret_cast<bf16x8 *>(lds);                        // [T][steps * 8]
  const int part = wave % PARTS, grp = wave / PARTS, c = lane & 7;
  const int f = min(f0 + 8 * grp + (lane >> 3), I - 1);  // past the end: the last, unused
  const unsigned short *pg = a.wg + (long)f * H + 8 * c, *pu = a.wu + (long)f * H + 8 * c;
  const int s0 = part * per, s1 = min(steps, s0 + per);
  struct Step {
    bf16x8 g, u;
  };
  auto load = [&](Step &w, int s) __attribute__((always_inline)) {
    const bool in = s < s1 && s * 64 + 8 * c < H;
    w.g = in ? __builtin_nontemporal_load(reinterpret_cast<const bf16x8 *>(pg + s * 64)) : bf16x8{};
    w.u = in ? __builtin_nontemporal_load(reinterpret_cast<const bf16x8 *>(pu + s * 64)) : bf16x8{};
  };
  Step w0, w1;
  load(w0, s0);
  load(w1, s0 + 1);
  for (int e = threadIdx.x; e < T * steps * 8; e += 256 * PARTS) {
    const int t = e / (steps * 8), k = (e - t * steps * 8) * 8;
    xs[e] = t < a.rows && k < H ? *reinterpret_cast<const bf16x8 *>(a.x + t * a.ldx + k) : bf16x8{};
  }
  __syncthreads();
  float g[T], u[T];
#pragma unroll
  for (int t = 0; t < T; ++t) g[t] = u[t] = 0.f;
  auto products = [&](const Step &w, int s) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const bf16x8 x = xs[(t * steps + s) * 8 + c];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bf16x2 xj = bf16x2{x[2 * j], x[2 * j + 1]};
        g[t] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w.g[2 * j], w.g[2 * j + 1]}, xj, g[t], false);
        u[t] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w.u[2 * j], w.u[2 * j + 1]}, xj, u[t], false);
      }
    }
  };
  for (int s = s0; s < s1; s += 2) {
    products(w0, s);
    load(w0, s + 2);
    if (s + 1 >= s1) break;
    products(w1, s + 1);
    load(w1, s + 3);
  }
#pragma unroll
  for (int t = 0; t < T; ++t) {
#pragma unroll
    for (int o = 1; o <= 4; o *= 2) {
      g[t] += __shfl_xor(g[t], o, 64);
      u[t] += __shfl_xor(u[t], o, 64);
    }
    if (c == 0) {
      sums[part][0][t][8 * grp + (lane >> 3)] = g[t];
      sums[part][1][t][8 * grp + (lane >> 3)] = u[t];
    }
  }
  __syncthreads();
  if (threadIdx.x >= FEATURES * T) return;
  const int t = threadIdx.x / FEATURES, fi = threadIdx.x % FEATURES;
  float gv = sums[0][0][t][fi], uv = sums[0][1][t][fi];
#pragma unroll
  for (int p = 1; p < PARTS; ++p) {
    gv += sums[p][0][t][fi];
    uv += sums[p][1][t][fi];
  }
  const bool in = t < a.rows && f0 + fi < I;
  const long off = (long)t * I + f0 + fi;
  if constexpr (KEEP == CODES) {
    unsigned tg = in ? act8::mag(gv) : 0u, tu = in ? act8::mag(uv) : 0u;
#pragma unroll
    for (int o = 1; o <= 16; o *= 2) {
      tg = max(tg, (unsigned)__shfl_xor((int)tg, o, 64));
      tu = max(tu, (unsigned)__shfl_xor((int)tu, o, 64));
    }
    const int eg = act8::exp_byte(tg), eu = act8::exp_byte(tu);
    if (in) {
      const long at = (long)t * ((I + act8::BLOCK - 1) / act8::BLOCK) + blockIdx.x;
      if (fi == 0) {
        ep.k.g8.exp[at] = (uint8_t)eg;
        ep.k.u8.exp[at] = (uint8_t)eu;
      }
      float vg[4] = {gv, 0.f, 0.f, 0.f}, vu[4] = {uv, 0.f, 0.f, 0.f};
      unsigned cg[1], cu[1];
      act8::codes(vg, eg, cg);
      act8::codes(vu, eu, cu);
      ep.k.g8.code[off] = (int8_t)cg[0];
      ep.k.u8.code[off] = (int8_t)cu[0];
    }
  }
  if (!in) return;
  const float ga[1] = {gv};
  float sg[1];
  sigmoids(ga, sg);
  ep.m[off] = f2bf_bits(gv * sg[0] * uv);
  if constexpr (KEEP == BF16) {
    ep.k.g16[off] = f2bf_bits(gv);
    ep.k.u16[off] = f2bf_bits(uv);
  }
}

// The forward for some tens of rows (16 NB at most): a block takes 32 features, its
// waves every WAVES-th step of 64 of K, and their sums are added up in LDS, in order.
// The weights' bytes are the work, and memory gives them fastest in whole 128-byte lines
// (k_glu_few), which are not the layout of a matrix product's operand: there a load
// takes 64 bytes of 16 rows.  So a lane's 16 bytes, 8 rows to a load, go through the
// wave's own 8 KB of LDS (chunk c of row r in slot c ^ (r & 7): no conflicts), first
// those of x, then the weights', while the loads of the wave's next step are under
// way; no wave waits for another.  Lanes past the last feature or row read the last
// one, and their sums go nowhere; what lies past K reads as zeros.  16 / 32 / 64 rows:
// 3,584 x 2 x 18,944 48.7 / 54.8 / 66 us (5.6 / 5.0 / 4.1 TB/s; the GEMM 62 to 66; both
// operands from memory in their layout 71 / 82 / 103, x alone 50 / 58 / 76); 2,048 x 2 x
// 5,504 11.5 / 13.7 / 18.0 (30).  x a step later, which saves its second set of registers,
// takes 53 / 62 / 82; four waves for 16 rows 51 and 13.0, eight for 64 rows 83 and 18.7.
template <int NB, int WAVES, Keep KEEP>
__global__ void __launch_bounds__(64 * WAVES, NB < 4 ? 4 : 2) k_glu_rows(const RowsArgs a, const EpiGlu<KEEP> ep) {
  // [wave][64 weight rows: 32 of wg, 32 of wu][8 chunks], then the waves' sums
  constexpr int STAGE = WAVES * 64 * 8, SUMS = WAVES * 4 * NB * 64;
  __shared__ __attribute__((aligned(1024))) f32x4 lds[STAGE > SUMS ? STAGE : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, grp = lane >> 4, lr = lane >> 3, lc = lane & 7;
  const int f0 = blockIdx.x * FEATURES, I = ep.features, H = a.hidden;
  const unsigned short *wg = a.wg + (long)f0 * H, *wu = a.wu + (long)f0 * H;
  unsigned off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) off[i] = (unsigned)min(8 * i + lr, I - 1 - f0) * (unsigned)H + 8 * lc;
  unsigned xoff[2 * NB];
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i) xoff[i] = (unsigned)min(8 * i + lr, a.rows - 1) * (unsigned)a.ldx + 8 * lc;
  bf16x8 w[8], x[2 * NB];
  auto load = [&](int k) __attribute__((always_inline)) {
    const bool in = k + 8 * lc < H;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned short *p = (i < 4 ? wg : wu) + k + off[i & 3];
      w[i] = in ? __builtin_nontemporal_load(reinterpret_cast<const bf16x8 *>(p)) : bf16x8{};
    }
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) x[i] = in ? *reinterpret_cast<const bf16x8 *>(a.x + k + xoff[i]) : bf16x8{};
  };
  f32x4 acc[4][NB];
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int n = 0; n < NB; ++n) acc[b][n] = f32x4{};
  bf16x8 *stage = reinterpret_cast<bf16x8 *>(lds) + wave * (64 * 8);
  bf16x8 *to = stage + lr * 8 + (lc ^ lr);
  const bf16x8 *from = stage + r * 8;
  int k = wave * 64;
  load(k);
  for (; k < H; k += 64 * WAVES) {
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) to[64 * i] = x[i];
    __builtin_amdgcn_wave_barrier();
    bf16x8 cx[2][NB];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < NB; ++n) cx[h][n] = from[n * 128 + ((4 * h + grp) ^ (r & 7))];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 8; ++i) to[64 * i] = w[i];
    __builtin_amdgcn_wave_barrier();
    load(k + 64 * WAVES);
    // features of block b against rows of block n: a lane holds row 16 n + lane % 16,
    // features 4 (lane / 16) .. + 3
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const bf16x8 cw = from[b * 128 + ((4 * h + grp) ^ (r & 7))];
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[b][n] = mfma16(cw, cx[h][n], acc[b][n]);
      }
    __builtin_amdgcn_wave_barrier();
  }
  f32x4(*sums)[4 * NB][64] = reinterpret_cast<f32x4(*)[4 * NB][64]>(lds);
  __syncthreads();
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int n = 0; n < NB; ++n) sums[wave][b * NB + n][lane] = acc[b][n];
  __syncthreads();
  if (wave >= NB) return;
  const int row = 16 * wave + r;
  f32x4 v[4];  // gate of features 4 grp .. and 16 + 4 grp .., up of the same
#pragma unroll
  for (int b = 0; b < 4; ++b) v[b] = sums[0][b * NB + wave][lane];
#pragma unroll 1  // (unrolled, these reads take more registers than the products)
  for (int q = 1; q < WAVES; ++q)
#pragma unroll
    for (int b = 0; b < 4; ++b) v[b] += sums[q][b * NB + wave][lane];
  int eg = 0, eu = 0;
  if constexpr (KEEP == CODES) {
    unsigned tg = 0, tu = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if (f0 + 16 * b + 4 * grp >= I) continue;  // I is a multiple of 8
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        tg = max(tg, act8::mag(v[b][j]));
        tu = max(tu, act8::mag(v[2 + b][j]));
      }
    }
    eg = act8::exp_byte(act8::max_groups(tg));
    eu = act8::exp_byte(act8::max_groups(tu));
    const long at = (long)row * ((I + act8::BLOCK - 1) / act8::BLOCK) + blockIdx.x;
    if (row < a.rows && grp == 0) ep.k.g8.exp[at] = (uint8_t)eg;
    if (row < a.rows && grp == 1) ep.k.u8.exp[at] = (uint8_t)eu;
  }
  if (row >= a.rows) return;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int f = f0 + 16 * b + 4 * grp;
    if (f >= I) continue;
    const f32x4 g = v[b], u = v[2 + b];
    const float ga[4] = {g[0], g[1], g[2], g[3]};
    float sg[4], m[4];
    sigmoids(ga, sg);
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = g[j] * sg[j] * u[j];
    const long off = (long)row * I + f;
    *reinterpret_cast<gemm::u32x2 *>(ep.m + off) = gemm::u32x2{gemm::pack2(m[0], m[1]), gemm::pack2(m[2], m[3])};
    if constexpr (KEEP == BF16) {
      *reinterpret_cast<gemm::u32x2 *>(ep.k.g16 + off) = gemm::u32x2{gemm::pack2(g[0], g[1]), gemm::pack2(g[2], g[3])};
      *reinterpret_cast<gemm::u32x2 *>(ep.k.u16 + off) = gemm::u32x2{gemm::pack2(u[0], u[1]), gemm::pack2(u[2], u[3])};
    }
    if constexpr (KEEP == CODES) {
      float vg[4] = {g[0], g[1], g[2], g[3]}, vu[4] = {u[0], u[1], u[2], u[3]};
      unsigned cg[1], cu[1];
      act8::codes(vg, eg, cg);
      act8::codes(vu, eu, cu);
      *reinterpret_cast<unsigned *>(ep.k.g8.code + off) = cg[0];
      *reinterpret_cast<unsigned *>(ep.k.u8.code + off) = cu[0];
    }
  }
}

// dg = dm * u * silu'(g), du = dm * silu(g), silu'(g) = s (1 + g (1 - s)),
// s = sigmoid(g), and m = silu(g) * u; 8 features a thread.  A streaming kernel:
// folded into the epilogue of the GEMM that makes dm its loads stall the one
// wave per SIMD.  dg and du round to bf16, as the matrix cores take them: dx and the
// weight gradients are then off by 0.0024 of their norm, not the 0.0017 of their own rounding
// (two bf16 terms each would double both products).  Gate and up values that the backward
// computes again come in bf16, too: their rounding is as large as that of dg and du, and fp32
// would write and read 8 more bytes an element beside the 16 of both kernels.
template <Keep KEEP>
__global__ void __launch_bounds__(256) k_glu_bwd(const glu::Kept k, const unsigned short *__restrict__ dm,
                                                 unsigned short *__restrict__ dg, unsigned short *__restrict__ du,
                                                 unsigned short *__restrict__ m, long n8, int row8) {
  for (long c = (long)blockIdx.x * 256 + threadIdx.x; c < n8; c += (long)gridDim.x * 256) {
    float g[8], u[8];
    if constexpr (KEEP == BF16) {
      const u16x8 gv = *reinterpret_cast<const u16x8 *>(k.g16 + c * 8);
      const u16x8 uv = *reinterpret_cast<const u16x8 *>(k.u16 + c * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        g[j] = bf_bits2f(gv[j]);
        u[j] = bf_bits2f(uv[j]);
      }
    } else {
      const long row = c / row8;
      const long at = row * ((row8 + 3) / 4) + (c - row * row8) / 4;
      const uint2 gc = *reinterpret_cast<const uint2 *>(k.g8.code + c * 8);
      const uint2 uc = *reinterpret_cast<const uint2 *>(k.u8.code + c * 8);
      const unsigned gw[2] = {gc.x, gc.y}, uw[2] = {uc.x, uc.y};
      act8::values8(gw, act8::scale(k.g8.exp[at]), g);
      act8::values8(uw, act8::scale(k.u8.exp[at]), u);
    }
    const u16x8 mv = *reinterpret_cast<const u16x8 *>(dm + c * 8);
    u16x8 og, ou, om;
    float sg[8];
    sigmoids(g, sg);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = bf_bits2f(mv[j]), s = sg[j];
      og[j] = f2bf_bits(d * u[j] * s * (1.f + g[j] * (1.f - s)));
      ou[j] = f2bf_bits(d * g[j] * s);
      om[j] = f2bf_bits(g[j] * s * u[j]);
    }
    *reinterpret_cast<u16x8 *>(dg + c * 8) = og;
    *reinterpret_cast<u16x8 *>(du + c * 8) = ou;
    if (m) *reinterpret_cast<u16x8 *>(m + c * 8) = om;
  }
}

unsigned few_lds(int rows, int hidden) { return (unsigned)((hidden + 63) / 64 * 128) * rows; }

// Rows of x that the kernel for few rows is built for (1 or 2; 16, 32 or 64 for
// k_glu_rows), or 0 where the GEMM serves.  One or two rows go to k_glu_few if x fits its
// LDS.  Beyond, the time of each is that of the weights' bytes, or of its steps where
// there are few blocks, as measured: k_glu_rows 5.3, 4.9 and 4.3 TB/s, and 2.0, 2.3 and
// 1.55 us for a wave's step of 64; the GEMM's tiles take 1.12 of what choose() expects
// when the weights come from memory, which give 5.4 TB/s at most.  Measured, 16 / 32 / 64
// rows, k_glu_rows / GEMM: 8,192 x 2 x 28,672 182 / 191 / 200 and 176 / 171 / 172 us;
// 4,096 x 2 x 14,336 43 / 47 / 52 and 69; 8,192 x 2 x 4,096 36 / 41 / 53 and 45 / 46 / 47;
// 512 x 2 x 18,944 10 / 14 / 14 and 15 / 14 / 14; 16,384 x 2 x 2,048 54 / 62 / 88 and 45.
int few_rows(int rows, int hidden, int inter, double gemm_us) {
  if (rows <= FEW && few_lds(rows, hidden) + PARTS * 2 * rows * FEATURES * 4 <= FEW_LDS) return rows;
  if (rows > ROWS) return 0;
  const int n = rows <= 16 ? 0 : rows <= 32 ? 1 : 2;
  constexpr double RATE[3] = {5.3, 4.9, 4.3}, STEP[3] = {2.0, 2.3, 1.55};
  const double mb = 4e-6 * hidden * inter, steps = (hidden + 63) / 64;
  const double us = 4 + std::max(mb / RATE[n], STEP[n] * std::ceil(steps / (n < 2 ? 8 : 4)));
  return us < std::max(1.12 * gemm_us, 4 + mb / 5.4) ? 16 << n : 0;
}

template <class Epi>
void launch_few(int t, const RowsArgs &a, const Epi &ep, hipStream_t st) {
  const unsigned nb = (unsigned)act8::blocks_of(ep.features), lds = t <= FEW ? few_lds(t, a.hidden) : 0;
  switch (t) {
    case 1: k_glu_few<1><<<nb, 256 * PARTS, lds, st>>>(a, ep); break;
    case 2: k_glu_few<2><<<nb, 256 * PARTS, lds, st>>>(a, ep); break;
    case 16: k_glu_rows<1, 8><<<nb, 64 * 8, 0, st>>>(a, ep); break;
    case 32: k_glu_rows<2, 8><<<nb, 64 * 8, 0, st>>>(a, ep); break;
    default: k_glu_rows<4, 4><<<nb, 64 * 4, 0, st>>>(a, ep); break;
  }
  SEG_LAUNCH_CHECK();
}

int pair_columns(int inter) { return 2 * (int)act8::blocks_of(inter) * act8::BLOCK; }

// How a forward of its own (not a chunk of a layer) is launched: few (few_rows), or a
// GEMM with up to MAX_SUMS partial sums.
struct Forward {
  gemm::Choice c;
  int few;
};

Forward choose_fwd(int rows, int hidden, int inter) {
  const int N = pair_columns(inter);
  const long steps = (hidden + gemm::BK - 1) / gemm::BK;
  const long t4 = gemm::tiles_of(rows, N, 4), t2 = gemm::tiles_of(rows, N, 2);
  const gemm::Choice c = gemm::choose_even(gemm::choose(t4, t2, steps, 1, 0), t4, steps, MAX_SUMS);
  return Forward{c, few_rows(rows, hidden, inter, c.us)};
}

size_t fwd_sums(int rows, int hidden, int inter) {
  const Forward f = choose_fwd(rows, hidden, inter);
  const gemm::Choice &c = f.c;
  if (f.few || !c.rest || c.parts == 1) return 256;
  return (size_t)c.parts * (gemm::tiles_of(rows, pair_columns(inter), 4) - c.full) * gemm::bm_of(4) * gemm::BN * 4;
}

}  // namespace

namespace glu {

void forward(const unsigned short *x, long ldx, const unsigned short *wg, const unsigned short *wu, int rows,
             int hidden, int inter, unsigned short *m, const Kept &keep, float *sums, hipStream_t st) {
  const int N = pair_columns(inter);
  const Forward how = sums ? choose_fwd(rows, hidden, inter) : Forward{gemm::Choice{4, 1, 0}, 0};
  const gemm::Choice &c = how.c;
  auto go = [&](auto ep) {
    if (how.few) {
      launch_few(how.few, RowsArgs{x, wg, wu, ldx, rows, hidden}, ep, st);
      return;
    }
    const auto g = gemm::one<false, false>(x, ldx, wg, hidden, rows, N, hidden, ep);
    if (!c.rest) {
      gemm::launch<false, false>(g, st);
      return;
    }
    gemm::launch_even<false, false>(g, c, sums, [&](const gemm::RestTiles<1> &t) {
      k_finish_glu<<<(unsigned)(t.cnt * 16), 256, 0, st>>>(t, ep);
      SEG_LAUNCH_CHECK();
    }, st);
  };
  if (keep.g16) go(EpiGlu<BF16>{wu, inter, m, keep});
  else if (keep.g8.code) go(EpiGlu<CODES>{wu, inter, m, keep});
  else go(EpiGlu<NONE>{wu, inter, m, keep});
}

void backward_act(const Kept &kept, const unsigned short *dm, int rows, int inter, unsigned short *dg,
                  unsigned short *du, unsigned short *m, hipStream_t st) {
  const long n8 = (long)rows * inter / 8;
  const unsigned nb = (unsigned)std::max<long>(1, std::min<long>(65536, (n8 + 255) / 256));
  if (kept.g16) k_glu_bwd<BF16><<<nb, 256, 0, st>>>(kept, dm, dg, du, m, n8, inter / 8);
  else k_glu_bwd<CODES><<<nb, 256, 0, st>>>(kept, dm, dg, du, m, n8, inter / 8);
  SEG_LAUNCH_CHECK();
}

}  // namespace glu

namespace {

struct GluWs {
  size_t dg, du, g, u, m, sums, total;
  long sum_elems;
};

GluWs glu_ws(int rows, int hidden, int inter, bool kept) {
  GluWs w{};
  Carver c(nullptr);
  auto take = [&](size_t bytes) {
    const size_t o = c.off;
    c.take<char>(std::max<size_t>(bytes, 1));
    return o;
  };
  const size_t R = std::max(rows, 1), H = hidden, I = inter;
  w.dg = take(R * I * 2);
  w.du = take(R * I * 2);
  if (!kept) {
    w.g = take(R * I * 2);
    w.u = take(R * I * 2);
    w.m = take(R * I * 2);
  }
  // partial sums of products cut over K: what 16 parts of the larger one take, its
  // tiles whole, up to MAX_SUMS (larger ones fill the chip uncut)
  const size_t t = std::max(gemm::tiles_of(R, H, 4), 2 * gemm::tiles_of(I, H, 4));
  w.sum_elems = (long)std::min<size_t>(MAX_SUMS, 16 * t * gemm::bm_of(4) * gemm::BN);
  w.sums = take(std::max<size_t>(w.sum_elems * 4, kept ? 0 : fwd_sums(rows, hidden, inter)));
  w.total = c.off;
  return w;
}

void check_glu(int32_t rows, int32_t hidden, int32_t inter, int64_t ldx) {
  SEG_CHECK(rows >= 0, SEG_ERR_ARG, "rows < 0");
  SEG_CHECK(hidden >= 8 && hidden % 8 == 0 && inter >= 8 && inter % 8 == 0, SEG_ERR_UNSUPPORTED,
            "hidden %d and inter %d must be positive multiples of 8", hidden, inter);
  SEG_CHECK(rows <= MAX_DIM && hidden <= MAX_DIM && inter <= MAX_DIM, SEG_ERR_UNSUPPORTED,
            "rows %d, hidden %d or inter %d above %d", rows, hidden, inter, MAX_DIM);
  const long f = act8::blocks_of(inter);  // (a launch holds fewer than 2^32 threads)
  SEG_CHECK(gemm::tiles_of(rows, 64 * f, 2) <= 1 << 22 && gemm::tiles_of(rows, hidden, 2) <= 1 << 22 &&
                2 * gemm::tiles_of(inter, hidden, 2) <= 1 << 22,
            SEG_ERR_CAPACITY, "rows %d, hidden %d and inter %d: too many tiles for one launch", rows, hidden, inter);
  SEG_CHECK(ldx >= hidden, SEG_ERR_ARG, "row stride %lld < hidden %d", (long long)ldx, hidden);
  SEG_CHECK(ldx % 8 == 0 && ldx <= MAX_DIM, SEG_ERR_UNSUPPORTED,
            "row stride %lld must be a multiple of 8 up to %d", (long long)ldx, MAX_DIM);
}

void check_aligned(std::initializer_list<const void *> p, uintptr_t to) {
  for (const void *x : p)
    SEG_CHECK(reinterpret_cast<uintptr_t>(x) % to == 0, SEG_ERR_UNSUPPORTED,
              "a tensor does not start on a %d-byte boundary", (int)to);
}

// both of g and u or none, whole
bool check_kept(const seg_act8 *g, const seg_act8 *u) {
  SEG_CHECK(!g == !u, SEG_ERR_ARG, "only one of the gate's and the up values' 8-bit arrays is given");
  if (!g) return false;
  SEG_CHECK(g->code && g->exp && u->code && u->exp, SEG_ERR_ARG, "an 8-bit array is NULL");
  check_aligned({g->code, u->code}, 8);
  return true;
}

#define US(p) reinterpret_cast<unsigned short *>(p)
#define CUS(p) reinterpret_cast<const unsigned short *>(p)

}  // namespace
}  // namespace seg

using namespace seg;

// For tests (not in seg.h; host only): how the forward (which = 0), dx (1) and the
// weight gradients (2) are launched; out = {rows of a tile, parts of K, 256-row
// tiles in whole rounds, whether there is a rest}, or {rows the kernel for few is
// built for, 0, 0, 0}.
extern "C" void seg_glu_gemm_choice(int32_t rows, int32_t hidden, int32_t inter, int32_t which, int32_t *out) {
  gemm::Choice c;
  const long sums = glu_ws(rows, hidden, inter, true).sum_elems;
  if (which == 0) {
    const Forward f = choose_fwd(rows, hidden, inter);
    if (f.few) {
      out[0] = f.few;
      out[1] = out[2] = out[3] = 0;
      return;
    }
    c = f.c;
  } else if (which == 1) {
    const int K[2] = {inter, inter};
    c = gemm::choose_even_group(1, &rows, &hidden, 2, K, sums);
  } else {
    const int M[2] = {inter, inter}, N[2] = {hidden, hidden};
    c = gemm::choose_even_group(2, M, N, 1, &rows, sums);
  }
  out[0] = gemm::bm_of(c.tm);
  out[1] = c.parts;
  out[2] = c.full;
  out[3] = c.rest;
}

extern "C" seg_status seg_glu_fwd(int32_t rows, int32_t hidden, int32_t inter, const void *x, int64_t ldx,
                                  const void *wg, const void *wu, void *m, const seg_act8 *g8,
                                  const seg_act8 *u8, void *ws, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    check_glu(rows, hidden, inter, ldx);
    if (rows == 0) return;
    SEG_CHECK(x && wg && wu && m, SEG_ERR_ARG, "x, a weight or m is NULL");
    check_aligned({x, wg, wu, m}, 16);
    const size_t need = fwd_sums(rows, hidden, inter);
    SEG_CHECK(ws_bytes >= need, SEG_ERR_WORKSPACE, "workspace of %zu bytes < required %zu", ws_bytes, need);
    SEG_CHECK(ws, SEG_ERR_ARG, "ws is NULL");
    check_aligned({ws}, 16);
    glu::Kept keep{};
    if (check_kept(g8, u8)) {
      keep.g8 = *g8;
      keep.u8 = *u8;
    }
    const size_t R = rows, H = hidden, I = inter, W = I * H * 2, E = R * act8::blocks_of(inter);
    check_apart({{m, R * I * 2}, {ws, need}, {keep.g8.code, R * I}, {keep.g8.exp, E}, {keep.u8.code, R * I}, {keep.u8.exp, E}},
                {{x, ((R - 1) * ldx + H) * 2}, {wg, W}, {wu, W}});
    ProfScope prof("glu_fwd", stream);
    glu::forward(CUS(x), ldx, CUS(wg), CUS(wu), rows, hidden, inter, US(m), keep, static_cast<float *>(ws), stream);
  });
}

extern "C" size_t seg_glu_workspace_bytes(int32_t rows, int32_t hidden, int32_t inter, int32_t bwd, int32_t kept) {
  if (rows < 0 || rows > MAX_DIM || hidden < 1 || hidden > MAX_DIM || inter < 1 || inter > MAX_DIM) return 0;
  return bwd ? glu_ws(rows, hidden, inter, kept != 0).total : fwd_sums(rows, hidden, inter);
}

extern "C" seg_status seg_glu_bwd(int32_t rows, int32_t hidden, int32_t inter, const void *x, int64_t ldx,
                                  const void *wg, const void *wu, const seg_act8 *g8, const seg_act8 *u8,
                                  const void *dm, void *m, void *dx, seg_dtype dw_dt, void *dwg, void *dwu,
                                  void *ws, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    check_glu(rows, hidden, inter, ldx);
    SEG_CHECK(dw_dt == SEG_BF16 || dw_dt == SEG_F32, SEG_ERR_UNSUPPORTED, "dtype %d not supported", (int)dw_dt);
    SEG_CHECK(dwg && dwu, SEG_ERR_ARG, "a gradient pointer is NULL");
    check_aligned({dwg, dwu}, 16);
    const long n = (long)inter * hidden;
    if (rows == 0) {
      fill32(dwg, dw_dt == SEG_BF16 ? n / 2 : n, 0u, stream);
      fill32(dwu, dw_dt == SEG_BF16 ? n / 2 : n, 0u, stream);
      return;
    }
    SEG_CHECK(x && wg && wu && dm && dx, SEG_ERR_ARG, "x, a weight, dm or dx is NULL");
    check_aligned({x, wg, wu, dm, m, dx}, 16);
    const bool has = check_kept(g8, u8);
    const GluWs W = glu_ws(rows, hidden, inter, has);
    SEG_CHECK(ws_bytes >= W.total, SEG_ERR_WORKSPACE, "workspace of %zu bytes < required %zu", ws_bytes, W.total);
    SEG_CHECK(ws, SEG_ERR_ARG, "ws is NULL");
    check_aligned({ws}, 16);
    const seg_act8 none{}, &gk = has ? *g8 : none, &uk = has ? *u8 : none;
    const size_t R = rows, H = hidden, I = inter, E = R * act8::blocks_of(inter), D = I * H * (dw_dt == SEG_BF16 ? 2 : 4);
    check_apart({{m, R * I * 2}, {dx, R * H * 2}, {dwg, D}, {dwu, D}, {ws, W.total}},
                {{x, ((R - 1) * ldx + H) * 2}, {wg, I * H * 2}, {wu, I * H * 2}, {dm, R * I * 2}, {gk.code, R * I},
                 {gk.exp, E}, {uk.code, R * I}, {uk.exp, E}});
    char *base = static_cast<char *>(ws);
    unsigned short *dg = US(base + W.dg), *du = US(base + W.du);
    const gemm::Scratch sums{reinterpret_cast<float *>(base + W.sums), W.sum_elems};
    {
      ProfScope prof("glu_act", stream);
      glu::Kept kept{};
      if (has) {
        kept.g8 = *g8;
        kept.u8 = *u8;
      } else {
        kept.g16 = US(base + W.g);
        kept.u16 = US(base + W.u);
        unsigned short *mm = m ? US(m) : US(base + W.m);
        glu::forward(CUS(x), ldx, CUS(wg), CUS(wu), rows, hidden, inter, mm, kept, sums.p, stream);
      }
      glu::backward_act(kept, CUS(dm), rows, inter, dg, du, has ? US(m) : nullptr, stream);
    }
    typedef EpiOut<unsigned short, ST> OutBf;
    {
      ProfScope prof("glu_dx", stream);
      gemm::Problems<OutBf, 1, 2> g{{{dg, du}}, {{CUS(wg), CUS(wu)}}, {{inter, inter}}, {{hidden, hidden}},
                                    {inter, inter}, {rows}, {hidden}, {OutBf::make(US(dx), hidden)}, {}, 1, 0};
      gemm::launch_even<false, true>(g, sums, stream);
    }
    ProfScope prof("glu_dw", stream);
    auto dw = [&](auto *a, auto *b) {
      typedef EpiOut<std::remove_pointer_t<decltype(a)>, ST> Out;
      gemm::Problems<Out, 2, 1> g{{{dg}, {du}}, {{CUS(x)}, {CUS(x)}}, {{inter}, {inter}}, {{ldx}, {ldx}}, {rows},
                                  {inter, inter}, {hidden, hidden}, {Out::make(a, hidden), Out::make(b, hidden)},
                                  {}, 1, 0};
      gemm::launch_even<true, true>(g, sums, stream);
    };
    if (dw_dt == SEG_BF16) dw(US(dwg), US(dwu));
    else dw(static_cast<float *>(dwg), static_cast<float *>(dwu));
  });
}
