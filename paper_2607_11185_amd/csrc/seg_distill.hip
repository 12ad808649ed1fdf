// Divergence of the student's distribution over the vocabulary from a teacher's top
// logits, with gradients (bf16 MFMA on gfx950):
//   z = logit_scale h W^T, q = softmax(z); t_j = teacher_scale logits_j at the columns
//   ids_j; p = softmax(t), or exp(t - t_lse)
//   loss_r = weight_r sum_j p_j (log p_j - log q(ids_j))
//   d loss_r / d z_v = weight_r (q_v sum_j p_j - sum_{j: ids_j = v} p_j)
// The softmax over the vocabulary is that of the action-token loss (logits.h); the
// teacher has values at k columns of a row alone, so the gradient is one streaming pass
// over zT with one factor a row, and k places a row that are written again behind it.
// Pipeline:
//   1. hb = the rows of h that are used, as bf16;
//   2. zT[v][r] (MFMA, fp32 out) with per-(row, slab of the vocabulary) max / sum-exp;
//   3. per row: LSE, p, the logits at the k columns, loss, the factor sum p, and the
//      gradients at the k columns;
//   4. dzT = factor q as bf16, then the k places of each row;
//   5. dH = s dz W and dW = s dz^T h (MFMA).
#include <climits>
#include <cmath>

#include "common.h"
#include "gemm.h"
#include "logits.h"

namespace seg {
namespace {

constexpr int MAX_K = 256;

// The rows of h as bf16 (zeros from `rows` to rows_pad; a row whose index is not one of h
// is NaN), and an fp32 projection as bf16.
template <class TI>
__global__ void __launch_bounds__(256) k_distill_prep(const TI *__restrict__ h, const int32_t *__restrict__ rowmap,
                                                      int n_h, int rows, int rows_pad, int cols, bool hvec,
                                                      unsigned short *__restrict__ y, const TI *__restrict__ w, long w8,
                                                      bool wvec, unsigned short *__restrict__ wb) {
  const unsigned c8 = cols / 8;
  const long n = (long)rows_pad * c8, step = (long)gridDim.x * 256, at = (long)blockIdx.x * 256 + threadIdx.x;
  for (long i = at; i < n; i += step) {
    const int r = n >> 32 ? (int)(i / c8) : (int)((unsigned)i / c8);
    const long c = i - (long)r * c8;
    u16x8 v = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (r < rows) {
      const int from = rowmap ? rowmap[r] : r;
      if ((unsigned)from < (unsigned)n_h) v = load8(h + (long)from * cols + c * 8, hvec);
      else v = u16x8{0x7fc0, 0x7fc0, 0x7fc0, 0x7fc0, 0x7fc0, 0x7fc0, 0x7fc0, 0x7fc0};
    }
    *reinterpret_cast<u16x8 *>(y + i * 8) = v;
  }
  if constexpr (sizeof(TI) == 4) {
    for (long i = at; i < w8; i += step) *reinterpret_cast<u16x8 *>(wb + i * 8) = load8(w + i * 8, wvec);
  }
}

// The logits of few rows (16 NB at most), where the projection's bytes are the work and a
// tile of the shared product would be mostly empty: a block takes 32 rows of the
// vocabulary, its waves every WAVES-th step of 64 of the hidden width, and their sums are
// added up in LDS, in order (as the gated block's kernel for some tens of rows: 16 bytes a
// lane in whole 128-byte lines, turned in the wave's own LDS).  It writes what EpiLogits
// writes, with slabs of 32.  Measured with events around the launch, us, x 1,032 x 1,472: 25
// rows 7.5, 100 rows by the shared product 27.6; x 2,048 x 32,000: 16 / 32 / 64 rows 26.0 /
// 28.5 / 38.0, 65 rows 44.2; x 3,584 x 151,936: 24 / 64 rows 273 / 323, 65 rows 334.
constexpr int FEW = 64, FEW_SLAB = 32;

template <int NB, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, NB < 4 ? 4 : 2) k_logits_few(const unsigned short *__restrict__ w,
                                                                         const unsigned short *__restrict__ hb, int V,
                                                                         int R, int Rp, int H, float scale,
                                                                         float *__restrict__ zt,
                                                                         float2 *__restrict__ stats) {
  constexpr int ROWS = 16 * (NB > 2 ? NB : 2), STAGE = WAVES * ROWS * 8, SUMS = WAVES * 2 * NB * 64;
  __shared__ __attribute__((aligned(1024))) f32x4 lds[STAGE > SUMS ? STAGE : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, lg = lane >> 4, lr = lane >> 3, lc = lane & 7;
  const int v0 = blockIdx.x * FEW_SLAB;
  const unsigned short *wp = w + (long)v0 * H;
  unsigned woff[4], xoff[2 * NB];
  bool xin[2 * NB];
#pragma unroll
  for (int i = 0; i < 4; ++i) woff[i] = (unsigned)min(8 * i + lr, V - 1 - v0) * (unsigned)H + 8 * lc;
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i) {
    xin[i] = 8 * i + lr < R;
    xoff[i] = (unsigned)(8 * i + lr) * (unsigned)H + 8 * lc;
  }
  bf16x8 wv[4], xv[2 * NB];
  auto load = [&](int k) __attribute__((always_inline)) {
    const bool in = k + 8 * lc < H;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      wv[i] = in ? *reinterpret_cast<const bf16x8 *>(wp + k + woff[i]) : bf16x8{};
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i)
      xv[i] = in && xin[i] ? *reinterpret_cast<const bf16x8 *>(hb + k + xoff[i]) : bf16x8{};
  };
  f32x4 acc[2][NB];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int n = 0; n < NB; ++n) acc[b][n] = f32x4{};
  bf16x8 *stage = reinterpret_cast<bf16x8 *>(lds) + wave * (ROWS * 8);
  bf16x8 *to = stage + lr * 8 + (lc ^ lr);
  const bf16x8 *from = stage + r * 8;
  int k = wave * 64;
  load(k);
  for (; k < H; k += 64 * WAVES) {
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) to[64 * i] = xv[i];
    __builtin_amdgcn_wave_barrier();
    bf16x8 cx[2][NB];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < NB; ++n) cx[h][n] = from[n * 128 + ((4 * h + lg) ^ (r & 7))];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 4; ++i) to[64 * i] = wv[i];
    __builtin_amdgcn_wave_barrier();
    load(k + 64 * WAVES);
    // rows of the vocabulary of block b against rows of h of block n: a lane holds row 16 n +
    // lane % 16, vocabulary rows 16 b + 4 (lane / 16) .. + 3
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const bf16x8 cw = from[b * 128 + ((4 * h + lg) ^ (r & 7))];
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[b][n] = mfma16(cw, cx[h][n], acc[b][n]);
      }
    __builtin_amdgcn_wave_barrier();
  }
  f32x4(*sums)[2 * NB][64] = reinterpret_cast<f32x4(*)[2 * NB][64]>(lds);
  __syncthreads();
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int n = 0; n < NB; ++n) sums[wave][b * NB + n][lane] = acc[b][n];
  __syncthreads();
  if (wave >= NB) return;
  f32x4 z[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) z[b] = sums[0][b * NB + wave][lane];
#pragma unroll 1
  for (int q = 1; q < WAVES; ++q)
#pragma unroll
    for (int b = 0; b < 2; ++b) z[b] += sums[q][b * NB + wave][lane];
  const int m = 16 * wave + r;
  float mx = -INFINITY;
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int v = v0 + 16 * b + 4 * lg + q;
      z[b][q] *= scale;
      if (v >= V) continue;
      if (m < Rp) zt[(long)v * Rp + m] = z[b][q];
      mx = fmaxf(mx, z[b][q]);
    }
  mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
  mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
  const float mx2 = mx * LOG2E;
  float sm = 0.f;
  if (mx != -INFINITY) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (v0 + 16 * b + 4 * lg + q < V) sm += __builtin_amdgcn_exp2f(fmaf(z[b][q], LOG2E, -mx2));
  } else {  // -inf and NaN alone
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (v0 + 16 * b + 4 * lg + q < V && z[b][q] != z[b][q]) sm = z[b][q];
  }
  sm += __shfl_xor(sm, 16, 64);
  sm += __shfl_xor(sm, 32, 64);
  if (lg == 0 && m < R) stats[(long)blockIdx.x * R + m] = part_of(mx2, sm);
}

struct RowArgs {
  const float2 *stats;  // [slabs][rows]
  const float *zt;      // [vocab][Rp]
  int slabs, rows, Rp, vocab, k, hidden, grad;
  const int32_t *ids;
  const float *logits, *t_lse, *weight;
  float teacher_scale, loss_scale;
  float *loss_tok, *lse, *factor;
  unsigned short *place;  // [rows][k] the gradients at the k columns
  unsigned short *hb;
};

template <class F>
__device__ __forceinline__ float over_wave(float v, F &&f) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v = f(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ float sum_wave(float v) {
  return over_wave(v, [](float a, float b) { return a + b; });
}

// ROWS rows a block: their LSE from the slabs as in the action-token loss, then a wave a
// row, up to four of its columns a lane.  16 rows read the slabs in whole lines; with few
// rows 4 to a block leave no wave a second row (37 rows x 1,001: 10.6 us with 16, 4.4 with
// 4; 1,024 x 32,000 20.8 / 9.6).
//   A row without weight, or whose teacher gives no probability to any column, has loss 0
// and no gradient whatever its h holds: its dz is zero, and so is its row of hb from here
// on, as 0 x NaN would reach dW.
//   The same column more than once: each of its places gets the sum over all of them, in
// order, so it does not matter which is written last.
template <int ROWS>
__global__ void __launch_bounds__(256) k_distill_rows(const RowArgs a) {
  constexpr int SL = 256 / ROWS, E = MAX_K / 64;
  __shared__ float2 red[SL][ROWS];
  __shared__ float lse_of[ROWS];
  __shared__ int col_of[4][MAX_K];
  __shared__ float p_of[4][MAX_K];
  {
    const int t = threadIdx.x % ROWS, part = threadIdx.x / ROWS, r = blockIdx.x * ROWS + t;
    float2 s = make_float2(-INFINITY, 0.f);
    if (r < a.rows) {
#pragma unroll 4
      for (int i = part; i < a.slabs; i += SL) s = meet(s, a.stats[(long)i * a.rows + r]);
    }
    if (ROWS == 4) {  // 16 threads of a row are lanes of a wave: their order first
#pragma unroll
      for (int o = 4; o < 64; o *= 2) s = meet(s, make_float2(__shfl_xor(s.x, o, 64), __shfl_xor(s.y, o, 64)));
    }
    red[part][t] = s;
    __syncthreads();
    if (part == 0) {
      for (int k = ROWS == 4 ? 16 : 1; k < SL; k += ROWS == 4 ? 16 : 1) s = meet(s, red[k][t]);
      // (no part with a sum: every logit of the row is -inf, and so is this)
      lse_of[t] = (s.x + log2f(s.y)) * LN2;
    }
    __syncthreads();
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int t = wave; t < ROWS; t += 4) {
    const int r = blockIdx.x * ROWS + t;
    if (r >= a.rows) return;
    const float lse = lse_of[t], weight = a.weight ? a.weight[r] : 1.f;
    int col[E];
    float tj[E], zj[E], p[E], top = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = lane + 64 * e;
      col[e] = j < a.k ? a.ids[(long)r * a.k + j] : -1;
      tj[e] = col[e] >= 0 ? a.logits[(long)r * a.k + j] * a.teacher_scale : -INFINITY;
      zj[e] = col[e] >= 0 && col[e] < a.vocab ? a.zt[(long)col[e] * a.Rp + r] : 0.f;
      top = fmaxf(top, tj[e]);
    }
    float norm;
    if (a.t_lse) {
      norm = a.t_lse[r];
    } else {
      top = over_wave(top, [](float x, float y) { return fmaxf(x, y); });
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s += tj[e] == -INFINITY ? 0.f : expf(tj[e] - top);
      norm = top + logf(sum_wave(s));
    }
    float loss = 0.f, total = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      p[e] = tj[e] == -INFINITY ? 0.f : expf(tj[e] - norm);
      if (col[e] >= a.vocab) p[e] = __builtin_nanf("");  // a column outside the vocabulary
      total += p[e];
      loss += p[e] == 0.f ? 0.f : p[e] * (tj[e] - norm - zj[e] + lse);
    }
    loss = sum_wave(loss);
    total = sum_wave(total);
    const bool none = weight == 0.f || total == 0.f;
    const float g = a.loss_scale * weight, factor = none ? 0.f : g * total;
    if (lane == 0) {
      a.loss_tok[r] = none ? 0.f : weight * loss;
      a.lse[r] = lse;
    }
    if (!a.grad) continue;
    if (lane == 0) a.factor[r] = factor;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = lane + 64 * e;
      if (j < a.k) {
        col_of[wave][j] = col[e];
        p_of[wave][j] = p[e];
      }
    }
    __builtin_amdgcn_wave_barrier();
    float d[E] = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < a.k; ++j) {
      const int c = col_of[wave][j];
      const float pj = p_of[wave][j];
#pragma unroll
      for (int e = 0; e < E; ++e) d[e] += c == col[e] ? pj : 0.f;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = lane + 64 * e;
      if (j < a.k) a.place[(long)r * a.k + j] = none ? 0 : f2bf_bits(factor * expf(zj[e] - lse) - g * d[e]);
    }
    if (none)
      for (int c = lane * 8; c < a.hidden; c += 512)
        *reinterpret_cast<u16x8 *>(a.hb + (long)r * a.hidden + c) = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
  }
}

// The k places of each row of dzT (2 bytes each, in lines of their own).
__global__ void __launch_bounds__(256) k_distill_places(const int32_t *__restrict__ ids,
                                                        const unsigned short *__restrict__ place, int rows, int k,
                                                        int vocab, int Rp, unsigned short *__restrict__ dzt) {
  const long n = (long)rows * k;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
    const int c = ids[i];
    if (c >= 0 && c < vocab) dzt[(long)c * Rp + i / k] = place[i];
  }
}

// dw of no rows, of 2-byte elements at any alignment of theirs.
__global__ void __launch_bounds__(256) k_zero16(unsigned short *__restrict__ d, long n) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) d[i] = 0;
}

struct DistillWs {
  size_t hb, wb, zt, stats, factor, place, dzt, total;
  long zt_elems;
  int Rp, slabs;
};

DistillWs distill_ws(int rows, int hidden, int vocab, int k, seg_dtype dt, bool grad) {
  DistillWs w{};
  w.Rp = (rows + 31) / 32 * 32;
  const int slab = rows <= FEW ? FEW_SLAB : 128;
  w.slabs = (vocab + slab - 1) / slab;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align_up(off + std::max<size_t>(bytes, 1));
    return o;
  };
  const size_t Rp = w.Rp, H = hidden;
  w.hb = take(Rp * H * 2);
  w.wb = dt == SEG_F32 ? take((size_t)vocab * H * 2) : 0;
  // (zT later holds dH's partial sums: room for 16 parts of a small one)
  w.zt_elems = std::max((long)(vocab * Rp), grad ? std::min(16 * (long)(rows * H), 4L << 20) : 0L);
  w.zt = take((size_t)w.zt_elems * 4);
  w.stats = take((size_t)w.slabs * rows * sizeof(float2));
  if (grad) {
    w.factor = take(Rp * 4);
    w.place = take((size_t)rows * k * 2);
    w.dzt = take((size_t)vocab * Rp * 2);
  }
  w.total = off;
  return w;
}

struct Distill {
  int rows, hidden, vocab, k, n_h;
  const void *h, *w;
  const int32_t *row_index;
  const int32_t *ids;
  const float *logits, *t_lse, *weight;
  seg_distill_cfg cfg;
  float *loss_tok, *lse, *loss_sum;
  void *dh, *dw;
  seg_dtype dw_dt;
};

template <class TI, class TO>
void distill_impl(const Distill &a, char *base, const DistillWs &L, hipStream_t st) {
  const int Rp = L.Rp, R = a.rows, H = a.hidden, V = a.vocab;
  unsigned short *hb = reinterpret_cast<unsigned short *>(base + L.hb);
  float *zt = reinterpret_cast<float *>(base + L.zt);
  float2 *stats = reinterpret_cast<float2 *>(base + L.stats);
  float *factor = reinterpret_cast<float *>(base + L.factor);
  unsigned short *place = reinterpret_cast<unsigned short *>(base + L.place);
  unsigned short *dzt = reinterpret_cast<unsigned short *>(base + L.dzt);
  const bool grad = a.cfg.want_grad != 0;
  const unsigned short *wb;
  {
    unsigned short *w2 = sizeof(TI) == 4 ? reinterpret_cast<unsigned short *>(base + L.wb) : nullptr;
    const long n8 = (long)Rp * (H / 8), w8 = sizeof(TI) == 4 ? (long)V * (H / 8) : 0;
    auto vec = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    ProfScope prof("lp_prep", st);
    k_distill_prep<TI><<<(int)std::min<long>(16384, (std::max(n8, w8) + 255) / 256), 256, 0, st>>>(
        static_cast<const TI *>(a.h), a.row_index, a.n_h, R, Rp, H, vec(a.h), hb, static_cast<const TI *>(a.w), w8,
        vec(a.w), w2);
    SEG_LAUNCH_CHECK();
    wb = w2 ? w2 : static_cast<const unsigned short *>(a.w);
  }
  {
    ProfScope prof("logits", st);
    const float scale = a.cfg.logit_scale;
    if (R <= 16) {
      k_logits_few<1, 8><<<L.slabs, 512, 0, st>>>(wb, hb, V, R, Rp, H, scale, zt, stats);
      SEG_LAUNCH_CHECK();
    } else if (R <= 32) {
      k_logits_few<2, 8><<<L.slabs, 512, 0, st>>>(wb, hb, V, R, Rp, H, scale, zt, stats);
      SEG_LAUNCH_CHECK();
    } else if (R <= FEW) {
      k_logits_few<4, 8><<<L.slabs, 512, 0, st>>>(wb, hb, V, R, Rp, H, scale, zt, stats);
      SEG_LAUNCH_CHECK();
    } else {
      EpiLogits<false> e{zt, Rp, stats, R, nullptr, nullptr, scale, (long)V * Rp * 4 > (256L << 20)};
      gemm::Problems<EpiLogits<false>, 1, 1> g{{{wb}}, {{hb}}, {{H}}, {{H}}, {H}, {V}, {R}, {e}, {}, 1,
                                               (H + gemm::BK - 1) / gemm::BK};
      gemm::launch_tm<false, false, 4>(g, st);
    }
  }
  {
    ProfScope prof("distill", st);
    const RowArgs r{stats, zt, L.slabs, R, Rp, V, a.k, H, grad, a.ids, a.logits, a.t_lse, a.weight, a.cfg.teacher_scale,
                    a.cfg.loss_scale, a.loss_tok, a.lse, factor, place, hb};
    if (R >= 4096) k_distill_rows<16><<<(R + 15) / 16, 256, 0, st>>>(r);
    else k_distill_rows<4><<<(R + 3) / 4, 256, 0, st>>>(r);
    SEG_LAUNCH_CHECK();
    if (!grad) {
      k_loss_sum<<<1, 256, 0, st>>>(a.loss_tok, R, a.cfg.loss_scale, a.loss_sum);
      SEG_LAUNCH_CHECK();
      return;
    }
  }
  {
    ProfScope prof("dz", st);
    const int vr = dz_rows(V, Rp);
    k_dz<false><<<dim3((Rp + DZ_COLS - 1) / DZ_COLS, (V + vr - 1) / vr + 1), 256, 0, st>>>(
        zt, V, R, Rp, vr, a.lse, factor, nullptr, dzt, a.loss_tok, a.cfg.loss_scale, a.loss_sum);
    SEG_LAUNCH_CHECK();
  }
  {
    ProfScope prof("distill", st);
    k_distill_places<<<(unsigned)std::min<long>(8192, ((long)R * a.k + 255) / 256), 256, 0, st>>>(a.ids, place, R, a.k, V,
                                                                                                 Rp, dzt);
    SEG_LAUNCH_CHECK();
  }
  {
    ProfScope prof("dh", st);
    // zT has served: its place holds partial sums when the vocabulary is cut
    gemm::launch_one<true, true>(dzt, Rp, wb, H, R, H, V,
                                 EpiOut<TO, ST>::make(static_cast<TO *>(a.dh), H, a.cfg.logit_scale),
                                 gemm::Scratch{zt, L.zt_elems}, 0, st);
  }
  {
    ProfScope prof("dw", st);
    if (a.dw_dt == SEG_F32)
      gemm::launch_one<false, true>(dzt, Rp, hb, H, V, H, Rp,
                                    EpiOut<float, ST>::make(static_cast<float *>(a.dw), H, a.cfg.logit_scale), st);
    else
      gemm::launch_one<false, true>(
          dzt, Rp, hb, H, V, H, Rp,
          EpiOut<unsigned short, ST>::make(static_cast<unsigned short *>(a.dw), H, a.cfg.logit_scale), st);
  }
}

bool sizes_ok(int rows, int hidden, int vocab, int k) {
  return rows >= 0 && hidden >= 1 && vocab >= 1 && k >= 1 && hidden <= (1 << 20) && vocab <= (1 << 20) - 256 &&
         rows <= (1 << 20) - 256 && k <= MAX_K;
}

}  // namespace
}  // namespace seg

using namespace seg;

extern "C" size_t seg_distill_workspace_bytes(int32_t rows, int32_t hidden, int32_t vocab, int32_t k, seg_dtype dt,
                                              int32_t want_grad) {
  if (!sizes_ok(rows, hidden, vocab, k)) return 0;
  return distill_ws(rows, hidden, vocab, k, dt, want_grad != 0).total;
}

extern "C" seg_status seg_distill_loss(int32_t rows, int32_t hidden, int32_t vocab, int32_t k, seg_dtype dt, int32_t n_h,
                                       const void *h, const int32_t *row_index, const void *w, const int32_t *ids,
                                       const float *logits, const float *t_lse, const float *row_weight,
                                       const seg_distill_cfg *cfg, float *loss_tok, float *lse, float *loss_sum,
                                       void *dh, seg_dtype dw_dt, void *dw, void *ws, size_t ws_bytes,
                                       hipStream_t stream) {
  return guarded([&] {
    SEG_CHECK(cfg != nullptr, SEG_ERR_ARG, "cfg is NULL");
    SEG_CHECK(dt == SEG_BF16 || dt == SEG_F32, SEG_ERR_ARG, "unknown dtype %d", (int)dt);
    SEG_CHECK(rows >= 0 && hidden >= 1 && vocab >= 1 && n_h >= 0, SEG_ERR_ARG, "bad sizes rows=%d hidden=%d vocab=%d n_h=%d",
              rows, hidden, vocab, n_h);
    SEG_CHECK(k >= 1 && k <= vocab, SEG_ERR_ARG, "k = %d of %d columns", k, vocab);
    SEG_CHECK(k <= MAX_K, SEG_ERR_UNSUPPORTED, "k = %d above %d", k, MAX_K);
    SEG_CHECK(hidden % 8 == 0, SEG_ERR_UNSUPPORTED, "hidden %d must be a multiple of 8", hidden);
    SEG_CHECK(sizes_ok(rows, hidden, vocab, k), SEG_ERR_CAPACITY, "rows %d, hidden %d or vocab %d above 2^20", rows, hidden,
              vocab);
    SEG_CHECK(std::isfinite(cfg->logit_scale) && std::isfinite(cfg->teacher_scale) && std::isfinite(cfg->loss_scale),
              SEG_ERR_ARG, "non-finite setting");
    const bool grad = cfg->want_grad != 0;
    SEG_CHECK(!grad || dw_dt == SEG_BF16 || dw_dt == SEG_F32, SEG_ERR_ARG, "unknown dtype %d of dw", (int)dw_dt);
    SEG_CHECK(row_index || rows <= n_h, SEG_ERR_ARG, "%d rows of %d", rows, n_h);
    const DistillWs L = distill_ws(rows, hidden, vocab, k, dt, grad);
    SEG_CHECK(ws_bytes >= L.total, SEG_ERR_WORKSPACE, "workspace of %zu bytes < required %zu", ws_bytes, L.total);
    SEG_CHECK(loss_sum != nullptr, SEG_ERR_ARG, "loss_sum is NULL");
    const size_t e = dt == SEG_BF16 ? 2 : 4, ew = dw_dt == SEG_BF16 ? 2 : 4, H = hidden, R = rows;
    if (rows == 0) {
      SEG_CHECK(!grad || dw, SEG_ERR_ARG, "dw is NULL with want_grad");
      SEG_CHECK(!grad || reinterpret_cast<uintptr_t>(dw) % ew == 0, SEG_ERR_ARG, "dw is not aligned to its type");
      fill32(loss_sum, 1, 0u, stream);
      if (!grad) return;
      if (reinterpret_cast<uintptr_t>(dw) % 4 == 0) {
        fill32(dw, (long)(vocab * H * ew / 4), 0u, stream);
      } else {
        const long n = (long)(vocab * H);
        k_zero16<<<(unsigned)std::min<long>(16384, (n + 255) / 256), 256, 0, stream>>>(static_cast<unsigned short *>(dw), n);
        SEG_LAUNCH_CHECK();
      }
      return;
    }
    SEG_CHECK(h && w && ids && logits && loss_tok && lse && ws, SEG_ERR_ARG, "a tensor pointer is NULL");
    SEG_CHECK(!grad || (dh && dw), SEG_ERR_ARG, "dh or dw is NULL with want_grad");
    SEG_CHECK(reinterpret_cast<uintptr_t>(h) % e == 0 &&
                  (!grad || (reinterpret_cast<uintptr_t>(dh) % e == 0 && reinterpret_cast<uintptr_t>(dw) % ew == 0)),
              SEG_ERR_ARG, "h, dh or dw is not aligned to its type");
    SEG_CHECK(reinterpret_cast<uintptr_t>(w) % (dt == SEG_BF16 ? 16 : 4) == 0 && reinterpret_cast<uintptr_t>(ws) % 16 == 0,
              SEG_ERR_UNSUPPORTED, "w or the workspace is not on a 16-byte boundary");
    const Span outs[] = {{loss_tok, R * 4}, {lse, R * 4}, {loss_sum, 4}, {ws, L.total}, {grad ? dh : nullptr, R * H * e},
                         {grad ? dw : nullptr, vocab * H * ew}};
    const Span ins[] = {{h, n_h * H * e}, {row_index, R * 4}, {w, vocab * H * e}, {ids, R * k * 4}, {logits, R * k * 4},
                        {t_lse, R * 4}, {row_weight, R * 4}};
    check_apart(outs, 6, ins, 7);
    const Distill a{rows, hidden, vocab, k, n_h, h, w, row_index, ids, logits, t_lse, row_weight, *cfg, loss_tok, lse,
                    loss_sum, dh, dw, dw_dt};
    if (dt == SEG_F32) distill_impl<float, float>(a, static_cast<char *>(ws), L, stream);
    else distill_impl<unsigned short, unsigned short>(a, static_cast<char *>(ws), L, stream);
  });
}
