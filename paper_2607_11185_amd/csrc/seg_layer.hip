// One decoder layer of the language model around the segmented attention
// (the policy-update model of Sec. 3.3 training items; the vision encoder is
// fixed during RL, App. E, so screenshot tokens enter as hidden states):
// pre-norm RMSNorm, q/k/v projections, rotary position embedding with the
// token's row inside its segment as position, the segmented attention of
// seg_attn.hip, output projection, RMSNorm and a SwiGLU MLP, with residual
// connections; forward and backward on gfx950.  Projections and the MLP run
// over row chunks with the shared GEMM (gemm.h), which reads weights and
// activations in place in either orientation: a data gradient contracts over
// the weight's rows, a weight gradient over the chunk's rows.
// Weight gradients are summed chunk after chunk and the norm-weight gradients
// through fixed-order partial sums, so results are bitwise reproducible.
#include <algorithm>
#include <cmath>
#include <vector>

#include "act8.h"
#include "common.h"
#include "gemm.h"
#include "glu.h"
#include "mrope.h"

extern "C" seg_status seg_attn_fwd(const seg_layout *, const seg_sizes *, seg_dtype, int32_t,
                                   int32_t, int32_t, float, const void *, const void *,
                                   const void *, void *, float *, void *, size_t, hipStream_t);
extern "C" seg_status seg_attn_bwd(const seg_layout *, const seg_sizes *, seg_dtype, int32_t,
                                   int32_t, int32_t, float, const void *, const void *,
                                   const void *, const void *, const float *, const void *, void *,
                                   void *, void *, void *, size_t, hipStream_t);
extern "C" size_t seg_attn_workspace_bytes(const seg_sizes *, seg_dtype, int32_t, int32_t, int32_t,
                                           int32_t);

namespace seg {
namespace {

using gemm::ACC;
using gemm::EpiOut;
using gemm::RESID;
using gemm::ST;
typedef EpiOut<unsigned short, ST> OutBf;
typedef EpiOut<unsigned short, RESID> OutResid;
typedef EpiOut<float, ST> OutF32;
typedef EpiOut<float, ACC> OutGrad;

constexpr int MAX_CH = 16;   // hidden <= 8 * 64 * MAX_CH
constexpr int RMS_ROWS = 32; // rows per block of the norm backward
constexpr int DEFAULT_CHUNK = 65536;     // rows per chunk when chunk_rows = 0
constexpr int MAX_CHUNK = 1 << 20;       // GEMM rows are addressed with 32-bit offsets

// ------------------------------------------------------------------ kernels

// pos[r] = row inside its segment, -1 for padding rows (segments sorted by start)
__global__ void k_positions(const int32_t *__restrict__ seg_info, int S, long P,
                            int32_t *__restrict__ pos) {
  for (long r = (long)blockIdx.x * blockDim.x + threadIdx.x; r < P; r += (long)gridDim.x * blockDim.x) {
    int lo = 0, hi = S - 1, s = -1;
    while (lo <= hi) {
      const int mid = (lo + hi) >> 1;
      if (seg_info[(long)mid * SEG_INFO_FIELDS + SEG_INFO_START] <= r) {
        s = mid;
        lo = mid + 1;
      } else {
        hi = mid - 1;
      }
    }
    int p = -1;
    if (s >= 0) {
      const long st = seg_info[(long)s * SEG_INFO_FIELDS + SEG_INFO_START];
      const long ln = seg_info[(long)s * SEG_INFO_FIELDS + SEG_INFO_LEN];
      if (r < st + ln) p = (int)(r - st);
    }
    pos[r] = p;
  }
}

// y = x / sqrt(mean(x^2) + eps) * g; one wave per row, fp32 arithmetic.
// Padding rows (pos < 0) give y = 0 and rstd = 0 whatever x holds there.
__global__ void __launch_bounds__(256) k_rms_fwd(const unsigned short *__restrict__ x, long ldx,
                                                 const unsigned short *__restrict__ g, float eps,
                                                 int rows, int H, const int32_t *__restrict__ pos,
                                                 unsigned short *__restrict__ y, long ldy,
                                                 float *__restrict__ rstd) {
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= rows) return;
  const int nch = H / 8;
  if (pos[row] < 0) {
    if (lane == 0 && rstd) rstd[row] = 0.f;
    for (int c = lane; c < nch; c += 64)
      *reinterpret_cast<u16x8 *>(y + (long)row * ldy + c * 8) = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
    return;
  }
  const unsigned short *xr = x + (long)row * ldx;
  float ss = 0.f;
  for (int c = lane; c < nch; c += 64) {
    const u16x8 v = *reinterpret_cast<const u16x8 *>(xr + c * 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float f = bf_bits2f(v[j]);
      ss = fmaf(f, f, ss);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
  const float r = 1.f / sqrtf(ss / (float)H + eps);
  if (lane == 0 && rstd) rstd[row] = r;
  unsigned short *yr = y + (long)row * ldy;
  for (int c = lane; c < nch; c += 64) {
    const u16x8 v = *reinterpret_cast<const u16x8 *>(xr + c * 8);
    const u16x8 gv = *reinterpret_cast<const u16x8 *>(g + c * 8);
    u16x8 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = f2bf_bits(bf_bits2f(v[j]) * r * bf_bits2f(gv[j]));
    *reinterpret_cast<u16x8 *>(yr + c * 8) = o;
  }
}

// Backward of y = x * r * g, r = (mean(x^2) + eps)^(-1/2), for dy (fp32):
//   out = resid + r g dy - r^3 x sum(g dy x) / H      (bf16; resid may alias out)
// and per-wave partial sums of dy x r for dg: part[(block*4 + wave)][H].
// Padding rows (pos < 0) pass resid through and add nothing to dg.
__global__ void __launch_bounds__(256) k_rms_bwd(const unsigned short *__restrict__ x, long ldx,
                                                 const unsigned short *__restrict__ g,
                                                 const float *__restrict__ rstd,
                                                 const float *__restrict__ dy, long lddy, int rows,
                                                 int H, const int32_t *__restrict__ pos,
                                                 const unsigned short *resid, long ldr,
                                                 unsigned short *out, long ldo,
                                                 float *__restrict__ part) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int nch = H / 8;
  float dg[MAX_CH][8];
#pragma unroll
  for (int t = 0; t < MAX_CH; ++t)
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[t][j] = 0.f;
  const int r_end = min(rows, (blockIdx.x + 1) * RMS_ROWS);
  for (int row = blockIdx.x * RMS_ROWS + wave; row < r_end; row += 4) {
    if (pos[row] < 0) {
      for (int c = lane; c < nch; c += 64)
        *reinterpret_cast<u16x8 *>(out + (long)row * ldo + c * 8) =
            *reinterpret_cast<const u16x8 *>(resid + (long)row * ldr + c * 8);
      continue;
    }
    const unsigned short *xr = x + (long)row * ldx;
    const float *dr = dy + (long)row * lddy;
    const float r = rstd[row];
    float s = 0.f;
#pragma unroll
    for (int t = 0; t < MAX_CH; ++t) {
      const int c = lane + 64 * t;
      if (c < nch) {
        const u16x8 xv = *reinterpret_cast<const u16x8 *>(xr + c * 8);
        const u16x8 gv = *reinterpret_cast<const u16x8 *>(g + c * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float xf = bf_bits2f(xv[j]), d = dr[c * 8 + j];
          s = fmaf(bf_bits2f(gv[j]) * d, xf, s);
          dg[t][j] = fmaf(d * xf, r, dg[t][j]);
        }
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    const float k3 = r * r * r * s / (float)H;
    for (int c = lane; c < nch; c += 64) {
      const u16x8 xv = *reinterpret_cast<const u16x8 *>(xr + c * 8);
      const u16x8 gv = *reinterpret_cast<const u16x8 *>(g + c * 8);
      const u16x8 rv = *reinterpret_cast<const u16x8 *>(resid + (long)row * ldr + c * 8);
      u16x8 o;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = dr[c * 8 + j];
        const float dx = r * bf_bits2f(gv[j]) * d - k3 * bf_bits2f(xv[j]);
        o[j] = f2bf_bits(bf_bits2f(rv[j]) + dx);
      }
      *reinterpret_cast<u16x8 *>(out + (long)row * ldo + c * 8) = o;
    }
  }
  float *pr = part + ((long)blockIdx.x * 4 + wave) * H;
#pragma unroll
  for (int t = 0; t < MAX_CH; ++t) {
    const int c = lane + 64 * t;
    if (c < nch) {
#pragma unroll
      for (int j = 0; j < 8; ++j) pr[c * 8 + j] = dg[t][j];
    }
  }
}

// Column sums of part[nparts][H] in a fixed order, in two passes: block
// (x, y) sums parts [y*per, (y+1)*per) of 256 columns into part2[y][H], then
// out[h] += sum over y (in order) of part2[y][h].
constexpr int COLSUM_SPLIT = 16;

__global__ void __launch_bounds__(256) k_colsum_part(const float *__restrict__ part, int nparts,
                                                     int H, float *__restrict__ part2) {
  const int h = blockIdx.x * 256 + threadIdx.x;
  if (h >= H) return;
  const int per = (nparts + COLSUM_SPLIT - 1) / COLSUM_SPLIT;
  const int p0 = blockIdx.y * per, p1 = min(nparts, p0 + per);
  float s = 0.f;
#pragma unroll 8
  for (int p = p0; p < p1; ++p) s += part[(long)p * H + h];
  part2[(long)blockIdx.y * H + h] = s;
}

__global__ void k_colsum_add(const float *__restrict__ part2, int H, float *__restrict__ out) {
  const int h = blockIdx.x * blockDim.x + threadIdx.x;
  if (h >= H) return;
  float s = 0.f;
#pragma unroll
  for (int y = 0; y < COLSUM_SPLIT; ++y) s += part2[(long)y * H + h];
  out[h] += s;
}

// cos and sin of pos * base^(-2i/d) for every position of the longest segment
// and pair i < half.  The angle is formed and reduced modulo 2 pi in fp64.
__global__ void __launch_bounds__(256) k_rope_table(int n, int half, double log2_base,
                                                    float2 *__restrict__ tab) {
  const double two_pi = 6.283185307179586;
  for (long e = (long)blockIdx.x * 256 + threadIdx.x; e < (long)n * half; e += (long)gridDim.x * 256) {
    const int p = (int)(e / half), i = (int)(e - (long)p * half);
    double a = (double)p * exp2(-2.0 * i / (2 * half) * log2_base);
    a -= two_pi * floor(a / two_pi);
    float s, c;
    sincosf((float)a, &s, &c);
    tab[e] = make_float2(c, s);
  }
}

// Rotary embedding in place on a [P, ha, d] and b [P, hb, d]: the pair (x_i,
// x_{i+d/2}) turns by pos * base^(-2i/d) (by minus that angle with inverse, the
// transpose used by the backward).  Padding rows are left unchanged; with
// inverse they are zeroed, those of c [P, hc, d] too.  Bound by HBM: a thread
// turns eight pairs with 16-byte accesses and angles from the table, which all
// heads of a row share (with the angle and sincos per pair, 1.0 ms for 137,895
// rows x 28 heads x 128; now 0.42 ms with its 4 key heads, 5.4 TB/s).
struct RopeArgs {
  unsigned short *a, *b, *c;
  int ha, hb, hc, d, inverse;
  long P;
  const int32_t *pos;
  const float2 *tab;
};

__global__ void __launch_bounds__(256) k_rope(const RopeArgs g) {
  const int half = g.d / 2, per = half / 8;  // chunks of 8 pairs of a head
  const int heads = g.ha + g.hb, row_chunks = heads * per, n_c = g.hc * (g.d / 8);
  const int lane_chunks = row_chunks + n_c;
  // a block takes whole rows
  for (long row = blockIdx.x; row < g.P; row += gridDim.x) {
    const int p = g.pos[row];
    const u16x8 zero = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
    for (int e = threadIdx.x; e < (p < 0 && g.inverse ? lane_chunks : row_chunks); e += 256) {
      if (e >= row_chunks) {
        *reinterpret_cast<u16x8 *>(g.c + (row * g.hc * g.d) + (long)(e - row_chunks) * 8) = zero;
        continue;
      }
      const int h = e / per, i = (e - h * per) * 8;
      unsigned short *x = h < g.ha ? g.a + (row * g.ha + h) * g.d + i
                                   : g.b + (row * g.hb + (h - g.ha)) * g.d + i;
      if (p < 0) {
        if (g.inverse) {
          *reinterpret_cast<u16x8 *>(x) = zero;
          *reinterpret_cast<u16x8 *>(x + half) = zero;
        }
        continue;
      }
      const u16x8 lo = *reinterpret_cast<const u16x8 *>(x), hi = *reinterpret_cast<const u16x8 *>(x + half);
      const f32x4 *t = reinterpret_cast<const f32x4 *>(g.tab + (long)p * half + i);
      u16x8 olo, ohi;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const f32x4 cs = t[j / 2];
        const float c = cs[(j & 1) * 2], s = g.inverse ? -cs[(j & 1) * 2 + 1] : cs[(j & 1) * 2 + 1];
        const float x1 = bf_bits2f(lo[j]), x2 = bf_bits2f(hi[j]);
        olo[j] = f2bf_bits(x1 * c - x2 * s);
        ohi[j] = f2bf_bits(x2 * c + x1 * s);
      }
      *reinterpret_cast<u16x8 *>(x) = olo;
      *reinterpret_cast<u16x8 *>(x + half) = ohi;
    }
  }
}

// zeros in the padding rows of x [P, W] (the other rows are not touched)
__global__ void __launch_bounds__(256) k_zero_pad(unsigned short *__restrict__ x,
                                                  const int32_t *__restrict__ pos, long P, int W) {
  // four rows a block and turn, one per wave
  for (long row = (long)blockIdx.x * 4 + (threadIdx.x >> 6); row < P; row += (long)gridDim.x * 4)
    if (pos[row] < 0)
      for (int c = threadIdx.x & 63; c < W / 8; c += 64)
        *reinterpret_cast<u16x8 *>(x + row * W + c * 8) = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
}

// dst[r] = pos[r] >= 0 ? src[r] : 0 for rows of W bf16 values
__global__ void k_mask_rows(const unsigned short *src, const int32_t *__restrict__ pos, long P, int W,
                            unsigned short *dst) {
  const long n8 = P * (W / 8);
  for (long c = (long)blockIdx.x * blockDim.x + threadIdx.x; c < n8; c += (long)gridDim.x * blockDim.x) {
    const long row = c / (W / 8);
    u16x8 v = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (pos[row] >= 0) v = *reinterpret_cast<const u16x8 *>(src + c * 8);
    *reinterpret_cast<u16x8 *>(dst + c * 8) = v;
  }
}

// ------------------------------------------------------------------ host side

int blocks_for(long n, int per = 256) { return (int)std::max<long>(1, std::min<long>(65536, (n + per - 1) / per)); }

struct Dims {
  long P;
  int H, I, hq, hkv, d, C, QD, KD;
};

Dims dims_of(const seg_sizes &sz, const seg_layer_cfg &c) {
  Dims m{};
  m.P = sz.packed_tokens;
  m.H = c.hidden;
  m.I = c.inter;
  m.hq = c.hq;
  m.hkv = c.hkv;
  m.d = c.d;
  m.QD = c.hq * c.d;
  m.KD = c.hkv * c.d;
  long C = c.chunk_rows > 0 ? c.chunk_rows : DEFAULT_CHUNK;
  C = std::max<long>(1, std::min<long>(C, std::max<long>(m.P, 1)));
  m.C = (int)C;
  return m;
}

struct LayerWs {
  size_t pos, tab, a, m, sums, attn;                             // forward
  size_t dy1, dO, dq, dk, dv;  // backward
  size_t g, u, dm, dg, du, dbf, part;
  size_t x, q, k, v, o, y1;  // with 8-bit saved activations: their values
  long sum_elems;
  size_t total;
};

LayerWs layer_ws(const seg_sizes &sz, const seg_layer_cfg &c, int bwd, bool packed = false) {
  const Dims m = dims_of(sz, c);
  LayerWs w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = align_up(off + std::max<size_t>(bytes, 1));
    return o;
  };
  const size_t P = std::max<long>(m.P, 1), C = m.C, H = m.H, I = m.I;
  w.pos = take(P * 4);
  w.tab = take((size_t)std::max(sz.max_seg_len, 1) * (c.d / 2) * sizeof(float2));
  w.a = take(C * H * 2);
  w.m = take(C * I * 2);
  // partial sums of products cut over K: what the largest cut product takes, up
  // to 128 MB (larger ones fill the chip uncut); the same for every chunk size
  w.sum_elems = (long)std::min<size_t>(
      (size_t)32 << 20, 16 * std::max(std::max(P, H) * std::max<size_t>(H, m.QD + 2 * m.KD), H * I));
  w.sums = take(w.sum_elems * 4);
  if (packed) {
    if (bwd) w.x = take(P * H * 2);
    w.q = take(P * m.QD * 2);
    w.k = take(P * m.KD * 2);
    w.v = take(P * m.KD * 2);
    w.o = take(P * m.QD * 2);
    w.y1 = take(P * H * 2);
  }
  w.attn = take(seg_attn_workspace_bytes(&sz, SEG_BF16, c.hq, c.hkv, c.d, bwd));
  if (bwd) {
    w.dy1 = take(P * H * 2);
    w.dO = take(P * m.QD * 2);
    w.dq = take(P * m.QD * 2);
    w.dk = take(P * m.KD * 2);
    w.dv = take(P * m.KD * 2);
    w.g = take(C * I * 2);
    w.u = take(C * I * 2);
    w.dm = take(C * I * 2);
    w.dg = take(C * I * 2);
    w.du = take(C * I * 2);
    w.dbf = take(C * H * 4);
    w.part = take((((C + RMS_ROWS - 1) / RMS_ROWS) * 4 + COLSUM_SPLIT) * H * 4);
  }
  w.total = std::max<size_t>(off, 256);
  return w;
}

void check_layer(const seg_layout *L, const seg_sizes *sz, const seg_layer_cfg *c,
                 const seg_layer_weights *w) {
  SEG_CHECK(L && sz && c && w, SEG_ERR_ARG, "layout, sizes, cfg or weights is NULL");
  SEG_CHECK(c->hidden >= 8 && c->hidden % 8 == 0 && c->inter >= 8 && c->inter % 8 == 0,
            SEG_ERR_UNSUPPORTED, "hidden %d and inter %d must be positive multiples of 8",
            c->hidden, c->inter);
  SEG_CHECK(c->hidden <= 8 * 64 * MAX_CH, SEG_ERR_UNSUPPORTED, "hidden %d > %d", c->hidden,
            8 * 64 * MAX_CH);
  SEG_CHECK(c->hq >= 1 && c->hkv >= 1 && c->hq % c->hkv == 0 && (c->d == 64 || c->d == 128),
            SEG_ERR_UNSUPPORTED, "heads %d/%d, head_dim %d not supported", c->hq, c->hkv, c->d);
  SEG_CHECK(std::isfinite(c->rms_eps) && c->rms_eps > 0.f, SEG_ERR_ARG, "rms_eps must be > 0");
  SEG_CHECK(std::isfinite(c->rope_base) && c->rope_base > 1.f, SEG_ERR_ARG,
            "rope_base must be > 1");
  SEG_CHECK(c->chunk_rows >= 0, SEG_ERR_ARG, "chunk_rows must be >= 0");
  SEG_CHECK(c->chunk_rows <= MAX_CHUNK && c->inter <= MAX_CHUNK && (long)c->hq * c->d <= MAX_CHUNK,
            SEG_ERR_UNSUPPORTED, "chunk_rows %d, inter %d or hq*d above %d", c->chunk_rows,
            c->inter, MAX_CHUNK);
  SEG_CHECK(w->g1 && w->wq && w->wk && w->wv && w->wo && w->g2 && w->wg && w->wu && w->wd,
            SEG_ERR_ARG, "a weight pointer is NULL");
  SEG_CHECK((long)std::max<long>(sz->packed_tokens, 1) * std::max(c->hidden, c->inter) < (1L << 40),
            SEG_ERR_CAPACITY, "tensor too large");
}

#define US(p) reinterpret_cast<unsigned short *>(p)
#define CUS(p) reinterpret_cast<const unsigned short *>(p)

void rms_fwd(const unsigned short *x, long ldx, const void *g, float eps, int rows, int H,
             const int32_t *pos, unsigned short *y, float *rstd, hipStream_t st) {
  k_rms_fwd<<<(rows + 3) / 4, 256, 0, st>>>(x, ldx, CUS(g), eps, rows, H, pos, y, H, rstd);
  SEG_LAUNCH_CHECK();
}

void rms_bwd(const unsigned short *x, const void *g, const float *rstd, const float *dy, int rows,
             int H, const int32_t *pos, const unsigned short *resid, unsigned short *out,
             float *part, float *dgrad, hipStream_t st) {
  const int nb = (rows + RMS_ROWS - 1) / RMS_ROWS;
  k_rms_bwd<<<nb, 256, 0, st>>>(x, H, CUS(g), rstd, dy, H, rows, H, pos, resid, H, out, H, part);
  SEG_LAUNCH_CHECK();
  float *part2 = part + (long)nb * 4 * H;
  k_colsum_part<<<dim3((H + 255) / 256, COLSUM_SPLIT), 256, 0, st>>>(part, nb * 4, H, part2);
  SEG_LAUNCH_CHECK();
  k_colsum_add<<<(H + 255) / 256, 256, 0, st>>>(part2, H, dgrad);
  SEG_LAUNCH_CHECK();
}

void positions(const seg_layout *L, const seg_sizes *sz, long P, int32_t *pos, hipStream_t st) {
  k_positions<<<blocks_for(P), 256, 0, st>>>(L->seg_info, sz->num_segments, P, pos);
  SEG_LAUNCH_CHECK();
}

// the angle table of a call
void rope_table(const seg_sizes &sz, const seg_layer_cfg &c, float2 *tab, hipStream_t st) {
  const int n = sz.max_seg_len, half = c.d / 2;
  k_rope_table<<<blocks_for((long)n * half), 256, 0, st>>>(n, half, std::log2((double)c.rope_base), tab);
  SEG_LAUNCH_CHECK();
}

void rope(const RopeArgs &g, hipStream_t st) {
  k_rope<<<(int)std::max<long>(1, std::min<long>(g.P, 8192)), 256, 0, st>>>(g);
  SEG_LAUNCH_CHECK();
}

void zero_grads(const seg_layer_grads &g, const seg_layer_cfg &c, hipStream_t st) {
  const long H = c.hidden, I = c.inter, QD = (long)c.hq * c.d, KD = (long)c.hkv * c.d;
  fill32(g.g1, H, 0u, st);
  fill32(g.g2, H, 0u, st);
  fill32(g.wq, QD * H, 0u, st);
  fill32(g.wk, KD * H, 0u, st);
  fill32(g.wv, KD * H, 0u, st);
  fill32(g.wo, H * QD, 0u, st);
  fill32(g.wg, I * H, 0u, st);
  fill32(g.wu, I * H, 0u, st);
  fill32(g.wd, H * I, 0u, st);
}

void check_status(seg_status s) {
  if (s != SEG_OK) throw Fail{s};
}

// What the extended entry points add to the layer.
struct Ext {
  const seg_mrope_cfg *rope;       // positions on three axes, or NULL
  const int32_t *pos;              // [3, P]
  const seg_layer_saved8 *packed;  // 8-bit saved activations, or NULL
};

void rotate(const seg_sizes &sz, const seg_layer_cfg &c, const Ext &ext, const RopeArgs &g, float2 *tab,
            hipStream_t st) {
  if (!ext.rope) {
    rope_table(sz, c, tab, st);
    rope(g, st);
    return;
  }
  mrope::Args r{};
  r.a = mrope::Heads{g.a, g.a, (long)g.ha * g.d, (long)g.ha * g.d, g.ha};
  r.b = mrope::Heads{g.b, g.b, (long)g.hb * g.d, (long)g.hb * g.d, g.hb};
  r.rows = g.P;
  r.d = g.d;
  r.inverse = g.inverse;
  r.set(*ext.rope);
  r.pos = ext.pos;
  r.pad = g.pos;
  r.zero = g.c;
  r.zero_width = g.hc * g.d;
  mrope::launch(SEG_BF16, r, st);
}

// the kept gate and up values from row r0 on (none: codes NULL)
glu::Kept kept_rows(const Ext &ext, long r0, int I) {
  glu::Kept k{};
  if (!ext.packed || !ext.packed->g.code) return k;
  const long nb = act8::blocks_of(I);
  k.g8 = seg_act8{ext.packed->g.code + r0 * I, ext.packed->g.exp + r0 * nb};
  k.u8 = seg_act8{ext.packed->u.code + r0 * I, ext.packed->u.exp + r0 * nb};
  return k;
}

void pack(long rows, int cols, const unsigned short *x, const seg_act8 &to, hipStream_t st) {
  act8::pack(rows, cols, SEG_BF16, x, cols, &to, nullptr, st);
}

void unpack(long rows, int cols, const seg_act8 &from, unsigned short *x, hipStream_t st) {
  act8::unpack(rows, cols, SEG_BF16, &from, x, cols, nullptr, st);
}

void layer_fwd_impl(const seg_layout *L, const seg_sizes *sz, const seg_layer_cfg &c,
                    const Ext &ext, const seg_layer_weights &w, const unsigned short *x,
                    unsigned short *y, const seg_layer_saved &sv, char *base, const LayerWs &W,
                    size_t ws_bytes, hipStream_t st) {
  const Dims m = dims_of(*sz, c);
  const long P = m.P;
  const int H = m.H, I = m.I;
  int32_t *pos = reinterpret_cast<int32_t *>(base + W.pos);
  float2 *tab = reinterpret_cast<float2 *>(base + W.tab);
  const gemm::Scratch sums{reinterpret_cast<float *>(base + W.sums), W.sum_elems};
  unsigned short *a = US(base + W.a), *mb = US(base + W.m);
  unsigned short *q = US(sv.q), *k = US(sv.k), *v = US(sv.v), *o = US(sv.o), *y1 = US(sv.y1);
  {
    ProfScope prof("ly_misc", st);
    positions(L, sz, P, pos, st);
  }
  if (ext.packed) {  // before y, which may be x, is written
    ProfScope prof("ly_act8", st);
    pack(P, H, x, ext.packed->x, st);
  }
  for (long r0 = 0; r0 < P; r0 += m.C) {
    const int cr = (int)std::min<long>(m.C, P - r0);
    {
      ProfScope prof("ly_norm", st);
      rms_fwd(x + r0 * H, H, w.g1, c.rms_eps, cr, H, pos + r0, a, sv.rstd1 + r0, st);
    }
    ProfScope prof("ly_proj", st);
    gemm::Problems<OutBf, 3, 1> g{
        {{a}, {a}, {a}}, {{CUS(w.wq)}, {CUS(w.wk)}, {CUS(w.wv)}}, {{H}, {H}, {H}}, {{H}, {H}, {H}}, {H},
        {cr, cr, cr}, {m.QD, m.KD, m.KD},
        {OutBf::make(q + r0 * m.QD, m.QD), OutBf::make(k + r0 * m.KD, m.KD),
         OutBf::make(v + r0 * m.KD, m.KD)}, {}, 1, 0};
    gemm::launch<false, false>(g, sums, P, st);
  }
  {
    ProfScope prof("ly_rope", st);
    rotate(*sz, c, ext, RopeArgs{q, k, nullptr, m.hq, m.hkv, 0, m.d, 0, P, pos, tab}, tab, st);
  }
  check_status(seg_attn_fwd(L, sz, SEG_BF16, m.hq, m.hkv, m.d, 1.f / std::sqrt((float)m.d), q, k, v,
                            o, sv.lse, base + W.attn, ws_bytes - W.attn, st));
  {
    ProfScope prof("ly_misc", st);
    k_zero_pad<<<(int)std::min<long>(4096, (P + 3) / 4), 256, 0, st>>>(o, pos, P, m.QD);
    SEG_LAUNCH_CHECK();
  }
  for (long r0 = 0; r0 < P; r0 += m.C) {
    const int cr = (int)std::min<long>(m.C, P - r0);
    {
      ProfScope prof("ly_proj", st);
      gemm::launch_one<false, false>(o + r0 * m.QD, m.QD, CUS(w.wo), m.QD, cr, H, m.QD,
                                     OutResid::make(y1 + r0 * H, H, 1.f, x + r0 * H, H), sums, P, st);
    }
    {
      ProfScope prof("ly_norm", st);
      rms_fwd(y1 + r0 * H, H, w.g2, c.rms_eps, cr, H, pos + r0, a, sv.rstd2 + r0, st);
    }
    ProfScope prof("ly_mlp", st);
    glu::forward(a, H, CUS(w.wg), CUS(w.wu), cr, H, I, mb, kept_rows(ext, r0, I), nullptr, st);
    gemm::launch_one<false, false>(mb, I, CUS(w.wd), I, cr, H, I,
                                   OutResid::make(y + r0 * H, H, 1.f, y1 + r0 * H, H), sums, P, st);
  }
  if (ext.packed) {
    const seg_layer_saved8 &s8 = *ext.packed;
    ProfScope prof("ly_act8", st);
    pack(P, m.QD, q, s8.q, st);
    pack(P, m.KD, k, s8.k, st);
    pack(P, m.KD, v, s8.v, st);
    pack(P, m.QD, o, s8.o, st);
    pack(P, H, y1, s8.y1, st);
  }
}

void layer_bwd_impl(const seg_layout *L, const seg_sizes *sz, const seg_layer_cfg &c,
                    const Ext &ext, const seg_layer_weights &w, const unsigned short *x,
                    const seg_layer_saved &sv, const unsigned short *dy, unsigned short *dx,
                    const seg_layer_grads &gr, char *base, const LayerWs &W, size_t ws_bytes,
                    hipStream_t st) {
  const Dims m = dims_of(*sz, c);
  const long P = m.P;
  const int H = m.H, I = m.I;
  int32_t *pos = reinterpret_cast<int32_t *>(base + W.pos);
  float2 *tab = reinterpret_cast<float2 *>(base + W.tab);
  const gemm::Scratch sums{reinterpret_cast<float *>(base + W.sums), W.sum_elems};
  unsigned short *a = US(base + W.a), *mb = US(base + W.m);
  unsigned short *dy1 = US(base + W.dy1), *dO = US(base + W.dO), *dq = US(base + W.dq),
                 *dk = US(base + W.dk), *dv = US(base + W.dv);
  unsigned short *dm = US(base + W.dm), *dgb = US(base + W.dg), *dub = US(base + W.du);
  float *dbf = reinterpret_cast<float *>(base + W.dbf);
  float *part = reinterpret_cast<float *>(base + W.part);
  const unsigned short *q = CUS(sv.q), *k = CUS(sv.k), *v = CUS(sv.v), *o = CUS(sv.o),
                       *y1 = CUS(sv.y1);
  {
    ProfScope prof("ly_misc", st);
    fill32(gr.g1, H, 0u, st);
    fill32(gr.g2, H, 0u, st);
    positions(L, sz, P, pos, st);
    // dy1 starts as dy with the padding rows zeroed
    k_mask_rows<<<blocks_for(P * (H / 8)), 256, 0, st>>>(dy, pos, P, H, dy1);
    SEG_LAUNCH_CHECK();
  }
  if (ext.packed) {
    const seg_layer_saved8 &s8 = *ext.packed;
    ProfScope prof("ly_act8", st);
    unpack(P, H, s8.x, US(base + W.x), st);
    unpack(P, m.QD, s8.q, US(base + W.q), st);
    unpack(P, m.KD, s8.k, US(base + W.k), st);
    unpack(P, m.KD, s8.v, US(base + W.v), st);
    unpack(P, m.QD, s8.o, US(base + W.o), st);
    unpack(P, H, s8.y1, US(base + W.y1), st);
  }
  // MLP and output projection, chunk by chunk
  for (long r0 = 0; r0 < P; r0 += m.C) {
    const int cr = (int)std::min<long>(m.C, P - r0);
    unsigned short *dy1c = dy1 + r0 * H;
    {
      ProfScope prof("ly_norm", st);
      rms_fwd(y1 + r0 * H, H, w.g2, c.rms_eps, cr, H, pos + r0, a, nullptr, st);  // b
    }
    {
      ProfScope prof("ly_mlp", st);
      // m, g and u: kept by the forward, or computed again
      glu::Kept kept = kept_rows(ext, r0, I);
      if (!kept.g8.code) {
        kept.g16 = US(base + W.g);
        kept.u16 = US(base + W.u);
        glu::forward(a, H, CUS(w.wg), CUS(w.wu), cr, H, I, mb, kept, nullptr, st);
      }
      gemm::launch_one<false, true>(dy1c, H, CUS(w.wd), I, cr, I, H, OutBf::make(dm, I), sums, P, st);  // dm = dy wd
      glu::backward_act(kept, dm, cr, I, dgb, dub, kept.g8.code ? mb : nullptr, st);
      // db = dg wg + du wu, one sum over both contractions
      gemm::Problems<OutF32, 1, 2> g{{{dgb, dub}}, {{CUS(w.wg), CUS(w.wu)}}, {{I, I}}, {{H, H}}, {I, I},
                                     {cr}, {H}, {OutF32::make(dbf, H)}, {}, 1, 0};
      gemm::launch<false, true>(g, sums, P, st);
    }
    {
      // dWd += dy^T m, dWg += dg^T b, dWu += du^T b in one launch
      ProfScope prof("ly_wgrad", st);
      const bool first = r0 == 0;
      gemm::Problems<OutGrad, 3, 1> g{
          {{dy1c}, {dgb}, {dub}}, {{mb}, {a}, {a}}, {{H}, {I}, {I}}, {{I}, {H}, {H}}, {cr}, {H, I, I},
          {I, H, H},
          {OutGrad::make(gr.wd, I, 1.f, nullptr, 0, first), OutGrad::make(gr.wg, H, 1.f, nullptr, 0, first),
           OutGrad::make(gr.wu, H, 1.f, nullptr, 0, first)}, {}, 1, 0};
      gemm::launch<true, true>(g, sums, 0, st);
    }
    {
      ProfScope prof("ly_norm", st);
      rms_bwd(y1 + r0 * H, w.g2, sv.rstd2 + r0, dbf, cr, H, pos + r0, dy1c, dy1c, part, gr.g2, st);
    }
    ProfScope prof("ly_proj", st);
    gemm::launch_one<true, true>(dy1c, H, o + r0 * m.QD, m.QD, H, m.QD, cr,
                                 OutGrad::make(gr.wo, m.QD, 1.f, nullptr, 0, r0 == 0), sums, 0, st);  // dWo
    gemm::launch_one<false, true>(dy1c, H, CUS(w.wo), m.QD, cr, m.QD, H,
                                  OutBf::make(dO + r0 * m.QD, m.QD), sums, P, st);
  }
  check_status(seg_attn_bwd(L, sz, SEG_BF16, m.hq, m.hkv, m.d, 1.f / std::sqrt((float)m.d), q, k, v,
                            o, sv.lse, dO, dq, dk, dv, base + W.attn, ws_bytes - W.attn, st));
  {
    ProfScope prof("ly_rope", st);
    rotate(*sz, c, ext, RopeArgs{dq, dk, dv, m.hq, m.hkv, m.hkv, m.d, 1, P, pos, tab}, tab, st);
  }
  // q/k/v projections and the first norm, chunk by chunk
  for (long r0 = 0; r0 < P; r0 += m.C) {
    const int cr = (int)std::min<long>(m.C, P - r0);
    {
      ProfScope prof("ly_norm", st);
      rms_fwd(x + r0 * H, H, w.g1, c.rms_eps, cr, H, pos + r0, a, nullptr, st);  // a
    }
    {
      ProfScope prof("ly_proj", st);
      // da = dq wq + dk wk + dv wv, one sum over the three contractions
      gemm::Problems<OutF32, 1, 3> g{{{dq + r0 * m.QD, dk + r0 * m.KD, dv + r0 * m.KD}},
                                     {{CUS(w.wq), CUS(w.wk), CUS(w.wv)}}, {{m.QD, m.KD, m.KD}},
                                     {{H, H, H}}, {m.QD, m.KD, m.KD}, {cr}, {H},
                                     {OutF32::make(dbf, H)}, {}, 1, 0};
      gemm::launch<false, true>(g, sums, P, st);
    }
    {
      // dWq += dq^T a, dWk += dk^T a, dWv += dv^T a in one launch
      ProfScope prof("ly_wgrad", st);
      const bool first = r0 == 0;
      gemm::Problems<OutGrad, 3, 1> g{
          {{dq + r0 * m.QD}, {dk + r0 * m.KD}, {dv + r0 * m.KD}}, {{a}, {a}, {a}},
          {{m.QD}, {m.KD}, {m.KD}}, {{H}, {H}, {H}}, {cr}, {m.QD, m.KD, m.KD}, {H, H, H},
          {OutGrad::make(gr.wq, H, 1.f, nullptr, 0, first), OutGrad::make(gr.wk, H, 1.f, nullptr, 0, first),
           OutGrad::make(gr.wv, H, 1.f, nullptr, 0, first)}, {}, 1, 0};
      gemm::launch<true, true>(g, sums, 0, st);
    }
    ProfScope prof("ly_norm", st);
    rms_bwd(x + r0 * H, w.g1, sv.rstd1 + r0, dbf, cr, H, pos + r0, dy1 + r0 * H, dx + r0 * H, part,
            gr.g1, st);
  }
}

}  // namespace
}  // namespace seg

using namespace seg;

// For tests (not in seg.h; host only): how a group of the layer's products is
// launched.  rows as in gemm::launch; out = {rows of a tile, parts of K}.
extern "C" void seg_layer_gemm_choice(const seg_sizes *sz, const seg_layer_cfg *cfg, int32_t bwd,
                                      int32_t np, const int32_t *M, const int32_t *N, int32_t ns,
                                      const int32_t *K, int64_t rows, int32_t *out) {
  const gemm::Choice c =
      gemm::choose_group(np, M, N, ns, K, layer_ws(*sz, *cfg, bwd).sum_elems, rows);
  out[0] = gemm::bm_of(c.tm);
  out[1] = c.parts;
}

extern "C" size_t seg_layer_workspace_bytes(const seg_sizes *sz, const seg_layer_cfg *cfg,
                                            int32_t bwd) {
  return seg_layer_ext_workspace_bytes(sz, cfg, 0, bwd);
}

extern "C" size_t seg_layer_ext_workspace_bytes(const seg_sizes *sz, const seg_layer_cfg *cfg,
                                                int32_t saved8, int32_t bwd) {
  if (!sz || !cfg || cfg->hidden < 1 || cfg->inter < 1 || cfg->hq < 1 || cfg->hkv < 1 ||
      cfg->d < 1)
    return 0;
  return layer_ws(*sz, *cfg, bwd ? 1 : 0, saved8 != 0).total;
}

namespace {

Ext check_ext(const seg_layer_ext *e, const seg_sizes &sz, const seg_layer_cfg &c) {
  Ext x{};
  if (!e) return x;
  if (e->rope) {
    mrope::check_cfg(e->rope, c.d);
    SEG_CHECK(e->pos, SEG_ERR_ARG, "rope without pos");
    mrope::check_launch(SEG_BF16, sz.packed_tokens, c.hq + c.hkv, c.d);
  }
  if (e->saved8) {
    const seg_act8 *a[] = {&e->saved8->x, &e->saved8->q, &e->saved8->k,
                           &e->saved8->v, &e->saved8->o, &e->saved8->y1};
    for (const seg_act8 *p : a) SEG_CHECK(p->code && p->exp, SEG_ERR_ARG, "an 8-bit saved array is NULL");
    const seg_act8 &g = e->saved8->g, &u = e->saved8->u;
    SEG_CHECK(!g.code == !u.code && (!g.code || (g.exp && u.exp)), SEG_ERR_ARG,
              "the gate's and the up values' 8-bit arrays: both or none");
    SEG_CHECK((reinterpret_cast<uintptr_t>(g.code) | reinterpret_cast<uintptr_t>(u.code)) % 8 == 0,
              SEG_ERR_UNSUPPORTED, "the gate's and up values' codes must start on 8-byte boundaries");
    SEG_CHECK(e->saved8->lse && e->saved8->rstd1 && e->saved8->rstd2, SEG_ERR_ARG, "a saved vector is NULL");
    act8::check_launch(sz.packed_tokens, std::max(c.hidden, c.hq * c.d), SEG_BF16);
  }
  x.rope = e->rope;
  x.pos = e->pos;
  x.packed = e->saved8;
  return x;
}

// With 8-bit saved activations: a forward's outputs (grads NULL) or a backward's, and the
// workspace, share no memory with its inputs or each other, but y may be x and dx may be dy
// (in: x or dy, out: y or dx).
void check_ext_apart(const Ext &ext, const seg_sizes &sz, const seg_layer_cfg &c, const seg_layer_weights &w,
                     const void *in, const void *out, const seg_layer_grads *grads, const void *ws, size_t ws_bytes) {
  if (!ext.packed) return;
  const size_t P = sz.packed_tokens, H = c.hidden, I = c.inter, QD = (size_t)c.hq * c.d, KD = (size_t)c.hkv * c.d;
  const seg_layer_saved8 &s = *ext.packed;
  std::vector<Span> kept, outs{{out, P * H * 2}, {ws, ws_bytes}}, ins;
  auto act = [&](const seg_act8 &a, size_t cols) {
    if (!a.code) return;
    kept.push_back({a.code, P * cols});
    kept.push_back({a.exp, P * act8::blocks_of(cols)});
  };
  act(s.x, H);
  act(s.y1, H);
  act(s.q, QD);
  act(s.o, QD);
  act(s.k, KD);
  act(s.v, KD);
  act(s.g, I);
  act(s.u, I);
  kept.push_back({s.lse, c.hq * P * 4});
  kept.push_back({s.rstd1, P * 4});
  kept.push_back({s.rstd2, P * 4});
  std::vector<Span> &to = grads ? ins : outs;
  to.insert(to.end(), kept.begin(), kept.end());
  if (in != out) ins.push_back({in, P * H * 2});
  if (ext.rope) ins.push_back({ext.pos, 3 * P * 4});
  const void *wp[9] = {w.g1, w.wq, w.wk, w.wv, w.wo, w.g2, w.wg, w.wu, w.wd};
  const size_t n[9] = {H, QD * H, KD * H, KD * H, H * QD, H, I * H, I * H, H * I};
  for (int i = 0; i < 9; ++i) ins.push_back({wp[i], n[i] * 2});
  if (grads) {
    const void *gp[9] = {grads->g1, grads->wq, grads->wk, grads->wv, grads->wo, grads->g2, grads->wg, grads->wu, grads->wd};
    for (int i = 0; i < 9; ++i) outs.push_back({gp[i], n[i] * 4});
  }
  check_apart(outs.data(), outs.size(), ins.data(), ins.size());
}

// bf16 saved activations as the caller's struct says, or those of the workspace with
// the vectors of the 8-bit struct
seg_layer_saved saved_of(const Ext &ext, const seg_layer_saved *saved, char *base, const LayerWs &W) {
  if (!ext.packed) {
    SEG_CHECK(saved, SEG_ERR_ARG, "saved is NULL");
    SEG_CHECK(saved->q && saved->k && saved->v && saved->o && saved->lse && saved->y1 &&
                  saved->rstd1 && saved->rstd2,
              SEG_ERR_ARG, "a saved-buffer pointer is NULL");
    return *saved;
  }
  return seg_layer_saved{base + W.q,  base + W.k,       base + W.v,         base + W.o, ext.packed->lse,
                         base + W.y1, ext.packed->rstd1, ext.packed->rstd2};
}

}  // namespace

extern "C" seg_status seg_layer_fwd_ext(const seg_layout *L, const seg_sizes *sz,
                                        const seg_layer_cfg *cfg, const seg_layer_ext *ext,
                                        const seg_layer_weights *w, const void *x, void *y,
                                        const seg_layer_saved *saved, void *ws, size_t ws_bytes,
                                        hipStream_t stream) {
  return guarded([&] {
    check_layer(L, sz, cfg, w);
    const Ext e = check_ext(ext, *sz, *cfg);
    const LayerWs W = layer_ws(*sz, *cfg, 0, e.packed != nullptr);
    SEG_CHECK(ws_bytes >= W.total, SEG_ERR_WORKSPACE, "workspace of %zu bytes < required %zu",
              ws_bytes, W.total);
    if (sz->packed_tokens == 0) return;
    SEG_CHECK(x && y && ws, SEG_ERR_ARG, "x, y or ws is NULL");
    check_ext_apart(e, *sz, *cfg, *w, x, y, nullptr, ws, W.total);
    char *base = static_cast<char *>(ws);
    layer_fwd_impl(L, sz, *cfg, e, *w, CUS(x), US(y), saved_of(e, saved, base, W), base, W, ws_bytes,
                   stream);
  });
}

extern "C" seg_status seg_layer_fwd(const seg_layout *L, const seg_sizes *sz,
                                    const seg_layer_cfg *cfg, const seg_layer_weights *w,
                                    const void *x, void *y, const seg_layer_saved *saved, void *ws,
                                    size_t ws_bytes, hipStream_t stream) {
  return seg_layer_fwd_ext(L, sz, cfg, nullptr, w, x, y, saved, ws, ws_bytes, stream);
}

extern "C" seg_status seg_layer_bwd_ext(const seg_layout *L, const seg_sizes *sz,
                                        const seg_layer_cfg *cfg, const seg_layer_ext *ext,
                                        const seg_layer_weights *w, const void *x,
                                        const seg_layer_saved *saved, const void *dy, void *dx,
                                        const seg_layer_grads *g, void *ws, size_t ws_bytes,
                                        hipStream_t stream) {
  return guarded([&] {
    check_layer(L, sz, cfg, w);
    const Ext e = check_ext(ext, *sz, *cfg);
    const LayerWs W = layer_ws(*sz, *cfg, 1, e.packed != nullptr);
    SEG_CHECK(ws_bytes >= W.total, SEG_ERR_WORKSPACE, "workspace of %zu bytes < required %zu",
              ws_bytes, W.total);
    SEG_CHECK(g && g->g1 && g->wq && g->wk && g->wv && g->wo && g->g2 && g->wg && g->wu && g->wd,
              SEG_ERR_ARG, "a gradient pointer is NULL");
    if (sz->packed_tokens == 0) {
      zero_grads(*g, *cfg, stream);
      return;
    }
    SEG_CHECK((x || e.packed) && dy && dx && ws, SEG_ERR_ARG, "x, dy, dx or ws is NULL");
    check_ext_apart(e, *sz, *cfg, *w, dy, dx, g, ws, W.total);
    char *base = static_cast<char *>(ws);
    const unsigned short *xs = e.packed ? CUS(base + W.x) : CUS(x);
    layer_bwd_impl(L, sz, *cfg, e, *w, xs, saved_of(e, saved, base, W), CUS(dy), US(dx), *g, base, W,
                   ws_bytes, stream);
  });
}

extern "C" seg_status seg_layer_bwd(const seg_layout *L, const seg_sizes *sz,
                                    const seg_layer_cfg *cfg, const seg_layer_weights *w,
                                    const void *x, const seg_layer_saved *saved, const void *dy,
                                    void *dx, const seg_layer_grads *g, void *ws, size_t ws_bytes,
                                    hipStream_t stream) {
  return seg_layer_bwd_ext(L, sz, cfg, nullptr, w, x, saved, dy, dx, g, ws, ws_bytes, stream);
}
