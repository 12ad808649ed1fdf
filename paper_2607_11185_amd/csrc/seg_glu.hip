// Gated feed-forward block silu(x Wg^T) * (x Wu^T) with its backward.
//
// Forward: one GEMM launch for both projections; its epilogue forms the product
// from the fp32 accumulators (one rounding, of m), and can keep the gate and up
// values for the backward, in bf16 or in 8 bits with a power of two per 32
// features (act8.h).  Backward: one streaming pass turns the kept values and dm
// into dg and du, and two GEMM launches give dx = dg Wg + du Wu (one sum over
// both contractions) and both weight gradients.
#include <algorithm>

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

__device__ __forceinline__ float sigmoidf_(float g) { return 1.f / (1.f + __expf(-g)); }

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
        int eg = 0, eu = 0;
        if constexpr (KEEP == CODES) {
          unsigned tg = 0, tu = 0;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              tg = max(tg, act8::mag(g[j][r]));
              tu = max(tu, act8::mag(u[j][r]));
            }
#pragma unroll
          for (int o = 16; o <= 32; o *= 2) {
            tg = max(tg, (unsigned)__shfl_xor((int)tg, o, 64));
            tu = max(tu, (unsigned)__shfl_xor((int)tu, o, 64));
          }
          eg = act8::exp_byte(tg);
          eu = act8::exp_byte(tu);
          const int row = t.m0 + t.wr + bm * 32 + i * 16 + t.col;
          const long at = (long)row * ((I + act8::BLOCK - 1) / act8::BLOCK) + f0 / act8::BLOCK;
          if (row < t.M && t.grp == 0) k.g8.exp[at] = (uint8_t)eg;
          if (row < t.M && t.grp == 1) k.u8.exp[at] = (uint8_t)eu;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x4 gv = g[j], uv = u[j];
          float mv[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) mv[r] = gv[r] * sigmoidf_(gv[r]) * uv[r];
          const int at = (i * 16 + t.col) * 8 + ((j * 4 + t.grp) ^ (t.col & 6));
          w[at] = gemm::u32x2{gemm::pack2(mv[0], mv[1]), gemm::pack2(mv[2], mv[3])};
          if constexpr (KEEP == BF16) {
            w[256 + at] = gemm::u32x2{gemm::pack2(gv[0], gv[1]), gemm::pack2(gv[2], gv[3])};
            w[512 + at] = gemm::u32x2{gemm::pack2(uv[0], uv[1]), gemm::pack2(uv[2], uv[3])};
          }
          if constexpr (KEEP == CODES) {
            wc[at] = act8::codes4(gv[0], gv[1], gv[2], gv[3], eg);
            wc[256 + at] = act8::codes4(uv[0], uv[1], uv[2], uv[3], eu);
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
#pragma unroll
    for (int o = 1; o <= 2; o *= 2) {
      tg = max(tg, (unsigned)__shfl_xor((int)tg, o, 64));
      tu = max(tu, (unsigned)__shfl_xor((int)tu, o, 64));
    }
    eg = act8::exp_byte(tg);
    eu = act8::exp_byte(tu);
  }
  if (!in) return;
  const long off = (long)row * I + f;
  u16x8 m;
#pragma unroll
  for (int j = 0; j < 8; ++j) m[j] = f2bf_bits(g[j] * sigmoidf_(g[j]) * u[j]);
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
    *reinterpret_cast<uint2 *>(ep.k.g8.code + off) = make_uint2(act8::codes4(g[0], g[1], g[2], g[3], eg),
                                                                 act8::codes4(g[4], g[5], g[6], g[7], eg));
    *reinterpret_cast<uint2 *>(ep.k.u8.code + off) = make_uint2(act8::codes4(u[0], u[1], u[2], u[3], eu),
                                                                 act8::codes4(u[4], u[5], u[6], u[7], eu));
  }
}

// dg = dm * u * silu'(g), du = dm * silu(g), silu'(g) = s (1 + g (1 - s)),
// s = sigmoid(g), and m = silu(g) * u; 8 features a thread.  A streaming kernel:
// folded into the epilogue of the GEMM that makes dm its loads stall the one
// wave per SIMD.
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
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = bf_bits2f(mv[j]), s = sigmoidf_(g[j]);
      og[j] = f2bf_bits(d * u[j] * s * (1.f + g[j] * (1.f - s)));
      ou[j] = f2bf_bits(d * g[j] * s);
      om[j] = f2bf_bits(g[j] * s * u[j]);
    }
    *reinterpret_cast<u16x8 *>(dg + c * 8) = og;
    *reinterpret_cast<u16x8 *>(du + c * 8) = ou;
    if (m) *reinterpret_cast<u16x8 *>(m + c * 8) = om;
  }
}

int pair_columns(int inter) { return 2 * (int)act8::blocks_of(inter) * act8::BLOCK; }

// How a forward of its own (not a chunk of a layer) is launched, with up to MAX_SUMS
// partial sums.
gemm::Choice choose_fwd(int rows, int hidden, int inter) {
  const int N = pair_columns(inter);
  const long steps = (hidden + gemm::BK - 1) / gemm::BK;
  const long t4 = gemm::tiles_of(rows, N, 4), t2 = gemm::tiles_of(rows, N, 2);
  return gemm::choose_even(gemm::choose(t4, t2, steps, 1, 0), t4, steps, MAX_SUMS);
}

size_t fwd_sums(int rows, int hidden, int inter) {
  const gemm::Choice c = choose_fwd(rows, hidden, inter);
  if (!c.rest || c.parts == 1) return 256;
  return (size_t)c.parts * (gemm::tiles_of(rows, pair_columns(inter), 4) - c.full) * gemm::bm_of(4) * gemm::BN * 4;
}

}  // namespace

namespace glu {

void forward(const unsigned short *x, long ldx, const unsigned short *wg, const unsigned short *wu, int rows,
             int hidden, int inter, unsigned short *m, const Kept &keep, float *sums, hipStream_t st) {
  const int N = pair_columns(inter);
  const gemm::Choice c = sums ? choose_fwd(rows, hidden, inter) : gemm::Choice{4, 1, 0};
  auto go = [&](auto ep) {
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
// tiles in whole rounds, whether there is a rest}.
extern "C" void seg_glu_gemm_choice(int32_t rows, int32_t hidden, int32_t inter, int32_t which, int32_t *out) {
  gemm::Choice c;
  const long sums = glu_ws(rows, hidden, inter, true).sum_elems;
  if (which == 0) {
    c = choose_fwd(rows, hidden, inter);
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
