// Fused action-token log-prob and clipped policy-ratio loss with gradients
// (Eq. (loss) of App. E: min(rho A, clip(rho, 1 - eps_l, 1 + eps_h) A) over the
// trained action tokens, rho = pi_theta / pi_rollout), bf16 MFMA on gfx950.
//
// Only the R action rows are projected onto the vocabulary.  Pipeline:
//   1. zT[v][r] = s * W[v] . h[r] (MFMA, fp32 out) with a fused epilogue that
//      writes per-(row, 128-vocab tile) max / sum-exp partials and captures the
//      target logit;
//   2. per row: LSE from the partials (fixed order), logp, rho, loss, the
//      clipped flag and g = d loss_sum / d logp;
//   3. dzT = g * (onehot(target) - softmax(z))^T as bf16 (one pass over zT);
//   4. dH = s * dz W and dW = s * dz^T h (MFMA).
// All products use the shared kernel of gemm.h, which reads each operand in
// the orientation it has: dzT [V][R] serves dH (contracting over its rows)
// and dW (contracting along them), W and h serve as they are.
#include <climits>
#include <cmath>

#include "common.h"
#include "gemm.h"
#include "logits.h"

namespace seg {
namespace {

// The row statistics and the loss of LOSS_ROWS rows per block.  16 threads
// share a row, each taking every 16th slab, so a block reads 128-byte pieces
// of the slab-major statistics (one block per row read 8 of every 64 bytes: 89
// us for 7,680 rows x 1,187 slabs, now 26); their results are combined
// in a fixed order.
constexpr int LOSS_ROWS = 16;

__global__ void __launch_bounds__(256) k_row_loss(
    const float2 *__restrict__ stats, int ntiles, int rows, const float *__restrict__ ztgt,
    const float *__restrict__ old_logp, const float *__restrict__ ref_logp,
    const float *__restrict__ adv, const int32_t *__restrict__ row_traj, int num_traj,
    seg_loss_cfg cfg, float *__restrict__ logp, float *__restrict__ loss_tok,
    uint8_t *__restrict__ clipped, float *__restrict__ kl_tok, float *__restrict__ lse_out,
    float *__restrict__ g_out) {
  constexpr int SL = 256 / LOSS_ROWS;
  __shared__ float2 red[SL][LOSS_ROWS];
  const int t = threadIdx.x % LOSS_ROWS, part = threadIdx.x / LOSS_ROWS;
  const int r = blockIdx.x * LOSS_ROWS + t;
  float mx = -INFINITY, sm = 0.f;
  if (r < rows) {
#pragma unroll 4
    for (int i = part; i < ntiles; i += SL) {
      const float2 s = meet(make_float2(mx, sm), stats[(long)i * rows + r]);
      mx = s.x;
      sm = s.y;
    }
  }
  red[part][t] = make_float2(mx, sm);
  __syncthreads();
  if (part == 0 && r < rows) {
    for (int k = 1; k < SL; ++k) {
      const float2 s = meet(make_float2(mx, sm), red[k][t]);
      mx = s.x;
      sm = s.y;
    }
    const float lse = (mx + log2f(sm)) * LN2;
    const float lp = ztgt[r] - lse;
    // an out-of-range trajectory index yields NaN rather than a stray read
    const int tj = row_traj[r];
    const float A = (tj >= 0 && tj < num_traj) ? adv[tj] : __builtin_nanf("");
    const float rho = expf(lp - old_logp[r]);
    const float lo = 1.f - cfg.eps_low, hi = 1.f + cfg.eps_high;
    const float unc = rho * A;
    const float clp = fminf(fmaxf(rho, lo), hi) * A;
    float obj = fminf(unc, clp);
    bool cl = (A > 0.f && rho > hi) || (A < 0.f && rho < lo);
    if (cfg.dual_clip_c > 0.f && A < 0.f) {
      obj = fmaxf(obj, cfg.dual_clip_c * A);
      cl = cl || rho > cfg.dual_clip_c;
    }
    // KL(pi_theta || pi_ref) per token: e^x - x - 1 with x = ref - logp,
    // written expm1(x) - x (no cancellation for small x); its logp
    // derivative is 1 - e^x = -expm1(x)
    float kl = 0.f, dkl = 0.f;
    if (ref_logp) {
      const float x = ref_logp[r] - lp, em1 = expm1f(x);
      kl = em1 - x;
      dkl = -em1;
    }
    logp[r] = lp;
    loss_tok[r] = -obj + cfg.kl_coef * kl;
    clipped[r] = cl ? 1 : 0;
    if (kl_tok) kl_tok[r] = kl;
    lse_out[r] = lse;
    g_out[r] = (cl ? 0.f : -cfg.loss_scale * rho * A) + cfg.loss_scale * cfg.kl_coef * dkl;
  }
}

// Preparation of a call in one launch: the gathered action rows as bf16
// (y[r] = h[rowmap[r]], zero from `rows` to rows_pad), for fp32 inputs the
// projection as bf16 (wb), and NaN in the target logits (a target outside the
// vocabulary keeps it).  8 elements a thread where `vec` (the tensors start on
// 16-byte boundaries; cols is a multiple of 8), else one by one.
template <class TI>
__global__ void __launch_bounds__(256) k_lp_prep(const TI *__restrict__ h,
                                                 const int32_t *__restrict__ rowmap, int rows,
                                                 int rows_pad, int cols, bool hvec,
                                                 unsigned short *__restrict__ y,
                                                 const TI *__restrict__ w, long w8, bool wvec,
                                                 unsigned short *__restrict__ wb,
                                                 float *__restrict__ ztgt) {
  const unsigned c8 = cols / 8;
  const long n = (long)rows_pad * c8, step = (long)gridDim.x * 256;
  const long at = (long)blockIdx.x * 256 + threadIdx.x;
  for (long i = at; i < rows_pad; i += step) ztgt[i] = __builtin_nanf("");
  for (long i = at; i < n; i += step) {
    const int r = n >> 32 ? (int)(i / c8) : (int)((unsigned)i / c8);
    const long c = i - (long)r * c8;
    u16x8 v = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (r < rows) v = load8(h + (long)(rowmap ? rowmap[r] : r) * cols + c * 8, hvec);
    *reinterpret_cast<u16x8 *>(y + i * 8) = v;
  }
  if constexpr (sizeof(TI) == 4) {
    for (long i = at; i < w8; i += step)
      *reinterpret_cast<u16x8 *>(wb + i * 8) = load8(w + i * 8, wvec);
  }
}

struct LpWs {
  size_t hb, wb, zt, stats, ztgt, lse, g, dzt, total;
  int Rp, ntiles;
};

LpWs lp_ws(int rows, int hidden, int vocab, seg_dtype dt) {
  LpWs w{};
  w.Rp = (rows + 31) / 32 * 32;
  w.ntiles = (vocab + 127) / 128;  // 128-row slabs of the logits epilogue
  size_t off = 0;
  auto take = [&](size_t bytes) {
    size_t o = off;
    off = align_up(off + std::max<size_t>(bytes, 1));
    return o;
  };
  const size_t Rp = w.Rp, H = hidden;
  w.hb = take(Rp * H * 2);
  w.wb = dt == SEG_F32 ? take((size_t)vocab * H * 2) : 0;
  w.zt = take((size_t)vocab * Rp * 4);
  w.stats = take((size_t)w.ntiles * std::max(rows, 1) * sizeof(float2));
  w.ztgt = take(Rp * 4);
  w.lse = take(Rp * 4);
  w.g = take(Rp * 4);
  w.dzt = take((size_t)vocab * Rp * 2);
  w.total = off;
  return w;
}

template <class TI, class TO>
void logprob_impl(int rows, int H, int V, const TI *h, const int32_t *row_index, const TI *w,
                  const int32_t *target, const float *old_logp, const float *ref_logp,
                  const float *adv, const int32_t *row_traj, int num_traj,
                  const seg_loss_cfg &cfg, float *logp, float *loss_tok, uint8_t *clipped,
                  float *kl_tok, float *loss_sum, void *dh, float *dw, char *base,
                  const LpWs &L, hipStream_t st) {
  const int Rp = L.Rp;
  unsigned short *hb = reinterpret_cast<unsigned short *>(base + L.hb);
  float *zt = reinterpret_cast<float *>(base + L.zt);
  float2 *stats = reinterpret_cast<float2 *>(base + L.stats);
  float *ztgt = reinterpret_cast<float *>(base + L.ztgt);
  float *lse = reinterpret_cast<float *>(base + L.lse);
  float *g = reinterpret_cast<float *>(base + L.g);
  unsigned short *dzt = reinterpret_cast<unsigned short *>(base + L.dzt);

  const unsigned short *wb;
  {
    unsigned short *w2 = sizeof(TI) == 4 ? reinterpret_cast<unsigned short *>(base + L.wb) : nullptr;
    const long n8 = (long)Rp * (H / 8), w8 = sizeof(TI) == 4 ? (long)V * (H / 8) : 0;
    auto vec = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    ProfScope prof("lp_prep", st);
    k_lp_prep<TI><<<(int)std::min<long>(16384, (std::max(n8, w8) + 255) / 256), 256, 0, st>>>(
        h, row_index, rows, Rp, H, vec(h), hb, w, w8, vec(w), w2, ztgt);
    SEG_LAUNCH_CHECK();
    wb = w2 ? w2 : reinterpret_cast<const unsigned short *>(w);
  }
  // 1. logits zT = s * W h^T with partial softmax stats; the target logit
  //    stays NaN for a target outside [0, vocab)
  {
    EpiLogits<true> e{cfg.want_grad ? zt : nullptr, Rp, stats, rows, target, ztgt, cfg.logit_scale,
                (long)V * Rp * 4 > (256L << 20)};
    ProfScope prof("logits", st);
    gemm::Problems<EpiLogits<true>, 1, 1> g{{{wb}}, {{hb}}, {{H}}, {{H}}, {H}, {V}, {rows}, {e}, {}, 1,
                                      (H + gemm::BK - 1) / gemm::BK};
    gemm::launch_tm<false, false, 4>(g, st);
  }
  // 2. per-row loss
  {
  ProfScope prof("row_loss", st);
  k_row_loss<<<(rows + LOSS_ROWS - 1) / LOSS_ROWS, 256, 0, st>>>(stats, L.ntiles, rows, ztgt, old_logp, ref_logp, adv, row_traj,
                                   num_traj, cfg, logp, loss_tok, clipped, kl_tok, lse, g);
  SEG_LAUNCH_CHECK();
  if (!cfg.want_grad) {
    k_loss_sum<<<1, 256, 0, st>>>(loss_tok, rows, cfg.loss_scale, loss_sum);
    SEG_LAUNCH_CHECK();
    return;
  }
  }
  // 3. dz
  {
    ProfScope prof("dz", st);
    const int vr = dz_rows(V, Rp);
    k_dz<true><<<dim3((Rp + DZ_COLS - 1) / DZ_COLS, (V + vr - 1) / vr + 1), 256, 0, st>>>(
        zt, V, rows, Rp, vr, lse, g, target, dzt, loss_tok, cfg.loss_scale, loss_sum);
    SEG_LAUNCH_CHECK();
  }
  // 4. dH = s * dz W: A = dz^T [V][Rp], B = W [V][H], contracting over the
  //    vocabulary rows of both
  {
    ProfScope prof("dh", st);
    // zT has served: its place holds partial sums when the vocabulary is cut
    gemm::launch_one<true, true>(dzt, Rp, wb, H, rows, H, V,
                                 EpiOut<TO, ST>::make(static_cast<TO *>(dh), H, cfg.logit_scale),
                                 gemm::Scratch{zt, (long)V * Rp}, 0, st);
  }
  //    dW = s * dz^T h: A = dz^T along its rows (zero in the padded columns),
  //    B = h [Rp][H] (zero in the padded rows)
  {
    ProfScope prof("dw", st);
    gemm::launch_one<false, true>(dzt, Rp, hb, H, V, H, Rp,
                                  EpiOut<float, ST>::make(dw, H, cfg.logit_scale), st);
  }
}

}  // namespace
}  // namespace seg

using namespace seg;

extern "C" size_t seg_logprob_workspace_bytes(int32_t rows, int32_t hidden, int32_t vocab,
                                              seg_dtype dt) {
  if (rows < 0 || hidden < 1 || vocab < 1) return 0;
  return lp_ws(rows, hidden, vocab, dt).total;
}

extern "C" seg_status seg_logprob_loss(int32_t rows, int32_t hidden, int32_t vocab, seg_dtype dt,
                                       const void *h, const int32_t *row_index, const void *w,
                                       const int32_t *target, const float *old_logp,
                                       const float *ref_logp, const float *adv,
                                       const int32_t *row_traj, int32_t num_traj,
                                       const seg_loss_cfg *cfg, float *logp, float *loss_tok,
                                       uint8_t *clipped, float *kl_tok, float *loss_sum,
                                       void *dh, float *dw, void *ws, size_t ws_bytes,
                                       hipStream_t stream) {
  return guarded([&] {
    SEG_CHECK(cfg != nullptr, SEG_ERR_ARG, "cfg is NULL");
    SEG_CHECK(dt == SEG_BF16 || dt == SEG_F32, SEG_ERR_ARG, "unknown dtype %d", (int)dt);
    SEG_CHECK(rows >= 0 && hidden >= 1 && vocab >= 1 && num_traj >= 0, SEG_ERR_ARG,
              "bad sizes rows=%d hidden=%d vocab=%d num_traj=%d", rows, hidden, vocab, num_traj);
    SEG_CHECK(hidden % 8 == 0, SEG_ERR_UNSUPPORTED, "hidden %d must be a multiple of 8", hidden);
    // GEMM operand rows (hidden, padded vocab, padded rows) are addressed with
    // 32-bit offsets inside a 256-row block
    SEG_CHECK(hidden <= (1 << 20) && vocab <= (1 << 20) - 256 && rows <= (1 << 20) - 256,
              SEG_ERR_CAPACITY, "rows %d, hidden %d or vocab %d above 2^20", rows, hidden, vocab);
    SEG_CHECK(std::isfinite(cfg->eps_low) && std::isfinite(cfg->eps_high) &&
                  std::isfinite(cfg->loss_scale) && std::isfinite(cfg->logit_scale) &&
                  std::isfinite(cfg->dual_clip_c) && std::isfinite(cfg->kl_coef),
              SEG_ERR_ARG, "non-finite loss setting");
    SEG_CHECK(cfg->eps_low >= 0.f && cfg->eps_high >= 0.f, SEG_ERR_ARG, "negative clip range");
    SEG_CHECK(cfg->kl_coef >= 0.f, SEG_ERR_ARG, "negative kl_coef");
    SEG_CHECK(cfg->kl_coef == 0.f || ref_logp != nullptr, SEG_ERR_ARG,
              "kl_coef > 0 needs ref_logp");
    const LpWs L = lp_ws(rows, hidden, vocab, dt);
    SEG_CHECK(ws_bytes >= L.total, SEG_ERR_WORKSPACE, "workspace of %zu bytes < required %zu",
              ws_bytes, L.total);
    SEG_CHECK(loss_sum != nullptr, SEG_ERR_ARG, "loss_sum is NULL");
    if (rows == 0) {
      fill32(loss_sum, 1, 0u, stream);
      if (cfg->want_grad && dw) fill32(dw, (long)vocab * hidden, 0u, stream);
      return;
    }
    SEG_CHECK(h && w && target && old_logp && adv && row_traj && logp && loss_tok && clipped && ws,
              SEG_ERR_ARG, "a tensor pointer is NULL");
    SEG_CHECK(num_traj >= 1, SEG_ERR_ARG, "num_traj must be >= 1 when rows > 0");
    if (cfg->want_grad) SEG_CHECK(dh && dw, SEG_ERR_ARG, "dh/dw is NULL with want_grad");
    char *base = static_cast<char *>(ws);
    if (dt == SEG_F32)
      logprob_impl<float, float>(rows, hidden, vocab, static_cast<const float *>(h), row_index,
                                 static_cast<const float *>(w), target, old_logp, ref_logp, adv,
                                 row_traj, num_traj, *cfg, logp, loss_tok, clipped, kl_tok,
                                 loss_sum, dh, dw, base, L, stream);
    else
      logprob_impl<unsigned short, unsigned short>(
          rows, hidden, vocab, static_cast<const unsigned short *>(h), row_index,
          static_cast<const unsigned short *>(w), target, old_logp, ref_logp, adv, row_traj,
          num_traj, *cfg, logp, loss_tok, clipped, kl_tok, loss_sum, dh, dw, base, L, stream);
  });
}
