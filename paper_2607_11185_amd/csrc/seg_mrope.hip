// Rotary embedding with positions on several axes (time, height, width): pair
// (x_i, x_{i + d/2}) of a head turns by pos[axis(i)] base^(-2i/d), where the
// first pairs belong to the time axis, the next to the height and the last to
// the width; the backward turns by minus that angle (the transpose).
//
// Bound by HBM: q and k are read once and written once (137,895 rows x 32 heads x
// 128, bf16: 375 us, 6.0 TB/s).  A block takes a few rows: it issues their loads,
// forms each row's d/2 cosines and sines once for all heads while they are on
// their way (loads behind the angles: 397 us; two or eight pairs of pieces a thread
// for four: 383, 401), and keeps those in LDS.  An angle of a
// far position needs more than fp32 (at position 10^6 its last place is 1/16
// of a radian), so the turns are formed and reduced in fp64 and only the part
// of a turn that is left goes to fp32.  That rounding moves an angle by up to 9.4e-8: next
// to nothing where results round to bf16, but more than the rest of an fp32 rotation, which
// turns by the remainder too (to first order: its square is below 10^-14).
#include <cmath>

#include "mrope.h"

namespace seg {
namespace {

constexpr int MAX_ROWS = 16;       // rows of a block
constexpr int ITEMS = 4;          // 16-byte pairs of pieces of a thread in flight
constexpr int CS = 512;            // (cos, sin) pairs of a block

// 16 bytes of a row
template <class T>
struct Piece;
template <>
struct Piece<unsigned short> {
  static constexpr int W = 8;
  u16x8 v;
  __device__ __forceinline__ float get(int j) const { return bf_bits2f(v[j]); }
  __device__ __forceinline__ void set(int j, float f) { v[j] = f2bf_bits(f); }
};
template <>
struct Piece<float> {
  static constexpr int W = 4;
  f32x4 v;
  __device__ __forceinline__ float get(int j) const { return v[j]; }
  __device__ __forceinline__ void set(int j, float f) { v[j] = f; }
};
template <class T, bool STREAM>
__device__ __forceinline__ Piece<T> load_piece(const T *p) {
  const auto *q = reinterpret_cast<const decltype(Piece<T>::v) *>(p);
  return Piece<T>{STREAM ? __builtin_nontemporal_load(q) : *q};
}
template <class T, bool STREAM>
__device__ __forceinline__ void store_piece(T *p, const Piece<T> &x) {
  auto *q = reinterpret_cast<decltype(Piece<T>::v) *>(p);
  if (STREAM) __builtin_nontemporal_store(x.v, q);
  else *q = x.v;
}

// rows_per rows a block; half_pow: d/2 rounded up to a power of two; STREAM: more
// than the caches hold is read and written, so accesses go past them.  Five waves a
// SIMD serve what comes from the caches (10,007 x 16 x 64, fp32: 14.0 us against 15.6
// with the four of its free choice of registers), four what comes from memory (375
// against 393).
template <class T, bool STREAM>
__global__ void __launch_bounds__(256, STREAM ? 1 : 5) k_mrope(const mrope::Args g, int rows_per, int half_pow) {
  __shared__ __attribute__((aligned(16))) float2 cs[CS];
  __shared__ int ok[MAX_ROWS];
  typedef Piece<T> E;
  constexpr int W = E::W;
  const int half = g.d / 2, per = half / W, chunks = (g.a.heads + g.b.heads) * per;
  const long row0 = (long)blockIdx.x * rows_per;
  const int rows = (int)min((long)rows_per, g.rows - row0);
  // a thread's pieces: ITEMS at a time, the first ones under way during the angles
  const int items = rows * chunks;
  E lo[ITEMS], hi[ITEMS];
  T *to[ITEMS];
  int at[ITEMS];  // (row, pair) in cs; -1: none
  auto load = [&](int base) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < ITEMS; ++n) {
      const int e = base + n * 256 + threadIdx.x;
      at[n] = -1;
      if (e >= items) continue;
      const int r = e / chunks, q = e - r * chunks, h = q / per, i = (q - h * per) * W;
      const long row = row0 + r;
      const bool first = h < g.a.heads;
      const int hh = first ? h : h - g.a.heads;
      const T *x = static_cast<const T *>(first ? g.a.x : g.b.x) + row * (first ? g.a.ldx : g.b.ldx) + hh * g.d + i;
      to[n] = static_cast<T *>(first ? g.a.y : g.b.y) + row * (first ? g.a.ldy : g.b.ldy) + hh * g.d + i;
      at[n] = r * half + i;
      lo[n] = load_piece<T, STREAM>(x);
      hi[n] = load_piece<T, STREAM>(x + half);
    }
  };
  load(0);
  for (int e = threadIdx.x; e < rows * half_pow; e += 256) {
    const int r = e / half_pow, i = e & (half_pow - 1);
    const long row = row0 + r;
    if (i == 0) {
      bool y = true;
      if (g.pad) y = g.pad[row] >= 0;
      else
        for (int a = 0; a < 3; ++a) y = y && g.pos[a * g.rows + row] >= 0;
      ok[r] = y;
    }
    if (i < half) {
      const int axis = i < g.s0 ? 0 : i < g.s01 ? 1 : 2;
      // turns = pos base^(-2i/d) / (2 pi)
      const double f = exp2(-(double)(2 * i) / g.d * g.log2_base) * 0.15915494309189535;
      const double t = (double)g.pos[axis * g.rows + row] * f, left = t - rint(t);
      const float turn = (float)left;
      float s, c;
      sincospif(2.f * turn, &s, &c);
      if constexpr (sizeof(T) == 4) {  // and by what that rounding left out
        const float rest = (float)(left - turn) * 6.2831855f, c0 = c;
        c = fmaf(-rest, s, c);
        s = fmaf(rest, c0, s);
      }
      cs[r * half + i] = make_float2(c, g.inverse ? -s : s);
    }
  }
  __syncthreads();
  for (int base = 0; base < items; base += ITEMS * 256) {
    if (base > 0) load(base);
#pragma unroll
    for (int n = 0; n < ITEMS; ++n) {
      if (at[n] < 0) continue;
      E olo, ohi;
      if (ok[at[n] / half]) {
        const f32x4 *t = reinterpret_cast<const f32x4 *>(cs + at[n]);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const f32x4 w = t[j / 2];
          const float c = w[(j & 1) * 2], s = w[(j & 1) * 2 + 1];
          olo.set(j, lo[n].get(j) * c - hi[n].get(j) * s);
          ohi.set(j, hi[n].get(j) * c + lo[n].get(j) * s);
        }
      } else if (g.inverse) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
          olo.set(j, 0.f);
          ohi.set(j, 0.f);
        }
      } else {
        olo = lo[n];
        ohi = hi[n];
      }
      store_piece<T, STREAM>(to[n], olo);
      store_piece<T, STREAM>(to[n] + half, ohi);
    }
  }
  if (g.zero && g.inverse)
    for (int r = 0; r < rows; ++r)
      if (!ok[r])
        for (int c = threadIdx.x; c < g.zero_width / 8; c += 256)
          *reinterpret_cast<u16x8 *>(g.zero + (row0 + r) * g.zero_width + c * 8) =
              u16x8{0, 0, 0, 0, 0, 0, 0, 0};
}

}  // namespace

namespace mrope {

void check_cfg(const seg_mrope_cfg *cfg, int32_t d) {
  SEG_CHECK(cfg, SEG_ERR_ARG, "the rotary cfg is NULL");
  SEG_CHECK(d >= 16 && d % 16 == 0 && d <= MAX_D, SEG_ERR_UNSUPPORTED,
            "head_dim %d must be a multiple of 16 up to %d", d, MAX_D);
  long sum = 0;
  for (int a = 0; a < 3; ++a) {
    SEG_CHECK(cfg->sections[a] >= 0, SEG_ERR_ARG, "sections[%d] < 0", a);
    sum += cfg->sections[a];
  }
  SEG_CHECK(sum == d / 2, SEG_ERR_ARG, "the sections sum to %ld, not to head_dim / 2 = %d", sum, d / 2);
  SEG_CHECK(std::isfinite(cfg->base) && cfg->base > 1.f, SEG_ERR_ARG, "the rotary base must be > 1");
}

namespace {

// rows of a block, d/2 rounded up to a power of two, blocks
struct Grid {
  int rows_per, half_pow;
  long blocks;
};

Grid grid_of(seg_dtype dt, long rows, int heads, int d) {
  const int half = d / 2, chunks = heads * half / (dt == SEG_BF16 ? Piece<unsigned short>::W : Piece<float>::W);
  int hp = 8;
  while (hp < half) hp *= 2;
  const int want = (ITEMS * 256 + chunks - 1) / chunks;
  const int rows_per = std::max(1, std::min(std::min(want, MAX_ROWS), CS / hp));
  return Grid{rows_per, hp, (rows + rows_per - 1) / rows_per};
}

}  // namespace

void check_launch(seg_dtype dt, long rows, int heads, int d) {
  SEG_CHECK(grid_of(dt, rows, heads, d).blocks <= 0x7fffffffL / 256, SEG_ERR_CAPACITY, "too many rows for one launch");
}

void launch(seg_dtype dt, const Args &g, hipStream_t st) {
  if (g.rows == 0) return;
  check_launch(dt, g.rows, g.a.heads + g.b.heads, g.d);
  const Grid grid = grid_of(dt, g.rows, g.a.heads + g.b.heads, g.d);
  const long bytes = g.rows * (g.a.heads + g.b.heads) * g.d * (dt == SEG_BF16 ? 2 : 4) * 2;
  const bool stream = bytes > STREAM_BYTES;
  auto go = [&](auto kernel) { kernel<<<(unsigned)grid.blocks, 256, 0, st>>>(g, grid.rows_per, grid.half_pow); };
  if (dt == SEG_BF16) go(stream ? k_mrope<unsigned short, true> : k_mrope<unsigned short, false>);
  else go(stream ? k_mrope<float, true> : k_mrope<float, false>);
  SEG_LAUNCH_CHECK();
}

}  // namespace mrope

namespace {

// rows of `width` bytes, `ld` bytes apart
struct Rows {
  const void *p;
  int64_t ld, width;
};

// Whether they share a byte.  At one stride they may be parts of the same wide
// rows: then the columns decide.
bool meet(const Rows &a, const Rows &b, int64_t rows) {
  const __int128 x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);  // strides up to 2^42
  if (x >= y + (__int128)(rows - 1) * b.ld + b.width || y >= x + (__int128)(rows - 1) * a.ld + a.width) return false;
  if (rows == 1 || a.ld != b.ld) return true;
  const int64_t at = (int64_t)(((y - x) % a.ld + a.ld) % a.ld);
  return at < a.width || at + b.width > a.ld;
}

// Whether rows share a byte with the n bytes from p on.
bool meet(const Rows &a, int64_t rows, const void *p, int64_t n) {
  const __int128 x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(p);
  const __int128 r = y < x + a.width ? 0 : (y - x - a.width) / a.ld + 1;  // the first row that ends behind p
  return r < rows && x + r * a.ld < y + n;
}

seg_status rotate(int64_t rows, seg_dtype dt, const seg_mrope_cfg *cfg, int32_t hq, int32_t hkv, int32_t d,
                  const int32_t *pos, const void *q, int64_t ldq, const void *k, int64_t ldk, void *qo,
                  int64_t ldqo, void *ko, int64_t ldko, int inverse, hipStream_t stream) {
  return guarded([&] {
    SEG_CHECK(dt == SEG_BF16 || dt == SEG_F32, SEG_ERR_UNSUPPORTED, "dtype %d not supported", (int)dt);
    mrope::check_cfg(cfg, d);
    SEG_CHECK(rows >= 0, SEG_ERR_ARG, "rows < 0");
    SEG_CHECK(hq >= 1 && hkv >= 0 && hq <= 65536 && hkv <= 65536, SEG_ERR_ARG, "heads %d/%d out of range", hq, hkv);
    SEG_CHECK(rows < (1LL << 31), SEG_ERR_CAPACITY, "more than 2^31-1 rows");
    if (rows == 0) return;
    SEG_CHECK(pos && q && qo && (hkv == 0 || (k && ko)), SEG_ERR_ARG, "pos, a tensor or an output is NULL");
    const int64_t e = dt == SEG_BF16 ? 2 : 4;
    const void *ptr[4] = {q, k, qo, ko};
    const int64_t ld[4] = {ldq, ldk, ldqo, ldko};
    for (int i = 0; i < 4; ++i) {
      const int64_t heads = i & 1 ? hkv : hq;
      if (heads == 0) continue;
      SEG_CHECK(ld[i] >= heads * d && ld[i] < (1LL << 40), SEG_ERR_ARG, "row stride %lld does not hold %lld heads of %d",
                (long long)ld[i], (long long)heads, d);
      SEG_CHECK(reinterpret_cast<uintptr_t>(ptr[i]) % 16 == 0 && ld[i] * e % 16 == 0, SEG_ERR_UNSUPPORTED,
                "rows must start on 16-byte boundaries");
    }
    Rows t[4];
    for (int i = 0; i < 4; ++i) t[i] = Rows{ptr[i], ld[i] * e, (i & 1 ? hkv : hq) * (int64_t)d * e};
    for (int o = 2; o < 4; ++o) {
      SEG_CHECK(!t[o].width || !meet(t[o], rows, pos, 12 * rows), SEG_ERR_ARG, "an output overlaps pos");
      for (int i = 0; i < o; ++i) {
        const bool itself = i == o - 2 && t[i].p == t[o].p && t[i].ld == t[o].ld;
        SEG_CHECK(!t[i].width || !t[o].width || itself || !meet(t[i], t[o], rows), SEG_ERR_ARG,
                  "an output overlaps an input that is not its own, or another output");
      }
    }
    mrope::Args g{};
    g.a = mrope::Heads{q, qo, ldq, ldqo, hq};
    g.b = mrope::Heads{k, ko, ldk, ldko, hkv};
    g.rows = rows;
    g.d = d;
    g.inverse = inverse;
    g.set(*cfg);
    g.pos = pos;
    ProfScope prof("mrope", stream);
    mrope::launch(dt, g, stream);
  });
}

}  // namespace
}  // namespace seg

using namespace seg;

extern "C" seg_status seg_mrope_fwd(int64_t rows, seg_dtype dt, const seg_mrope_cfg *cfg, int32_t hq,
                                    int32_t hkv, int32_t d, const int32_t *pos, const void *q,
                                    int64_t ldq, const void *k, int64_t ldk, void *q_out,
                                    int64_t ldqo, void *k_out, int64_t ldko, hipStream_t stream) {
  return rotate(rows, dt, cfg, hq, hkv, d, pos, q, ldq, k, ldk, q_out, ldqo, k_out, ldko, 0, stream);
}

extern "C" seg_status seg_mrope_bwd(int64_t rows, seg_dtype dt, const seg_mrope_cfg *cfg, int32_t hq,
                                    int32_t hkv, int32_t d, const int32_t *pos, const void *dq,
                                    int64_t ldq, const void *dk, int64_t ldk, void *dq_out,
                                    int64_t ldqo, void *dk_out, int64_t ldko, hipStream_t stream) {
  return rotate(rows, dt, cfg, hq, hkv, d, pos, dq, ldq, dk, ldk, dq_out, ldqo, dk_out, ldko, 1, stream);
}
