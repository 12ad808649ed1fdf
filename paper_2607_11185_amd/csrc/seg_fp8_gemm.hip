// Product of two tensors in 8-bit floating point with blocks of 128 (format: fp8.h):
//   y(m, n) = sum_b 2^(sa(m, b) + sb(n, b)) sum_{k in block b} a(m, k) b(n, k)
// A step of the inner loop is one block of columns, 128 bytes of a row, and one matrix
// instruction (16x16x128) takes a whole step and both operands' powers of two, so the
// scales cost no arithmetic.  Inside the instruction the products of groups of 16
// columns (each whole on its own) are aligned to the group's largest and lose what is
// 2^-13 of it and below; the groups' sums and the accumulator add up in fp32.  (An
// 8-bit instruction without scales rounds the same way.)
//
// The compiler does not always keep vector instructions that read the result of such an
// instruction away from it for long enough (copies of an accumulator at the end of a
// loop got the one of before).  So every loop with such instructions ends with settled(),
// which waits longer than they take, and results are read behind it; other matrix
// instructions may follow at once, the hardware orders them.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "fp8.h"
#include "gemm.h"

namespace seg {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// one step: SW and SX pick the byte of each lane's row in sw and sx
template <int SW, int SX>
__device__ __forceinline__ f32x4 mfma8(const i32x8 &w, const i32x8 &x, const f32x4 &c, unsigned sw, unsigned sx) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, SW, (int)sw, SX, (int)sx);
}
__device__ __forceinline__ i32x8 join(const i32x4 &a, const i32x4 &b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <class F, int... I>
__device__ __forceinline__ void each_of(F &&f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F &&f) {
  each_of(f, std::make_integer_sequence<int, N>());
}
// the matrix instructions of before have written their results to acc
template <int NI, int NJ>
__device__ __forceinline__ void settled(f32x4 (&acc)[NI][NJ]) {
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(acc[i][j]));
  asm volatile("s_nop 15\n\ts_nop 3" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

struct Operand {
  const uint8_t *code, *exp;
  long ld, lde;  // bytes of a row of codes, of a block of columns' bytes
  int rows, square;
};

// N consecutive columns of a row of y, from its sums: whole where the row holds them
// (accesses of any width take any alignment of an element)
template <class T, int N>
__device__ __forceinline__ void store_run(T *d, int left, const float (&v)[N]) {
  if (left >= N) {
    constexpr int W = N < 16 / (int)sizeof(T) ? N : 16 / (int)sizeof(T);  // columns of an access
    static_assert(N % W == 0, "whole accesses");
    typedef T V __attribute__((ext_vector_type(W), aligned(sizeof(T))));
#pragma unroll
    for (int q = 0; q < N / W; ++q) {
      V o;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        if constexpr (sizeof(T) == 2) o[j] = f2bf_bits(v[q * W + j]);
        else o[j] = v[q * W + j];
      }
      *reinterpret_cast<V *>(d + q * W) = o;
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (j < left) store_val(d, j, v[j]);
}

struct Gemm8 {
  Operand a, b;
  void *y;
  long ldy, split_stride;  // elements between rows, and between the partial sums of parts
  int steps, part, splits, tiles;
};

// ------------------------------------------------------------------ many rows
//
// Tiles, waves and schedule are those of the bf16 product (k_gemm of gemm.h): 64 TM x
// 256 a block of 8 waves in two groups half a step apart, 128 bytes of every row a
// step, direct loads to two slots of A and three of B in LDS.  A step of 128 codes
// takes the matrix cores the time of 64 bf16 values.
//
// Rows of a wave tile are dealt to the operand's fragments in turn: row q of fragment i
// of F is row F q + i of the tile (the loads put it there).  So a lane's scales of all
// its fragments are F neighbouring bytes, one load a step, picked by the instruction;
// and a lane ends with 16 consecutive columns of a row, which it stores as they are.
constexpr int STEP = fp8::BLOCK, THREADS = gemm::THREADS;

struct Load8 {
  gemm::gemm_i32x4 rs;
  int voff, joff[8], chunk, bytes, add;

  // F (2, 4 or 8) fragments of 16 rows a wave tile; wave w of the group's four, load j: rows
  // 8 (w + 4 j) .. of the tile in LDS
  __device__ __forceinline__ void init(const uint8_t *code, long ld, int row0, int left, int F, int w, int lane) {
    rs = gemm::gemm_desc(code + (long)row0 * ld, (long)left * ld);
    const int p = 8 * (w & 1) + (lane >> 3);  // row of its fragment
    chunk = ((lane & 7) ^ (p >> 1)) * 16;
    bytes = (int)ld;
    voff = (F * p + (w >> 1)) * (int)ld + chunk;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      joff[j] = (F == 2 ? 32 * j : F == 4 ? 64 * (j / 2) + 2 * (j % 2) : 128 * (j / 4) + 2 * (j % 4)) * (int)ld;
  }
  __device__ __forceinline__ void prep(int k0) { add = k0 + chunk < bytes ? voff + k0 : 0x40000000; }
  __device__ __forceinline__ void load(unsigned dst, int j, int w) const {
    gemm::dma16(dst + (w + 4 * j) * 1024, add + joff[j], rs);
  }
};

// The bytes of F fragments' rows of one step.
template <int F>
struct Scales {
  static constexpr int N = (F + 3) / 4;
  const uint8_t *p;
  long lde;
  int square;
  __device__ __forceinline__ void init(const Operand &o, int row0, int q, int step) {
    square = o.square;
    lde = o.lde;
    // rows past the end: any byte in range, their codes are zeros and their sums unused
    const long at = square ? (row0 < o.rows ? row0 : o.rows - 1) / fp8::BLOCK : min((long)row0 + F * q, o.lde - F);
    p = o.exp + (long)step * lde + at;
  }
  __device__ __forceinline__ void fetch(unsigned (&s)[N]) {
    if (square) {
      s[0] = *p;
    } else if constexpr (N == 2) {
      const uint2 v = *reinterpret_cast<const uint2 *>(p);
      s[0] = v.x;
      s[1] = v.y;
    } else if constexpr (F == 4) {
      s[0] = *reinterpret_cast<const unsigned *>(p);
    } else if constexpr (F == 2) {
      s[0] = *reinterpret_cast<const unsigned short *>(p);
    } else {
      s[0] = *p;
    }
    p += lde;
  }
  // what was fetched, waited for, as four rows' bytes a register
  __device__ __forceinline__ void take(unsigned (&s)[N], unsigned (&to)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(s[i]));
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = square ? s[0] * 0x01010101u : s[i];
  }
};

// What a grid with a block a CU is given instead of a second block: four slots for each
// operand, and the scales of the block's steps in LDS before the first of them.  (A scale
// from memory is waited for with all loads before it, also those of later steps.)
constexpr int DEEP_STEPS = 128;

template <int TM, int BN, bool DEEP, class T>
__global__ void __launch_bounds__(THREADS, BN == 128 && !DEEP ? 4 : 2) k_gemm8(const Gemm8 g) {
  constexpr int BM = gemm::bm_of(TM), SA = BM * STEP, SB = BN * STEP;
  constexpr int SLOTS_A = DEEP ? 4 : gemm::SLOTS_A, SLOTS_B = DEEP ? 4 : gemm::SLOTS_B;
  constexpr int LDS_B = SA * SLOTS_A, LDS_S = LDS_B + SB * SLOTS_B;  // scales: [step][BM + BN]
  __shared__ __attribute__((aligned(1024))) char lds[LDS_S + (DEEP ? DEEP_STEPS * (BM + BN) : 0)];
  int idx = gemm::xcd_index(g.tiles * g.splits);
  if (idx >= g.tiles * g.splits) return;
  const int split = idx / g.tiles;
  idx -= split * g.tiles;
  int mt, nt;
  gemm::tile_of(idx, (g.a.rows + BM - 1) / BM, (g.b.rows + BN - 1) / BN, mt, nt);
  const int m0 = mt * BM, n0 = nt * BN;
  const int lane = threadIdx.x & 63, col = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int grp = wave >> 2, w4 = wave & 3;  // waves w and w + 4 share a SIMD
  const int wr = grp * 32 * TM, wc = w4 * (BN / 4);
  const int s0 = split * g.part, nk = min(g.part, g.steps - s0);

  constexpr int FA = 2 * TM, FB = BN / 64;
  static_assert(BM <= BN, "a group has as many loads of B as of A, or more");
  Load8 ldr;  // the group's operand
  if (grp == 0) ldr.init(g.a.code, g.a.ld, m0, min(BM, g.a.rows - m0), FA, w4, lane);
  else ldr.init(g.b.code, g.b.ld, n0, min(BN, g.b.rows - n0), FB, w4, lane);
  gemm::Frag<false, BM, FA> fA;
  gemm::Frag<false, BN, FB> fB;
  fA.init(0, wr, lane);
  fB.init(LDS_B, wc, lane);
  Scales<FA> ea;
  Scales<FB> eb;
  unsigned sa_next[Scales<FA>::N], sb_next[1], sa[Scales<FA>::N], sb[1];

  f32x4 acc[FA][FB];
#pragma unroll
  for (int i = 0; i < FA; ++i)
#pragma unroll
    for (int j = 0; j < FB; ++j) acc[i][j] = f32x4{};

  const unsigned base = (unsigned)(unsigned long)(__attribute__((address_space(3))) char *)lds;
  const unsigned ring = base + (grp == 0 ? 0 : LDS_B);
  constexpr int LA = BM / 32, LB = BN / 32;  // loads per wave of an A and of a B step
  int k_next = s0 * STEP;
  auto prep = [&]() __attribute__((always_inline)) {
    ldr.prep(k_next);
    k_next += STEP;
  };
  auto load = [&](int slot, int j) __attribute__((always_inline)) {
    if (LA == LB || j < LA || grp == 1) ldr.load(ring + slot, j, w4);
  };
  if (!DEEP && nk > 0) {
    ea.init(g.a, m0 + wr, col, s0);
    eb.init(g.b, n0 + wc, col, s0);
    ea.fetch(sa_next);
    eb.fetch(sb_next);
    ea.take(sa_next, sa);
    eb.take(sb_next, sb);
  }
  // the first SLOTS - 1 steps of the group's operand; the first of them has landed
#pragma unroll
  for (int d = 0; d + 1 < (SLOTS_A > SLOTS_B ? SLOTS_A : SLOTS_B); ++d) {
    if (grp == 0 && d + 1 >= SLOTS_A) continue;
    prep();
#pragma unroll
    for (int j = 0; j < LB; ++j) load(d * (grp == 0 ? SA : SB), j);
  }
  if constexpr (DEEP) {
    for (int i = threadIdx.x; i < nk * ((BM + BN) / 16); i += THREADS) {
      const int step = i / ((BM + BN) / 16), at = i % ((BM + BN) / 16) * 16;
      const Operand &o = at < BM ? g.a : g.b;
      const int row = at < BM ? m0 + at : n0 + at - BM;
      const uint8_t *p = o.exp + (long)(s0 + step) * o.lde;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (o.square) {
        v.x = v.y = v.z = v.w = row < o.rows ? p[row / fp8::BLOCK] * 0x01010101u : 0u;
      } else if (row < o.lde) {
        v = *reinterpret_cast<const uint4 *>(p + row);
      }
      *reinterpret_cast<uint4 *>(lds + LDS_S + step * (BM + BN) + at) = v;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  } else if (grp == 0 || nk <= 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  } else {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LB) : "memory");
  }
  __builtin_amdgcn_s_barrier();
  GEMM_FENCE();
  if (grp == 1 && nk > 0) __builtin_amdgcn_s_barrier();  // half a step behind group 0
  GEMM_FENCE();

  // Barriers and waits are those of k_gemm: before the barrier that opens group 0's reads
  // of step t + 1, both groups have waited for their loads of that step, and those of the
  // SLOTS - 2 steps behind it stay in flight.  The scales of step t + 1 are fetched before
  // the direct loads of step t's phase go out and waited for when its products are issued
  // (DEEP: read with the fragments).
  int slot_a = 0, slot_b = 0, old_a = (SLOTS_A - 1) * SA, old_b = (SLOTS_B - 1) * SB;  // of steps t and t - 1
#pragma unroll 1
  for (int t = 0; t < nk; ++t) {
    const int slot_n = grp == 0 ? old_a : old_b;
    bf16x8 a[2][FA], b[2][FB];
    if constexpr (DEEP) {
      const char *sc = lds + LDS_S + t * (BM + BN);
      static_assert(!DEEP || (FA == 4 && FB == 2), "a word of scales of a, a half of b");
      sa[0] = *reinterpret_cast<const unsigned *>(sc + wr + FA * col);
      sb[0] = *reinterpret_cast<const unsigned short *>(sc + BM + wc + FB * col);
    } else if (t + 1 < nk) {
      ea.fetch(sa_next);
      eb.fetch(sb_next);
    }
    prep();
    constexpr int NR = FA + FB, PER = LB / 2;  // reads and loads per half of a row's bytes
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int f = 0; f < NR; ++f) {
#pragma unroll
        for (int j = f * PER / NR; j < PER; ++j)
          if (j * NR / PER == f) load(slot_n, kk * PER + j);
        if (f < FB) b[kk][f] = fB.read(lds, slot_b, kk, f);
        else a[kk][f - FB] = fA.read(lds, slot_a, kk, f - FB);
      }
    }
    if (grp == 0) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((SLOTS_B - 2) * LB) : "memory");
    __builtin_amdgcn_s_barrier();
    GEMM_FENCE();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
    each<FA>([&](auto i) __attribute__((always_inline)) {
      each<FB>([&](auto jj) __attribute__((always_inline)) {
        constexpr int I = decltype(i)::value, J = (I & 1) ? FB - 1 - decltype(jj)::value : decltype(jj)::value;
        acc[I][J] = mfma8<J, I & 3>(
            join(__builtin_bit_cast(i32x4, b[0][J]), __builtin_bit_cast(i32x4, b[1][J])),
            join(__builtin_bit_cast(i32x4, a[0][I]), __builtin_bit_cast(i32x4, a[1][I])), acc[I][J], sb[0], sa[I / 4]);
      });
    });
    // here and not behind the next barrier, where the compiler would move them (51% of the
    // matrix cores' time, 2,140 TFLOP/s at 8192^3)
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
      for (int j = 0; j < FB; j += 2) asm volatile("" : "+v"(acc[i][j]), "+v"(acc[i][j + 1]));
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    old_a = slot_a;
    old_b = slot_b;
    slot_a = slot_a == (SLOTS_A - 1) * SA ? 0 : slot_a + SA;
    slot_b = slot_b == (SLOTS_B - 1) * SB ? 0 : slot_b + SB;
    if (grp == 0) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((SLOTS_A - 2) * LA) : "memory");
    if (!DEEP && t + 1 < nk) {
      ea.take(sa_next, sa);
      eb.take(sb_next, sb);
    }
    if (grp == 0 || t + 1 < nk) __builtin_amdgcn_s_barrier();
    GEMM_FENCE();
    // behind the barrier, where the other group's products are under way: 777 x 5,001 x 2,040
    // 19.3 -> 19.8 us, 1,500 x 18,944 x 3,584 85.6 -> 86.1, 8,192^3 386 -> 387
    settled(acc);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the block
  const int n = n0 + wc + 4 * FB * lg;
  if (n >= g.b.rows) return;
  T *y = static_cast<T *>(g.y) + (long)split * g.split_stride;
#pragma unroll
  for (int i = 0; i < FA; ++i) {
    const int m = m0 + wr + FA * col + i;
    if (m >= g.a.rows) continue;
    float v[4 * FB];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < FB; ++j) v[FB * r + j] = acc[i][j][r];
    // (partial sums: rows are filled up to 16)
    store_run(y + (long)m * g.ldy + n, g.splits > 1 ? 4 * FB : g.b.rows - n, v);
  }
}

// Sums the parts in order: 8 columns of a row a thread.
template <class T>
__global__ void __launch_bounds__(256) k_finish8(const float *__restrict__ part, int parts, long stride, long ldp, int M,
                                                 int N, T *__restrict__ y, long ldy) {
  const unsigned n8 = (unsigned)(ldp / 8);
  const long total = (long)M * n8;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long)gridDim.x * 256) {
    const long m = i / n8;
    const int n = (int)(i - m * n8) * 8;
    if (n >= N) continue;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < parts; ++k) {
      const f32x4 *p = reinterpret_cast<const f32x4 *>(part + k * stride + m * ldp + n);
      const f32x4 a = p[0], b = p[1];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] += a[j];
        v[4 + j] += b[j];
      }
    }
    store_run(y + m * ldy + n, N - n, v);
  }
}

// ------------------------------------------------------------------ few rows
//
// Up to 16 NB rows of a, where the bytes of b are the work (k_glu_rows of the gated
// block, in 8 bits): a block takes 16 CB rows of b, its waves every WAVES-th step, and
// their sums are added up in LDS, in order.  Memory gives the codes fastest in whole
// 128-byte lines, which is not the instruction's operand, so a lane's 16 bytes go
// through the wave's own piece of LDS (chunk c of row r in slot c ^ (r & 7)), while the
// loads of the wave's next DEPTH steps are under way; no wave waits for another.  Rows of
// b past the end read the last one, and their sums go nowhere; rows of a past the end are
// not read, and codes past a row's end read as zeros.
template <int NB, int CB, int WAVES, int DEPTH, int OCC, class T>
__global__ void __launch_bounds__(64 * WAVES, OCC) k_few8(const Gemm8 g) {
  constexpr int ROWS = 16 * (CB > NB ? CB : NB), STAGE = WAVES * ROWS * 8, SUMS = WAVES * CB * NB * 64;
  __shared__ __attribute__((aligned(1024))) f32x4 lds[STAGE > SUMS ? STAGE : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, lg = lane >> 4, lr = lane >> 3, lc = lane & 7;
  const int n0 = blockIdx.x * 16 * CB, ld = (int)g.b.ld;
  // row p of a piece is row CB (p % 16) + p / 16 of b's (NB of a's): see k_gemm8
  const uint8_t *bp = g.b.code + (long)n0 * ld;
  unsigned boff[2 * CB], aoff[2 * NB];
  bool ain[2 * NB];
#pragma unroll
  for (int i = 0; i < 2 * CB; ++i) {
    const int p = 8 * i + lr;
    boff[i] = (unsigned)min(CB * (p & 15) + (p >> 4), g.b.rows - 1 - n0) * (unsigned)ld + 16 * lc;
  }
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i) {
    const int p = 8 * i + lr;
    const int row = NB * (p & 15) + (p >> 4);
    ain[i] = row < g.a.rows;
    aoff[i] = (unsigned)row * (unsigned)ld + 16 * lc;
  }
  struct Set {  // a step of the wave
    i32x4 w[2 * CB], x[2 * NB];
    unsigned sw[1], sx[1];
  };
  Scales<CB> eb;
  Scales<NB> ea;
  eb.init(g.b, n0, r, wave);
  ea.init(g.a, 0, r, wave);
  eb.lde *= WAVES;
  ea.lde *= WAVES;
  auto load = [&](Set &t, int s) __attribute__((always_inline)) {
    const int k = s * STEP;
    const bool in = k + 16 * lc < ld;
#pragma unroll
    for (int i = 0; i < 2 * CB; ++i)
      t.w[i] = in ? __builtin_nontemporal_load(reinterpret_cast<const i32x4 *>(bp + k + boff[i])) : i32x4{};
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i)
      t.x[i] = in && ain[i] ? *reinterpret_cast<const i32x4 *>(g.a.code + k + aoff[i]) : i32x4{};
    t.sw[0] = t.sx[0] = 0;
    if (s < g.steps) {
      eb.fetch(t.sw);
      ea.fetch(t.sx);
    }
  };
  f32x4 acc[CB][NB];
#pragma unroll
  for (int b = 0; b < CB; ++b)
#pragma unroll
    for (int n = 0; n < NB; ++n) acc[b][n] = f32x4{};
  i32x4 *stage = reinterpret_cast<i32x4 *>(lds) + wave * (ROWS * 8);
  i32x4 *to = stage + lr * 8 + (lc ^ lr);
  const i32x4 *from = stage + r * 8;
  const int c0 = lg ^ (r & 7), c1 = (4 + lg) ^ (r & 7);
  // the products of a step, and the loads of the wave's step `next` in its place
  auto step = [&](Set &t, int next) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) to[64 * i] = t.x[i];
    __builtin_amdgcn_wave_barrier();
    i32x8 cx[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) cx[n] = join(from[n * 128 + c0], from[n * 128 + c1]);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 2 * CB; ++i) to[64 * i] = t.w[i];
    __builtin_amdgcn_wave_barrier();
    const unsigned sw = eb.square ? t.sw[0] * 0x01010101u : t.sw[0], sx = ea.square ? t.sx[0] * 0x01010101u : t.sx[0];
    load(t, next);
    each<CB>([&](auto b) __attribute__((always_inline)) {
      constexpr int B = decltype(b)::value;
      const i32x8 cw = join(from[B * 128 + c0], from[B * 128 + c1]);
      each<NB>([&](auto n) __attribute__((always_inline)) {
        constexpr int N = decltype(n)::value;
        acc[B][N] = mfma8<B, N>(cw, cx[N], acc[B][N], sw, sx);
      });
    });
    settled(acc);
    __builtin_amdgcn_wave_barrier();
  };
  Set t[DEPTH];
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) load(t[d], wave + d * WAVES);
  for (int s = wave; s < g.steps; s += WAVES * DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (d == 0 || s + d * WAVES < g.steps) step(t[d], s + (d + DEPTH) * WAVES);
  }
  f32x4(*sums)[CB * NB][64] = reinterpret_cast<f32x4(*)[CB * NB][64]>(lds);
  __syncthreads();
#pragma unroll
  for (int b = 0; b < CB; ++b)
#pragma unroll
    for (int n = 0; n < NB; ++n) sums[wave][b * NB + n][lane] = acc[b][n];
  __syncthreads();
  if (wave >= NB) return;
  f32x4 v[CB];
#pragma unroll
  for (int b = 0; b < CB; ++b) v[b] = sums[0][b * NB + wave][lane];
#pragma unroll 1
  for (int q = 1; q < WAVES; ++q)
#pragma unroll
    for (int b = 0; b < CB; ++b) v[b] += sums[q][b * NB + wave][lane];
  const int m = NB * r + wave, n = n0 + 4 * CB * lg;
  if (m >= g.a.rows || n >= g.b.rows) return;
  float o[4 * CB];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int b = 0; b < CB; ++b) o[CB * q + b] = v[b][q];
  store_run(static_cast<T *>(g.y) + (long)m * g.ldy + n, g.b.rows - n, o);
}

constexpr int FEW = 64;  // rows that k_few8 takes at most

// Partial sums: rows of `outs` filled up to 16.
long ld_part(int outs) { return (outs + 15) / 16 * 16; }
bool sizes_ok(int32_t rows, int32_t outs, int32_t cols) {
  return rows >= 0 && outs >= 1 && cols >= 1 && rows <= (1 << 20) && outs <= (1 << 20) && cols <= (1 << 20);
}
// 256 x 256, 128 x 256, 128 x 128 with two blocks a CU, or with one (DEEP)
enum Tiles { WIDE, HALF, TWO, ONE };
struct Choice {
  Tiles tiles;
  int parts, part;
};
long tiles_of(int rows, int outs, Tiles v) {
  const long bm = v == WIDE ? 256 : 128, bn = v == WIDE || v == HALF ? 256 : 128;
  return (rows + bm - 1) / bm * ((outs + bn - 1) / bn);
}

// How a product is launched, by the time that each way is expected to take: us of blocks
// that fill u of the chip's CUs, by steps s of 128 columns; a full chip's clocks are lower.
//   256 x 256 tiles: 6 + s (1.06 + 0.49 u) a round;  128 x 256: 4 + s (0.8 + 0.3 u);
//   128 x 128, two of them on a CU: 4 + s (0.6 + 0.1 u) for the first 256, another s (0.25 +
//   0.2 u) with the second; DEEP, for one round alone: 4 + s (0.52 + 0.12 u);
// and for parts of K their fp32 sums, 4.5 + 0.3 a MB.  Measured, us, rows x outs x cols (parts
// of K in brackets), 256 x 256 tiles / 128 x 256 / 128 x 128 / DEEP, the one taken first:
//   128 x 18,944 x 3,584     DEEP 26.2; 41.6 / 40.4 / 30.5
//   256 x 3,584 x 18,944     DEEP (4) 37.2; (8) 48.9 / (8) 43.5 / (8) 41.6
//   512 x 5,504 x 2,048      DEEP 14.0; 24.8 / 18.3 / 14.9
//   1,024 x 5,504 x 2,048    128 x 128 20.0; 25.7 / 20.3 / - / 25.6
//   1,500 x 5,001 x 2,040    128 x 256 22.9; 29.0 / - / 23.5 / 28.4
//   1,500 x 18,944 x 3,584   256 x 256 97.4; - / 128 / 128 / 140
// (The wait at the end of the loop came later: it adds 0.2 to 0.6 us to each but DEEP.  8,192 x
// 18,944 x 3,584 in two launches, nine rounds and the rest in quarters of tiles: 478, in one 470.)
double expect(int v, long blocks, double s) {
  const long slots = v == TWO ? 512 : 256, full = blocks / slots, rest = blocks % slots;
  auto round = [&](double n) {  // n blocks, at most the slots
    const double u = std::min(n, 256.0) / 256, second = std::max(n - 256, 0.0) / 256;
    return v == WIDE ? 6 + s * (1.06 + 0.49 * u)
         : v == HALF ? 4 + s * (0.8 + 0.3 * u)
         : v == TWO ? 4 + s * (0.6 + 0.1 * u + (second > 0 ? 0.25 + 0.2 * second : 0))
                    : 4 + s * (0.52 + 0.12 * u);
  };
  return full * round((double)slots) + (rest ? round((double)rest) : 0.0);
}

Choice choice_of(int rows, int outs, int cols) {
  const int steps = (int)fp8::blocks_of(cols);
  const double mb = (double)rows * ld_part(outs) * 4e-6;
  Choice best{};
  double best_us = 0;
  for (Tiles v : {WIDE, HALF, TWO, ONE}) {
    const long tiles = tiles_of(rows, outs, v);
    for (int p = 1; p <= 16; ++p) {
      const int per = (steps + p - 1) / p;
      if (p > 1 && (per < 2 || (p - 1) * per >= steps || tiles * p > 2048)) continue;
      if (v == ONE && (tiles * p > 256 || per > DEEP_STEPS)) continue;
      const double us = expect(v, tiles * p, per) + (p > 1 ? 4.5 + 0.3 * mb * p : 0.0);
      if (best_us == 0 || us < best_us) {
        best = Choice{v, p, per};
        best_us = us;
      }
    }
  }
  return best;
}

template <int NB, int CB, int WAVES, int DEPTH, int OCC, class T>
void few_as(const Gemm8 &g, hipStream_t st) {
  k_few8<NB, CB, WAVES, DEPTH, OCC, T><<<(unsigned)((g.b.rows + 16 * CB - 1) / (16 * CB)), 64 * WAVES, 0, st>>>(g);
  SEG_LAUNCH_CHECK();
}

// Above 32 rows many of b's bytes are better read by tiles, or as well: us, rows x outs x
// cols, this way / by tiles, 64 x 4,096 x 4,096 9.5 / 15.0; 64 x 8,192 x 8,192 19.7 / 19.5; 64 x
// 3,584 x 18,944 31.9 / 21.3; 64 x 18,944 x 3,584 23.8 / 19.0, 40 rows 22.3 / 18.7; the rule loses
// a little only where there are very many outs: 64 x 151,936 x 3,584 121.1 / 122.5, 48 rows
// 113 / 119.
bool is_few(int rows, int outs, int cols) {
  return rows <= FEW / 2 || (rows <= FEW && (double)outs * cols < (1 << 25));
}

struct Few {
  int nb, cb, waves;
};
// Narrow blocks where there are few of them (each CU then has more waves on its rows of b),
// wide ones, which read a less often, where there are many.  Measured, us, rows x outs x
// cols, the kernel taken / another: 1 x 18,944 x 3,584 12.9 / 14.2 (16 waves), 16.7 (32 rows
// of b a block, one step ahead); 1 x 3,584 x 18,944 13.2 / 15.5 (8 waves, two steps ahead); 24
// x 18,944 x 3,584 17.1 / 20.4 (16 rows of b); 24 x 3,584 x 18,944 23.5 / 26.4 (32 rows); 64
// x 3,584 x 3,584 8.7 / 9.8 (32 rows); 64 x 5,504 x 2,048 7.6 / 10.0 (64 rows).
Few few_choice(int rows, int outs, int cols) {
  if (rows <= 16) return {1, 1, outs <= 16 * 256 && cols > 16 * STEP ? 16 : 8};
  if (rows <= 32) return outs <= 32 * 128 ? Few{2, 1, 8} : Few{2, 2, 4};
  return outs <= 32 * 128 ? Few{4, 1, 8} : outs <= 32 * 512 ? Few{4, 2, 8} : Few{4, 4, 4};
}

template <class T>
void few(const Gemm8 &g, const Few &f, hipStream_t st) {
  if (f.nb == 1) {
    if (f.waves == 16) few_as<1, 1, 16, 1, 4, T>(g, st);
    else few_as<1, 1, 8, 2, 4, T>(g, st);
  } else if (f.nb == 2) {
    if (f.cb == 1) few_as<2, 1, 8, 2, 4, T>(g, st);
    else few_as<2, 2, 4, 2, 2, T>(g, st);
  } else if (f.cb == 1) {
    few_as<4, 1, 8, 1, 2, T>(g, st);
  } else if (f.cb == 2) {
    few_as<4, 2, 8, 1, 2, T>(g, st);
  } else {
    few_as<4, 4, 4, 1, 2, T>(g, st);
  }
}

template <class T>
void many(Gemm8 g, const Choice &c, hipStream_t st) {
  g.tiles = (int)tiles_of(g.a.rows, g.b.rows, c.tiles);
  const unsigned grid = (unsigned)(((long)g.tiles * g.splits + 7) / 8 * 8);
  switch (c.tiles) {
    case WIDE: k_gemm8<4, 256, false, T><<<grid, THREADS, 0, st>>>(g); break;
    case HALF: k_gemm8<2, 256, false, T><<<grid, THREADS, 0, st>>>(g); break;
    case TWO: k_gemm8<2, 128, false, T><<<grid, THREADS, 0, st>>>(g); break;
    case ONE: k_gemm8<2, 128, true, T><<<grid, THREADS, 0, st>>>(g); break;
  }
  SEG_LAUNCH_CHECK();
}

}  // namespace
}  // namespace seg

using namespace seg;

// How a product is launched (for tests): out = {Tiles, 0, parts of K}, or for few rows
// {16-row blocks of a, of b, - waves}.
extern "C" void seg_fp8_gemm_choice(int32_t rows, int32_t outs, int32_t cols, int32_t *out) {
  if (is_few(rows, outs, cols)) {
    const Few f = few_choice(rows, outs, cols);
    out[0] = f.nb;
    out[1] = f.cb;
    out[2] = -f.waves;
    return;
  }
  const Choice c = choice_of(rows, outs, cols);
  out[0] = c.tiles;
  out[1] = 0;
  out[2] = c.parts;
}

extern "C" size_t seg_fp8_gemm_workspace_bytes(int32_t rows, int32_t outs, int32_t cols) {
  if (!sizes_ok(rows, outs, cols) || is_few(rows, outs, cols)) return 0;
  const Choice c = choice_of(rows, outs, cols);
  return c.parts > 1 ? align_up((size_t)c.parts * rows * ld_part(outs) * 4) : 0;
}

extern "C" seg_status seg_fp8_gemm(int32_t rows, int32_t outs, int32_t cols, const seg_fp8 *a, const seg_fp8 *b,
                                   seg_dtype dt, void *y, int64_t ldy, void *ws, size_t ws_bytes,
                                   hipStream_t stream) {
  return guarded([&] {
    SEG_CHECK(dt == SEG_BF16 || dt == SEG_F32, SEG_ERR_UNSUPPORTED, "dtype %d not supported", (int)dt);
    SEG_CHECK(rows >= 0 && outs >= 1 && cols >= 1, SEG_ERR_ARG, "bad sizes rows=%d outs=%d cols=%d", rows, outs, cols);
    SEG_CHECK(sizes_ok(rows, outs, cols), SEG_ERR_CAPACITY, "rows %d, outs %d or cols %d above 2^20", rows, outs, cols);
    SEG_CHECK(ldy >= outs && ldy < (1LL << 40), SEG_ERR_ARG, "row stride %lld of y for %d columns", (long long)ldy, outs);
    if (rows == 0) return;
    fp8::check(a, "a");
    fp8::check(b, "b");
    const size_t need = seg_fp8_gemm_workspace_bytes(rows, outs, cols), e = dt == SEG_BF16 ? 2 : 4;
    SEG_CHECK(ws_bytes >= need, SEG_ERR_WORKSPACE, "workspace of %zu bytes < required %zu", ws_bytes, need);
    SEG_CHECK(y && (ws || need == 0), SEG_ERR_ARG, "y or the workspace is NULL");
    SEG_CHECK(reinterpret_cast<uintptr_t>(y) % e == 0, SEG_ERR_ARG, "y is not aligned to its type");
    SEG_CHECK(need == 0 || reinterpret_cast<uintptr_t>(ws) % 16 == 0, SEG_ERR_UNSUPPORTED,
              "the workspace is not on a 16-byte boundary");
    check_apart({{y, ((size_t)(rows - 1) * ldy + outs) * e}, {need ? ws : nullptr, need}},
                {{a->code, fp8::code_bytes(rows, cols)}, {a->exp, fp8::exp_bytes(rows, cols, a->block_rows)},
                 {b->code, fp8::code_bytes(outs, cols)}, {b->exp, fp8::exp_bytes(outs, cols, b->block_rows)}});
    auto operand = [&](const seg_fp8 *p, int n) {
      return Operand{p->code, p->exp, fp8::ld_code(cols), fp8::ld_exp(n, p->block_rows), n, p->block_rows != 1};
    };
    Gemm8 g{operand(a, rows), operand(b, outs), y, ldy, 0, (int)fp8::blocks_of(cols), (int)fp8::blocks_of(cols), 1, 0};
    ProfScope prof("fp8_gemm", stream);
    if (is_few(rows, outs, cols)) {
      const Few f = few_choice(rows, outs, cols);
      if (dt == SEG_BF16) few<unsigned short>(g, f, stream);
      else few<float>(g, f, stream);
      return;
    }
    const Choice c = choice_of(rows, outs, cols);
    if (c.parts == 1) {
      if (dt == SEG_BF16) many<unsigned short>(g, c, stream);
      else many<float>(g, c, stream);
      return;
    }
    g.y = ws;
    g.ldy = ld_part(outs);
    g.split_stride = (long)rows * g.ldy;
    g.splits = c.parts;
    g.part = c.part;
    many<float>(g, c, stream);
    const unsigned grid = (unsigned)std::min<long>(8192, ((long)rows * g.ldy / 8 + 255) / 256);
    if (dt == SEG_BF16)
      k_finish8<<<grid, 256, 0, stream>>>(static_cast<const float *>(ws), c.parts, g.split_stride, g.ldy, rows, outs,
                                          static_cast<unsigned short *>(y), ldy);
    else
      k_finish8<<<grid, 256, 0, stream>>>(static_cast<const float *>(ws), c.parts, g.split_stride, g.ldy, rows, outs,
                                          static_cast<float *>(y), ldy);
    SEG_LAUNCH_CHECK();
  });
}
