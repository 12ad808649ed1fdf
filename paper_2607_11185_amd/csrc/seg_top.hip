// The k largest logits of each row, with their columns, and the row's log-sum-exp.
//
// Order: by value, descending, then by column, ascending; NaN counts as larger than
// all numbers, -0 as 0.  Two steps:
//
//   scan   one pass over the logits: running maximum and sum of the softmax, and the
//          largest of every 64 columns (a group) as a whole number in order;
//   pick   of each row: the k largest groups (ties: the first ones), and of their columns
//          the k largest;
//
// as two kernels over parts of rows and over rows (k_top_scan, k_top_pick) or as one over
// rows (k_top_row).  Small vocabularies take one step without groups (k_top_small).
//
// The k largest logits lie in the k largest groups: a column outside them is preceded
// by the largest of each of those groups, which is larger, or as large and further to
// the front, as the groups are runs of columns.  So the second step reads k groups
// again and not the row, and no order of the values makes it do more.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "act8.h"
#include "common.h"
#include "fp8.h"

namespace seg {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float FAR = 3.4028234663852886e38f;
constexpr int GROUP = 64;    // columns
constexpr int MAX_K = 256;
constexpr int SPAN = 16384;  // columns of a block of the scan, at most

template <class T>
struct Piece;
template <>
struct Piece<unsigned short> {
  typedef unsigned short X __attribute__((ext_vector_type(8), aligned(2)));
};
template <>
struct Piece<float> {
  typedef float X __attribute__((ext_vector_type(8), aligned(4)));
};
template <class T>
__device__ __forceinline__ float value(T v) {
  if constexpr (sizeof(T) == 2) return bf_bits2f(v);
  else return v;
}

// Whole numbers in the order of the values: NaN first, zeros alike; 16 bits for bf16, whose
// thresholds then take one pass less.  No value has 0.
template <class T>
__device__ __forceinline__ unsigned order(float x) {
  unsigned u = __builtin_bit_cast(unsigned, x);
  if (x == 0.f) u = 0;
  u ^= (unsigned)((int)u >> 31) | 0x80000000u;
  if (x != x) u = 0xffffffffu;
  return sizeof(T) == 2 ? u >> 16 : u;
}

struct TopArgs {
  const void *z;
  long ldz;
  int rows, vocab, k, groups, parts, span;
  float scale;
  unsigned *gmax;   // [rows][groups]
  float2 *stats;    // [rows][parts]: maximum of a part, and sum of the exponentials below it
  int32_t *ids;
  float *logits, *lse;
};

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

// maximum and sum of the exponentials of two parts
__device__ __forceinline__ float2 meet(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  return make_float2(m, a.y * exp_of(a.x - m) + b.y * exp_of(b.x - m));
}

// A block takes `span` columns of a row, a lane 8 neighbouring ones at a time, so 8
// lanes a group.  The reference in front of the sum is the largest value so far, kept
// inside fp32's numbers, so that infinities meet no infinity: -inf adds 0, inf gives inf,
// NaN stays NaN.  Bound by the vector units and HBM about alike (7,680 x 151,936 bf16): nine
// issue slots an element, four of them the exponential; whole numbers are formed of a
// lane's largest value only, and NaN looked for two values at a time.
template <class T, bool STREAM>
__device__ __forceinline__ float2 scan(const TopArgs &a, const T *__restrict__ z, int c0, int c1, unsigned *gmax,
                                       float2 (&red)[4]) {
  float2 s = make_float2(-FAR, 0.f);
  // U pieces of 2,048 columns; WHOLE: all of them are there
  auto step = [&](int first, auto pieces, auto whole) __attribute__((always_inline)) {
    constexpr int U = decltype(pieces)::value;
    constexpr bool WHOLE = decltype(whole)::value;
    const int c = first + threadIdx.x * 8;
    typename Piece<T>::X v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = c + 2048 * u;
      if (WHOLE || at + 8 <= c1) {
        const typename Piece<T>::X *p = reinterpret_cast<const typename Piece<T>::X *>(z + at);
        v[u] = STREAM ? __builtin_nontemporal_load(p) : *p;
      } else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] = at + j < c1 ? z[at + j] : T();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = c + 2048 * u;
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = value<T>(v[u][j]);
      auto in = [&](int j) { return WHOLE || at + j < c1; };
      float most = -INFINITY, m;
      bool nan = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) most = in(j) ? fmaxf(most, x[j]) : most;
#pragma unroll
      for (int j = 0; j < 8; j += 2) nan = nan || __builtin_isunordered(x[j], x[j + 1]);
      if (a.scale >= 0.f) {
        m = most * a.scale;
      } else {
        float least = INFINITY;
#pragma unroll
        for (int j = 0; j < 8; ++j) least = in(j) ? fminf(least, x[j]) : least;
        m = least * a.scale;
      }
      m = fminf(fmaxf(s.x, m), FAR);
      s.y *= exp_of(s.x - m);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = exp_of(fmaf(x[j], a.scale, -m));
        s.y += in(j) ? e : 0.f;
      }
      s.x = m;
      const unsigned top = act8::max8(WHOLE || at < c1 ? order<T>(nan ? __builtin_nanf("") : most) : 0u);
      if ((threadIdx.x & 7) == 0 && (WHOLE || at < c1)) gmax[at / GROUP] = top;
    }
  };
  int first = c0;
  typedef std::integral_constant<int, 4> Four;
  typedef std::integral_constant<int, 1> One;
  for (; first + 4 * 2048 <= c1; first += 4 * 2048) step(first, Four(), std::true_type());
  if (first + 2048 < c1) step(first, Four(), std::false_type());
  else if (first < c1) step(first, One(), std::false_type());
#pragma unroll
  for (int o = 1; o < 64; o *= 2) s = meet(s, make_float2(__shfl_xor(s.x, o, 64), __shfl_xor(s.y, o, 64)));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  return meet(meet(red[0], red[1]), meet(red[2], red[3]));
}

template <class T>
__global__ void __launch_bounds__(256) k_top_scan(const TopArgs a) {
  __shared__ float2 red[4];
  const int row = blockIdx.x / (unsigned)a.parts, part = blockIdx.x - row * (unsigned)a.parts;
  const int c0 = part * a.span;
  const float2 s = scan<T, false>(a, static_cast<const T *>(a.z) + (long)row * a.ldz, c0, min(a.vocab, c0 + a.span),
                                  a.gmax + (long)row * a.groups, red);
  if (threadIdx.x == 0) a.stats[(long)row * a.parts + part] = s;
}

typedef unsigned long long u64;

// What a block's threads share to find a threshold.
struct Pick {
  __attribute__((aligned(16))) unsigned hist[256];
  unsigned least, most, own, digit, want, done;
};

// The threshold t such that exactly `want` (at least 1, at most all) of the numbers of the
// block are >= t, or, where that cuts equal ones, the number t that is cut, with how many of
// the equal ones are wanted.  each(f) calls f(number) for every one of the thread.  The
// numbers between the least and the most that may still be t are counted in up to 256 equal
// ranges, and the range that holds t is the next to be cut: two or three times for values of
// one size, four at most (digits of the bits from the top down would meet values of one
// exponent in one or two counters first).  Counters that many threads meet in are what a
// pass costs, so it starts from a bound that leaves most numbers out.
struct Cut {
  unsigned t, want;  // want: of the numbers equal to t; 0: all that are >= t
};
__device__ __forceinline__ unsigned max_wave(unsigned x) { return act8::max_groups(fp8::max16(x)); }

template <int THREADS, class K>
__device__ __forceinline__ Cut threshold(K &&each, unsigned want, Pick &p) {
  unsigned lo = 0xffffffffu, hi = 0;
  each([&](unsigned x) {
    lo = min(lo, x);
    hi = max(hi, x);
  });
  const unsigned own = ~max_wave(~hi);  // of the threads' largest (0 where one has none), the smallest
  lo = ~max_wave(~lo);
  hi = max_wave(hi);
  if (threadIdx.x == 0) {
    p.least = p.own = 0xffffffffu;
    p.most = 0;
  }
  if (threadIdx.x < 256) p.hist[threadIdx.x] = 0;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    atomicMin(&p.least, lo);
    atomicMin(&p.own, own);
    atomicMax(&p.most, hi);
  }
  __syncthreads();
  lo = p.least;
  hi = p.most;
  // as many numbers as threads are at least the smallest of the threads' largest
  if (want <= THREADS && p.own > 0) lo = p.own;
  if (lo >= hi) __syncthreads();  // all have read these before another search of the block writes them
  while (lo < hi) {
    const int shift = max(0, 24 - (int)__builtin_clz(hi - lo));  // (hi - lo) >> shift is at most 255
    each([&](unsigned x) {
      if (x >= lo && x <= hi) atomicAdd(&p.hist[(x - lo) >> shift], 1u);
    });
    __syncthreads();
    if (threadIdx.x < 64) {  // four counters a lane, those of the largest numbers in lane 0
      uint4 *h = reinterpret_cast<uint4 *>(p.hist) + (63 - threadIdx.x);
      const uint4 c = *h;
      *h = make_uint4(0, 0, 0, 0);
      unsigned above = c.x + c.y + c.z + c.w;  // with all above them
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const unsigned t = __shfl_up(above, o, 64);
        if ((int)threadIdx.x >= o) above += t;
      }
      const unsigned n[5] = {above - (c.x + c.y + c.z + c.w), above - (c.x + c.y + c.z), above - (c.x + c.y), above - c.x, above};
#pragma unroll
      for (int j = 0; j < 4; ++j)  // counter 3 - j: n[j] numbers above it, n[j + 1] with it
        if (n[j] < want && n[j + 1] >= want) {
          p.digit = 4 * (63 - threadIdx.x) + 3 - j;
          p.want = want - n[j];
          p.done = n[j + 1] == want;
        }
    }
    __syncthreads();
    lo += p.digit << shift;
    hi = lo + min(hi - lo, (1u << shift) - 1);
    want = p.want;
    if (p.done) return Cut{lo, 0};
  }
  return Cut{lo, want};
}

// The selection from the groups' numbers, `key` of group threadIdx.x + THREADS i.  They, and
// every pass over them, stay in registers: from memory a pass cost a latency (7,680 rows,
// k = 64: 212 us).
constexpr int CANDS = 1024, PER = 16, COLS = 8;

struct Pool {
  Pick pick;
  u64 cand[CANDS];
  int group[MAX_K];
  unsigned count, low;
};

// The first k of n candidates to their places: each counts those in front of it.
template <class T, int THREADS>
__device__ __forceinline__ void place(const TopArgs &a, int row, const T *__restrict__ z, const u64 (&cand)[CANDS], int n) {
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const u64 own = cand[i];
    const int c = (int)~(unsigned)own;
    const T v = z[c];
    int at = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) at += cand[j] > own;
    if (at < a.k) {
      a.ids[(long)row * a.k + at] = c;
      a.logits[(long)row * a.k + at] = value<T>(v);
    }
  }
}

template <class T, int THREADS>
__device__ __forceinline__ void pick_row(const TopArgs &a, int row, const T *__restrict__ z, const unsigned (&key)[PER],
                                         Pool &p) {
  Pick &pick = p.pick;
  u64(&cand)[CANDS] = p.cand;
  int(&group)[MAX_K] = p.group;
  unsigned &count = p.count, &low = p.low;
  if (threadIdx.x == 0) {
    count = 0;
    low = 0xffffffffu;
  }
  __syncthreads();
  // the groups: by value, then the first ones
  const int ng = min(a.k, a.groups);
  auto groups = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (key[i]) f(key[i], threadIdx.x + THREADS * i);
  };
  Cut c{0, 0}, ci{0, 0};
  if (ng < a.groups) {
    c = threshold<THREADS>([&](auto f) __attribute__((always_inline)) { groups([&](unsigned x, int) { f(x); }); }, ng, pick);
    if (c.want)
      ci = threshold<THREADS>(
          [&](auto f) __attribute__((always_inline)) { groups([&](unsigned x, int g) { if (x == c.t) f(~(unsigned)g); }); }, c.want, pick);
  }
  groups([&](unsigned x, int g) {
    if (x > c.t || (x == c.t && (!c.want || ~(unsigned)g >= ci.t))) {
      group[atomicAdd(&count, 1u)] = g;
      atomicMin(&low, x);
    }
  });
  __syncthreads();
  // their columns that are as large as the smallest of these groups' largest (k of them
  // are, unless all groups were taken)
  const unsigned least = ng < a.groups ? low : 0u;
  __syncthreads();
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  // 8 columns a piece, 8 pieces a group
  auto columns = [&](auto f) __attribute__((always_inline)) {
    for (int i = threadIdx.x; i < ng * (GROUP / COLS); i += THREADS) {
      const int c0 = group[i / (GROUP / COLS)] * GROUP + i % (GROUP / COLS) * COLS;
      typename Piece<T>::X v{};
      if (c0 + COLS <= a.vocab) v = *reinterpret_cast<const typename Piece<T>::X *>(z + c0);
      else
#pragma unroll
        for (int j = 0; j < COLS; ++j)
          if (c0 + j < a.vocab) v[j] = z[c0 + j];
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        const unsigned o = order<T>(value<T>(v[j]));
        if (c0 + j < a.vocab && o >= least) f(o, c0 + j);
      }
    }
  };
  columns([&](unsigned x, int at) {
    const unsigned n = atomicAdd(&count, 1u);
    if (n < CANDS) cand[n] = (u64)x << 32 | (unsigned)~at;
  });
  __syncthreads();
  int n = (int)count;
  if (n > CANDS) {  // many of the same value: the k first by a threshold of their own
    __syncthreads();
    const Cut t = threshold<THREADS>([&](auto f) __attribute__((always_inline)) { columns([&](unsigned x, int) { f(x); }); }, a.k, pick);
    Cut ti{0, 0};
    if (t.want)
      ti = threshold<THREADS>(
          [&](auto f) __attribute__((always_inline)) { columns([&](unsigned x, int at) { if (x == t.t) f(~(unsigned)at); }); }, t.want, pick);
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    columns([&](unsigned x, int at) {
      if (x > t.t || (x == t.t && (!t.want || ~(unsigned)at >= ti.t)))
        cand[atomicAdd(&count, 1u)] = (u64)x << 32 | (unsigned)~at;
    });
    __syncthreads();
    n = a.k;
  }
  place<T, THREADS>(a, row, z, cand, n);
}

// A block a row, behind the scan.
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS) k_top_pick(const TopArgs a) {
  __shared__ Pool pool;
  const int row = blockIdx.x;
  const unsigned *gm = a.gmax + (long)row * a.groups;
  unsigned key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int g = threadIdx.x + THREADS * i;
    key[i] = g < a.groups ? gm[g] : 0;  // (0 is below every value's number)
  }
  if (threadIdx.x < 64) {  // the parts' sums, each lane's in order and then the lanes'
    float2 s = make_float2(-FAR, 0.f);
    for (int i = threadIdx.x; i < a.parts; i += 64) s = meet(s, a.stats[(long)row * a.parts + i]);
#pragma unroll
    for (int o = 1; o < 64; o *= 2) s = meet(s, make_float2(__shfl_xor(s.x, o, 64), __shfl_xor(s.y, o, 64)));
    if (threadIdx.x == 0) a.lse[row] = s.x + log2f(s.y) * LN2;
  }
  pick_row<T, THREADS>(a, row, static_cast<const T *>(a.z) + (long)row * a.ldz, key, pool);
}

// Both for a row, a block each: with many rows some blocks select while others read.
template <class T, bool STREAM>
__global__ void __launch_bounds__(256) k_top_row(const TopArgs a) {
  __shared__ Pool pool;
  __shared__ float2 red[4];
  extern __shared__ unsigned gmax[];
  const int row = blockIdx.x;
  const T *z = static_cast<const T *>(a.z) + (long)row * a.ldz;
  const float2 s = scan<T, STREAM>(a, z, 0, a.vocab, gmax, red);
  if (threadIdx.x == 0) a.lse[row] = s.x + log2f(s.y) * LN2;
  unsigned key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int g = threadIdx.x + 256 * i;
    key[i] = g < a.groups ? gmax[g] : 0;
  }
  pick_row<T, 256>(a, row, z, key, pool);
}

// Up to 16 THREADS columns, a block a row: the columns themselves stay in registers, without
// groups (where k is near their number nearly all columns would be read again and sorted
// out a second time).
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS) k_top_small(const TopArgs a) {
  __shared__ Pool p;
  __shared__ float2 red[THREADS / 64];
  const int row = blockIdx.x;
  const T *z = static_cast<const T *>(a.z) + (long)row * a.ldz;
  T v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = threadIdx.x + THREADS * i;
    v[i] = at < a.vocab ? z[at] : T();
  }
  unsigned key[PER];
  float y[PER];
  float2 s = make_float2(-FAR, 0.f);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool in = threadIdx.x + THREADS * i < a.vocab;
    key[i] = in ? order<T>(value<T>(v[i])) : 0;  // (0 is below every value's number)
    y[i] = in ? value<T>(v[i]) * a.scale : -INFINITY;
    s.x = fmaxf(s.x, y[i]);
  }
  s.x = fminf(s.x, FAR);
#pragma unroll
  for (int i = 0; i < PER; ++i) s.y += exp_of(y[i] - s.x);
#pragma unroll
  for (int o = 1; o < 64; o *= 2) s = meet(s, make_float2(__shfl_xor(s.x, o, 64), __shfl_xor(s.y, o, 64)));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  if (threadIdx.x == 0) p.count = 0;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < THREADS / 64; ++w) s = meet(s, red[w]);
    a.lse[row] = s.x + log2f(s.y) * LN2;
  }
  auto columns = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (key[i]) f(key[i], (int)threadIdx.x + THREADS * i);
  };
  Cut c{0, 0}, ci{0, 0};
  if (a.k < a.vocab) {
    c = threshold<THREADS>([&](auto f) __attribute__((always_inline)) { columns([&](unsigned x, int) { f(x); }); }, a.k, p.pick);
    if (c.want)
      ci = threshold<THREADS>(
          [&](auto f) __attribute__((always_inline)) { columns([&](unsigned x, int at) { if (x == c.t) f(~(unsigned)at); }); }, c.want, p.pick);
  }
  columns([&](unsigned x, int at) {
    if (x > c.t || (x == c.t && (!c.want || ~(unsigned)at >= ci.t)))
      p.cand[atomicAdd(&p.count, 1u)] = (u64)x << 32 | (unsigned)~at;
  });
  __syncthreads();
  place<T, THREADS>(a, row, z, p.cand, a.k);
}

// Without groups: up to 4,096 columns (2,000 x 4,000 fp32, k = 20: 19.4 us, with them 23.4),
// and up to 16,384 where there are fewer groups than twice k.
inline bool is_small(int vocab, int k) {
  return vocab <= 256 * PER || (vocab <= 1024 * PER && (vocab + GROUP - 1) / GROUP < 2 * k);
}

// Whether a block takes a whole row: with many rows, or some of moderate length (the parts'
// way / this, us: 1,024 x 151,936 bf16 89.8 / 71.9, 300 38.5 / 50.1; 400 x 32,000 bf16 23.0 /
// 19.6, 200 fp32 17.4 / 14.9).
inline bool is_whole(int rows, int vocab) {
  return vocab <= 256 * PER * GROUP && (rows >= 512 || (rows >= 64 && vocab <= 65536));
}

template <class T>
void launch(const TopArgs &a, hipStream_t st) {
  if (is_small(a.vocab, a.k)) {
    if (a.vocab <= 256 * PER) k_top_small<T, 256><<<a.rows, 256, 0, st>>>(a);
    else k_top_small<T, 1024><<<a.rows, 1024, 0, st>>>(a);
    SEG_LAUNCH_CHECK();
    return;
  }
  if (is_whole(a.rows, a.vocab)) {
    const size_t lds = (size_t)a.groups * 4;
    if ((double)a.rows * a.vocab * sizeof(T) > STREAM_BYTES) k_top_row<T, true><<<a.rows, 256, lds, st>>>(a);
    else k_top_row<T, false><<<a.rows, 256, lds, st>>>(a);
    SEG_LAUNCH_CHECK();
    return;
  }
  k_top_scan<T><<<(unsigned)((long)a.rows * a.parts), 256, 0, st>>>(a);
  SEG_LAUNCH_CHECK();
  // (1,024 threads hold the groups of any vocabulary, 256 those of 262,144 columns)
  if (a.groups <= 256 * PER) k_top_pick<T, 256><<<a.rows, 256, 0, st>>>(a);
  else k_top_pick<T, 1024><<<a.rows, 1024, 0, st>>>(a);
  SEG_LAUNCH_CHECK();
}

struct TopWs {
  size_t gmax, stats, total;
  int groups, parts, span;
};

// Parts of a row: spans of SPAN columns, halved down to the 2,048 of one piece while the
// chip has more CUs than blocks (one row of 151,936 fp32: 4.8 us in 10 parts, 3.3 in 75)
TopWs top_ws(int rows, int vocab) {
  TopWs w{};
  w.groups = (vocab + GROUP - 1) / GROUP;
  w.span = SPAN;
  while (w.span > 2048 && (long)rows * ((vocab + w.span - 1) / w.span) < 256) w.span /= 2;
  w.parts = (vocab + w.span - 1) / w.span;
  if (is_small(vocab, 1) || is_whole(rows, vocab)) return w;  // none
  w.stats = align_up((size_t)rows * w.groups * 4);
  w.total = w.stats + align_up((size_t)rows * w.parts * sizeof(float2));
  return w;
}

}  // namespace
}  // namespace seg

using namespace seg;

extern "C" size_t seg_top_logits_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab < 1 || rows > (1 << 20) || vocab > (1 << 20)) return 0;
  return top_ws(rows, vocab).total;
}

extern "C" seg_status seg_top_logits(int32_t rows, int32_t vocab, int32_t k, seg_dtype dt, const void *z,
                                     int64_t ldz, float scale, int32_t *ids, float *logits, float *lse, void *ws,
                                     size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    SEG_CHECK(dt == SEG_BF16 || dt == SEG_F32, SEG_ERR_UNSUPPORTED, "dtype %d not supported", (int)dt);
    SEG_CHECK(rows >= 0 && vocab >= 1, SEG_ERR_ARG, "bad sizes rows=%d vocab=%d", rows, vocab);
    SEG_CHECK(rows <= (1 << 20) && vocab <= (1 << 20), SEG_ERR_CAPACITY, "rows %d or vocab %d above 2^20", rows, vocab);
    SEG_CHECK(k >= 1 && k <= vocab, SEG_ERR_ARG, "k = %d of %d columns", k, vocab);
    SEG_CHECK(k <= MAX_K, SEG_ERR_UNSUPPORTED, "k = %d above %d", k, MAX_K);
    SEG_CHECK(ldz >= vocab && ldz < (1LL << 40), SEG_ERR_ARG, "row stride %lld < vocab %d", (long long)ldz, vocab);
    SEG_CHECK(std::isfinite(scale), SEG_ERR_ARG, "non-finite scale");
    if (rows == 0) return;
    const TopWs w = top_ws(rows, vocab);
    SEG_CHECK(ws_bytes >= w.total, SEG_ERR_WORKSPACE, "workspace of %zu bytes < required %zu", ws_bytes, w.total);
    SEG_CHECK(z && ids && logits && lse && (ws || w.total == 0), SEG_ERR_ARG, "a tensor pointer is NULL");
    const size_t e = dt == SEG_BF16 ? 2 : 4;
    SEG_CHECK(reinterpret_cast<uintptr_t>(z) % e == 0, SEG_ERR_ARG, "z is not aligned to its type");
    SEG_CHECK(w.total == 0 || reinterpret_cast<uintptr_t>(ws) % 16 == 0, SEG_ERR_UNSUPPORTED, "the workspace is not on a 16-byte boundary");
    // (the way by parts alone launches more than a block a row)
    SEG_CHECK(w.total == 0 || (double)rows * w.parts <= 0x7fffffffL / 256, SEG_ERR_CAPACITY, "too many rows for one launch");
    check_apart({{ids, (size_t)rows * k * 4}, {logits, (size_t)rows * k * 4}, {lse, (size_t)rows * 4},
                 {w.total ? ws : nullptr, w.total}},
                {{z, ((size_t)(rows - 1) * ldz + vocab) * e}});
    char *base = static_cast<char *>(ws);
    const TopArgs a{z, ldz, rows, vocab, k, w.groups, w.parts, w.span, scale, reinterpret_cast<unsigned *>(base + w.gmax),
                    reinterpret_cast<float2 *>(base + w.stats), ids, logits, lse};
    ProfScope prof("top_logits", stream);
    if (dt == SEG_BF16) launch<unsigned short>(a, stream);
    else launch<float>(a, stream);
  });
}
