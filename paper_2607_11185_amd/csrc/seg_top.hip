// The k largest logits of each row, with their columns, and the row's log-sum-exp.
//
// Order: by value, descending, then by column, ascending; NaN counts as larger than
// all numbers, -0 as 0.  Two kernels:
//
//   k_top_scan   one pass over the logits: running maximum and sum of the softmax, and
//                the largest of every 64 columns (a group) as a whole number in order;
//   k_top_pick   of each row: the k largest groups (ties: the first ones), and of their
//                columns the k largest.
//
// The k largest logits lie in the k largest groups: a column outside them is preceded
// by the largest of each of those groups, which is larger, or as large and further to
// the front, as the groups are runs of columns.  So the second kernel reads k groups
// again and not the row, and no order of the values makes it do more.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"

namespace seg {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float FAR = 3.4028234663852886e38f;
constexpr int GROUP = 64;    // columns
constexpr int MAX_K = 256;
constexpr int SPAN = 16384;  // columns of a block of the scan, at most

// Whole numbers in the order of the values: NaN first, zeros alike.  No value has 0.
__device__ __forceinline__ unsigned order(float x) {
  unsigned u = __builtin_bit_cast(unsigned, x);
  if (x != x) return 0xffffffffu;
  if (x == 0.f) u = 0;
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}

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
// lanes a group.  The maximum in front of the sum stays inside fp32's numbers, so that
// infinities meet no infinity: -inf adds 0, inf gives inf, NaN stays NaN.
template <class T>
__global__ void __launch_bounds__(256) k_top_scan(const TopArgs a) {
  __shared__ float2 red[4];
  const int row = blockIdx.x / (unsigned)a.parts, part = blockIdx.x - row * (unsigned)a.parts;
  const T *z = static_cast<const T *>(a.z) + (long)row * a.ldz;
  const int c0 = part * a.span, c1 = min(a.vocab, c0 + a.span);
  float2 s = make_float2(-FAR, 0.f);
  constexpr int U = 4;
  auto step = [&](int first, auto whole) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int c = first + threadIdx.x * 8;
    typename Piece<T>::X v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = c + 2048 * u;
      if (WHOLE || at + 8 <= c1) v[u] = *reinterpret_cast<const typename Piece<T>::X *>(z + at);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] = at + j < c1 ? z[at + j] : T();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = c + 2048 * u;
      float y[8], m = s.x;
      unsigned top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = WHOLE || at + j < c1;
        const float x = value<T>(v[u][j]);
        top = max(top, in ? order(x) : 0u);
        y[j] = in ? x * a.scale : -INFINITY;
        m = fmaxf(m, y[j]);
      }
      m = fminf(m, FAR);
      s.y *= exp_of(s.x - m);
#pragma unroll
      for (int j = 0; j < 8; ++j) s.y += exp_of(y[j] - m);
      s.x = m;
      top = max(top, (unsigned)__shfl_xor((int)top, 1, 64));
      top = max(top, (unsigned)__shfl_xor((int)top, 2, 64));
      top = max(top, (unsigned)__shfl_xor((int)top, 4, 64));
      if ((threadIdx.x & 7) == 0 && (WHOLE || at < c1)) a.gmax[(long)row * a.groups + at / GROUP] = top;
    }
  };
  int first = c0;
  for (; first + 2048 * U <= c1; first += 2048 * U) step(first, std::true_type());
  if (first < c1) step(first, std::false_type());
#pragma unroll
  for (int o = 1; o < 64; o *= 2) s = meet(s, make_float2(__shfl_xor(s.x, o, 64), __shfl_xor(s.y, o, 64)));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    a.stats[(long)row * a.parts + part] = meet(meet(red[0], red[1]), meet(red[2], red[3]));
}

typedef unsigned long long u64;

// The threshold t such that exactly `want` (at least 1, at most all) of the block's keys
// are >= t; keys are distinct and none is 0.  keys(f) calls f(key) for every key of the thread.  8 bits of the
// key a pass, from bit `shift` on down; ends early where a digit's keys are wanted whole.
struct Pick {
  unsigned hist[256];
  unsigned wave[4];
  u64 prefix;
  unsigned want, done;
};

template <class K>
__device__ __forceinline__ u64 threshold(K &&keys, unsigned want, Pick &p) {
  u64 prefix = 0;
  for (int shift = 56; shift >= 0; shift -= 8) {
    p.hist[threadIdx.x] = 0;
    __syncthreads();
    keys([&](u64 key) {
      if (shift == 56 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&p.hist[(key >> shift) & 255], 1u);
    });
    __syncthreads();
    // keys with a digit >= that of the thread
    const unsigned own = p.hist[threadIdx.x];
    unsigned n = own;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const unsigned t = __shfl_down(n, o, 64);
      if ((threadIdx.x & 63) + o < 64) n += t;
    }
    if ((threadIdx.x & 63) == 0) p.wave[threadIdx.x >> 6] = n;
    __syncthreads();
    for (int w = (threadIdx.x >> 6) + 1; w < 4; ++w) n += p.wave[w];
    if (n >= want && n - own < want) {
      p.prefix = prefix | (u64)threadIdx.x << shift;
      p.want = want - (n - own);
      p.done = n == want;
    }
    __syncthreads();
    prefix = p.prefix;
    want = p.want;
    const bool done = p.done;
    __syncthreads();
    if (done) break;
  }
  return prefix;
}

// A block a row.
constexpr int CANDS = 1024;

template <class T>
__global__ void __launch_bounds__(256) k_top_pick(const TopArgs a) {
  __shared__ Pick pick;
  __shared__ u64 cand[CANDS];
  __shared__ int group[MAX_K];
  __shared__ unsigned count, low;
  const int row = blockIdx.x;
  const T *z = static_cast<const T *>(a.z) + (long)row * a.ldz;
  const unsigned *gm = a.gmax + (long)row * a.groups;
  if (threadIdx.x == 0) {
    float2 s = a.stats[(long)row * a.parts];
    for (int i = 1; i < a.parts; ++i) s = meet(s, a.stats[(long)row * a.parts + i]);
    a.lse[row] = s.x + log2f(s.y) * LN2;
    count = 0;
    low = 0xffffffffu;
  }
  __syncthreads();
  // the groups: value, then the first ones
  const int ng = min(a.k, a.groups);
  auto groups = [&](auto f) __attribute__((always_inline)) {
    for (int i = threadIdx.x; i < a.groups; i += 256) f((u64)gm[i] << 32 | (unsigned)~i);
  };
  const u64 tg = ng < a.groups ? threshold(groups, ng, pick) : 0;
  groups([&](u64 key) {
    if (key >= tg) {
      group[atomicAdd(&count, 1u)] = (int)~(unsigned)key;
      atomicMin(&low, (unsigned)(key >> 32));
    }
  });
  __syncthreads();
  // their columns that are as large as the smallest of these groups' largest (k of them
  // are, unless all groups were taken)
  const unsigned least = ng < a.groups ? low : 0u;
  __syncthreads();
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  auto columns = [&](auto f) __attribute__((always_inline)) {
    for (int i = threadIdx.x; i < ng * GROUP; i += 256) {
      const int c = group[i / GROUP] * GROUP + i % GROUP;
      if (c >= a.vocab) continue;
      const unsigned o = order(value<T>(z[c]));
      if (o >= least) f((u64)o << 32 | (unsigned)~c);
    }
  };
  columns([&](u64 key) {
    const unsigned n = atomicAdd(&count, 1u);
    if (n < CANDS) cand[n] = key;
  });
  __syncthreads();
  int n = (int)count;
  if (n > CANDS) {  // many of the same value: the k first by their own threshold
    __syncthreads();
    const u64 t = threshold(columns, a.k, pick);
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    columns([&](u64 key) {
      if (key >= t) cand[atomicAdd(&count, 1u)] = key;
    });
    __syncthreads();
    n = a.k;
  }
  // each candidate's place is the number of those in front of it
  for (int i = threadIdx.x; i < n; i += 256) {
    const u64 key = cand[i];
    int at = 0;
    for (int j = 0; j < n; ++j) at += cand[j] > key;
    if (at < a.k) {
      const int c = (int)~(unsigned)key;
      a.ids[(long)row * a.k + at] = c;
      a.logits[(long)row * a.k + at] = value<T>(z[c]);
    }
  }
}

struct TopWs {
  size_t gmax, stats, total;
  int groups, parts, span;
};

// Parts of a row: blocks of SPAN columns, fewer where that leaves the chip idle
TopWs top_ws(int rows, int vocab) {
  TopWs w{};
  w.groups = (vocab + GROUP - 1) / GROUP;
  w.span = SPAN;
  w.parts = (vocab + w.span - 1) / w.span;
  w.gmax = 0;
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
    SEG_CHECK(z && ids && logits && lse && ws, SEG_ERR_ARG, "a tensor pointer is NULL");
    const size_t e = dt == SEG_BF16 ? 2 : 4;
    SEG_CHECK(reinterpret_cast<uintptr_t>(z) % e == 0, SEG_ERR_ARG, "z is not aligned to its type");
    SEG_CHECK(reinterpret_cast<uintptr_t>(ws) % 16 == 0, SEG_ERR_UNSUPPORTED, "the workspace is not on a 16-byte boundary");
    SEG_CHECK((double)rows * w.parts <= 0x7fffffffL / 256, SEG_ERR_CAPACITY, "too many rows for one launch");
    check_apart({{ids, (size_t)rows * k * 4}, {logits, (size_t)rows * k * 4}, {lse, (size_t)rows * 4}, {ws, w.total}},
                {{z, ((size_t)(rows - 1) * ldz + vocab) * e}});
    char *base = static_cast<char *>(ws);
    const TopArgs a{z, ldz, rows, vocab, k, w.groups, w.parts, w.span, scale, reinterpret_cast<unsigned *>(base + w.gmax),
                    reinterpret_cast<float2 *>(base + w.stats), ids, logits, lse};
    ProfScope prof("top_logits", stream);
    const unsigned grid = (unsigned)((long)rows * w.parts);
    if (dt == SEG_BF16) {
      k_top_scan<unsigned short><<<grid, 256, 0, stream>>>(a);
      SEG_LAUNCH_CHECK();
      k_top_pick<unsigned short><<<rows, 256, 0, stream>>>(a);
    } else {
      k_top_scan<float><<<grid, 256, 0, stream>>>(a);
      SEG_LAUNCH_CHECK();
      k_top_pick<float><<<rows, 256, 0, stream>>>(a);
    }
    SEG_LAUNCH_CHECK();
  });
}
