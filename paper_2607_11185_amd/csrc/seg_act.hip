// Activations kept in 8 bits between a layer's forward and backward (format:
// act8.h), packed from and unpacked to rows of bf16 or fp32.
//
// Both kernels are bound by HBM: one pass, 3.03 (bf16) or 5.03 (fp32) bytes an
// element.  A lane takes 16 bytes of x, so four (bf16) or eight lanes a block, whose
// largest magnitude is two or three lane permutations.  Rows may start anywhere:
// global accesses of any width take any alignment of an element, and a row's last,
// shorter chunk goes element by element.  Measured, pack / unpack: 137,895 x 3,584
// bf16 230 / 241 us (6.5 / 6.2 TB/s); 100,000 x 2,147 bf16, rows on odd addresses, 115 /
// 128 (with a column a lane 395 / 333).
#include <algorithm>

#include "act8.h"
#include "common.h"

namespace seg {
namespace {

struct ActArgs {
  void *x;
  long ldx;
  int8_t *code;
  uint8_t *exp;
  long rows;
  int cols, per_row, blocks;   // of a row: chunks, and blocks of 32 columns
  int step_rows, step_chunks;  // 64 chunks further: rows and chunks
  bool narrow;                 // all chunks count in 32 bits
};

// accesses of a chunk, at the alignment of an element
template <class T>
struct Chunk;
template <>
struct Chunk<unsigned short> {
  static constexpr int W = 8;
  typedef unsigned short X __attribute__((ext_vector_type(8), aligned(2)));
  typedef unsigned C __attribute__((ext_vector_type(2), aligned(1)));
};
template <>
struct Chunk<float> {
  static constexpr int W = 4;
  typedef float X __attribute__((ext_vector_type(4), aligned(4)));
  typedef unsigned C __attribute__((ext_vector_type(1), aligned(1)));
};

// A lane's chunk of columns; a wave takes 64 consecutive chunks at a time, a row
// holding whole blocks of them.
struct Walk {
  long row;
  int c;
  __device__ __forceinline__ Walk(const ActArgs &a, long i) {
    row = a.narrow ? (long)((unsigned)i / (unsigned)a.per_row) : i / a.per_row;
    c = (int)(i - row * a.per_row);
  }
  __device__ __forceinline__ void next(const ActArgs &a) {
    row += a.step_rows;
    c += a.step_chunks;
    if (c >= a.per_row) {
      c -= a.per_row;
      ++row;
    }
  }
};

// bf16 bits of a value that bf16 holds: its upper half (the conversion
// instruction makes zeros of subnormal numbers, and 2^-127 is one)
__device__ __forceinline__ unsigned short bf_exact(float v) {
  return (unsigned short)(__builtin_bit_cast(unsigned, v) >> 16);
}
template <class T>
__device__ __forceinline__ float to_float(T v) {
  if constexpr (sizeof(T) == 2) return bf_bits2f(v);
  else return v;
}
template <class T>
__device__ __forceinline__ T of_exact(float v) {
  if constexpr (sizeof(T) == 2) return bf_exact(v);
  else return v;
}

template <bool STREAM, class V, class P>
__device__ __forceinline__ V load_piece(const P *p) {
  const V *q = reinterpret_cast<const V *>(p);
  return STREAM ? __builtin_nontemporal_load(q) : *q;
}
template <bool STREAM, class V, class P>
__device__ __forceinline__ void store_piece(P *p, const V &x) {
  V *q = reinterpret_cast<V *>(p);
  if (STREAM) __builtin_nontemporal_store(x, q);
  else *q = x;
}

// U chunks a lane; more than one: past the caches (STREAM_BYTES) or not
template <class T, int U, bool STREAM>
__global__ void __launch_bounds__(256) k_pack(const ActArgs a) {
  typedef Chunk<T> K;
  constexpr int W = K::W;
  const int lane = threadIdx.x & 63;
  Walk w(a, ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 * U) + lane);
  typename K::X v[U];
  long row[U];
  int col[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    row[u] = w.row;
    col[u] = w.c * W;
    const int n = row[u] < a.rows ? a.cols - col[u] : 0;
    const T *p = static_cast<const T *>(a.x) + row[u] * a.ldx + col[u];
    v[u] = typename K::X{};
    if (n >= W) v[u] = load_piece<STREAM, typename K::X>(p);
    else
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        if (j < n) v[u][j] = p[j];
    w.next(a);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float f[W];
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      f[j] = to_float<T>(v[u][j]);
      top = max(top, act8::mag(f[j]));
    }
    top = W == 8 ? act8::max4(top) : act8::max8(top);
    const int n = row[u] < a.rows ? a.cols - col[u] : 0;
    if (n <= 0) continue;
    const int e = act8::exp_byte(top);
    if (col[u] % act8::BLOCK == 0) a.exp[row[u] * a.blocks + col[u] / act8::BLOCK] = (uint8_t)e;
    unsigned cw[W / 4];
    act8::codes(f, e, cw);
    typename K::C c;
#pragma unroll
    for (int q = 0; q < W / 4; ++q) c[q] = cw[q];
    int8_t *d = a.code + row[u] * a.cols + col[u];
    if (n >= W) store_piece<STREAM>(d, c);
    else
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        if (j < n) d[j] = (int8_t)(c[j / 4] >> (8 * (j & 3)));
  }
}

template <class T, int U, bool STREAM>
__global__ void __launch_bounds__(256) k_unpack(const ActArgs a) {
  typedef Chunk<T> K;
  constexpr int W = K::W;
  const int lane = threadIdx.x & 63;
  Walk w(a, ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 * U) + lane);
  typename K::C cd[U];
  int e[U], col[U];
  long row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    row[u] = w.row;
    col[u] = w.c * W;
    const int n = row[u] < a.rows ? a.cols - col[u] : 0;
    const int8_t *p = a.code + row[u] * a.cols + col[u];
    e[u] = n > 0 ? a.exp[row[u] * a.blocks + col[u] / act8::BLOCK] : 0;
    cd[u] = typename K::C{};
    if (n >= W) cd[u] = load_piece<STREAM, typename K::C>(p);
    else
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        if (j < n) cd[u][j / 4] |= (unsigned)(uint8_t)p[j] << (8 * (j & 3));
    w.next(a);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int n = row[u] < a.rows ? a.cols - col[u] : 0;
    if (n <= 0) continue;
    const float sc = act8::scale(e[u]);
    typename K::X o;
#pragma unroll
    for (int j = 0; j < W; ++j) o[j] = of_exact<T>(act8::value(cd[u][j / 4], j & 3, sc));
    T *d = static_cast<T *>(a.x) + row[u] * a.ldx + col[u];
    if (n >= W) store_piece<STREAM>(d, o);
    else
#pragma unroll
      for (int j = 0; j < W - 1; ++j)
        if (j < n) d[j] = o[j];
  }
}

bool act_args(int64_t rows, int32_t cols, seg_dtype dt, const void *x, int64_t ldx,
              const seg_act8 *p, ActArgs &a) {
  SEG_CHECK(dt == SEG_BF16 || dt == SEG_F32, SEG_ERR_UNSUPPORTED, "dtype %d not supported", (int)dt);
  SEG_CHECK(rows >= 0 && cols >= 1, SEG_ERR_ARG, "rows %lld or cols %d out of range", (long long)rows, cols);
  SEG_CHECK(ldx >= cols, SEG_ERR_ARG, "row stride %lld < cols %d", (long long)ldx, cols);
  SEG_CHECK(p, SEG_ERR_ARG, "the 8-bit arrays' struct is NULL");
  SEG_CHECK(cols <= (1 << 30) && rows < (1LL << 40) && ldx < (1LL << 40) && (double)rows * ldx < 1e15, SEG_ERR_CAPACITY,
            "tensor too large");
  if (rows == 0) return false;
  SEG_CHECK(x && p->code && p->exp, SEG_ERR_ARG, "x or an 8-bit array is NULL");
  SEG_CHECK(reinterpret_cast<uintptr_t>(x) % (dt == SEG_BF16 ? 2 : 4) == 0, SEG_ERR_ARG, "x is not aligned to its type");
  a.x = const_cast<void *>(x);
  a.ldx = ldx;
  a.code = p->code;
  a.exp = p->exp;
  a.rows = rows;
  a.cols = cols;
  a.blocks = (int)act8::blocks_of(cols);
  return true;
}

// chunks of a row, whole blocks of them
long chunks_of(long cols, seg_dtype dt) {
  return act8::blocks_of(cols) * (act8::BLOCK / (dt == SEG_BF16 ? Chunk<unsigned short>::W : Chunk<float>::W));
}

// Chunks a lane: one until the chip is full, four in flight beyond that.
struct Grid {
  int unroll;
  long blocks;
  explicit Grid(long chunks) : unroll(chunks > 2048 * 256 ? 4 : 1), blocks((chunks + 256 * unroll - 1) / (256 * unroll)) {}
};

// Launches kernel(T, U, STREAM): U chunks a lane, past the caches where they cannot
// hold the tensors.
template <class F>
void act_launch(ActArgs &a, seg_dtype dt, const char *name, hipStream_t st, F &&kernel) {
  act8::check_launch(a.rows, a.cols, dt);
  a.per_row = (int)chunks_of(a.cols, dt);
  a.step_rows = 64 / a.per_row;
  a.step_chunks = 64 % a.per_row;
  const Grid grid(a.rows * a.per_row);
  const int unroll = grid.unroll;
  const long nb = grid.blocks;
  check_apart({{a.code, (size_t)a.rows * a.cols}, {a.exp, (size_t)a.rows * a.blocks}},
              {{a.x, ((size_t)(a.rows - 1) * a.ldx + a.cols) * (dt == SEG_BF16 ? 2 : 4)}});
  a.narrow = nb * 256 * unroll <= 0xffffffffL;
  const double bytes = (double)a.rows * a.cols * (dt == SEG_BF16 ? 3 : 5);
  ProfScope prof(name, st);
  auto go = [&](auto t) {
    if (unroll == 1) kernel((unsigned)nb, t, std::integral_constant<int, 1>(), std::false_type());
    else if (bytes <= STREAM_BYTES) kernel((unsigned)nb, t, std::integral_constant<int, 4>(), std::false_type());
    else kernel((unsigned)nb, t, std::integral_constant<int, 4>(), std::true_type());
  };
  if (dt == SEG_BF16) go((unsigned short)0);
  else go(0.f);
  SEG_LAUNCH_CHECK();
}

}  // namespace

void act8::check_launch(long rows, long cols, seg_dtype dt) {
  SEG_CHECK(Grid(rows * chunks_of(cols, dt)).blocks <= 0x7fffffffL / 256, SEG_ERR_CAPACITY,
            "tensor too large for one launch");
}

void act8::pack(int64_t rows, int32_t cols, seg_dtype dt, const void *x, int64_t ldx, const seg_act8 *out,
                const char *name, hipStream_t st) {
  ActArgs a{};
  if (!act_args(rows, cols, dt, x, ldx, out, a)) return;
  act_launch(a, dt, name, st, [&](unsigned nb, auto t, auto u, auto past) {
    k_pack<decltype(t), decltype(u)::value, decltype(past)::value><<<nb, 256, 0, st>>>(a);
  });
}

void act8::unpack(int64_t rows, int32_t cols, seg_dtype dt, const seg_act8 *in, void *x, int64_t ldx,
                  const char *name, hipStream_t st) {
  ActArgs a{};
  if (!act_args(rows, cols, dt, x, ldx, in, a)) return;
  act_launch(a, dt, name, st, [&](unsigned nb, auto t, auto u, auto past) {
    k_unpack<decltype(t), decltype(u)::value, decltype(past)::value><<<nb, 256, 0, st>>>(a);
  });
}

}  // namespace seg

using namespace seg;

extern "C" seg_status seg_act_pack(int64_t rows, int32_t cols, seg_dtype dt, const void *x,
                                   int64_t ldx, const seg_act8 *out, hipStream_t stream) {
  return guarded([&] { act8::pack(rows, cols, dt, x, ldx, out, "act_pack", stream); });
}

extern "C" seg_status seg_act_unpack(int64_t rows, int32_t cols, seg_dtype dt, const seg_act8 *in,
                                     void *x, int64_t ldx, hipStream_t stream) {
  return guarded([&] { act8::unpack(rows, cols, dt, in, x, ldx, "act_unpack", stream); });
}
