// Tensors packed to 8-bit floating point with blocks of 128 (format: fp8.h) and read
// again.
//
// One pass each, bound by HBM: 3 bytes an element of bf16, 5 of fp32.  A lane takes
// 8 columns, so 16 lanes a row of a block, whose largest magnitude is four lane
// permutations.  Blocks of one row: a thread block takes 16 rows and up to four blocks
// of columns of each, one after another in the lane, so that a row is read in pieces of
// 1 KB (bf16).  Blocks of 128 rows: a thread block takes one of them, its 8 rows a lane
// held in registers until the four waves have met in LDS.  Rows may start at any
// element: accesses of any width take any alignment of one.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "fp8.h"

namespace seg {
namespace {

struct PackArgs {
  void *x;
  long ldx;
  uint8_t *code, *exp;
  long rows, ldc, lde;
  int cols, groups;  // groups: of column blocks, in a row
};

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
typedef unsigned Code8 __attribute__((ext_vector_type(2)));

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

// 8 columns from c on of a row (those past the end: 0)
template <class T, bool STREAM>
__device__ __forceinline__ typename Piece<T>::X load8(const T *row, int c, int cols) {
  typename Piece<T>::X v{};
  if (c + 8 <= cols) return load_piece<STREAM, typename Piece<T>::X>(row + c);
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (c + j < cols) v[j] = row[c + j];
  return v;
}
template <class T>
__device__ __forceinline__ void floats8(const typename Piece<T>::X &v, float (&f)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (sizeof(T) == 2) f[j] = bf_bits2f(v[j]);
    else f[j] = v[j];
  }
}

// Blocks of one row: 16 rows, U blocks of columns.
template <class T, int U, bool STREAM>
__global__ void __launch_bounds__(256) k_pack_rows(const PackArgs a) {
  const long rg = blockIdx.x / (unsigned)a.groups;
  const int g = blockIdx.x - (unsigned)rg * (unsigned)a.groups;
  const long row = rg * 16 + (threadIdx.x >> 4);
  const int c0 = g * U * fp8::BLOCK + (threadIdx.x & 15) * 8;
  const bool ok = row < a.rows;
  const T *x = static_cast<const T *>(a.x) + (ok ? row : 0) * a.ldx;
  typename Piece<T>::X v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    v[u] = load8<T, STREAM>(x, c0 + u * fp8::BLOCK, ok ? a.cols : 0);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * fp8::BLOCK;
    float f[8];
    floats8<T>(v[u], f);
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, fp8::mag(f[j]));
    const int e = fp8::exp_byte(fp8::max16(top));
    const uint2 w = fp8::codes8(f, e);
    if (ok && c < a.ldc) store_piece<STREAM>(a.code + row * a.ldc + c, Code8{w.x, w.y});
    // (rows behind the last, up to 16, get the byte 0)
    if ((threadIdx.x & 15) == 0 && c < a.cols) a.exp[(long)(c / fp8::BLOCK) * a.lde + row] = (uint8_t)e;
  }
}

// Blocks of 128 rows: one of them a thread block, lane rows 16 apart.
template <class T, bool STREAM>
__global__ void __launch_bounds__(256) k_pack_square(const PackArgs a) {
  __shared__ unsigned tops[4];
  const long rb = blockIdx.x / (unsigned)a.groups;
  const int b = blockIdx.x - (unsigned)rb * (unsigned)a.groups;
  const long r0 = rb * fp8::BLOCK + (threadIdx.x >> 4);
  const int c = b * fp8::BLOCK + (threadIdx.x & 15) * 8;
  typename Piece<T>::X v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long row = r0 + 16 * i;
    const bool ok = row < a.rows;
    v[i] = load8<T, STREAM>(static_cast<const T *>(a.x) + (ok ? row : 0) * a.ldx, c, ok ? a.cols : 0);
  }
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float f[8];
    floats8<T>(v[i], f);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, fp8::mag(f[j]));
  }
  top = fp8::max16(top);
  top = max(top, (unsigned)__shfl_xor((int)top, 16, 64));
  top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  const int e = fp8::exp_byte(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long row = r0 + 16 * i;
    float f[8];
    floats8<T>(v[i], f);
    const uint2 w = fp8::codes8(f, e);
    if (row < a.rows && c < a.ldc)
      store_piece<STREAM>(a.code + row * a.ldc + c, Code8{w.x, w.y});
  }
  // (bytes behind the last block of rows, up to 16: 0)
  if (threadIdx.x == 0) a.exp[(long)b * a.lde + rb] = (uint8_t)e;
  const long end = rb + 1 + threadIdx.x;
  if ((rb + 1) * fp8::BLOCK >= a.rows && end < a.lde) a.exp[(long)b * a.lde + end] = 0;
}

// bf16 bits of v, to nearest, ties to even (the conversion instruction makes zeros of
// subnormal numbers, which the smallest blocks hold)
__device__ __forceinline__ unsigned short bf_rne(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  return (unsigned short)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

template <class T, int U, bool STREAM>
__global__ void __launch_bounds__(256) k_unpack_rows(const PackArgs a, int shift) {
  const long rg = blockIdx.x / (unsigned)a.groups;
  const int g = blockIdx.x - (unsigned)rg * (unsigned)a.groups;
  const long row = rg * 16 + (threadIdx.x >> 4);
  const int c0 = g * U * fp8::BLOCK + (threadIdx.x & 15) * 8;
  if (row >= a.rows) return;
  Code8 w[U];
  int e[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * fp8::BLOCK;
    w[u] = Code8{0, 0};
    e[u] = 0;
    if (c < a.cols) {
      w[u] = load_piece<STREAM, Code8>(a.code + row * a.ldc + c);
      e[u] = a.exp[(long)(c / fp8::BLOCK) * a.lde + (row >> shift)];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = c0 + u * fp8::BLOCK;
    if (c >= a.cols) break;
    const float sc = fp8::scale(e[u]);
    float f[8];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      f[4 * q] = __builtin_amdgcn_cvt_f32_fp8((int)w[u][q], 0) * sc;
      f[4 * q + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[u][q], 1) * sc;
      f[4 * q + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[u][q], 2) * sc;
      f[4 * q + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[u][q], 3) * sc;
    }
    typename Piece<T>::X o;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (sizeof(T) == 2) o[j] = bf_rne(f[j]);
      else o[j] = f[j];
    }
    T *d = static_cast<T *>(a.x) + row * a.ldx + c;
    if (c + 8 <= a.cols) store_piece<STREAM, typename Piece<T>::X>(d, o);
    else
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (c + j < a.cols) d[j] = o[j];
  }
}

// The launch of the kernels that take 16 rows a thread block: blocks of columns a lane, one
// where there are few of them, so that more thread blocks start.
struct Grid {
  int unroll, groups;
  double blocks;
  Grid(long rows, long cols) {
    const long nb = fp8::blocks_of(cols), rg = (rows + 15) / 16;
    unroll = rg * nb > 4096 && nb >= 3 ? 4 : 1;
    groups = (int)((nb + unroll - 1) / unroll);
    blocks = (double)rg * groups;
  }
};

// Thread blocks of a launch: 2^31 threads (a launch may have 2^32 - 1).
constexpr double MAX_BLOCKS = 1 << 23;

// What both entry points check (packing: x is read); false where there is nothing to do.
bool pack_args(int64_t rows, int32_t cols, seg_dtype dt, const void *x, int64_t ldx, const seg_fp8 *p, bool packing,
               PackArgs &a) {
  SEG_CHECK(dt == SEG_BF16 || dt == SEG_F32, SEG_ERR_UNSUPPORTED, "dtype %d not supported", (int)dt);
  SEG_CHECK(rows >= 0 && cols >= 1, SEG_ERR_ARG, "rows %lld or cols %d out of range", (long long)rows, cols);
  SEG_CHECK(ldx >= cols, SEG_ERR_ARG, "row stride %lld < cols %d", (long long)ldx, cols);
  SEG_CHECK(cols <= (1 << 30) && rows < (1LL << 36) && ldx < (1LL << 40) && (double)rows * ldx < 1e15,
            SEG_ERR_CAPACITY, "tensor too large");
  SEG_CHECK(p, SEG_ERR_ARG, "the struct of the 8-bit arrays is NULL");
  SEG_CHECK(p->block_rows == 1 || p->block_rows == fp8::BLOCK, SEG_ERR_UNSUPPORTED,
            "blocks of %d rows, not of 1 or 128", p->block_rows);
  if (rows == 0) return false;
  SEG_CHECK(x, SEG_ERR_ARG, "x is NULL");
  fp8::check(p, "8 bits");
  SEG_CHECK(reinterpret_cast<uintptr_t>(x) % (dt == SEG_BF16 ? 2 : 4) == 0, SEG_ERR_ARG, "x is not aligned to its type");
  // (packing of 128 x 128 blocks has a grid of its own: of few rows it is up to four times as large)
  const double blocks = packing && p->block_rows != 1 ? (double)fp8::blocks_of(rows) * fp8::blocks_of(cols)
                                                      : Grid(rows, cols).blocks;
  SEG_CHECK(blocks <= MAX_BLOCKS, SEG_ERR_CAPACITY, "tensor too large for one launch");
  a = PackArgs{const_cast<void *>(x), ldx, p->code, p->exp, rows, fp8::ld_code(cols), fp8::ld_exp(rows, p->block_rows),
               cols, 0};
  return true;
}

struct Memory {
  Span x, code, exp;
  bool stream;
};
Memory memory_of(const PackArgs &a, int block_rows, seg_dtype dt) {
  const size_t e = dt == SEG_BF16 ? 2 : 4;
  return {{a.x, ((size_t)(a.rows - 1) * a.ldx + a.cols) * e}, {a.code, fp8::code_bytes(a.rows, a.cols)},
          {a.exp, fp8::exp_bytes(a.rows, a.cols, block_rows)}, (double)a.rows * a.cols * (e + 1) > STREAM_BYTES};
}

// kernel(T, U, STREAM): past the caches where they cannot hold the tensors
template <class F>
void launch_rows(PackArgs &a, seg_dtype dt, bool stream, F &&kernel) {
  const Grid g(a.rows, a.cols);
  a.groups = g.groups;
  const unsigned grid = (unsigned)g.blocks;
  auto go = [&](auto t) {
    if (g.unroll == 1) kernel(grid, t, std::integral_constant<int, 1>(), std::false_type());
    else if (!stream) kernel(grid, t, std::integral_constant<int, 4>(), std::false_type());
    else kernel(grid, t, std::integral_constant<int, 4>(), std::true_type());
  };
  if (dt == SEG_BF16) go((unsigned short)0);
  else go(0.f);
  SEG_LAUNCH_CHECK();
}

}  // namespace
}  // namespace seg

using namespace seg;

extern "C" seg_status seg_fp8_pack(int64_t rows, int32_t cols, seg_dtype dt, const void *x, int64_t ldx,
                                   const seg_fp8 *out, hipStream_t stream) {
  return guarded([&] {
    PackArgs a{};
    if (!pack_args(rows, cols, dt, x, ldx, out, true, a)) return;
    const Memory m = memory_of(a, out->block_rows, dt);
    check_apart({m.code, m.exp}, {m.x});
    ProfScope prof("fp8_pack", stream);
    if (out->block_rows == 1) {
      launch_rows(a, dt, m.stream, [&](unsigned nb, auto t, auto u, auto past) {
        k_pack_rows<decltype(t), decltype(u)::value, decltype(past)::value><<<nb, 256, 0, stream>>>(a);
      });
      return;
    }
    a.groups = (int)fp8::blocks_of(cols);
    const unsigned grid = (unsigned)(fp8::blocks_of(rows) * a.groups);
    auto go = [&](auto t) {
      if (m.stream) k_pack_square<decltype(t), true><<<grid, 256, 0, stream>>>(a);
      else k_pack_square<decltype(t), false><<<grid, 256, 0, stream>>>(a);
    };
    if (dt == SEG_BF16) go((unsigned short)0);
    else go(0.f);
    SEG_LAUNCH_CHECK();
  });
}

extern "C" seg_status seg_fp8_unpack(int64_t rows, int32_t cols, seg_dtype dt, const seg_fp8 *in, void *x,
                                     int64_t ldx, hipStream_t stream) {
  return guarded([&] {
    PackArgs a{};
    if (!pack_args(rows, cols, dt, x, ldx, in, false, a)) return;
    const Memory m = memory_of(a, in->block_rows, dt);
    check_apart({m.x}, {m.code, m.exp});
    const int shift = in->block_rows == 1 ? 0 : 7;
    ProfScope prof("fp8_unpack", stream);
    launch_rows(a, dt, m.stream, [&](unsigned nb, auto t, auto u, auto past) {
      k_unpack_rows<decltype(t), decltype(u)::value, decltype(past)::value><<<nb, 256, 0, stream>>>(a, shift);
    });
  });
}
