// Activations kept in 8 bits between a layer's forward and backward (format:
// act8.h), packed from and unpacked to rows of bf16 or fp32.
//
// Both kernels are bound by HBM: one pass, 3.03 (bf16) or 5.03 (fp32) bytes an
// element.  A lane takes 8 columns (16-byte accesses for bf16), four lanes a
// block, so the block's largest magnitude is two exchanges inside a quad.
#include <algorithm>

#include "act8.h"
#include "common.h"

namespace seg {
namespace {

constexpr int UNROLL = 4;  // chunks of a lane in flight

struct ActArgs {
  void *x;
  long ldx;
  int8_t *code;
  uint8_t *exp;
  long rows, chunks;  // chunks of 8 columns, whole blocks (four chunks) a row
  int cols, per_row;  // per_row: chunks of a row
  int step_rows, step_chunks;  // 64 chunks further: rows and chunks
};

// A lane's place in the chunks, which a wave takes 64 consecutive ones at a time.
struct Walk {
  long row;
  int c;
  __device__ __forceinline__ void next(const ActArgs &a) {
    row += a.step_rows;
    c += a.step_chunks;
    if (c >= a.per_row) {
      c -= a.per_row;
      ++row;
    }
  }
};

template <class T, bool VEC>
__device__ __forceinline__ void load8(const T *p, int n, float (&v)[8]) {
  if constexpr (VEC && sizeof(T) == 2) {
    const u16x8 w = *reinterpret_cast<const u16x8 *>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = bf_bits2f(w[j]);
  } else if constexpr (VEC) {
    const f32x4 lo = reinterpret_cast<const f32x4 *>(p)[0], hi = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = lo[j];
      v[4 + j] = hi[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = 0.f;
      if (j < n) {
        if constexpr (sizeof(T) == 2) v[j] = bf_bits2f(p[j]);
        else v[j] = p[j];
      }
    }
  }
}

// VEC: cols a multiple of 8, x rows on 16-byte boundaries, codes on 8-byte ones
template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_pack(const ActArgs a) {
  const int lane = threadIdx.x & 63;
  const long wave = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long first = wave * (64 * UNROLL) + lane;
  const T *x = static_cast<const T *>(a.x);
  Walk w{first / a.per_row, 0};
  w.c = (int)(first - w.row * a.per_row);
  float v[UNROLL][8];
  long row[UNROLL];
  int col[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    row[u] = w.row;
    col[u] = w.c * 8;
    const int n = w.row < a.rows ? a.cols - col[u] : 0;
    if (n > 0) load8<T, VEC>(x + w.row * a.ldx + col[u], n, v[u]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] = 0.f;
    w.next(a);
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, act8::mag(v[u][j]));
    top = max(top, (unsigned)__shfl_xor((int)top, 1, 64));
    top = max(top, (unsigned)__shfl_xor((int)top, 2, 64));
    const int n = row[u] < a.rows ? a.cols - col[u] : 0;
    if (n <= 0) continue;
    const int e = act8::exp_byte(top);
    if ((lane & 3) == 0) a.exp[row[u] * (a.per_row / 4) + col[u] / act8::BLOCK] = (uint8_t)e;
    const unsigned lo = act8::codes4(v[u][0], v[u][1], v[u][2], v[u][3], e);
    const unsigned hi = act8::codes4(v[u][4], v[u][5], v[u][6], v[u][7], e);
    int8_t *d = a.code + row[u] * a.cols + col[u];
    if constexpr (VEC) {
      *reinterpret_cast<uint2 *>(d) = make_uint2(lo, hi);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) d[j] = (int8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
    }
  }
}

// bf16 bits of a value that bf16 holds: its upper half (the conversion
// instruction makes zeros of subnormal numbers, and 2^-127 is one)
__device__ __forceinline__ unsigned short bf_exact(float v) {
  return (unsigned short)(__builtin_bit_cast(unsigned, v) >> 16);
}

template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_unpack(const ActArgs a) {
  const int lane = threadIdx.x & 63;
  const long wave = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long first = wave * (64 * UNROLL) + lane;
  T *x = static_cast<T *>(a.x);
  Walk w{first / a.per_row, 0};
  w.c = (int)(first - w.row * a.per_row);
  unsigned cd[UNROLL][2];
  int e[UNROLL], col[UNROLL];
  long row[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    row[u] = w.row;
    col[u] = w.c * 8;
    const int n = w.row < a.rows ? a.cols - col[u] : 0;
    cd[u][0] = cd[u][1] = 0u;
    e[u] = 0;
    if (n > 0) {
      e[u] = a.exp[w.row * (a.per_row / 4) + col[u] / act8::BLOCK];
      const int8_t *s = a.code + w.row * a.cols + col[u];
      if constexpr (VEC) {
        const uint2 t = *reinterpret_cast<const uint2 *>(s);
        cd[u][0] = t.x;
        cd[u][1] = t.y;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < n) cd[u][j / 4] |= (unsigned)(uint8_t)s[j] << (8 * (j & 3));
      }
    }
    w.next(a);
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const int n = row[u] < a.rows ? a.cols - col[u] : 0;
    if (n <= 0) continue;
    float v[8];
    act8::values8(cd[u], act8::scale(e[u]), v);
    T *d = x + row[u] * a.ldx + col[u];
    if constexpr (VEC && sizeof(T) == 2) {
      u16x8 o;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = bf_exact(v[j]);
      *reinterpret_cast<u16x8 *>(d) = o;
    } else if constexpr (VEC) {
      reinterpret_cast<f32x4 *>(d)[0] = f32x4{v[0], v[1], v[2], v[3]};
      reinterpret_cast<f32x4 *>(d)[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) {
          if constexpr (sizeof(T) == 2) d[j] = bf_exact(v[j]);
          else d[j] = v[j];
        }
    }
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
  a.per_row = (int)act8::blocks_of(cols) * (act8::BLOCK / 8);
  a.chunks = rows * a.per_row;
  a.step_rows = 64 / a.per_row;
  a.step_chunks = 64 % a.per_row;
  return true;
}

// 16-byte accesses of x rows and 8-byte ones of code rows (both strides and both
// pointers; otherwise element by element)
bool vectors(const ActArgs &a, seg_dtype dt) {
  const long e = dt == SEG_BF16 ? 2 : 4;
  return a.cols % 8 == 0 && reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx * e % 16 == 0 &&
         reinterpret_cast<uintptr_t>(a.code) % 8 == 0;
}

unsigned act_blocks(const ActArgs &a) {
  const long per = 256L * UNROLL;
  const long n = (a.chunks + per - 1) / per;
  SEG_CHECK(n <= 0x7fffffffL / 256, SEG_ERR_CAPACITY, "tensor too large for one launch");
  return (unsigned)n;
}

}  // namespace
}  // namespace seg

using namespace seg;

extern "C" seg_status seg_act_pack(int64_t rows, int32_t cols, seg_dtype dt, const void *x,
                                   int64_t ldx, const seg_act8 *out, hipStream_t stream) {
  return guarded([&] {
    ActArgs a{};
    if (!act_args(rows, cols, dt, x, ldx, out, a)) return;
    const unsigned nb = act_blocks(a);
    ProfScope prof("act_pack", stream);
    const bool v = vectors(a, dt);
    if (dt == SEG_BF16) {
      if (v) k_pack<unsigned short, true><<<nb, 256, 0, stream>>>(a);
      else k_pack<unsigned short, false><<<nb, 256, 0, stream>>>(a);
    } else {
      if (v) k_pack<float, true><<<nb, 256, 0, stream>>>(a);
      else k_pack<float, false><<<nb, 256, 0, stream>>>(a);
    }
    SEG_LAUNCH_CHECK();
  });
}

extern "C" seg_status seg_act_unpack(int64_t rows, int32_t cols, seg_dtype dt, const seg_act8 *in,
                                     void *x, int64_t ldx, hipStream_t stream) {
  return guarded([&] {
    ActArgs a{};
    if (!act_args(rows, cols, dt, x, ldx, in, a)) return;
    const unsigned nb = act_blocks(a);
    ProfScope prof("act_unpack", stream);
    const bool v = vectors(a, dt);
    if (dt == SEG_BF16) {
      if (v) k_unpack<unsigned short, true><<<nb, 256, 0, stream>>>(a);
      else k_unpack<unsigned short, false><<<nb, 256, 0, stream>>>(a);
    } else {
      if (v) k_unpack<float, true><<<nb, 256, 0, stream>>>(a);
      else k_unpack<float, false><<<nb, 256, 0, stream>>>(a);
    }
    SEG_LAUNCH_CHECK();
  });
}
