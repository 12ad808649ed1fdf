// Rotation of heads by positions on three axes (seg_mrope.hip), also called by
// the decoder layer.
#pragma once

#include <cmath>

#include "common.h"

namespace seg {
namespace mrope {

constexpr int MAX_D = 256;

// x and y [rows, heads, d] at row strides (elements); y may be x
struct Heads {
  const void *x;
  void *y;
  long ldx, ldy;
  int heads;
};

struct Args {
  Heads a, b;          // b.heads may be 0
  long rows;
  int d, inverse;
  int s0, s01;         // pairs below s0 turn with axis 0, below s01 with axis 1
  double log2_base;
  const int32_t *pos;  // [3, rows]
  // rows to rotate: pad[row] >= 0, or with pad NULL the rows whose three
  // positions are >= 0.  The others are copied; with inverse they become zeros
  // in y, and in zero [rows, zero_width] (or NULL) too.
  const int32_t *pad;
  unsigned short *zero;
  int zero_width;

  void set(const seg_mrope_cfg &c) {
    s0 = c.sections[0];
    s01 = s0 + c.sections[1];
    log2_base = std::log2((double)c.base);
  }
};

// sections, base, head counts and head size as seg_mrope_fwd takes them
void check_cfg(const seg_mrope_cfg *cfg, int32_t d);
// refuses what one launch does not hold (heads: of q and k together)
void check_launch(seg_dtype dt, long rows, int heads, int d);
void launch(seg_dtype dt, const Args &g, hipStream_t st);

}  // namespace mrope
}  // namespace seg
