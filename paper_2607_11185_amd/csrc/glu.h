// The gated feed-forward block's own parts (seg_glu.hip), also called by the
// decoder layer.
#pragma once

#include "common.h"
#include "seg.h"

namespace seg {
namespace glu {

// What a forward keeps of the gate and up values g and u [rows, inter], or a
// backward reads: bf16 (g16 set), 8 bits (g8.code set) or nothing.
struct Kept {
  unsigned short *g16, *u16;
  seg_act8 g8, u8;
};

// m = silu(x wg^T) * (x wu^T), with the gate and up values to `keep`.  sums: memory for
// partial sums (seg_glu_workspace_bytes), or NULL: a row's result then does not depend
// on the other rows
void forward(const unsigned short *x, long ldx, const unsigned short *wg, const unsigned short *wu,
             int rows, int hidden, int inter, unsigned short *m, const Kept &keep, float *sums,
             hipStream_t st);

// dg = dm * u * silu'(g), du = dm * silu(g), from the kept values; with m set
// also m = silu(g) * u.  All [rows, inter].
void backward_act(const Kept &kept, const unsigned short *dm, int rows, int inter, unsigned short *dg,
                  unsigned short *du, unsigned short *m, hipStream_t st);

}  // namespace glu
}  // namespace seg
