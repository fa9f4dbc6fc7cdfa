// Norm and rotary positions of queries and keys: what the kernels are given.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/ppll.h"

namespace ppll {

constexpr int ROTARY_PAIRS = 128;          // pairs of a head, at most
constexpr int ROTARY_PARTIALS = 512;       // workgroups of a backward pass (a side), each leaving a row of partial sums in [.][2][head_dim]

struct RotaryPlan {
  int32_t rows, tokens, heads[2], hd, axes, pairs, neighbours;
  int32_t end[3];                          // first pair behind those of an axis
  float eps;
  double turns[ROTARY_PAIRS];              // of a pair, at position 1: base^(-i / n) / (2 pi)
};
// One side (0: queries, 1: keys) of a call.  forward: y = R norm(x); backward: y -> dx, from dy
struct RotarySide {
  const void *x, *dy;
  void *y, *keep;
  int64_t x_ld, dy_ld, y_ld, keep_ld;
  const float* scale;
};

int rotary_plan(const ppll_rotary_config* cfg, RotaryPlan* plan);
inline size_t rotary_partial_floats(int hd) { return (size_t)ROTARY_PARTIALS * 2 * hd; }

}  // namespace ppll
