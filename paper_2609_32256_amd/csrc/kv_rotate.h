// Arguments of the kernels that norm and turn heads (kv_rotate.hip).
#pragma once

#include <cstdint>

#include "lam_internal.h"

namespace lam {

struct RotateHeads {   // heads of rows: strides in elements
  const uint16_t* x;
  int64_t x_row, x_head;
  uint16_t* y;
  int64_t y_row, y_head;
  const void* gain;    // of each channel, null: no norm
  int gain_f32;        // float32, else of the rows' type
  int heads;
  int x_wide, y_wide, gain_wide;   // every eight channels are a 16-byte access (gains in float32: two)
};

struct RotateArgs {
  RotateHeads h[2];      // queries and keys
  const double* freq;    // radians a position, of each pair
  int pairs, interleaved;
  float amplitude;
  double amplitude64, eps, inv_dim;
  const int32_t* positions;   // of each row
  int64_t rows;
  int dim;
  int parts;             // waves that share a row's heads
};

lam_status launch_kv_rotate(lam_ctx* ctx, RotateArgs a, int dtype);
lam_status launch_kv_rotate_append(lam_ctx* ctx, const lam_kv_view& v, const RotateArgs& r, const void* val,
                                   int64_t v_row, int64_t v_head, const lam_kv_slots& weights,
                                   const lam_kv_slots& positions, const int32_t* first, uint32_t* status);

}  // namespace lam
