// Arguments of the residual norm's kernel (vq_residual_norm).
#pragma once

#include "vq_common.cuh"

namespace vq {

struct ResidualNorm {
  const void* x;          // binary16 or binary32 (wide)
  const __half* y;        // null: nothing is added
  const __half* gate;     // null: 1
  const __half* post_w;   // null: no norm of y
  const __half* post_b;
  const __half* pre_w;    // null: no norm behind
  const __half* pre_b;
  void* x_out;            // null: not stored
  __half* h;
  int rows, cols, layer, wide;
  long long x_stride, y_stride, gate_stride, x_out_stride, h_stride;   // gate_stride 0: one row for all
  float eps, scale;
};

vq_status launch_residual_norm(const ResidualNorm& a, cudaStream_t s);

}  // namespace vq
