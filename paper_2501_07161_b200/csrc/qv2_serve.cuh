// Page planning and norm with rotation: what their kernels are given, and the launch wrappers.
#pragma once

#include <type_traits>

#include "qv2_mx.cuh"

namespace qv2 {

cudaError_t launch_kv_plan(const Launch& l, const qv2_page_plan& p, uint32_t* ticket, uint64_t* launches);

struct HeadRows {                 // qv2_head_rows of queries and keys
  const void* x[2];
  void* y[2];
  uint64_t x_token_ld[2], x_head_ld[2], y_token_ld[2], y_head_ld[2];
  const float* weight[2];
  uint32_t heads[2];
};
struct Rotation {
  const int64_t* positions;
  const float* freqs;
  uint64_t tokens;
  uint32_t dtype, dim, rot, pairs;
  float eps;
};
cudaError_t launch_norm_rotate(const Launch& l, const HeadRows& h, const Rotation& r, uint64_t* launches);

}  // namespace qv2
