// Page planning, norm with rotation, and attention over the cache: what their kernels are given, and the launch wrappers.
#pragma once

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

struct AttendArgs {
  KvView c;
  const void* q;
  uint64_t q_token_ld, q_head_ld;
  uint32_t q_heads, group, total, seqs;
  const int64_t *starts, *lens;
  const int32_t* table;
  uint64_t table_ld;
  float scale, cap;
  int64_t window;                 // 2^62: none
  const float* slopes;
  void* out;
  float* lse;
  uint32_t dtype, max_new;
};
cudaError_t launch_kv_attend(const Launch& l, const AttendArgs& a, uint64_t* launches);

// Sequence s of a call: its rows of q, and its length; lengths are held to 2^40.
struct AttendSeq {
  uint32_t row0, n;
  int64_t len;
};
__device__ __forceinline__ AttendSeq attend_seq(const AttendArgs& a, uint32_t s) {
  const int64_t total = a.total, lo = min(max(__ldg(a.starts + s), (int64_t)0), total), hi = min(max(__ldg(a.starts + s + 1), lo), total);
  AttendSeq r;
  r.row0 = (uint32_t)lo;
  r.n = (uint32_t)(hi - lo);
  r.len = min(max(__ldg(a.lens + s), (int64_t)0), (int64_t)1 << 40);
  return r;
}

}  // namespace qv2
