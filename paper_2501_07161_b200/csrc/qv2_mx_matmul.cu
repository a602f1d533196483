// Products of microscaled 4-bit matrices, dense and grouped by expert.
#include "qv2_mx.cuh"

namespace qv2 {

namespace {

constexpr int kTile = 64;

// Rows [begin, end) of group g.  Offsets are clamped to 0..m and never decrease, whatever the caller passed.
__device__ __forceinline__ void store_one(void* y, uint64_t at, uint32_t dtype, float v) {
  if (dtype == kF16) ((__half*)y)[at] = __float2half_rn(v);
  else if (dtype == kBF16) ((__nv_bfloat16*)y)[at] = __float2bfloat16_rn(v);
  else ((float*)y)[at] = v;
}

// One CTA per 64 x 64 tile of y: blocks of 32 columns are decoded into shared memory and multiplied.
// blockIdx.y numbers the row tiles of all groups one after the other.
__global__ void __launch_bounds__(256) mx_matmul_kernel(MxProduct p) {
  __shared__ float sa[kTile][33], sw[kTile][33];
  dependency_wait();
  allow_dependents();
  uint32_t g = 0, row0 = 0, row_end = p.m, tile = blockIdx.y;
  if (p.offsets) {
    int64_t lo = min(max(__ldg(p.offsets), (int64_t)0), (int64_t)p.m);
    for (;; ++g) {
      if (g == p.groups) return;
      int64_t hi = min(max(__ldg(p.offsets + g + 1), lo), (int64_t)p.m);
      const uint32_t tiles = (uint32_t)((hi - lo + kTile - 1) / kTile);
      if (tile < tiles) { row0 = (uint32_t)lo + tile * kTile; row_end = (uint32_t)hi; break; }
      tile -= tiles;
      lo = hi;
    }
  } else {
    row0 = tile * kTile;
  }
  const uint32_t col0 = blockIdx.x * kTile;
  const uint32_t blocks = (p.k + 31) / 32;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  for (uint32_t b = 0; b < blocks; ++b) {
    for (uint32_t i = threadIdx.x; i < 2 * kTile * 4; i += 256) {
      const bool is_w = i >= kTile * 4;
      const uint32_t r = (i / 4) % kTile, ch = i % 4;
      const MxView& v = is_w ? p.w : p.a;
      const uint64_t row = is_w ? col0 + r : row0 + r;
      const bool in = is_w ? row < p.n : row < row_end;
      float f[8] = {};
      if (in) {
        const uint64_t base = is_w ? (uint64_t)g * v.codes_gs : 0, sbase = is_w ? (uint64_t)g * v.scales_gs : 0;
        const uint32_t c = *reinterpret_cast<const uint32_t*>(v.codes + base + row * v.codes_ld + 16ull * b + 4 * ch);
        mx_decode8(c, mx_scale(v.scales[sbase + row * v.scales_ld + b]), f);
      }
      float* dst = (is_w ? sw[r] : sa[r]) + 8 * ch;
#pragma unroll
      for (int k = 0; k < 8; ++k) dst[k] = f[k];
    }
    __syncthreads();
    for (int k = 0; k < 32; ++k) {
      float av[4], wv[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) { av[i] = sa[ty + 16 * i][k]; wv[i] = sw[tx + 16 * i][k]; }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], wv[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t r = row0 + ty + 16 * i, n = col0 + tx + 16 * j;
      if (r < row_end && n < p.n)
        store_one(p.y, r * p.y_ld + n, p.dtype, acc[i][j] + (p.bias ? p.bias[(uint64_t)g * p.n + n] : 0.0f));
    }
}

}  // namespace

cudaError_t launch_mx_matmul(const Launch& l, const MxProduct& p, uint64_t* launches) {
  const uint32_t row_tiles = (p.m + kTile - 1) / kTile + (p.offsets ? p.groups : 0);
  if (row_tiles > 65535u) return cudaErrorInvalidValue;
  cudaError_t e = launch_grid(l, mx_matmul_kernel, dim3((p.n + kTile - 1) / kTile, row_tiles), 256, 0, p);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace qv2
