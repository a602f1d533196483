// Attention of new tokens over the quantized paged cache.
#include "qv2_serve.cuh"

namespace qv2 {

namespace {

constexpr uint32_t kAttendThreads = 256;

template <class T> __device__ __forceinline__ float widen1(T v);
template <> __device__ __forceinline__ float widen1(float v) { return v; }
template <> __device__ __forceinline__ float widen1(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float widen1(__nv_bfloat16 v) { return __bfloat162float(v); }

// Element d of a cached row.
template <int FORMAT>
__device__ __forceinline__ float cached(const KvView& c, int which, uint64_t at, uint32_t d, uint32_t blocks) {
  if (FORMAT == QV2_KV_I8) return (float)(int8_t)__ldg(c.codes[which] + at * c.dim + d) * __ldg(reinterpret_cast<const float*>(c.scales[which]) + at);
  const uint32_t code = __ldg(c.codes[which] + at * 16 * blocks + d / 2) >> (4 * (d & 1));
  float v[8];
  mx_decode8(code & 15u, mx_scale(__ldg(c.scales[which] + at * blocks + d / 32)), v);
  return v[0];
}

// A CTA has one query head of one sequence, a warp one query at a time; lane l holds elements l, l + 32, ...
template <class T, int FORMAT>
__global__ void __launch_bounds__(kAttendThreads) attend_simple_kernel(AttendArgs a, FastDiv page) {
  dependency_wait();
  allow_dependents();
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, head = blockIdx.x, kv = head / a.group, blocks = (a.c.dim + 31) / 32;
  const AttendSeq s = attend_seq(a, blockIdx.y);
  const int64_t room = (int64_t)a.table_ld * page.d;
  const float slope = a.slopes ? __ldg(a.slopes + head) : 0.f;
  for (uint32_t i = warp; i < s.n; i += kAttendThreads / 32) {
    const uint64_t row = s.row0 + i;
    const int64_t pos = s.len - s.n + i, j0 = max(pos - a.window + 1, (int64_t)0), j1 = min(pos + 1, room);
    float q[8], o[8], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t d = lane + 32 * k;
      q[k] = d < a.c.dim ? widen1<T>(((const T*)a.q)[row * a.q_token_ld + head * a.q_head_ld + d]) : 0.f;
      o[k] = 0.f;
    }
    for (int64_t j = j0; j < j1; ++j) {
      const uint32_t pg = page.div((uint32_t)j);
      const int32_t id = __ldg(a.table + blockIdx.y * a.table_ld + pg);
      if (id < 0 || (uint32_t)id >= a.c.pages) continue;
      const uint64_t at = ((uint64_t)id * page.d + ((uint32_t)j - pg * page.d)) * a.c.heads + kv;
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (lane + 32 * k < a.c.dim) x = fmaf(q[k], cached<FORMAT>(a.c, 0, at, lane + 32 * k, blocks), x);
#pragma unroll
      for (int b = 16; b > 0; b >>= 1) x += __shfl_xor_sync(0xffffffffu, x, b);
      x *= a.scale;
      if (a.cap > 0.f) x = a.cap * tanhf(x / a.cap);
      x += slope * (float)(j - pos);
      float v[8];
      bool bad = false;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        v[k] = lane + 32 * k < a.c.dim ? cached<FORMAT>(a.c, 1, at, lane + 32 * k, blocks) : 0.f;
        bad |= isnan(v[k]);
      }
      const float poison = __any_sync(0xffffffffu, bad) ? NAN : 0.f;
      const float now = isnan(x) ? x : fmaxf(top, x), was = top == -INFINITY ? 0.f : expf(top - now), p = expf(x - now);
      top = now;
      sum = sum * was + p;
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = fmaf(p, v[k] + poison, o[k] * was);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (lane + 32 * k < a.c.dim) ((T*)a.out)[(row * a.q_heads + head) * a.c.dim + lane + 32 * k] = Chunk8<T>::narrow(sum == 0.f ? 0.f : o[k] / sum);
    if (a.lse && lane == 0) a.lse[row * a.q_heads + head] = sum == 0.f ? -INFINITY : top + logf(sum);
  }
}

template <class T>
cudaError_t attend_typed(const Launch& l, const AttendArgs& a, uint64_t* launches) {
  auto* kernel = a.c.format == QV2_KV_MX4 ? attend_simple_kernel<T, QV2_KV_MX4> : attend_simple_kernel<T, QV2_KV_I8>;
  cudaError_t e = launch_grid(l, kernel, dim3(a.q_heads, a.seqs), kAttendThreads, 0, a, FastDiv(a.c.page_size));
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace

cudaError_t launch_kv_attend(const Launch& l, const AttendArgs& a, uint64_t* launches) {
  if (a.dtype == kF16) return attend_typed<__half>(l, a, launches);
  if (a.dtype == kBF16) return attend_typed<__nv_bfloat16>(l, a, launches);
  return attend_typed<float>(l, a, launches);
}

}  // namespace qv2
