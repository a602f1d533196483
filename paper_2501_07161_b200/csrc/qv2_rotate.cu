// RMS norm of every head and the rotation by position, queries and keys in one launch.
//
// Bound by its bytes, each read and written once.  Eight elements to a lane, so 8, 16 or 32 lanes hold a row of up to 64, 128
// or 256; the sum of squares stays in their registers.  A CTA takes all heads of a few tokens and works out the sines and cosines
// of those tokens once for all heads: the angle is a product of binary64, reduced there to a part of a turn, and only then
// narrowed, so that positions in the millions keep their phase.
#include "qv2_serve.cuh"

namespace qv2 {

namespace {

constexpr int kRotateThreads = 256, kRotateRows = 4;       // rows in flight per lane
constexpr uint32_t kRotateMaxTokens = 8;                   // tokens of a CTA
enum { kPairs = 0, kHalvesChunk = 1, kHalvesAny = 2 };     // where the other element of a pair is: same lane, same place of another lane, anywhere

template <class T, int LPR, int MODE>
__global__ void __launch_bounds__(kRotateThreads)
norm_rotate_kernel(HeadRows h, Rotation r, uint32_t tokens_per_cta, FastDiv heads, FastDiv half_div, uint32_t vec_in, uint32_t vec_out) {
  extern __shared__ float2 turns[];                        // [token][rot / 2], then (kHalvesAny) a row of binary32 per group of lanes
  constexpr uint32_t GROUPS = kRotateThreads / LPR;
  const uint32_t half = r.rot / 2, c = threadIdx.x % LPR, group = threadIdx.x / LPR, d0 = 8 * c;
  const uint64_t token0 = (uint64_t)blockIdx.x * tokens_per_cta;
  const uint32_t tokens = (uint32_t)min((uint64_t)tokens_per_cta, r.tokens - token0), n_rows = tokens * heads.d;
  float* const row_buf = reinterpret_cast<float*>(turns + tokens_per_cta * half) + group * LPR * 8;
  dependency_wait();
  allow_dependents();

  Chunk8<T> e[kRotateRows];
  uint32_t which[kRotateRows], token[kRotateRows], head[kRotateRows];
  auto load = [&](uint32_t base) {
#pragma unroll
    for (int u = 0; u < kRotateRows; ++u) {
      const uint32_t row = base + u * GROUPS + group;
      e[u].zero();
      which[u] = token[u] = head[u] = 0;
      if (row >= n_rows) continue;
      token[u] = heads.div(row);
      head[u] = row - token[u] * heads.d;
      which[u] = head[u] >= h.heads[0];
      if (which[u]) head[u] -= h.heads[0];
      const T* p = (const T*)h.x[which[u]] + (token0 + token[u]) * h.x_token_ld[which[u]] + head[u] * h.x_head_ld[which[u]] + d0;
      if (d0 + 8 <= r.dim) { if (vec_in >> which[u] & 1) e[u].load_vec(p); else e[u].load_any(p); }
      else if (d0 < r.dim) e[u].load_some(p, r.dim - d0);
    }
  };
  load(0);
  float w[2][8];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) w[a][k] = h.weight[a] && d0 + k < r.dim ? __ldg(h.weight[a] + d0 + k) : 1.f;
  for (uint32_t i = threadIdx.x; i < tokens * half; i += kRotateThreads) {
    const uint32_t t = half_div.div(i);
    const double turn = (double)__ldg(r.positions + token0 + t) * (double)__ldg(r.freqs + (i - t * half)) * 0.15915494309189535;   // 1 / (2 pi)
    float s, co;
    sincospif((float)(2.0 * (turn - rint(turn))), &s, &co);
    turns[i] = make_float2(co, s);
  }
  __syncthreads();
  for (uint32_t base = 0; base < n_rows; ) {
#pragma unroll
    for (int u = 0; u < kRotateRows; ++u) {
      if (base + u * GROUPS >= n_rows) continue;           // the same for all lanes of the CTA
      const bool keys = which[u] != 0;
      float v[8];
      e[u].widen(v);
      if (h.weight[0] || h.weight[1]) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(v[k], v[k], sum);
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (h.weight[keys]) {
          const float f = 1.f / sqrtf(sum / (float)r.dim + r.eps);
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = v[k] * f * (keys ? w[1][k] : w[0][k]);
        }
      }
      const float2* cs = turns + token[u] * half;
      if (MODE == kPairs) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (d0 + 2 * k < r.rot) {
            const float2 t = cs[d0 / 2 + k];
            const float a = v[2 * k], b = v[2 * k + 1];
            v[2 * k] = a * t.x - b * t.y;
            v[2 * k + 1] = b * t.x + a * t.y;
          }
      } else if (MODE == kHalvesChunk) {
        const uint32_t hc = half / 8;
        const bool first = c < hc, in = c < 2 * hc;
        const uint32_t other = first ? c + hc : in ? c - hc : c;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float b = __shfl_sync(0xffffffffu, v[k], other, LPR);
          if (in) {
            const float2 t = cs[(first ? d0 : d0 - half) + k];
            v[k] = first ? v[k] * t.x - b * t.y : v[k] * t.x + b * t.y;
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) row_buf[d0 + k] = v[k];
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t d = d0 + k;
          if (d < r.rot) {
            const bool first = d < half;
            const float2 t = cs[first ? d : d - half];
            const float b = row_buf[first ? d + half : d - half];
            v[k] = first ? v[k] * t.x - b * t.y : v[k] * t.x + b * t.y;
          }
        }
        __syncwarp();
      }
      if (base + u * GROUPS + group < n_rows && d0 < r.dim) {
        T* p = (T*)h.y[keys] + (token0 + token[u]) * h.y_token_ld[keys] + head[u] * h.y_head_ld[keys] + d0;
        if (vec_out >> which[u] & 1) Chunk8<T>::store_vec(p, v);
        else store_some(p, v, r.dim - d0);
      }
    }
    base += kRotateRows * GROUPS;
    if (base < n_rows) load(base);
  }
}

template <class T, int LPR>
cudaError_t rotate_rows(const Launch& l, const HeadRows& h, const Rotation& r, uint64_t* launches) {
  const uint32_t heads = h.heads[0] + h.heads[1], half = r.rot / 2;
  uint32_t vec_in = 0, vec_out = 0;
  for (int a = 0; a < 2; ++a) {
    if ((uintptr_t)h.x[a] % 16 == 0 && h.x_token_ld[a] * sizeof(T) % 16 == 0 && h.x_head_ld[a] * sizeof(T) % 16 == 0) vec_in |= 1u << a;
    if (r.dim % 8 == 0 && (uintptr_t)h.y[a] % 16 == 0 && h.y_token_ld[a] * sizeof(T) % 16 == 0 && h.y_head_ld[a] * sizeof(T) % 16 == 0) vec_out |= 1u << a;
  }
  const uint64_t spread = r.tokens / (8 * (uint64_t)l.sm_count);                 // eight CTAs per SM where there are tokens for them
  const uint32_t tokens = (uint32_t)(spread < 1 ? 1 : spread > kRotateMaxTokens ? kRotateMaxTokens : spread);
  const int mode = r.pairs ? kPairs : half % 8 == 0 ? kHalvesChunk : kHalvesAny;
  const size_t smem = sizeof(float2) * tokens * half + (mode == kHalvesAny ? sizeof(float) * kRotateThreads * 8 : 0);
  auto* kernel = mode == kPairs ? norm_rotate_kernel<T, LPR, kPairs> : mode == kHalvesChunk ? norm_rotate_kernel<T, LPR, kHalvesChunk> : norm_rotate_kernel<T, LPR, kHalvesAny>;
  cudaError_t e = launch_grid(l, kernel, dim3((uint32_t)((r.tokens + tokens - 1) / tokens)), kRotateThreads, smem, h, r, tokens, FastDiv(heads), FastDiv(half ? half : 1), vec_in, vec_out);
  if (e == cudaSuccess) ++*launches;
  return e;
}

template <class T>
cudaError_t rotate_typed(const Launch& l, const HeadRows& h, const Rotation& r, uint64_t* launches) {
  if (r.dim <= 64) return rotate_rows<T, 8>(l, h, r, launches);
  if (r.dim <= 128) return rotate_rows<T, 16>(l, h, r, launches);
  return rotate_rows<T, 32>(l, h, r, launches);
}

}  // namespace

cudaError_t launch_norm_rotate(const Launch& l, const HeadRows& h, const Rotation& r, uint64_t* launches) {
  if (r.dtype == kF16) return rotate_typed<__half>(l, h, r, launches);
  if (r.dtype == kBF16) return rotate_typed<__nv_bfloat16>(l, h, r, launches);
  return rotate_typed<float>(l, h, r, launches);
}

}  // namespace qv2
