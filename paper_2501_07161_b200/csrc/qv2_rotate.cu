// RMS norm of every head and the rotation by position, queries and keys in one launch.
//
// Bound by its bytes, each read and written once.  A lane has eight elements of a row that are four pairs of the rotation: neighbours, or
// (halves) four elements and the four rot / 2 further on, so nothing but the sum of squares leaves the lane; 8, 16 or 32 lanes hold
// a row of up to 64, 128 or 256.  (Eight neighbouring elements to a lane and the other half by shuffles took 260 instructions for
// them, and the time that those take: 129 us for 16384 tokens of 40 heads x 128 in 16 bits.)  A CTA takes all heads of a few
// tokens and works out the sines and cosines of those tokens once for all heads: the angle is a product of binary64, reduced there to
// a part of a turn, and only then narrowed, so that positions in the millions keep their phase.
//
// 16384 tokens of 32 + 8 heads x 128 in 16 bits (336 MB) take 67 us, 5.0 TB/s: a copy of as much takes 51.  One token of a few sequences is the call's
// host time (14 us).
#include "qv2_serve.cuh"

namespace qv2 {

namespace {

constexpr int kRotateThreads = 256, kRotateRows = 4;       // rows in flight per lane
constexpr uint32_t kRotateMaxTokens = 8;                   // tokens of a CTA

// Four consecutive elements as loaded, and back.
template <class T> struct Quad;
template <> struct Quad<float> {
  float4 a;
  __device__ __forceinline__ void load(const float* p) { a = Chunk8<float>::load4(p); }
  __device__ __forceinline__ void gather(const float* p) { a = make_float4(__ldg(p), __ldg(p + 1), __ldg(p + 2), __ldg(p + 3)); }
  __device__ __forceinline__ void widen(float* v) const { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; }
  static __device__ __forceinline__ void store(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <class T> struct Quad {
  uint32_t w[2];
  __device__ __forceinline__ void load(const T* p) {
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));      // volatile: stays behind dependency_wait()
  }
  __device__ __forceinline__ void gather(const T* p) {
    const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
    w[0] = __ldg(q) | (uint32_t)__ldg(q + 1) << 16; w[1] = __ldg(q + 2) | (uint32_t)__ldg(q + 3) << 16;
  }
  __device__ __forceinline__ void widen(float* v) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
      } else { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
  }
  static __device__ __forceinline__ void store(T* p, const float* v) { *reinterpret_cast<uint2*>(p) = make_uint2(Chunk8<T>::pack(v[0], v[1]), Chunk8<T>::pack(v[2], v[3])); }
};

// QUADS: rows of a multiple of 8 elements, rot / 2 of 4.  Otherwise a lane has eight neighbouring elements and halves meet in shared memory.
// VEC: rows on 16-byte addresses, in and out, strides below 2^20.  (How rows lie changes nothing of what is added to what.)
template <class T, int LPR, bool PAIRS, bool QUADS, bool VEC>
__global__ void __launch_bounds__(kRotateThreads, VEC && LPR == 16 ? 4 : 1)
norm_rotate_kernel(HeadRows h, Rotation r, uint32_t tokens_per_cta, FastDiv heads_q, FastDiv heads_k, FastDiv half_div) {
  extern __shared__ float4 turns_raw[];                    // [token][cosines, sines][pitch], then (halves, not QUADS) a row of binary32 per group of lanes
  float* const turns = reinterpret_cast<float*>(turns_raw);
  constexpr uint32_t GROUPS = kRotateThreads / LPR;
  const uint32_t half = r.rot / 2, c = threadIdx.x % LPR, group = threadIdx.x / LPR;
  const uint64_t token0 = (uint64_t)blockIdx.x * tokens_per_cta;
  const uint32_t tokens = (uint32_t)min((uint64_t)tokens_per_cta, r.tokens - token0);
  const uint32_t pitch = (half + 3) / 4 * 4;               // 16-byte addresses
  float* const row_buf = turns + 2 * tokens_per_cta * pitch + group * LPR * 8;
  // this lane's elements: d0 .. d0 + 3 and d1 .. d1 + 3
  const bool turned = QUADS ? (PAIRS ? 8 * c < r.rot : 4 * c < half) : false;
  const uint32_t d0 = !QUADS || PAIRS ? 8 * c : turned ? 4 * c : r.rot + 8 * (c - half / 4), d1 = QUADS && !PAIRS && turned ? half + 4 * c : d0 + 4;
  const bool in = d0 < r.dim;
  dependency_wait();
  allow_dependents();

  for (uint32_t i = threadIdx.x; i < tokens * half; i += kRotateThreads) {
    const uint32_t t = half_div.div(i), k = i - t * half;
    const double turn = (double)__ldg(r.positions + token0 + t) * (double)__ldg(r.freqs + k) * 0.15915494309189535;   // 1 / (2 pi)
    float s, co;
    sincospif((float)(2.0 * (turn - rint(turn))), &s, &co);
    turns[2 * t * pitch + k] = co;
    turns[(2 * t + 1) * pitch + k] = s;
  }
  __syncthreads();
  const float per = 1.f / (float)r.dim;
  auto run = [&](const int a, const FastDiv& heads) {      // queries, keys
    const uint32_t n_rows = tokens * h.heads[a];
    if (n_rows == 0) return;
    const T* const x = (const T*)h.x[a] + token0 * h.x_token_ld[a];
    T* const y = (T*)h.y[a] + token0 * h.y_token_ld[a];
    using Step = typename std::conditional<VEC, uint32_t, uint64_t>::type;
    const Step xt = (Step)h.x_token_ld[a], xh = (Step)h.x_head_ld[a], yt = (Step)h.y_token_ld[a], yh = (Step)h.y_head_ld[a];
    const float* const weight = h.weight[a];
    float w[8];
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k) {
      const uint32_t d = (k < 4 ? d0 : d1 - 4) + k;
      w[k] = weight && d < r.dim ? __ldg(weight + d) : 1.f;
    }
    for (uint32_t base = 0; base < n_rows; base += kRotateRows * GROUPS) {
      Quad<T> lo[kRotateRows], hi[kRotateRows];
      Chunk8<T> e[kRotateRows];
      uint32_t token[kRotateRows], head[kRotateRows];
#pragma unroll
      for (int u = 0; u < kRotateRows; ++u) {
        // Loads without a branch stay in flight together: rows and elements that are not there take others' (elements become zeros below).
        const uint32_t row = min(base + u * GROUPS + group, n_rows - 1);
        token[u] = heads.div(row);
        head[u] = row - token[u] * heads.d;
        const T* p = x + token[u] * xt + head[u] * xh;
        if (VEC) { lo[u].load(p + (in ? d0 : 0)); hi[u].load(p + (in ? d1 : 0)); }
        else if (QUADS) { lo[u].gather(p + (in ? d0 : 0)); hi[u].gather(p + (in ? d1 : 0)); }
        else {
          e[u].zero();
          if (d0 + 8 <= r.dim) e[u].load_any(p + d0);
          else if (in) e[u].load_some(p + d0, r.dim - d0);
        }
      }
#pragma unroll
      for (int u = 0; u < kRotateRows; ++u) {
        if (base + u * GROUPS >= n_rows) continue;         // the same for all lanes of the CTA
        float v[8];
        if (QUADS) { lo[u].widen(v); hi[u].widen(v + 4); }
        else e[u].widen(v);
        float f = 1.f;
        if (weight) {
          float sum = v[0] * v[0], more = v[1] * v[1];
#pragma unroll
          for (int k = 2; k < 8; k += 2) { sum = fmaf(v[k], v[k], sum); more = fmaf(v[k + 1], v[k + 1], more); }
          sum += more;
          if (QUADS && !in) sum = 0.f;
#pragma unroll
          for (int o = LPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          f = rsqrtf(fmaf(sum, per, r.eps));
#pragma unroll
          for (int k = 0; k < 8; k += 2) mul2(v[k], v[k + 1], w[k], w[k + 1]);
        }
        const float *const co = turns + 2 * token[u] * pitch, *const si = co + pitch;
        if (QUADS) {
          if (turned) {
            const float4 c4 = *reinterpret_cast<const float4*>(co + 4 * c), s4 = *reinterpret_cast<const float4*>(si + 4 * c);
            if (PAIRS) {
              const float ck[4] = {c4.x, c4.y, c4.z, c4.w}, sk[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float p = v[2 * k], q = v[2 * k + 1];
                v[2 * k] = fmaf(p, ck[k], -(q * sk[k]));
                v[2 * k + 1] = fmaf(q, ck[k], p * sk[k]);
              }
            } else {                                       // p cos - q sin, q cos + p sin
              float ps[4] = {v[0], v[1], v[2], v[3]}, qs[4] = {-v[4], -v[5], -v[6], -v[7]};
              mul2(ps[0], ps[1], s4.x, s4.y); mul2(ps[2], ps[3], s4.z, s4.w);
              mul2(qs[0], qs[1], s4.x, s4.y); mul2(qs[2], qs[3], s4.z, s4.w);
              fma2(v[0], v[1], c4.x, c4.y, qs[0], qs[1]); fma2(v[2], v[3], c4.z, c4.w, qs[2], qs[3]);
              fma2(v[4], v[5], c4.x, c4.y, ps[0], ps[1]); fma2(v[6], v[7], c4.z, c4.w, ps[2], ps[3]);
            }
          }
        } else if (PAIRS) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (d0 + 2 * k < r.rot) {
              const float ck = co[d0 / 2 + k], sk = si[d0 / 2 + k], p = v[2 * k], q = v[2 * k + 1];
              v[2 * k] = fmaf(p, ck, -(q * sk));
              v[2 * k + 1] = fmaf(q, ck, p * sk);
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
              const float ck = co[first ? d : d - half], sk = si[first ? d : d - half], q = row_buf[first ? d + half : d - half];
              v[k] = fmaf(v[k], ck, first ? -(q * sk) : q * sk);
            }
          }
          __syncwarp();
        }
        if (weight) {
#pragma unroll
          for (int k = 0; k < 8; k += 2) mul2(v[k], v[k + 1], f, f);
        }
        if (base + u * GROUPS + group < n_rows && in) {
          T* p = y + token[u] * yt + head[u] * yh;
          if (VEC) { Quad<T>::store(p + d0, v); Quad<T>::store(p + d1, v + 4); }
          else if (QUADS) {
#pragma unroll
            for (int k = 0; k < 8; ++k) p[(k < 4 ? d0 : d1 - 4) + k] = Chunk8<T>::narrow(v[k]);
          } else store_some(p + d0, v, r.dim - d0);
        }
      }
    }
  };
  run(0, heads_q);
  run(1, heads_k);
}

template <class T, int LPR>
cudaError_t rotate_rows(const Launch& l, const HeadRows& h, const Rotation& r, uint64_t* launches) {
  const uint32_t half = r.rot / 2;
  const bool quads = r.dim % 8 == 0 && half % 4 == 0;
  uintptr_t where = quads ? 0 : 1;
  for (int a = 0; a < 2; ++a)
    if (h.heads[a]) {
      if ((h.x_token_ld[a] | h.x_head_ld[a] | h.y_token_ld[a] | h.y_head_ld[a]) >> 20 || h.heads[a] > 2048) where |= 1;
      where |= (uintptr_t)h.x[a] | (uintptr_t)h.y[a] | (h.x_token_ld[a] | h.x_head_ld[a] | h.y_token_ld[a] | h.y_head_ld[a]) * sizeof(T);
    }
  const bool vec = where % 16 == 0;
  const uint64_t spread = r.tokens / (8 * (uint64_t)l.sm_count);                 // eight CTAs per SM where there are tokens for them
  const uint32_t tokens = (uint32_t)(spread < 1 ? 1 : spread > kRotateMaxTokens ? kRotateMaxTokens : spread);
  const size_t smem = 2 * sizeof(float) * tokens * ((half + 3) / 4 * 4) + (!quads && !r.pairs ? sizeof(float) * kRotateThreads * 8 : 0);
  auto* kernel = r.pairs ? (vec ? norm_rotate_kernel<T, LPR, true, true, true> : quads ? norm_rotate_kernel<T, LPR, true, true, false> : norm_rotate_kernel<T, LPR, true, false, false>)
                         : (vec ? norm_rotate_kernel<T, LPR, false, true, true> : quads ? norm_rotate_kernel<T, LPR, false, true, false> : norm_rotate_kernel<T, LPR, false, false, false>);
  auto heads = [&](int a) { return FastDiv(h.heads[a] ? h.heads[a] : 1); };
  cudaError_t e = launch_grid(l, kernel, dim3((uint32_t)((r.tokens + tokens - 1) / tokens)), kRotateThreads, smem, h, r, tokens, heads(0), heads(1), FastDiv(half ? half : 1));
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
