// Microscaled 4-bit format and quantized cache: device helpers shared by their kernels, and the
// launch wrappers that the C-ABI layer calls.
#pragma once

#include "qv2_device.cuh"

namespace qv2 {

// n / d for n < 2^31 by one wide multiplication: with s = ceil(log2 d) and m = ceil(2^(31+s) / d),
// m < 2^32 and m*d - 2^(31+s) < 2^s, so n*m exceeds n*2^(31+s)/d by less than 2^(31+s)/d and the
// shifted product is the quotient.
struct FastDiv {
  uint32_t d = 1, m = 1u << 31, s = 31;
  FastDiv() = default;
  explicit FastDiv(uint32_t div) : d(div) {
    uint32_t k = 0;
    while ((1ull << k) < div) ++k;
    s = 31 + k;
    m = (uint32_t)(((1ull << s) + div - 1) / div);
  }
  __host__ __device__ __forceinline__ uint32_t div(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> s); }
};

// launch_kernel for grids of more than one dimension and kernels with dynamic shared memory.
template <class... KArgs, class... Args>
inline cudaError_t launch_grid(const Launch& l, void (*kernel)(KArgs...), dim3 grid, uint32_t block, size_t smem, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = l.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = l.pdl ? 1u : 0u;
  return cudaLaunchKernelEx(&cfg, kernel, KArgs(static_cast<Args&&>(args))...);
}

struct MxView {                  // qv2_mx_matrix as the kernels see it
  uint8_t* codes; uint8_t* scales;
  uint64_t codes_ld, scales_ld, codes_gs, scales_gs;
};

// NW words from p, whatever its alignment (a multiple of 2): aligned 16-byte loads, each of which holds at least one
// of the wanted bytes, shifted into place.
template <int NW>
__device__ __forceinline__ void load_shifted(uint32_t (&out)[NW], const void* p) {
  const uint32_t off = (uint32_t)((uintptr_t)p & 15u);
  const uint4* q = reinterpret_cast<const uint4*>((uintptr_t)p & ~(uintptr_t)15u);
  uint32_t w[NW + 4];
#pragma unroll
  for (int i = 0; i <= NW / 4; ++i) {
    const uint4 v = i < NW / 4 || off ? __ldg(q + i) : make_uint4(0, 0, 0, 0);
    w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
  }
  if (off & 8u)
#pragma unroll
    for (int i = 0; i < NW + 2; ++i) w[i] = w[i + 2];
  if (off & 4u)
#pragma unroll
    for (int i = 0; i < NW + 1; ++i) w[i] = w[i + 1];
#pragma unroll
  for (int i = 0; i < NW; ++i) out[i] = __funnelshift_r(w[i], w[i + 1], 8 * (off & 3u));
}

// --- eight consecutive elements, as loaded ---------------------------------------------------------
template <class T> struct Chunk8;
template <> struct Chunk8<float> {
  float4 a, b;
  static __device__ __forceinline__ float4 load4(const float* p) {     // volatile: stays behind dependency_wait()
    float4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
    return v;
  }
  __device__ __forceinline__ void load_vec(const float* p) { a = load4(p); b = load4(p + 4); }
  __device__ __forceinline__ void load_any(const float* p) {
    uint32_t w[8];
    load_shifted<8>(w, p);
    a = make_float4(__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3]));
    b = make_float4(__uint_as_float(w[4]), __uint_as_float(w[5]), __uint_as_float(w[6]), __uint_as_float(w[7]));
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load_some(const float* p, uint32_t n) {
    float* e = &a.x; float* f = &b.x;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) { e[i] = i < n ? p[i] : 0.f; f[i] = i + 4 < n ? p[i + 4] : 0.f; }
  }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  // Largest magnitude as the bits of a binary32 (which order like the numbers, with infinity and
  // NaN above every finite value).
  __device__ __forceinline__ uint32_t top_bits() const {
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
  }
  static __device__ __forceinline__ void store_vec(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
  static __device__ __forceinline__ float narrow(float v) { return v; }
};
struct Chunk8Half {              // the two 16-bit types: four words of two elements
  uint32_t w[4];
  __device__ __forceinline__ void load_words(const void* p) {
    // volatile: stays behind dependency_wait()
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
  }
  __device__ __forceinline__ void load_any(const void* p) { load_shifted<4>(w, p); }
  __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
  __device__ __forceinline__ void load_halves(const unsigned short* p, uint32_t n) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      w[i] = (2 * i < n ? (uint32_t)p[2 * i] : 0u) | ((2 * i + 1 < n ? (uint32_t)p[2 * i + 1] : 0u) << 16);
  }
  __device__ __forceinline__ uint32_t top16() const {
    uint32_t m = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16);
  }
};
template <> struct Chunk8<__nv_bfloat16> : Chunk8Half {
  __device__ __forceinline__ void load_vec(const __nv_bfloat16* p) { load_words(p); }
  __device__ __forceinline__ void load_some(const __nv_bfloat16* p, uint32_t n) { load_halves(reinterpret_cast<const unsigned short*>(p), n); }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  __device__ __forceinline__ uint32_t top_bits() const { return top16() << 16; }
  static __device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pack(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); }
  static __device__ __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Chunk8<__half> : Chunk8Half {
  __device__ __forceinline__ void load_vec(const __half* p) { load_words(p); }
  __device__ __forceinline__ void load_some(const __half* p, uint32_t n) { load_halves(reinterpret_cast<const unsigned short*>(p), n); }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
  }
  __device__ __forceinline__ uint32_t top_bits() const {
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)top16()))) & 0x7fffffffu;
  }
  static __device__ __forceinline__ void store_vec(__half* p, const float (&v)[8]) {
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pack(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); }
  static __device__ __forceinline__ __half narrow(float v) { return __float2half_rn(v); }
};
template <class T>
__device__ __forceinline__ void store_some(T* p, const float (&v)[8], uint32_t n) {
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i)
    if (i < n) p[i] = Chunk8<T>::narrow(v[i]);
}

// Sixteen results as whole 32-byte sectors; p is 32-byte aligned.
__device__ __forceinline__ void store_sector(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
template <class T>
__device__ __forceinline__ void store_sectors(T* p, const float (&a)[8], const float (&b)[8]) {
  uint32_t w[8];
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(a[i]);
    store_sector(p, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(b[i]);
    store_sector(p + 8, w);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) { w[i] = Chunk8<T>::pack(a[2 * i], a[2 * i + 1]); w[4 + i] = Chunk8<T>::pack(b[2 * i], b[2 * i + 1]); }
    store_sector(p, w);
  }
}

// --- the 4-bit format ------------------------------------------------------------------------------
// Scale byte of a block from the bits of its largest magnitude.  The exponent field of a binary32
// is floor(log2) + 127 for normal numbers and 0 below them, so floor(log2 A) - 2 + 127 is the
// field less 2, held at 0 from below; the field of infinities and NaN, 255, is passed on.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top_bits) {
  const uint32_t field = top_bits >> 23;
  return field == 255u ? 255u : (field > 2u ? field - 2u : 0u);
}
// 2^(byte - 127); NaN for byte 255.
__device__ __forceinline__ float mx_scale(uint32_t byte) {
  return __uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
}
// Codes of eight elements of a block, element i in bits 4i .. 4i+3.  The multiplication by
// 2^(127 - byte) is exact wherever it matters: it is a shift of the exponent, and what underflows
// is far below the smallest midpoint 0.25.  (byte <= 252 for a finite block, so the factor is normal.)
__device__ __forceinline__ uint32_t mx_encode8(const float (&v)[8], uint32_t byte) {
  if (byte == 255u) return 0u;
  const float r = __uint_as_float((254u - byte) << 23);
  uint32_t out;
  asm("{\n\t.reg .b8 c0, c1, c2, c3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c3, %8, %7;\n\t"
      "mov.b32 %0, {c0, c1, c2, c3};\n\t}"
      : "=r"(out)
      : "f"(v[0] * r), "f"(v[1] * r), "f"(v[2] * r), "f"(v[3] * r), "f"(v[4] * r), "f"(v[5] * r), "f"(v[6] * r), "f"(v[7] * r));
  return out;
}
// The eight numbers that the codes stand for, times `scale` (exact unless it leaves binary32's range).
__device__ __forceinline__ void mx_decode8(uint32_t codes, float scale, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 c0, c1, c2, c3;\n\t"
      "mov.b32 {c0, c1, c2, c3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, c0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, c1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, c3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = f.x * scale; v[2 * i + 1] = f.y * scale;
  }
}

// --- launch wrappers -------------------------------------------------------------------------------
cudaError_t launch_mx_quantize(const Launch& l, const void* x, uint32_t dtype, uint64_t x_ld, uint64_t rows, uint32_t cols,
                               const MxView& out, void* values, uint64_t values_ld, uint64_t* launches);
cudaError_t launch_mx_dequantize(const Launch& l, const MxView& m, uint64_t groups, uint64_t rows, uint32_t cols, void* y,
                                 uint32_t dtype, uint64_t y_ld, uint64_t* launches);
struct MxProduct {
  MxView a, w;
  const float* bias; const int64_t* offsets;
  void* y; uint64_t y_ld;
  uint32_t dtype, m, n, k, groups;
  uint32_t early;        // only `a` may still be on its way when the launch begins (see mx_matmul_kernel)
  uint32_t* fault;       // host-mapped word, set when a kernel gave up waiting
};
cudaError_t launch_mx_matmul(const Launch& l, const MxProduct& p, uint64_t* launches);
uint32_t mx_product_form(uint32_t m, uint32_t n, uint32_t groups, uint32_t sm_count, uint64_t* tiles);

struct KvView {
  uint8_t* codes[2]; uint8_t* scales[2];       // keys, values
  uint64_t slots;
  uint32_t pages, page_size, heads, dim, format;
};
struct KvNew {
  const void* x[2]; uint64_t token_ld[2], head_ld[2];
  const int64_t* slots;
  uint64_t tokens;
  uint32_t dtype;
};
struct KvRead {
  const int32_t* table; uint64_t table_ld;
  const int64_t* starts;
  uint32_t seqs;
  uint64_t total;
  void* y[2];
  uint32_t dtype;
};
cudaError_t launch_kv_write(const Launch& l, const KvView& c, const KvNew& n, uint64_t* launches);
cudaError_t launch_kv_read(const Launch& l, const KvView& c, const KvRead& r, uint64_t* launches);

}  // namespace qv2
