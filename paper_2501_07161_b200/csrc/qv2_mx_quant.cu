// Rounding rows to the microscaled 4-bit format and back.  Both are one pass over the data: four
// lanes share a block of 32 elements, eight consecutive elements each, so that a warp reads and
// writes runs of consecutive bytes, and the block's largest magnitude takes two shuffles.  Bound by
// memory: 16384 x 8192 bfloat16 elements with their values (608 MB) take 93 us = 6.5 TB/s, the copy rate;
// 1001 x 25088 binary32 ones (214 MB) 34 us (back to back, at the clocks that hold then, 102 and 35).  Rows on any
// address are loaded twice over (load_shifted): 8192 x 8191 codes 46 us beside 33 us aligned, with values 93 beside
// 52; dequantized to them, element by element, 187 us beside 26 us for the bytes.
#include "qv2_mx.cuh"

namespace qv2 {

namespace {

constexpr uint32_t kMxThreads = 256;

// Work item i: chunk i % cpr of row i / cpr, cpr = 4 * blocks per row; n_items is a multiple of 4,
// so the four lanes of a block are all in range or all out of it.
template <class T, bool VEC, bool VALUES, int U>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const T* x, uint64_t x_ld, uint32_t cols, FastDiv cpr, uint32_t n_items, MxView out, T* values,
                   uint64_t values_ld) {
  dependency_wait();
  allow_dependents();
  const uint32_t base = blockIdx.x * (kMxThreads * U) + threadIdx.x;
  Chunk8<T> e[U];
  uint32_t row[U], c[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = base + u * kMxThreads;
    row[u] = cpr.div(i); c[u] = i - row[u] * cpr.d;
    e[u].zero();
    if (i < n_items) {
      const T* p = x + row[u] * x_ld + 8ull * c[u];
      if (c[u] * 8 + 8 <= cols) { if (VEC) e[u].load_vec(p); else e[u].load_any(p); }
      else if (c[u] * 8 < cols) e[u].load_some(p, cols - c[u] * 8);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t top = e[u].top_bits();
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t byte = mx_scale_byte(top);
    float v[8];
    e[u].widen(v);
    const uint32_t codes = mx_encode8(v, byte);
    if (base + u * kMxThreads < n_items) {
      *reinterpret_cast<uint32_t*>(out.codes + row[u] * out.codes_ld + 4ull * c[u]) = codes;
      if ((c[u] & 3u) == 0) out.scales[row[u] * out.scales_ld + (c[u] >> 2)] = (uint8_t)byte;
      if (VALUES) {
        mx_decode8(codes, mx_scale(byte), v);
        T* q = values + row[u] * values_ld + 8ull * c[u];
        if (VEC) {
          if (c[u] * 8 + 8 <= cols) Chunk8<T>::store_vec(q, v);
          else if (c[u] * 8 < cols) store_some(q, v, cols - c[u] * 8);
        }
      }
    }
    if (VALUES && !VEC) {
      // Rows on any address: the warp's 256 results change places so that neighbouring lanes store neighbouring elements.
      __shared__ T swap[kMxThreads * 8];
      T* const mine = swap + (threadIdx.x & ~31u) * 8;
      const uint32_t lane = threadIdx.x % 32;
#pragma unroll
      for (int k = 0; k < 8; ++k) mine[8 * lane + k] = Chunk8<T>::narrow(v[k]);
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t from = 4 * k + lane / 8;
        const uint32_t r = __shfl_sync(0xffffffffu, row[u], from), col = 8 * __shfl_sync(0xffffffffu, c[u], from) + lane % 8;
        const bool in = base - lane + from + u * kMxThreads < n_items;
        if (in && col < cols) values[r * values_ld + col] = mine[32 * k + lane];
      }
      __syncwarp();
    }
  }
}

template <class T, bool VEC, int U>
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize_kernel(MxView m, uint64_t row0, FastDiv cpr, FastDiv rows_of_group, uint32_t group0, uint32_t row_in_group0,
                     uint32_t cols, uint32_t n_items, T* y, uint64_t y_ld) {
  dependency_wait();
  allow_dependents();
  const uint32_t base = blockIdx.x * (kMxThreads * U) + threadIdx.x;
  uint32_t codes[U], byte[U];
  uint32_t row[U], c[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = base + u * kMxThreads;
    row[u] = cpr.div(i); c[u] = i - row[u] * cpr.d;
    codes[u] = 0; byte[u] = 0;
    if (i < n_items) {
      const uint32_t r = row[u] + row_in_group0, g = rows_of_group.div(r);
      const uint64_t group = group0 + g, rg = r - g * rows_of_group.d;
      codes[u] = __ldg(reinterpret_cast<const uint32_t*>(m.codes + group * m.codes_gs + rg * m.codes_ld) + c[u]);
      byte[u] = __ldg(m.scales + group * m.scales_gs + rg * m.scales_ld + (c[u] >> 2));
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (base + u * kMxThreads >= n_items) continue;
    float v[8];
    mx_decode8(codes[u], mx_scale(byte[u]), v);
    T* q = y + (row0 + row[u]) * y_ld + 8ull * c[u];
    if (VEC && c[u] * 8 + 8 <= cols) Chunk8<T>::store_vec(q, v);
    else if (c[u] * 8 < cols) store_some(q, v, cols - c[u] * 8);
  }
}

// Item numbers stay below 2^31: rows are taken in slices of that many items.
uint64_t slice_rows(uint32_t cpr) { return (1ull << 30) / cpr; }

template <class T, bool VEC, bool VALUES>
cudaError_t quantize_slices(const Launch& l, const T* x, uint64_t x_ld, uint64_t rows, uint32_t cols, const MxView& out, T* values,
                            uint64_t values_ld, uint64_t* launches) {
  const uint32_t cpr = 4 * ((cols + 31) / 32);
  const uint64_t step = slice_rows(cpr);
  for (uint64_t r = 0; r < rows; r += step) {
    const uint64_t n_rows = rows - r < step ? rows - r : step;
    const uint32_t n = (uint32_t)(n_rows * cpr);
    MxView o = out;
    o.codes += r * out.codes_ld; o.scales += r * out.scales_ld;
    const T* xs = x + r * x_ld;
    T* vs = VALUES ? values + r * values_ld : nullptr;
    // Few items: one per thread spreads them over more SMs; many: four loads in flight per thread.
    cudaError_t e;
    if (n <= (uint32_t)l.sm_count * 8u * kMxThreads)
      e = launch_kernel(l, mx_quantize_kernel<T, VEC, VALUES, 1>, (n + kMxThreads - 1) / kMxThreads, kMxThreads, xs, x_ld, cols, FastDiv(cpr), n, o, vs, values_ld);
    else
      e = launch_kernel(l, mx_quantize_kernel<T, VEC, VALUES, 4>, (n + 4 * kMxThreads - 1) / (4 * kMxThreads), kMxThreads, xs, x_ld, cols, FastDiv(cpr), n, o, vs, values_ld);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

template <class T>
cudaError_t quantize_typed(const Launch& l, const void* x, uint64_t x_ld, uint64_t rows, uint32_t cols, const MxView& out, void* values,
                           uint64_t values_ld, uint64_t* launches) {
  const T* xt = (const T*)x; T* vt = (T*)values;
  const bool vec = ((uintptr_t)x % 16 == 0) && (x_ld * sizeof(T)) % 16 == 0 && ((uintptr_t)values % 16 == 0) && (!values || (values_ld * sizeof(T)) % 16 == 0);
  if (values)
    return vec ? quantize_slices<T, true, true>(l, xt, x_ld, rows, cols, out, vt, values_ld, launches)
               : quantize_slices<T, false, true>(l, xt, x_ld, rows, cols, out, vt, values_ld, launches);
  return vec ? quantize_slices<T, true, false>(l, xt, x_ld, rows, cols, out, vt, values_ld, launches)
             : quantize_slices<T, false, false>(l, xt, x_ld, rows, cols, out, vt, values_ld, launches);
}

template <class T, bool VEC>
cudaError_t dequantize_slices(const Launch& l, const MxView& m, uint64_t all_rows, uint32_t group_rows, uint32_t cols, T* y, uint64_t y_ld,
                              uint64_t* launches) {
  const uint32_t cpr = 4 * ((cols + 31) / 32);
  const uint64_t step = slice_rows(cpr);
  for (uint64_t r = 0; r < all_rows; r += step) {
    const uint64_t n_rows = all_rows - r < step ? all_rows - r : step;
    const uint32_t n = (uint32_t)(n_rows * cpr);
    const uint32_t g0 = (uint32_t)(r / group_rows), in0 = (uint32_t)(r % group_rows);
    cudaError_t e = launch_kernel(l, mx_dequantize_kernel<T, VEC, 4>, (n + 4 * kMxThreads - 1) / (4 * kMxThreads), kMxThreads, m, r, FastDiv(cpr),
                                  FastDiv(group_rows), g0, in0, cols, n, y, y_ld);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

template <class T>
cudaError_t dequantize_typed(const Launch& l, const MxView& m, uint64_t all_rows, uint32_t group_rows, uint32_t cols, void* y, uint64_t y_ld,
                             uint64_t* launches) {
  const bool vec = ((uintptr_t)y % 16 == 0) && (y_ld * sizeof(T)) % 16 == 0;
  return vec ? dequantize_slices<T, true>(l, m, all_rows, group_rows, cols, (T*)y, y_ld, launches)
             : dequantize_slices<T, false>(l, m, all_rows, group_rows, cols, (T*)y, y_ld, launches);
}

}  // namespace

cudaError_t launch_mx_quantize(const Launch& l, const void* x, uint32_t dtype, uint64_t x_ld, uint64_t rows, uint32_t cols,
                               const MxView& out, void* values, uint64_t values_ld, uint64_t* launches) {
  if (dtype == kF16) return quantize_typed<__half>(l, x, x_ld, rows, cols, out, values, values_ld, launches);
  if (dtype == kBF16) return quantize_typed<__nv_bfloat16>(l, x, x_ld, rows, cols, out, values, values_ld, launches);
  return quantize_typed<float>(l, x, x_ld, rows, cols, out, values, values_ld, launches);
}

cudaError_t launch_mx_dequantize(const Launch& l, const MxView& m, uint64_t groups, uint64_t rows, uint32_t cols, void* y,
                                 uint32_t dtype, uint64_t y_ld, uint64_t* launches) {
  const uint64_t all = groups * rows;
  if (dtype == kF16) return dequantize_typed<__half>(l, m, all, (uint32_t)rows, cols, y, y_ld, launches);
  if (dtype == kBF16) return dequantize_typed<__nv_bfloat16>(l, m, all, (uint32_t)rows, cols, y, y_ld, launches);
  return dequantize_typed<float>(l, m, all, (uint32_t)rows, cols, y, y_ld, launches);
}

}  // namespace qv2
