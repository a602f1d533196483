// The quantized key / value cache: rows of one head rounded on their way into their slots, and
// whole sequences gathered back through a page table.  Both directions are bound by the bytes of
// the unquantized side (256 of 256 + 68 bytes per row of 128 bfloat16 elements at 4 bits).
#include "qv2_mx.cuh"

namespace qv2 {

namespace {

constexpr uint32_t kKvThreads = 256;

// ---------------------------------------------------------------------------------- writing, 4 bits
// Work item: eight elements, as in mx_quantize_kernel; blockIdx.y picks keys or values.
template <class T>
__global__ void __launch_bounds__(kKvThreads)
kv_write_mx4_kernel(KvView c, KvNew n, uint64_t token0, FastDiv cpr, FastDiv heads, uint32_t n_items, bool vec_k, bool vec_v) {
  dependency_wait();
  allow_dependents();
  const uint32_t which = blockIdx.y;
  const bool vec = which ? vec_v : vec_k;
  const uint32_t i = blockIdx.x * kKvThreads + threadIdx.x;
  const uint32_t row = cpr.div(i), ch = i - row * cpr.d;
  const uint32_t t = heads.div(row), h = row - t * heads.d;
  Chunk8<T> e;
  e.zero();
  int64_t slot = -1;
  if (i < n_items) {
    slot = __ldg(n.slots + token0 + t);
    const T* p = (const T*)n.x[which] + (token0 + t) * n.token_ld[which] + h * n.head_ld[which] + 8ull * ch;
    if (vec && ch * 8 + 8 <= c.dim) e.load_vec(p);
    else if (ch * 8 < c.dim) e.load_some(p, c.dim - ch * 8);
  }
  uint32_t top = e.top_bits();
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t byte = mx_scale_byte(top);
  float v[8];
  e.widen(v);
  const uint32_t codes = mx_encode8(v, byte);
  if (slot < 0 || (uint64_t)slot >= c.slots) return;
  const uint64_t at = (uint64_t)slot * c.heads + h;
  reinterpret_cast<uint32_t*>(c.codes[which])[at * cpr.d + ch] = codes;
  if ((ch & 3u) == 0) c.scales[which][at * (cpr.d >> 2) + (ch >> 2)] = (uint8_t)byte;
}

// ---------------------------------------------------------------------------------- writing, 8 bits
// LPR lanes share a row; a row of more than 8 * LPR elements (LPR = 32, head_dim > 256) is walked
// twice, the second time out of L1.
template <class T, int LPR>
__global__ void __launch_bounds__(kKvThreads)
kv_write_i8_kernel(KvView c, KvNew n, uint64_t token0, FastDiv heads, uint32_t n_rows, bool vec_k, bool vec_v) {
  dependency_wait();
  allow_dependents();
  const uint32_t which = blockIdx.y;
  const bool vec = which ? vec_v : vec_k;
  const uint32_t lane = threadIdx.x % LPR;
  const uint32_t row = blockIdx.x * (kKvThreads / LPR) + threadIdx.x / LPR;
  const uint32_t t = heads.div(row), h = row - t * heads.d;
  const bool in = row < n_rows;
  const T* p = (const T*)n.x[which] + (token0 + t) * n.token_ld[which] + h * n.head_ld[which];
  const int64_t slot = in ? __ldg(n.slots + token0 + t) : -1;
  auto load = [&](Chunk8<T>& e, uint32_t d) {
    e.zero();
    if (!in || d >= c.dim) return;
    if (vec && d + 8 <= c.dim) e.load_vec(p + d);
    else e.load_some(p + d, c.dim - d);
  };
  Chunk8<T> e;
  load(e, 8 * lane);
  uint32_t top = e.top_bits();
  for (uint32_t d = 8 * (lane + LPR); d < c.dim; d += 8 * LPR) {
    Chunk8<T> more;
    load(more, d);
    top = max(top, more.top_bits());
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (slot < 0 || (uint64_t)slot >= c.slots) return;
  const float R = __uint_as_float(top);
  float step = __fdiv_rn(R, 127.0f), inv = __fdiv_rn(127.0f, R);
  const bool finite = top < 0x7f800000u;
  if (finite && (!(R > 0.0f) || !isfinite(inv) || !(step > 0.0f))) { step = 1.0f; inv = 1.0f; }
  const uint64_t at = (uint64_t)slot * c.heads + h;
  uint8_t* q = c.codes[which] + at * c.dim;
  const bool vec_out = (c.dim % 8 == 0) && ((uintptr_t)c.codes[which] % 8 == 0);
  for (uint32_t d = 8 * lane; d < c.dim; d += 8 * LPR) {
    if (d >= 8 * LPR) load(e, d);
    float v[8];
    e.widen(v);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float s = fminf(fmaxf(rintf(v[k] * inv), -127.0f), 127.0f);
      const uint32_t code = finite ? (uint32_t)(int)s & 0xffu : 0u;
      w[k / 4] |= code << (8 * (k % 4));
    }
    if (vec_out) {
      *reinterpret_cast<uint2*>(q + d) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (uint32_t k = 0; k < 8; ++k)
        if (d + k < c.dim) q[d + k] = (uint8_t)(w[k / 4] >> (8 * (k % 4)));
    }
  }
  if (lane == 0) reinterpret_cast<float*>(c.scales[which])[at] = finite ? step : __uint_as_float(0x7fc00000u);
}

// ---------------------------------------------------------------------------------- reading
constexpr uint32_t kKvMaxTokens = 32;     // tokens of one CTA

// Slot of output row r, or -1: the sequence is the last one that starts at or before r.
__device__ __forceinline__ int64_t slot_of(const KvView& c, const KvRead& rd, uint64_t r) {
  uint32_t lo = 0, hi = rd.seqs + 1;      // starts[lo - 1] <= r < starts[hi]
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    if (__ldg(rd.starts + mid) <= (int64_t)r) lo = mid + 1; else hi = mid;
  }
  if (lo == 0 || lo > rd.seqs) return -1;
  const uint64_t i = r - (uint64_t)__ldg(rd.starts + lo - 1);
  const uint64_t page = i / c.page_size;
  if (page >= rd.table_ld) return -1;
  const int32_t id = __ldg(rd.table + (lo - 1) * rd.table_ld + page);
  if (id < 0 || (uint32_t)id >= c.pages) return -1;
  return (int64_t)((uint64_t)id * c.page_size + i % c.page_size);
}

template <class T, int FORMAT>
__global__ void __launch_bounds__(kKvThreads)
kv_read_kernel(KvView c, KvRead rd, uint32_t tokens, FastDiv cpr, FastDiv per_token, uint32_t which0) {
  __shared__ int64_t slots[kKvMaxTokens];
  dependency_wait();
  allow_dependents();
  const uint32_t which = which0 + blockIdx.y;
  const uint64_t token0 = blockIdx.x * (uint64_t)tokens;
  if (threadIdx.x < tokens) slots[threadIdx.x] = token0 + threadIdx.x < rd.total ? slot_of(c, rd, token0 + threadIdx.x) : -1;
  __syncthreads();
  const uint32_t left = (uint32_t)min((uint64_t)tokens, rd.total - token0);
  const uint32_t n_items = left * per_token.d;
  T* y = (T*)rd.y[which] + token0 * c.heads * c.dim;
  const uint8_t* codes = c.codes[which];
  const bool vec_out = (c.dim % 8 == 0) && ((uintptr_t)rd.y[which] % 16 == 0);
  const bool vec_in = (c.dim % 8 == 0) && ((uintptr_t)codes % 8 == 0);
  constexpr int U = 4;
  for (uint32_t i0 = threadIdx.x; i0 < n_items; i0 += U * kKvThreads) {
    uint2 w[U]; float scale[U]; uint32_t row[U], ch[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = i0 + u * kKvThreads;
      w[u] = make_uint2(0, 0); scale[u] = 0.f; row[u] = ch[u] = 0;
      if (i >= n_items) continue;
      const uint32_t t = per_token.div(i);
      row[u] = cpr.div(i); ch[u] = i - row[u] * cpr.d;
      const int64_t slot = slots[t];
      if (slot < 0) continue;
      const uint64_t at = (uint64_t)slot * c.heads + (row[u] - t * c.heads);
      if (FORMAT == QV2_KV_MX4) {
        w[u].x = __ldg(reinterpret_cast<const uint32_t*>(codes) + at * cpr.d + ch[u]);
        scale[u] = mx_scale(__ldg(c.scales[which] + at * (cpr.d >> 2) + (ch[u] >> 2)));
      } else {
        const uint8_t* p = codes + at * c.dim + 8ull * ch[u];
        if (vec_in) w[u] = __ldg(reinterpret_cast<const uint2*>(p));
        else
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k)
            if (8 * ch[u] + k < c.dim) (k < 4 ? w[u].x : w[u].y) |= (uint32_t)__ldg(p + k) << (8 * (k % 4));
        scale[u] = __ldg(reinterpret_cast<const float*>(c.scales[which]) + at);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * kKvThreads >= n_items) continue;
      float v[8];
      if (FORMAT == QV2_KV_MX4) {
        mx_decode8(w[u].x, scale[u], v);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (float)(int8_t)((k < 4 ? w[u].x : w[u].y) >> (8 * (k % 4))) * scale[u];
      }
      T* q = y + (uint64_t)row[u] * c.dim + 8ull * ch[u];
      if (8 * ch[u] >= c.dim) continue;              // a chunk of the last block past the row's end
      if (vec_out) Chunk8<T>::store_vec(q, v);
      else store_some(q, v, c.dim - 8 * ch[u]);
    }
  }
}

template <class T>
cudaError_t write_typed(const Launch& l, const KvView& c, const KvNew& n, uint64_t* launches) {
  bool vec[2];
  for (int w = 0; w < 2; ++w)
    vec[w] = (uintptr_t)n.x[w] % 16 == 0 && n.token_ld[w] * sizeof(T) % 16 == 0 && n.head_ld[w] * sizeof(T) % 16 == 0;
  const uint32_t cpr = c.format == QV2_KV_MX4 ? 4 * ((c.dim + 31) / 32) : 32;
  const uint64_t step = (1ull << 30) / ((uint64_t)cpr * c.heads);      // item numbers stay below 2^31
  for (uint64_t t = 0; t < n.tokens; t += step) {
    const uint64_t nt = n.tokens - t < step ? n.tokens - t : step;
    const uint32_t rows = (uint32_t)(nt * c.heads);
    cudaError_t e;
    if (c.format == QV2_KV_MX4) {
      const uint32_t items = rows * cpr;
      e = launch_grid(l, kv_write_mx4_kernel<T>, dim3((items + kKvThreads - 1) / kKvThreads, 2), kKvThreads, 0, c, n, t, FastDiv(cpr), FastDiv(c.heads), items, vec[0], vec[1]);
    } else if (c.dim <= 64) {
      e = launch_grid(l, kv_write_i8_kernel<T, 8>, dim3((rows + kKvThreads / 8 - 1) / (kKvThreads / 8), 2), kKvThreads, 0, c, n, t, FastDiv(c.heads), rows, vec[0], vec[1]);
    } else if (c.dim <= 128) {
      e = launch_grid(l, kv_write_i8_kernel<T, 16>, dim3((rows + kKvThreads / 16 - 1) / (kKvThreads / 16), 2), kKvThreads, 0, c, n, t, FastDiv(c.heads), rows, vec[0], vec[1]);
    } else {
      e = launch_grid(l, kv_write_i8_kernel<T, 32>, dim3((rows + kKvThreads / 32 - 1) / (kKvThreads / 32), 2), kKvThreads, 0, c, n, t, FastDiv(c.heads), rows, vec[0], vec[1]);
    }
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

template <class T>
cudaError_t read_typed(const Launch& l, const KvView& c, const KvRead& r, uint64_t* launches) {
  const uint32_t cpr = c.format == QV2_KV_MX4 ? 4 * ((c.dim + 31) / 32) : (c.dim + 7) / 8;
  const uint32_t per_token = cpr * c.heads;
  uint32_t tokens = 2048 / per_token;
  tokens = tokens < 1 ? 1 : tokens > kKvMaxTokens ? kKvMaxTokens : tokens;
  const uint64_t grid = (r.total + tokens - 1) / tokens;
  const uint32_t which0 = r.y[0] ? 0 : 1, n_which = (r.y[0] ? 1 : 0) + (r.y[1] ? 1 : 0);
  auto* kernel = c.format == QV2_KV_MX4 ? kv_read_kernel<T, QV2_KV_MX4> : kv_read_kernel<T, QV2_KV_I8>;
  cudaError_t e = launch_grid(l, kernel, dim3((uint32_t)grid, n_which), kKvThreads, 0, c, r, tokens, FastDiv(cpr), FastDiv(per_token), which0);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace

cudaError_t launch_kv_write(const Launch& l, const KvView& c, const KvNew& n, uint64_t* launches) {
  if (n.dtype == kF16) return write_typed<__half>(l, c, n, launches);
  if (n.dtype == kBF16) return write_typed<__nv_bfloat16>(l, c, n, launches);
  return write_typed<float>(l, c, n, launches);
}

cudaError_t launch_kv_read(const Launch& l, const KvView& c, const KvRead& r, uint64_t* launches) {
  if (r.dtype == kF16) return read_typed<__half>(l, c, r, launches);
  if (r.dtype == kBF16) return read_typed<__nv_bfloat16>(l, c, r, launches);
  return read_typed<float>(l, c, r, launches);
}

}  // namespace qv2
