// The quantized key / value cache: rows of one head rounded on their way into their slots, and
// whole sequences gathered back through a page table.  Both directions are bound by the bytes of
// the unquantized side (256 of 256 + 68 bytes per row of 128 bfloat16 elements at 4 bits).  204 K tokens
// of 8 heads x 128 read back from 4 bits (1.06 GB) take 177 us = 5.9 TB/s, 23 K tokens written in 8 bits
// (145 MB) 39 us = 3.7 TB/s, and read back 30 us = 4.8 TB/s.  A CTA begins with a chain of look-ups (sequence, page,
// codes: some 2.5 us), so it takes up to 128 tokens (the same read: 232 us at 16 tokens, 190 at 64).
#include "qv2_mx.cuh"

namespace qv2 {

namespace {

constexpr uint32_t kKvThreads = 128;

// ---------------------------------------------------------------------------------- writing, 4 bits
// Work item: eight elements, as in mx_quantize_kernel; blockIdx.y picks keys or values.
template <class T, int U>
__global__ void __launch_bounds__(kKvThreads)
kv_write_mx4_kernel(KvView c, KvNew n, uint64_t token0, FastDiv cpr, FastDiv heads, uint32_t n_items, bool vec_k, bool vec_v) {
  dependency_wait();
  allow_dependents();
  const uint32_t which = blockIdx.y;
  const bool vec = which ? vec_v : vec_k;
  const uint32_t base = blockIdx.x * (kKvThreads * U) + threadIdx.x;
  Chunk8<T> e[U];
  int64_t slot[U];
  uint32_t h[U], ch[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = base + u * kKvThreads, row = cpr.div(i), t = heads.div(row);
    ch[u] = i - row * cpr.d;
    h[u] = row - t * heads.d;
    e[u].zero();
    slot[u] = -1;
    if (i < n_items) {
      slot[u] = __ldg(n.slots + token0 + t);
      const T* p = (const T*)n.x[which] + (token0 + t) * n.token_ld[which] + h[u] * n.head_ld[which] + 8ull * ch[u];
      if (ch[u] * 8 + 8 <= c.dim) { if (vec) e[u].load_vec(p); else e[u].load_any(p); }
      else if (ch[u] * 8 < c.dim) e[u].load_some(p, c.dim - ch[u] * 8);
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
    if (slot[u] < 0 || (uint64_t)slot[u] >= c.slots) continue;
    const uint64_t at = (uint64_t)slot[u] * c.heads + h[u];
    reinterpret_cast<uint32_t*>(c.codes[which])[at * cpr.d + ch[u]] = codes;
    if ((ch[u] & 3u) == 0) c.scales[which][at * (cpr.d >> 2) + (ch[u] >> 2)] = (uint8_t)byte;
  }
}

// ---------------------------------------------------------------------------------- writing, 8 bits
// Eight codes from elements and 127 / R.  |x| <= R, so |x * (127/R)| <= 127 (1 + 2^-22) and the rounded code needs no
// clamp; adding 1.5 * 2^23 rounds to the nearest whole number (ties to even) and leaves its two's complement in the
// low bits of the sum.
__device__ __forceinline__ uint2 i8_encode8(const float (&v)[8], float inv) {
  uint32_t q[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) q[k] = __float_as_uint(__fadd_rn(__fmul_rn(v[k], inv), 12582912.0f));
  const uint32_t a = __byte_perm(q[0], q[1], 0x0040), b = __byte_perm(q[2], q[3], 0x0040);
  const uint32_t c = __byte_perm(q[4], q[5], 0x0040), d = __byte_perm(q[6], q[7], 0x0040);
  return make_uint2(__byte_perm(a, b, 0x5410), __byte_perm(c, d, 0x5410));
}

// LPR lanes share a row, 16 elements each, and R rows are in flight per thread; a row of more than 16 * LPR elements
// (LPR = 32, head_dim > 512) is walked twice, the second time out of the caches.
template <class T, int LPR, int R>
__global__ void __launch_bounds__(kKvThreads)
kv_write_i8_kernel(KvView c, KvNew n, uint64_t token0, FastDiv heads, uint32_t n_rows, bool vec_k, bool vec_v, uint32_t out_align) {
  dependency_wait();
  allow_dependents();
  constexpr uint32_t ROWS = kKvThreads / LPR;              // rows of a CTA per round
  const uint32_t which = blockIdx.y;
  const bool vec = which ? vec_v : vec_k;
  const uint32_t lane = threadIdx.x % LPR;
  auto load = [&](Chunk8<T> (&e)[2], const T* p, uint32_t d) {
#pragma unroll
    for (uint32_t g = 0; g < 2; ++g, d += 8) {
      e[g].zero();
      if (!p || d >= c.dim) continue;
      if (d + 8 <= c.dim) { if (vec) e[g].load_vec(p + d); else e[g].load_any(p + d); }
      else e[g].load_some(p + d, c.dim - d);
    }
  };
  Chunk8<T> e[R][2];
  const T* p[R];
  int64_t slot[R];
  uint32_t h[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const uint32_t row = (blockIdx.x * R + r) * ROWS + threadIdx.x / LPR, t = heads.div(row);
    h[r] = row - t * heads.d;
    p[r] = row < n_rows ? (const T*)n.x[which] + (token0 + t) * n.token_ld[which] + h[r] * n.head_ld[which] : nullptr;
    slot[r] = row < n_rows ? __ldg(n.slots + token0 + t) : -1;
    load(e[r], p[r], 16 * lane);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    uint32_t top = max(e[r][0].top_bits(), e[r][1].top_bits());
    if (LPR == 32)
      for (uint32_t d = 16 * (lane + LPR); d < c.dim; d += 16 * LPR) {
        Chunk8<T> more[2];
        load(more, p[r], d);
        top = max(top, max(more[0].top_bits(), more[1].top_bits()));
      }
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (slot[r] < 0 || (uint64_t)slot[r] >= c.slots) continue;
    const float most = __uint_as_float(top);
    float step = __fdiv_rn(most, 127.0f), inv = __fdiv_rn(127.0f, most);
    const bool finite = top < 0x7f800000u;
    if (finite && (!(most > 0.0f) || !isfinite(inv) || !(step > 0.0f))) { step = 1.0f; inv = 1.0f; }
    const uint64_t at = (uint64_t)slot[r] * c.heads + h[r];
    uint8_t* q = c.codes[which] + at * c.dim;
    for (uint32_t d = 16 * lane; d < c.dim; d += 16 * LPR) {
      if (LPR == 32 && d >= 16 * LPR) load(e[r], p[r], d);
      float v[8];
      e[r][0].widen(v);
      uint2 a = i8_encode8(v, inv);
      e[r][1].widen(v);
      uint2 b = i8_encode8(v, inv);
      if (!finite) a = b = make_uint2(0, 0);
      if (out_align == 16) {
        *reinterpret_cast<uint4*>(q + d) = make_uint4(a.x, a.y, b.x, b.y);
      } else if (out_align == 8) {
        *reinterpret_cast<uint2*>(q + d) = a;
        if (d + 8 < c.dim) *reinterpret_cast<uint2*>(q + d + 8) = b;
      } else {
#pragma unroll
        for (uint32_t k = 0; k < 16; ++k)
          if (d + k < c.dim) q[d + k] = (uint8_t)((k < 8 ? (k < 4 ? a.x : a.y) : (k < 12 ? b.x : b.y)) >> (8 * (k % 4)));
      }
    }
    if (lane == 0) reinterpret_cast<float*>(c.scales[which])[at] = finite ? step : __uint_as_float(0x7fc00000u);
  }
}

// ---------------------------------------------------------------------------------- reading
constexpr uint32_t kKvMaxTokens = 128;     // tokens of one CTA

// Number of starts that are <= r, among count of them (non-decreasing); the warp narrows the range 32-fold a step.
__device__ __forceinline__ uint32_t warp_upper_bound(const int64_t* starts, uint32_t count, int64_t r, uint32_t lane) {
  uint32_t lo = 0, n = count;             // the answer lies in lo .. lo + n
  while (n > 0) {
    const uint32_t step = (n + 31) / 32, i = lane * step + step - 1;        // the last entry of this lane's piece
    const bool le = i < n && __ldg(starts + lo + i) <= r;
    const uint32_t pieces = __popc(__ballot_sync(0xffffffffu, le));         // whole pieces that are <= r
    lo += pieces * step;
    n = pieces * step < n ? min(step - 1, n - pieces * step) : 0;           // what is left of the next piece
  }
  return lo;
}

// Slots of the output rows row0 + lane, or -1.
__device__ __forceinline__ int64_t warp_slots(const KvView& c, const KvRead& rd, uint64_t row0, uint32_t lane) {
  const uint32_t first = warp_upper_bound(rd.starts, rd.seqs + 1, (int64_t)row0, lane);
  const uint64_t r = row0 + lane;
  uint32_t after = first;                 // sequences that start at or before r: the rows follow one another
  while (after <= rd.seqs && __ldg(rd.starts + after) <= (int64_t)r) ++after;
  if (r >= rd.total || after == 0 || after > rd.seqs) return -1;
  const uint64_t i = r - (uint64_t)__ldg(rd.starts + after - 1);
  const uint64_t page = i / c.page_size;
  if (page >= rd.table_ld) return -1;
  const int32_t id = __ldg(rd.table + (after - 1) * rd.table_ld + page);
  if (id < 0 || (uint32_t)id >= c.pages) return -1;
  return (int64_t)((uint64_t)id * c.page_size + i % c.page_size);
}

// Work item: E consecutive elements of a row.  E = 32, 16: rows of whole items, aligned, stores of whole 32-byte
// sectors; E = 8: any alignment and length.
template <class T, int FORMAT, uint32_t E>
__global__ void __launch_bounds__(kKvThreads)
kv_read_kernel(KvView c, KvRead rd, uint32_t tokens, FastDiv cpr, FastDiv per_token, uint32_t which0, bool vec_in, bool vec_out) {
  __shared__ int64_t slots[kKvMaxTokens];
  dependency_wait();
  allow_dependents();
  const uint32_t which = which0 + blockIdx.y;
  const uint64_t token0 = blockIdx.x * (uint64_t)tokens;
  if (threadIdx.x < kKvMaxTokens) slots[threadIdx.x] = warp_slots(c, rd, token0 + (threadIdx.x & ~31u), threadIdx.x % 32);
  __syncthreads();
  const uint32_t left = (uint32_t)min((uint64_t)tokens, rd.total - token0);
  const uint32_t n_items = left * per_token.d;
  T* y = (T*)rd.y[which] + token0 * c.heads * c.dim;
  const uint8_t* codes = c.codes[which];
  const uint8_t* scales = c.scales[which];
  const uint32_t blocks = (c.dim + 31) / 32;
  constexpr int U = 4;
  constexpr uint32_t BYTES = FORMAT == QV2_KV_MX4 ? E / 2 : E, WORDS = BYTES / 4;
  for (uint32_t i0 = threadIdx.x; i0 < n_items; i0 += U * kKvThreads) {
    uint32_t w[U][WORDS]; float scale[U]; uint32_t row[U], ch[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = i0 + u * kKvThreads;
#pragma unroll
      for (uint32_t k = 0; k < WORDS; ++k) w[u][k] = 0;
      scale[u] = 0.f; row[u] = ch[u] = 0;
      if (i >= n_items) continue;
      const uint32_t t = per_token.div(i);
      row[u] = cpr.div(i); ch[u] = i - row[u] * cpr.d;
      const int64_t slot = slots[t];
      if (slot < 0) continue;
      const uint64_t at = (uint64_t)slot * c.heads + (row[u] - t * c.heads);
      const uint8_t* p = codes + at * (FORMAT == QV2_KV_MX4 ? 16 * blocks : c.dim) + BYTES * ch[u];
      if (E > 8 || FORMAT == QV2_KV_MX4 || vec_in) {
#pragma unroll
        for (uint32_t k = 0; k < WORDS; k += 4) {
          if (WORDS >= 4) { const uint4 q = __ldg(reinterpret_cast<const uint4*>(p) + k / 4); w[u][k] = q.x; w[u][k + 1 < WORDS ? k + 1 : 0] = q.y; w[u][k + 2 < WORDS ? k + 2 : 0] = q.z; w[u][k + 3 < WORDS ? k + 3 : 0] = q.w; }
          else if (WORDS == 2) { const uint2 q = __ldg(reinterpret_cast<const uint2*>(p)); w[u][0] = q.x; w[u][WORDS - 1] = q.y; }
          else w[u][0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        }
      } else {
#pragma unroll
        for (uint32_t k = 0; k < BYTES; ++k)
          if (8 * ch[u] + k < c.dim) w[u][k / 4] |= (uint32_t)__ldg(p + k) << (8 * (k % 4));
      }
      scale[u] = FORMAT == QV2_KV_MX4 ? mx_scale(__ldg(scales + at * blocks + ch[u] / (32 / E))) : __ldg(reinterpret_cast<const float*>(scales) + at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * kKvThreads >= n_items) continue;
      T* q = y + (uint64_t)row[u] * c.dim + E * ch[u];
      float v[2][8];
#pragma unroll
      for (uint32_t g = 0; g < E / 8; ++g) {
        if (FORMAT == QV2_KV_MX4) {
          mx_decode8(w[u][g], scale[u], v[g % 2]);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[g % 2][k] = (float)(int8_t)(w[u][(2 * g + k / 4) % WORDS] >> (8 * (k % 4))) * scale[u];
        }
        if (E > 8 && g % 2 == 1) store_sectors(q + 8 * (g - 1), v[0], v[1]);
      }
      if (E == 8) {
        if (8 * ch[u] >= c.dim) continue;              // an item of the last block past the row's end
        if (vec_out) Chunk8<T>::store_vec(q, v[0]);
        else store_some(q, v[0], c.dim - 8 * ch[u]);
      }
    }
  }
}

template <class T>
cudaError_t write_typed(const Launch& l, const KvView& c, const KvNew& n, uint64_t* launches) {
  bool vec[2];
  for (int w = 0; w < 2; ++w)
    vec[w] = (uintptr_t)n.x[w] % 16 == 0 && n.token_ld[w] * sizeof(T) % 16 == 0 && n.head_ld[w] * sizeof(T) % 16 == 0;
  const uint64_t to = (uint64_t)c.dim | (uintptr_t)c.codes[0] | (uintptr_t)c.codes[1];
  const uint32_t out_align = to % 16 == 0 ? 16 : to % 8 == 0 ? 8 : 1;
  const uint32_t cpr = c.format == QV2_KV_MX4 ? 4 * ((c.dim + 31) / 32) : 32;
  const uint64_t step = (1ull << 30) / ((uint64_t)cpr * c.heads);      // item numbers stay below 2^31
  for (uint64_t t = 0; t < n.tokens; t += step) {
    const uint64_t nt = n.tokens - t < step ? n.tokens - t : step;
    const uint32_t rows = (uint32_t)(nt * c.heads);
    // Few items: one per thread spreads them over more SMs; many: several loads in flight per thread.
    const bool many = (uint64_t)rows * ((c.dim + 7) / 8) > (uint64_t)l.sm_count * 8 * kKvThreads;
    cudaError_t e;
    if (c.format == QV2_KV_MX4) {
      const uint32_t items = rows * cpr, per = kKvThreads * (many ? 4 : 1);
      auto* kernel = many ? kv_write_mx4_kernel<T, 4> : kv_write_mx4_kernel<T, 1>;
      e = launch_grid(l, kernel, dim3((items + per - 1) / per, 2), kKvThreads, 0, c, n, t, FastDiv(cpr), FastDiv(c.heads), items, vec[0], vec[1]);
    } else {
      const uint32_t lpr = c.dim <= 64 ? 4 : c.dim <= 128 ? 8 : c.dim <= 256 ? 16 : 32, per = kKvThreads / lpr * (many ? 4 : 1);
      auto* kernel = lpr == 4    ? (many ? kv_write_i8_kernel<T, 4, 4> : kv_write_i8_kernel<T, 4, 1>)
                     : lpr == 8  ? (many ? kv_write_i8_kernel<T, 8, 4> : kv_write_i8_kernel<T, 8, 1>)
                     : lpr == 16 ? (many ? kv_write_i8_kernel<T, 16, 4> : kv_write_i8_kernel<T, 16, 1>)
                                 : (many ? kv_write_i8_kernel<T, 32, 4> : kv_write_i8_kernel<T, 32, 1>);
      e = launch_grid(l, kernel, dim3((rows + per - 1) / per, 2), kKvThreads, 0, c, n, t, FastDiv(c.heads), rows, vec[0], vec[1], out_align);
    }
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

template <class T>
cudaError_t read_typed(const Launch& l, const KvView& c, const KvRead& r, uint64_t* launches) {
  const uintptr_t out = (uintptr_t)r.y[0] | (uintptr_t)r.y[1], in = (uintptr_t)c.codes[0] | (uintptr_t)c.codes[1];
  const uint32_t wide = out % 32 || in % 16 ? 8 : c.dim % 32 == 0 ? 32 : c.dim % 16 == 0 ? 16 : 8;
  const bool vec_out = c.dim % 8 == 0 && out % 16 == 0, vec_in = c.dim % 8 == 0 && in % 8 == 0;
  const uint32_t cpr = wide > 8 ? c.dim / wide : c.format == QV2_KV_MX4 ? 4 * ((c.dim + 31) / 32) : (c.dim + 7) / 8;
  const uint32_t per_token = cpr * c.heads;
  uint32_t tokens = 131072 / wide / per_token;              // many rounds of loads per thread (a CTA begins with a
                                                           // chain of look-ups), but four CTAs per SM where there is work for them
  const uint64_t spread = r.total / (4 * (uint64_t)l.sm_count);
  if (tokens > spread) tokens = (uint32_t)spread;
  tokens = tokens < 1 ? 1 : tokens > kKvMaxTokens ? kKvMaxTokens : tokens;
  const uint64_t grid = (r.total + tokens - 1) / tokens;
  const uint32_t which0 = r.y[0] ? 0 : 1, n_which = (r.y[0] ? 1 : 0) + (r.y[1] ? 1 : 0);
  auto* kernel = c.format == QV2_KV_MX4 ? (wide == 32 ? kv_read_kernel<T, QV2_KV_MX4, 32> : wide == 16 ? kv_read_kernel<T, QV2_KV_MX4, 16> : kv_read_kernel<T, QV2_KV_MX4, 8>)
                                        : (wide == 32 ? kv_read_kernel<T, QV2_KV_I8, 32> : wide == 16 ? kv_read_kernel<T, QV2_KV_I8, 16> : kv_read_kernel<T, QV2_KV_I8, 8>);
  cudaError_t e = launch_grid(l, kernel, dim3((uint32_t)grid, n_which), kKvThreads, 0, c, r, tokens, FastDiv(cpr), FastDiv(per_token), which0, vec_in, vec_out);
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
