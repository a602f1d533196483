// Products of microscaled 4-bit matrices, dense and grouped by expert, on the fifth-generation tensor
// cores: y[i][j] = sum_k a[i][k] w[j][k], both operands in blocks of 32 codes with a power-of-two scale.
//
// tcgen05.mma.kind::mxf4 multiplies codes straight from shared memory and applies the two scales of each
// block of 32 inside the instruction; the accumulator (binary32) stays in tensor memory.  One CTA has
//   warp 0       fetches code tiles by TMA (128 bytes = 256 columns per row and step, 128-byte swizzle),
//   warp 1       copies the scales from shared to tensor memory and issues the products,
//   warp 2       owns the tensor memory,
//   warps 4-7    move finished accumulators out (one warp per quarter of the 128 accumulator rows),
//   warps 8-11   bring the scales: they lie row by row in memory, the tensor core wants them four to a
//                word and 32 rows to a column, so they pass through registers, 16 bytes per row and two
//                steps, fetched four steps ahead.
// A ring of shared-memory stages decouples them; accumulators are double-buffered.
//
// The 128-row operand X and the BN-row operand Y take either role:
//   tokens as X, weights as Y (BN = 256): the many-row form, bound by the tensor cores;
//   weights as X, tokens as Y (BN = 16..128): few rows per weight, bound by reading the weights once; the
//   columns may be cut over the CTAs of a cluster, whose partial sums are added through distributed
//   shared memory in the order of the ranks.
#include <cuda.h>

#include "qv2_mx.cuh"

namespace qv2 {

namespace {

constexpr int kProductThreads = 384;
constexpr uint32_t kStepCols = 256;              // columns per stage: 128 bytes of codes
constexpr uint64_t kWaitLimitNs = 2000000000ull; // a wait that lasts this long gives up
constexpr uint32_t kMaxGroups = QV2_MX_MAX_GROUPS;

// ------------------------------------------------------------------------------------ PTX wrappers
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns() { uint64_t t; asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t)); return t; }

// Waits for the phase of `parity` to complete.  false: this wait or another of the CTA has given up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* failed) {
  if (bar_try(bar, parity)) return true;
  uint64_t begin = 0;
  for (uint32_t i = 1;; ++i) {
    if (bar_try(bar, parity)) return true;
    if ((i & 255u) == 0) {
      if (*failed) return false;
      const uint64_t t = now_ns();
      if (!begin) begin = t;
      else if (t - begin > kWaitLimitNs) { *failed = 1; return false; }
    }
  }
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Scales of 128 rows by 4 blocks: 512 consecutive bytes, 16 for each of 32 lanes, into 4 columns of all
// four lane quarters.
__device__ __forceinline__ void tc_copy_scales(uint32_t column, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(column), "l"(desc) : "memory");
}
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_load32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
                 "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
                 "=r"(r[30]), "=r"(r[31])
               : "r"(taddr));
}
__device__ __forceinline__ void tc_load16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
__device__ __forceinline__ void tc_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Shared-memory matrix descriptors (address and strides in units of 16 bytes, version 1 in bits 46-47).
// Codes: rows of 128 bytes in the 128-byte swizzle, 1024 bytes from one group of 8 rows to the next.
__device__ __forceinline__ uint64_t codes_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Scales: no swizzle, 128 bytes from one group of 8 lanes to the next.
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
}

// ------------------------------------------------------------------------------------ geometry
template <int BN_, bool TOKENS_X_, int STAGES_>
struct Shape {
  static constexpr int BN = BN_, STAGES = STAGES_;
  static constexpr bool TOKENS_X = TOKENS_X_;              // X are the tokens (else the weights)
  static constexpr int ROW_TILE = TOKENS_X ? 128 : BN;     // tokens per tile
  static constexpr int W_TILE = TOKENS_X ? BN : 128;       // weight rows per tile
  static constexpr int YB = (BN + 127) / 128;              // 128-row groups of Y's scales
  static constexpr uint32_t X_BYTES = 128 * 128, Y_BYTES = BN * 128;
  static constexpr uint32_t SF_BYTES = 2 * 512 * (1 + YB);
  static constexpr uint32_t STAGE = X_BYTES + Y_BYTES + SF_BYTES;
  // Two accumulators of 256 columns and the scales do not fit 512 columns: the second one begins 64
  // columns before the first one's end, and a tile waits for those columns of its predecessor only.
  static constexpr bool OVERLAP = BN == 256;
  static constexpr uint32_t ACC_STEP = OVERLAP ? 192 : BN;
  static constexpr uint32_t SF_COL = OVERLAP ? 448 : 2 * BN;
  static constexpr uint32_t SF_SET = 8 + 8 * YB;           // columns of one step's scales; two sets alternate
  static_assert(SF_COL + 2 * SF_SET <= 512, "tensor memory");
  static constexpr uint32_t STAGING = TOKENS_X ? 4 * 4096 : 0;
  static constexpr uint32_t TABLES = 2 * 4 * (kMaxGroups + 2);
  static constexpr uint32_t SMEM = 1024 + STAGES * STAGE + STAGING + TABLES + 512;
  static_assert(SMEM <= 232448, "shared memory");
  static constexpr uint32_t IDESC = (1u << 7) | (1u << 10) | ((uint32_t)(BN / 8) << 17) | (1u << 23) | (8u << 24);   // E2M1 x E2M1, E8M0 scales, 128 x BN
};

struct ProductArgs {
  const uint8_t *x_scales, *y_scales;
  uint64_t x_sld, y_sld, x_sgs, y_sgs;       // bytes between rows and between groups
  uint32_t x_rows, y_rows;                   // rows of the matrices (of one group)
  uint32_t x_vec, y_vec;                     // 16-byte loads of scales are aligned
  const float* bias;
  const int64_t* offsets;
  void* out;
  uint64_t out_ld;
  uint32_t dtype, out_vec;                   // out_vec: 16-byte stores of whole rows are aligned
  uint32_t m, n, blocks, steps, groups, w_tiles, splits;
  uint32_t early;                            // everything but `a` was complete before this launch could begin
  uint32_t* fault;
};

struct Where {                               // one tile
  uint32_t group, token0, token_end, w0;
};

template <class S>
__device__ __forceinline__ bool find_tile(const uint32_t* lo, const uint32_t* cum, uint32_t groups, uint32_t w_tiles, uint32_t tile, Where* out) {
  if (tile >= cum[groups] * w_tiles) return false;
  const uint32_t q = tile / w_tiles;
  uint32_t a = 0, b = groups;                // cum[a] <= q < cum[b]
  while (b - a > 1) {
    const uint32_t mid = (a + b) / 2;
    if (cum[mid] <= q) a = mid; else b = mid;
  }
  // within a group: bands of BAND row tiles, inside a band the row tile runs fastest, so that the CTAs at work
  // at one time share few tiles of either operand
  constexpr uint32_t BAND = S::TOKENS_X ? 8 : 0x7fffffff;
  const uint32_t rt = cum[a + 1] - cum[a];
  uint32_t t = tile - cum[a] * w_tiles, first = 0, height = rt;
  if (S::TOKENS_X && rt > BAND) {
    const uint32_t band = t / (BAND * w_tiles);
    t -= band * BAND * w_tiles;
    first = band * BAND;
    height = min(BAND, rt - first);
  }
  out->group = a;
  out->token0 = lo[a] + (first + t % height) * S::ROW_TILE;
  out->token_end = lo[a + 1];
  out->w0 = (t / height) * S::W_TILE;
  return true;
}

// Scale bytes 16*v .. 16*v+15 of a row, zeros behind the last block.
__device__ __forceinline__ uint4 load_scales(const uint8_t* row, uint32_t v, uint32_t blocks, bool vec) {
  const uint32_t at = 16 * v;
  if (vec && at + 16 <= blocks) return __ldg(reinterpret_cast<const uint4*>(row + at));
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (uint32_t i = 0; i < 16; ++i)
    if (at + i < blocks) w[i / 4] |= (uint32_t)__ldg(row + at + i) << (8 * (i % 4));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void store_as(void* y, uint64_t at, uint32_t dtype, float v) {
  if (dtype == kBF16) ((__nv_bfloat16*)y)[at] = __float2bfloat16_rn(v);
  else if (dtype == kF16) ((__half*)y)[at] = __float2half_rn(v);
  else ((float*)y)[at] = v;
}
__device__ __forceinline__ uint32_t pack2(uint32_t dtype, float a, float b) {
  if (dtype == kBF16) { __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); }
  __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&h);
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// ------------------------------------------------------------------------------------ the kernel
template <class S>
__global__ void __launch_bounds__(kProductThreads, 1)
mx_matmul_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_y, const ProductArgs p) {
  extern __shared__ uint8_t raw[];
  const uint32_t raw_addr = smem_addr(raw);
  uint8_t* const base = raw + ((1024u - (raw_addr & 1023u)) & 1023u);     // swizzled tiles start at multiples of 1024
  const uint32_t base_addr = smem_addr(base);
  // codes of all stages, then scales of all stages, then the rest
  constexpr uint32_t CODES = S::X_BYTES + S::Y_BYTES;
  uint8_t* const sf = base + S::STAGES * CODES;
  const uint32_t sf_addr = base_addr + S::STAGES * CODES;
  uint8_t* const staging = sf + S::STAGES * S::SF_BYTES;
  uint32_t* const lo = reinterpret_cast<uint32_t*>(staging + S::STAGING);
  uint32_t* const cum = lo + kMaxGroups + 2;
  uint64_t* const bars = reinterpret_cast<uint64_t*>(cum + kMaxGroups + 2);
  const uint32_t bar0 = smem_addr(bars);
  auto full_codes = [&](uint32_t s) { return bar0 + 8 * s; };
  auto full_scales = [&](uint32_t s) { return bar0 + 8 * (S::STAGES + s); };
  auto empty = [&](uint32_t s) { return bar0 + 8 * (2 * S::STAGES + s); };
  auto acc_full = [&](uint32_t b) { return bar0 + 8 * (3 * S::STAGES + b); };
  auto acc_free = [&](uint32_t b) { return bar0 + 8 * (3 * S::STAGES + 2 + b); };
  const uint32_t drained = bar0 + 8 * (3 * S::STAGES + 4);
  static_assert(8 * (3 * S::STAGES + 5) + 8 <= 512, "barriers");
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 3 * S::STAGES + 5);
  volatile uint32_t* const failed = tmem_slot + 1;

  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (!p.early) dependency_wait();
  allow_dependents();

  // group tables: lo[g] = first token of group g (clamped, never decreasing), cum[g] = row tiles before it
  for (uint32_t g = threadIdx.x; g <= p.groups; g += kProductThreads) {
    int64_t o = p.offsets ? __ldg(p.offsets + g) : (g ? (int64_t)p.m : 0);
    lo[g] = (uint32_t)(o < 0 ? 0 : o > (int64_t)p.m ? (int64_t)p.m : o);
  }
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < S::STAGES; ++s) { bar_init(full_codes(s), 1); bar_init(full_scales(s), 4); bar_init(empty(s), 1); }
    for (uint32_t b = 0; b < 2; ++b) { bar_init(acc_full(b), 1); bar_init(acc_free(b), 4); }
    bar_init(drained, 1);
    *failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_y) : "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) {
    uint32_t carry = 0;
    for (uint32_t g0 = 0; g0 <= p.groups; g0 += 32) {      // running maximum
      uint32_t v = g0 + lane <= p.groups ? lo[g0 + lane] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v = max(v, u); }
      v = max(v, carry);
      if (g0 + lane <= p.groups) lo[g0 + lane] = v;
      carry = __shfl_sync(0xffffffffu, v, 31);
    }
    __syncwarp();
    carry = 0;
    for (uint32_t g0 = 0; g0 < p.groups; g0 += 32) {       // running sum of row tiles
      const uint32_t g = g0 + lane;
      uint32_t v = g < p.groups ? (lo[g + 1] - lo[g] + S::ROW_TILE - 1) / S::ROW_TILE : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += u; }
      v += carry;
      if (g < p.groups) cum[g + 1] = v;
      carry = __shfl_sync(0xffffffffu, v, 31);
    }
    if (lane == 0) cum[0] = 0;
  }
  __syncthreads();
  const uint32_t tmem = *tmem_slot;

  // this CTA's tiles: tile0, tile0 + stride, ...; the steps of a tile are cut over the cluster in pairs
  const uint32_t rank = p.splits > 1 ? blockIdx.x % p.splits : 0;
  const uint32_t tile0 = blockIdx.x / p.splits, stride = gridDim.x / p.splits;
  const uint32_t pairs = (p.steps + 1) / 2;
  const uint32_t step_begin = 2 * (uint32_t)((uint64_t)pairs * rank / p.splits);
  const uint32_t step_end = min(p.steps, 2 * (uint32_t)((uint64_t)pairs * (rank + 1) / p.splits));
  Where at;

  if (warp == 0) {
    // ---------------------------------------------------------------------------------- codes
    if (lane == 0) {
      uint32_t it = 0;                        // fills so far
      auto fetch_w = [&](uint32_t s, uint32_t step) {
        if (S::TOKENS_X) tma_load(base_addr + s * CODES + S::X_BYTES, &map_y, full_codes(s), step * 128, at.w0, at.group);
        else tma_load(base_addr + s * CODES, &map_x, full_codes(s), step * 128, at.w0, at.group);
      };
      auto fetch_a = [&](uint32_t s, uint32_t step) {
        if (S::TOKENS_X) tma_load(base_addr + s * CODES, &map_x, full_codes(s), step * 128, at.token0, 0);
        else tma_load(base_addr + s * CODES + S::X_BYTES, &map_y, full_codes(s), step * 128, at.token0, 0);
      };
      bool first = p.early != 0;
      for (uint32_t tile = tile0; find_tile<S>(lo, cum, p.groups, p.w_tiles, tile, &at); tile += stride) {
        uint32_t step = step_begin;
        if (first) {
          // the weights of the first stages do not depend on the kernel that is rounding the activations
          const uint32_t n = min(step_end - step, (uint32_t)S::STAGES);
          for (uint32_t i = 0; i < n; ++i) { bar_expect(full_codes(i), CODES); fetch_w(i, step + i); }
          dependency_wait();
          for (uint32_t i = 0; i < n; ++i) fetch_a(i, step + i);
          step += n; it = n;
          first = false;
        }
        for (; step < step_end; ++step, ++it) {
          const uint32_t s = it % S::STAGES;
          if (it >= S::STAGES && !bar_wait(empty(s), (it / S::STAGES - 1) & 1, failed)) goto out;
          bar_expect(full_codes(s), CODES);
          fetch_w(s, step);
          fetch_a(s, step);
        }
      }
    out:
      if (*failed)                            // leave no copy in flight
        for (uint32_t i = it > S::STAGES ? it - S::STAGES : 0; i < it; ++i) {
          const uint64_t begin = now_ns();
          while (!bar_try(full_codes(i % S::STAGES), (i / S::STAGES) & 1) && now_ns() - begin < kWaitLimitNs) {}
        }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------------------------- products
    if (lane == 0) {
      uint32_t it = 0, done = 0;              // steps and tiles so far
      for (uint32_t tile = tile0; find_tile<S>(lo, cum, p.groups, p.w_tiles, tile, &at); tile += stride, ++done) {
        const uint32_t b = done & 1;
        // OVERLAP: the predecessor has left the shared columns; else: the tile before it has left this buffer
        if (S::OVERLAP ? done >= 1 && !bar_wait(acc_free(b ^ 1), ((done - 1) / 2) & 1, failed)
                       : done >= 2 && !bar_wait(acc_free(b), (done / 2 - 1) & 1, failed)) break;
        tc_fence_after();
        const uint32_t acc = tmem + b * S::ACC_STEP;
        bool ok = true;
        for (uint32_t step = step_begin; step < step_end; ++step, ++it) {
          const uint32_t s = it % S::STAGES, phase = (it / S::STAGES) & 1;
          if (!bar_wait(full_scales(s), phase, failed) || !bar_wait(full_codes(s), phase, failed)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sfx = tmem + S::SF_COL + (it & 1) * S::SF_SET, sfy = sfx + 8;
          const uint32_t src = sf_addr + s * S::SF_BYTES;
#pragma unroll
          for (uint32_t h = 0; h < 2; ++h) {
            tc_copy_scales(sfx + 4 * h, scales_desc(src + 512 * h));
#pragma unroll
            for (uint32_t y = 0; y < S::YB; ++y)
              tc_copy_scales(sfy + 4 * (h * S::YB + y), scales_desc(src + 1024 + 512 * (h * S::YB + y)));
          }
          const uint64_t dx = codes_desc(base_addr + s * CODES), dy = codes_desc(base_addr + s * CODES + S::X_BYTES);
#pragma unroll
          for (uint32_t k = 0; k < 4; ++k) {  // 64 columns each: 32 bytes along the row, two of the word's four scales
            const uint32_t id = 2 * (k & 1);
            tc_mma(acc, dx + 2 * k, dy + 2 * k, S::IDESC | (id << 29) | (id << 4), sfx + 4 * (k / 2), sfy + 4 * S::YB * (k / 2),
                   step > step_begin || k > 0);
          }
          tc_commit(empty(s));
        }
        if (!ok) break;
        tc_commit(acc_full(b));
      }
      if (*failed) {                          // leave no product in flight
        tc_commit(drained);
        const uint64_t begin = now_ns();
        while (!bar_try(drained, 0) && now_ns() - begin < kWaitLimitNs) {}
      }
    }
  } else if (warp >= 8) {
    // ---------------------------------------------------------------------------------- scales
    const uint32_t t = threadIdx.x - 256;
    if (p.early) dependency_wait();
    constexpr int AHEAD = 4;                  // pairs of steps in flight
    constexpr int YV = S::YB;
    struct Pair { uint4 x, y[YV]; uint32_t n; } ring[AHEAD];
    // the sequence of pairs to fetch
    uint32_t tile = tile0, pair = 0;
    const uint8_t *px = nullptr, *py[YV];
    bool live = true, begun = false;
    auto fetch = [&](Pair& r) {
      r.n = 0; r.x = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < YV; ++i) r.y[i] = make_uint4(0, 0, 0, 0);
      if (!live) return;
      if (!begun || 2 * pair >= step_end) {
        if (begun) tile += stride;
        begun = true;
        if (!find_tile<S>(lo, cum, p.groups, p.w_tiles, tile, &at)) { live = false; return; }
        pair = step_begin / 2;
        const uint32_t xr = (S::TOKENS_X ? at.token0 : at.w0) + t;
        px = xr < p.x_rows ? p.x_scales + (S::TOKENS_X ? 0 : at.group * p.x_sgs) + xr * p.x_sld : nullptr;
#pragma unroll
        for (int i = 0; i < YV; ++i) {
          const uint32_t yr = (S::TOKENS_X ? at.w0 : at.token0) + t + 128 * i;
          py[i] = t + 128 * i < S::BN && yr < p.y_rows ? p.y_scales + (S::TOKENS_X ? at.group * p.y_sgs : 0) + yr * p.y_sld : nullptr;
        }
      }
      if (px) r.x = load_scales(px, pair, p.blocks, p.x_vec);
#pragma unroll
      for (int i = 0; i < YV; ++i)
        if (py[i]) r.y[i] = load_scales(py[i], pair, p.blocks, p.y_vec);
      r.n = min(2u, step_end - 2 * pair);
      ++pair;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(ring[i]);
    uint32_t it = 0;
    const uint32_t word = (t % 32) * 16 + (t / 32) * 4;
    for (bool more = true; more;) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (!more) break;
        Pair& r = ring[i];
        if (r.n == 0) { more = false; break; }
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
          if (h >= r.n) break;
          const uint32_t s = it % S::STAGES;
          if (it >= S::STAGES && !bar_wait(empty(s), (it / S::STAGES - 1) & 1, failed)) { more = false; break; }
          uint8_t* dst = sf + s * S::SF_BYTES + word;
          *reinterpret_cast<uint32_t*>(dst) = h ? r.x.z : r.x.x;
          *reinterpret_cast<uint32_t*>(dst + 512) = h ? r.x.w : r.x.y;
#pragma unroll
          for (int y = 0; y < YV; ++y) {
            *reinterpret_cast<uint32_t*>(dst + 1024 + 512 * y) = h ? r.y[y].z : r.y[y].x;
            *reinterpret_cast<uint32_t*>(dst + 1024 + 512 * (YV + y)) = h ? r.y[y].w : r.y[y].y;
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive(full_scales(s));
          ++it;
        }
        if (more) fetch(r);
      }
    }
  } else if (warp >= 4) {
    // ---------------------------------------------------------------------------------- results
    const uint32_t quarter = warp - 4;        // warp w may read lanes 32 * (w % 4) and up
    const uint32_t lanes = (quarter * 32) << 16;
    if (p.early) dependency_wait();
    uint32_t done = 0;
    for (uint32_t tile = tile0; find_tile<S>(lo, cum, p.groups, p.w_tiles, tile, &at); tile += stride, ++done) {
      const uint32_t b = done & 1;
      if (!bar_wait(acc_full(b), (done / 2) & 1, failed)) break;
      tc_fence_after();
      const uint32_t acc = tmem + b * S::ACC_STEP + lanes;
      if constexpr (S::TOKENS_X) {
        // lane = token, columns = weight rows: 64 columns at a time, the ones shared with the next tile first
        uint8_t* const mine = staging + quarter * 4096;
        const uint32_t esz = p.dtype == kF32 ? 4 : 2;
        const float* bias = p.bias ? p.bias + (uint64_t)at.group * p.n : nullptr;
        const uint32_t row0 = at.token0 + quarter * 32;
        const uint32_t rows = row0 < at.token_end ? min(32u, at.token_end - row0) : 0;
#pragma unroll 1
        for (uint32_t c = 0; c < S::BN / 64; ++c) {
          const uint32_t cc = b == 0 ? (c + S::BN / 64 - 1) % (S::BN / 64) : c;
          uint32_t v[2][32];
          tc_load32(acc + 64 * cc, v[0]);
          tc_load32(acc + 64 * cc + 32, v[1]);
          tc_load_wait();
          if (c == 0) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_free(b));
          }
          const uint32_t col0 = at.w0 + 64 * cc;
          if (col0 >= p.n) continue;
#pragma unroll
          for (uint32_t h = 0; h < 2; ++h) {
            const uint32_t col = col0 + 32 * h;
            if (bias) {
#pragma unroll
              for (uint32_t j = 0; j < 32; ++j)
                if (col + j < p.n) v[h][j] = __float_as_uint(__uint_as_float(v[h][j]) + __ldg(bias + col + j));
            }
            // rows of 128 bytes, 16-byte pieces swizzled by the row so that neither side meets bank conflicts
            if (esz == 2) {
#pragma unroll
              for (uint32_t j = 0; j < 4; ++j) {
                uint32_t o[4];
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
                  o[e] = pack2(p.dtype, __uint_as_float(v[h][8 * j + 2 * e]), __uint_as_float(v[h][8 * j + 2 * e + 1]));
                *reinterpret_cast<uint4*>(mine + lane * 128 + (((4 * h + j) ^ (lane & 7)) * 16)) = make_uint4(o[0], o[1], o[2], o[3]);
              }
              if (h == 0) continue;
            } else {
#pragma unroll
              for (uint32_t j = 0; j < 8; ++j)
                *reinterpret_cast<uint4*>(mine + lane * 128 + ((j ^ (lane & 7)) * 16)) = make_uint4(v[h][4 * j], v[h][4 * j + 1], v[h][4 * j + 2], v[h][4 * j + 3]);
            }
            __syncwarp();
            const uint32_t begin = esz == 2 ? col0 : col;          // first column of the staged rows
            const uint32_t bytes = min((p.n - begin) * esz, 128u); // (col0 < n; the second half may lie behind the end)
            if (begin < p.n) {
#pragma unroll
              for (uint32_t i = 0; i < 8; ++i) {
                const uint32_t r = 4 * i + lane / 8, piece = lane % 8;
                if (r >= rows || 16 * piece >= bytes) continue;
                const uint4 o = *reinterpret_cast<const uint4*>(mine + r * 128 + ((piece ^ (r & 7)) * 16));
                uint8_t* dst = (uint8_t*)p.out + ((uint64_t)(row0 + r) * p.out_ld + begin) * esz + 16 * piece;
                if (p.out_vec && 16 * piece + 16 <= bytes) {
                  *reinterpret_cast<uint4*>(dst) = o;
                } else {
                  const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                  for (uint32_t e = 0; e < 8; ++e) {
                    if (esz == 2) { if (16 * piece + 2 * e < bytes) reinterpret_cast<uint16_t*>(dst)[e] = (uint16_t)(w[e / 2] >> (16 * (e % 2))); }
                    else if (e < 4 && 16 * piece + 4 * e < bytes) reinterpret_cast<uint32_t*>(dst)[e] = w[e];
                  }
                }
              }
            }
            __syncwarp();
          }
        }
      } else {
        // lane = weight row, columns = tokens: 32 lanes write neighbouring results
        const uint32_t n = at.w0 + quarter * 32 + lane;
        const float bias = p.bias && n < p.n ? __ldg(p.bias + (uint64_t)at.group * p.n + n) : 0.f;
        const uint32_t tokens = min((uint32_t)S::BN, at.token_end - at.token0);
        float* part = reinterpret_cast<float*>(base) + quarter * 32 + lane;     // [token][128], over stages that are done with
#pragma unroll 1
        for (uint32_t c = 0; c < S::BN; c += 16) {
          if (c >= tokens) break;
          uint32_t v[16];
          tc_load16(acc + c, v);
          tc_load_wait();
#pragma unroll
          for (uint32_t j = 0; j < 16; ++j) {
            if (p.splits > 1) part[(c + j) * 128] = __uint_as_float(v[j]);
            else if (c + j < tokens && n < p.n) store_as(p.out, (uint64_t)(at.token0 + c + j) * p.out_ld + n, p.dtype, __uint_as_float(v[j]) + bias);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(acc_free(b));
      }
    }
  }
  __syncwarp();

  if (!S::TOKENS_X && p.splits > 1) {
    // One tile per cluster: each rank adds up its share of the tokens over all ranks, in their order.
    cluster_sync();
    if (warp >= 4 && warp < 8 && find_tile<S>(lo, cum, p.groups, p.w_tiles, tile0, &at)) {
      const uint32_t col = threadIdx.x - 128, n = at.w0 + col;
      const uint32_t tokens = min((uint32_t)S::BN, at.token_end - at.token0);
      const float bias = p.bias && n < p.n ? __ldg(p.bias + (uint64_t)at.group * p.n + n) : 0.f;
      for (uint32_t tok = rank; tok < tokens; tok += p.splits) {
        float sum = 0.f;
        for (uint32_t r = 0; r < p.splits; ++r) {
          uint32_t remote;
          float v;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(base_addr + (tok * 128 + col) * 4), "r"(r));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote) : "memory");
          sum += v;
        }
        if (n < p.n) store_as(p.out, (uint64_t)(at.token0 + tok) * p.out_ld + n, p.dtype, sum + bias);
      }
    }
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *failed) { *p.fault = 1; __threadfence_system(); }
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// Products over no columns: the bias, or zero.
__global__ void __launch_bounds__(256) mx_bias_kernel(ProductArgs p) {
  dependency_wait();
  allow_dependents();
  for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < (uint64_t)p.m * p.n; i += gridDim.x * 256ull) {
    const uint64_t row = i / p.n, n = i % p.n;
    uint32_t g = 0;
    if (p.offsets) {
      int64_t lo = min(max(__ldg(p.offsets), (int64_t)0), (int64_t)p.m);
      if ((int64_t)row < lo) continue;
      for (g = 0; g < p.groups; ++g) {
        lo = min(max(__ldg(p.offsets + g + 1), lo), (int64_t)p.m);
        if ((int64_t)row < lo) break;
      }
      if (g == p.groups) continue;
    }
    store_as(p.out, row * p.out_ld + n, p.dtype, p.bias ? p.bias[(uint64_t)g * p.n + n] : 0.f);
  }
}

// ------------------------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
  static EncodeTiled fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult how;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess) p = nullptr;
    return (EncodeTiled)p;
  }();
  return fn;
}

bool make_map(CUtensorMap* map, const MxView& m, uint32_t blocks, uint64_t rows, uint64_t groups, uint32_t box_rows) {
  EncodeTiled fn = encoder();
  if (!fn) return false;
  const cuuint64_t dims[3] = {16ull * blocks, rows, groups};
  const cuuint64_t strides[2] = {m.codes_ld, groups > 1 ? m.codes_gs : m.codes_ld};
  const cuuint32_t box[3] = {128, box_rows, 1}, ones[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, m.codes, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool vec16(const MxView& v) { return ((uintptr_t)v.scales | v.scales_ld | v.scales_gs) % 16 == 0; }

template <class S>
cudaError_t launch_shape(const Launch& l, const MxProduct& q, ProductArgs p, uint64_t* launches) {
  const MxView &x = S::TOKENS_X ? q.a : q.w, &y = S::TOKENS_X ? q.w : q.a;
  p.x_scales = x.scales; p.y_scales = y.scales;
  p.x_sld = x.scales_ld; p.y_sld = y.scales_ld; p.x_sgs = x.scales_gs; p.y_sgs = y.scales_gs;
  p.x_rows = S::TOKENS_X ? q.m : q.n; p.y_rows = S::TOKENS_X ? q.n : q.m;
  p.x_vec = vec16(x); p.y_vec = vec16(y);
  CUtensorMap mx, my;
  const uint64_t xg = S::TOKENS_X ? 1 : q.groups, yg = S::TOKENS_X ? q.groups : 1;
  if (!make_map(&mx, x, p.blocks, p.x_rows, xg, 128) || !make_map(&my, y, p.blocks, p.y_rows, yg, S::BN)) return cudaErrorNotSupported;
  p.w_tiles = (q.n + S::W_TILE - 1) / S::W_TILE;
  // no more row tiles than this, whatever the offsets say: every group has at most one tile that is not full
  uint64_t row_tiles = (q.m + S::ROW_TILE - 1) / S::ROW_TILE;
  if (q.groups > 1) row_tiles += q.groups < q.m ? q.groups : q.m;
  const uint64_t tiles = row_tiles * p.w_tiles;
  if (tiles > 0x7fffffffull) return cudaErrorInvalidValue;
  p.splits = 1;
  if (!S::TOKENS_X) {
    const uint32_t pairs = (p.steps + 1) / 2;
    while (p.splits < 8 && p.splits * 2 <= pairs && tiles * p.splits * 2 <= (uint64_t)l.sm_count) p.splits *= 2;
  }
  const uint32_t grid = p.splits > 1 ? (uint32_t)tiles * p.splits : (uint32_t)(tiles < (uint64_t)l.sm_count ? tiles : l.sm_count);
  static bool ready[64] = {};                // per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !ready[dev]) {
    e = cudaFuncSetAttribute(mx_matmul_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) ready[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(kProductThreads); cfg.dynamicSmemBytes = S::SMEM; cfg.stream = l.stream;
  cudaLaunchAttribute attr[2];
  uint32_t na = 0;
  if (l.pdl) { attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization; attr[na++].val.programmaticStreamSerializationAllowed = 1; }
  if (p.splits > 1) {
    attr[na].id = cudaLaunchAttributeClusterDimension;
    attr[na].val.clusterDim.x = p.splits; attr[na].val.clusterDim.y = 1; attr[na++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr; cfg.numAttrs = na;
  e = cudaLaunchKernelEx(&cfg, mx_matmul_kernel<S>, mx, my, p);
  if (e == cudaSuccess) ++*launches;
  return e;
}

using ManyRows = Shape<256, true, 4>;
using Few16 = Shape<16, false, 10>;
using Few32 = Shape<32, false, 9>;
using Few64 = Shape<64, false, 8>;
using Few128 = Shape<128, false, 6>;

}  // namespace

cudaError_t launch_mx_matmul(const Launch& l, const MxProduct& q, uint64_t* launches) {
  ProductArgs p = {};
  p.bias = q.bias; p.offsets = q.offsets; p.out = q.y; p.out_ld = q.y_ld; p.dtype = q.dtype;
  p.m = q.m; p.n = q.n; p.blocks = (q.k + 31) / 32; p.steps = (q.k + kStepCols - 1) / kStepCols; p.groups = q.groups;
  p.early = q.early; p.fault = q.fault;
  p.out_vec = ((uintptr_t)q.y % 16 == 0) && (q.y_ld * dtype_size(q.dtype)) % 16 == 0;
  if (p.steps == 0) {
    const uint64_t want = ((uint64_t)q.m * q.n + 255) / 256;
    cudaError_t e = launch_kernel(l, mx_bias_kernel, (uint32_t)(want < 4096 ? want : 4096), 256, p);
    if (e == cudaSuccess) ++*launches;
    return e;
  }
  const uint32_t per_weight = (q.m + q.groups - 1) / q.groups;     // average rows that meet one weight
  const uint64_t many_tiles = (uint64_t)((q.m + 127) / 128) * ((q.n + 255) / 256);
  if (per_weight > 64 && 2 * many_tiles > (uint64_t)l.sm_count) return launch_shape<ManyRows>(l, q, p, launches);
  if (per_weight <= 16) return launch_shape<Few16>(l, q, p, launches);
  if (per_weight <= 32) return launch_shape<Few32>(l, q, p, launches);
  if (per_weight <= 64) return launch_shape<Few64>(l, q, p, launches);
  return launch_shape<Few128>(l, q, p, launches);
}

}  // namespace qv2
