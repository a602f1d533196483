// Products of microscaled 4-bit matrices, dense and grouped by expert, on the fifth-generation tensor
// cores: y[i][j] = sum_k a[i][k] w[j][k], both operands in blocks of 32 codes with a power-of-two scale.
//
// tcgen05.mma.kind::mxf4 multiplies codes straight from shared memory and applies the two scales of each
// block of 32 inside the instruction; the accumulator (binary32) stays in tensor memory.  One CTA has
//   warp 0       fetches code tiles by TMA (128 bytes = 256 columns per row and step, 128-byte swizzle),
//   warp 1       copies the scales from shared to tensor memory and issues the products,
//   warp 2       owns the tensor memory,
//   warps 4-11   move finished accumulators out (two warps per quarter of the 128 accumulator rows),
//   warps 12-15  bring the scales: they lie row by row in memory, the tensor core wants them four to a
//                word and 32 rows to a column, so each thread fetches 16 bytes of its row (two steps) with
//                cp.async, four of those ahead, and deals them out through registers.
// A ring of shared-memory stages decouples them; accumulators are double-buffered.
//
// The 128-row operand X and the BN-row operand Y take either role:
//   tokens as X, weights as Y (BN = 256): the many-row form.  Two CTAs share a 256 x 256 tile
//   (cta_group::2), since a 128 x 256 tile of one asks L2 for 48 KB a step of 512 tensor cycles, 96 bytes a
//   cycle and SM, more than it delivers (880 cycles a step; 580 in pairs).  8192 x 8192 x 8192 takes 239 us
//   back to back (4.6 PFLOP/s, 2.8 times the measured bf16 rate; the clock settles at 1380 MHz) and 203 in a
//   burst after a pause, 16411 x 4096 x 2048 in 16 groups 92 and 78 us.  What bounds it: the tensor cores under
//   the power limit (constant codes take 167 instead of 203 us in a burst), and some 700 cycles between tiles,
//   in which the shared columns of the accumulators are read out.
//   weights as X, tokens as Y (BN = 16..128): few rows per weight, bound by reading the weights once; the
//   columns may be cut over the CTAs of a cluster, whose partial sums are added through distributed
//   shared memory in the order of the ranks.  A step takes at least 480 cycles whatever BN (four products
//   and four copies of scales), 8 TB/s over all SMs; 1 x 4096 x 25088 takes 14.3 us beside 8.4 us for its bytes
//   at the copy rate: 128 of 148 SMs, 2.4 us until the first tile is there, 2 us to join the four partial sums.
#include <cuda.h>

#include "qv2_mx.cuh"

namespace qv2 {

namespace {

constexpr int kProductThreads = 512;
constexpr uint32_t kStepCols = 256;              // columns per stage: 128 bytes of codes
constexpr uint64_t kWaitLimitNs = 2000000000ull; // a wait that lasts this long gives up
constexpr uint32_t kMaxGroups = QV2_MX_MAX_GROUPS;

// ------------------------------------------------------------------------------------ PTX wrappers
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
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

// One lane of the warp, the same each time.  Work issued by one thread stands behind this test and not behind a
// lane number: the values it needs are then known to be the warp's own and are kept in uniform registers (with
// `lane == 0` a step of the product took 950 cycles to issue).
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
  return ok != 0;
}

// The warp waits for the phase of `parity` to complete.  false, for all of its lanes: this wait or another of the
// CTA has given up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* failed) {
  bool ok = bar_try(bar, parity);
  if (__all_sync(0xffffffffu, ok)) return true;
  uint64_t begin = 0;
  for (uint32_t i = 1; !ok; ++i) {
    ok = bar_try(bar, parity);
    if (!ok && (i & 255u) == 0) {
      if (*failed) break;
      const uint64_t t = now_ns();
      if (!begin) begin = t;
      else if (t - begin > kWaitLimitNs) { *failed = 1; break; }
    }
  }
  return __all_sync(0xffffffffu, ok);
}

// PAIR: the two CTAs of a cluster work on one tile; copies of either report to the first one's barrier.
template <bool PAIR>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  if constexpr (PAIR)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_store(uint32_t src, const CUtensorMap* map, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y) : "memory");
}
// Arrives at `bar` (PAIR: at the same place in both CTAs) when the tensor work issued so far is done.
template <bool PAIR>
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {      // the same place in another CTA of the cluster
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// Arrives at a barrier of this CTA, or (PAIR) at one given by at_rank.  What has to be seen with the arrival is shared
// memory of the arriving CTA, read by its own tensor core after fence.proxy.async, and tensor memory, ordered by
// tcgen05.fence; a release to the whole cluster would besides wait for all global traffic that the thread has in
// flight, and took 1500 to 2200 cycles a step.
template <bool PAIR>
__device__ __forceinline__ void bar_arrive_at(uint32_t bar) {
  if constexpr (PAIR) asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
  else asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Scales of 128 rows by 4 blocks: 512 consecutive bytes, 16 for each of 32 lanes, into 4 columns of all
// four lane quarters.  (PAIR: each CTA from its own shared to its own tensor memory.)
template <bool PAIR>
__device__ __forceinline__ void tc_copy_scales(uint32_t column, uint64_t desc) {
  if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(column), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(column), "l"(desc) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  if constexpr (PAIR)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
  else
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
  static constexpr bool PAIR = TOKENS_X;                   // two CTAs per tile: each has half of X's and of Y's rows
  static constexpr int CTAS = PAIR ? 2 : 1;
  static constexpr int ROW_TILE = TOKENS_X ? 128 * CTAS : BN;     // tokens per tile
  static constexpr int W_TILE = TOKENS_X ? BN : 128;       // weight rows per tile
  static constexpr int Y_ROWS = BN / CTAS;                 // rows of Y's codes that a CTA holds; it holds the scales of all
  static constexpr int YB = (BN + 127) / 128;              // 128-row groups of Y's scales
  static constexpr uint32_t X_BYTES = 128 * 128, Y_BYTES = Y_ROWS * 128;
  static constexpr uint32_t SF_BYTES = 2 * 512 * (1 + YB);
  static constexpr uint32_t STAGE = X_BYTES + Y_BYTES + SF_BYTES;
  // Two accumulators of 256 columns and the scales do not fit 512 columns: the second one begins 64
  // columns before the first one's end, and a tile waits for those columns of its predecessor only.
  static constexpr bool OVERLAP = BN == 256;
  static constexpr uint32_t ACC_STEP = OVERLAP ? 192 : BN;
  static constexpr uint32_t SF_COL = OVERLAP ? 448 : 2 * BN;
  static constexpr uint32_t SF_SET = 8 + 8 * YB;           // columns of one step's scales; two sets alternate
  static_assert(SF_COL + 2 * SF_SET <= 512, "tensor memory");
  static constexpr uint32_t AHEAD = 4;                     // pairs of steps whose scales are on their way
  static constexpr uint32_t RAW_SLOT = 128 * 16 * (1 + YB), RAW = AHEAD * RAW_SLOT;
  static constexpr uint32_t STAGING = TOKENS_X ? 8 * 2048 : 0;    // per result warp: 32 rows of 64 bytes
  static constexpr uint32_t BIAS = TOKENS_X ? 8 * (BN / 2) * 4 : 0;
  static constexpr uint32_t TABLES = 2 * 4 * (kMaxGroups + 2);
  static constexpr uint32_t SMEM = 1024 + STAGES * STAGE + RAW + STAGING + BIAS + TABLES + 512;
  static_assert(SMEM <= 232448, "shared memory");
  // E2M1 x E2M1, E8M0 scales, 128 (PAIR: 256) x BN
  static constexpr uint32_t IDESC = (1u << 7) | (1u << 10) | ((uint32_t)(BN / 8) << 17) | (1u << 23) | ((8u * CTAS) << 24);
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
  uint32_t dtype, out_align;                 // out_align: rows of the result start at multiples of 16 (as TMA needs), 4 or 2 bytes
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

// n <= 16 scale bytes into this thread's 16 bytes of shared memory, zeros behind them.  Aligned ones are fetched
// in the background (cp.async, completed by its group).
__device__ __noinline__ void bring_bytes(uint8_t* dst, const uint8_t* src, uint32_t n) {
  for (uint32_t i = 0; i < 16; ++i) dst[i] = i < n ? __ldg(src + i) : (uint8_t)0;
}
__device__ __forceinline__ void bring_scales(uint8_t* dst, const uint8_t* src, uint32_t n, bool vec) {
  if (vec) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(n) : "memory");
  else bring_bytes(dst, src, n);
}

__device__ __forceinline__ void store_as(void* y, uint64_t at, uint32_t dtype, float v) {
  if (dtype == kBF16) ((__nv_bfloat16*)y)[at] = __float2bfloat16_rn(v);
  else if (dtype == kF16) ((__half*)y)[at] = __float2half_rn(v);
  else ((float*)y)[at] = v;
}
// 16 results that lie `ld` apart.
template <class T>
__device__ __forceinline__ void store_column(T* y, uint64_t ld, const uint32_t (&v)[16], float bias, uint32_t n) {
#pragma unroll
  for (uint32_t j = 0; j < 16; ++j)
    if (j < n) y[j * ld] = Chunk8<T>::narrow(__uint_as_float(v[j]) + bias);
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
mx_matmul_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_out,
                 const ProductArgs p) {
  constexpr bool PAIR = S::PAIR;
  extern __shared__ uint8_t raw[];
  const uint32_t raw_addr = smem_addr(raw);
  uint8_t* const base = raw + ((1024u - (raw_addr & 1023u)) & 1023u);     // swizzled tiles start at multiples of 1024
  const uint32_t base_addr = smem_addr(base);
  // codes of all stages, scales of all stages, scales as they lie in memory, then the rest
  constexpr uint32_t CODES = S::X_BYTES + S::Y_BYTES;
  uint8_t* const sf = base + S::STAGES * CODES;
  const uint32_t sf_addr = base_addr + S::STAGES * CODES;
  uint8_t* const bytes_ring = sf + S::STAGES * S::SF_BYTES;
  uint8_t* const staging = bytes_ring + S::RAW;
  float* const bias_rows = reinterpret_cast<float*>(staging + S::STAGING);
  uint32_t* const lo = reinterpret_cast<uint32_t*>(staging + S::STAGING + S::BIAS);
  uint32_t* const cum = lo + kMaxGroups + 2;
  uint64_t* const bars = reinterpret_cast<uint64_t*>(cum + kMaxGroups + 2);
  const uint32_t bar0 = smem_addr(bars);
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t half = PAIR ? blockIdx.x % 2 : 0;                         // place in the pair; the first one issues the products
  auto full = [&](uint32_t s) { return bar0 + 8 * s; };                    // codes and scales of a stage are there (first CTA's counts)
  auto empty = [&](uint32_t s) { return bar0 + 8 * (S::STAGES + s); };
  auto acc_full = [&](uint32_t b) { return bar0 + 8 * (2 * S::STAGES + b); };
  auto acc_free = [&](uint32_t b) { return bar0 + 8 * (2 * S::STAGES + 2 + b); };   // (first CTA's counts)
  const uint32_t drained = bar0 + 8 * (2 * S::STAGES + 4);
  static_assert(8 * (2 * S::STAGES + 5) + 8 <= 512, "barriers");
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * S::STAGES + 5);
  volatile uint32_t* const failed = tmem_slot + 1;

  if (!p.early) dependency_wait();
  allow_dependents();

  // group tables: lo[g] = first token of group g (clamped, never decreasing), cum[g] = row tiles before it
  for (uint32_t g = threadIdx.x; p.groups > 1 && g <= p.groups; g += kProductThreads) {
    const int64_t o = __ldg(p.offsets + g);
    lo[g] = (uint32_t)(o < 0 ? 0 : o > (int64_t)p.m ? (int64_t)p.m : o);
  }
  if (warp == 3) {
    if (elect_one()) {
#pragma unroll 1
      for (uint32_t s = 0; s < S::STAGES; ++s) { bar_init(full(s), 1 + 4 * S::CTAS); bar_init(empty(s), 1); }
#pragma unroll 1
      for (uint32_t b = 0; b < 2; ++b) { bar_init(acc_full(b), 1); bar_init(acc_free(b), 8 * S::CTAS); }
      bar_init(drained, 1);
      *failed = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
  } else if (warp == 2) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(tmem_slot)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(tmem_slot)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  } else if (warp == 0) {
    if (elect_one()) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&map_y) : "memory");
    }
    __syncwarp();
  }
  if (p.groups > 1) {
    __syncthreads();
    if (warp == 4) {
      uint32_t carry = 0;
#pragma unroll 1
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
#pragma unroll 1
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
  } else if (threadIdx.x == 128) {
    const int64_t m = p.m, first = p.offsets ? min(max(__ldg(p.offsets), (int64_t)0), m) : 0, last = p.offsets ? min(max(__ldg(p.offsets + 1), first), m) : m;
    lo[0] = (uint32_t)first; lo[1] = (uint32_t)last;
    cum[0] = 0; cum[1] = (uint32_t)(last - first + S::ROW_TILE - 1) / S::ROW_TILE;
  }
  __syncwarp();
  tc_fence_before();
  if constexpr (PAIR) cluster_sync(); else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  // this CTA's (pair's) tiles: tile0, tile0 + stride, ...; the steps of a tile are cut over the cluster in twos
  const uint32_t rank = PAIR ? 0 : blockIdx.x % p.splits, width = PAIR ? 2 : p.splits;
  const uint32_t tile0 = blockIdx.x / width, stride = gridDim.x / width;
  const uint32_t twos = (p.steps + 1) / 2;
  const uint32_t step_begin = 2 * (uint32_t)((uint64_t)twos * rank / p.splits);
  const uint32_t step_end = min(p.steps, 2 * (uint32_t)((uint64_t)twos * (rank + 1) / p.splits));
  Where at = {};

  if (warp == 0) {
    // ---------------------------------------------------------------------------------- codes
    uint32_t s = 0, phase = 1, fills = 0;     // the first wait for an empty stage is for the phase before the first
    const uint32_t full0 = PAIR ? at_rank(full(0), 0) : full(0);
    auto fetch = [&](uint32_t stage, uint32_t step, bool weights) {
      const bool x = weights != S::TOKENS_X;
      const int row = (int)(weights ? at.w0 + (x ? 0 : S::Y_ROWS * half) : at.token0 + (x ? 128 * half : 0));
      tma_load<PAIR>(base_addr + stage * CODES + (x ? 0 : S::X_BYTES), x ? &map_x : &map_y, full0 + 8 * stage, (int)step * 128, row, weights ? (int)at.group : 0);
    };
    bool first = p.early != 0, ok = true;
#pragma unroll 1
    for (uint32_t tile = tile0; ok && find_tile<S>(lo, cum, p.groups, p.w_tiles, tile, &at); tile += stride) {
      uint32_t step = step_begin;
      if (first) {
        // the weights of the first stages do not depend on the kernel that is rounding the activations
        const uint32_t n = min(step_end - step, (uint32_t)S::STAGES);
        if (elect_one()) {
#pragma unroll 1
          for (uint32_t i = 0; i < n; ++i) {
            if (half == 0) bar_expect(full(i), S::CTAS * CODES);
            fetch(i, step + i, true);
          }
        }
        __syncwarp();
        dependency_wait();
        if (elect_one()) {
#pragma unroll 1
          for (uint32_t i = 0; i < n; ++i) fetch(i, step + i, false);
        }
        __syncwarp();
        step += n; fills = n; s = n;
        if (s == S::STAGES) { s = 0; phase = 0; }
        first = false;
      }
#pragma unroll 1
      for (; step < step_end; ++step) {
        if (!bar_wait(empty(s), phase, failed)) { ok = false; break; }
        if (elect_one()) {
          if (half == 0) bar_expect(full(s), S::CTAS * CODES);
          fetch(s, step, true);
          fetch(s, step, false);
        }
        __syncwarp();
        ++fills;
        if (++s == S::STAGES) { s = 0; phase ^= 1; }
      }
    }
    if (*failed) {                            // leave no copy in flight: what was asked for last has landed long before the limit passes
      const uint64_t begin = now_ns();
      for (uint32_t i = fills > S::STAGES ? fills - S::STAGES : 0; i < fills; ++i)
        while (!bar_try(full(i % S::STAGES), (i / S::STAGES) & 1) && now_ns() - begin < kWaitLimitNs / 20) {}
    }
  } else if (warp == 1 && half == 0) {
    // ---------------------------------------------------------------------------------- products
    uint32_t s = 0, phase = 0, set = 0, done = 0;
#pragma unroll 1
    for (uint32_t tile = tile0; find_tile<S>(lo, cum, p.groups, p.w_tiles, tile, &at); tile += stride, ++done) {
      const uint32_t b = done & 1;
      // OVERLAP: the predecessor has left the shared columns; else: the tile before it has left this buffer
      if (S::OVERLAP ? done >= 1 && !bar_wait(acc_free(b ^ 1), ((done - 1) / 2) & 1, failed)
                     : done >= 2 && !bar_wait(acc_free(b), (done / 2 - 1) & 1, failed)) break;
      tc_fence_after();
      const uint32_t acc = tmem + b * S::ACC_STEP;
      bool ok = true;
#pragma unroll 1
      for (uint32_t step = step_begin; step < step_end; ++step) {
        if (!bar_wait(full(s), phase, failed)) { ok = false; break; }
        tc_fence_after();
        if (elect_one()) {
          const uint32_t sfx = tmem + S::SF_COL + set, sfy = sfx + 8;
          const uint64_t src = scales_desc(sf_addr + s * S::SF_BYTES);
#pragma unroll
          for (uint32_t h = 0; h < 2; ++h) {
            tc_copy_scales<PAIR>(sfx + 4 * h, src + 32 * h);
#pragma unroll
            for (uint32_t y = 0; y < S::YB; ++y) tc_copy_scales<PAIR>(sfy + 4 * (h * S::YB + y), src + 64 + 32 * (h * S::YB + y));
          }
          const uint64_t dx = codes_desc(base_addr + s * CODES), dy = codes_desc(base_addr + s * CODES + S::X_BYTES);
#pragma unroll
          for (uint32_t k = 0; k < 4; ++k) {  // 64 columns each: 32 bytes along the row, two of the word's four scales
            const uint32_t id = 2 * (k & 1);
            tc_mma<PAIR>(acc, dx + 2 * k, dy + 2 * k, S::IDESC | (id << 29) | (id << 4), sfx + 4 * (k / 2), sfy + 4 * S::YB * (k / 2),
                         step > step_begin || k > 0);
          }
          tc_commit<PAIR>(empty(s));
        }
        __syncwarp();
        set ^= S::SF_SET;
        if (++s == S::STAGES) { s = 0; phase ^= 1; }
      }
      if (!ok) break;
      if (elect_one()) tc_commit<PAIR>(acc_full(b));
      __syncwarp();
    }
    if (*failed) {                            // leave no product in flight
      if (elect_one()) tc_commit<PAIR>(drained);
      __syncwarp();
      const uint64_t begin = now_ns();
      while (!bar_try(drained, 0) && now_ns() - begin < kWaitLimitNs) {}
    }
  } else if (warp >= 12) {
    // ---------------------------------------------------------------------------------- scales
    const uint32_t t = threadIdx.x - 384;
    if (p.early) dependency_wait();
    const uint32_t full0 = PAIR ? at_rank(full(0), 0) : full(0);
    const bool vec_x = p.x_vec != 0, vec_y = p.y_vec != 0;
    uint8_t* const mine = bytes_ring + 16 * t;     // of slot i: + i * RAW_SLOT; X's row, then 2048 bytes on Y's, and its row 128 below
    // The sequence of pairs of steps, fetched AHEAD of the one that is unpacked.  Rows past the end of a matrix keep what
    // the slot held: they scale results that nobody stores.  (Fetching the last row's scales for them made a product
    // of 333 rows take 41 us, one of 512 rows 19: hundreds of lanes asked for the same few bytes.)
    uint32_t tile = tile0, two = 0, slot_in = 0;
    const uint8_t *px = nullptr, *py[S::YB];
    bool in_x = false, in_y[S::YB];
    bool live = find_tile<S>(lo, cum, p.groups, p.w_tiles, tile, &at);
    auto enter = [&] {
      two = step_begin / 2;
      const uint32_t xr = (S::TOKENS_X ? at.token0 + 128 * half : at.w0) + t;
      in_x = xr < p.x_rows;
      px = p.x_scales + (S::TOKENS_X ? 0 : at.group * p.x_sgs) + xr * p.x_sld + 16ull * two;
#pragma unroll
      for (int i = 0; i < S::YB; ++i) {
        const uint32_t yr = (S::TOKENS_X ? at.w0 : at.token0) + t + 128 * i;
        in_y[i] = t + 128 * i < S::BN && yr < p.y_rows;
        py[i] = p.y_scales + (S::TOKENS_X ? at.group * p.y_sgs : 0) + yr * p.y_sld + 16ull * two;
      }
    };
    auto fetch = [&] {                             // one pair of steps into the next slot, or nothing; always one group
      if (live) {
        uint8_t* dst = mine + slot_in * S::RAW_SLOT;
        const uint32_t n = min(p.blocks - 16 * two, 16u);
        if (in_x) bring_scales(dst, px, n, vec_x);
        px += 16;
#pragma unroll
        for (int i = 0; i < S::YB; ++i) {
          if (in_y[i]) bring_scales(dst + 2048 * (1 + i), py[i], n, vec_y);
          py[i] += 16;
        }
        if (2 * ++two >= step_end) {
          tile += stride;
          live = find_tile<S>(lo, cum, p.groups, p.w_tiles, tile, &at);
          if (live) enter();
        }
      }
      slot_in = slot_in + 1 == S::AHEAD ? 0 : slot_in + 1;
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (live) enter();
#pragma unroll 1
    for (uint32_t i = 0; i + 1 < S::AHEAD; ++i) fetch();
    uint32_t s = 0, phase = 1, slot = 0;
    const uint32_t word = (t % 32) * 16 + (t / 32) * 4;
    Where now;
    bool ok = true;
#pragma unroll 1
    for (uint32_t tile_now = tile0; ok && find_tile<S>(lo, cum, p.groups, p.w_tiles, tile_now, &now); tile_now += stride) {
#pragma unroll 1
      for (uint32_t step = step_begin; step < step_end; step += 2) {
        fetch();
        asm volatile("cp.async.wait_group %0;" ::"n"(S::AHEAD - 1) : "memory");
        // both steps at once
        const bool both = step + 1 < step_end;
        const uint32_t s1 = s + 1 == S::STAGES ? 0 : s + 1, phase1 = s + 1 == S::STAGES ? phase ^ 1 : phase;
        if (!bar_wait(empty(s), phase, failed) || (both && !bar_wait(empty(s1), phase1, failed))) { ok = false; break; }
        const uint8_t* src = mine + slot * S::RAW_SLOT;
        uint8_t *d0 = sf + s * S::SF_BYTES + word, *d1 = sf + s1 * S::SF_BYTES + word;
#pragma unroll
        for (int i = 0; i <= S::YB; ++i) {         // X, then Y's groups of 128 rows
          const uint4 v = *reinterpret_cast<const uint4*>(src + 2048 * i);
          const uint32_t at0 = i == 0 ? 0 : 1024 + 512 * (i - 1), at1 = i == 0 ? 512 : 1024 + 512 * (S::YB + i - 1);
          *reinterpret_cast<uint32_t*>(d0 + at0) = v.x;
          *reinterpret_cast<uint32_t*>(d0 + at1) = v.y;
          if (both) {
            *reinterpret_cast<uint32_t*>(d1 + at0) = v.z;
            *reinterpret_cast<uint32_t*>(d1 + at1) = v.w;
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          bar_arrive_at<PAIR>(full0 + 8 * s);
          if (both) bar_arrive_at<PAIR>(full0 + 8 * s1);
        }
        slot = slot + 1 == S::AHEAD ? 0 : slot + 1;
        s = s1; phase = phase1;
        if (both && ++s == S::STAGES) { s = 0; phase ^= 1; }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= 4) {
    // ---------------------------------------------------------------------------------- results
    const uint32_t quarter = warp % 4;        // the lanes that a warp may read follow from its number
    const uint32_t side = (warp - 4) / 4;     // which half of the columns
    const uint32_t lanes = (quarter * 32) << 16;
    if (p.early) dependency_wait();
    const uint32_t free0 = PAIR ? at_rank(acc_free(0), 0) : acc_free(0);
    constexpr uint32_t COLS = S::BN / 2;      // TOKENS_X: columns of this warp
    float* const bias_row = bias_rows + (warp - 4) * COLS;
    float ahead[COLS / 32 ? COLS / 32 : 1];   // TOKENS_X: this lane's part of the next tile's bias, fetched a tile ahead
    auto fetch_bias = [&](const Where& w) {
#pragma unroll
      for (uint32_t i = 0; i < COLS / 32; ++i) {
        const uint32_t n = w.w0 + side * COLS + 32 * i + lane;
        ahead[i] = n < p.n ? __ldg(p.bias + (uint64_t)w.group * p.n + n) : 0.f;
      }
    };
    uint32_t done = 0;
    Where then;
    bool more = find_tile<S>(lo, cum, p.groups, p.w_tiles, tile0, &then);
    if (S::TOKENS_X && p.bias && more) fetch_bias(then);
#pragma unroll 1
    for (uint32_t tile = tile0; more; tile += stride, ++done) {
      const uint32_t b = done & 1;
      at = then;
      if constexpr (S::TOKENS_X) {
        const uint32_t w0 = at.w0 + side * COLS;
        if (p.bias) {
#pragma unroll
          for (uint32_t i = 0; i < COLS / 32; ++i) bias_row[32 * i + lane] = ahead[i];
          __syncwarp();
        }
        more = find_tile<S>(lo, cum, p.groups, p.w_tiles, tile + stride, &then);
        if (p.bias && more) fetch_bias(then);
        if (!bar_wait(acc_full(b), (done / 2) & 1, failed)) break;
        tc_fence_after();
        const uint32_t acc = tmem + b * S::ACC_STEP + side * COLS + lanes;
        // The columns shared with the next tile are the last 64 of the first buffer and the first 64 of the second:
        // they go first, and a warp that has none of them lets the next tile in at once.
        const bool shares = side != b;
        if (!shares && lane == 0) bar_arrive_at<PAIR>(free0 + 8 * b);        // (also: done with the tile before)
        // lane = token, columns = weight rows, 32 at a time.  They pass through 2 KB of shared memory (rows
        // of 64 bytes: 32 results of 16 bits, or in two rounds 16 of 32 bits) and leave as a tile by TMA.  Where the result's
        // rows are not aligned for TMA, or a group ends inside the tile, the warp stores the rows side by side itself.  (Every
        // lane storing its own row took 4096 or more cycles of the load/store unit a tile and held up the products, whose
        // barriers and operands share that unit; in single elements a product of 6385 x 3738 x 262 took 262 us.)
        const uint32_t row0 = at.token0 + 128 * half + quarter * 32;
        const uint32_t rows = row0 < at.token_end ? min(32u, at.token_end - row0) : 0;
        const bool by_tma = p.out_align == 16 && rows == 32;
        const uint32_t shift = p.dtype == kF32 ? 2 : 1;
        uint8_t* const mine = staging + (warp - 4) * 2048;
        uint8_t* const put = mine + lane * 64;
        const uint32_t put_sw = ((lane >> 1) & 3) * 16;                          // the 64-byte swizzle
        auto column = [&](uint32_t c) { return 32 * (b == 0 ? c ^ 2 : c); };
        uint32_t next[32];
        tc_load32(acc + column(0), next);
        tc_load_wait();
#pragma unroll 1
        for (uint32_t c = 0; c < COLS / 32; ++c) {
          uint32_t v[32];
#pragma unroll
          for (uint32_t j = 0; j < 32; ++j) v[j] = next[j];
          if (c + 1 < COLS / 32) {
            tc_load32(acc + column(c + 1), next);
            tc_load_wait();
          }
          if (c == 0 && shares) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive_at<PAIR>(free0 + 8 * b);
          }
          const uint32_t col = column(c), cols = w0 + col < p.n ? min(p.n - w0 - col, 32u) : 0;
          if (cols == 0 || rows == 0) continue;
          if (p.bias) {
#pragma unroll
            for (uint32_t j = 0; j < 32; j += 4) {
              const float4 f = *reinterpret_cast<const float4*>(bias_row + col + j);
              v[j] = __float_as_uint(__uint_as_float(v[j]) + f.x); v[j + 1] = __float_as_uint(__uint_as_float(v[j + 1]) + f.y);
              v[j + 2] = __float_as_uint(__uint_as_float(v[j + 2]) + f.z); v[j + 3] = __float_as_uint(__uint_as_float(v[j + 3]) + f.w);
            }
          }
          if (p.dtype == kBF16) {
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) v[j] = pack2(kBF16, __uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
          } else if (p.dtype == kF16) {
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) v[j] = pack2(kF16, __uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
          }
#pragma unroll 1
          for (uint32_t round = 0; round < shift; ++round) {
            if (elect_one()) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");     // the last tile has been read out
            __syncwarp();
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
              *reinterpret_cast<uint4*>(put + ((16 * j) ^ put_sw)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) v[j] = v[16 + j];
            if (by_tma) {
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (elect_one()) {
                tma_store(smem_addr(mine), &map_out, (int)(w0 + col + 16 * round), (int)row0);
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
              }
            } else {
              __syncwarp();
              const uint32_t left = cols > 16 * round ? cols - 16 * round : 0, bytes = min(left << shift, 64u);
              uint8_t* const to = (uint8_t*)p.out + (((uint64_t)row0 * p.out_ld + w0 + col + 16 * round) << shift);
              const uint64_t pitch = p.out_ld << shift;
              auto staged = [&](uint32_t r, uint32_t b) { return mine + r * 64 + (((b / 16) ^ ((r >> 1) & 3)) * 16) + b % 16; };
              if (p.out_align == 16 && bytes == 64) {          // a row by four lanes
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                  const uint32_t r = 8 * i + lane / 4, at_byte = 16 * (lane % 4);
                  if (r < rows) *reinterpret_cast<uint4*>(to + r * pitch + at_byte) = *reinterpret_cast<const uint4*>(staged(r, at_byte));
                }
              } else if (p.out_align >= 4) {                   // by sixteen
                const uint32_t at_byte = 4 * (lane % 16);
#pragma unroll 4
                for (uint32_t r = lane / 16; r < rows; r += 2) {
                  if (at_byte + 4 <= bytes) *reinterpret_cast<uint32_t*>(to + r * pitch + at_byte) = *reinterpret_cast<const uint32_t*>(staged(r, at_byte));
                  else if (at_byte < bytes) *reinterpret_cast<uint16_t*>(to + r * pitch + at_byte) = *reinterpret_cast<const uint16_t*>(staged(r, at_byte));
                }
              } else {                                         // by all (16-bit results on odd addresses of two bytes)
                const uint32_t at_byte = 2 * lane;
#pragma unroll 4
                for (uint32_t r = 0; r < rows; ++r)
                  if (at_byte < bytes) *reinterpret_cast<uint16_t*>(to + r * pitch + at_byte) = *reinterpret_cast<const uint16_t*>(staged(r, at_byte));
              }
            }
            __syncwarp();
          }
        }
        // What was read from this buffer above is ordered before the warp's next arrival (which lets the products into it).
        tc_fence_before();
        __syncwarp();
      } else {
        more = find_tile<S>(lo, cum, p.groups, p.w_tiles, tile + stride, &then);
        if (!bar_wait(acc_full(b), (done / 2) & 1, failed)) break;
        tc_fence_after();
        const uint32_t acc = tmem + b * S::ACC_STEP + lanes;
        // lane = weight row, columns = tokens: 32 lanes write neighbouring results
        const uint32_t n = at.w0 + quarter * 32 + lane;
        const float bias = p.bias && n < p.n ? __ldg(p.bias + (uint64_t)at.group * p.n + n) : 0.f;
        const uint32_t tokens = min((uint32_t)S::BN, at.token_end - at.token0);
        float* part = reinterpret_cast<float*>(base) + quarter * 32 + lane;     // [token][128], over stages that are done with
#pragma unroll 1
        for (uint32_t c = 16 * side; c < tokens; c += 32) {
          uint32_t v[16];
          tc_load16(acc + c, v);
          tc_load_wait();
          if (p.splits > 1) {
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) part[(c + j) * 128] = __uint_as_float(v[j]);
          } else if (n < p.n) {
            const uint64_t to = (uint64_t)(at.token0 + c) * p.out_ld + n;
            if (p.dtype == kBF16) store_column<__nv_bfloat16>((__nv_bfloat16*)p.out + to, p.out_ld, v, bias, tokens - c);
            else if (p.dtype == kF16) store_column<__half>((__half*)p.out + to, p.out_ld, v, bias, tokens - c);
            else store_column<float>((float*)p.out + to, p.out_ld, v, bias, tokens - c);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_at<false>(free0 + 8 * b);
      }
    }
  }
  if constexpr (S::TOKENS_X) {
    if (warp >= 4 && warp < 12 && elect_one()) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  __syncwarp();

  if (!S::TOKENS_X && p.splits > 1) {
    // One tile per cluster: each rank adds up its share of the tokens over all ranks, in their order.  A warp takes a
    // token, a lane four weight rows of it: remote shared memory is bound by requests, 16 bytes a lane are the widest.
    cluster_sync();
    if (find_tile<S>(lo, cum, p.groups, p.w_tiles, tile0, &at)) {
      const uint32_t n = at.w0 + 4 * lane;
      const uint32_t tokens = min((uint32_t)S::BN, at.token_end - at.token0);
      float bias[4];
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) bias[k] = p.bias && n + k < p.n ? __ldg(p.bias + (uint64_t)at.group * p.n + n + k) : 0.f;
#pragma unroll 1
      for (uint32_t tok = rank + p.splits * warp; tok < tokens; tok += p.splits * (kProductThreads / 32)) {
        float4 v[8];
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r) {
          v[r] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (r < p.splits)
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[r].x), "=f"(v[r].y), "=f"(v[r].z), "=f"(v[r].w)
                         : "r"(at_rank(base_addr + tok * 512 + lane * 16, r)));
        }
        float4 sum = v[0];
#pragma unroll
        for (uint32_t r = 1; r < 8; ++r)
          if (r < p.splits) { sum.x += v[r].x; sum.y += v[r].y; sum.z += v[r].z; sum.w += v[r].w; }
        const uint64_t to = (uint64_t)(at.token0 + tok) * p.out_ld + n;
        const float y[4] = {sum.x + bias[0], sum.y + bias[1], sum.z + bias[2], sum.w + bias[3]};
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
          if (n + k < p.n) store_as(p.out, to + k, p.dtype, y[k]);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  // no CTA of a cluster leaves while another may still read its memory or arrive at its barriers
  if (PAIR || p.splits > 1) cluster_sync(); else __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *failed) { *p.fault = 1; __threadfence_system(); }
  if (warp == 2) {
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
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

// The result as the many-row form stores it: boxes of 32 rows by 64 bytes.
bool make_out_map(CUtensorMap* map, const MxProduct& q) {
  const uint32_t esz = dtype_size(q.dtype);
  const cuuint64_t dims[2] = {q.n, q.m}, strides[1] = {q.y_ld * esz};
  const cuuint32_t box[2] = {64 / esz, 32}, ones[2] = {1, 1};
  return encoder()(map, esz == 4 ? CU_TENSOR_MAP_DATA_TYPE_UINT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, q.y, dims, strides, box, ones,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool vec16(const MxView& v) { return ((uintptr_t)v.scales | v.scales_ld | v.scales_gs) % 16 == 0; }

// No more tiles than this, whatever the offsets say: every group has at most one row tile that is not full.
template <class S>
uint64_t most_tiles(uint64_t m, uint64_t n, uint64_t groups) {
  uint64_t row_tiles = (m + S::ROW_TILE - 1) / S::ROW_TILE;
  if (groups > 1) row_tiles += groups < m ? groups : m;
  return row_tiles * ((n + S::W_TILE - 1) / S::W_TILE);
}

constexpr int kDevices = 64;                 // answers are kept for this many devices

template <class S>
cudaError_t allow_shared(int dev) {
  static bool done[kDevices] = {};
  if (dev < kDevices && done[dev]) return cudaSuccess;
  cudaError_t e = cudaFuncSetAttribute(mx_matmul_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM);
  if (e == cudaSuccess && dev < kDevices) done[dev] = true;
  return e;
}

// Clusters of `width` CTAs that the device holds at one time (0: it could not be asked).
template <class S>
uint32_t resident_clusters(int dev, uint32_t width) {
  static uint32_t known[kDevices][4] = {};   // per log2 of the width; stored plus one
  const uint32_t w = width == 8 ? 3 : width == 4 ? 2 : 1;
  if (dev < kDevices && known[dev][w]) return known[dev][w] - 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(width); cfg.blockDim = dim3(kProductThreads); cfg.dynamicSmemBytes = S::SMEM;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = width; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, mx_matmul_kernel<S>, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
  if (dev < kDevices) known[dev][w] = (uint32_t)n + 1;
  return (uint32_t)n;
}

template <class S>
cudaError_t launch_shape(const Launch& l, const MxProduct& q, ProductArgs p, uint64_t* launches) {
  const MxView &x = S::TOKENS_X ? q.a : q.w, &y = S::TOKENS_X ? q.w : q.a;
  p.x_scales = x.scales; p.y_scales = y.scales;
  p.x_sld = x.scales_ld; p.y_sld = y.scales_ld; p.x_sgs = x.scales_gs; p.y_sgs = y.scales_gs;
  p.x_rows = S::TOKENS_X ? q.m : q.n; p.y_rows = S::TOKENS_X ? q.n : q.m;
  p.x_vec = vec16(x); p.y_vec = vec16(y);
  CUtensorMap mx, my, mo = {};
  const uint64_t xg = S::TOKENS_X ? 1 : q.groups, yg = S::TOKENS_X ? q.groups : 1;
  if (!make_map(&mx, x, p.blocks, p.x_rows, xg, 128) || !make_map(&my, y, p.blocks, p.y_rows, yg, S::Y_ROWS)) return cudaErrorNotSupported;
  const uint64_t row_bytes = q.y_ld * dtype_size(q.dtype);
  const uint64_t where = (uintptr_t)q.y | row_bytes;
  p.out_align = where % 16 == 0 && row_bytes < (1ull << 40) ? 16 : where % 4 == 0 ? 4 : 2;
  if (S::TOKENS_X && p.out_align == 16 && !make_out_map(&mo, q)) return cudaErrorNotSupported;
  p.w_tiles = (q.n + S::W_TILE - 1) / S::W_TILE;
  const uint64_t tiles = most_tiles<S>(q.m, q.n, q.groups);
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = allow_shared<S>(dev);
  if (e != cudaSuccess) return e;
  p.splits = 1;
  if (!S::TOKENS_X) {
    const uint32_t pairs = (p.steps + 1) / 2;              // the steps are cut in twos
    // as many as fill the SMs, as long as all clusters fit the device at once (16 of eight do not, on a B200)
    while (p.splits < 8 && p.splits * 2 <= pairs && tiles * p.splits * 2 <= (uint64_t)l.sm_count) p.splits *= 2;
    while (p.splits > 1 && tiles > resident_clusters<S>(dev, p.splits)) p.splits /= 2;
  }
  const uint32_t width = S::PAIR ? 2 : p.splits;           // CTAs of a cluster
  const uint64_t most = p.splits > 1 ? tiles : (uint64_t)l.sm_count / width;
  const uint32_t grid = (uint32_t)(tiles < most ? tiles : most) * width;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(kProductThreads); cfg.dynamicSmemBytes = S::SMEM; cfg.stream = l.stream;
  cudaLaunchAttribute attr[2];
  uint32_t na = 0;
  if (l.pdl) { attr[na].id = cudaLaunchAttributeProgrammaticStreamSerialization; attr[na++].val.programmaticStreamSerializationAllowed = 1; }
  if (width > 1) {
    attr[na].id = cudaLaunchAttributeClusterDimension;
    attr[na].val.clusterDim.x = width; attr[na].val.clusterDim.y = 1; attr[na++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr; cfg.numAttrs = na;
  e = cudaLaunchKernelEx(&cfg, mx_matmul_kernel<S>, mx, my, mo, p);
  if (e == cudaSuccess) ++*launches;
  return e;
}

using ManyRows = Shape<256, true, 5>;
using Few16 = Shape<16, false, 9>;
using Few32 = Shape<32, false, 8>;
using Few64 = Shape<64, false, 7>;
using Few128 = Shape<128, false, 5>;

}  // namespace

// Rows of a tile of the form that a product takes (256: the many-row form), and the most tiles that it may walk.
uint32_t mx_product_form(uint32_t m, uint32_t n, uint32_t groups, uint32_t sm_count, uint64_t* tiles) {
  // Rows that meet one weight, on average.  Up to 64 of them are one tile beside the weights (the next wider tile
  // costs up to a fifth more: 16 rows x 4096 x 4096 6.7 us at 16, 7.1 at 64 and 7.9 at 128).  More rows take the
  // narrowest tile whose count does not exceed the SMs: at 4096 x 4096, 128 rows 8.9 us at 64 and 13.1 at 16 wide,
  // 256 rows 10.0 at 64, 13.4 at 32 and 12.5 in the many-row form.  Where 128 wide is too many tiles the many-row form
  // is faster: 768 rows 13.9 us against 16.3, 2048 rows 20.6 against 27.1.  (All of them bursts with the weights in L2.
  // Other shapes were not measured against the rule, and of groups it knows only the average.)
  const uint32_t per_weight = (m + groups - 1) / groups;
  const uint64_t t16 = most_tiles<Few16>(m, n, groups), t32 = most_tiles<Few32>(m, n, groups), t64 = most_tiles<Few64>(m, n, groups),
                 t128 = most_tiles<Few128>(m, n, groups);
  uint32_t form = 256;
  uint64_t t = most_tiles<ManyRows>(m, n, groups);
  if (per_weight <= 16) { form = 16; t = t16; }
  else if (per_weight <= 32 || (per_weight > 64 && t32 <= sm_count)) { form = 32; t = t32; }
  else if (per_weight <= 64 || t64 <= sm_count) { form = 64; t = t64; }
  else if (t128 <= sm_count) { form = 128; t = t128; }
  if (tiles) *tiles = t;
  return form;
}

cudaError_t launch_mx_matmul(const Launch& l, const MxProduct& q, uint64_t* launches) {
  ProductArgs p = {};
  p.bias = q.bias; p.offsets = q.offsets; p.out = q.y; p.out_ld = q.y_ld; p.dtype = q.dtype;
  p.m = q.m; p.n = q.n; p.blocks = (q.k + 31) / 32; p.steps = (q.k + kStepCols - 1) / kStepCols; p.groups = q.groups;
  p.early = q.early; p.fault = q.fault;
  if (p.steps == 0) {
    const uint64_t want = ((uint64_t)q.m * q.n + 255) / 256;
    cudaError_t e = launch_kernel(l, mx_bias_kernel, (uint32_t)(want < 4096 ? want : 4096), 256, p);
    if (e == cudaSuccess) ++*launches;
    return e;
  }
  switch (mx_product_form(q.m, q.n, q.groups, (uint32_t)l.sm_count, nullptr)) {
    case 16: return launch_shape<Few16>(l, q, p, launches);
    case 32: return launch_shape<Few32>(l, q, p, launches);
    case 64: return launch_shape<Few64>(l, q, p, launches);
    case 128: return launch_shape<Few128>(l, q, p, launches);
    default: return launch_shape<ManyRows>(l, q, p, launches);
  }
}

}  // namespace qv2
