// Attention of new tokens over the quantized paged cache, many query rows to a key head: prompts and chunks of them, 16-bit queries.
//
// A CTA takes 256 query rows (two tiles of 128; one tile where a head has more than 128 elements) against tiles of 64 tokens:
//   warps 0-3, 4-7   the softmax of one query tile each, a thread to a row: scores from tensor memory, weights back into it in
//                    binary16, where the second product reads them; results out at the end,
//   warps 8-11       turn codes of keys and values into operands in shared memory, once for both query tiles,
//   warps 12, 13     look up the tokens of a tile ahead: where their rows lie, what their scales come to,
//   warp 14          issues the products (tcgen05.mma): scores S = Q K^T two tiles ahead, results O += P V.
// While one query tile's softmax runs the tensor cores are at the other's products.
//
// What bounds it: instructions and their latencies, not a unit.  Per 64 tokens and 256 rows of 128 elements the products are 512 cycles at the
// full rate and the exponentials 1024 (16 a cycle); a tile takes some 3000, the tensor cores are active 25 % of the time, special functions 25 %, and leaving out all exponentials
// was worth 3 %.  A prompt of 8192 tokens, 32 heads over 8, takes 740 us (744 TFLOP/s of what is seen).  Steps that told: two bodies of the softmax,
// one of them without masks, so that it need not jump over what it does not use; half the code of the converting warps (785 -> 740 us: a quarter of what
// a warp waits for is the next instruction); 64 tokens to a tile, since 128 scores of a row do not fit in registers (840 us with 128).
// 8 bits cost more: a multiplication for each score and each weight that the 4-bit form has in its operands (4 chunks of 512 over 4096 tokens
// each, 16 heads over 4: 154 us without a cap, 210 with one, whose exponential and reciprocal come on top).
//
// Codes are exact in binary16.  At 4 bits they are multiplied by their block's scale over the largest of the tile (keys) or of the item so far
// (values), a power of two: exact unless a scale is 2^36 below that.  8-bit integers enter as they are, and what is left is one number per
// token: keys' multiply their column of scores, values' their weights, held against the largest so far.  When that grows,
// results are brought along.  The reference of a row's softmax follows its maximum only when the largest weight has grown
// 2^kSlack-fold, so results are seldom rescaled.  A poisoned key is a NaN among the operands; a poisoned value must not be (it would
// reach the rows that do not see it, too): it is left out there and enters through the weights of those that do.
#include "qv2_attend.cuh"
#include "qv2_tensor.cuh"

namespace qv2 {

namespace {

constexpr uint32_t kConvert = 4, kScout = 2;                         // converting and looking-up warps
constexpr uint32_t kFirstScout = 8 + kConvert, kProducts = kFirstScout + kScout, kChunkThreads = (kProducts + 1) * 32;
constexpr uint32_t kSetup = 8;              // what an item costs besides its tiles, in tiles
constexpr int kChunkFactor = 13;            // 4 bits: operands stand 2^13 above code * scale / (largest scale): 6 * 2^13 at most
constexpr float kSlack = 4.f;               // a row's largest weight is 2^kSlack at most ...
constexpr int kWeightBits = 10;             // ... and weights stand 2^10 above that: at most 2^15 (8 bits: times up to 2), and what binary16 loses below 2^-35

__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void tensor_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D[128][N] (+)= A B: A from shared memory or from tensor memory (binary16, two to a column).
__device__ __forceinline__ void tensor_product(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void tensor_product_from(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
// 32 columns of this warp's lanes; the numbers are there when it returns.
__device__ __forceinline__ void tensor_read(uint32_t at, float (&v)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
               "tcgen05.wait::ld.sync.aligned;"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                 "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]),
                 "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]),
                 "=f"(v[30]), "=f"(v[31])
               : "r"(at) : "memory");
}
// The same, but they are there only after tc_load_wait().
__device__ __forceinline__ void tensor_read_begin(uint32_t at, float* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                 "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]),
                 "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]),
                 "=f"(v[30]), "=f"(v[31])
               : "r"(at) : "memory");
}
__device__ __forceinline__ void tensor_read16(uint32_t at, float (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
               "tcgen05.wait::ld.sync.aligned;"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                 "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
               : "r"(at) : "memory");
}
__device__ __forceinline__ void tensor_write16(uint32_t at, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
                 "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(at) : "memory");
}
__device__ __forceinline__ void tensor_write_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float4 shared_quad(uint32_t at) {           // (volatile: as plain loads all of a tile's are brought forward, at the price of 72 spilled registers)
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float reciprocal_fast(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
// Whether all threads of the looking-up warps say yes.
__device__ __forceinline__ bool all_scouts(bool ok) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)ok), "n"(32 * kScout) : "memory");
  return r != 0;
}

// Operands lie in panels of 64 columns, rows of 128 bytes in the 128-byte swizzle, 1024 bytes from one group of 8 rows to the next.
// Along the rows (queries and keys: the sum runs along the columns) ...
__device__ __forceinline__ uint64_t rows_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// ... and across them (values: the sum runs along the rows), `panel` bytes from one panel to the next.
__device__ __forceinline__ uint64_t columns_desc(uint32_t addr, uint32_t panel) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(panel >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

template <int FORMAT_, int DP_, bool PLAIN_>
struct Chunk {
  static constexpr int FORMAT = FORMAT_, DP = DP_;
  static constexpr bool PLAIN = PLAIN_;                               // no cap, no slopes
  static constexpr bool MX = FORMAT == QV2_KV_MX4;
  static constexpr uint32_t QT = DP == 256 ? 1 : 2;                   // query tiles
  static constexpr uint32_t ROWS = 128 * QT;
  static constexpr uint32_t KT = 64;                                  // tokens of a tile
  static constexpr uint32_t NB = DP / 32, RB = MX ? DP / 2 : DP;      // blocks of a row, bytes of its codes
  static constexpr uint32_t Q_PANEL = 128 * 128, Q_TILE = Q_PANEL * (DP / 64);
  static constexpr uint32_t PANEL = KT * 128, KV_TILE = PANEL * (DP / 64);
  static constexpr uint32_t STAGES = DP == 256 ? 2 : 4;
  // What is known of a tile's tokens: where each row lies; 4 bits: factors of keys' and values' blocks [2][block][token], 8 bits: scales of keys, of
  // values [2][token]; then which tokens there are, whose value is poisoned (4 words each), the largest exponents and flags.
  static constexpr uint32_t INFO = 8;                                 // tiles ahead
  static_assert(INFO == 8 && STAGES <= 4, "barriers");
  static constexpr uint32_t FACTOR_LD = KT + 8;                       // (blocks of a token in different banks)
  static constexpr uint32_t AT_SCALES = 8 * KT, AT_BITS = AT_SCALES + (MX ? 2 * 2 * NB * FACTOR_LD : 2 * 4 * KT), META = AT_BITS + 48;
  static constexpr uint32_t SMEM = 1024 + QT * Q_TILE + STAGES * 2 * KV_TILE + INFO * META;
  static constexpr uint32_t O_COL = QT * 2 * KT;                      // tensor memory: scores, two tiles of tokens ahead, then the results
  static_assert(O_COL + QT * DP <= 512, "tensor memory");
  static constexpr uint32_t S_IDESC = (1u << 4) | ((KT / 8) << 17) | (8u << 24);                    // binary16 x binary16, binary32 sums
  static constexpr uint32_t O_IDESC = (1u << 4) | (1u << 16) | ((DP / 8) << 17) | (8u << 24);       // second operand across its rows
  static constexpr uint32_t TOK = KT / kConvert;                             // tokens of a converting warp
  static constexpr uint32_t PIECES = RB / 16, WIDE = PIECES < 4 ? PIECES : 4;   // 16-byte pieces of a row; how many of a row in one instruction
  static constexpr uint32_t HIGH = 32 / WIDE;                         // rows in one instruction
  static constexpr uint32_t LOADS = TOK * PIECES / 32;                // of a lane, for keys or values
  static constexpr uint32_t SCALE_WORDS = MX ? (NB + 6) / 4 : 1;
};

struct ChunkArgs {
  AttendArgs a;
  FastDiv page, group;
  uint32_t few;                             // sequences of as many rows or fewer are the other kernel's
  uint32_t vec_q, vec_codes, vec_out;       // 16-byte loads of queries and of codes, stores of eight results
  float* parts;
  AttendPiece* pieces;
  uint32_t* fault;
};

// One row tile of a sequence: the tokens that its rows see between them.
struct ChunkTile {
  uint32_t rows, row0, row1;                // of the sequence; of the tile
  int32_t pos0;                             // position of the sequence's first query
  uint32_t j0, j1, units;
};
template <class F>
__device__ __forceinline__ ChunkTile chunk_tile(const ChunkArgs& p, const AttendSeq& s, uint32_t tile) {
  ChunkTile t;
  t.rows = s.n * p.a.group;
  t.row0 = tile * F::ROWS;
  t.row1 = min(t.rows, t.row0 + F::ROWS);
  t.pos0 = s.len - (int32_t)s.n;
  const int32_t first = t.pos0 + (int32_t)p.group.div(t.row0), last = t.pos0 + (int32_t)p.group.div(t.row1 - 1);
  t.j0 = min(first >= p.a.window ? (uint32_t)(first - p.a.window + 1) : 0u, p.a.room);
  t.j1 = max(min((uint32_t)(max(last, -1) + 1), p.a.room), t.j0);
  t.units = max(1u, (t.j1 - t.j0 + F::KT - 1) / F::KT);
  return t;
}
template <class F>
__device__ __forceinline__ uint32_t chunk_tiles(const ChunkArgs& p, const AttendSeq& s) {
  const uint64_t rows = (uint64_t)s.n * p.a.group;
  return rows <= p.few ? 0 : (uint32_t)((rows + F::ROWS - 1) / F::ROWS);
}

// Where a CTA stands in the row of all items: sequence, row tile, key head, and its part of that item.  An item takes kSetup + units;
// what a CTA has of the setup alone is nothing.  Every warp keeps one of its own.
template <class F>
struct Walk {
  uint32_t seq, tile, tiles, kv;
  uint32_t x0, x1, unit, unit1;                  // the part in those terms, and its units unit .. unit1 - 1
  uint64_t left;                                 // of this CTA, from x0 on
  AttendSeq s;
  ChunkTile t;
  __device__ __forceinline__ void enter(const ChunkArgs& p) {
    t = chunk_tile<F>(p, s, tile);
    const uint32_t all = t.units + kSetup;
    x1 = (uint32_t)min((uint64_t)all, x0 + left);
    unit = max(x0, kSetup) - kSetup;
    unit1 = max(x1, kSetup) - kSetup;
  }
  __device__ __forceinline__ bool next(const ChunkArgs& p) {       // on to the next item of which this CTA has a unit
    do {
      left -= x1 - x0;
      if (left == 0) return false;
      x0 = 0;
      if (++kv == p.a.c.heads) {
        kv = 0;
        if (++tile == tiles) {
          tile = 0;
          do { s = attend_seq(p.a, ++seq); tiles = chunk_tiles<F>(p, s); } while (tiles == 0);
        }
      }
      enter(p);
    } while (unit == unit1);
    return true;
  }
};

template <class F>
__global__ void __launch_bounds__(kChunkThreads, 1) attend_chunk_kernel(const ChunkArgs p) {
  constexpr bool MX = F::MX;
  constexpr uint32_t DP = F::DP, KT = F::KT, QT = F::QT, NB = F::NB;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t scan[kChunkThreads / 32];
  __shared__ struct { uint64_t before; uint32_t seq; } found;
  __shared__ uint64_t bars[36];
  __shared__ int32_t highest[2][2][kScout];
  __shared__ uint32_t tmem_slot, failed_flag;
  const AttendArgs& a = p.a;
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  uint8_t* const base = raw + ((1024u - (smem_addr(raw) & 1023u)) & 1023u);
  const uint32_t q_at = smem_addr(base), k_at = q_at + QT * F::Q_TILE, v_at = k_at + F::STAGES * F::KV_TILE;
  uint8_t* const meta = base + QT * F::Q_TILE + 2 * F::STAGES * F::KV_TILE;
  const uint32_t bar0 = smem_addr(bars);
  // Of tile n (counted over all items): operands are there (k_full, v_full, by stage), its tokens are known (m_full); the products for the scores of both
  // query tiles, for the results, are done (s_done, o_done: eight in turn, so that whoever waits is never two rounds late); the weights are there (p_full, two
  // in turn).
  auto k_full = [&](uint32_t s) { return bar0 + 8 * s; };
  auto v_full = [&](uint32_t s) { return bar0 + 8 * (4 + s); };
  auto m_full = [&](uint32_t n) { return bar0 + 8 * (8 + n % 8); };
  auto s_done = [&](uint32_t n) { return bar0 + 8 * (16 + n % 8); };
  auto o_done = [&](uint32_t n) { return bar0 + 8 * (24 + n % 8); };
  auto p_full = [&](uint32_t n) { return bar0 + 8 * (32 + n % 2); };
  const uint32_t q_full = bar0 + 8 * 34, drained = bar0 + 8 * 35;
  volatile uint32_t* const failed = &failed_flag;
  dependency_wait();
  allow_dependents();

  if (tid == 0) {
    for (uint32_t s = 0; s < 4; ++s) { bar_init(k_full(s), kConvert); bar_init(v_full(s), kConvert); }
    for (uint32_t s = 0; s < 8; ++s) { bar_init(m_full(s), kScout); bar_init(s_done(s), 1); bar_init(o_done(s), 1); }
    bar_init(p_full(0), 4 * QT); bar_init(p_full(1), 4 * QT); bar_init(q_full, 4 * QT);
    bar_init(drained, 1);
    *failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }

  // ---- this CTA's units
  auto units_in = [&](uint32_t s) -> uint64_t {
    if (s >= a.seqs) return 0;
    const AttendSeq q = attend_seq(a, s);
    const uint32_t tiles = chunk_tiles<F>(p, q);
    uint64_t sum = 0;
    for (uint32_t t = 0; t < tiles; ++t) sum += chunk_tile<F>(p, q, t).units + kSetup;
    return sum * a.c.heads;
  };
  uint64_t all = 0;
  for (uint32_t b = 0; b < a.seqs; b += kChunkThreads) all += units_in(b + tid);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  if (lane == 0) scan[warp] = all;
  __syncthreads();
  all = 0;
#pragma unroll
  for (uint32_t w = 0; w < kChunkThreads / 32; ++w) all += scan[w];
  const uint32_t ctas = (uint32_t)min((uint64_t)gridDim.x, all);
  if (tid == 0) p.pieces[blockIdx.x].followers = 0;
  if (blockIdx.x >= ctas) return;
  const uint64_t u_begin = all * blockIdx.x / ctas, u_end = all * (blockIdx.x + 1) / ctas;
  for (uint64_t b = 0, before = 0; b < a.seqs; b += kChunkThreads) {
    __syncthreads();
    const uint64_t mine = units_in((uint32_t)b + tid);
    uint64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint64_t v = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += v; }
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    uint64_t whole = 0;
#pragma unroll
    for (uint32_t w = 0; w < kChunkThreads / 32; ++w) { if (w < warp) sum += scan[w]; whole += scan[w]; }
    const uint64_t first = before + sum - mine;
    if (mine && u_begin >= first && u_begin < first + mine) { found.before = first; found.seq = (uint32_t)b + tid; }
    before += whole;
    if (u_begin < before) break;
  }
  if (warp == kProducts) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;

  Walk<F> at;
  at.seq = found.seq; at.tile = 0; at.left = u_end - u_begin;
  at.s = attend_seq(a, at.seq);
  at.tiles = chunk_tiles<F>(p, at.s);
  uint64_t in_seq = u_begin - found.before;
  for (;; ++at.tile) {
    const uint64_t n = (uint64_t)(chunk_tile<F>(p, at.s, at.tile).units + kSetup) * a.c.heads;
    if (in_seq < n) break;
    in_seq -= n;
  }
  {
    const uint32_t n = chunk_tile<F>(p, at.s, at.tile).units + kSetup;
    at.kv = (uint32_t)(in_seq / n);
    at.x0 = (uint32_t)(in_seq % n);
    at.enter(p);
  }
  const bool any = at.unit < at.unit1 || at.next(p);         // (a CTA that has nothing but the beginning of a setup has no unit)

  if (!any) {
  } else if (warp < 8) {
    // ---------------------------------------------------------------------------------- softmax
    const uint32_t t = warp / 4, lanes = ((warp % 4) * 32) << 16, r_in = 128 * t + (warp % 4) * 32 + lane;
    const uint32_t s_tile = tmem + t * 2 * KT + lanes, o_at = tmem + F::O_COL + t * DP + lanes;
    uint32_t n = 0;                                          // tiles so far
    // What a thread knows about its row of an item.
    struct Row {
      int32_t pos, pos_first, pos_last;                      // of the row, and of the first and last one of the warp
      uint32_t out_row, head;                                // row of the results, query head
      float back, slope;                                     // what the scores are multiplied by (to powers of two unless they are capped)
      bool there, part;                                      // the row exists; the tile takes part in the item
    } row = {}, ahead = {};
    Walk<F> to = at;
    bool more = true, ok = t < QT;
    float ref = -INFINITY, sum = 0.f;
    int v_top = -126;
#pragma unroll 1
    for (bool begin = true; ok; begin = false) {
      if (!begin) { to = at; more = to.next(p); }
      ahead.part = more && (t == 0 || to.t.row1 - to.t.row0 > 128);
      if (ahead.part) {
        // the next item's row, brought to the top of binary16's range by a power of two, signed like the scale.  (The products with the
        // last item's rows are done: their scores have been read.)
        const uint32_t r = to.t.row0 + r_in, rc = min(r, to.t.row1 - 1), i = p.group.div(rc), in_group = rc - i * p.group.d;
        ahead.head = to.kv * p.group.d + in_group;
        ahead.there = r < to.t.row1;
        ahead.out_row = to.s.row0 + i;
        ahead.pos = to.t.pos0 + (int32_t)i;
        ahead.pos_first = __shfl_sync(0xffffffffu, ahead.pos, 0);
        ahead.pos_last = __shfl_sync(0xffffffffu, ahead.pos, 31);
        // A row by DP / 8 lanes, ROUND rows in one round of loads; rows that are not there take another's elements, times zero.
        const uint64_t from = (uint64_t)ahead.out_row * a.q_token_ld + (uint64_t)ahead.head * a.q_head_ld;
        uint32_t top = 0;                                    // bits of the largest magnitude of this lane's row
        auto bring = [&](auto zero, const auto* q) {
          constexpr uint32_t LPR = DP / 8, ROUND = 32 / LPR, HELD = 8;       // lanes of a row, rows and rounds in flight
          const uint32_t c8 = 8 * (lane % LPR), in = lane / LPR;
#pragma unroll 1
          for (uint32_t r0 = 0; r0 < 32; r0 += HELD * ROUND) {
            decltype(zero) c[HELD];
            if (p.vec_q) {
#pragma unroll
              for (uint32_t k = 0; k < HELD; ++k) c[k].load_vec(q + __shfl_sync(0xffffffffu, from, r0 + k * ROUND + in) + min(c8, a.c.dim - 8));
            } else {
#pragma unroll
              for (uint32_t k = 0; k < HELD; ++k) {
                const uint64_t row_at = __shfl_sync(0xffffffffu, from, r0 + k * ROUND + in);
                c[k].zero();
                if (c8 + 8 <= a.c.dim) c[k].load_any(q + row_at + c8);
                else if (c8 < a.c.dim) c[k].load_some(q + row_at + c8, a.c.dim - c8);
              }
            }
#pragma unroll
            for (uint32_t k = 0; k < HELD; ++k) {
              uint32_t high = c[k].top_bits();
#pragma unroll
              for (uint32_t o = LPR / 2; o > 0; o >>= 1) high = max(high, __shfl_xor_sync(0xffffffffu, high, o));
              const uint32_t r = r0 + k * ROUND + in;                        // this lane's row of the round, of the warp's 32
              const uint32_t mine = __shfl_sync(0xffffffffu, high, (lane % ROUND) * LPR);
              if (lane / ROUND == r0 / ROUND + k) top = mine;
              const bool there = __shfl_sync(0xffffffffu, (uint32_t)ahead.there, r) != 0;
              const int e = high ? max((int)(high >> 23) - 127, -100) : 0;
              // (a row that holds a NaN or an infinity becomes NaN throughout: then all of its scores are, and no factor needs to be)
              const float up = !there || c8 >= a.c.dim ? 0.f : high >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : copysignf(power_of_two(14 - min(e, 127)), a.scale);
              float v[8];
              c[k].widen(v);
              uint32_t h[4];
#pragma unroll
              for (int i2 = 0; i2 < 4; ++i2) h[i2] = pack_half(v[2 * i2] * up, v[2 * i2 + 1] * up);
              const uint32_t row_in = (warp % 4) * 32 + r, where = q_at + t * F::Q_TILE + (c8 / 64) * F::Q_PANEL + row_in * 128 + (((c8 / 8) ^ row_in) & 7) * 16;
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(where), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
            }
          }
        };
        if (a.dtype == kBF16) bring(Chunk8<__nv_bfloat16>(), (const __nv_bfloat16*)a.q);
        else bring(Chunk8<__half>(), (const __half*)a.q);
        const int e = top ? max((int)(top >> 23) - 127, -100) : 0;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        ahead.back = power_of_two(min(e, 127) - 14) * power_of_two(MX ? -kChunkFactor : 0) * fabsf(a.scale) * (!F::PLAIN && a.cap > 0.f ? 1.f : kLog2e);
        ahead.slope = !F::PLAIN && a.slopes ? kLog2e * __ldg(a.slopes + ahead.head) : 0.f;
      }
      __syncwarp();
      if (more && lane == 0) bar_arrive(q_full);
      if (!begin && row.part) {
        // ---- results of the item that is done
        if (!bar_wait(o_done(n - 1), (n - 1) / 8 & 1, failed)) break;
        tc_fence_after();
        const bool whole = at.unit == 0 && at.unit1 == at.t.units;
        const uint32_t place = at.unit == 0 ? 1 : 0;
        float* const part = p.parts + ((uint64_t)blockIdx.x * 2 + place) * F::ROWS * (DP + 2);
        sum *= power_of_two(-kWeightBits);
        const float f0 = power_of_two(-kWeightBits - (MX ? kChunkFactor : 0)) * (!whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum), f1 = power_of_two(v_top);
        const uint64_t out_at = (uint64_t)row.out_row * a.q_heads + row.head;
        if (!whole && row.there) *reinterpret_cast<float2*>(part + F::ROWS * DP + 2 * r_in) = make_float2(ref, sum);
        if (whole && row.there && a.lse) a.lse[out_at] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * kLn2;
#pragma unroll 1
        for (uint32_t c = 0; c < DP / 32; ++c) {
          float o[32];
          tensor_read(o_at + 32 * c, o);
          if (!row.there) continue;
#pragma unroll
          for (uint32_t k = 0; k < 32; ++k) o[k] = o[k] * f0 * f1;
          if (!whole) {
#pragma unroll
            for (uint32_t k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(part + r_in * DP + 32 * c + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
          } else {
            auto store = [&](auto* out) {
              using T = typename std::remove_pointer<decltype(out)>::type;
#pragma unroll
              for (uint32_t k = 0; k < 32; k += 8) {
                const float v[8] = {o[k], o[k + 1], o[k + 2], o[k + 3], o[k + 4], o[k + 5], o[k + 6], o[k + 7]};
                const uint32_t d = 32 * c + k;
                T* const where = out + out_at * a.c.dim + d;
                if (p.vec_out) { if (d < a.c.dim) Chunk8<T>::store_vec(where, v); }
                else if (d < a.c.dim) store_some(where, v, a.c.dim - d);
              }
            };
            if (a.dtype == kBF16) store((__nv_bfloat16*)a.out);
            else store((__half*)a.out);
          }
        }
        if (!whole && place == 1 && tid == 0) {
          const uint64_t last = u_end - at.left - at.x0 + at.t.units + kSetup - 1;
          uint32_t c = (uint32_t)(last * ctas / all);
          while (all * c / ctas > last) --c;
          while (all * (c + 1) / ctas <= last) ++c;
          AttendPiece h;
          h.followers = c - blockIdx.x; h.row0 = at.s.row0; h.rows = at.t.rows; h.tile = at.tile; h.heads = at.kv;
          p.pieces[blockIdx.x] = h;
        }
        tc_fence_before();
        __syncwarp();
      }
      if (!more) break;
      at = to;
      row = ahead;
      const uint32_t n_units = at.unit1 - at.unit;
      ref = -INFINITY; sum = 0.f; v_top = -126;
#pragma unroll 1
      for (uint32_t u = 0; u < n_units; ++u, ++n) {
        const uint8_t* const m = meta + n % F::INFO * F::META;
        const uint32_t k_scale = smem_addr(m + F::AT_SCALES), v_scale = k_scale + 4 * KT;
        const uint32_t* const real = reinterpret_cast<const uint32_t*>(m + F::AT_BITS);
        const uint32_t* const bad = real + 4;
        const uint32_t j = at.t.j0 + (at.unit + u) * KT, s_at = s_tile + (n & 1) * KT;
        if (!bar_wait(m_full(n), n / 8 & 1, failed)) { ok = false; break; }
        const int4 tops = *reinterpret_cast<const int4*>(m + F::AT_BITS + 32);       // exponents of the tile's keys (4 bits), of the values so far; flags
        const bool every = (tops.z & 1) && (int32_t)(j + KT - 1) <= row.pos_first && row.pos_last - (int32_t)j < a.window, poisoned = MX && (tops.z & 2);
        // what turns a score of the product into one to powers of two; not 0, since it multiplies minus infinity, too
        const float unit = MX ? row.back * power_of_two(tops.x) : row.back, mul = !F::PLAIN ? 1.f : unit < 1.2e-38f ? 1.2e-38f : unit;
        if (!bar_wait(s_done(n), n / 8 & 1, failed)) { ok = false; break; }
        // EVERY: all tokens are seen by all rows of the warp, and none is poisoned.  (Two bodies instead of branches in one: jumping over the unused code cost
        // more than the softmax itself.)
        auto weights = [&](auto every_) -> bool {
          constexpr bool EVERY = decltype(every_)::value;
          tc_fence_after();
          float x[KT];
          tensor_read_begin(s_at, x);
          tensor_read_begin(s_at + 32, x + 32);
          tc_load_wait();
          if (!MX) {
#pragma unroll
            for (uint32_t k = 0; k < KT / 4; ++k) {
              const float4 f = shared_quad(k_scale + 16 * k);
              mul2(x[4 * k], x[4 * k + 1], f.x, f.y);
              mul2(x[4 * k + 2], x[4 * k + 3], f.z, f.w);
            }
          }
          if (!F::PLAIN) {
            // the bias of the tile's first token; of the others, `slope` for each token more
            const float bias = row.slope * (float)(int32_t)(j - (uint32_t)row.pos);
            if (a.cap > 0.f) {                               // cap * tanh(y / cap) = cap - 2 cap / (1 + e^(2 y / cap)), off by some 2^-22 of cap
              const float cap_in = 2.f * kLog2e * unit / a.cap, cap_out = kLog2e * a.cap;
#pragma unroll
              for (uint32_t k = 0; k < KT; k += 2) {
                mul2(x[k], x[k + 1], cap_in, cap_in);
                x[k] = 1.f + exp2_fast(x[k]);
                x[k + 1] = 1.f + exp2_fast(x[k + 1]);
                x[k] = reciprocal_fast(x[k]);
                x[k + 1] = reciprocal_fast(x[k + 1]);
                fma2(x[k], x[k + 1], -2.f * cap_out, cap_out + bias);
              }
            } else {
#pragma unroll
              for (uint32_t k = 0; k < KT; k += 2) fma2(x[k], x[k + 1], unit, bias);
            }
            if (a.slopes)
#pragma unroll
              for (uint32_t k = 1; k < KT; ++k) x[k] = fmaf(row.slope, (float)k, x[k]);
          }
          uint32_t seen[2] = {~0u, ~0u};
          if constexpr (!EVERY) {
            // tokens that there are, up to the row's position, within its window
            const int32_t upto = row.pos - (int32_t)j, from = upto - a.window;      // first unseen one on either side, relative to the tile
#pragma unroll
            for (uint32_t c = 0; c < 2; ++c) {
              const int32_t hi = min(max(upto + 1 - (int32_t)(32 * c), 0), 32), lo = row.pos < a.window ? 0 : min(max(from + 1 - (int32_t)(32 * c), 0), 32);
              seen[c] = real[c] & (hi == 32 ? ~0u : (1u << hi) - 1u) & (lo == 32 ? 0u : ~0u << lo);
#pragma unroll
              for (uint32_t k = 0; k < 32; ++k)
                if (!(seen[c] >> k & 1u)) x[32 * c + k] = -INFINITY;
            }
          }
          float h4[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
          for (uint32_t k = 4; k < KT - 4; k += 8)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) h4[i] = max3(h4[i], x[k + i], x[k + 4 + i]);
#pragma unroll
          for (uint32_t i = 0; i < 4; ++i) h4[i] = fmaxf(h4[i], x[KT - 4 + i]);
          float high = fmaxf(max3(h4[0], h4[1], h4[2]), h4[3]);
          high = high == -INFINITY ? high : high * mul;      // (NaN scores are not seen here: their weights are NaN below)
          float soft = 1.f, values = 1.f;
          if (high > ref + kSlack) { soft = exp2_fast(ref - high); ref = high; }
          if (tops.y != v_top) { values = power_of_two(max(v_top - tops.y, -126)); v_top = tops.y; }
          sum *= soft;
          if (u > 0 && __any_sync(0xffffffffu, soft * values != 1.f)) {
            if (!bar_wait(o_done(n - 1), (n - 1) / 8 & 1, failed)) return false;
            tc_fence_after();
            const float f = soft * values;
#pragma unroll 1
            for (uint32_t c = 0; c < DP / 16; ++c) {
              float o[16];
              tensor_read16(o_at + 16 * c, o);
#pragma unroll
              for (uint32_t k = 0; k < 16; k += 2) mul2(o[k], o[k + 1], f, f);
              uint32_t bits[16];
#pragma unroll
              for (uint32_t k = 0; k < 16; ++k) bits[k] = __float_as_uint(o[k]);
              tensor_write16(o_at + 16 * c, bits);
            }
          }
          const float less = (float)kWeightBits - (ref == -INFINITY ? 0.f : ref);
          float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (uint32_t c = 0; c < 2; ++c) {
            float* const y = x + 32 * c;
#pragma unroll
            for (uint32_t k = 0; k < 32; k += 2) fma2(y[k], y[k + 1], mul, less);
#pragma unroll
            for (uint32_t k = 0; k < 32; ++k) y[k] = exp2_fast(y[k]);
#pragma unroll
            for (uint32_t k = 0; k < 32; k += 4) { add2(sums[0], sums[1], y[k], y[k + 1]); add2(sums[2], sums[3], y[k + 2], y[k + 3]); }
            if (!MX) {
#pragma unroll
              for (uint32_t k = 0; k < 8; ++k) {
                const float4 f = shared_quad(v_scale + 16 * (8 * c + k));
                mul2(y[4 * k], y[4 * k + 1], f.x, f.y);
                mul2(y[4 * k + 2], y[4 * k + 3], f.z, f.w);
              }
            } else if (!EVERY && poisoned) {
              const uint32_t nan = bad[c] & seen[c];
#pragma unroll
              for (uint32_t k = 0; k < 32; ++k)
                if (nan >> k & 1u) y[k] = __uint_as_float(0x7fc00000u);
            }
            uint32_t h[16];
#pragma unroll
            for (uint32_t k = 0; k < 16; ++k) {
              h[k] = pack_half(y[2 * k], y[2 * k + 1]);
              if (!MX && !EVERY) h[k] &= (0u - (seen[c] >> 2 * k & 1u) & 0xffffu) | (0u - (seen[c] >> (2 * k + 1) & 1u) & 0xffff0000u);      // not zero times a poisoned scale
            }
            tensor_write16(s_at + 16 * c, h);
          }
          sum += (sums[0] + sums[1]) + (sums[2] + sums[3]);
          tensor_write_wait();
          tc_fence_before();
          return true;
        };
        if (row.part) {
          if (every && !poisoned) ok = weights(std::true_type());
          else ok = weights(std::false_type());
          if (!ok) break;
        }
        __syncwarp();
        if (lane == 0) bar_arrive(p_full(n));                // (a query tile without rows says so, too)
      }
      if (!ok) break;
    }
  } else if (warp < kFirstScout) {
    // ---------------------------------------------------------------------------------- codes into operands
    constexpr uint32_t TOK = F::TOK, LOADS = F::LOADS, HIGH = F::HIGH;
    const uint32_t first = (warp - 8) * TOK;                                 // this warp's tokens of a tile
    const uint32_t row_bytes = MX ? 16 * ((a.c.dim + 31) / 32) : a.c.dim;
    uint4 code[2][LOADS];                                                    // of keys and of values
    auto at_load = [&](uint32_t i, uint32_t* in, uint32_t* piece) {          // token of the tile, 16-byte piece of its row
      *in = first + (i % (TOK / HIGH)) * HIGH + lane % HIGH;
      *piece = (i / (TOK / HIGH)) * F::WIDE + lane / HIGH;
    };
    auto fetch = [&](uint4 (&code)[LOADS], int w, uint32_t n) {
      const uint8_t* const m = meta + n % F::INFO * F::META;
#pragma unroll
      for (uint32_t i = 0; i < LOADS; ++i) {
        uint32_t in, piece;
        at_load(i, &in, &piece);
        const int64_t row = reinterpret_cast<const int64_t*>(m)[in];
        code[i] = make_uint4(0, 0, 0, 0);
        if (row >= 0 && 16 * piece < row_bytes && (MX || p.vec_codes)) code[i] = __ldg(reinterpret_cast<const uint4*>(a.c.codes[w] + row + 16 * piece));
      }
      if constexpr (!MX) {
        if (p.vec_codes) return;
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {                               // rows on any address
          uint32_t in, piece, v[4] = {0, 0, 0, 0};
          at_load(i, &in, &piece);
          const int64_t row = reinterpret_cast<const int64_t*>(m)[in];
#pragma unroll 1
          for (uint32_t b = 0; b < 16 && row >= 0 && 16 * piece + b < row_bytes; ++b) {
            const uint32_t byte = (uint32_t)__ldg(a.c.codes[w] + row + 16 * piece + b) << (8 * (b % 4));
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) if (b / 4 == k) v[k] |= byte;
          }
          code[i] = make_uint4(v[0], v[1], v[2], v[3]);
        }
      }
    };
    bool ok = bar_wait(m_full(0), 0, failed);
    auto last = [&](uint32_t n) { return (*reinterpret_cast<const int32_t*>(meta + n % F::INFO * F::META + F::AT_BITS + 40) & 4) != 0; };
    if (ok) {
      fetch(code[0], 0, 0); fetch(code[1], 1, 0);
    }
    // One tile; its registers take the codes of the next as soon as they are free.  false: that was the last, or a wait gave up.
    auto convert = [&](uint32_t n) -> bool {
      const uint32_t s = n % F::STAGES, before = n - F::STAGES;              // the tile that had this stage
      const uint8_t* const m = meta + n % F::INFO * F::META;
      const bool more = !last(n);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if (n >= F::STAGES && !bar_wait(w ? o_done(before) : s_done(before), before / 8 & 1, failed)) return false;
        const uint32_t tile = (w ? v_at : k_at) + s * F::KV_TILE;
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
          uint32_t in, piece;
          at_load(i, &in, &piece);
          // 16 bytes of operands after 16: where they lie differs from the first in bits that the swizzle turns over
          const uint32_t d = (MX ? 32 : 16) * piece, to = tile + in * 128 + (d / 64) * F::PANEL + (((d / 8) ^ in) & 7) * 16;
          auto put = [&](uint32_t k, uint32_t x, uint32_t y, uint32_t z, uint32_t t) {
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to ^ 16 * k), "r"(x), "r"(y), "r"(z), "r"(t) : "memory");
          };
          const uint32_t word[4] = {code[w][i].x, code[w][i].y, code[w][i].z, code[w][i].w};
          if (MX) {
            const uint32_t h = reinterpret_cast<const uint16_t*>(m + F::AT_SCALES)[(w * NB + piece) * F::FACTOR_LD + in], factor = h | h << 16;
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) {
              uint32_t c[4];
              four_bits(word[k], c);
              put(k, half_mul(c[0], factor), half_mul(c[1], factor), half_mul(c[2], factor), half_mul(c[3], factor));
            }
          } else {
#pragma unroll
            for (uint32_t k = 0; k < 4; k += 2) {
              const uint32_t x = word[k] ^ 0x80808080u, y = word[k + 1] ^ 0x80808080u;
              put(k / 2, eight_bits<0x4140>(x), eight_bits<0x4342>(x), eight_bits<0x4140>(y), eight_bits<0x4342>(y));
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive(w ? v_full(s) : k_full(s));
        if (more) {
          if (w == 0 && !bar_wait(m_full(n + 1), (n + 1) / 8 & 1, failed)) return false;
          fetch(code[w], w, n + 1);
        }
      }
      return more;
    };
    if (ok)
#pragma unroll 1
      for (uint32_t n = 0; convert(n); ++n) {}
  } else if (warp < kProducts) {
    // ---------------------------------------------------------------------------------- tokens
    constexpr uint32_t PER = KT / (32 * kScout), WORDS = F::SCALE_WORDS, PACKS = MX ? (NB + 3) / 4 : 1;
    const uint32_t part = warp - kFirstScout, first = part * 32 * PER + lane;     // this lane's tokens of a tile: first, first + 32
    const uint32_t blocks = (a.c.dim + 31) / 32, row_bytes = MX ? 16 * blocks : a.c.dim;
    struct Token {
      int32_t id, id_next;                                                   // its page in this tile and in the next; negative: no such token
      uint32_t scale_word[2][WORDS], lead;                                   // its scales, where they begin in their first word (keys, values)
      uint64_t row;                                                          // in the cache
    } tok[PER];
    auto page_of = [&](uint32_t u, uint32_t q) -> int32_t {
      const uint64_t j = (uint64_t)at.t.j0 + (uint64_t)u * KT + first + 32 * q;
      if (u >= at.unit1 || j >= at.t.j1) return -1;
      const int32_t id = __ldg(a.table + at.seq * a.table_ld + p.page.div((uint32_t)j));
      return id >= 0 && (uint32_t)id < a.c.pages ? id : -1;
    };
    auto fetch_scales = [&](uint32_t u, uint32_t q) {
      Token& k = tok[q];
      const uint32_t j = at.t.j0 + u * KT + first + 32 * q, off = j - p.page.div(j) * p.page.d;
      k.row = k.id < 0 ? 0 : ((uint64_t)(uint32_t)k.id * p.page.d + off) * a.c.heads + at.kv;
      k.lead = 0;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
#pragma unroll
        for (uint32_t i = 0; i < WORDS; ++i) k.scale_word[w][i] = 0;
        if (k.id < 0) continue;
        if (MX) {                                                            // whole words, each of which holds a wanted byte
          const uintptr_t from = (uintptr_t)a.c.scales[w] + k.row * blocks;
          const uint32_t l = (uint32_t)(from & 3u);
          k.lead |= l << (4 * w);
#pragma unroll
          for (uint32_t i = 0; i < WORDS; ++i)
            if (4 * i < l + blocks) k.scale_word[w][i] = __ldg(reinterpret_cast<const uint32_t*>(from & ~(uintptr_t)3u) + i);
        } else k.scale_word[w][0] = __ldg(reinterpret_cast<const uint32_t*>(a.c.scales[w]) + k.row);
      }
    };
    uint32_t u = at.unit;
    auto begin_item = [&] {
#pragma unroll
      for (uint32_t q = 0; q < PER; ++q) { tok[q].id = page_of(u, q); tok[q].id_next = page_of(u + 1, q); }
    };
    begin_item();
#pragma unroll
    for (uint32_t q = 0; q < PER; ++q) fetch_scales(u, q);
    int v_top = -126;
    bool more = true;
#pragma unroll 1
    for (uint32_t n = 0; more; ++n) {
      const uint32_t s = n % F::INFO;
      float scale[PER][2];
      uint32_t bytes[PER][2][PACKS], high_byte[PER][2], real[PER], poisoned[PER];      // 4 bits: scales of the blocks, and the largest
      int64_t here[PER];
      int v_most = -126, flags = 0;
      uint32_t k_most = 0;
#pragma unroll
      for (uint32_t q = 0; q < PER; ++q) {
        const Token& k = tok[q];
        real[q] = __ballot_sync(0xffffffffu, k.id >= 0);
        here[q] = k.id >= 0 ? (int64_t)(k.row * row_bytes) : -1;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          high_byte[q][w] = 0;
          scale[q][w] = MX ? 0.f : __uint_as_float(k.scale_word[w][0]);
          if (!MX) continue;
          const uint32_t shift = 8 * (k.lead >> (4 * w) & 3u);
#pragma unroll
          for (uint32_t i = 0; i < PACKS; ++i) {
            bytes[q][w][i] = __funnelshift_r(k.scale_word[w][i], i + 1 < WORDS ? k.scale_word[w][i + 1 < WORDS ? i + 1 : 0] : 0u, shift);
            const uint32_t have = blocks - min(blocks, 4 * i);
            if (have < 4) bytes[q][w][i] &= (1u << (8 * have)) - 1u;
#pragma unroll
            for (uint32_t b = 0; b < 4; ++b) high_byte[q][w] = max(high_byte[q][w], bytes[q][w][i] >> (8 * b) & 255u);
          }
        }
        // the largest exponents: 4 bits, of the tile's keys, as bytes; of the values (8 bits: finite scales are positive)
        const uint32_t field = MX ? (high_byte[q][1] == 255u ? 0u : high_byte[q][1]) : (__float_as_uint(scale[q][1]) >> 23 & 255u);
        if (field != 255u) v_most = max(v_most, min((int)field - 127, MX ? 127 : 126));
        if (high_byte[q][0] != 255u) k_most = max(k_most, high_byte[q][0]);
        poisoned[q] = __ballot_sync(0xffffffffu, MX && high_byte[q][1] == 255u);
        flags |= (real[q] != 0xffffffffu) | (poisoned[q] != 0) << 1;         // some token is not there; some value is poisoned
      }
      v_most = __reduce_max_sync(0xffffffffu, v_most);
      k_most = MX ? __reduce_max_sync(0xffffffffu, k_most) : 0;
      if (lane == 0) { highest[n & 1][0][part] = (int)k_most | flags << 16; highest[n & 1][1][part] = v_most; }
      // on to the next tile: its scales are fetched meanwhile
      const bool new_item = ++u == at.unit1;
      if (new_item) {
        more = at.next(p);
        u = at.unit;
        if (more) begin_item();
      } else {
#pragma unroll
        for (uint32_t q = 0; q < PER; ++q) { tok[q].id = tok[q].id_next; tok[q].id_next = page_of(u + 1, q); }
      }
      if (more) {
#pragma unroll
        for (uint32_t q = 0; q < PER; ++q) fetch_scales(u, q);
      }
      if (!all_scouts(n < F::INFO || bar_wait(o_done(n - F::INFO), (n - F::INFO) / 8 & 1, failed))) break;
      int k_top = 1, any_flag = 0;
#pragma unroll
      for (uint32_t k = 0; k < kScout; ++k) {
        const int v = highest[n & 1][0][k];
        k_top = max(k_top, v & 0xffff); any_flag |= v >> 16;
        v_top = max(v_top, highest[n & 1][1][k]);
      }
      uint8_t* const m = meta + s * F::META;
#pragma unroll
      for (uint32_t q = 0; q < PER; ++q) {
        const uint32_t in = first + 32 * q;
        reinterpret_cast<int64_t*>(m)[in] = here[q];
        if (MX) {
          const bool nan_key = high_byte[q][0] == 255u, no_value = high_byte[q][1] == 255u;
#pragma unroll
          for (uint32_t b = 0; b < NB; ++b)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              // 2^(own - largest + kChunkFactor) in binary16, down to its smallest number 2^-24
              const int f = (int)(bytes[q][w][MX ? b / 4 : 0] >> (8 * (b % 4)) & 255u) - (w ? v_top + 127 : k_top) + kChunkFactor;
              uint32_t h = f < -24 ? 0u : f >= -14 ? (uint32_t)(min(f, kChunkFactor) + 15) << 10 : 1u << (f + 24);
              if (w == 0 && nan_key) h = 0x7e00u;
              if (w == 1 && no_value) h = 0;
              reinterpret_cast<uint16_t*>(m + F::AT_SCALES)[(w * NB + b) * F::FACTOR_LD + in] = (uint16_t)h;
            }
        } else {
          reinterpret_cast<float*>(m + F::AT_SCALES)[in] = scale[q][0];
          reinterpret_cast<float*>(m + F::AT_SCALES + 4 * KT)[in] = scale[q][1] * power_of_two(-v_top);
        }
        if (lane == 0) {
          reinterpret_cast<uint32_t*>(m + F::AT_BITS)[part * PER + q] = real[q];
          reinterpret_cast<uint32_t*>(m + F::AT_BITS + 16)[part * PER + q] = poisoned[q];
        }
      }
      if (part == 0 && lane == 0) *reinterpret_cast<int4*>(m + F::AT_BITS + 32) = make_int4(k_top - 127, v_top, (any_flag ^ 1) | (more ? 0 : 4), 0);
      __syncwarp();
      if (lane == 0) bar_arrive(m_full(s));
      if (new_item) v_top = -126;
    }
  } else {
    // ---------------------------------------------------------------------------------- products
    // Scores run two tiles of tokens ahead of the results, so that a softmax finds the next ones ready.  Descriptors are made once and moved by
    // constants (in units of 16 bytes): the one warp that issues is soon the slowest.
    uint32_t n = 0, items = 0;
    const uint64_t q_desc = rows_desc(q_at), k_desc = rows_desc(k_at), v_desc = columns_desc(v_at, F::PANEL);
    bool ok = true;
    do {
      const uint32_t n_units = at.unit1 - at.unit;
      const bool both = QT == 2 && at.t.row1 - at.t.row0 > 128;
      auto scores = [&](uint32_t m) {                                        // of tile m
        const uint32_t s = m % F::STAGES;
        ok = ok && bar_wait(k_full(s), m / F::STAGES & 1, failed);
        if (!ok) return;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t kd = k_desc + s * (F::KV_TILE >> 4);
          const uint32_t to = tmem + (m & 1) * KT;
#pragma unroll
          for (uint32_t t = 0; t < QT; ++t)
            if (t == 0 || both)
#pragma unroll
              for (uint32_t k = 0; k < DP / 16; ++k)
                tensor_product(to + 2 * t * KT, q_desc + ((t * F::Q_TILE + (k / 4) * F::Q_PANEL) >> 4) + 2 * (k % 4), kd + ((k / 4) * F::PANEL >> 4) + 2 * (k % 4),
                               F::S_IDESC, k > 0);
          tensor_commit(s_done(m));
        }
        __syncwarp();
      };
      ok = bar_wait(q_full, items++ & 1, failed);
      scores(n);
      if (n_units > 1) scores(n + 1);
#pragma unroll 1
      for (uint32_t u = 0; ok && u < n_units; ++u, ++n) {
        const uint32_t s = n % F::STAGES;
        ok = bar_wait(v_full(s), n / F::STAGES & 1, failed) && bar_wait(p_full(n), n / 2 & 1, failed);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t vd = v_desc + s * (F::KV_TILE >> 4);
          const uint32_t from = tmem + (n & 1) * KT, add = u > 0;
#pragma unroll
          for (uint32_t t = 0; t < QT; ++t)
            if (t == 0 || both)
#pragma unroll
              for (uint32_t k = 0; k < KT / 16; ++k)
                tensor_product_from(tmem + F::O_COL + t * DP, from + 2 * t * KT + 8 * k, vd + 128 * k, F::O_IDESC, k > 0 ? 1u : add);
          tensor_commit(o_done(n));
        }
        __syncwarp();
        if (u + 2 < n_units) scores(n + 2);
      }
    } while (ok && at.next(p));
    if (*failed) {                                                           // leave no product in flight
      if (elect_one()) tensor_commit(drained);
      __syncwarp();
      const uint64_t begin = now_ns();
      while (!bar_try(drained, 0) && now_ns() - begin < kWaitLimitNs) {}
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (tid == 0 && *failed) { *p.fault = 1; __threadfence_system(); }
  if (warp == kProducts) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

constexpr int kDevices = 64;

template <class F>
cudaError_t launch_chunk(const Launch& l, ChunkArgs p, const AttendRun& run, uint64_t* launches) {
  static bool allowed[kDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= kDevices || !allowed[dev]) {
    e = cudaFuncSetAttribute(attend_chunk_kernel<F>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::SMEM);
    if (e != cudaSuccess) return e;
    if (dev < kDevices) allowed[dev] = true;
  }
  static_assert(F::ROWS == chunk_rows(F::DP) && F::SMEM <= 232448 - 1024, "shared memory");
  p.parts = reinterpret_cast<float*>(run.scratch);
  p.pieces = reinterpret_cast<AttendPiece*>(run.scratch + attend_parts_bytes(run.chunk_ctas, 1, F::ROWS, F::DP));
  e = launch_grid(l, attend_chunk_kernel<F>, dim3(run.chunk_ctas), kChunkThreads, F::SMEM, p);
  if (e != cudaSuccess) return e;
  ++*launches;
  return launch_attend_join(l, p.a, p.parts, p.pieces, run.chunk_ctas, 0, F::ROWS, F::DP, launches);
}

template <int FORMAT, bool PLAIN>
cudaError_t launch_dim(const Launch& l, const ChunkArgs& p, const AttendRun& run, uint64_t* launches) {
  if (run.dp == 64) return launch_chunk<Chunk<FORMAT, 64, PLAIN>>(l, p, run, launches);
  if (run.dp == 128) return launch_chunk<Chunk<FORMAT, 128, PLAIN>>(l, p, run, launches);
  return launch_chunk<Chunk<FORMAT, 256, PLAIN>>(l, p, run, launches);
}

}  // namespace

cudaError_t launch_attend_chunk(const Launch& l, const AttendArgs& a, const AttendRun& run, uint64_t* launches) {
  ChunkArgs p;
  p.a = a; p.page = FastDiv(a.c.page_size); p.group = FastDiv(a.group); p.few = run.few;
  p.vec_codes = a.c.dim % 16 == 0 && ((uintptr_t)a.c.codes[0] | (uintptr_t)a.c.codes[1]) % 16 == 0;
  p.vec_q = a.c.dim % 8 == 0 && ((uintptr_t)a.q | a.q_token_ld * 2 | a.q_head_ld * 2) % 16 == 0;
  p.vec_out = a.c.dim % 8 == 0 && (uintptr_t)a.out % 16 == 0; p.fault = run.fault;
  if (!(a.cap > 0.f) && !a.slopes) return a.c.format == QV2_KV_MX4 ? launch_dim<QV2_KV_MX4, true>(l, p, run, launches) : launch_dim<QV2_KV_I8, true>(l, p, run, launches);
  return a.c.format == QV2_KV_MX4 ? launch_dim<QV2_KV_MX4, false>(l, p, run, launches) : launch_dim<QV2_KV_I8, false>(l, p, run, launches);
}

}  // namespace qv2
