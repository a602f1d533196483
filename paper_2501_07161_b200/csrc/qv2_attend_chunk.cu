// Attention of new tokens over the quantized paged cache, many query rows to a key head: prompts and chunks of them, 16-bit queries.
//
// A CTA takes 256 query rows (two tiles of 128; one tile where a head has more than 128 elements) against tiles of 128 (64) tokens:
//   warps 0-3, 4-7   the softmax of one tile each, a thread to a row: scores from tensor memory, weights back into it in
//                    binary16, where the second product reads them; results out at the end,
//   warps 8-11       turn codes and scales of keys and values into operands in shared memory, once for both tiles,
//   warp 12          issues the products (tcgen05.mma): scores S = Q K^T, results O += P V.
// While one tile's softmax runs the tensor cores are at the other tile's products.  Bound by the exponentials (16 a cycle and SM: 2048
// cycles for 2 x 128 x 128 scores) next to the products (2 x 2 x 512 cycles for 128 elements).
//
// Codes are exact in binary16: 8-bit integers as they are, 4-bit codes times a power of two that says how far their block's scale is below
// the row's largest.  What is left is one number per token: keys' multiply their column of scores, values' their weights, held
// against the largest so far (its exponent is the CTA's; results are brought along when it grows).  The
// reference of a row's softmax follows its maximum only when that has doubled its largest weight, so results are seldom rescaled.
#include "qv2_attend.cuh"
#include "qv2_tensor.cuh"

namespace qv2 {

namespace {

constexpr uint32_t kChunkThreads = 13 * 32;
constexpr int kChunkBits = 13;              // weights stand 2^13 above p * scale / (largest scale): at most 2^15, p being at most 2
constexpr int kChunkFactor = 13;            // 4 bits: numbers stand 2^13 above code * scale / (largest of the row): 6 * 2^13 at most
constexpr float kSlack = 1.f;               // the reference of a row's softmax follows its maximum when that is above it by more (a power of two)

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
__device__ __forceinline__ void tensor_write(uint32_t at, const float (&v)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
               ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
                 "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]),
                 "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]),
                 "f"(v[30]), "f"(v[31]), "r"(at) : "memory");
}
__device__ __forceinline__ void tensor_write16(uint32_t at, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
                 "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(at) : "memory");
}
__device__ __forceinline__ void tensor_write_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Whether all 128 threads of the four converting warps say yes.
__device__ __forceinline__ bool all_converting(bool ok) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)ok) : "memory");
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

template <int FORMAT_, int DP_>
struct Chunk {
  static constexpr int FORMAT = FORMAT_, DP = DP_;
  static constexpr bool MX = FORMAT == QV2_KV_MX4;
  static constexpr uint32_t QT = DP == 256 ? 1 : 2;                   // query tiles
  static constexpr uint32_t ROWS = 128 * QT;
  static constexpr uint32_t KT = DP == 256 ? 64 : 128;                // tokens of a tile
  static constexpr uint32_t NB = DP / 32, RB = MX ? DP / 2 : DP;      // blocks of a row, bytes of its codes
  static constexpr uint32_t Q_PANEL = 128 * 128, Q_TILE = Q_PANEL * (DP / 64);
  static constexpr uint32_t PANEL = KT * 128, KV_TILE = PANEL * (DP / 64);
  static constexpr uint32_t STAGES = 2;
  static constexpr uint32_t META = 2 * 4 * KT + 16 + 16;              // scales of keys, of values, which tokens there are, the exponent of the values' scales
  static constexpr uint32_t SMEM = 1024 + QT * Q_TILE + STAGES * (2 * KV_TILE + META) + 256;
  static constexpr uint32_t O_COL = QT * KT;                          // tensor memory: scores of the tiles, then their results
  static_assert(O_COL + QT * DP <= 512, "tensor memory");
  static constexpr uint32_t S_IDESC = (1u << 4) | ((KT / 8) << 17) | (8u << 24);                    // binary16 x binary16, binary32 sums
  static constexpr uint32_t O_IDESC = (1u << 4) | (1u << 16) | ((DP / 8) << 17) | (8u << 24);       // second operand across its rows
  static constexpr uint32_t TOK = KT / 4;                             // tokens of a converting warp
  static constexpr uint32_t PIECES = RB / 16, WIDE = PIECES < 4 ? PIECES : 4;   // 16-byte pieces of a row; how many of a row in one instruction
  static constexpr uint32_t HIGH = 32 / WIDE;                         // rows in one instruction
  static constexpr uint32_t LOADS = TOK * PIECES / 32;                // of a lane, for keys or values
  static constexpr uint32_t SCALE_WORDS = MX ? (NB + 6) / 4 : 1;
};

struct ChunkArgs {
  AttendArgs a;
  FastDiv page, group;
  uint32_t few;                             // sequences of as many rows or fewer are the other kernel's
  uint32_t vec_codes, vec_out;
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

// Where a CTA stands in the row of all units: sequence, row tile, key head, unit of that item.  Every warp keeps one of its own.
template <class F>
struct Walk {
  uint32_t seq, tile, tiles, kv, unit, unit1;    // units unit .. unit1 - 1 of the item are this CTA's
  uint64_t left;                                 // units of this CTA from here on
  AttendSeq s;
  ChunkTile t;
  __device__ __forceinline__ void enter(const ChunkArgs& p) {
    t = chunk_tile<F>(p, s, tile);
    unit1 = (uint32_t)min((uint64_t)t.units, unit + left);
  }
  __device__ __forceinline__ bool next(const ChunkArgs& p) {       // on to the next item
    left -= unit1 - unit;
    if (left == 0) return false;
    unit = 0;
    if (++kv == p.a.c.heads) {
      kv = 0;
      if (++tile == tiles) {
        tile = 0;
        do { s = attend_seq(p.a, ++seq); tiles = chunk_tiles<F>(p, s); } while (tiles == 0);
      }
    }
    enter(p);
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
  __shared__ uint64_t bars[17];
  __shared__ uint32_t tmem_slot, failed_flag;
  __shared__ int32_t highest[2][4];
  const AttendArgs& a = p.a;
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  uint8_t* const base = raw + ((1024u - (smem_addr(raw) & 1023u)) & 1023u);
  const uint32_t q_at = smem_addr(base), k_at = q_at + QT * F::Q_TILE, v_at = k_at + F::STAGES * F::KV_TILE;
  uint8_t* const meta = base + QT * F::Q_TILE + 2 * F::STAGES * F::KV_TILE;
  const uint32_t bar0 = smem_addr(bars);
  auto k_full = [&](uint32_t s) { return bar0 + 8 * s; };
  auto k_empty = [&](uint32_t s) { return bar0 + 8 * (2 + s); };
  auto v_full = [&](uint32_t s) { return bar0 + 8 * (4 + s); };
  auto v_empty = [&](uint32_t s) { return bar0 + 8 * (6 + s); };
  auto q_full = [&](uint32_t t) { return bar0 + 8 * (8 + t); };
  auto s_full = [&](uint32_t t) { return bar0 + 8 * (10 + t); };
  auto p_full = [&](uint32_t t) { return bar0 + 8 * (12 + t); };
  auto o_done = [&](uint32_t t) { return bar0 + 8 * (14 + t); };
  const uint32_t drained = bar0 + 8 * 16;
  volatile uint32_t* const failed = &failed_flag;
  dependency_wait();
  allow_dependents();

  if (tid == 0) {
    for (uint32_t s = 0; s < 2; ++s) {
      bar_init(k_full(s), 4); bar_init(k_empty(s), 1); bar_init(v_full(s), 4); bar_init(v_empty(s), 1);
      bar_init(q_full(s), 4); bar_init(s_full(s), 1); bar_init(p_full(s), 4); bar_init(o_done(s), 1);
    }
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
    for (uint32_t t = 0; t < tiles; ++t) sum += chunk_tile<F>(p, q, t).units;
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
  if (warp == 12) {
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
    const uint64_t n = (uint64_t)chunk_tile<F>(p, at.s, at.tile).units * a.c.heads;
    if (in_seq < n) break;
    in_seq -= n;
  }
  {
    const uint32_t units = chunk_tile<F>(p, at.s, at.tile).units;
    at.kv = (uint32_t)(in_seq / units);
    at.unit = (uint32_t)(in_seq % units);
    at.enter(p);
  }

  if (warp < 4 * QT) {
    // ---------------------------------------------------------------------------------- softmax
    const uint32_t t = warp / 4, lanes = ((warp % 4) * 32) << 16, r_in = 128 * t + (warp % 4) * 32 + lane;
    const uint32_t s_at = tmem + t * KT + lanes, o_at = tmem + F::O_COL + t * DP + lanes;
    uint32_t turn = 0;                                       // tiles done: phases of s_full, o_done; stage of the metadata
    const bool plain = !(a.cap > 0.f) && !a.slopes;
    uint32_t tiles_before = 0;                               // tiles of all items so far, with or without this warp's query tile
    do {
      const uint32_t n_units = at.unit1 - at.unit;
      const bool takes_part = t == 0 || at.t.row1 - at.t.row0 > 128;
      if (takes_part) {
        // the row: brought to the top of binary16's range by a power of two, signed like the scale
        const uint32_t r = at.t.row0 + r_in, i = p.group.div(min(r, at.t.row1 - 1)), head = at.kv * p.group.d + (min(r, at.t.row1 - 1) - i * p.group.d);
        const bool there = r < at.t.row1;
        const int32_t pos = at.t.pos0 + (int32_t)i;
        const int32_t pos_first = __shfl_sync(0xffffffffu, pos, 0), pos_last = __shfl_sync(0xffffffffu, pos, 31);
        const uint64_t from = (uint64_t)(at.s.row0 + i) * a.q_token_ld + (uint64_t)head * a.q_head_ld;
        uint32_t top = 0;
        auto each = [&](auto zero, const auto* q, auto&& use) {
#pragma unroll 1
          for (uint32_t d = 0; d < DP; d += 8) {
            auto e = zero;
            e.zero();
            if (there && d + 8 <= a.c.dim) e.load_any(q + from + d);
            else if (there && d < a.c.dim) e.load_some(q + from + d, a.c.dim - d);
            use(e, d);
          }
        };
        auto most = [&](auto& e, uint32_t) { top = max(top, e.top_bits()); };
        if (a.dtype == kBF16) each(Chunk8<__nv_bfloat16>(), (const __nv_bfloat16*)a.q, most);
        else each(Chunk8<__half>(), (const __half*)a.q, most);
        const int e = top ? max((int)(top >> 23) - 127, -100) : 0;
        const float up = copysignf(power_of_two(14 - min(e, 127)), a.scale);
        auto put = [&](auto& c, uint32_t d) {
          float v[8];
          c.widen(v);
          uint32_t h[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) h[k] = pack_half(v[2 * k] * up, v[2 * k + 1] * up);
          const uint32_t row = r_in % 128, to = q_at + t * F::Q_TILE + (d / 64) * F::Q_PANEL + row * 128 + (((d / 8) ^ row) & 7) * 16;
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
        };
        if (a.dtype == kBF16) each(Chunk8<__nv_bfloat16>(), (const __nv_bfloat16*)a.q, put);
        else each(Chunk8<__half>(), (const __half*)a.q, put);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive(q_full(t));
        const float back = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : power_of_two(min(e, 127) - 14) * power_of_two(MX ? -kChunkFactor : 0) * fabsf(a.scale) * (a.cap > 0.f ? 1.f : kLog2e);
        const float slope = a.slopes ? kLog2e * __ldg(a.slopes + head) : 0.f;

        float ref = -INFINITY, sum = 0.f;
        int v_top = -126;
        bool ok = true;
#pragma unroll 1
        for (uint32_t u = 0; u < n_units; ++u, ++turn) {
          const uint32_t stage = (tiles_before + u) % F::STAGES;
          const uint8_t* const m = meta + stage * F::META;
          const float4* const k_scale = reinterpret_cast<const float4*>(m);
          const float4* const v_scale = reinterpret_cast<const float4*>(m + 4 * KT);
          const uint32_t* const real = reinterpret_cast<const uint32_t*>(m + 8 * KT);
          if (!bar_wait(s_full(t), turn & 1, failed)) { ok = false; break; }
          tc_fence_after();
          const int v_now = *reinterpret_cast<const int32_t*>(m + 8 * KT + 16);
          const uint32_t j = at.t.j0 + (at.unit + u) * KT;
          bool every = (int32_t)(j + KT - 1) <= pos_first && pos_last - (int32_t)j < a.window;
#pragma unroll
          for (uint32_t k = 0; k < KT / 32; ++k) every &= real[k] == 0xffffffffu;

          // scores, to powers of two: the largest
          auto scores = [&](uint32_t c, float (&x)[32]) {
            tensor_read(s_at + 32 * c, x);
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) {
              const float4 f = k_scale[8 * c + k];
              x[4 * k] *= f.x; x[4 * k + 1] *= f.y; x[4 * k + 2] *= f.z; x[4 * k + 3] *= f.w;
            }
            if (!plain) {
#pragma unroll
              for (uint32_t k = 0; k < 32; ++k) {
                float v = x[k] * back;
                if (a.cap > 0.f) v = kLog2e * capped_fast(v, a.cap);
                x[k] = fmaf(slope, (float)(int32_t)(j + 32 * c + k - (uint32_t)pos), v);
              }
            }
            if (!every) {
              const uint32_t there_bits = real[c];
#pragma unroll
              for (uint32_t k = 0; k < 32; ++k) {
                const int32_t tok = (int32_t)(j + 32 * c + k);
                if (!((there_bits >> k & 1u) && tok <= pos && (uint32_t)pos - (uint32_t)tok < (uint32_t)a.window)) x[k] = -INFINITY;
              }
            }
          };
          const float mul = !plain ? 1.f : back < 1.2e-38f ? 1.2e-38f : back;      // not 0: it multiplies minus infinity, too
          float x[32], high = -INFINITY;
#pragma unroll 1
          for (uint32_t c = 0; c < KT / 32; ++c) {
            scores(c, x);
#pragma unroll
            for (uint32_t k = 0; k < 32; ++k) high = fmaxf(high, x[k]);
          }
          high = high == -INFINITY ? high : high * mul;      // (NaN from a poisoned query: its scores are NaN below)
          float soft = 1.f, values = 1.f;
          if (high > ref + kSlack) { soft = exp2_fast(ref - high); ref = high; }
          if (v_now != v_top) { values = power_of_two(max(v_top - v_now, -126)); v_top = v_now; }
          sum *= soft;
          if (u > 0 && __any_sync(0xffffffffu, soft * values != 1.f)) {
            if (!bar_wait(o_done(t), (turn - 1) & 1, failed)) { ok = false; break; }
            tc_fence_after();
#pragma unroll 1
            for (uint32_t c = 0; c < DP / 32; ++c) {
              float o[32];
              tensor_read(o_at + 32 * c, o);
#pragma unroll
              for (uint32_t k = 0; k < 32; ++k) o[k] *= soft * values;
              tensor_write(o_at + 32 * c, o);
            }
          }
          const float from_ref = ref == -INFINITY ? 0.f : ref;
#pragma unroll 1
          for (uint32_t c = 0; c < KT / 32; ++c) {
            scores(c, x);
            uint32_t h[16];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) {
              const float4 f = v_scale[8 * c + k];
              float w[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
              for (uint32_t i2 = 0; i2 < 4; ++i2) {
                const float e2 = exp2_fast(fmaf(x[4 * k + i2], mul, -from_ref));
                sum += e2;
                w[i2] = every || x[4 * k + i2] != -INFINITY ? e2 * w[i2] : 0.f;
              }
              h[2 * k] = pack_half(w[0], w[1]);
              h[2 * k + 1] = pack_half(w[2], w[3]);
            }
            tensor_write16(s_at + 16 * c, h);
          }
          tensor_write_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(p_full(t));
        }
        if (!ok) break;
        // ---- the rows' results
        if (!bar_wait(o_done(t), (turn - 1) & 1, failed)) break;
        tc_fence_after();
        const bool whole = at.unit == 0 && at.unit1 == at.t.units;
        const uint32_t place = at.unit == 0 ? 1 : 0;
        float* const part = p.parts + ((uint64_t)blockIdx.x * 2 + place) * F::ROWS * (DP + 2);
        const float f0 = power_of_two(-kChunkBits - (MX ? kChunkFactor : 0)), f1 = power_of_two(v_top);
        if (!whole && there) *reinterpret_cast<float2*>(part + F::ROWS * DP + 2 * r_in) = make_float2(ref, sum);
#pragma unroll 1
        for (uint32_t c = 0; c < DP / 32; ++c) {
          float o[32];
          tensor_read(o_at + 32 * c, o);
          if (!there) continue;
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k) {
            const float4 v = make_float4(o[4 * k] * f0 * f1, o[4 * k + 1] * f0 * f1, o[4 * k + 2] * f0 * f1, o[4 * k + 3] * f0 * f1);
            if (whole) attend_store(a, at.s.row0, r, p.group, at.kv, 32 * c + 4 * k, v, ref, sum, p.vec_out);
            else *reinterpret_cast<float4*>(part + r_in * DP + 32 * c + 4 * k) = v;
          }
        }
        if (!whole && place == 1 && tid == 0) {
          const uint64_t last = u_end - at.left + at.t.units - 1;     // u_end - left: the item's first unit
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
      tiles_before += n_units;
    } while (at.next(p));
  } else if (warp >= 8 && warp < 12) {
    // ---------------------------------------------------------------------------------- codes into operands
    constexpr uint32_t TOK = F::TOK, LOADS = F::LOADS, HIGH = F::HIGH, WORDS = F::SCALE_WORDS, PACKS = MX ? (NB + 3) / 4 : 1;
    const uint32_t part = warp - 8, first = part * TOK;                      // this warp's tokens of a tile
    const uint32_t blocks = (a.c.dim + 31) / 32, row_bytes = MX ? 16 * blocks : a.c.dim;
    uint4 code[2][LOADS];
    uint32_t scale_word[2][WORDS];
    uint32_t lead = 0;                                                       // where the scales begin in their first word, keys' and values'
    uint32_t n = 0;                                                          // tiles so far
    bool ok = true;
    do {
      const uint32_t n_units = at.unit1 - at.unit;
      const int32_t* const pages = a.table + at.seq * a.table_ld;
      auto token = [&](uint32_t u) { return (uint64_t)at.t.j0 + (uint64_t)(at.unit + u) * KT + first + lane; };
      auto page_of = [&](uint32_t u) -> int32_t {                            // of this lane's token of a tile; negative: no such token
        const uint64_t j = token(u);
        if (u >= n_units || lane >= TOK || j >= at.t.j1) return -1;
        const int32_t id = __ldg(pages + p.page.div((uint32_t)j));
        return id >= 0 && (uint32_t)id < a.c.pages ? id : -1;
      };
      auto fetch = [&](uint32_t u, int32_t id) {
        const uint32_t j = (uint32_t)token(u), off = j - p.page.div(j) * p.page.d;
        const uint64_t row = id < 0 ? 0 : ((uint64_t)(uint32_t)id * p.page.d + off) * a.c.heads + at.kv;
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (uint32_t k = 0; k < WORDS; ++k) scale_word[w][k] = 0;
        lead = 0;
        if (id >= 0) {
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            if (MX) {                                                        // whole words, each of which holds a wanted byte
              const uintptr_t from = (uintptr_t)a.c.scales[w] + row * blocks;
              const uint32_t l = (uint32_t)(from & 3u);
              lead |= l << (4 * w);
#pragma unroll
              for (uint32_t k = 0; k < WORDS; ++k)
                if (4 * k < l + blocks) scale_word[w][k] = __ldg(reinterpret_cast<const uint32_t*>(from & ~(uintptr_t)3u) + k);
            } else scale_word[w][0] = __ldg(reinterpret_cast<const uint32_t*>(a.c.scales[w]) + row);
          }
        }
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
          const uint32_t r = (i % (TOK / HIGH)) * HIGH + lane % HIGH, c16 = 16 * ((i / (TOK / HIGH)) * F::WIDE + lane / HIGH);
          const uint64_t src = __shfl_sync(0xffffffffu, row, r) * row_bytes + c16;
          const bool there = __shfl_sync(0xffffffffu, id, r) >= 0 && c16 < row_bytes;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            code[w][i] = make_uint4(0, 0, 0, 0);
            if (!there) continue;
            if (MX || p.vec_codes) code[w][i] = __ldg(reinterpret_cast<const uint4*>(a.c.codes[w] + src));
            else {
              uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
              for (uint32_t b = 0; b < 16; ++b)
                if (c16 + b < row_bytes) v[b / 4] |= (uint32_t)__ldg(a.c.codes[w] + src + b) << (8 * (b % 4));
              code[w][i] = make_uint4(v[0], v[1], v[2], v[3]);
            }
          }
        }
      };
      int32_t id = page_of(0), id_next = page_of(1);
      fetch(0, id);
      int v_top = -126;
#pragma unroll 1
      for (uint32_t u = 0; u < n_units; ++u, ++n) {
        const uint32_t s = n % F::STAGES, phase = (n / F::STAGES & 1) ^ 1;
        // scales, a token to a lane: the row's, and (4 bits) how far below it each block's is
        float scale[2] = {0.f, 0.f};
        uint32_t below[2][PACKS];
        const uint32_t real = __ballot_sync(0xffffffffu, id >= 0);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          if (MX) {
            const uint32_t shift = 8 * (lead >> (4 * w) & 3u);
            uint32_t bytes[PACKS], most = 0;
#pragma unroll
            for (uint32_t k = 0; k < PACKS; ++k) {
              bytes[k] = __funnelshift_r(scale_word[w][k], k + 1 < WORDS ? scale_word[w][k + 1 < WORDS ? k + 1 : 0] : 0u, shift);
              const uint32_t have = blocks - min(blocks, 4 * k);
              if (have < 4) bytes[k] &= (1u << (8 * have)) - 1u;
#pragma unroll
              for (uint32_t b = 0; b < 4; ++b) most = max(most, bytes[k] >> (8 * b) & 255u);
            }
            scale[w] = id >= 0 ? mx_scale(most) : 0.f;                       // NaN if any block is poisoned
#pragma unroll
            for (uint32_t k = 0; k < PACKS; ++k) below[w][k] = most == 255u || id < 0 ? ~0u : __vsubus4(most * 0x01010101u, bytes[k]);
          } else {
            scale[w] = __uint_as_float(scale_word[w][0]);
            below[w][0] = 0;
          }
        }
        const uint32_t field = __float_as_uint(scale[1]) >> 23 & 255u;       // finite scales are positive
        const int most = __reduce_max_sync(0xffffffffu, field == 255u ? -126 : min(max((int)field - 127, -126), 126));
        if (lane == 0) highest[n & 1][part] = most;
        ok = bar_wait(k_empty(s), phase, failed);
        ok = bar_wait(v_empty(s), phase, failed) && ok;
        ok = all_converting(ok);
        if (!ok) break;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) v_top = max(v_top, highest[n & 1][k]);
        uint8_t* const m = meta + s * F::META;
        if (lane < TOK) {
          reinterpret_cast<float*>(m)[first + lane] = scale[0];
          reinterpret_cast<float*>(m + 4 * KT)[first + lane] = scale[1] * power_of_two(-v_top) * (float)(1 << kChunkBits);
        }
        if (lane == 0) {
          if (TOK == 32) reinterpret_cast<uint32_t*>(m + 8 * KT)[part] = real;
          else reinterpret_cast<uint16_t*>(m + 8 * KT)[part] = (uint16_t)real;
          if (part == 0) *reinterpret_cast<int32_t*>(m + 8 * KT + 16) = v_top;
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t tile = (w ? v_at : k_at) + s * F::KV_TILE;
#pragma unroll
          for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t r = (i % (TOK / HIGH)) * HIGH + lane % HIGH, piece = (i / (TOK / HIGH)) * F::WIDE + lane / HIGH;
            const uint32_t row = first + r;
            auto put = [&](uint32_t d, uint32_t x, uint32_t y, uint32_t z, uint32_t t) {
              const uint32_t to = tile + (d / 64) * F::PANEL + row * 128 + (((d / 8) ^ row) & 7) * 16;
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(x), "r"(y), "r"(z), "r"(t) : "memory");
            };
            const uint32_t word[4] = {code[w][i].x, code[w][i].y, code[w][i].z, code[w][i].w};
            if (MX) {
              uint32_t pack = __shfl_sync(0xffffffffu, below[w][0], r);
              if (PACKS > 1) { const uint32_t more = __shfl_sync(0xffffffffu, below[w][PACKS - 1], r); if (piece >= 4) pack = more; }
              const int f = kChunkFactor - (int)(pack >> (8 * (piece & 3u)) & 255u);
              const uint32_t h = f < -24 ? 0u : f >= -14 ? (uint32_t)(f + 15) << 10 : 1u << (f + 24), factor = h | h << 16;
#pragma unroll
              for (uint32_t k = 0; k < 4; ++k) {
                uint32_t c[4];
                four_bits(word[k], c);
                put(32 * piece + 8 * k, half_mul(c[0], factor), half_mul(c[1], factor), half_mul(c[2], factor), half_mul(c[3], factor));
              }
            } else {
#pragma unroll
              for (uint32_t k = 0; k < 4; k += 2) {
                const uint32_t x = word[k] ^ 0x80808080u, y = word[k + 1] ^ 0x80808080u;
                put(16 * piece + 4 * k, eight_bits<0x4140>(x), eight_bits<0x4342>(x), eight_bits<0x4140>(y), eight_bits<0x4342>(y));
              }
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive(w ? v_full(s) : k_full(s));
        }
        id = id_next;
        id_next = page_of(u + 2);
        if (u + 1 < n_units) fetch(u + 1, id);
      }
    } while (ok && at.next(p));
  } else if (warp == 12) {
    // ---------------------------------------------------------------------------------- products
    uint32_t n = 0, q_turn[2] = {0, 0}, p_turn[2] = {0, 0};
    auto scores = [&](uint32_t t, uint32_t s) {                              // by one lane
#pragma unroll
      for (uint32_t k = 0; k < DP / 16; ++k)
        tensor_product(tmem + t * KT, rows_desc(q_at + t * F::Q_TILE + (k / 4) * F::Q_PANEL) + 2 * (k % 4), rows_desc(k_at + s * F::KV_TILE + (k / 4) * F::PANEL) + 2 * (k % 4),
                       F::S_IDESC, k > 0);
      tensor_commit(s_full(t));
    };
    auto results = [&](uint32_t t, uint32_t s, bool add) {
#pragma unroll
      for (uint32_t k = 0; k < KT / 16; ++k)
        tensor_product_from(tmem + F::O_COL + t * DP, tmem + t * KT + 8 * k, columns_desc(v_at + s * F::KV_TILE, F::PANEL) + 128 * k, F::O_IDESC, add || k > 0);
      tensor_commit(o_done(t));
    };
    bool ok = true;
    do {
      const uint32_t n_units = at.unit1 - at.unit, nt = QT == 2 && at.t.row1 - at.t.row0 > 128 ? 2 : 1;
      for (uint32_t t = 0; ok && t < nt; ++t) { ok = bar_wait(q_full(t), q_turn[t] & 1, failed); ++q_turn[t]; }
      ok = ok && bar_wait(k_full(n % 2), n / 2 & 1, failed);
      if (!ok) break;
      tc_fence_after();
      if (elect_one()) {
        for (uint32_t t = 0; t < nt; ++t) scores(t, n % 2);
        tensor_commit(k_empty(n % 2));
      }
      __syncwarp();
#pragma unroll 1
      for (uint32_t u = 0; u < n_units; ++u, ++n) {
        const bool more = u + 1 < n_units;
        if (!bar_wait(v_full(n % 2), n / 2 & 1, failed)) { ok = false; break; }
        for (uint32_t t = 0; t < nt; ++t) {
          if (!bar_wait(p_full(t), p_turn[t] & 1, failed)) { ok = false; break; }
          ++p_turn[t];
          tc_fence_after();
          if (elect_one()) {
            results(t, n % 2, u > 0);
            if (t + 1 == nt) tensor_commit(v_empty(n % 2));
          }
          __syncwarp();
          if (!more) continue;
          if (t == 0 && !bar_wait(k_full((n + 1) % 2), (n + 1) / 2 & 1, failed)) { ok = false; break; }
          if (t == 0) tc_fence_after();
          if (elect_one()) {
            scores(t, (n + 1) % 2);
            if (t + 1 == nt) tensor_commit(k_empty((n + 1) % 2));
          }
          __syncwarp();
        }
        if (!ok) break;
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
  if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
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

template <int FORMAT>
cudaError_t launch_dim(const Launch& l, const ChunkArgs& p, const AttendRun& run, uint64_t* launches) {
  if (run.dp == 64) return launch_chunk<Chunk<FORMAT, 64>>(l, p, run, launches);
  if (run.dp == 128) return launch_chunk<Chunk<FORMAT, 128>>(l, p, run, launches);
  return launch_chunk<Chunk<FORMAT, 256>>(l, p, run, launches);
}

}  // namespace

cudaError_t launch_attend_chunk(const Launch& l, const AttendArgs& a, const AttendRun& run, uint64_t* launches) {
  ChunkArgs p;
  p.a = a; p.page = FastDiv(a.c.page_size); p.group = FastDiv(a.group); p.few = run.few;
  p.vec_codes = a.c.dim % 16 == 0 && ((uintptr_t)a.c.codes[0] | (uintptr_t)a.c.codes[1]) % 16 == 0;
  p.vec_out = attend_vec_out(a); p.fault = run.fault;
  return a.c.format == QV2_KV_MX4 ? launch_dim<QV2_KV_MX4>(l, p, run, launches) : launch_dim<QV2_KV_I8>(l, p, run, launches);
}

}  // namespace qv2
