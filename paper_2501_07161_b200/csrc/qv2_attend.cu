// Attention of new tokens over the quantized paged cache, few query rows to a key head: decoding steps and drafts.
//
// Bound by reading the cache (a key or value of 128 elements is 68 bytes at 4 bits, 132 at 8), next by turning codes into
// operands.  A warp has one key head and a run of tokens and needs no other warp until the end: codes of TOK tokens
// come by cp.async into its own ring in shared memory, go through registers as operands of mma.sync (16 tokens x 8 query rows
// for the scores, transposed probabilities for the values), and the softmax runs along (running maximum and sum).
//
// Measured: 8 sequences of up to 32000 tokens, 32 heads over 8 of 128 elements, 4 bits (231 MB, all that is read): 77 us, 3.0 TB/s; 64 sequences of
// up to 2000 at 8 bits (208 MB): 61 us, 3.4 TB/s.  What bounds it is issue: 2.5 instructions a cycle and SM, of them 23 % for turning codes of values into
// operands and multiplying them, 10 % for scales, 9 % for the softmax.
//
// Codes enter as they are: 4-bit codes and 8-bit integers are exact in binary16.  Scales of keys multiply the scores of their block
// (32 columns: two products), or of the row; scales of values are split into the row's (multiplied into its weight) and
// a power of two per block (multiplied into the codes, exactly).  Queries are brought to the top of binary16's range by
// a power of two per row, so 16-bit ones are exact; of 32-bit ones (TERMS = 2) the rest of the rounding enters as a second
// operand, and so for the weights.  Weights p_j * scale_j are held against the largest value scale met so far and
// rounded to binary16, 2^14 at most, so what binary16 loses is below 2^-38 of the largest.
#include "qv2_attend.cuh"

namespace qv2 {

namespace {

constexpr uint32_t kDepth = 2;                             // stages of a warp's ring
constexpr uint32_t kBegin = 3;                             // what an item costs besides its units, in units
constexpr int kWeightBits = 13;                            // weights stand 2^13 above p * scale / (largest scale)
constexpr int kFactorBits = 12;                            // 4 bits: block factors stand 2^12 above scale / (largest of the row)

__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {      // the rest of the 16 becomes zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
template <uint32_t N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t* p) {
  if constexpr (N == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (N == 2) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
  else
#pragma unroll
    for (uint32_t i = 0; i < N; i += 4) { const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i); w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w; }
}

template <uint32_t N>
__device__ __forceinline__ void load_floats(float (&f)[N], const float* p) {
  if constexpr (N == 2) { const float2 v = *reinterpret_cast<const float2*>(p); f[0] = v.x; f[1] = v.y; }
  else
#pragma unroll
    for (uint32_t i = 0; i < N; i += 4) { const float4 v = *reinterpret_cast<const float4*>(p + i); f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w; }
}

template <int FORMAT_, int DP_, int NT_, int TERMS_>
struct Form {
  static constexpr int FORMAT = FORMAT_, DP = DP_, NT = NT_, TERMS = TERMS_;
  static constexpr bool MX = FORMAT == QV2_KV_MX4;
  static constexpr uint32_t ROWS = 8 * NT;                 // query rows of an item
  static constexpr uint32_t NB = DP / 32;                  // blocks of a row
  static constexpr uint32_t RB = MX ? DP / 2 : DP;         // bytes of a row's codes
  static constexpr uint32_t TOK = RB <= 64 ? 32 : 16;      // tokens of a stage: some 4 KB of codes
  static constexpr uint32_t TILES = TOK / 16;
  // Rows in shared memory lie so far apart that the loads of a warp (keys: 8 rows, 4 lanes each; values: 4 pairs of rows, 8
  // lanes each) meet every bank once.
  static constexpr uint32_t KS = RB + (MX ? 16 : 32), VS = RB + 16;
  static constexpr uint32_t RAW = MX ? 4 * ((NB + 6) / 4) : 4;      // bytes of a row's scales as they lie in memory: whole words
  static constexpr uint32_t STAGE = TOK * (KS + VS + 2 * RAW + 4);  // ... and a word that says where they begin, or that there is no such token
  static constexpr uint32_t READY = MX ? TOK * (4 * NB + 4) + TOK * 2 * NB : TOK * 8;   // scales as the products want them
  static constexpr uint32_t WARP = (kDepth * STAGE + READY + 15) / 16 * 16;
  // One CTA per SM: sixteen warps where a thread's accumulators and operands leave room in 128 registers, else eight.
  static constexpr uint32_t WARPS = (DP / 16) * 4 * NT + 4 * NB * NT * TERMS > 64 ? 8 : 16, THREADS = 32 * WARPS;
  static constexpr uint32_t EXCHANGE = WARPS * ROWS * DP * 4;
  static constexpr uint32_t SMEM = WARPS * WARP > EXCHANGE ? WARPS * WARP : EXCHANGE;
  static_assert(SMEM + 4096 <= 232448, "shared memory");
  static constexpr uint32_t PIECE = ROWS * (DP + 2);       // floats of a head of a partial result
};

struct RowsArgs {
  AttendArgs a;
  FastDiv page, group;
  uint32_t hw, hw_log;                                     // key heads of a CTA (a power of two), warps / hw warps share the tokens
  uint32_t row_limit;                                      // sequences of more rows are not this kernel's
  uint32_t vec_q, vec_codes, vec_out;                      // queries and codes by 16 bytes, results by four elements
  uint32_t quick;                                          // ... and rows of scales are whole aligned words
  uint32_t token_codes, token_scales;                      // bytes of a token's codes and scales, all heads
  float* parts;
  AttendPiece* pieces;
};

// Units of every item of a sequence, and its items.
template <class F>
__device__ __forceinline__ void units_of(const RowsArgs& p, const AttendSeq& s, uint32_t* units, uint32_t* tiles) {
  const uint64_t rows = (uint64_t)s.n * p.a.group;
  *tiles = rows > p.row_limit ? 0 : (uint32_t)((rows + F::ROWS - 1) / F::ROWS);
  const uint32_t sees = (uint32_t)p.a.window + (F::ROWS + p.a.group - 1) / p.a.group;       // tokens that a tile of rows sees at most
  const uint32_t wide = min(min((uint32_t)s.len, p.a.room), sees), unit = F::TOK * (F::WARPS >> p.hw_log);
  *units = max(1u, (wide + unit - 1) / unit);
}

template <class F>
__global__ void __launch_bounds__(F::THREADS, 1) attend_rows_kernel(const RowsArgs p) {
  constexpr bool MX = F::MX;
  constexpr int NT = F::NT, DP = F::DP, TERMS = F::TERMS;
  constexpr uint32_t kWarps = F::WARPS, kThreads = F::THREADS, NB = F::NB, TOK = F::TOK, TILES = F::TILES, ROWS = F::ROWS;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ uint64_t scan[kWarps];
  __shared__ AttendUnits found;
  __shared__ float2 top_sum[kWarps][ROWS];
  const AttendArgs& a = p.a;
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, t = lane % 4;
  dependency_wait();
  allow_dependents();

  // ---- this CTA's units
  const uint32_t groups = a.c.heads >> p.hw_log;                               // groups of key heads
  auto units_in = [&](uint32_t s) -> uint64_t {
    if (s >= a.seqs) return 0;
    uint32_t units, tiles;
    units_of<F>(p, attend_seq(a, s), &units, &tiles);
    return (uint64_t)(units + kBegin) * tiles * groups;
  };
  uint64_t all = 0;
  for (uint32_t base = 0; base < a.seqs; base += kThreads) all += units_in(base + tid);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  if (lane == 0) scan[warp] = all;
  __syncthreads();
  all = 0;
#pragma unroll
  for (uint32_t w = 0; w < kWarps; ++w) all += scan[w];
  const uint32_t ctas = (uint32_t)min((uint64_t)gridDim.x, all);                // every one of these has a unit at least
  if (tid == 0) p.pieces[blockIdx.x].followers = 0;
  if (blockIdx.x >= ctas) return;
  const uint64_t u_begin = all * blockIdx.x / ctas, u_end = all * (blockIdx.x + 1) / ctas;
  for (uint64_t base = 0, before = 0; base < a.seqs; base += kThreads) {        // which sequence u_begin falls into
    __syncthreads();
    const uint64_t mine = units_in((uint32_t)base + tid);
    uint64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint64_t v = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += v; }
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    uint64_t whole = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) { if (w < warp) sum += scan[w]; whole += scan[w]; }
    const uint64_t first = before + sum - mine;
    if (mine && u_begin >= first && u_begin < first + mine) { found.before = first; found.seq = (uint32_t)base + tid; }
    before += whole;
    if (u_begin < before) break;
  }
  __syncthreads();
  uint32_t seq = found.seq;
  uint64_t at_unit = u_begin, seq_begin = found.before;

  const uint32_t head_in = warp & (p.hw - 1), part = warp >> p.hw_log, parts = kWarps >> p.hw_log;
  uint8_t* const mine = smem + warp * F::WARP;
  const uint32_t ring = shared_at(mine);
  uint8_t* const ready = mine + kDepth * F::STAGE;
  float* const k_scale = reinterpret_cast<float*>(ready);                       // 4 bits: [token][block], 8 bits: [token]
  float* const v_scale = k_scale + TOK * (MX ? NB : 1);                         // [token], against the largest
  __half* const v_factor = reinterpret_cast<__half*>(v_scale + TOK);            // 4 bits: [block][token]
  const uint32_t blocks = (a.c.dim + 31) / 32, row_bytes = MX ? 16 * blocks : a.c.dim;

  while (at_unit < u_end) {
    // ---- the next item, or the part of it that is this CTA's
    AttendSeq s = attend_seq(a, seq);
    uint32_t units, tiles;
    units_of<F>(p, s, &units, &tiles);
    const uint32_t cost = units + kBegin;
    const uint64_t in_seq = (uint64_t)cost * tiles * groups;
    if (at_unit - seq_begin >= in_seq) { seq_begin += in_seq; ++seq; continue; }
    const uint32_t item = (uint32_t)((at_unit - seq_begin) / cost), x0 = (uint32_t)((at_unit - seq_begin) % cost);
    const uint32_t x1 = (uint32_t)min((uint64_t)cost, x0 + (u_end - at_unit));
    const uint32_t unit0 = max(x0, kBegin) - kBegin, unit1 = max(x1, kBegin) - kBegin;
    if (unit0 == unit1) { at_unit += x1 - x0; continue; }                       // (of the setup alone there is nothing to do)
    const uint32_t tile = item / groups, hg = item % groups, kv = (hg << p.hw_log) + head_in;
    const uint32_t rows = s.n * a.group, row0 = tile * ROWS, row1 = min(rows, row0 + ROWS);
    const int32_t pos0 = s.len - (int32_t)s.n;                                  // position of the sequence's first query
    const int32_t p_first = pos0 + (int32_t)p.group.div(row0), p_last = pos0 + (int32_t)p.group.div(row1 - 1);
    const uint32_t j0 = min(p_first >= a.window ? (uint32_t)(p_first - a.window + 1) : 0u, a.room);   // tokens that any of the rows sees: j0 .. j1 - 1
    const uint32_t j1 = max(min((uint32_t)(max(p_last, -1) + 1), a.room), j0);
    const int32_t* const pages = a.table + seq * a.table_ld;

    // ---- tokens: stage k of this warp begins at j0 + (first + k * parts) * TOK
    const uint32_t n_stages = unit1 - unit0;
    auto stage_token = [&](uint32_t k) { return (uint64_t)j0 + (uint64_t)((unit0 + k) * parts + part) * TOK; };
    auto page_of = [&](uint32_t k) -> int32_t {                                  // of token `lane` of a stage; negative: no such token
      const uint64_t j = stage_token(k) + lane;
      if (k >= n_stages || lane >= TOK || j >= j1) return -1;
      const int32_t id = __ldg(pages + p.page.div((uint32_t)j));
      return id >= 0 && (uint32_t)id < a.c.pages ? id : -1;
    };
    constexpr uint32_t CH = F::RB / 16, PER = 32 / CH;                           // 16-byte pieces of a row, rows of one instruction
    const uint32_t c16 = 16 * (lane % CH), tok0 = lane / CH;
    const bool piece = c16 < row_bytes;
    const uint32_t piece_bytes = piece ? 16 : 0;
    const uint64_t row_in_token = (uint64_t)kv * row_bytes;
    const uint8_t *const k_src = a.c.codes[0] + row_in_token + c16, *const v_src = a.c.codes[1] + row_in_token + c16;
    const uint32_t k_dst = tok0 * F::KS + c16, v_dst = TOK * F::KS + tok0 * F::VS + c16;
    const uint32_t scale_bytes = MX ? blocks : 4;                                // of a row
    const uint8_t *const ks_src = a.c.scales[0] + (uint64_t)kv * scale_bytes, *const vs_src = a.c.scales[1] + (uint64_t)kv * scale_bytes;
    auto fetch = [&](uint32_t k, int32_t id) {                                   // codes and scales of a stage into its place of the ring
      const uint32_t place = (k % kDepth) * F::STAGE;
      if (k < n_stages) {
        const uint32_t j = (uint32_t)stage_token(k) + lane, off = j - p.page.div(j) * p.page.d;
        const uint64_t token = (uint64_t)(uint32_t)max(id, 0) * p.page.d + (id < 0 ? 0 : off);      // in the cache
        const int64_t bytes = (int64_t)(token * p.token_codes);
        const uint32_t raw = place + TOK * (F::KS + F::VS), where = ring + place;
        if (p.quick && __all_sync(0xffffffffu, id >= 0 || lane >= TOK)) {          // whole aligned words and pieces, and every token is there
#pragma unroll
          for (uint32_t i = 0; i < TOK / PER; ++i) {
            const int64_t row = __shfl_sync(0xffffffffu, bytes, i * PER + tok0);
            copy16(where + k_dst + i * PER * F::KS, k_src + row, piece_bytes);
            copy16(where + v_dst + i * PER * F::VS, v_src + row, piece_bytes);
          }
          if (lane < TOK) {
            const uint64_t first = token * p.token_scales;
#pragma unroll
            for (uint32_t i = 0; i < (MX ? (NB + 3) / 4 : 1); ++i)
              if (!MX || 4 * i + 4 <= blocks) {
                copy4(ring + raw + lane * F::RAW + 4 * i, ks_src + first + 4 * i, true);
                copy4(ring + raw + TOK * F::RAW + lane * F::RAW + 4 * i, vs_src + first + 4 * i, true);
              }
            *reinterpret_cast<uint32_t*>(mine + raw + 2 * TOK * F::RAW + 4 * lane) = 0u;
          }
        } else {
          const int64_t known = id < 0 ? -1 : bytes;
#pragma unroll 1
          for (uint32_t i = 0; i < TOK / PER; ++i) {
            const int64_t row = __shfl_sync(0xffffffffu, known, i * PER + tok0);
            const bool there = row >= 0 && piece;
            const uint64_t from = there ? (uint64_t)row : 0;
            if (MX || p.vec_codes) {
              copy16(where + k_dst + i * PER * F::KS, k_src + from, there ? 16 : 0);
              copy16(where + v_dst + i * PER * F::VS, v_src + from, there ? 16 : 0);
            } else
              for (uint32_t b = 0; b < 16; ++b) {
                const bool has = there && c16 + b < row_bytes;
                mine[place + k_dst + i * PER * F::KS + b] = has ? __ldg(k_src + from + b) : (uint8_t)0;
                mine[place + v_dst + i * PER * F::VS + b] = has ? __ldg(v_src + from + b) : (uint8_t)0;
              }
          }
          if (lane < TOK) {
            const uint64_t first = token * p.token_scales;
            uint32_t skip = 0;
#pragma unroll
            for (int w = 0; w < 2; ++w) {                                        // whole words, each of which holds a wanted byte
              const uintptr_t from = (uintptr_t)(w ? vs_src : ks_src) + first;
              const uint32_t lead = (uint32_t)(from & 3u);
              skip |= lead << (8 * w);
#pragma unroll
              for (uint32_t i = 0; i < F::RAW / 4; ++i)
                if (4 * i < lead + scale_bytes) copy4(ring + raw + w * TOK * F::RAW + lane * F::RAW + 4 * i, (const void*)((from & ~(uintptr_t)3u) + 4 * i), id >= 0);
            }
            *reinterpret_cast<uint32_t*>(mine + raw + 2 * TOK * F::RAW + 4 * lane) = id >= 0 ? skip : ~0u;
          }
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int32_t next_id = page_of(0);
#pragma unroll 1
    for (uint32_t k = 0; k < kDepth; ++k) {
      const int32_t id = next_id;
      next_id = page_of(k + 1);
      fetch(k, id);
    }
    // ---- queries, while the first stages are on their way: as operands, with what brings their scores back (to powers of two unless they are capped)
    uint32_t qf[TERMS][NT][4 * NB];
    float back[NT][2];
    int32_t pos[NT][2];
    float slope[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint32_t r = row0 + 8 * n + g;
      const bool there = r < row1;
      float v[NB][8];
      uint32_t top = 0;
      const uint32_t rc = min(r, row1 - 1), ic = p.group.div(rc);                // (rows that are not there take another's elements, times zero)
      const uint64_t q_at = (uint64_t)(s.row0 + ic) * a.q_token_ld + (uint64_t)(kv * a.group + (rc - ic * a.group)) * a.q_head_ld;
      auto bring = [&](auto zero, const auto* from) {
        decltype(zero) chunk[NB];
        if (p.vec_q) {
#pragma unroll
          for (uint32_t b = 0; b < NB; ++b) chunk[b].load_vec(from + q_at + min(32 * b + 8 * t, a.c.dim - 8));
        } else {
#pragma unroll
          for (uint32_t b = 0; b < NB; ++b) {
            const uint32_t d = 32 * b + 8 * t;
            chunk[b].zero();
            if (d + 8 <= a.c.dim) chunk[b].load_any(from + q_at + d);
            else if (d < a.c.dim) chunk[b].load_some(from + q_at + d, a.c.dim - d);
          }
        }
#pragma unroll
        for (uint32_t b = 0; b < NB; ++b) {
          chunk[b].widen(v[b]);
          top = max(top, chunk[b].top_bits());
          if (32 * b + 8 * t >= a.c.dim)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[b][k] = 0.f;
        }
      };
      if (a.dtype == kBF16) bring(Chunk8<__nv_bfloat16>(), (const __nv_bfloat16*)a.q);
      else if (a.dtype == kF16) bring(Chunk8<__half>(), (const __half*)a.q);
      else bring(Chunk8<float>(), (const float*)a.q);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = top ? max((int)(top >> 23) - 127, -100) : 0;                // the largest element is 2^e to 2^(e+1)
      const float up = there ? power_of_two(14 - min(e, 127)) : 0.f;
#pragma unroll
      for (uint32_t b = 0; b < NB; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float x = v[b][2 * k] * up, y = v[b][2 * k + 1] * up;
          qf[0][n][4 * b + k] = pack_half(x, y);
          if (TERMS == 2) {
            const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&qf[0][n][4 * b + k]));
            qf[TERMS - 1][n][4 * b + k] = pack_half(x - h.x, y - h.y);
          }
        }
      const float down = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : power_of_two(min(e, 127) - 14) * a.scale * (a.cap > 0.f ? 1.f : kLog2e);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        back[n][k] = __shfl_sync(0xffffffffu, down, 4 * (2 * t + k));
        const uint32_t rr = row0 + 8 * n + 2 * t + k, ii = p.group.div(rr);
        pos[n][k] = rr < row1 ? pos0 + (int32_t)ii : p_last;                    // (rows that are not there hold nothing up)
        slope[n][k] = a.slopes && rr < row1 ? kLog2e * __ldg(a.slopes + kv * a.group + (rr - ii * a.group)) : 0.f;
      }
    }
    float o[NT][DP / 16][4], top_x[NT][2], sum[NT][2];
    int v_top = -126;                                                          // exponent of the largest value scale so far
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      top_x[n][0] = top_x[n][1] = -INFINITY; sum[n][0] = sum[n][1] = 0.f;
#pragma unroll
      for (int m = 0; m < DP / 16; ++m)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[n][m][k] = 0.f;
    }

#pragma unroll 1
    for (uint32_t k = 0; k < n_stages; ++k) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
      __syncwarp();
      const int32_t id = next_id;                                                // of stage k + kDepth
      next_id = page_of(k + kDepth + 1);
      const uint32_t place = (k % kDepth) * F::STAGE, raw = place + TOK * (F::KS + F::VS);
      const uint32_t j_stage = (uint32_t)stage_token(k);

      // ---- scales of the stage's tokens, one to a lane
      uint32_t meta = ~0u;
      if (lane < TOK) meta = *reinterpret_cast<const uint32_t*>(mine + raw + 2 * TOK * F::RAW + 4 * lane);
      const uint32_t real = __ballot_sync(0xffffffffu, meta != ~0u);             // tokens that there are
      float v_row = 0.f;                                                         // scale of this lane's value
      if (MX) {
        constexpr uint32_t PACKS = (NB + 3) / 4, WORDS = F::RAW / 4;
        const uint32_t *kw = reinterpret_cast<const uint32_t*>(mine + raw + lane * F::RAW), *vw = reinterpret_cast<const uint32_t*>(mine + raw + TOK * F::RAW + lane * F::RAW);
        uint32_t kb[PACKS], vb[PACKS], v_most = 0;                               // bytes of the row's blocks; 0 where there is none
        float ks[NB];
        if (lane < TOK) {
#pragma unroll
          for (uint32_t i = 0; i < PACKS; ++i) {
            const uint32_t have = blocks - min(blocks, 4 * i), keep = meta == ~0u ? 0u : have < 4 ? (1u << (8 * have)) - 1u : ~0u;
            kb[i] = __funnelshift_r(kw[i], i + 1 < WORDS ? kw[i + 1] : 0u, 8 * (meta & 3u)) & keep;
            vb[i] = __funnelshift_r(vw[i], i + 1 < WORDS ? vw[i + 1] : 0u, 8 * (meta >> 8 & 3u)) & keep;
            const uint32_t two = __vmaxu2(vb[i] & 0x00ff00ffu, vb[i] >> 8 & 0x00ff00ffu);
            v_most = max(v_most, max(two & 0xffffu, two >> 16));
          }
#pragma unroll
          for (uint32_t b = 0; b < NB; ++b) {
            const uint32_t byte = kb[b / 4] >> (8 * (b % 4)) & 255u;
            ks[b] = __uint_as_float(byte << 23 | (byte + 1) >> 8 << 22);         // 2^(byte - 127); 255: NaN; 0: none, for the 2^-127 that it means
          }
          if constexpr (NB == 2) *reinterpret_cast<float2*>(k_scale + lane * NB) = make_float2(ks[0], ks[1]);
          else
#pragma unroll
            for (uint32_t b = 0; b < NB; b += 4) *reinterpret_cast<float4*>(k_scale + lane * NB + b) = make_float4(ks[b], ks[b + 1], ks[b + 2], ks[b + 3]);
          v_row = meta == ~0u ? 0.f : mx_scale(v_most);                          // NaN if any block is poisoned
          // 2^(own - row's largest + kFactorBits) in binary16, down to its smallest number 2^-24
          const uint32_t base = (uint32_t)(127 + kFactorBits) - v_most;
#pragma unroll
          for (uint32_t b = 0; b < NB; ++b) {
            const int e = (int)((vb[b / 4] >> (8 * (b % 4)) & 255u) + base);
            v_factor[b * TOK + lane] = __float2half_rn(v_most == 255u ? 0.f : __uint_as_float((uint32_t)max(e, 0) << 23));
          }
        }
      } else if (lane < TOK) {
        k_scale[lane] = *reinterpret_cast<const float*>(mine + raw + 4 * lane);
        v_row = *reinterpret_cast<const float*>(mine + raw + TOK * F::RAW + 4 * lane);
      }
      const uint32_t field = __float_as_uint(v_row) >> 23 & 255u;                // finite scales are positive
      const int highest = __reduce_max_sync(0xffffffffu, field == 255u ? -126 : min(max((int)field - 127, -126), 126));
      if (highest > v_top) {
        const float f = v_top == -126 ? 0.f : power_of_two(max(v_top - highest, -126));   // (nothing has been added at -126 that could be seen)
        v_top = highest;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int m = 0; m < DP / 16; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][m][i] *= f;
      }
      if (lane < TOK) v_scale[lane] = v_row * power_of_two(-v_top) * (float)(1 << kWeightBits);
      __syncwarp();

      // ---- scores: rows are tokens, columns queries
      float x[TILES][NT][4];
#pragma unroll
      for (uint32_t l = 0; l < TILES; ++l) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[l][n][i] = 0.f;
        float s0[MX ? NB : 1], s1[MX ? NB : 1];
        if constexpr (MX) {
          load_floats<NB>(s0, k_scale + (16 * l + g) * NB);
          load_floats<NB>(s1, k_scale + (16 * l + g + 8) * NB);
        } else { s0[0] = k_scale[16 * l + g]; s1[0] = k_scale[16 * l + g + 8]; }
        const uint8_t* k0 = mine + place + (16 * l + g) * F::KS;
        const uint8_t* k1 = k0 + 8 * F::KS;
#pragma unroll
        for (uint32_t b = 0; b < NB; ++b) {
          uint32_t c0[4], c1[4];
          if (MX) {
            four_bits(*reinterpret_cast<const uint32_t*>(k0 + 16 * b + 4 * t), c0);
            four_bits(*reinterpret_cast<const uint32_t*>(k1 + 16 * b + 4 * t), c1);
          } else {
            const uint2 w0 = *reinterpret_cast<const uint2*>(k0 + 32 * b + 8 * t), w1 = *reinterpret_cast<const uint2*>(k1 + 32 * b + 8 * t);
            c0[0] = eight_bits<0x4140>(w0.x ^ 0x80808080u); c0[1] = eight_bits<0x4342>(w0.x ^ 0x80808080u);
            c0[2] = eight_bits<0x4140>(w0.y ^ 0x80808080u); c0[3] = eight_bits<0x4342>(w0.y ^ 0x80808080u);
            c1[0] = eight_bits<0x4140>(w1.x ^ 0x80808080u); c1[1] = eight_bits<0x4342>(w1.x ^ 0x80808080u);
            c1[2] = eight_bits<0x4140>(w1.y ^ 0x80808080u); c1[3] = eight_bits<0x4342>(w1.y ^ 0x80808080u);
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
            float (&into)[4] = MX ? acc : x[l][n];
#pragma unroll
            for (int term = TERMS - 1; term >= 0; --term) {
              mma16816(into, c0[0], c1[0], c0[1], c1[1], qf[term][n][4 * b], qf[term][n][4 * b + 1]);
              mma16816(into, c0[2], c1[2], c0[3], c1[3], qf[term][n][4 * b + 2], qf[term][n][4 * b + 3]);
            }
            if (MX) {
              const float f0 = s0[MX ? b : 0], f1 = s1[MX ? b : 0];
              x[l][n][0] = fmaf(acc[0], f0, x[l][n][0]); x[l][n][1] = fmaf(acc[1], f0, x[l][n][1]);
              x[l][n][2] = fmaf(acc[2], f1, x[l][n][2]); x[l][n][3] = fmaf(acc[3], f1, x[l][n][3]);
            }
          }
        }
        if (!MX) {
#pragma unroll
          for (int n = 0; n < NT; ++n) { x[l][n][0] *= s0[0]; x[l][n][1] *= s0[0]; x[l][n][2] *= s1[0]; x[l][n][3] *= s1[0]; }
        }
      }

      // ---- what is seen, and the softmax so far
      const bool plain = !(a.cap > 0.f) && !a.slopes;
      const bool every = real == 0xffffffffu >> (32 - TOK) && (int32_t)(j_stage + TOK - 1) <= p_first && p_last - (int32_t)j_stage < a.window;
      uint32_t seen = 0xffffffffu;                                               // bit of x[l][n][i]: 4 * (l * NT + n) + i
      static_assert(4 * TILES * NT <= 32, "bits");
#pragma unroll
      for (uint32_t l = 0; l < TILES; ++l)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = x[l][n][i] * back[n][i & 1];
            const uint32_t tok = 16 * l + g + 8 * (i >> 1);
            const int32_t at = (int32_t)(j_stage + tok), mine_pos = pos[n][i & 1];
            if (!plain) {
              if (a.cap > 0.f) v = kLog2e * (TERMS == 2 ? a.cap * tanhf(v / a.cap) : capped_fast(v, a.cap));
              v = fmaf(slope[n][i & 1], (float)(int32_t)((uint32_t)at - (uint32_t)mine_pos), v);
            }
            if (!every) {
              const bool ok = (real >> tok & 1u) && at <= mine_pos && (uint32_t)mine_pos - (uint32_t)at < (uint32_t)a.window;
              if (!ok) { v = -INFINITY; seen &= ~(1u << (4 * (l * NT + n) + i)); }
            }
            x[l][n][i] = v;
          }
      bool moved = false;
      float shrink[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float m = fmaxf(x[0][n][k], x[0][n][k + 2]);
#pragma unroll
          for (uint32_t l = 1; l < TILES; ++l) m = fmaxf(m, fmaxf(x[l][n][k], x[l][n][k + 2]));
#pragma unroll
          for (int b = 4; b < 32; b <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, b));
          m = fmaxf(m, top_x[n][k]);
          const float from = m == -INFINITY ? 0.f : m;
          shrink[n][k] = exp2_fast(top_x[n][k] - from);
          moved |= top_x[n][k] != m;
          top_x[n][k] = m;
          float add = 0.f;
#pragma unroll
          for (uint32_t l = 0; l < TILES; ++l) {
            x[l][n][k] = exp2_fast(x[l][n][k] - from); x[l][n][k + 2] = exp2_fast(x[l][n][k + 2] - from);
            add += x[l][n][k] + x[l][n][k + 2];
          }
          sum[n][k] = fmaf(sum[n][k], shrink[n][k], add);
        }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int m = 0; m < DP / 16; ++m) {
            o[n][m][0] *= shrink[n][0]; o[n][m][1] *= shrink[n][1]; o[n][m][2] *= shrink[n][0]; o[n][m][3] *= shrink[n][1];
          }
      }
      uint32_t wf[TERMS][TILES][NT][2];                                          // weights as operands: rows tokens, columns queries
#pragma unroll
      for (uint32_t l = 0; l < TILES; ++l)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float vs = v_scale[16 * l + g + 8 * r];
            const uint32_t bit = 4 * (l * NT + n) + 2 * r;
            float w0 = x[l][n][2 * r] * vs, w1 = x[l][n][2 * r + 1] * vs;
            if (!every) {                                                        // not zero times a poisoned scale
              if (!(seen >> bit & 1u)) w0 = 0.f;
              if (!(seen >> (bit + 1) & 1u)) w1 = 0.f;
            }
            const uint32_t h = pack_half(w0, w1);
            wf[0][l][n][r] = transpose8x8(h);
            if (TERMS == 2) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
              wf[TERMS - 1][l][n][r] = transpose8x8(pack_half(w0 - f.x, w1 - f.y));
            }
          }

      // ---- values: rows are elements (this lane's DP / 8 neighbouring ones, two by two), columns queries
      const uint8_t* v0 = mine + place + TOK * F::KS + 2 * t * F::VS + g * (F::RB / 8);
      auto product = [&](uint32_t l, int m, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, float (&into)[NT][4]) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int term = TERMS - 1; term >= 0; --term)
            mma16816(TERMS == 2 ? into[n] : o[n][m], a0, a1, a2, a3, wf[term][l][n][0], wf[term][l][n][1]);
      };
      constexpr uint32_t WORDS = F::RB / 32;                                     // words of a row that are this lane's
      constexpr int PER_WORD = MX ? 4 : 2;                                       // products of a word
      uint32_t code[TILES][4][WORDS];                                            // of tokens 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
      for (uint32_t l = 0; l < TILES; ++l)
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) load_words<WORDS>(code[l][i], v0 + (16 * l + (i & 1) + 8 * (i >> 1)) * F::VS);
#pragma unroll
      for (uint32_t w = 0; w < WORDS; ++w) {
        float fresh[PER_WORD][NT][4];                                            // TERMS = 2: sums of this stage alone, added in binary32 below
        if (TERMS == 2)
#pragma unroll
          for (int m = 0; m < PER_WORD; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int i = 0; i < 4; ++i) fresh[m][n][i] = 0.f;
#pragma unroll
        for (uint32_t l = 0; l < TILES; ++l) {
          const uint32_t wa = code[l][0][w], wb = code[l][1][w], wc = code[l][2][w], wd = code[l][3][w];
          if (MX) {
            const uint32_t block = g * NB / 8;
            const uint32_t f0 = *reinterpret_cast<const uint32_t*>(v_factor + block * TOK + 16 * l + 2 * t);
            const uint32_t f1 = *reinterpret_cast<const uint32_t*>(v_factor + block * TOK + 16 * l + 2 * t + 8);
            constexpr uint32_t LOW = 0x0f0f0f0fu;
            uint32_t e0[4], d0[4], e1[4], d1[4];                                 // even and odd elements, two tokens to a pair
            four_bits((wa & LOW) | ((wb & LOW) << 4), e0);
            four_bits(((wa >> 4) & LOW) | (wb & ~LOW), d0);
            four_bits((wc & LOW) | ((wd & LOW) << 4), e1);
            four_bits(((wc >> 4) & LOW) | (wd & ~LOW), d1);
#pragma unroll
            for (int m = 0; m < 4; ++m) product(l, 4 * w + m, half_mul(e0[m], f0), half_mul(d0[m], f0), half_mul(e1[m], f1), half_mul(d1[m], f1), fresh[m % PER_WORD]);
          } else {
            const uint32_t xa = wa ^ 0x80808080u, xb = wb ^ 0x80808080u, xc = wc ^ 0x80808080u, xd = wd ^ 0x80808080u;
            const uint32_t ab0 = __byte_perm(xa, xb, 0x5140), ab1 = __byte_perm(xa, xb, 0x7362), cd0 = __byte_perm(xc, xd, 0x5140), cd1 = __byte_perm(xc, xd, 0x7362);
            product(l, 2 * w, eight_bits<0x4140>(ab0), eight_bits<0x4342>(ab0), eight_bits<0x4140>(cd0), eight_bits<0x4342>(cd0), fresh[0]);
            product(l, 2 * w + 1, eight_bits<0x4140>(ab1), eight_bits<0x4342>(ab1), eight_bits<0x4140>(cd1), eight_bits<0x4342>(cd1), fresh[1]);
          }
        }
        if (TERMS == 2)
#pragma unroll
          for (int m = 0; m < PER_WORD; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[n][PER_WORD * w + m][i] += fresh[m][n][i];
      }
      __syncwarp();
      fetch(k + kDepth, id);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");

    // ---- the warps' results meet in shared memory
    __syncthreads();
    float* const o_all = reinterpret_cast<float*>(smem);                          // [warp][row][DP]
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float total = sum[n][k];
#pragma unroll
        for (int b = 4; b < 32; b <<= 1) total += __shfl_xor_sync(0xffffffffu, total, b);
        const uint32_t r = 8 * n + 2 * t + k;
        if (g == 0) top_sum[warp][r] = make_float2(top_x[n][k], total);
        float* to = o_all + (warp * ROWS + r) * DP + g * (DP / 8);
        const float f0 = power_of_two(-kWeightBits - (MX ? kFactorBits : 0)), f1 = power_of_two(v_top);
#pragma unroll
        for (int m = 0; m < DP / 16; ++m) *reinterpret_cast<float2*>(to + 2 * m) = make_float2(o[n][m][k] * f0 * f1, o[n][m][k + 2] * f0 * f1);
      }
    __syncthreads();
    const bool whole = unit0 == 0 && unit1 == units;
    const uint32_t place = unit0 == 0 ? 1 : 0;
    float* const to_part = p.parts + ((uint64_t)blockIdx.x * 2 + place) * p.hw * F::PIECE;
    if (!whole && place == 1 && tid == 0) {
      // the item's last unit is among those of CTA c where c * all / ctas <= last < (c + 1) * all / ctas
      const uint64_t last = at_unit - x0 + cost - 1;
      uint32_t c = (uint32_t)(last * ctas / all);
      while (all * c / ctas > last) --c;
      while (all * (c + 1) / ctas <= last) ++c;
      AttendPiece h;
      h.followers = c - blockIdx.x; h.row0 = s.row0; h.rows = rows; h.tile = tile; h.heads = hg;
      p.pieces[blockIdx.x] = h;
    }
    const uint32_t n_rows = row1 - row0, quads = DP / 4;
    for (uint32_t i = tid; i < p.hw * n_rows * quads; i += kThreads) {
      const uint32_t d = 4 * (i % quads), r = i / quads % n_rows, h = i / quads / n_rows;
      float top = -INFINITY, total = 0.f;
      for (uint32_t w = h; w < kWarps; w += p.hw) top = fmaxf(top, top_sum[w][r].x);
      const float from = top == -INFINITY ? 0.f : top;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (uint32_t w = h; w < kWarps; w += p.hw) {
        const float2 ts = top_sum[w][r];
        const float f = exp2_fast(ts.x - from);
        const float4 ov = *reinterpret_cast<const float4*>(o_all + (w * ROWS + r) * DP + d);
        total = fmaf(ts.y, f, total);
        v.x = fmaf(ov.x, f, v.x); v.y = fmaf(ov.y, f, v.y); v.z = fmaf(ov.z, f, v.z); v.w = fmaf(ov.w, f, v.w);
      }
      if (whole) attend_store(a, s.row0, row0 + r, p.group, (hg << p.hw_log) + h, d, v, top, total, p.vec_out);
      else {
        *reinterpret_cast<float4*>(to_part + (h * ROWS + r) * DP + d) = v;
        if (d == 0) *reinterpret_cast<float2*>(to_part + p.hw * ROWS * DP + 2 * (h * ROWS + r)) = make_float2(top, total);
      }
    }
    __syncthreads();
    at_unit += x1 - x0;
  }
}

// Adds up the items that were cut.  Their rows of results (query row, key head) stand in one row of all of them and are dealt out to the warps of
// all CTAs, several warps to a row when there are few: those share its pieces and meet in shared memory.  (CTA c for what main CTA c began left one
// sequence of 32000 tokens, 8 key heads and 8 rows to 8 CTAs: 77 us with the main kernel.)
constexpr uint32_t kJoinThreads = 256, kJoinMost = kJoinThreads;      // main CTAs at most: a thread for each
template <uint32_t K>                                         // float4 of a row to a lane
__global__ void __launch_bounds__(kJoinThreads)
attend_join_kernel(const AttendArgs a, FastDiv group, const float* parts, const AttendPiece* pieces, uint32_t ctas, uint32_t hw_log, uint32_t tile_rows, uint32_t dp,
                   uint32_t vec_out) {
  constexpr uint32_t WARPS = kJoinThreads / 32, HELD = 8;      // pieces in flight
  __shared__ float4 sums[WARPS][32 * K];
  __shared__ float2 top_sum[WARPS];
  __shared__ uint32_t begin[kJoinMost], scan[WARPS];
  dependency_wait();
  allow_dependents();
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, quads = dp / 4;
  // rows of what each main CTA began and did not end, and their running sum
  uint32_t sum = 0;
  if (tid < ctas) {
    const AttendPiece h = pieces[tid];
    if (h.followers) sum = min(tile_rows, h.rows - h.tile * tile_rows) << hw_log;
  }
  uint32_t upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
  if (lane == 31) scan[warp] = upto;
  __syncthreads();
  uint32_t all = 0, before = upto - sum;
#pragma unroll
  for (uint32_t w = 0; w < WARPS; ++w) { if (w < warp) before += scan[w]; all += scan[w]; }
  begin[tid] = before;
  __syncthreads();
  const uint64_t piece = (uint64_t)(tile_rows << hw_log) * (dp + 2);
  uint32_t share = WARPS;                                    // warps of a row: a power of two
  while (share > 1 && gridDim.x * (WARPS / share) < all) share /= 2;
  const uint32_t sub = warp & (share - 1), step = gridDim.x * (WARPS / share);
  for (uint32_t i0 = blockIdx.x; i0 < all; i0 += step) {
    const uint32_t i = i0 + gridDim.x * (warp / share);
    const bool there = i < all;
    float top = -INFINITY, total = 0.f;
    float4 v[K] = {};
    AttendPiece h = {};
    uint32_t r = 0, head = 0;
    if (there) {
      uint32_t c = 0, end = ctas;                            // the last one that begins at i or before (those without rows begin where the next one does)
      while (end - c > 1) {
        const uint32_t mid = (c + end) / 2;
        if (begin[mid] <= i) c = mid; else end = mid;
      }
      h = pieces[c];
      const uint32_t in = i - begin[c];
      r = in >> hw_log; head = in & ((1u << hw_log) - 1);
      const uint32_t at = head * tile_rows + r;
#pragma unroll 1
      for (uint32_t f0 = sub; f0 <= h.followers; f0 += HELD * share) {
        float2 ts[HELD];
        float4 x[HELD][K];
#pragma unroll
        for (uint32_t b = 0; b < HELD; ++b) {                // (loads without branches: past the end the last piece, past the row its last elements)
          const uint32_t f = min(f0 + b * share, h.followers);
          const float* from = parts + ((uint64_t)(c + f) * 2 + (f == 0 ? 1 : 0)) * piece;
          ts[b] = *reinterpret_cast<const float2*>(from + (tile_rows << hw_log) * dp + 2 * at);
#pragma unroll
          for (uint32_t k = 0; k < K; ++k) x[b][k] = *reinterpret_cast<const float4*>(from + at * dp + 4 * min(lane + 32 * k, quads - 1));
        }
        float high = top;
#pragma unroll
        for (uint32_t b = 0; b < HELD; ++b) {
          if (f0 + b * share > h.followers) {
            ts[b] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (uint32_t k = 0; k < K; ++k) x[b][k] = make_float4(0.f, 0.f, 0.f, 0.f);
          }
          high = fmaxf(high, ts[b].x);
        }
        const float base = high == -INFINITY ? 0.f : high, was = exp2_fast(top - base);
        top = high;
        total *= was;
#pragma unroll
        for (uint32_t k = 0; k < K; ++k) { v[k].x *= was; v[k].y *= was; v[k].z *= was; v[k].w *= was; }
#pragma unroll
        for (uint32_t b = 0; b < HELD; ++b) {
          const float is = exp2_fast(ts[b].x - base);
          total = fmaf(ts[b].y, is, total);
#pragma unroll
          for (uint32_t k = 0; k < K; ++k) {
            v[k].x = fmaf(x[b][k].x, is, v[k].x); v[k].y = fmaf(x[b][k].y, is, v[k].y); v[k].z = fmaf(x[b][k].z, is, v[k].z); v[k].w = fmaf(x[b][k].w, is, v[k].w);
          }
        }
      }
    }
    if (share > 1) {                                         // (the same in all threads)
#pragma unroll
      for (uint32_t k = 0; k < K; ++k) sums[warp][lane + 32 * k] = v[k];
      if (lane == 0) top_sum[warp] = make_float2(top, total);
      __syncthreads();
      if (there && sub == 0) {
        top = -INFINITY; total = 0.f;
        for (uint32_t w = 0; w < share; ++w) top = fmaxf(top, top_sum[warp + w].x);
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (uint32_t k = 0; k < K; ++k) v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (uint32_t w = 0; w < share; ++w) {
          const float f = exp2_fast(top_sum[warp + w].x - base);
          total = fmaf(top_sum[warp + w].y, f, total);
#pragma unroll
          for (uint32_t k = 0; k < K; ++k) {
            const float4 x = sums[warp + w][lane + 32 * k];
            v[k].x = fmaf(x.x, f, v[k].x); v[k].y = fmaf(x.y, f, v[k].y); v[k].z = fmaf(x.z, f, v[k].z); v[k].w = fmaf(x.w, f, v[k].w);
          }
        }
      }
      __syncthreads();
    }
    if (there && sub == 0)
#pragma unroll
      for (uint32_t k = 0; k < K; ++k)
        if (lane + 32 * k < quads) attend_store(a, h.row0, h.tile * tile_rows + r, group, (h.heads << hw_log) + head, 4 * (lane + 32 * k), v[k], top, total, vec_out);
  }
}

// The same where an item has many rows and few pieces: a warp adds up a row.
__global__ void __launch_bounds__(kJoinThreads)
attend_join_rows_kernel(const AttendArgs a, FastDiv group, const float* parts, const AttendPiece* pieces, uint32_t tile_rows, uint32_t dp, uint32_t vec_out) {
  dependency_wait();
  allow_dependents();
  const AttendPiece h = pieces[blockIdx.x];
  if (h.followers == 0) return;
  const uint32_t lane = threadIdx.x % 32, quads = dp / 4, n_rows = min(tile_rows, h.rows - h.tile * tile_rows);
  const uint64_t piece = (uint64_t)tile_rows * (dp + 2);
  for (uint32_t r = blockIdx.y * (kJoinThreads / 32) + threadIdx.x / 32; r < n_rows; r += gridDim.y * (kJoinThreads / 32)) {
    float top = -INFINITY, total = 0.f;
    float4 v[2] = {};
#pragma unroll 2
    for (uint32_t f = 0; f <= h.followers; ++f) {
      const float* from = parts + ((uint64_t)(blockIdx.x + f) * 2 + (f == 0 ? 1 : 0)) * piece;
      const float2 ts = *reinterpret_cast<const float2*>(from + tile_rows * dp + 2 * r);
      const float m = fmaxf(top, ts.x), base = m == -INFINITY ? 0.f : m, was = exp2_fast(top - base), is = exp2_fast(ts.x - base);
      top = m;
      total = total * was + ts.y * is;
#pragma unroll
      for (uint32_t k = 0; k < 2; ++k)
        if (lane + 32 * k < quads) {
          const float4 x = *reinterpret_cast<const float4*>(from + (uint64_t)r * dp + 4 * (lane + 32 * k));
          v[k].x = v[k].x * was + x.x * is; v[k].y = v[k].y * was + x.y * is; v[k].z = v[k].z * was + x.z * is; v[k].w = v[k].w * was + x.w * is;
        }
    }
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k)
      if (lane + 32 * k < quads) attend_store(a, h.row0, h.tile * tile_rows + r, group, h.heads, 4 * (lane + 32 * k), v[k], top, total, vec_out);
  }
}

constexpr int kDevices = 64;

template <class F>
cudaError_t launch_rows(const Launch& l, RowsArgs p, const AttendRun& run, uint64_t* launches) {
  static bool allowed[kDevices] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= kDevices || !allowed[dev]) {
    e = cudaFuncSetAttribute(attend_rows_kernel<F>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::SMEM);
    if (e != cudaSuccess) return e;
    if (dev < kDevices) allowed[dev] = true;
  }
  p.parts = reinterpret_cast<float*>(run.scratch);
  p.pieces = reinterpret_cast<AttendPiece*>(run.scratch + attend_parts_bytes(run.ctas, p.hw, F::ROWS, F::DP));
  e = launch_grid(l, attend_rows_kernel<F>, dim3(run.ctas), F::THREADS, F::SMEM, p);
  if (e != cudaSuccess) return e;
  ++*launches;
  return launch_attend_join(l, p.a, p.parts, p.pieces, run.ctas, p.hw_log, F::ROWS, F::DP, launches);
}

template <int FORMAT, int DP>
cudaError_t launch_format(const Launch& l, const RowsArgs& p, const AttendRun& run, uint64_t* launches) {
  if (run.terms == 2) {
    if constexpr (DP <= 128) if (run.rows == 16) return launch_rows<Form<FORMAT, DP, 2, 2>>(l, p, run, launches);
    return launch_rows<Form<FORMAT, DP, 1, 2>>(l, p, run, launches);
  }
  if constexpr (DP <= 128) if (run.rows == 16) return launch_rows<Form<FORMAT, DP, 2, 1>>(l, p, run, launches);
  return launch_rows<Form<FORMAT, DP, 1, 1>>(l, p, run, launches);
}

template <int FORMAT>
cudaError_t launch_dim(const Launch& l, const RowsArgs& p, const AttendRun& run, uint64_t* launches) {
  if (run.dp == 64) return launch_format<FORMAT, 64>(l, p, run, launches);
  if (run.dp == 128) return launch_format<FORMAT, 128>(l, p, run, launches);
  return launch_format<FORMAT, 256>(l, p, run, launches);
}

}  // namespace

cudaError_t launch_attend_join(const Launch& l, const AttendArgs& a, const float* parts, const AttendPiece* pieces, uint32_t ctas, uint32_t hw_log, uint32_t tile_rows,
                               uint32_t dp, uint64_t* launches) {
  const FastDiv group(a.group);
  const uint32_t vec = attend_vec_out(a);
  cudaError_t e;
  if (tile_rows >= 128) e = launch_grid(l, attend_join_rows_kernel, dim3(ctas, 8), kJoinThreads, 0, a, group, parts, pieces, tile_rows, dp, vec);
  else if (dp <= 128) e = launch_grid(l, attend_join_kernel<1>, dim3(2 * ctas), kJoinThreads, 0, a, group, parts, pieces, ctas, hw_log, tile_rows, dp, vec);
  else e = launch_grid(l, attend_join_kernel<2>, dim3(2 * ctas), kJoinThreads, 0, a, group, parts, pieces, ctas, hw_log, tile_rows, dp, vec);
  if (e == cudaSuccess) ++*launches;
  return e;
}

// Which forms a call takes, and the scratch that it needs.
AttendRun plan_kv_attend(const AttendArgs& a, int sm_count) {
  AttendRun r = {};
  r.dp = a.c.dim <= 64 ? 64 : a.c.dim <= 128 ? 128 : 256;
  r.terms = a.dtype == kF32 ? 2 : 1;
  const uint64_t most = (uint64_t)a.max_new * a.group;             // query rows of a sequence and key head
  // Sequences of more than 32 rows go to the tensor cores' tiles of 128 rows, which binary32 has no operands for.  (32 sequences of 2000 tokens, 8 key heads of
  // 128, 4 bits, 32 rows each: 85 us here, 106 there; 64 rows: 147 and 109; 8 bits: 104 and 162, 179 and 166.)
  r.few = r.terms == 2 || most <= 32 ? 0xffffffffu : a.seqs == 1 ? 0 : 32;
  // Sixteen rows to an item where sequences have more than eight (drafts), or a single token has (16 rows as above: 56 us beside 57, 8 bits 68 and 74; 8 rows,
  // half of the sixteen empty: 48 beside 38).  Where long chunks are mixed with single tokens, the latter get eight.
  r.rows = r.dp <= 128 && most > 8 && (most <= 32 || r.terms == 2 || a.group > 8) ? 16 : 8;
  r.hw_log = 0;
  while (r.hw_log < 3 && a.c.heads % (2u << r.hw_log) == 0) ++r.hw_log;
  // A CTA per SM, fewer where there cannot be a unit of 16 tokens for each
  const uint64_t tiles = (uint64_t)a.total * a.group / r.rows + a.seqs, units = tiles * (a.c.heads >> r.hw_log) * (a.room / 16 + 1);
  const uint64_t ctas = (uint64_t)(sm_count < (int)kJoinMost ? sm_count : (int)kJoinMost);
  r.ctas = (uint32_t)(units < ctas ? units : ctas);
  uint64_t most_bytes = r.few == 0 ? 0 : attend_parts_bytes(r.ctas, 1u << r.hw_log, r.rows, r.dp) + r.ctas * sizeof(AttendPiece);
  if (r.few != 0xffffffffu) {
    const uint64_t many = ((uint64_t)a.total * a.group / chunk_rows(r.dp) + a.seqs) * a.c.heads * (a.room / 64 + 1);
    r.chunk_ctas = (uint32_t)(many < ctas ? many : ctas);
    const uint64_t bytes = attend_parts_bytes(r.chunk_ctas, 1, chunk_rows(r.dp), r.dp) + r.chunk_ctas * sizeof(AttendPiece);
    if (bytes > most_bytes) most_bytes = bytes;
  }
  r.scratch_bytes = most_bytes;
  return r;
}

cudaError_t launch_kv_attend(const Launch& l, const AttendArgs& a, const AttendRun& run, uint64_t* launches) {
  if (run.few != 0) {
    RowsArgs p;
    p.a = a; p.page = FastDiv(a.c.page_size); p.group = FastDiv(a.group);
    p.hw = 1u << run.hw_log; p.hw_log = run.hw_log; p.row_limit = run.few;
    p.vec_codes = a.c.dim % 16 == 0 && ((uintptr_t)a.c.codes[0] | (uintptr_t)a.c.codes[1]) % 16 == 0;
    const uint32_t blocks = (a.c.dim + 31) / 32;
    const bool mx = a.c.format == QV2_KV_MX4;
    p.token_codes = a.c.heads * (mx ? 16 * blocks : a.c.dim); p.token_scales = a.c.heads * (mx ? blocks : 4);
    p.quick = (mx || p.vec_codes) && (!mx || blocks % 4 == 0) && ((uintptr_t)a.c.scales[0] | (uintptr_t)a.c.scales[1]) % 4 == 0;
    p.vec_q = a.c.dim % 8 == 0 && ((uintptr_t)a.q | a.q_token_ld * dtype_size(a.dtype) | a.q_head_ld * dtype_size(a.dtype)) % 16 == 0;
    p.vec_out = attend_vec_out(a);
    cudaError_t e = a.c.format == QV2_KV_MX4 ? launch_dim<QV2_KV_MX4>(l, p, run, launches) : launch_dim<QV2_KV_I8>(l, p, run, launches);
    if (e != cudaSuccess || run.few == 0xffffffffu) return e;
  }
  return launch_attend_chunk(l, a, run, launches);
}

}  // namespace qv2
