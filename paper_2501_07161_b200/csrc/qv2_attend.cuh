// What the two forms of the attention share: sequences, the cutting of the work over the CTAs, partial results.
#pragma once

#include <type_traits>

#include "qv2_mx.cuh"

namespace qv2 {

struct AttendArgs {
  KvView c;
  const void* q;
  uint64_t q_token_ld, q_head_ld;
  uint32_t q_heads, group, total, seqs;
  const int64_t *starts, *lens;
  const int32_t* table;
  uint64_t table_ld;
  uint32_t room;                  // tokens that a row of the table has pages for; 0: the cache has no pages
  float scale, cap;
  int32_t window;                 // 2^31 - 1: none
  const float* slopes;
  void* out;
  float* lse;
  uint32_t dtype, max_new;
};

// Sequence s of a call: its rows of q, and its length, which is held to 2^31 - 1.
struct AttendSeq {
  uint32_t row0, n;
  int32_t len;
};
__device__ __forceinline__ AttendSeq attend_seq(const AttendArgs& a, uint32_t s) {
  const int64_t total = a.total, lo = min(max(__ldg(a.starts + s), (int64_t)0), total), hi = min(max(__ldg(a.starts + s + 1), lo), total);
  AttendSeq r;
  r.row0 = (uint32_t)lo;
  r.n = (uint32_t)(hi - lo);
  r.len = (int32_t)min(max(__ldg(a.lens + s), (int64_t)0), (int64_t)0x7fffffff);
  return r;
}

// The work of a call is cut evenly however ragged its sequences are.  An item is a tile of query rows of one sequence with one
// group of key heads; it takes as many units (runs of tokens) as its sequence's other items.  All units of all items stand
// in one row, and CTA c of C takes those from c*T/C to (c+1)*T/C: the end of one item, whole items, the beginning
// of another.  What is not whole goes to scratch: at most one piece that continues an item (place 0) and one that begins one
// (place 1).  A second kernel adds up each item that was cut, in the order of its tokens; the CTA that began it says so here.
struct AttendPiece {
  uint32_t followers;             // CTAs after this one that hold more of the item that it began; 0: it began none that is cut
  uint32_t row0, rows;            // the item's sequence: first row of q, rows (query, head of the group) in all
  uint32_t tile, heads;           // which tile of those, which group of key heads
};

// Where unit u of the row of all units lies.
struct AttendUnits {
  uint64_t before;                // units of the sequences before this one
  uint32_t seq;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }     // -126..127
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) { const __half2 h = __floats2half2_rn(lo, hi); return *reinterpret_cast<const uint32_t*>(&h); }
__device__ __forceinline__ uint32_t half_mul(uint32_t a, uint32_t b) {
  const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The four pairs of numbers of a word of 4-bit codes, as they lie.
__device__ __forceinline__ void four_bits(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 c0, c1, c2, c3;\n\t"
      "mov.b32 {c0, c1, c2, c3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, c0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, c1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, c3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// Bytes S and T of w, which are 8-bit integers plus 128, as a pair: 0x6400 + byte is the number 1024 + byte in binary16.
template <uint32_t SELECT>
__device__ __forceinline__ uint32_t eight_bits(uint32_t w) {
  const uint32_t biased = __byte_perm(w, 0x64646464u, SELECT);
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&biased), __half2half2(__ushort_as_half((unsigned short)0x6480)));
  return *reinterpret_cast<const uint32_t*>(&h);
}

// cap * tanh(x / cap) for results of 16 bits: tanh(y) = 1 - 2 / (1 + e^2y), off by some 2^-23 of cap.
__device__ __forceinline__ float capped_fast(float x, float cap) {
  return cap - __fdividef(2.f * cap, 1.f + exp2_fast(2.f * kLog2e * __fdividef(x, cap)));
}

// Elements d .. d + 3 of the result of query row r (of a sequence and key head), from sums of which the largest score, to powers of two, is `top`.
__device__ __forceinline__ void attend_store(const AttendArgs& a, uint32_t q_row0, uint32_t r, const FastDiv& group, uint32_t kv, uint32_t d, float4 v,
                                             float top, float total, bool vec) {
  const uint32_t i = group.div(r);
  const uint64_t at = (uint64_t)(q_row0 + i) * a.q_heads + kv * group.d + (r - i * group.d);
  const float f = total == 0.f ? 0.f : 1.f / total;                // nothing seen: zeros
  const float y[4] = {v.x * f, v.y * f, v.z * f, v.w * f};
  if (a.lse && d == 0) a.lse[at] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
  auto store = [&](auto* out) {
    using T = typename std::remove_pointer<decltype(out)>::type;
    T* to = out + at * a.c.dim + d;
    if (vec) {
      if (d >= a.c.dim) return;
      if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to) = make_float4(y[0], y[1], y[2], y[3]);
      else *reinterpret_cast<uint2*>(to) = make_uint2(Chunk8<T>::pack(y[0], y[1]), Chunk8<T>::pack(y[2], y[3]));
    } else {
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k)
        if (d + k < a.c.dim) to[k] = Chunk8<T>::narrow(y[k]);
    }
  };
  if (a.dtype == kBF16) store((__nv_bfloat16*)a.out);
  else if (a.dtype == kF16) store((__half*)a.out);
  else store((float*)a.out);
}

// The form of a call, and its scratch: partial results, then an AttendPiece per CTA.
struct AttendRun {
  uint32_t dp, terms, rows, hw_log, ctas;      // the form for few rows
  uint32_t few;                                // sequences of more query rows (per key head) take the other form; 2^32 - 1: none does, 0: all do
  uint32_t chunk_ctas;
  uint64_t scratch_bytes;
  uint8_t* scratch;
  uint32_t* fault;                             // host-mapped word, set when a kernel gave up waiting
};
AttendRun plan_kv_attend(const AttendArgs& a, int sm_count);
constexpr uint32_t chunk_rows(uint32_t dp) { return dp == 256 ? 128 : 256; }      // query rows of an item of the form for many
cudaError_t launch_attend_chunk(const Launch& l, const AttendArgs& a, const AttendRun& run, uint64_t* launches);
// Adds up what was cut: parts as a form left them, hw key heads (a power of two) and tile_rows query rows to an item.
cudaError_t launch_attend_join(const Launch& l, const AttendArgs& a, const float* parts, const AttendPiece* pieces, uint32_t ctas, uint32_t hw_log, uint32_t tile_rows,
                               uint32_t dp, uint64_t* launches);
inline uint32_t attend_vec_out(const AttendArgs& a) { return a.c.dim % 4 == 0 && (uintptr_t)a.out % (4 * dtype_size(a.dtype)) == 0; }
inline uint64_t attend_parts_bytes(uint32_t ctas, uint32_t hw, uint32_t tile_rows, uint32_t dp) { return (uint64_t)ctas * 2 * hw * tile_rows * (dp + 2) * sizeof(float); }
cudaError_t launch_kv_attend(const Launch& l, const AttendArgs& a, const AttendRun& run, uint64_t* launches);

}  // namespace qv2
