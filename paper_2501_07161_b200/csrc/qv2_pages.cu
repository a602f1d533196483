// Pages, positions and slots of a step's new tokens from the lengths of its requests.
//
// Everything is a running sum over the sequences (new tokens, new pages, tokens in all).  Each CTA makes that sum for itself,
// 1024 sequences at a time, and then serves its own part of the tokens and pages by searching it, so that one launch does it
// all and no CTA waits for another.  The arrays that may be an input and an output at once are written by the CTA that
// arrives last, when all have read them.
//
// Bound by latency.  64 sequences with a token each: 15 us a call, nearly all of it the host's.  1500 sequences with up to 700 new
// tokens (9 MB, 1.4 us at the copy rate) take 23 to 26 us: the running sums over two rounds of 1024 sequences, then a search of ten steps and a chain of
// look-ups for each token, four tokens of a thread at a time so that their steps overlap.
#include "qv2_serve.cuh"

namespace qv2 {

namespace {

constexpr uint32_t kPlanThreads = 256, kPlanSeqs = 4 * kPlanThreads;

// Largest i < n with sums[i] <= x; sums[0] is 0 and x is not negative.
__device__ __forceinline__ uint32_t last_at_most(const int64_t* sums, uint32_t n, int64_t x) {
  uint32_t a = 0, b = n;
  while (b - a > 1) {
    const uint32_t mid = (a + b) / 2;
    if (sums[mid] <= x) a = mid; else b = mid;
  }
  return a;
}

__device__ __forceinline__ int64_t held_to(int64_t v) { return min(max(v, (int64_t)0), (int64_t)1 << 40); }

__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(qv2_page_plan p, FastDiv page, uint32_t* ticket) {
  __shared__ int64_t tok[kPlanSeqs], pag[kPlanSeqs], held[kPlanSeqs];
  __shared__ int64_t part[3][kPlanThreads / 32];
  __shared__ uint32_t last;
  dependency_wait();
  allow_dependents();
  const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const int64_t count = min(max(*(volatile const int64_t*)p.free_count, (int64_t)0), (int64_t)p.free_size);
  const int64_t span = (int64_t)page.d * (int64_t)p.width;           // tokens that a row of the table has pages for, below 2^31
  auto pages_of = [&](int64_t tokens) { return tokens >= span ? (int64_t)p.width : (int64_t)page.div((uint32_t)tokens + page.d - 1); };
  auto page_number = [&](int64_t taken) { return taken < count ? __ldg(p.free_pages + (count - 1 - taken)) : -1; };
  const uint64_t per = (p.total + gridDim.x - 1) / gridDim.x;
  const int64_t t_begin = (int64_t)min(p.total, per * blockIdx.x), t_end = (int64_t)min(p.total, per * (blockIdx.x + 1));
  int64_t tok0 = 0, pag0 = 0, all0 = 0;                              // sums over the sequences before this round's
  for (uint32_t base = 0; base < p.seqs; base += kPlanSeqs) {
    const uint32_t n = min(kPlanSeqs, p.seqs - base);
    int64_t h[4], v[3][4], sum[3] = {0, 0, 0};
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      const uint32_t i = 4 * tid + k;
      int64_t more = 0;
      h[k] = 0;
      if (i < n) {
        h[k] = held_to(((volatile const int64_t*)p.lens)[base + i]);
        more = held_to(__ldg(p.fresh + base + i));
      }
      const int64_t now[3] = {more, pages_of(h[k] + more) - pages_of(h[k]), h[k] + more};
#pragma unroll
      for (int a = 0; a < 3; ++a) { v[a][k] = sum[a]; sum[a] += now[a]; }
    }
    int64_t before[3];
#pragma unroll
    for (int a = 0; a < 3; ++a) {
      int64_t s = sum[a];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int64_t u = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += u; }
      before[a] = s - sum[a];
      if (lane == 31) part[a][warp] = s;
    }
    __syncthreads();
    int64_t whole[3] = {0, 0, 0};
#pragma unroll
    for (uint32_t w = 0; w < kPlanThreads / 32; ++w)
#pragma unroll
      for (int a = 0; a < 3; ++a) { if (w < warp) before[a] += part[a][w]; whole[a] += part[a][w]; }
    const bool mine = (base / kPlanSeqs) % gridDim.x == blockIdx.x;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) {
      const uint32_t i = 4 * tid + k;
      tok[i] = before[0] + v[0][k]; pag[i] = before[1] + v[1][k]; held[i] = h[k];
      if (mine && i < n) {
        p.q_starts[base + i] = tok0 + before[0] + v[0][k];
        p.starts[base + i] = all0 + before[2] + v[2][k];
      }
    }
    __syncthreads();
    // Four tokens of a thread at a time: a token is a chain of look-ups.
    const int64_t stop = min(t_end, tok0 + whole[0]);
    for (int64_t t0 = max(t_begin, tok0) + tid; t0 < stop; t0 += 4 * kPlanThreads) {
      uint32_t i[4], b[4];
      int64_t at[4], slot[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) { i[k] = 0; b[k] = n; }
      for (uint32_t wide = n; wide > 1; wide = (wide + 1) / 2) {                // as last_at_most
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t mid = (i[k] + b[k]) / 2;
          if (b[k] - i[k] > 1) { if (tok[mid] <= t0 + k * kPlanThreads - tok0) i[k] = mid; else b[k] = mid; }
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t t = t0 + k * kPlanThreads;
        at[k] = held[i[k]] + (t - tok0 - tok[i[k]]);
        slot[k] = -1;
        if (t < stop && at[k] < span) {
          const uint32_t pg = page.div((uint32_t)at[k]);
          const int64_t have = pages_of(held[i[k]]);
          const int32_t id = pg < have ? __ldg(p.table + (base + i[k]) * p.table_ld + pg) : page_number(pag0 + pag[i[k]] + pg - have);
          if (id >= 0) slot[k] = (int64_t)id * page.d + ((uint32_t)at[k] - pg * page.d);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t t = t0 + k * kPlanThreads;
        if (t < stop) { p.slots[t] = slot[k]; p.positions[t] = at[k]; }
      }
    }
    for (int64_t a = blockIdx.x * kPlanThreads + tid; a < whole[1]; a += gridDim.x * kPlanThreads) {
      const uint32_t i = last_at_most(pag, n, a);
      p.table[(base + i) * p.table_ld + pages_of(held[i]) + (a - pag[i])] = page_number(pag0 + a);
    }
    tok0 += whole[0]; pag0 += whole[1]; all0 += whole[2];
    __syncthreads();
  }
  for (int64_t t = max(t_begin, tok0) + tid; t < t_end; t += kPlanThreads) { p.slots[t] = -1; p.positions[t] = 0; }
  if (gridDim.x > 1) {
    __syncthreads();
    if (tid == 0) {
      __threadfence();
      last = atomicAdd(ticket, 1u) == gridDim.x - 1;
      if (last) *ticket = 0;
    }
    __syncthreads();
    if (!last) return;
  }
  for (uint32_t s = tid; s < p.seqs; s += kPlanThreads) p.lens_out[s] = held_to(((volatile const int64_t*)p.lens)[s]) + held_to(__ldg(p.fresh + s));
  if (tid == 0) {
    p.q_starts[p.seqs] = tok0;
    p.starts[p.seqs] = all0;
    *p.count_out = max(count - pag0, (int64_t)0);
    if (p.missing) *p.missing = max(pag0 - count, (int64_t)0);
  }
}

}  // namespace

cudaError_t launch_kv_plan(const Launch& l, const qv2_page_plan& p, uint32_t* ticket, uint64_t* launches) {
  // A CTA for every 1024 new tokens, one per SM at most.
  const uint64_t want = (p.total + 1023) / 1024;
  const uint32_t grid = (uint32_t)(want < 1 ? 1 : want < (uint64_t)l.sm_count ? want : l.sm_count);
  cudaError_t e = launch_kernel(l, kv_plan_kernel, grid, kPlanThreads, p, FastDiv(p.page_size), ticket);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace qv2
