// C-ABI layer of page planning, norm with rotation, and attention over the cache.
#include <cmath>

#include "qv2_attend.cuh"
#include "qv2_call.cuh"
#include "qv2_serve.cuh"

using namespace qv2;

namespace {

constexpr uint64_t kMaxStride = 1ull << 40, kMaxTokens = 1ull << 30;

int check_rows(const qv2_head_rows* h, int dtype, uint64_t tokens) {
  if (!h || h->heads == 0 || tokens == 0) return QV2_OK;
  if (h->heads > 65536) return QV2_ERR_SIZE;
  if (!h->x || !h->y) return QV2_ERR_NULL;
  if (((uintptr_t)h->x | (uintptr_t)h->y) % dtype_size((uint32_t)dtype) || (uintptr_t)h->weight % 4) return QV2_ERR_ALIGN;
  if (h->x_token_ld > kMaxStride || h->x_head_ld > kMaxStride || h->y_token_ld > kMaxStride || h->y_head_ld > kMaxStride) return QV2_ERR_SIZE;
  return QV2_OK;
}

}  // namespace

extern "C" int qv2_kv_plan(qv2_ctx* c, const qv2_page_plan* p) {
  if (!c || !p) return QV2_ERR_NULL;
  TraceRange range("qv2_kv_plan");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    if (p->page_size == 0) return QV2_ERR_ARG;
    if (p->seqs > QV2_PLAN_MAX_SEQS || p->width > (1ull << 31) || p->page_size * (p->width + 1) >= (1ull << 31) || p->table_ld > kMaxStride ||
        p->free_size > (1ull << 40) || p->total > (1ull << 40)) return QV2_ERR_SIZE;
    if (p->seqs > 1 && p->table_ld < p->width) return QV2_ERR_ARG;
    if (!p->q_starts || !p->starts || !p->free_count || !p->count_out || (p->total && (!p->slots || !p->positions))) return QV2_ERR_NULL;
    if (p->seqs && (!p->lens || !p->fresh || !p->lens_out || (p->width && !p->table))) return QV2_ERR_NULL;
    if (p->free_size && !p->free_pages) return QV2_ERR_NULL;
    if (((uintptr_t)p->lens | (uintptr_t)p->fresh | (uintptr_t)p->free_count | (uintptr_t)p->lens_out | (uintptr_t)p->q_starts | (uintptr_t)p->starts |
         (uintptr_t)p->slots | (uintptr_t)p->positions | (uintptr_t)p->count_out | (uintptr_t)p->missing) % 8 ||
        ((uintptr_t)p->table | (uintptr_t)p->free_pages) % 4) return QV2_ERR_ALIGN;
    int st = take_fault(c);
    if (st != QV2_OK) return st;
    DeviceGuard guard(c->device);
    QV2_CUDA(c, launch_kv_plan(launch_of(c), *p, c->d_plan_ticket, &c->launches));
    return QV2_OK;
  };
  return logged(c, "qv2_kv_plan", before, run());
}

extern "C" int qv2_norm_rotate(qv2_ctx* c, const qv2_head_rows* queries, const qv2_head_rows* keys, uint32_t type, uint32_t head_dim,
                               uint32_t rot, uint32_t order, float eps, uint64_t tokens, const int64_t* positions, const float* freqs) {
  if (!c) return QV2_ERR_NULL;
  TraceRange range("qv2_norm_rotate");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    const int dtype = dtype_of(type);
    if (dtype < 0 || order > QV2_ROTATE_PAIRS || head_dim == 0 || rot % 2 || rot > head_dim || !(eps >= 0.f) || std::isinf(eps)) return QV2_ERR_ARG;
    if (head_dim > QV2_SERVE_MAX_DIM || tokens > kMaxTokens) return QV2_ERR_SIZE;
    int st;
    if ((st = check_rows(queries, dtype, tokens)) != QV2_OK || (st = check_rows(keys, dtype, tokens)) != QV2_OK) return st;
    if (tokens && rot && (!positions || !freqs)) return QV2_ERR_NULL;
    if (tokens && rot && ((uintptr_t)positions % 8 || (uintptr_t)freqs % 4)) return QV2_ERR_ALIGN;
    if ((st = take_fault(c)) != QV2_OK) return st;
    HeadRows h = {};
    const qv2_head_rows* part[2] = {queries, keys};
    for (int a = 0; a < 2; ++a) {
      if (!part[a] || part[a]->heads == 0) continue;
      h.x[a] = part[a]->x; h.y[a] = part[a]->y; h.weight[a] = part[a]->weight; h.heads[a] = part[a]->heads;
      h.x_token_ld[a] = part[a]->x_token_ld; h.x_head_ld[a] = part[a]->x_head_ld;
      h.y_token_ld[a] = part[a]->y_token_ld; h.y_head_ld[a] = part[a]->y_head_ld;
    }
    if (tokens == 0 || h.heads[0] + h.heads[1] == 0) return QV2_OK;
    DeviceGuard guard(c->device);
    Rotation r;
    r.positions = positions; r.freqs = freqs; r.tokens = tokens; r.dtype = (uint32_t)dtype; r.dim = head_dim; r.rot = rot; r.pairs = order == QV2_ROTATE_PAIRS; r.eps = eps;
    QV2_CUDA(c, launch_norm_rotate(launch_of(c), h, r, &c->launches));
    return QV2_OK;
  };
  return logged(c, "qv2_norm_rotate", before, run());
}

extern "C" int qv2_kv_attend(qv2_ctx* c, const qv2_kv_cache* cache, const void* q, uint64_t q_token_ld, uint64_t q_head_ld, uint32_t q_heads,
                             uint32_t type, uint64_t total, const int64_t* q_starts, const int64_t* lens, uint32_t seqs, const int32_t* table,
                             uint64_t table_ld, const qv2_attend_cfg* cfg, void* out, float* lse) {
  if (!c || !cfg) return QV2_ERR_NULL;
  TraceRange range("qv2_kv_attend");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    const int dtype = dtype_of(type);
    int st = check_cache(cache);
    if (st != QV2_OK) return st;
    if (dtype < 0 || q_heads == 0 || q_heads % cache->heads || !std::isfinite(cfg->scale) || !(cfg->cap >= 0.f) || std::isinf(cfg->cap)) return QV2_ERR_ARG;
    if (cache->head_dim > QV2_SERVE_MAX_DIM || q_heads > 65536 || total > kMaxTokens || total * q_heads >= (1ull << 31) || seqs > 65536 ||
        table_ld >= (1ull << 31) || table_ld * cache->page_size >= (1ull << 31) || q_token_ld > kMaxStride || q_head_ld > kMaxStride) return QV2_ERR_SIZE;
    if (total && seqs && (!q || !out || !q_starts || !lens || (table_ld && !table))) return QV2_ERR_NULL;
    if (((uintptr_t)q | (uintptr_t)out) % dtype_size((uint32_t)dtype) || ((uintptr_t)q_starts | (uintptr_t)lens) % 8 ||
        ((uintptr_t)table | (uintptr_t)lse | (uintptr_t)cfg->slopes) % 4) return QV2_ERR_ALIGN;
    if ((st = take_fault(c)) != QV2_OK) return st;
    if (total == 0 || seqs == 0) return QV2_OK;
    DeviceGuard guard(c->device);
    AttendArgs a;
    a.c = view_of(cache);
    a.q = q; a.q_token_ld = q_token_ld; a.q_head_ld = q_head_ld; a.q_heads = q_heads; a.group = q_heads / cache->heads;
    a.total = (uint32_t)total; a.seqs = seqs; a.starts = q_starts; a.lens = lens; a.table = table; a.table_ld = table_ld;
    a.scale = cfg->scale; a.cap = cfg->cap; a.window = cfg->window && cfg->window < 0x7fffffffull ? (int32_t)cfg->window : 0x7fffffff;
    a.slopes = cfg->slopes; a.out = out; a.lse = lse; a.dtype = (uint32_t)dtype;
    a.max_new = cfg->max_new && cfg->max_new < total ? (uint32_t)cfg->max_new : (uint32_t)total;
    a.room = cache->pages ? (uint32_t)(table_ld * cache->page_size) : 0;
    AttendRun r = plan_kv_attend(a, c->sm_count);
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    QV2_CUDA(c, cudaStreamIsCapturing(c->stream, &capture));
    if ((st = grow_capturable(c, &c->d_attend, &c->cap_attend, r.scratch_bytes, capture != cudaStreamCaptureStatusNone, &c->attend_captured)) != QV2_OK) return st;
    r.scratch = c->d_attend; r.fault = c->d_fault;
    QV2_CUDA(c, launch_kv_attend(launch_of(c), a, r, &c->launches));
    return QV2_OK;
  };
  return logged(c, "qv2_kv_attend", before, run());
}
