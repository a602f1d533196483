// What the files that implement calls on 4-bit matrices and on the cache share: launch settings, element types, the report of
// a kernel that gave up waiting, checks of a cache.
#pragma once

#include "qv2_context.cuh"
#include "qv2_mx.cuh"

namespace qv2 {

inline Launch launch_of(const qv2_ctx* c) {
  Launch l; l.stream = c->stream; l.sm_count = c->sm_count; l.pdl = c->dependent_launch;
  return l;
}

// Element type of a flag word, or -1.
inline int dtype_of(uint32_t type) {
  return type == QV2_IN_F32 ? (int)kF32 : type == QV2_IN_F16 ? (int)kF16 : type == QV2_IN_BF16 ? (int)kBF16 : -1;
}

// Whether a kernel of an earlier call gave up waiting; asking clears it.  Every call asks once its arguments are in order, so
// that what a failed product left behind is not taken further unnoticed.
inline int take_fault(qv2_ctx* c) {
  if (!*(volatile uint32_t*)c->h_fault) return QV2_OK;
  *(volatile uint32_t*)c->h_fault = 0;
  return QV2_ERR_TIMEOUT;
}

inline int check_cache(const qv2_kv_cache* k) {
  if (!k) return QV2_ERR_NULL;
  if (k->format > QV2_KV_I8 || k->page_size == 0 || k->heads == 0 || k->head_dim == 0) return QV2_ERR_ARG;
  if (k->head_dim > 4096 || k->heads > 65536 || k->pages > 0x7fffffffull) return QV2_ERR_SIZE;
  if (k->pages == 0) return QV2_OK;
  if (!k->k_codes || !k->k_scales || !k->v_codes || !k->v_scales) return QV2_ERR_NULL;
  if (k->format == QV2_KV_MX4 && (((uintptr_t)k->k_codes | (uintptr_t)k->v_codes) & 15u)) return QV2_ERR_ALIGN;
  if (k->format == QV2_KV_I8 && (((uintptr_t)k->k_scales | (uintptr_t)k->v_scales) & 3u)) return QV2_ERR_ALIGN;
  return QV2_OK;
}

inline KvView view_of(const qv2_kv_cache* k) {
  KvView v;
  v.codes[0] = (uint8_t*)k->k_codes; v.codes[1] = (uint8_t*)k->v_codes;
  v.scales[0] = (uint8_t*)k->k_scales; v.scales[1] = (uint8_t*)k->v_scales;
  v.slots = k->pages * k->page_size;
  v.pages = (uint32_t)k->pages; v.page_size = k->page_size; v.heads = k->heads; v.dim = k->head_dim; v.format = k->format;
  return v;
}

inline int logged(const qv2_ctx* c, const char* call, uint64_t before, int status) {
  if (c->log)
    std::fprintf(stderr, "qv2: %s launches=%llu status=%d (%s)\n", call, (unsigned long long)(c->launches - before), status, qv2_status_string(status));
  return status;
}

}  // namespace qv2
