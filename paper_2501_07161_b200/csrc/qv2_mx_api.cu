// C-ABI layer of the microscaled 4-bit operators and the quantized cache: argument checks, scratch
// and the launches of each call.
#include "qv2_context.cuh"
#include "qv2_mx.cuh"

using namespace qv2;

namespace {

constexpr uint64_t kMaxCols = 1ull << 26, kMaxRows = 1ull << 30, kMaxQuantRows = 1ull << 40;

Launch launch_of(const qv2_ctx* c) {
  Launch l; l.stream = c->stream; l.sm_count = c->sm_count; l.pdl = c->dependent_launch;
  return l;
}

// Element type of a flag word, or -1.
int dtype_of(uint32_t type) {
  return type == QV2_IN_F32 ? (int)kF32 : type == QV2_IN_F16 ? (int)kF16 : type == QV2_IN_BF16 ? (int)kBF16 : -1;
}

int check_dense(const void* p, int dtype, uint64_t ld, uint64_t rows, uint64_t cols) {
  if (dtype < 0) return QV2_ERR_ARG;
  if (rows == 0 || cols == 0) return QV2_OK;
  if (!p) return QV2_ERR_NULL;
  if ((uintptr_t)p % dtype_size((uint32_t)dtype)) return QV2_ERR_ALIGN;
  if (rows > 1 && ld < cols) return QV2_ERR_ARG;
  if (ld > (1ull << 40)) return QV2_ERR_SIZE;
  return QV2_OK;
}

int check_matrix(const qv2_mx_matrix* m, uint64_t max_groups, uint64_t max_rows) {
  if (!m) return QV2_ERR_NULL;
  if (m->groups == 0) return QV2_ERR_ARG;
  if (m->cols > kMaxCols || m->rows > max_rows || m->groups > max_groups) return QV2_ERR_SIZE;
  if (m->rows == 0 || m->cols == 0) return QV2_OK;
  if (!m->codes || !m->scales) return QV2_ERR_NULL;
  const uint64_t blocks = (m->cols + QV2_MX_BLOCK - 1) / QV2_MX_BLOCK;
  if (m->codes_ld < 16 * blocks || m->scales_ld < blocks) return QV2_ERR_ARG;
  if (m->codes_ld > (1ull << 36) || m->scales_ld > (1ull << 36)) return QV2_ERR_SIZE;
  if ((uintptr_t)m->codes % 16 || m->codes_ld % 16) return QV2_ERR_ALIGN;
  if (m->groups > 1) {
    // groups may not overlap, and their strides stay far from overflowing 64 bits
    if (m->codes_gs < (m->rows - 1) * m->codes_ld + 16 * blocks || m->scales_gs < (m->rows - 1) * m->scales_ld + blocks) return QV2_ERR_ARG;
    if (m->codes_gs >= (1ull << 40) || m->scales_gs >= (1ull << 40)) return QV2_ERR_SIZE;
    if (m->codes_gs % 16) return QV2_ERR_ALIGN;
  }
  return QV2_OK;
}

MxView view_of(const qv2_mx_matrix* m) {
  return MxView{(uint8_t*)m->codes, (uint8_t*)m->scales, m->codes_ld, m->scales_ld, m->groups > 1 ? m->codes_gs : 0, m->groups > 1 ? m->scales_gs : 0};
}

int check_product(const qv2_mx_matrix* w, uint64_t rows, const float* bias, const int64_t* offsets, const void* y, int dtype, uint64_t y_ld) {
  int st = check_matrix(w, QV2_MX_MAX_GROUPS, kMaxRows);
  if (st != QV2_OK) return st;
  if (!offsets && w->groups != 1) return QV2_ERR_ARG;
  if (rows > kMaxRows) return QV2_ERR_SIZE;
  // tile numbers stay below 2^31, whichever of the product's shapes is taken (16 rows by 128 are its smallest tile)
  if (((rows + 15) / 16 + w->groups) * ((w->rows + 127) / 128) > 0x7fffffffull) return QV2_ERR_SIZE;
  if ((uintptr_t)bias % 4 || (uintptr_t)offsets % 8) return QV2_ERR_ALIGN;
  return check_dense(y, dtype, y_ld, rows, w->rows);
}

// Whether a kernel of an earlier call gave up waiting; asking clears it.  Every call asks once its arguments are in order, so
// that what a failed product left behind is not taken further unnoticed.
int take_fault(qv2_ctx* c) {
  if (!*(volatile uint32_t*)c->h_fault) return QV2_OK;
  *(volatile uint32_t*)c->h_fault = 0;
  return QV2_ERR_TIMEOUT;
}

int run_product(qv2_ctx* c, const MxView& a, uint64_t rows, const qv2_mx_matrix* w, const float* bias, const int64_t* offsets, void* y,
                int dtype, uint64_t y_ld, bool early) {
  MxProduct p;
  p.early = early && c->dependent_launch; p.fault = c->d_fault;
  p.a = a; p.w = view_of(w);
  p.bias = bias; p.offsets = offsets; p.y = y; p.y_ld = y_ld;
  p.dtype = (uint32_t)dtype; p.m = (uint32_t)rows; p.n = (uint32_t)w->rows; p.k = (uint32_t)w->cols; p.groups = (uint32_t)w->groups;
  QV2_CUDA(c, launch_mx_matmul(launch_of(c), p, &c->launches));
  return QV2_OK;
}

int check_cache(const qv2_kv_cache* k) {
  if (!k) return QV2_ERR_NULL;
  if (k->format > QV2_KV_I8 || k->page_size == 0 || k->heads == 0 || k->head_dim == 0) return QV2_ERR_ARG;
  if (k->head_dim > 4096 || k->heads > 65536 || k->pages > 0x7fffffffull) return QV2_ERR_SIZE;
  if (k->pages == 0) return QV2_OK;
  if (!k->k_codes || !k->k_scales || !k->v_codes || !k->v_scales) return QV2_ERR_NULL;
  if (k->format == QV2_KV_MX4 && (((uintptr_t)k->k_codes | (uintptr_t)k->v_codes) & 15u)) return QV2_ERR_ALIGN;
  if (k->format == QV2_KV_I8 && (((uintptr_t)k->k_scales | (uintptr_t)k->v_scales) & 3u)) return QV2_ERR_ALIGN;
  return QV2_OK;
}

KvView view_of(const qv2_kv_cache* k) {
  KvView v;
  v.codes[0] = (uint8_t*)k->k_codes; v.codes[1] = (uint8_t*)k->v_codes;
  v.scales[0] = (uint8_t*)k->k_scales; v.scales[1] = (uint8_t*)k->v_scales;
  v.slots = k->pages * k->page_size;
  v.pages = (uint32_t)k->pages; v.page_size = k->page_size; v.heads = k->heads; v.dim = k->head_dim; v.format = k->format;
  return v;
}

int logged(const qv2_ctx* c, const char* call, uint64_t before, int status) {
  if (c->log)
    std::fprintf(stderr, "qv2: %s launches=%llu status=%d (%s)\n", call, (unsigned long long)(c->launches - before), status, qv2_status_string(status));
  return status;
}

}  // namespace

extern "C" int qv2_mx_quantize(qv2_ctx* c, const void* x, uint32_t x_type, uint64_t x_ld, const qv2_mx_matrix* out, void* values,
                               uint64_t values_ld) {
  if (!c) return QV2_ERR_NULL;
  TraceRange range("qv2_mx_quantize");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    const int dtype = dtype_of(x_type);
    int st = check_matrix(out, 1, kMaxQuantRows);
    if (st != QV2_OK) return st;
    if ((st = check_dense(x, dtype, x_ld, out->rows, out->cols)) != QV2_OK) return st;
    if (values && (st = check_dense(values, dtype, values_ld, out->rows, out->cols)) != QV2_OK) return st;
    if ((st = take_fault(c)) != QV2_OK) return st;
    if (out->rows == 0 || out->cols == 0) return QV2_OK;
    DeviceGuard guard(c->device);
    QV2_CUDA(c, launch_mx_quantize(launch_of(c), x, (uint32_t)dtype, x_ld, out->rows, (uint32_t)out->cols, view_of(out), values, values_ld, &c->launches));
    return QV2_OK;
  };
  return logged(c, "qv2_mx_quantize", before, run());
}

extern "C" int qv2_mx_dequantize(qv2_ctx* c, const qv2_mx_matrix* m, void* y, uint32_t y_type, uint64_t y_ld) {
  if (!c) return QV2_ERR_NULL;
  TraceRange range("qv2_mx_dequantize");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    const int dtype = dtype_of(y_type);
    int st = check_matrix(m, 1ull << 20, kMaxRows);
    if (st != QV2_OK) return st;
    if ((st = check_dense(y, dtype, y_ld, m->groups * m->rows, m->cols)) != QV2_OK) return st;
    if ((st = take_fault(c)) != QV2_OK) return st;
    if (m->rows == 0 || m->cols == 0) return QV2_OK;
    DeviceGuard guard(c->device);
    QV2_CUDA(c, launch_mx_dequantize(launch_of(c), view_of(m), m->groups, m->rows, (uint32_t)m->cols, y, (uint32_t)dtype, y_ld, &c->launches));
    return QV2_OK;
  };
  return logged(c, "qv2_mx_dequantize", before, run());
}

extern "C" int qv2_mx_matmul(qv2_ctx* c, const qv2_mx_matrix* a, const qv2_mx_matrix* w, const float* bias, const int64_t* offsets, void* y,
                             uint32_t y_type, uint64_t y_ld) {
  if (!c) return QV2_ERR_NULL;
  TraceRange range("qv2_mx_matmul");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    const int dtype = dtype_of(y_type);
    int st = check_matrix(a, 1, kMaxRows);
    if (st != QV2_OK) return st;
    if ((st = check_product(w, a->rows, bias, offsets, y, dtype, y_ld)) != QV2_OK) return st;
    if (a->cols != w->cols) return QV2_ERR_ARG;
    if ((st = take_fault(c)) != QV2_OK) return st;
    if (a->rows == 0 || w->rows == 0) return QV2_OK;
    DeviceGuard guard(c->device);
    return run_product(c, view_of(a), a->rows, w, bias, offsets, y, dtype, y_ld, false);
  };
  return logged(c, "qv2_mx_matmul", before, run());
}

extern "C" int qv2_check_waits(qv2_ctx* c) {
  if (!c) return QV2_ERR_NULL;
  DeviceGuard guard(c->device);
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  QV2_CUDA(c, cudaStreamIsCapturing(c->stream, &capture));
  if (capture != cudaStreamCaptureStatusNone) return QV2_ERR_UNSUPPORTED;
  ++c->syncs;
  QV2_CUDA(c, cudaStreamSynchronize(c->stream));
  return take_fault(c);
}

extern "C" int qv2_debug_fail_wait(qv2_ctx* c) {
  if (!c) return QV2_ERR_NULL;
  *(volatile uint32_t*)c->h_fault = 1;
  return QV2_OK;
}

extern "C" int qv2_debug_mx_form(uint64_t rows, uint64_t n, uint64_t groups, uint32_t sm_count, uint64_t* tiles) {
  if (groups == 0 || sm_count == 0) return QV2_ERR_ARG;
  if (rows > kMaxRows || n > kMaxRows || groups > QV2_MX_MAX_GROUPS) return QV2_ERR_SIZE;
  return (int)mx_product_form((uint32_t)rows, (uint32_t)n, (uint32_t)groups, sm_count, tiles);
}

extern "C" int qv2_mx_linear(qv2_ctx* c, const void* x, uint32_t x_type, uint64_t x_ld, uint64_t rows, const qv2_mx_matrix* w,
                             const float* bias, const int64_t* offsets, void* y, uint32_t y_type, uint64_t y_ld) {
  if (!c) return QV2_ERR_NULL;
  TraceRange range("qv2_mx_linear");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    const int xt = dtype_of(x_type), yt = dtype_of(y_type);
    int st = check_product(w, rows, bias, offsets, y, yt, y_ld);
    if (st != QV2_OK) return st;
    if ((st = check_dense(x, xt, x_ld, rows, w->cols)) != QV2_OK) return st;
    if ((st = take_fault(c)) != QV2_OK) return st;
    if (rows == 0 || w->rows == 0) return QV2_OK;
    DeviceGuard guard(c->device);
    const uint64_t blocks = (w->cols + QV2_MX_BLOCK - 1) / QV2_MX_BLOCK;
    MxView a;
    a.codes_ld = 16 * blocks; a.scales_ld = (blocks + 15) / 16 * 16; a.codes_gs = a.scales_gs = 0;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    QV2_CUDA(c, cudaStreamIsCapturing(c->stream, &capture));
    const bool capturing = capture != cudaStreamCaptureStatusNone;
    if ((st = grow_capturable(c, &c->d_mx_codes, &c->cap_mx_codes, rows * a.codes_ld, capturing, &c->mx_codes_captured)) != QV2_OK) return st;
    if ((st = grow_capturable(c, &c->d_mx_scales, &c->cap_mx_scales, rows * a.scales_ld, capturing, &c->mx_scales_captured)) != QV2_OK) return st;
    a.codes = c->d_mx_codes; a.scales = c->d_mx_scales;
    if (w->cols) QV2_CUDA(c, launch_mx_quantize(launch_of(c), x, (uint32_t)xt, x_ld, rows, (uint32_t)w->cols, a, nullptr, 0, &c->launches));
    // The kernel that rounds x waits for all work before it and only then lets the product begin, so
    // weights, bias and offsets are complete when the product starts to fetch them.
    return run_product(c, a, rows, w, bias, offsets, y, yt, y_ld, w->cols != 0);
  };
  return logged(c, "qv2_mx_linear", before, run());
}

extern "C" int qv2_kv_write(qv2_ctx* c, const qv2_kv_cache* cache, const void* k, uint64_t k_token_ld, uint64_t k_head_ld, const void* v,
                            uint64_t v_token_ld, uint64_t v_head_ld, uint32_t type, uint64_t tokens, const int64_t* slots) {
  if (!c) return QV2_ERR_NULL;
  TraceRange range("qv2_kv_write");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    const int dtype = dtype_of(type);
    int st = check_cache(cache);
    if (st != QV2_OK) return st;
    if (dtype < 0) return QV2_ERR_ARG;
    if (tokens > (1ull << 40)) return QV2_ERR_SIZE;
    if (tokens && (!k || !v || !slots)) return QV2_ERR_NULL;
    if (tokens && (((uintptr_t)k | (uintptr_t)v) % dtype_size((uint32_t)dtype) || (uintptr_t)slots % 8)) return QV2_ERR_ALIGN;
    if ((st = take_fault(c)) != QV2_OK) return st;
    if (tokens == 0) return QV2_OK;
    if (cache->pages == 0) return QV2_OK;                      // no slot exists: every token is skipped
    DeviceGuard guard(c->device);
    KvNew n;
    n.x[0] = k; n.x[1] = v; n.token_ld[0] = k_token_ld; n.token_ld[1] = v_token_ld; n.head_ld[0] = k_head_ld; n.head_ld[1] = v_head_ld;
    n.slots = slots; n.tokens = tokens; n.dtype = (uint32_t)dtype;
    QV2_CUDA(c, launch_kv_write(launch_of(c), view_of(cache), n, &c->launches));
    return QV2_OK;
  };
  return logged(c, "qv2_kv_write", before, run());
}

extern "C" int qv2_kv_read(qv2_ctx* c, const qv2_kv_cache* cache, const int32_t* table, uint64_t table_ld, uint32_t seqs,
                           const int64_t* starts, uint64_t total, void* k, void* v, uint32_t type) {
  if (!c) return QV2_ERR_NULL;
  TraceRange range("qv2_kv_read");
  const uint64_t before = c->launches;
  auto run = [&]() -> int {
    const int dtype = dtype_of(type);
    int st = check_cache(cache);
    if (st != QV2_OK) return st;
    if (dtype < 0) return QV2_ERR_ARG;
    if (total > (1ull << 30) || seqs > (1u << 30) || table_ld > (1ull << 40)) return QV2_ERR_SIZE;
    if (total && ((!k && !v) || !starts || (seqs && table_ld && !table))) return QV2_ERR_NULL;
    if (total && (((uintptr_t)k | (uintptr_t)v) % dtype_size((uint32_t)dtype) || (uintptr_t)starts % 8 || (uintptr_t)table % 4)) return QV2_ERR_ALIGN;
    if ((st = take_fault(c)) != QV2_OK) return st;
    if (total == 0) return QV2_OK;
    DeviceGuard guard(c->device);
    KvRead r;
    r.table = table; r.table_ld = table_ld; r.starts = starts; r.seqs = seqs; r.total = total; r.y[0] = k; r.y[1] = v; r.dtype = (uint32_t)dtype;
    QV2_CUDA(c, launch_kv_read(launch_of(c), view_of(cache), r, &c->launches));
    return QV2_OK;
  };
  return logged(c, "qv2_kv_read", before, run());
}
