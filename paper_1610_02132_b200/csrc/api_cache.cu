// C ABI of the 4-bit cache: argument validation and dispatch. See include/qsgd.h for the contract of every entry point.
#include <math.h>

#include "cache.cuh"

namespace qsgd {

namespace {

constexpr uint32_t kMostPageTokens = 1u << 16, kMostHeads = 1u << 16;

bool dim_taken(uint32_t dim) { return dim == 64 || dim == 128 || dim == 192 || dim == 256; }

bool page_taken(uint32_t page_tokens, uint32_t heads, uint32_t dim) {
  return dim_taken(dim) && heads >= 1 && heads <= kMostHeads && page_tokens >= kCacheTile && page_tokens <= kMostPageTokens &&
         page_tokens % kCacheTile == 0;
}

uint64_t head_bytes(uint32_t page_tokens, uint32_t dim) { return (uint64_t)(page_tokens / kCacheTile) * 18 * dim; }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// a * b, or the largest number where 64 bits do not hold it.
uint64_t span(uint64_t a, uint64_t b) {
  const __uint128_t v = (__uint128_t)a * b;
  return v >> 64 ? ~0ull : (uint64_t)v;
}

int check_dense(const void* p, uint64_t row_stride, uint64_t head_stride) {
  if (!p) return QSGD_ERR_NULL;
  if (!aligned16(p) || (row_stride & 7u) || (head_stride & 7u)) return QSGD_ERR_ALIGN;
  if (row_stride >> 40 || head_stride >> 40) return QSGD_ERR_LAYOUT;
  return QSGD_OK;
}

// An output's rows and heads must lie apart.
int check_apart(uint64_t rows, uint64_t row_stride, uint64_t heads, uint64_t head_stride, uint32_t dim) {
  const bool rows_outside = (rows <= 1 || row_stride >= span(heads - 1, head_stride) + dim) && (heads <= 1 || head_stride >= dim);
  const bool heads_outside = (heads <= 1 || head_stride >= span(rows ? rows - 1 : 0, row_stride) + dim) && (rows <= 1 || row_stride >= dim);
  return rows_outside || heads_outside ? QSGD_OK : QSGD_ERR_LAYOUT;
}

}  // namespace

int resolve_cache(const qsgd_cache* cache, const qsgd_cache_rows* rows, uint32_t* status_dev, CacheView* view) {
  if (!cache || !rows || !status_dev) return QSGD_ERR_NULL;
  if (cache->type != QSGD_TYPE_F16 && cache->type != QSGD_TYPE_BF16) return QSGD_ERR_TYPE;
  if (!page_taken(cache->page_tokens, cache->heads, cache->head_dim)) return QSGD_ERR_LAYOUT;
  if (cache->n_pages < 1 || cache->n_pages > 0x7fffffffull || rows->rows > 0x7fffffffull || rows->sequences > 0x7fffffffu)
    return QSGD_ERR_SHAPE;
  if (rows->rows == 0 || rows->sequences == 0) {
    view->rows = 0;                                          // nothing to do, whatever the pointers are
    return rows->starts || rows->rows == rows->sequences ? QSGD_OK : QSGD_ERR_SHAPE;
  }
  if (!rows->starts && rows->rows != rows->sequences) return QSGD_ERR_SHAPE;
  if (!cache->data || !rows->table || !rows->lengths) return QSGD_ERR_NULL;
  if (!aligned16(cache->data) || (cache->page_stride & 15u) || (cache->head_stride & 15u)) return QSGD_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(rows->table) | reinterpret_cast<uintptr_t>(rows->lengths) | reinterpret_cast<uintptr_t>(rows->starts)) & 3u)
    return QSGD_ERR_ALIGN;
  const uint64_t bytes = head_bytes(cache->page_tokens, cache->head_dim);
  if (cache->page_stride >> 40 || cache->head_stride >> 40) return QSGD_ERR_LAYOUT;
  const bool pages_outside = (cache->n_pages == 1 || cache->page_stride >= span(cache->heads - 1, cache->head_stride) + bytes) &&
                             (cache->heads == 1 || cache->head_stride >= bytes);
  const bool heads_outside = (cache->heads == 1 || cache->head_stride >= span(cache->n_pages - 1, cache->page_stride) + bytes) &&
                             (cache->n_pages == 1 || cache->page_stride >= bytes);
  if (!pages_outside && !heads_outside) return QSGD_ERR_LAYOUT;
  if (rows->table_pages < 1 || rows->table_pages > 0x7fffffffu || (rows->sequences > 1 && rows->table_stride < rows->table_pages))
    return QSGD_ERR_SHAPE;
  *view = CacheView{static_cast<uint8_t*>(cache->data), cache->page_stride, cache->head_stride, rows->table, rows->table_stride,
                    rows->lengths, rows->starts, (uint32_t)cache->n_pages, cache->page_tokens / kCacheTile, rows->table_pages,
                    rows->sequences, (uint32_t)rows->rows, cache->heads, status_dev};
  return QSGD_OK;
}

}  // namespace qsgd

using namespace qsgd;

extern "C" {

size_t qsgd_cache_page_bytes(uint32_t page_tokens, uint32_t heads, uint32_t head_dim) {
  return page_taken(page_tokens, heads, head_dim) ? (size_t)(heads * head_bytes(page_tokens, head_dim)) : 0;
}

static int store(const qsgd_cache* cache, const qsgd_cache_rows* rows, void* k, uint64_t k_row, uint64_t k_head, void* v, uint64_t v_row,
                 uint64_t v_head, uint32_t* status_dev, qsgd_stream_t stream, bool write) {
  CacheView view;
  int st = resolve_cache(cache, rows, status_dev, &view);
  if (st || view.rows == 0) return st;
  st = check_dense(k, k_row, k_head);
  if (!st) st = check_dense(v, v_row, v_head);
  if (!st && !write) st = check_apart(view.rows, k_row, view.heads, k_head, cache->head_dim);
  if (!st && !write) st = check_apart(view.rows, v_row, view.heads, v_head, cache->head_dim);
  if (st) return st;
  return (write ? launch_cache_write(view, cache->head_dim, cache->type, k, k_row, k_head, v, v_row, v_head, static_cast<cudaStream_t>(stream))
                : launch_cache_read(view, cache->head_dim, cache->type, k, k_row, k_head, v, v_row, v_head, static_cast<cudaStream_t>(stream)));
}

int qsgd_cache_write(const qsgd_cache* cache, const qsgd_cache_rows* rows, const void* k, uint64_t k_row_stride, uint64_t k_head_stride,
                     const void* v, uint64_t v_row_stride, uint64_t v_head_stride, uint32_t* status_dev, qsgd_stream_t stream) {
  return store(cache, rows, const_cast<void*>(k), k_row_stride, k_head_stride, const_cast<void*>(v), v_row_stride, v_head_stride, status_dev,
               stream, true);
}

int qsgd_cache_read(const qsgd_cache* cache, const qsgd_cache_rows* rows, void* k, uint64_t k_row_stride, uint64_t k_head_stride, void* v,
                    uint64_t v_row_stride, uint64_t v_head_stride, uint32_t* status_dev, qsgd_stream_t stream) {
  return store(cache, rows, k, k_row_stride, k_head_stride, v, v_row_stride, v_head_stride, status_dev, stream, false);
}

size_t qsgd_cache_attend_workspace_bytes(const qsgd_cache* cache, uint32_t q_heads) {
  if (!cache || !page_taken(cache->page_tokens, cache->heads, cache->head_dim) || q_heads == 0 || q_heads > kMostHeads || q_heads % cache->heads) return 0;
  return cache_attend_workspace_bytes(cache->head_dim);
}

int qsgd_cache_attend(const qsgd_cache* cache, const qsgd_cache_rows* rows, const void* q, uint64_t q_row_stride, uint64_t q_head_stride,
                      uint32_t q_heads, float scale, void* out, uint64_t out_row_stride, uint64_t out_head_stride, float* lse, void* workspace,
                      uint32_t* status_dev, qsgd_stream_t stream) {
  CacheView view;
  int st = resolve_cache(cache, rows, status_dev, &view);
  if (st) return st;
  if (q_heads == 0 || q_heads > kMostHeads || q_heads % cache->heads || !isfinite(scale)) return QSGD_ERR_LAYOUT;
  if (view.rows == 0) return QSGD_OK;
  if ((uint64_t)view.rows * (q_heads / cache->heads) > 0x7fffffffull) return QSGD_ERR_SHAPE;
  st = check_dense(q, q_row_stride, q_head_stride);
  if (!st) st = check_dense(out, out_row_stride, out_head_stride);
  if (!st) st = check_apart(view.rows, out_row_stride, q_heads, out_head_stride, cache->head_dim);
  if (st) return st;
  if (!workspace) return QSGD_ERR_NULL;
  if (!aligned16(workspace) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return QSGD_ERR_ALIGN;
  const AttendArgs args{q, q_row_stride, q_head_stride, out, out_row_stride, out_head_stride, lse, q_heads, scale,
                        static_cast<uint8_t*>(workspace)};
  return launch_cache_attend(view, cache->head_dim, cache->type, args, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
