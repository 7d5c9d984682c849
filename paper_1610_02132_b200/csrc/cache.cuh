// The 4-bit cache of keys and values: layout, and how a row of a call finds its place in it.
//
// A (page, head) holds page_tokens / 16 tiles of 16 tokens, one after another, each of 18 * head_dim bytes:
//   key codes     [head_dim / 64][16 tokens][32 bytes]      nibble i of a 32-bit word = coordinate 8 * word + i
//   key pairs     [16 tokens][head_dim / 64] (lo, step)     two numbers of the cache's 16-bit type
//   value codes, value pairs                                likewise
// so that everything attention needs of 16 tokens is one stretch of memory (2304 bytes at head_dim 128), which one bulk copy
// brings in, and 8 tokens' codes of a group lie in 256 bytes, which a warp reads from shared memory without a bank conflict.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "qsgd_common.cuh"

namespace qsgd {

constexpr uint32_t kCacheTile = 16;       // tokens per tile
constexpr uint32_t kCacheGroup = 64;      // values per (lo, step)

struct CacheView {                        // qsgd_cache and qsgd_cache_rows as the kernels take them
  uint8_t* data;
  uint64_t page_stride, head_stride;      // bytes
  const int32_t* table;
  uint64_t table_stride;                  // entries
  const int32_t* lengths;
  const int32_t* starts;                  // nullptr: row r is the last token of sequence r
  uint32_t n_pages, page_tiles, table_pages, sequences, rows, heads;
  uint32_t* status;
};

// Fills `view`; head_dim and type are the caller's to dispatch on.
int resolve_cache(const qsgd_cache* cache, const qsgd_cache_rows* rows, uint32_t* status_dev, CacheView* view);

int launch_cache_write(const CacheView& view, uint32_t head_dim, int type, const void* k, uint64_t k_token, uint64_t k_head,
                       const void* v, uint64_t v_token, uint64_t v_head, cudaStream_t stream);
int launch_cache_read(const CacheView& view, uint32_t head_dim, int type, void* k, uint64_t k_token, uint64_t k_head, void* v,
                      uint64_t v_token, uint64_t v_head, cudaStream_t stream);

struct AttendArgs {
  const void* q;
  uint64_t q_token, q_head;               // elements
  void* out;
  uint64_t out_token, out_head;
  float* lse;                             // [rows][q_heads] or nullptr
  uint32_t q_heads;
  float scale;
  uint8_t* workspace;
};
size_t cache_attend_workspace_bytes(uint32_t head_dim);
// For many rows a key head (cache_attend_wide.cu): whether it takes a call, and the launch.
bool cache_attend_wide_takes(const CacheView& view, uint32_t head_dim, int type, uint32_t q_heads);
int launch_cache_attend_wide(const CacheView& view, uint32_t head_dim, const AttendArgs& args, cudaStream_t stream);

int launch_cache_attend(const CacheView& view, uint32_t head_dim, int type, const AttendArgs& args, cudaStream_t stream);

// The power of two that sums of p v have to lose so that they stay in fp32 whatever the values are, p being 2^8 at most: from the longest sequence
// that the table can name.
inline int attend_sums_lose(const CacheView& view) {
  const uint64_t longest = (uint64_t)view.table_pages * view.page_tiles * kCacheTile;
  int lost = 9;
  while (lost < 40 && longest >> (lost - 9)) ++lost;
  return lost;
}

#ifdef __CUDACC__
// Pattern of a 16-bit number <-> fp32.
template <int TYPE>
__device__ __forceinline__ float from_bits16(uint32_t bits) {
  if (TYPE == QSGD_TYPE_BF16) return __uint_as_float(bits << 16);
  return __half2float(__ushort_as_half((unsigned short)bits));
}
template <int TYPE>
__device__ __forceinline__ uint32_t to_bits16(float v) {
  if (TYPE == QSGD_TYPE_BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
  return __half_as_ushort(__float2half_rn(v));
}
// The pair (low half, high half), rounded to nearest.
template <int TYPE>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  uint32_t r;
  if (TYPE == QSGD_TYPE_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Rows of one sequence: rows [start, start + n) are its last n tokens. What `starts` holds is looked at, not trusted.
struct SequenceRows {
  uint32_t start, n;
  int64_t length;                         // tokens in the cache, never more than its table row can name
};
__device__ __forceinline__ SequenceRows rows_of(const CacheView& c, uint32_t b, bool* bad) {
  SequenceRows s;
  const int64_t most = (int64_t)c.table_pages * c.page_tiles * kCacheTile;
  const int64_t length = __ldg(c.lengths + b);
  s.length = length < 0 ? 0 : length > most ? most : length;
  *bad = length != s.length;
  if (c.starts) {
    const int64_t first = __ldg(c.starts + b), last = __ldg(c.starts + b + 1);
    const bool fine = first >= 0 && last >= first && last <= (int64_t)c.rows;
    s.start = fine ? (uint32_t)first : 0u;
    s.n = fine ? (uint32_t)(last - first) : 0u;
    *bad |= !fine;
  } else {
    s.start = b;
    s.n = 1;
  }
  return s;
}

// The sequence of row r: the last one that starts at or before it. (sequences >= 1)
__device__ __forceinline__ uint32_t sequence_of(const CacheView& c, uint32_t r) {
  if (!c.starts) return r;
  uint32_t lo = 0, hi = c.sequences;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (__ldg(c.starts + mid) <= (int64_t)r) lo = mid; else hi = mid;
  }
  return lo;
}
#endif

}  // namespace qsgd
