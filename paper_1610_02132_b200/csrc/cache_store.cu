// Quantising keys and values into the 4-bit cache, and reading them back.
//
// A group of 64 values x of one token and head becomes lo = min x, step = the smallest number of the cache's type with
// 15 * step >= max x - min x, and codes c = the nearest of 0 .. 15 to (x - lo) / step, the lower one of two as near; it reads back as lo + step * c.
// lo is one of the values, so storing it in their type rounds nothing; rounding step up keeps the largest value within reach,
// and the codes are taken against the rounded step, so a value is never further than step / 2 from what is held for it.
//
// Both directions move 2 * head_dim * 2 dense bytes and 9/8 * head_dim held bytes a token and head and compute little: HBM
// bounds them. Eight lanes share a group (16 dense bytes and one word of codes each), so a warp's accesses to either side are whole sectors. Where
// a row lies in the cache takes a search in `starts` and two dependent reads; a CTA looks that up for up to 32 rows at once, a lane to a
// row, before it moves any of them.
#include <float.h>

#include "cache.cuh"

namespace qsgd {

namespace {

constexpr uint32_t kThreads = 256, kTeams = kThreads / 8, kMostRows = 32;

struct StoreArgs {
  CacheView c;
  const uint16_t* k;
  const uint16_t* v;
  uint64_t k_token, k_head, v_token, v_head;
  uint32_t rows_shift;          // log2 of the rows a CTA takes at a time
  uint32_t head_dim;
};

constexpr uint64_t kNowhere = ~0ull, kBefore = ~0ull - 1;

// Byte offset of a row's tile (head 0) with its token's place in the tile in the low four bits (tiles begin on 16-byte boundaries); kNowhere for a
// row of no sequence or of a place that the cache has not, kBefore for a row in front of its sequence's first token.
__device__ uint64_t place_of(const CacheView& c, uint32_t r, uint32_t tile_bytes) {
  if (r >= c.rows) return kNowhere;
  const uint32_t b = sequence_of(c, r);
  bool bad;
  const SequenceRows s = rows_of(c, b, &bad);
  if (bad) { atomicOr(c.status, QSGD_DEV_PAGE); return kNowhere; }
  if (r < s.start || r - s.start >= s.n) return kNowhere;
  const int64_t pos = s.length - (int64_t)(s.n - (r - s.start));
  if (pos < 0) return kBefore;
  const uint32_t tile = (uint32_t)(pos / kCacheTile), page = tile / c.page_tiles;
  const int32_t at = __ldg(c.table + (uint64_t)b * c.table_stride + page);
  if (at < 0 || (uint32_t)at >= c.n_pages) { atomicOr(c.status, QSGD_DEV_PAGE); return kNowhere; }
  return (uint64_t)at * c.page_stride + (uint64_t)(tile - page * c.page_tiles) * tile_bytes + (uint32_t)(pos % kCacheTile);
}

// What a lane of a team holds of a group: unit u of a CTA's rows, the row fastest.
struct Unit {
  uint64_t at;
  uint32_t row, head, half, group;
};
__device__ __forceinline__ Unit unit_of(const StoreArgs& a, const uint64_t* place, uint32_t u) {
  Unit t;
  const uint32_t groups = a.head_dim / kCacheGroup;
  t.row = u & ((1u << a.rows_shift) - 1u);
  uint32_t rest = u >> a.rows_shift;
  t.half = rest & 1u;
  rest >>= 1;
  t.head = rest / groups;
  t.group = rest - t.head * groups;
  t.at = place[t.row];
  return t;
}
__device__ __forceinline__ uint64_t dense_at(const StoreArgs& a, const Unit& t, uint32_t r, uint32_t lane8) {
  return (uint64_t)r * (t.half ? a.v_token : a.k_token) + (uint64_t)t.head * (t.half ? a.v_head : a.k_head) + t.group * kCacheGroup +
         lane8 * 8;
}
// Addresses of the lane's word of codes and of the group's pair.
__device__ __forceinline__ void held_at(const StoreArgs& a, const Unit& t, uint32_t lane8, uint32_t** word, uint32_t** pair) {
  const uint32_t slot = (uint32_t)t.at & (kCacheTile - 1u), D = a.head_dim;
  uint8_t* p = a.c.data + (t.at - slot) + (uint64_t)t.head * a.c.head_stride + t.half * 9 * D;
  *word = reinterpret_cast<uint32_t*>(p + (t.group * kCacheTile + slot) * 32 + lane8 * 4);
  *pair = reinterpret_cast<uint32_t*>(p + 8 * D + (slot * (D / kCacheGroup) + t.group) * 4);
}

// A row is looked up in one sequence only: that every sequence's rows ascend inside the call's is looked at here, by all CTAs together.
__device__ void check_starts(const CacheView& c) {
  if (!c.starts) return;
  for (uint64_t b = (uint64_t)blockIdx.x * kThreads + threadIdx.x; b < c.sequences; b += (uint64_t)gridDim.x * kThreads) {
    bool bad;
    rows_of(c, (uint32_t)b, &bad);
    if (bad) atomicOr(c.status, QSGD_DEV_PAGE);
  }
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const __grid_constant__ StoreArgs a) {
  __shared__ uint64_t place[kMostRows];
  const uint32_t team = threadIdx.x / 8, lane8 = threadIdx.x % 8, rows = 1u << a.rows_shift;
  const uint32_t units = (a.head_dim / kCacheGroup * a.c.heads * 2) << a.rows_shift;
  chain_wait();
  for (uint64_t first = (uint64_t)blockIdx.x << a.rows_shift; first < a.c.rows; first += (uint64_t)gridDim.x << a.rows_shift) {
    if (threadIdx.x < rows) place[threadIdx.x] = place_of(a.c, (uint32_t)first + threadIdx.x, 18 * a.head_dim);
    __syncthreads();
    // (all lanes of a warp go round together: the shuffles below are of the whole warp)
    for (uint32_t u0 = 0; u0 < units; u0 += kTeams) {
      const uint32_t u = u0 + team;
      Unit t = unit_of(a, place, u < units ? u : 0u);
      if (u >= units) t.at = kNowhere;
      const bool live = t.at < kBefore;
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (live) raw = __ldg(reinterpret_cast<const uint4*>((t.half ? a.v : a.k) + dense_at(a, t, (uint32_t)first + t.row, lane8)));
      const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[2 * i] = from_bits16<TYPE>(w[i] & 0xffffu); x[2 * i + 1] = from_bits16<TYPE>(w[i] >> 16); }
      float lo = x[0], hi = x[0];
      bool fine = fabsf(x[0]) <= FLT_MAX;
#pragma unroll
      for (int i = 1; i < 8; ++i) { lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]); fine &= fabsf(x[i]) <= FLT_MAX; }
#pragma unroll
      for (int m = 1; m < 8; m <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, m));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, m));
      }
      const uint32_t votes = __ballot_sync(0xffffffffu, fine);
      fine = ((votes >> (threadIdx.x & 24u)) & 0xffu) == 0xffu;
      lo += 0.0f;                                           // -0 becomes +0: the pair's bits do not depend on the order
      fine &= hi - lo <= FLT_MAX;
      // The span in 64 bits (exact but for wildly different exponents), so that step is the smallest number in reach, not one near it.
      const double span = (double)hi - (double)lo;
      uint32_t step_bits = to_bits16<TYPE>((float)span * (1.0f / 15.0f));
      if (15.0 * (double)from_bits16<TYPE>(step_bits) < span) ++step_bits;
      else if (step_bits && 15.0 * (double)from_bits16<TYPE>(step_bits - 1u) >= span) --step_bits;
      if (span < 15.0 * 1.1754943508222875e-38) step_bits = 0;      // step below the smallest normal fp32: every code is 0
      const float step = from_bits16<TYPE>(step_bits), inverse = step > 0.0f ? 1.0f / step : 0.0f;
      const float half = step > 0.0f ? 0.5f * step : INFINITY;           // without a step no value leaves code 0
      uint32_t codes = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = x[i] - lo;
        float c = rintf(d * inverse);
        // The quotient's last places may have crossed a border: the remainder, exact in one fused operation, says so.
        const float r = fmaf(-c, step, d);
        if (r > half) c += 1.0f;
        if (r <= -half && c > 0.0f) c -= 1.0f;
        codes |= (uint32_t)fminf(c, 15.0f) << (4 * i);
      }
      uint32_t pair = to_bits16<TYPE>(lo) | step_bits << 16;
      if (!fine) { codes = 0; pair = TYPE == QSGD_TYPE_BF16 ? 0x7fc07fc0u : 0x7e007e00u; }     // reads back as NaN
      if (live) {
        uint32_t *word_at, *pair_at;
        held_at(a, t, lane8, &word_at, &pair_at);
        *word_at = codes;
        if (lane8 == 0) *pair_at = pair;
      }
    }
    __syncthreads();
  }
  check_starts(a.c);
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const __grid_constant__ StoreArgs a) {
  __shared__ uint64_t place[kMostRows];
  const uint32_t team = threadIdx.x / 8, lane8 = threadIdx.x % 8, rows = 1u << a.rows_shift;
  const uint32_t units = (a.head_dim / kCacheGroup * a.c.heads * 2) << a.rows_shift;
  chain_wait();
  for (uint64_t first = (uint64_t)blockIdx.x << a.rows_shift; first < a.c.rows; first += (uint64_t)gridDim.x << a.rows_shift) {
    if (threadIdx.x < rows) place[threadIdx.x] = place_of(a.c, (uint32_t)first + threadIdx.x, 18 * a.head_dim);
    __syncthreads();
    constexpr int kAhead = 4;                               // units whose reads are in flight together
    for (uint32_t u0 = team; u0 < units; u0 += kAhead * kTeams) {
      uint32_t word[kAhead], pair[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const uint32_t u = u0 + i * kTeams;
        word[i] = pair[i] = 0;
        if (u < units) {
          const Unit t = unit_of(a, place, u);
          if (t.at < kBefore) {
            uint32_t *word_at, *pair_at;
            held_at(a, t, lane8, &word_at, &pair_at);
            word[i] = __ldg(word_at);
            pair[i] = __ldg(pair_at);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const uint32_t u = u0 + i * kTeams;
        if (u >= units) break;
        const Unit t = unit_of(a, place, u);
        if (t.at == kNowhere) continue;
        const float lo = from_bits16<TYPE>(pair[i] & 0xffffu), step = from_bits16<TYPE>(pair[i] >> 16);
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)                         // step * code is exact in fp32: one rounding there, one to the type
          o[j] = pack16<TYPE>(fmaf(step, (float)((word[i] >> (8 * j)) & 15u), lo), fmaf(step, (float)((word[i] >> (8 * j + 4)) & 15u), lo));
        *reinterpret_cast<uint4*>(const_cast<uint16_t*>(t.half ? a.v : a.k) + dense_at(a, t, (uint32_t)first + t.row, lane8)) =
            make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
    __syncthreads();
  }
  check_starts(a.c);
}

template <typename Kernel>
int launch_store(Kernel kern, KernelSite& site, KernelId id, StoreArgs& a, cudaStream_t stream) {
  int sms = 0, occ = 0;
  const int st = site.lookup(kern, kThreads, 0, &sms, &occ);
  if (st) return st;
  // As many rows to a CTA as leave every resident CTA some: one row at a time where there are few.
  const uint64_t ctas = (uint64_t)sms * occ;
  a.rows_shift = 0;
  while (a.rows_shift < 5 && (a.c.rows >> (a.rows_shift + 1)) >= ctas) ++a.rows_shift;
  const uint64_t blocks = ((uint64_t)a.c.rows + (1u << a.rows_shift) - 1) >> a.rows_shift;
  ScopedKernel sk(id, stream);
  return (int)launch_chained(kern, (uint32_t)(blocks < ctas ? blocks : ctas), kThreads, 0, stream, a);
}

}  // namespace

int launch_cache_write(const CacheView& view, uint32_t head_dim, int type, const void* k, uint64_t k_token, uint64_t k_head,
                       const void* v, uint64_t v_token, uint64_t v_head, cudaStream_t stream) {
  StoreArgs a{view, static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), k_token, k_head, v_token, v_head, 0, head_dim};
  static KernelSite site[2];
  if (type == QSGD_TYPE_BF16) return launch_store(cache_write_kernel<QSGD_TYPE_BF16>, site[0], kKernCacheWrite, a, stream);
  return launch_store(cache_write_kernel<QSGD_TYPE_F16>, site[1], kKernCacheWrite, a, stream);
}

int launch_cache_read(const CacheView& view, uint32_t head_dim, int type, void* k, uint64_t k_token, uint64_t k_head, void* v,
                      uint64_t v_token, uint64_t v_head, cudaStream_t stream) {
  StoreArgs a{view, static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), k_token, k_head, v_token, v_head, 0, head_dim};
  static KernelSite site[2];
  if (type == QSGD_TYPE_BF16) return launch_store(cache_read_kernel<QSGD_TYPE_BF16>, site[0], kKernCacheRead, a, stream);
  return launch_store(cache_read_kernel<QSGD_TYPE_F16>, site[1], kKernCacheRead, a, stream);
}

}  // namespace qsgd
