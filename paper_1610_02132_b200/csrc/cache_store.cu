// Quantising keys and values into the 4-bit cache, and reading them back.
//
// A group of 64 values x of one token and head becomes lo = min x, step = the smallest number of the cache's type with
// 15 * step >= max x - min x, and codes c = the nearest of 0 .. 15 to (x - lo) / step, the lower one of two as near; it reads back as lo + step * c.
// lo is one of the values, so storing it in their type rounds nothing; rounding step up keeps the largest value within reach,
// and the codes are taken against the rounded step, so a value is never further than step / 2 from what is held for it.
//
// Both directions move 2 * head_dim * 2 dense bytes and 9/8 * head_dim held bytes a token and head and compute little: HBM
// bounds them, once the conversions stay off the slow conversion pipe (codes become floats, and floats codes, by adding 2^23) and nobody waits for
// places: where a row lies in the cache takes a search in `starts` and two dependent reads, and a ninth warp looks that up for the next rows
// of its CTA while the others move the present ones.
// Four lanes share a group (two times 16 dense bytes and two words of codes each: with eight lanes what a group takes once, its span and step,
// was done twice as often), a warp's eight teams neighbouring rows or heads; a team goes along its row's keys, or values, head by head.
// 65536 tokens of 8 heads of 128 read back: 60 us, 5.7 TB/s (102 with a conversion instruction a code). 15.6 K tokens written and read back: 47 us (78 at
// first, 53 with eight lanes to a group). Writing takes ten operations a value; its issue slots are two thirds full, and its warps wait most for what they
// read (the next head's numbers are asked for when the present one's codes are stored) and at the CTA's meetings.
#include <float.h>

#include "cache.cuh"

namespace qsgd {

namespace {

constexpr uint32_t kMovers = 256, kThreads = kMovers + 32, kLanes = 4, kTeams = kMovers / kLanes, kMostShift = 5;

struct StoreArgs {
  CacheView c;
  const uint16_t* k;
  const uint16_t* v;
  uint64_t k_token, k_head, v_token, v_head;
  uint32_t rows_shift;          // log2 of the rows that a CTA takes at a time
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

constexpr float kTwo23 = 8388608.0f;

// Goes through the CTA's rows, 1 << rows_shift at a time: `move` by all movers with the rows' places, while the ninth warp looks up the next.
template <int J, typename Move>
__device__ __forceinline__ void for_rows(const StoreArgs& a, Move&& move) {
  __shared__ uint64_t place[2][1u << kMostShift];
  const uint32_t rows = 1u << a.rows_shift;
  const uint64_t stride = (uint64_t)gridDim.x << a.rows_shift;
  const bool scout = threadIdx.x >= kMovers;
  const uint32_t i = threadIdx.x - kMovers;
  uint64_t first = (uint64_t)blockIdx.x << a.rows_shift;
  if (scout && i < rows) place[0][i] = first + i < a.c.rows ? place_of(a.c, (uint32_t)(first + i), 1152 * J) : kNowhere;
  __syncthreads();
  for (uint32_t turn = 0; first < a.c.rows; first += stride, turn ^= 1u) {
    if (scout) {
      const uint64_t next = first + stride + i;
      if (i < rows) place[turn ^ 1u][i] = next < a.c.rows ? place_of(a.c, (uint32_t)next, 1152 * J) : kNowhere;
    } else {
      move(place[turn], first);
    }
    __syncthreads();
  }
}

// A team's way along its row: the heads first, first + step, ... of the keys or of the values.
struct Way {
  uint64_t at;                 // the row's place
  uint32_t head, step;
  uint8_t* held;               // of `head`: the lane's first word of codes, the other lies 16 bytes, the pairs `pair` bytes further
  uint64_t held_step;
  uint32_t pair;
  const uint16_t* dense;       // the lane's first eight numbers, the others lie 32 further
  uint64_t dense_step;
};
template <int J>
__device__ __forceinline__ Way way_of(const StoreArgs& a, const uint64_t* place, uint64_t first) {
  const uint32_t team = threadIdx.x / kLanes, lane4 = threadIdx.x % kLanes, r = team & ((1u << a.rows_shift) - 1u);
  const uint32_t side = team >> a.rows_shift;               // the last bit of it: keys or values (two teams at least to a row)
  Way w;
  w.at = place[r];
  w.head = side >> 1;
  w.step = kTeams >> (a.rows_shift + 1);
  const uint32_t slot = (uint32_t)w.at & (kCacheTile - 1u);
  w.held = a.c.data + (w.at - slot) + (uint64_t)w.head * a.c.head_stride + (side & 1u) * 576 * J + slot * 32 + lane4 * 4;
  w.held_step = (uint64_t)w.step * a.c.head_stride;
  w.pair = J * 512 + slot * J * 4 - slot * 32 - lane4 * 4;
  const uint64_t row = first + r;
  w.dense = (side & 1u ? a.v + row * a.v_token + (uint64_t)w.head * a.v_head : a.k + row * a.k_token + (uint64_t)w.head * a.k_head) + lane4 * 8;
  w.dense_step = (uint64_t)w.step * (side & 1u ? a.v_head : a.k_head);
  return w;
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

// Smaller and larger of two pairs of numbers; not a number where one of them is none.
template <int TYPE>
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (TYPE == QSGD_TYPE_BF16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <int TYPE>
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (TYPE == QSGD_TYPE_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float reciprocal(float v) {
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// Codes and pair of a team's group; all lanes of the warp take part.
template <int TYPE>
__device__ __forceinline__ void quantize_group(const uint4 (&raw)[2], uint32_t (&codes_out)[2], uint32_t* pair_out) {
  uint32_t small = min2<TYPE>(min2<TYPE>(min2<TYPE>(raw[0].x, raw[0].y), min2<TYPE>(raw[0].z, raw[0].w)),
                              min2<TYPE>(min2<TYPE>(raw[1].x, raw[1].y), min2<TYPE>(raw[1].z, raw[1].w)));
  uint32_t large = max2<TYPE>(max2<TYPE>(max2<TYPE>(raw[0].x, raw[0].y), max2<TYPE>(raw[0].z, raw[0].w)),
                              max2<TYPE>(max2<TYPE>(raw[1].x, raw[1].y), max2<TYPE>(raw[1].z, raw[1].w)));
#pragma unroll
  for (int m = 1; m < (int)kLanes; m <<= 1) {
    small = min2<TYPE>(small, __shfl_xor_sync(0xffffffffu, small, m));
    large = max2<TYPE>(large, __shfl_xor_sync(0xffffffffu, large, m));
  }
  small = min2<TYPE>(small, __byte_perm(small, small, 0x1032));
  large = max2<TYPE>(large, __byte_perm(large, large, 0x1032));
  const float lo = from_bits16<TYPE>(small & 0xffffu) + 0.0f;               // -0 becomes +0: the pair's bits do not depend on the order
  const float hi = from_bits16<TYPE>(large & 0xffffu);
  // The span as the sum of two numbers, so that step is the smallest number with 15 * step (exact in fp32) at least as large, not one near it.
  const float span = hi - lo, back = span - hi, rest = (hi - (span - back)) - (lo + back);
  const bool fine = fabsf(span) <= FLT_MAX;                 // not with an infinity or what is no number among the values
  uint32_t step_bits = to_bits16<TYPE>(span * (1.0f / 15.0f));
  const float near = 15.0f * from_bits16<TYPE>(step_bits), below = 15.0f * from_bits16<TYPE>(step_bits - 1u);
  if (near < span || (near == span && rest > 0.0f)) ++step_bits;
  else if (step_bits && (below > span || (below == span && rest <= 0.0f))) --step_bits;
  if (span < 15.0f * 1.1754943508222875e-38f) step_bits = 0;                // step below the smallest normal fp32: every code is 0
  // Slightly too large on purpose (the approximation is off by 2^-23 at most, the difference by 2^-24): a quotient is rounded to its nearest code or to
  // one too high, never too low. The border below that code tells the two apart: rounded down, since then a number of 24 bits or fewer lies above it
  // exactly where it lies above lo + (code - 1/2) * step itself, however far apart the exponents of the three are.
  const float step = from_bits16<TYPE>(step_bits), inverse = step > 0.0f ? reciprocal(step) * (1.0f + 0x1p-21f) : 0.0f;
  const float base = step > 0.0f ? lo : -INFINITY;          // without a step no value leaves code 0
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const uint32_t w[4] = {raw[x].x, raw[x].y, raw[x].z, raw[x].w};
    uint32_t codes = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
      const float v = from_bits16<TYPE>(i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu);
      const float t = fmaf(v - lo, inverse, kTwo23);        // 2^23 + the quotient, rounded to a whole number
      const float border = __fmaf_rd((t - kTwo23) - 0.5f, step, base);
      codes = codes * 16u + (__float_as_uint(t) - (v <= border ? 1u : 0u));
    }
    codes_out[x] = fine ? codes - 0xfb000000u : 0u;         // less the exponents of the 2^23, as far as they lie in 32 bits
  }
  *pair_out = fine ? to_bits16<TYPE>(lo) | step_bits << 16 : TYPE == QSGD_TYPE_BF16 ? 0x7fc07fc0u : 0x7e007e00u;     // reads back as NaN
}

template <int TYPE, int J>
__global__ void __launch_bounds__(kThreads, 3) cache_write_kernel(const __grid_constant__ StoreArgs a) {
  const uint32_t lane4 = threadIdx.x % kLanes;
  chain_wait();
  for_rows<J>(a, [&](const uint64_t* place, uint64_t first) {
    Way w = way_of<J>(a, place, first);
    const uint32_t heads = w.at < kBefore ? a.c.heads : 0u;
    // (the lanes of a warp go round together: the shuffles are of the whole warp)
    const uint32_t rounds = (a.c.heads + w.step - 1) / w.step;
#pragma unroll 1
    for (uint32_t i = 0; i < rounds; ++i) {
      uint4 raw[J][2];
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          raw[j][x] = w.head < heads ? __ldg(reinterpret_cast<const uint4*>(w.dense + j * kCacheGroup + x * 32)) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        uint32_t codes[2], pair;
        quantize_group<TYPE>(raw[j], codes, &pair);
        if (w.head < heads) {
          *reinterpret_cast<uint32_t*>(w.held + j * 512) = codes[0];
          *reinterpret_cast<uint32_t*>(w.held + j * 512 + 16) = codes[1];
          if (lane4 == 0) *reinterpret_cast<uint32_t*>(w.held + w.pair + j * 4) = pair;
        }
      }
      w.head += w.step;
      w.held += w.held_step;
      w.dense += w.dense_step;
    }
  });
  check_starts(a.c);
}

// Whether lo + step * code may need more than the 24 bits of fp32: a number of the type is a multiple of 2^-bits of its size, so the sums are not
// if all of them lie below 2^24 times the smaller multiple. (Not the case in ordinary groups: lo is zero or of the values' size.)
template <int TYPE>
__device__ __forceinline__ bool sums_are_long(uint32_t pair) {
  const float lo = fabsf(from_bits16<TYPE>(pair & 0xffffu)), step = from_bits16<TYPE>(pair >> 16);
  return lo > 0.0f && fmaf(16.0f, step, lo) > (TYPE == QSGD_TYPE_BF16 ? 65536.0f : 8192.0f) * fminf(lo, step);
}

// Eight values of the group's type from a word of codes, rounded once. ODD: by way of fp32 numbers rounded to odd, which keep on which side of a
// number of the type, or of the middle between two, the sum lies.
template <int TYPE, bool ODD>
__device__ __forceinline__ uint4 expand_word(uint32_t word, float lo, float step) {
  const uint32_t even = word & 0x0f0f0f0fu, odd = (word >> 4) & 0x0f0f0f0fu;
  auto sum = [&](float code) {
    if (!ODD) return fmaf(step, code, lo);                  // step * code is exact in fp32, and so is the sum
    const float below = __fmaf_rd(step, code, lo), above = __fmaf_ru(step, code, lo);
    return __float_as_uint(below) & 1u ? below : above;     // (the same where it is exact)
  };
  uint32_t o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float c0 = __uint_as_float(__byte_perm(even, 0x4b000000u, 0x7440 + j)) - kTwo23;         // 2^23 + code, less 2^23
    const float c1 = __uint_as_float(__byte_perm(odd, 0x4b000000u, 0x7440 + j)) - kTwo23;
    o[j] = pack16<TYPE>(sum(c0), sum(c1));
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}
template <int TYPE>
__device__ __forceinline__ uint4 expand(uint32_t word, uint32_t pair) {
  const float lo = from_bits16<TYPE>(pair & 0xffffu), step = from_bits16<TYPE>(pair >> 16);
  return sums_are_long<TYPE>(pair) ? expand_word<TYPE, true>(word, lo, step) : expand_word<TYPE, false>(word, lo, step);
}

template <int TYPE, int J>
__global__ void __launch_bounds__(kThreads, 3) cache_read_kernel(const __grid_constant__ StoreArgs a) {
  chain_wait();
  for_rows<J>(a, [&](const uint64_t* place, uint64_t first) {
    Way w = way_of<J>(a, place, first);
    if (w.at == kNowhere) return;
    constexpr int kAhead = J <= 2 ? 4 / J : 1;              // heads whose reads are in flight together
#pragma unroll 1
    for (; w.head < a.c.heads; w.head += kAhead * w.step) {
      uint32_t word[kAhead][J][2], pair[kAhead][J];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
          word[i][j][0] = word[i][j][1] = pair[i][j] = 0;   // in front of the first token: zeros
          if (w.at != kBefore && w.head + i * w.step < a.c.heads) {
            const uint8_t* const at = w.held + i * w.held_step;
            word[i][j][0] = __ldg(reinterpret_cast<const uint32_t*>(at + j * 512));
            word[i][j][1] = __ldg(reinterpret_cast<const uint32_t*>(at + j * 512 + 16));
            pair[i][j] = __ldg(reinterpret_cast<const uint32_t*>(at + w.pair + j * 4));
          }
        }
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (w.head + i * w.step < a.c.heads) {
          uint16_t* const to = const_cast<uint16_t*>(w.dense) + i * w.dense_step;
#pragma unroll
          for (int j = 0; j < J; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x) *reinterpret_cast<uint4*>(to + j * kCacheGroup + x * 32) = expand<TYPE>(word[i][j][x], pair[i][j]);
        }
      w.held += kAhead * w.held_step;
      w.dense += kAhead * w.dense_step;
    }
  });
  check_starts(a.c);
}

template <typename Kernel>
int launch_store(Kernel kern, KernelSite& site, KernelId id, StoreArgs& a, cudaStream_t stream) {
  int sms = 0, occ = 0;
  const int st = site.lookup(kern, kThreads, 0, &sms, &occ);
  if (st) return st;
  // As many rows at a time as keep the teams busy, and more, up to 32, as long as every CTA goes round six times: then the last round, which
  // not all take part in, makes up little of the time.
  const uint64_t places = (uint64_t)sms * occ;
  a.rows_shift = 0;
  while (a.rows_shift < kMostShift && kTeams >> a.rows_shift > 2 * a.c.heads) ++a.rows_shift;
  while (a.rows_shift < kMostShift && (a.c.rows >> (a.rows_shift + 1)) >= 6 * places) ++a.rows_shift;
  const uint64_t blocks = ((uint64_t)a.c.rows + (1u << a.rows_shift) - 1) >> a.rows_shift;
  ScopedKernel sk(id, stream);
  return (int)launch_chained(kern, (uint32_t)(blocks < places ? blocks : places), kThreads, 0, stream, a);
}

template <int TYPE, int J>
int launch_way(StoreArgs& a, bool write, cudaStream_t stream) {
  static KernelSite site[2];
  if (write) return launch_store(cache_write_kernel<TYPE, J>, site[0], kKernCacheWrite, a, stream);
  return launch_store(cache_read_kernel<TYPE, J>, site[1], kKernCacheRead, a, stream);
}

template <int TYPE>
int launch_dim(StoreArgs& a, uint32_t head_dim, bool write, cudaStream_t stream) {
  switch (head_dim / kCacheGroup) {
    case 1: return launch_way<TYPE, 1>(a, write, stream);
    case 2: return launch_way<TYPE, 2>(a, write, stream);
    case 3: return launch_way<TYPE, 3>(a, write, stream);
    default: return launch_way<TYPE, 4>(a, write, stream);
  }
}

}  // namespace

int launch_cache_write(const CacheView& view, uint32_t head_dim, int type, const void* k, uint64_t k_token, uint64_t k_head,
                       const void* v, uint64_t v_token, uint64_t v_head, cudaStream_t stream) {
  StoreArgs a{view, static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), k_token, k_head, v_token, v_head, 0};
  return type == QSGD_TYPE_BF16 ? launch_dim<QSGD_TYPE_BF16>(a, head_dim, true, stream) : launch_dim<QSGD_TYPE_F16>(a, head_dim, true, stream);
}

int launch_cache_read(const CacheView& view, uint32_t head_dim, int type, void* k, uint64_t k_token, uint64_t k_head, void* v,
                      uint64_t v_token, uint64_t v_head, cudaStream_t stream) {
  StoreArgs a{view, static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), k_token, k_head, v_token, v_head, 0};
  return type == QSGD_TYPE_BF16 ? launch_dim<QSGD_TYPE_BF16>(a, head_dim, false, stream) : launch_dim<QSGD_TYPE_F16>(a, head_dim, false, stream);
}

}  // namespace qsgd
