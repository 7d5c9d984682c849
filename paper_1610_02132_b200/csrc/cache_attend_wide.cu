// Attention over the 4-bit cache for many query rows a key head (chunks of a prompt), head sizes 64 and 128, bf16.
//
// The mathematics is that of cache_attend.cu. Here 128 rows share what is unpacked, so the codes become numbers once, k = lo + step * c and v likewise in
// fp16, and both products run on the fifth-generation tensor cores, sums in tensor memory:
//   S = Q K^T   128 rows x 64 tokens,   O += P V   128 rows x head_dim
// A CTA has 128 rows of one (sequence, key head) and goes over its tokens 64 at a time:
//   warp 0       brings the packed tiles in by bulk copies, four steps ahead
//   warp 1       issues the products (one lane of it)
//   warps 2, 3   the (lo, step) pairs of the keys, of the values: their largest number, and the pairs in fp16
//   warps 4-11   softmax: a thread to a row of S, four warps to every other step; P goes to shared memory; O is scaled in tensor memory when a maximum
//                rises by 2^8
//   warps 12-15  unpack the keys as rows of a token, 128-byte swizzle, two buffers
//   warps 16-19  unpack the values turned round (rows of a coordinate), three buffers
// Range: bf16 numbers need not fit fp16. The keys of a step, and its values, are multiplied by a power of two that puts their largest at 2^14, a query row
// likewise at 2^11; P holds p times a power of two of each row that follows its own largest p * v. Numbers 2^-28 below the largest of 64 tokens lose bits.
// Where that is more than the rounding to 11 bits (a group of a key or of a query much smaller than another one, of values than another of the same step: a row
// need not see the other, its weight may be low, a small query may meet a large key) or scores are so large that a power of two beside them is lost, the tile is done again in fp32: attend_plainly.
// Roundings: k and v to 11 bits, p to 11 bits, next to the output's 8. (For an fp16 output they would weigh as much as its own rounding: those go through
// cache_attend.cu.)
//
// What bounds it: a step is 2 * 128 * 64 * head_dim multiply-adds, 512 cycles of the tensor cores at head_dim 128, 8192 exponentials, another 512 cycles
// of the special-function units, and about 5000 warp instructions, half of them unpacking. It takes 1800 cycles at 1.72 GHz (1500 at head size 64), and no role waits
// for long: softmax warps 80 percent of the time at work, unpacking ones as much; issue slots 65 percent, tensor pipe 27. What took it there from 2700: issuing warps that go round as a whole
// (addresses in uniform registers; one lane by itself took 1250 cycles a step to issue and let P wait for 2200), softmax warps in two halves on
// alternate steps, and buffers enough that neither waits for the other's last step. Waits out of line, since the roles' code together is as
// large as the instruction cache (in line: 500 cycles more).
// Four chunks of 256 queries, 32 heads on 8 of 128, over 700 to 4096 tokens: 78.5 us, 0.39 PFLOP/s; by cache_attend.cu 204.
#include <float.h>

#include "cache.cuh"

namespace qsgd {

namespace {

constexpr uint32_t kRows = 128, kStep = 64, kThreads = 640, kUnpackWarps = 8, kSoftmaxWarps = 8, kRawStages = 4, kPairs = 4, kValues = 3;
constexpr uint32_t kMostSorted = 256;
constexpr uint32_t kDrainPolls = 1u << 22;                 // bound of the waits for copies and products in flight
constexpr float kNoMax = -FLT_MAX;                         // maximum of nothing: below any score, and finite, so that differences of maxima are numbers
// What the tiles' 11 bits and common powers of two are good for; a tile with more goes through attend_plainly. The largest number of one group of a step's
// keys next to that of another (groups of zeros aside), of its values, of a query row; the largest value at all; the size of a score.
constexpr float kKeyRange = 65536.0f, kValueRange = 4096.0f, kQueryRange = 4096.0f, kMostValue = 8.5070591730234616e+37f, kMostScore = 8192.0f;
constexpr float kLeastCap = 7.5231638452626401e-37f, kMostCap = 8.5070591730234616e+37f;      // 2^-120, 2^126

struct WideParams {
  CacheView c;
  const uint16_t* q;
  uint16_t* out;
  uint64_t q_token, q_head, out_token, out_head;
  float* lse;
  uint32_t q_heads, group;
  float scale_log2;
  uint32_t polls;              // bound of the roles' waits
  float times, back;           // for sums of p v in fp32: 2^-lost and 2^lost
};

template <int D>
struct Shape {
  static constexpr int kGroups = D / 64;
  static constexpr uint32_t kTile = 18 * D;                // 16 packed tokens
  static constexpr uint32_t kRaw = 4 * kTile;
  static constexpr uint32_t kQ = kRows * D * 2, kK = kStep * D * 2, kV = D * kStep * 2, kP = kRows * kStep * 2;
  static constexpr uint32_t kAtK = kQ, kAtV = kAtK + 2 * kK, kAtP = kAtV + kValues * kV, kAtRaw = kAtP + 2 * kP;
  static constexpr uint32_t kTmem = 4 * D;                 // two tiles of S, 64 columns each, and two of O (at least a power of two)
  static constexpr uint32_t kSmem = kAtRaw + kRawStages * kRaw + 1024;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Without the suspension that a try may bring.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// False when the wait ran out or another role's has. (Out of line: the roles' loops share the instruction cache, and each step goes through all of
// them; with every wait's loop in its place a step took 3000 cycles, most of them waiting for instructions.)
__device__ __noinline__ bool mbar_poll(uint32_t bar, uint32_t parity, volatile uint32_t* given_up, uint32_t polls) {
#pragma unroll 1
  for (uint32_t i = 0; i < polls; ++i) {
    if (mbar_try(bar, parity)) return true;
    if ((i & 63u) == 63u && *given_up) return false;
  }
  *given_up = 1;
  return false;
}
struct Waits {
  volatile uint32_t* given_up;
  uint32_t polls;
};
__device__ __forceinline__ bool given_up_now(const Waits& w) { return *w.given_up != 0; }
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const Waits& w) {
  return (w.polls && mbar_try(bar, parity)) || mbar_poll(bar, parity, w.given_up, w.polls);
}
// In line, where a call would have to save a row of scores.
__device__ __forceinline__ bool mbar_wait_here(uint32_t bar, uint32_t parity, const Waits& w) {
#pragma unroll 1
  for (uint32_t i = 0; i < w.polls; ++i) {
    if (mbar_try(bar, parity)) return true;
    if ((i & 63u) == 63u && *w.given_up) return false;
  }
  *w.given_up = 1;
  return false;
}
// One lane of a whole warp, the same each time.
__device__ __forceinline__ bool elected() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Rows of 128 bytes, 128-byte swizzle: 8 rows are 1024 bytes apart.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr) {
  return ((uint64_t)0x40004040u << 32) | (1u << 16) | ((addr >> 4) & 0x3fffu);
}
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
               "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_load64(uint32_t at, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
      "%25,%26,%27,%28,%29,%30,%31}, [%64];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,"
      "%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%65];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
        "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]),
        "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]),
        "=f"(v[31]), "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]), "=f"(v[40]),
        "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]), "=f"(v[48]), "=f"(v[49]), "=f"(v[50]),
        "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]), "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]),
        "=f"(v[61]), "=f"(v[62]), "=f"(v[63])
      : "r"(at), "r"(at + 32) : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const float* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n\t"
      "tcgen05.wait::st.sync.aligned;" ::"r"(at),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]),
      "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float exp2_approx(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// 2^(put - e) for a number of [2^e, 2^(e + 1)), as the exponent to build it from; 0 for zero, an infinity or what is no number.
__device__ __forceinline__ int32_t lift(float largest, int32_t put) {
  const int32_t e = (int32_t)(__float_as_uint(largest) >> 23) - 127;
  if (!(largest > 0.0f) || e == 128) return 0;
  const int32_t up = put - e;
  return up > 120 ? 120 : up;
}
__device__ __forceinline__ float power_above(float v) { return __uint_as_float((__float_as_uint(v) + 0x007fffffu) & 0xff800000u); }
__device__ __forceinline__ float inverse_of_power(float v) { return __uint_as_float((254u << 23) - __float_as_uint(v)); }      // of 2^-126 to 2^126
__device__ __forceinline__ float power2(int32_t e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// A named barrier of 64 threads; whether all of them said yes.
__device__ __forceinline__ bool meet(uint32_t id, bool yes) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %2, 0;\n\tbar.red.and.pred p, %1, 64, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(all) : "r"(id), "r"((uint32_t)yes) : "memory");
  return all != 0;
}
// Nibble s of either half of a word as lo + step * code.
__device__ __forceinline__ void values_of(uint32_t w, uint32_t step, uint32_t lo, uint32_t (&v)[4]) {
  const uint32_t u = w >> 8;
  v[0] = fma_f16x2(sub_f16x2((w & 0x000f000fu) | 0x64006400u, 0x64006400u), step, lo);      // 1024 + c, less 1024
  v[1] = fma_f16x2(sub_f16x2((w & 0x00f000f0u) | 0x54005400u, 0x54005400u), step, lo);      // 64 + c, less 64
  v[2] = fma_f16x2(sub_f16x2((u & 0x000f000fu) | 0x64006400u, 0x64006400u), step, lo);
  v[3] = fma_f16x2(sub_f16x2((u & 0x00f000f0u) | 0x54005400u, 0x54005400u), step, lo);
}

// A tile's rows token by token in fp32, four rows to a warp: for tiles whose numbers differ too much in size. Keys and values are halved or smaller on the
// way, since lo + 15 * step may lie outside fp32. (Four chunks of 256 queries over 4096 tokens, all tiles this way: 11 ms against 0.15. Ordinary models'
// keys and values lie within a factor of a hundred.)
template <int D>
__device__ __noinline__ void attend_plainly(const WideParams& p, const SequenceRows& seq, uint32_t b, uint32_t head, uint32_t row0, uint32_t rows) {
  constexpr int TYPE = QSGD_TYPE_BF16, V = D / 32, J = D / 64, kTogether = 4;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, j = lane * V / 64, byte = lane * V % 64 / 2;
#pragma unroll 1
  for (uint32_t r0 = warp * kTogether; r0 < rows; r0 += kThreads / 32 * kTogether) {
    float q[kTogether][V], o[kTogether][V], top[kTogether], l[kTogether];
    uint32_t see[kTogether], most = 0;
#pragma unroll
    for (int x = 0; x < kTogether; ++x) {
      const bool live = r0 + x < rows;
      const uint32_t query = (row0 + r0 + x) / p.group, hh = head * p.group + (row0 + r0 + x) - query * p.group;
      const int64_t far = live ? seq.length - (int64_t)(seq.n - 1 - query) : 0;
      see[x] = far > 0 ? (uint32_t)far : 0u;
      most = see[x] > most ? see[x] : most;
      const uint16_t* const src = p.q + (uint64_t)(seq.start + query) * p.q_token + (uint64_t)hh * p.q_head + lane * V;
#pragma unroll
      for (int y = 0; y < V; ++y) { q[x][y] = live ? from_bits16<TYPE>(__ldg(src + y)) : 0.0f; o[x][y] = 0.0f; }
      top[x] = kNoMax;
      l[x] = 0.0f;
    }
#pragma unroll 1
    for (uint32_t t0 = 0; t0 < most; t0 += kCacheTile) {
      const uint32_t tile = t0 / kCacheTile, page = tile / p.c.page_tiles;
      int32_t at = __ldg(p.c.table + (uint64_t)b * p.c.table_stride + page);
      if (at < 0 || (uint32_t)at >= p.c.n_pages) at = 0;    // (said by the role that brings the tiles in)
      const uint8_t* const held = p.c.data + (uint64_t)at * p.c.page_stride + (uint64_t)head * p.c.head_stride +
                                  (uint64_t)(tile - page * p.c.page_tiles) * Shape<D>::kTile;
      const uint32_t end = most - t0 < kCacheTile ? most - t0 : kCacheTile;
#pragma unroll 2
      for (uint32_t slot = 0; slot < end; ++slot) {
        float kv[2][V];                                     // half a key, and p.times a value
#pragma unroll
        for (int side = 0; side < 2; ++side) {
          const uint8_t* const part = held + side * 9 * D;
          const uint32_t pair = __ldg(reinterpret_cast<const uint32_t*>(part + 8 * D) + slot * J + j);
          const uint8_t* const codes = part + (j * 16 + slot) * 32 + byte;
          const uint32_t word = V == 4 ? (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(codes)) : (uint32_t)__ldg(codes);
          const float by = side ? p.times : 0.5f, lo = from_bits16<TYPE>(pair & 0xffffu) * by, step = from_bits16<TYPE>(pair >> 16) * by;
#pragma unroll
          for (int y = 0; y < V; ++y) kv[side][y] = fmaf(step, (float)((word >> (4 * y)) & 15u), lo);
        }
#pragma unroll
        for (int x = 0; x < kTogether; ++x) {
          float s = 0.0f;
#pragma unroll
          for (int y = 0; y < V; ++y) s = fmaf(q[x][y], kv[0][y], s);
#pragma unroll
          for (int m = 1; m < 32; m <<= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
          if (t0 + slot < see[x]) {
            s *= 2.0f * p.scale_log2;
            const float high = fmaxf(top[x], s), f = exp2_approx(top[x] - high), e = exp2_approx(s - high);
            top[x] = high;
            l[x] = fmaf(l[x], f, e);
#pragma unroll
            for (int y = 0; y < V; ++y) o[x][y] = fmaf(e, kv[1][y], o[x][y] * f);
          }
        }
      }
    }
#pragma unroll
    for (int x = 0; x < kTogether; ++x) {
      if (r0 + x >= rows) continue;
      const uint32_t query = (row0 + r0 + x) / p.group, hh = head * p.group + (row0 + r0 + x) - query * p.group;
      const uint64_t row = (uint64_t)seq.start + query;
      uint16_t* const out = p.out + row * p.out_token + (uint64_t)hh * p.out_head + lane * V;
      const float over = see[x] ? 1.0f / l[x] : 0.0f;
#pragma unroll
      for (int y = 0; y < V; ++y) out[y] = (uint16_t)to_bits16<TYPE>(see[x] ? o[x][y] * over * p.back : 0.0f);
      if (p.lse && lane == 0) p.lse[row * p.q_heads + hh] = see[x] ? (top[x] + log2f(l[x])) * 0.69314718055994531f : -INFINITY;
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) cache_attend_wide_kernel(const __grid_constant__ WideParams p) {
  using S = Shape<D>;
  constexpr int J = S::kGroups;
  constexpr int TYPE = QSGD_TYPE_BF16;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars[2 * kRawStages + 2 * kValues + 2 * kPairs + 13];
  __shared__ uint64_t scan[kThreads / 32];
  __shared__ uint64_t found_base;
  __shared__ uint32_t found_b, tmem_base, given_up;
  __shared__ uint32_t far_apart;                           // numbers too far apart for the tile: attend_plainly does it again
  __shared__ int32_t length_of[kMostSorted];
  __shared__ uint32_t order[kMostSorted];
  __shared__ float key_back[8], value_size[8];             // of a step's keys: what undoes their scaling; of its values: the power of two below the largest, or 0
  __shared__ uint2 key_pair[kPairs][kStep * J];                 // (step, step), (lo, lo) in fp16
  __shared__ uint32_t value_pair[kPairs][kStep * J];            // step, lo
  __shared__ float row_max[2][kRows], row_sum[2][kRows], row_cap[2][kRows];
  __shared__ uint32_t row_nan[2][kRows];
  __shared__ uint8_t poison[8][kStep];                     // groups of a token's values that hold what is no number
  __shared__ uint32_t poisoned[8];                         // (of eight steps: the pairs may be seven ahead of the softmax)
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  const Waits waits{&given_up, p.polls};
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const mem = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar0 = smem_u32(bars);
  const uint32_t raw_full = bar0, raw_empty = raw_full + 8 * kRawStages, k_full = raw_empty + 8 * kRawStages, k_empty = k_full + 16,
                 v_full = k_empty + 16, v_empty = v_full + 8 * kValues, s_full = v_empty + 8 * kValues, s_empty = s_full + 16, p_full = s_empty + 16, pv = p_full + 16,
                 q_full = pv + 16, pairs_full = q_full + 8, pairs_empty = pairs_full + 8 * kPairs;
  if (tid == 0) {
    for (uint32_t s = 0; s < kRawStages; ++s) { mbar_init(raw_full + 8 * s, 1); mbar_init(raw_empty + 8 * s, kUnpackWarps); }
    for (uint32_t s = 0; s < 2; ++s) {
      mbar_init(k_full + 8 * s, kUnpackWarps / 2); mbar_init(k_empty + 8 * s, 1);
      mbar_init(s_full + 8 * s, 1); mbar_init(s_empty + 8 * s, kSoftmaxWarps / 2);
    }
    for (uint32_t s = 0; s < 2; ++s) {
      mbar_init(p_full + 8 * s, kSoftmaxWarps / 2);
      mbar_init(pv + 8 * s, 1);                             // a product P V is done
    }
    mbar_init(q_full, kSoftmaxWarps);
    for (uint32_t s = 0; s < kPairs; ++s) { mbar_init(pairs_full + 8 * s, 2); mbar_init(pairs_empty + 8 * s, kUnpackWarps); }
    for (uint32_t s = 0; s < kValues; ++s) { mbar_init(v_full + 8 * s, kUnpackWarps / 2); mbar_init(v_empty + 8 * s, 1); }
    given_up = far_apart = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(S::kTmem) : "memory");
  chain_wait();

  // ---- which rows of which sequence -----------------------------------------------------------------------------------
  // Items in the order of the sequences' lengths, the longest first, as long as those are few: CTAs are placed in their order, and the last ones to
  // start should be short. (Four sequences of 700 to 4096 tokens as they came: 122 us against 97.)
  const uint32_t item = blockIdx.x;
  const bool sorted = p.c.sequences <= kMostSorted;
  if (sorted) {
    if (tid < p.c.sequences) length_of[tid] = __ldg(p.c.lengths + tid);
    __syncthreads();
    if (tid < p.c.sequences) {
      const int32_t mine = length_of[tid];
      uint32_t rank = 0;
#pragma unroll 4
      for (uint32_t b = 0; b < p.c.sequences; ++b) rank += length_of[b] > mine || (length_of[b] == mine && b < tid);
      order[rank] = tid;
    }
    __syncthreads();
  }
  uint64_t before = 0;
  bool found = false;
  auto items_of = [&](uint32_t b, SequenceRows* s) -> uint32_t {
    bool bad;
    *s = rows_of(p.c, b, &bad);
    if (bad) atomicOr(p.c.status, QSGD_DEV_PAGE);
    return p.c.heads * ((s->n * p.group + kRows - 1) / kRows);
  };
  for (uint32_t b0 = 0; b0 < p.c.sequences && !found; b0 += kThreads) {
    SequenceRows s;
    const uint32_t at = b0 + tid, b = at < p.c.sequences ? (sorted ? order[at] : at) : 0u;
    const uint32_t mine = at < p.c.sequences ? items_of(b, &s) : 0u;
    uint64_t sum = mine;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const uint64_t up = __shfl_up_sync(0xffffffffu, sum, m);
      if (lane >= (uint32_t)m) sum += up;
    }
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    uint64_t here = before + sum - mine, all = before;
#pragma unroll 1
    for (uint32_t w = 0; w < kThreads / 32; ++w) {
      if (w < warp) here += scan[w];
      all += scan[w];
    }
    if (here <= item && item < here + mine) { found_base = here; found_b = b; }
    found = item < all;
    before = all;
    __syncthreads();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_base, tmem_o = tmem + 2 * kStep;
  uint32_t steps = 0, see_any = 0, head = 0, row0 = 0, rows = 0;
  SequenceRows seq{};
  if (found) {
    bool bad;
    seq = rows_of(p.c, found_b, &bad);
    const uint32_t row_tiles = (seq.n * p.group + kRows - 1) / kRows, at = (uint32_t)(item - found_base);
    head = at / row_tiles;
    row0 = (at - head * row_tiles) * kRows;
    rows = seq.n * p.group - row0 < kRows ? seq.n * p.group - row0 : kRows;
    const int64_t any = seq.length - (int64_t)(seq.n - 1 - (row0 + rows - 1) / p.group);
    see_any = any > 0 ? (uint32_t)any : 0u;
    steps = (see_any + kStep - 1) / kStep;
  }

  if (warp == 0) {                                          // ---- packed tiles in -------------------------------------------------
    const uint32_t tiles = (see_any + kCacheTile - 1) / kCacheTile;
    auto look_up = [&](uint32_t tile) -> const uint8_t* {   // by lanes 0 to 3
      if (lane >= 4 || tile >= tiles) return nullptr;
      const uint32_t page = tile / p.c.page_tiles;
      int32_t at = __ldg(p.c.table + (uint64_t)found_b * p.c.table_stride + page);
      if (at < 0 || (uint32_t)at >= p.c.n_pages) { atomicOr(p.c.status, QSGD_DEV_PAGE); at = 0; }
      return p.c.data + (uint64_t)at * p.c.page_stride + (uint64_t)head * p.c.head_stride + (uint64_t)(tile - page * p.c.page_tiles) * S::kTile;
    };
    const uint8_t* next = look_up(lane);
    uint32_t i = 0;
#pragma unroll 1
    for (; i < steps; ++i) {
      const uint8_t* const src = next;
      next = look_up(4 * (i + 1) + lane);
      const uint32_t s = i % kRawStages, round = i / kRawStages;
      const bool fine = i < kRawStages || mbar_wait(raw_empty + 8 * s, (round - 1) & 1u, waits);
      if (!__all_sync(0xffffffffu, fine)) break;
      const uint32_t have = tiles - 4 * i < 4 ? tiles - 4 * i : 4u;
      if (lane == 0)
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(raw_full + 8 * s), "r"(have * S::kTile) : "memory");
      __syncwarp();
      if (src)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                         base + S::kAtRaw + s * S::kRaw + lane * S::kTile), "l"(src), "r"(S::kTile), "r"(raw_full + 8 * s) : "memory");
    }
    // What is in flight lands before the CTA's shared memory goes away, whether anybody still waits for it or not.
    for (uint32_t back = 1; back <= kRawStages && back <= i; ++back) {
      const uint32_t fill = i - back;
#pragma unroll 1
      for (uint32_t t = 0; t < kDrainPolls && !mbar_try(raw_full + 8 * (fill % kRawStages), (fill / kRawStages) & 1u); ++t) {}
    }
  } else if (warp == 1) {                                   // ---- the products ------------------------------------------------------
    if (steps) {                                            // (the whole warp goes round, so that addresses are in uniform registers, and one lane issues:
                                                            // 133 us against 161 with one lane in the loop)
      constexpr uint32_t idesc_s = (1u << 4) | ((kStep >> 3) << 17) | ((kRows >> 4) << 24);        // fp32 += fp16 * fp16
      constexpr uint32_t idesc_o = (1u << 4) | ((D >> 3) << 17) | ((kRows >> 4) << 24);
      bool fine = __all_sync(0xffffffffu, mbar_wait(q_full, 0, waits));
      uint32_t issued = 0, done = 0;                        // products Q K^T, P V issued
      // S of a step as soon as its keys are there and S of the step before the last one has been read, O of a step as soon as P is there: whichever
      // can go first, since the two halves of the softmax warps run by themselves.
      uint32_t idle = 0;
#pragma unroll 1
      while (fine && done < steps) {
        const uint32_t bs = issued & 1u, bo = done & 1u;
        bool moved = false;
        if (issued < steps && __all_sync(0xffffffffu, mbar_test(k_full + 8 * bs, (issued >> 1) & 1u) &&
                                                          (issued < 2 || mbar_test(s_empty + 8 * bs, ((issued >> 1) - 1) & 1u)))) {
          if (elected()) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (uint32_t x = 0; x < D / 16; ++x)
              mma_f16(tmem + bs * kStep, tile_desc(base + (x / 4) * (kRows * 128)) + 2 * (x % 4),
                      tile_desc(base + S::kAtK + bs * S::kK + (x / 4) * (kStep * 128)) + 2 * (x % 4), idesc_s, x != 0);
            tc_commit(k_empty + 8 * bs);
            tc_commit(s_full + 8 * bs);
          }
          __syncwarp();
          ++issued;
          moved = true;
        }
        if (done < issued && __all_sync(0xffffffffu, mbar_test(v_full + 8 * (done % kValues), (done / kValues) & 1u) &&
                                                         mbar_test(p_full + 8 * bo, (done >> 1) & 1u))) {
          if (elected()) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t pa = tile_desc(base + S::kAtP + bo * S::kP), vb = tile_desc(base + S::kAtV + (done % kValues) * S::kV);
#pragma unroll
            for (uint32_t x = 0; x < kStep / 16; ++x) mma_f16(tmem_o + bo * D, pa + 2 * x, vb + 2 * x, idesc_o, done >= 2 || x != 0);
            tc_commit(v_empty + 8 * (done % kValues));
            tc_commit(pv + 8 * bo);
          }
          __syncwarp();
          ++done;
          moved = true;
        }
        idle = moved ? 0u : idle + 1;
        if (idle >= waits.polls || ((idle & 63u) == 63u && __any_sync(0xffffffffu, given_up_now(waits)))) fine = false;
      }
      if (!fine) *waits.given_up = 1;
      if (!fine && issued) {                                     // products in flight are done before tensor memory is freed
#pragma unroll 1
        for (uint32_t t = 0; t < kDrainPolls && !mbar_try(k_empty + 8 * ((issued - 1) & 1u), ((issued - 1) >> 1) & 1u); ++t) {}
#pragma unroll 1
        for (uint32_t t = 0; done && t < kDrainPolls && !mbar_try(pv + 8 * ((done - 1) & 1u), ((done - 1) >> 1) & 1u); ++t) {}
      }
    }
  } else if (warp < 4) {                                    // ---- pairs: warp 2 the keys', warp 3 the values' ---------------------
    const bool value = warp == 3;
#pragma unroll 1
    for (uint32_t i = 0; i < steps; ++i) {
      const uint32_t b = i % kPairs, s = i % kRawStages;
      const uint32_t first = i * kStep, have = see_any - first < kStep ? see_any - first : kStep;     // tokens of the step that some row sees
      bool fine = mbar_wait(raw_full + 8 * s, (i / kRawStages) & 1u, waits);
      fine = fine && (i < kPairs || mbar_wait(pairs_empty + 8 * b, (i / kPairs - 1) & 1u, waits));
      if (!__all_sync(0xffffffffu, fine)) break;
      const uint8_t* const raw = mem + S::kAtRaw + s * S::kRaw + (value ? 17 : 8) * D;
      float largest = 0.0f, smallest = FLT_MAX;             // (the groups' largest numbers)
      uint32_t pair[2][J];
      bool bad = false;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint32_t token = lane + 32 * x;
        uint32_t groups = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          pair[x][j] = token < have ? *reinterpret_cast<const uint32_t*>(raw + (token >> 4) * S::kTile + ((token & 15u) * J + j) * 4) : 0u;
          const float lo = from_bits16<TYPE>(pair[x][j] & 0xffffu);
          const float size = fmaxf(fabsf(lo), fabsf(fmaf(15.0f, from_bits16<TYPE>(pair[x][j] >> 16), lo)));
          largest = fmaxf(largest, size);
          if (size > 0.0f) smallest = fminf(smallest, size);
          if (value && lo != lo) {                          // no number: zeros here, and the rows that see it are told
            groups |= 1u << j;
            pair[x][j] = 0;
          }
        }
        if (value) poison[i & 7u][token] = (uint8_t)groups;
        bad |= groups != 0;
      }
      largest = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(largest)));
      smallest = __uint_as_float(__reduce_min_sync(0xffffffffu, __float_as_uint(smallest)));
      if (lane == 0 && (largest > smallest * (value ? kValueRange : kKeyRange) || largest >= (value ? kMostValue : INFINITY))) far_apart = 1;
      const int32_t up = lift(largest, 14);
      const float times = power2(up);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const float lo = from_bits16<TYPE>(pair[x][j] & 0xffffu) * times, step = from_bits16<TYPE>(pair[x][j] >> 16) * times;
          const uint32_t at = (lane + 32 * x) * J + j;
          if (value) value_pair[b][at] = pack16<QSGD_TYPE_F16>(step, lo);
          else key_pair[b][at] = make_uint2(pack16<QSGD_TYPE_F16>(step, step), pack16<QSGD_TYPE_F16>(lo, lo));
        }
      const bool any = __any_sync(0xffffffffu, bad);
      if (lane == 0) {
        if (value) { value_size[i & 7u] = largest > 0.0f ? power2(14 - up) : 0.0f; poisoned[i & 7u] = any; }
        else key_back[i & 7u] = power2(-up);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(pairs_full + 8 * b);
    }
  } else if (warp >= 12) {                                  // ---- unpacking ---------------------------------------------------------
    const bool value = warp >= 16;
#pragma unroll 1
    for (uint32_t i = 0; i < steps; ++i) {
      const uint32_t b = i & 1u, s = i % kRawStages, vs = i % kValues, ps = i % kPairs;
      const uint32_t first = i * kStep, have = see_any - first < kStep ? see_any - first : kStep;
      bool fine = mbar_wait(pairs_full + 8 * ps, (i / kPairs) & 1u, waits) && mbar_wait(raw_full + 8 * s, (i / kRawStages) & 1u, waits);
      if (value) fine = fine && (i < kValues || mbar_wait(v_empty + 8 * vs, (i / kValues - 1) & 1u, waits));
      else fine = fine && (i < 2 || mbar_wait(k_empty + 8 * b, ((i >> 1) - 1) & 1u, waits));
      if (!__all_sync(0xffffffffu, fine)) break;
      const uint8_t* const raw = mem + S::kAtRaw + s * S::kRaw;
      if (!value) {
        // Keys: a thread has half the words (of 8 coordinates) of one token; a word becomes 16 bytes of the token's row, in the order that the
        // queries have too (0 4 1 5 2 6 3 7).
        const uint32_t ut = tid - 384, token = ut & 63u, part = ut >> 6;
        constexpr int kWords = D / 16;
        const int j = (int)(part * kWords) / 8;
        const uint32_t word0 = part * kWords - 8 * j;
        const uint2 pair = key_pair[ps][token * J + j];
        const uint8_t* const src = raw + (token >> 4) * S::kTile + (j * 16 + (token & 15u)) * 32 + word0 * 4;
        uint8_t* const row = mem + S::kAtK + b * S::kK + j * (kStep * 128) + token * 128;
        uint4 c[kWords / 4];
#pragma unroll
        for (int x = 0; x < kWords / 4; ++x) c[x] = token < have ? *reinterpret_cast<const uint4*>(src + 16 * x) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int x = 0; x < kWords; ++x) {
          const uint4& q = c[x / 4];
          uint32_t v[4];
          values_of(x % 4 == 0 ? q.x : x % 4 == 1 ? q.y : x % 4 == 2 ? q.z : q.w, pair.x, pair.y, v);
          *reinterpret_cast<uint4*>(row + (((word0 + x) ^ (token & 7u)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
      } else {
        // Values: a lane has two tokens, 16 apart (so that a warp's reads of the codes meet fewer banks twice; P's columns are in the same order), a
        // warp a quarter of their words; a word becomes pairs in 8 coordinates' rows.
        const uint32_t w = warp - 16, token = (lane & 15u) + 2 * (lane & 16u);
        constexpr int kWords = 2 * J;
        const int j = (int)(w * kWords) / 8;
        const uint32_t word0 = w * kWords - 8 * j;
        const uint32_t pair0 = value_pair[ps][token * J + j], pair1 = value_pair[ps][(token + 16) * J + j];
        const uint32_t step = __byte_perm(pair0, pair1, 0x5410), lo = __byte_perm(pair0, pair1, 0x7632);
        const uint8_t* const src = raw + (token >> 4) * S::kTile + 9 * D + (j * 16 + (token & 15u)) * 32 + word0 * 4;
        uint8_t* const to = mem + S::kAtV + vs * S::kV + (lane & 3u) * 4;
        uint2 c0[J], c1[J];
#pragma unroll
        for (int x = 0; x < J; ++x) {
          c0[x] = token < have ? *reinterpret_cast<const uint2*>(src + 8 * x) : make_uint2(0u, 0u);
          c1[x] = token + 16 < have ? *reinterpret_cast<const uint2*>(src + S::kTile + 8 * x) : make_uint2(0u, 0u);
        }
#pragma unroll
        for (int x = 0; x < kWords; ++x) {
          const uint32_t w0 = x % 2 ? c0[x / 2].y : c0[x / 2].x, w1 = x % 2 ? c1[x / 2].y : c1[x / 2].x;
          uint32_t front[4], behind[4];
          values_of(__byte_perm(w0, w1, 0x5410), step, lo, front);
          values_of(__byte_perm(w0, w1, 0x7632), step, lo, behind);
          uint8_t* const row = to + (64 * j + 8 * (word0 + x)) * 128;
#pragma unroll
          for (uint32_t y = 0; y < 4; ++y) {
            *reinterpret_cast<uint32_t*>(row + y * 128 + (((lane >> 2) ^ y) << 4)) = front[y];
            *reinterpret_cast<uint32_t*>(row + (y + 4) * 128 + (((lane >> 2) ^ (y + 4)) << 4)) = behind[y];
          }
        }
      }
      async_fence();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(value ? v_full + 8 * vs : k_full + 8 * b);
        mbar_arrive(pairs_empty + 8 * ps);
        mbar_arrive(raw_empty + 8 * s);
      }
    }
  } else {                                                  // ---- softmax -----------------------------------------------------------
    // A thread has a row; warps 4-7 take the even steps and warps 8-11 the odd ones, each with its own maximum, sum and O, joined at the end. (With
    // two threads to a row at every step each step waited for the latencies of the whole chain from S to P.)
    const uint32_t quarter = warp & 3u, r = 32 * quarter + lane, side = (warp - 4) >> 2, lanes = (32 * quarter) << 16;
    const uint32_t twins = 1 + quarter;                     // named barrier of the two warps that share their rows
    const bool live = r < rows;
    const uint32_t query = (row0 + r) / p.group, hh = head * p.group + (row0 + r) - query * p.group;
    // (A row that is not there sees what any other does: a warp without masks is a fifth faster, 366 us against 467 for 64 rows of 16384 tokens.)
    const int64_t far = live ? seq.length - (int64_t)(seq.n - 1 - query) : (int64_t)see_any;
    const uint32_t see = far > 0 ? (uint32_t)far : 0u;
    float factor = 0.0f, top = kNoMax, l = 0.0f, cap = kLeastCap;
    uint32_t nan_groups = 0;
    bool fine = true;
    if (steps) {
      // Half of the row of q, scaled, in the keys' order of coordinates.
      const uint16_t* const src = p.q + (uint64_t)(seq.start + query) * p.q_token + (uint64_t)hh * p.q_head;
      float largest = 0.0f;
#pragma unroll 1
      for (uint32_t j = 0; j < J; ++j) {
        float group = 0.0f;
#pragma unroll 2
        for (uint32_t c = 8 * j; c < 8 * j + 8; ++c) {
          const uint4 x = live ? __ldg(reinterpret_cast<const uint4*>(src + 8 * c)) : make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int y = 0; y < 4; ++y) group = fmaxf(group, fmaxf(fabsf(from_bits16<TYPE>(w[y] & 0xffffu)), fabsf(from_bits16<TYPE>(w[y] >> 16))));
        }
        // (One of zeros has no say. The largest so far of two is the other one.)
        if (j && group > 0.0f && largest > 0.0f && fmaxf(group, largest) > kQueryRange * fminf(group, largest)) far_apart = 1;
        largest = fmaxf(largest, group);
      }
      const int32_t up = lift(largest, 11);
      const float times = power2(up);
      factor = p.scale_log2 * power2(-up);
#pragma unroll 1
      for (uint32_t c = side * (D / 16); c < (side + 1) * (D / 16); ++c) {
        const uint4 x = live ? __ldg(reinterpret_cast<const uint4*>(src + 8 * c)) : make_uint4(0, 0, 0, 0);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        float v[8];
#pragma unroll
        for (int y = 0; y < 4; ++y) { v[2 * y] = from_bits16<TYPE>(w[y] & 0xffffu) * times; v[2 * y + 1] = from_bits16<TYPE>(w[y] >> 16) * times; }
        *reinterpret_cast<uint4*>(mem + (c >> 3) * (kRows * 128) + r * 128 + (((c & 7u) ^ (r & 7u)) << 4)) =
            make_uint4(pack16<QSGD_TYPE_F16>(v[0], v[4]), pack16<QSGD_TYPE_F16>(v[1], v[5]), pack16<QSGD_TYPE_F16>(v[2], v[6]),
                       pack16<QSGD_TYPE_F16>(v[3], v[7]));
      }
      async_fence();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
    }
#pragma unroll 1
    for (uint32_t i = side; i < steps; i += 2) {
      const uint32_t round = i >> 1, first = i * kStep;
      fine = __all_sync(0xffffffffu, mbar_wait(s_full + 8 * side, round & 1u, waits));        // (the keys are unpacked, so both kinds' pairs have been seen to)
      if (!fine) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      float sc[kStep];
      tmem_load64(tmem + side * kStep + lanes, sc);
      const float scale = factor * key_back[i & 7u];
      float size = value_size[i & 7u];
      if (size == 0.0f) size = cap;                         // values that are all zero are of any size
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(s_empty + 8 * side);
      // The largest of scale * s: with a negative scale it comes from the smallest.
      float times = fabsf(scale);
      if (!(scale > 0.0f)) {
        const float turn = scale < 0.0f ? -1.0f : scale;    // (a scale of zero: products of zero, from here on by a scale of one)
#pragma unroll
        for (int x = 0; x < (int)kStep; ++x) sc[x] *= turn;
        if (scale == 0.0f) times = 1.0f;
      }
      if (first + kStep > see) {
#pragma unroll
        for (int x = 0; x < (int)kStep; ++x)
          if (first + x >= see) sc[x] = -INFINITY;
      }
      float highs[4] = {sc[0], sc[1], sc[2], sc[3]};
#pragma unroll
      for (int x = 4; x < (int)kStep; ++x) highs[x & 3] = fmaxf(highs[x & 3], sc[x]);
      float high = fmaxf(fmaxf(highs[0], highs[1]), fmaxf(highs[2], highs[3])) * times;
      if (poisoned[i & 7u]) {
#pragma unroll 1
        for (uint32_t x = 0; x < kStep; ++x)
          if (first + x < see) nan_groups |= poison[i & 7u][x];
      }
      if (high == -INFINITY) high = kNoMax;                 // nothing seen
      // cap, a power of two of the row's own, follows its largest p * size: what it does not see, or hardly weighs, does not count.
      const bool higher = high > top + 8.0f;
      const float most = higher ? size : exp2_approx(high - top - 8.0f) * size;       // (2^-8 of the largest where the maximum stays: p is 2^8 at most)
      const bool raise = higher || most > cap;
      float f = 1.0f;
      if (raise) {
        float held = cap;
        if (higher) {
          f = exp2_approx(top - high);
          l *= f;
          held *= f;
          top = high;
          if (!(fabsf(top) <= kMostScore)) far_apart = 1;   // (the sum of it and of a shift would not be exact enough)
        }
        cap = power_above(fminf(fmaxf(fmaxf(held, higher ? most : 256.0f * most), kLeastCap), kMostCap));
        f = held * inverse_of_power(cap);                   // (1 at most)
      }
      // P holds p * 2^7 * size / cap: at most 2^15, and 2^-14, where fp16 begins to lose bits, for p * size = 2^-21 * cap. (Below 2^-60 p itself would
      // leave fp32; P is zero long before.)
      int32_t shift = (int32_t)(__float_as_uint(size) >> 23) - (int32_t)(__float_as_uint(cap) >> 23) + 7;
      if (shift < -60) shift = -60;
      const float off = (float)shift - top;
      // The product before this one of the same half reads the same buffer of P, and adds to the same O.
      if (round) {
        fine = __all_sync(0xffffffffu, mbar_wait_here(pv + 8 * side, (round - 1) & 1u, waits));
        if (!fine) break;
        if (__any_sync(0xffffffffu, raise)) {
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
          for (uint32_t c = 0; c < D; c += 16) {            // (as many as find room in registers beside the scores)
            float o[16];
            tmem_load16(tmem_o + side * D + c + lanes, o);
#pragma unroll
            for (int x = 0; x < 16; ++x) o[x] *= f;
            tmem_store16(tmem_o + side * D + c + lanes, o);
          }
        }
      }
      float sums[2] = {0.0f, 0.0f};
#pragma unroll
      for (uint32_t c = 0; c < 8; ++c) {                    // 16 bytes: tokens x and x + 16, as the values' columns
        uint32_t packed[4];
#pragma unroll
        for (uint32_t y = 0; y < 4; ++y) {
          const uint32_t x = 32 * (c >> 2) + 4 * (c & 3u) + y;
          const float p0 = exp2_approx(fmaf(sc[x], times, off)), p1 = exp2_approx(fmaf(sc[x + 16], times, off));
          sums[y & 1u] += p0 + p1;
          packed[y] = pack16<QSGD_TYPE_F16>(p0, p1);
        }
        *reinterpret_cast<uint4*>(mem + S::kAtP + side * S::kP + r * 128 + ((c ^ (r & 7u)) << 4)) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
      }
      l = fmaf(sums[0] + sums[1], power2(shift < 126 ? -shift : -126), l);       // (from there on p is nothing beside l)
      async_fence();
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full + 8 * side);
    }
    // A half waits for its own products, whose phases it has followed: of the other half's it has seen none, and a wait for a phase by its parity is over at
    // once when an earlier one of the same parity is. That those are done it learns from its twins at the barrier, where the halves' maxima, sums and
    // sizes change hands, too. Each writes half of the coordinates.
    const uint32_t turns = (steps + 1 - side) / 2;
    if (turns) fine = fine && mbar_wait(pv + 8 * side, (turns - 1) & 1u, waits);
    fine = __all_sync(0xffffffffu, fine);
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    row_max[side][r] = top;
    row_sum[side][r] = l;
    row_cap[side][r] = cap;
    row_nan[side][r] = nan_groups;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    fine = meet(twins, fine);
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const float high = fmaxf(row_max[0][r], row_max[1][r]), e0 = exp2_approx(row_max[0][r] - high), e1 = exp2_approx(row_max[1][r] - high);
    l = fmaf(row_sum[0][r], e0, row_sum[1][r] * e1);        // (the same in both)
    top = high;
    nan_groups = row_nan[0][r] | row_nan[1][r];
    if (fine && found && !*(volatile uint32_t*)&far_apart) {
      const uint64_t row = (uint64_t)seq.start + query;
      uint16_t* const out = p.out + row * p.out_token + (uint64_t)hh * p.out_head;
      const bool saw = see != 0;
      // O is sum (p 2^7 size / cap) (v 2^14 / size). (The division first: a sum that is not divided may lie outside fp32, and 2^-21 cap below its range.)
      const float w0 = e0 / l, w1 = e1 / l, back0 = row_cap[0][r] * power2(-21), back1 = row_cap[1][r] * power2(-21);
#pragma unroll 1
      for (uint32_t c = side * (D / 2); c < (side + 1) * (D / 2); c += 16) {
        float o[16], o1[16] = {};
        if (steps) tmem_load16(tmem_o + c + lanes, o);
        if (steps > 1) tmem_load16(tmem_o + D + c + lanes, o1);
        if (live) {
          const float nan = nan_groups >> (c / 64) & 1u ? NAN : 0.0f;
#pragma unroll
          for (int x = 0; x < 16; ++x) o[x] = saw ? o[x] * w0 * back0 + o1[x] * w1 * back1 + nan : 0.0f;
#pragma unroll
          for (int x = 0; x < 16; x += 8)
            *reinterpret_cast<uint4*>(out + c + x) =
                make_uint4(pack16<TYPE>(o[x], o[x + 1]), pack16<TYPE>(o[x + 2], o[x + 3]), pack16<TYPE>(o[x + 4], o[x + 5]), pack16<TYPE>(o[x + 6], o[x + 7]));
        }
        __syncwarp();
      }
      if (live && side == 0 && p.lse) p.lse[row * p.q_heads + hh] = saw ? (top + log2f(l)) * 0.69314718055994531f : -INFINITY;
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 0) {
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmem));
  }
  if (tid == 0 && given_up) atomicOr(p.c.status, QSGD_DEV_TIMEOUT);
  if (far_apart && !given_up) attend_plainly<D>(p, seq, found_b, head, row0, rows);
}

template <int D>
int look_up(int* sms) {
  static KernelSite site;
  int occ = 0;
  return site.lookup(cache_attend_wide_kernel<D>, kThreads, Shape<D>::kSmem, sms, &occ);
}

template <int D>
int launch_wide(const WideParams& p, cudaStream_t stream) {
  int sms = 0;
  const int st = look_up<D>(&sms);
  if (st) return st;
  // At most this many row tiles: where the sequences' rows end inside one is known on the device only.
  const uint64_t ctas = (uint64_t)p.c.heads * ((uint64_t)p.c.rows * p.group / kRows + p.c.sequences);
  ScopedKernel sk(kKernCacheAttend, stream);
  return (int)launch_chained(cache_attend_wide_kernel<D>, (uint32_t)ctas, kThreads, Shape<D>::kSmem, stream, p);
}

}  // namespace

// A CTA has a row tile for itself, and all of its tokens, so that few tiles leave SMs idle, while cache_attend.cu spreads any rows over all SMs. A round of
// tiles over the SMs takes 43, 131 and 247 us for 2048, 8192 and 16384 tokens at head size 128, however few or empty the tiles are; cache_attend.cu
// 46, 114 and 212 for 4096 rows in all heads, 48, 126 and 236 for 4608, and 69, 213 and 406 for 8192. At head size 64: 35, 109 and 208 against 30, 73 and
// 132 for 4608 rows, 42, 120 and 224 for 8192. So the rows have to fill that part of the rounds' room, 18944 on 148 SMs, from which on it pays. (The rows'
// average counts: one kernel has the whole call, a long run and single tokens beside it too.)
bool cache_attend_wide_takes(const CacheView& view, uint32_t head_dim, int type, uint32_t q_heads) {
  if (type != QSGD_TYPE_BF16 || (head_dim != 64 && head_dim != 128) || !view.starts || !view.sequences) return false;
  const uint64_t rows = (uint64_t)view.rows * (q_heads / view.heads);        // of a key head
  if ((rows / kRows + view.sequences) * view.heads >= (1ull << 31)) return false;
  int sms = 0;
  if ((head_dim == 64 ? look_up<64>(&sms) : look_up<128>(&sms)) || sms < 1) return false;
  const uint64_t each = (rows + view.sequences - 1) / view.sequences, tiles = (each + kRows - 1) / kRows * view.sequences * view.heads;
  const uint64_t room = (tiles + sms - 1) / sms * sms * kRows;
  return rows * view.heads * 24 >= room * (head_dim == 64 ? 10 : 7);
}

int launch_cache_attend_wide(const CacheView& view, uint32_t head_dim, const AttendArgs& a, cudaStream_t stream) {
  WideParams p;
  p.c = view;
  p.q = static_cast<const uint16_t*>(a.q);
  p.out = static_cast<uint16_t*>(a.out);
  p.q_token = a.q_token; p.q_head = a.q_head; p.out_token = a.out_token; p.out_head = a.out_head;
  p.lse = a.lse;
  p.q_heads = a.q_heads;
  p.group = a.q_heads / view.heads;
  p.scale_log2 = (float)((double)a.scale * 1.4426950408889634);
  p.polls = quantize_poll_limit();
  const int lost = attend_sums_lose(view);
  p.times = ldexpf(1.0f, -lost);
  p.back = ldexpf(1.0f, lost);
  return head_dim == 64 ? launch_wide<64>(p, stream) : launch_wide<128>(p, stream);
}

}  // namespace qsgd
