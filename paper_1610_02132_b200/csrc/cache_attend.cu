// Attention over the 4-bit cache.
//
// For a query row q (one head of one query), with keys k_t = lo + step * c_t (a group g of 64 coordinates has its own pair):
//   s_t = sum_g step_tg * (q_g . c_tg) + lo_tg * sum(q_g),   p_t = 2^(a s_t - m),   a = scale * log2(e),
//   o   = (sum_t p_t v_t) / sum_t p_t,    sum_t p_t v_tg = sum_t (p_t step_tg) (c_tg - 8) + sum_t p_t (lo_tg + 8 step_tg).
// The codes go to the tensor cores as they are and the pairs are applied in fp32:
//   scores   A = codes of 16 tokens, B = up to 8 query rows of one key head (m16n8k16, fp16 operands, fp32 sums). Each group of a row of q is multiplied
//            by a power of two that puts its largest number at 2^11: 16-bit numbers of either type fit fp16 then, but for what lies 2^-21 and more
//            below the group's largest, of which it keeps 2^-36.
//   output   A = codes of 16 coordinates x 16 tokens, B = p * step in fp16, times a power of two, of each row and group by itself, that puts the
//            largest p * step so far at 32 to 64 and is lowered only when one passes it by 2^9. It follows p * step and not step, each row's own:
//            a group beside a much larger one, a row in front of much larger values that it does not see, or sees with little weight, keep their bits.
//            (With one power of two for all, 2^24 between two groups' steps left nothing of the smaller one's output.)
//            For a bf16 output 11 bits of p are enough: a rounding of 2^-12 at most, next to 2^-9 of the output's own.
//            For fp16 p * step goes as the sum of two fp16 numbers, since one would put as much error into the output as rounding it does.
//            Both sums are held under that power of two, which no p * lo exceeds by more than 2^10 either, until they are divided: the values may
//            be as large as their type has them, the undivided sums then lie outside fp32.
//            The codes are centred here because these sums run over the whole sequence: 8 sum(p step) would grow until what is left
//            after taking it off at the end is the error of its rounded sums.
// A nibble in bits 4 to 7 of an fp16 number is c * 2^-20, below the normal ones: a mask and at most a shift each make the keys' operands. The values' are
// centred by a multiply-add that makes normal numbers of them, (c - 8) * 2^-9, so that a nibble may lie in the last four bits, too (c * 2^-24), and one
// shift does for four masks. The powers of two are undone in q's scale and in the output's at the end. (The tensor cores line products up by their exponents
// as written, 2^-14 for numbers below the normal ones, and drop what lies 2^24 below the largest: beside c * 2^-20 that is 2^-18 of the largest q, beside c * 2^-24
// it was 2^-14, an error of 10^-6 in fp16 scores and of 2^-13 * p * step in the output.)
// For 64 sequences of 100 to 8000 tokens, 8 heads of 128: nibbles moved into place under a bf16 exponent, p in two bf16 numbers 143 us; nibbles under the
// exponents of 1024 and 64 and a subtraction each 101; as now, with the -8 by a product with a constant operand 87; with an addition 84;
// as now, with powers of two of each row and group and these operands, 89 by 16 warps and 80 by 12.
// The rows of a score tile are permuted (token_of) so that the transpose of p between the two products is one movmatrix, and reads
// of codes from shared memory meet no bank twice.
//
// What bounds it: HBM holds 9/8 * head_dim bytes a token and head, each read once; issue slots and the integer pipe are nearly as busy (350 warp
// instructions per 16 tokens at head size 128, of which 104 unpack codes and pairs; issue 60 %, integer pipe 54 %, tensor pipe 21 %). 64 sequences of
// 16000 tokens: 271 us, 4.4 TB/s; the 2.9 us in front of the first copies and the 7 us behind the last tile are what shorter calls feel.
// So everything is arranged around the stream of tiles. The tiles of all (sequence, key
// head, row tile) segments form one line of units, kSegmentCost more to a segment for what starting one takes, and every WARP of the grid
// takes an equal stretch of it, whatever the lengths are, through a ring of its own that bulk copies fill. A segment inside a stretch is
// written out by its warp; what spans warps of a CTA is joined in shared memory; what spans CTAs leaves (m, sum, o) in the workspace,
// at most two parts a CTA, and a second kernel joins those. (With tiles dealt out to the eight warps of a CTA, which met at the end of each
// segment, 33 sequences of 17 to 1500 tokens with 16 heads took 85 us against 22, and 20 now: a CTA had up to 40 segments one after another.)
// Few and short segments need no such line: a cluster of CTAs has one each and joins it over its shared memory (one user's step, 1000 tokens, with
// the write in front of it: 11.5 us against 13.9).
#include <float.h>

#include "cache.cuh"

namespace qsgd {

namespace {

constexpr uint32_t kJoinWarps = 8, kJoinThreads = 32 * kJoinWarps;
constexpr uint32_t kMostCtas = 1024;      // what the workspace is laid out for
constexpr uint32_t kLeastStretch = 2;     // units of a warp's stretch at least, and of a CTA's
constexpr uint32_t kLeastCta = 8;
// Of a sequence at most to a CTA of a cluster: 8000 tokens take 13.6 us by a cluster of 8 and 15.4 by the line. And at least, before one more is worth it:
// 16 tokens take 6.4 us by one CTA and 7.6 by eight, 1000 take 11.5 and 8.8.
constexpr uint32_t kDirectTokens = 1024, kClusterTokens = 96;
constexpr uint32_t kMostCluster = 8, kMostDirect = 128;     // CTAs that share a segment, and all of those
// What a segment costs beside its tiles, in tiles. (Counted as 2, 4, 6 and 8: 64 users of 100 to 8000 tokens take 93.9, 84.4, 80.3 and 79.5 us, 128 of 50 to
// 2000 64.0, 55.7, 52.2 and 51.0, 64 of 4000 each 78.3, 77.7, 77.5 and 79.5, 33 of 17 to 1500 with 16 heads of 64 22.2, 20.9, 20.1 and 21.4.)
constexpr uint32_t kSegmentCost = 6;
constexpr uint32_t kMostRowTile = 16;
constexpr uint32_t kDrainPolls = 1u << 22;   // bound of the waits for copies in flight
constexpr float kLeastCap = 1.9259299443872359e-34f, kMostCap = 8.5070591730234616e+37f;     // 2^-112, 2^126
constexpr float kNoMax = -FLT_MAX;        // maximum of nothing: below any score, and finite, so that differences of maxima are numbers

template <bool V>
struct Constant { static constexpr bool value = V; };

struct Rows {                             // of a segment: which rows of which sequence
  uint32_t head, row0, rows;              // key head, first row (query * group + head in group), number of rows
  uint32_t start;                         // first query row of the sequence
};

struct Span {                             // of a segment in a CTA: where its first part lies, its first and last warp, whether it ends here (and began here)
  uint8_t slot, first, last, ends;
};

struct JoinInfo {                         // of the segment that a CTA's stretch begins inside of, written by every CTA of every call
  Rows rows;
  uint32_t parts, first;                  // CTAs from `first` on hold a part each; 0: another CTA says so, or there is none
  uint32_t unused[2];
};

struct AttendParams {
  CacheView c;
  const uint16_t* q;
  uint16_t* out;
  uint64_t q_token, q_head, out_token, out_head;
  float* lse;
  uint32_t q_heads, group;
  float scale_log2;
  uint32_t polls;                         // bound of the waits for tiles
  uint32_t direct;                        // CTAs, a cluster, to a segment (0: a line of units)
  // A segment's parts go with their sums times 2^-part_lost, so that all of them add up to no more than the largest value. (One power of two for all, from
  // the longest sequence that the table can name: with each part's own, in its maximum, scores of 2^27 left no room for it there.)
  float part_lost, part_times;
  JoinInfo* join;
  float* parts;                           // [CTA][2][rows * (dim + 2)]
};

__host__ __device__ constexpr size_t part_floats(uint32_t rows, uint32_t dim) { return (size_t)rows * (dim + 2); }

// Token of a tile that row r (of 8) of a score tile stands for; rows 8 .. 15 are the same behind 8. Lane (g, t) of a warp reads key
// codes of token token_of(g) and value codes of tokens token_of(2 t) and token_of(2 t + 1): both sets of four rows of 32 bytes that go
// together differ modulo 4.
__device__ __forceinline__ uint32_t token_of(uint32_t r) { return (0x57463120u >> (4 * r)) & 7u; }

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Waits for a phase, `polls` times at most (0: not at all) as long as the hardware suspends a thread that tries; false if that was not enough.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, uint32_t polls) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .u32 n;\n\t"
      "mov.u32 n, 0;\n\t"
      "setp.ne.u32 p, %3, 0;\n\t"
      "@!p bra done;\n\t"
      "again:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra done;\n\t"
      "add.u32 n, n, 1;\n\t"
      "setp.lt.u32 p, n, %3;\n\t"
      "@p bra again;\n\t"
      "setp.ne.u32 p, n, n;\n\t"
      "done:\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity), "r"(polls) : "memory");
  return ok != 0;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// From the same place in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ float cluster_load(uint32_t at, uint32_t rank) {
  float v;
  asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(v) : "r"(at), "r"(rank) : "memory");
  return v;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t at, uint32_t rank) {
  float4 v;
  asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [a];\n\t}"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at), "r"(rank) : "memory");
  return v;
}

// One lane's copies of one or two tiles into a stage, two places one behind the other.
__device__ __forceinline__ void copy_tiles(bool mine, uint32_t dst, const uint8_t* src0, const uint8_t* src1, uint32_t tile_bytes, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .u32 d, n;\n\t"
      "setp.ne.u32 p, %0, 0;\n\t"
      "setp.ne.and.u64 q, %3, 0, p;\n\t"
      "add.u32 d, %1, %4;\n\t"
      "selp.u32 n, %4, 0, q;\n\t"
      "add.u32 n, n, %4;\n\t"
      "@p mbarrier.arrive.expect_tx.shared::cta.b64 _, [%5], n;\n\t"
      "@p cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%1], [%2], %4, [%5];\n\t"
      "@q cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [d], [%3], %4, [%5];\n\t}"
      ::"r"((uint32_t)mine), "r"(dst), "l"(src0), "l"(src1), "r"(tile_bytes), "r"(bar) : "memory");
}

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

__device__ __forceinline__ float exp2_approx(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// Of either half by itself.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// What a power of two is held against: the step of a pair, or 2^-10 of its lo.
template <int TYPE>
__device__ __forceinline__ float size_of_pair(uint32_t pair) {
  return fmaxf(from_bits16<TYPE>(pair >> 16), fabsf(from_bits16<TYPE>(pair & 0xffffu)) * (1.0f / 1024.0f));
}

// The largest pair (as a number) of that size.
template <int TYPE>
__device__ __forceinline__ uint32_t pair_of_size(float size) {
  const float lo = size * 1024.0f, most = TYPE == QSGD_TYPE_F16 ? 65504.0f : 3.3895314e38f;
  return to_bits16<TYPE>(size < most ? size : most) << 16 | to_bits16<TYPE>(lo < most ? lo : most);
}
// Of a power of two from 2^-126 to 2^126.
__device__ __forceinline__ float inverse_of_power(float v) { return __uint_as_float((254u << 23) - __float_as_uint(v)); }

__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
// The codes of a word as fp16 pairs, pair s = nibble s of either half: c * 2^-20.
__device__ __forceinline__ void unpack(uint32_t w, uint32_t (&c)[4]) {
  c[0] = (w << 4) & 0x00f000f0u;
  c[1] = w & 0x00f000f0u;
  c[2] = (w >> 4) & 0x00f000f0u;
  c[3] = (w >> 8) & 0x00f000f0u;
}
// The same as (c - 8) * 2^-9, exact: c * 2^-24 or c * 2^-20, times 2^15 or 2^11, less 2^-6.
__device__ __forceinline__ void unpack_centred(uint32_t w, uint32_t (&c)[4]) {
  const uint32_t v = w >> 8;
  c[0] = fma_f16x2(w & 0x000f000fu, 0x78007800u, 0xa400a400u);
  c[1] = fma_f16x2(w & 0x00f000f0u, 0x68006800u, 0xa400a400u);
  c[2] = fma_f16x2(v & 0x000f000fu, 0x78007800u, 0xa400a400u);
  c[3] = fma_f16x2(v & 0x00f000f0u, 0x68006800u, 0xa400a400u);
}

template <int J>
__device__ __forceinline__ void load_pairs(const uint32_t* at, uint32_t (&v)[J]) {      // at: on a boundary of J words if that is a power of two
  if constexpr (J == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(at);
    v[0] = x.x; v[1] = x.y;
  } else if constexpr (J == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(at);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  } else {
#pragma unroll
    for (int j = 0; j < J; ++j) v[j] = at[j];
  }
}

// One sequence on the line of units.
struct Sequence {
  uint32_t b, start, n, tiles, row_tiles;
  int64_t length;
  uint64_t units;
};
template <int ROWS>
__device__ __forceinline__ Sequence sequence_at(const AttendParams& p, uint32_t b) {
  bool bad;
  const SequenceRows s = rows_of(p.c, b, &bad);
  if (bad) atomicOr(p.c.status, QSGD_DEV_PAGE);
  Sequence q;
  q.b = b; q.start = s.start; q.n = s.n; q.length = s.length;
  q.tiles = (uint32_t)((s.length + kCacheTile - 1) / kCacheTile);
  if (q.tiles == 0) q.tiles = 1;          // nothing to attend to: a unit that writes the empty result
  q.row_tiles = (s.n * p.group + ROWS - 1) / ROWS;
  q.units = (uint64_t)p.c.heads * q.row_tiles * (q.tiles + kSegmentCost);
  return q;
}

template <int TYPE, int D, int NT>
struct Shape {
  static constexpr int kRows = 8 * NT, kGroups = D / 64;
  // A CTA fills its SM: at head size 64 with 128 registers a thread 16 warps, with 168 12, as at 128; else 8. (At 128, 16 warps have the registers of a row's and
  // group's numbers in local memory: one user's step 12.4 us against 11.5, 131 K tokens 50.6 and 48.4, 64 users of 4000 tokens 82.4 and 78.4. As two CTAs
  // of 8, the second one's warps were given 18 % less of the SM's time than the first one's, and worked on alone at the end.)
  static constexpr uint32_t kWarps = D > 128 ? 8 : NT == 2 ? (D == 64 ? 12 : 8) : D == 64 ? 16 : 12, kThreads = 32 * kWarps;
  static constexpr uint32_t kTileBytes = 18 * D;
  // Ring stages of a warp, two tiles each: 9 KB at head sizes 64 and 128 (12 or 16 warps: 110 or 150 KB), and room for the warp's part of the join.
  static constexpr uint32_t kStages = D == 64 ? 4 : 2;
  static constexpr uint32_t kRing = kStages * 2 * kTileBytes;
  static constexpr uint32_t kRowFloats = D + 8;                             // of a part: rows shifted by 8 banks
  static constexpr uint32_t kPart = kRows * kRowFloats * 4;
  static constexpr uint32_t kRingSpace = ((kRing > kPart ? kRing : kPart) + 127) / 128 * 128;
  // A warp's memory: the ring, whose place its last part takes, and the part of the segment that its stretch begins inside of.
  static constexpr uint32_t kPerWarp = kRingSpace + (kPart + 127) / 128 * 128;
  static constexpr uint32_t kSmem = kWarps * kPerWarp;
};

__device__ __forceinline__ uint64_t divide(uint64_t a, uint32_t b) {      // nearly always in 32 bits, a fraction of the latency
  return a >> 32 ? a / b : (uint64_t)((uint32_t)a / b);
}

// Where a row of a segment goes, and its logarithm of the sum.
__device__ __forceinline__ uint16_t* out_row(const AttendParams& p, const Rows& s, uint32_t r, uint64_t* lse_at) {
  const uint32_t query = (s.row0 + r) / p.group, hh = s.head * p.group + (s.row0 + r) - query * p.group;
  const uint64_t row = (uint64_t)s.start + query;
  *lse_at = row * p.q_heads + hh;
  return p.out + row * p.out_token + (uint64_t)hh * p.out_head;
}
// A row that saw no token has no maximum and no sum.
__device__ __forceinline__ bool saw(float m, float l) { return m > kNoMax || !(l == 0.0f); }
// lost: the power of two that the sum lacks.
__device__ __forceinline__ float log_sum(float m, float l, float lost) { return saw(m, l) ? (m + (lost + log2f(l))) * 0.69314718055994531f : -INFINITY; }

template <int TYPE, int D, int NT>
__global__ void __launch_bounds__((Shape<TYPE, D, NT>::kThreads), 1) cache_attend_kernel(const __grid_constant__ AttendParams p) {
  using S = Shape<TYPE, D, NT>;
  constexpr int J = S::kGroups, R = S::kRows;
  constexpr uint32_t kWarps = S::kWarps, kThreads = S::kThreads;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t bars[kWarps][S::kStages];
  __shared__ uint64_t scan[kWarps];
  __shared__ uint64_t found_base[kWarps];
  __shared__ uint32_t found_b[kWarps];
  __shared__ float part_m[2][kWarps][R], part_l[2][kWarps][R];
  __shared__ float cta_m[R], cta_l[R];                      // of the CTA's part of a segment that a cluster has
  __shared__ Rows part_rows[2][kWarps];
  __shared__ uint32_t late[kWarps];                         // a wait ran out
  __shared__ __align__(8) uint32_t row_see[kWarps][R];      // tokens that a row sees, in front of the end of the warp's tiles
  __shared__ uint32_t row_see_any[kWarps];                  // and that some row does
  __shared__ Span spans[kWarps + 1];
  __shared__ uint32_t n_spans;
  __shared__ uint32_t part_open[2][kWarps];                 // 0: no part; 1: the segment ends inside the warp's stretch; 2: it goes on
  __shared__ uint64_t head_begin, head_end;                 // of the segment that the CTA's stretch begins inside of, on the line of units

  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, g = lane >> 2, t = lane & 3u;
  uint8_t* const ring = smem + warp * S::kPerWarp;
  const uint32_t ring_u32 = smem_u32(ring), bar_u32 = smem_u32(&bars[warp][0]);
  if (lane == 0) {
#pragma unroll
    for (uint32_t s = 0; s < S::kStages; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar_u32 + 8 * s) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    part_open[0][warp] = part_open[1][warp] = late[warp] = 0;
  }
  if (tid < R) { cta_m[tid] = kNoMax; cta_l[tid] = 0.0f; }
  __syncwarp();
  chain_wait();

  // ---- the warps' stretches of the line of units, and the sequences that they begin in -----------------------------------
  uint64_t u0, u1, per_cta = 0, seq_base = 0;
  Sequence seq{};
  if (p.direct) {                                           // segment blockIdx.x / p.direct, of sequences with as many segments each
    const uint32_t row_tiles = (p.group + R - 1) / R, each = p.c.heads * row_tiles, segment = blockIdx.x / p.direct, rank = blockIdx.x % p.direct;
    seq = sequence_at<R>(p, segment / each);
    const uint32_t mine = (seq.tiles + p.direct - 1) / p.direct, front = rank * mine, back = front + mine < seq.tiles ? front + mine : seq.tiles;
    uint32_t stretch = (mine + kWarps - 1) / kWarps;
    if (stretch < kLeastStretch) stretch = kLeastStretch;
    const uint64_t begin = (uint64_t)(segment % each) * (seq.tiles + kSegmentCost) + kSegmentCost;
    u0 = begin + front + warp * stretch;
    u1 = u0 + stretch < begin + back ? u0 + stretch : begin + back;
  } else {
    uint64_t total = 0;
    for (uint32_t b = tid; b < p.c.sequences; b += kThreads) total += sequence_at<R>(p, b).units;
#pragma unroll
    for (int m = 16; m; m >>= 1) total += __shfl_xor_sync(0xffffffffu, total, m);
    if (lane == 0) scan[warp] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) total += scan[w];
    per_cta = divide(total + gridDim.x - 1, gridDim.x);
    if (per_cta < kLeastCta) per_cta = kLeastCta;
    uint64_t stretch = (per_cta + kWarps - 1) / kWarps;
    if (stretch < kLeastStretch) stretch = kLeastStretch;
    const uint64_t cta0 = blockIdx.x * per_cta, cta1 = cta0 + per_cta < total ? cta0 + per_cta : total;
    if (cta0 >= total) {
      if (tid == 0) p.join[blockIdx.x].parts = 0;
      return;
    }
    uint64_t base = 0;
    for (uint32_t b0 = 0;; b0 += kThreads) {                 // ends: cta1 <= total
      const uint64_t mine = b0 + tid < p.c.sequences ? sequence_at<R>(p, b0 + tid).units : 0;
      uint64_t sum = mine;
#pragma unroll
      for (int m = 1; m < 32; m <<= 1) {
        const uint64_t up = __shfl_up_sync(0xffffffffu, sum, m);
        if (lane >= (uint32_t)m) sum += up;
      }
      __syncthreads();
      if (lane == 31) scan[warp] = sum;
      __syncthreads();
      uint64_t here = base, all = 0;
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w) {
        if (w < warp) here += scan[w];
        all += scan[w];
      }
      here += sum - mine;
      if (mine && here < cta1 && here + mine > cta0) {
#pragma unroll
        for (uint32_t w = 0; w < kWarps; ++w) {
          const uint64_t at = cta0 + w * stretch;
          if (here <= at && at < here + mine) { found_base[w] = here; found_b[w] = b0 + tid; }
        }
      }
      base += all;
      if (base >= cta1) break;
    }
    __syncthreads();

    u0 = cta0 + warp * stretch;
    u1 = u0 + stretch < cta1 ? u0 + stretch : cta1;
    if (u0 < u1) {
      seq = sequence_at<R>(p, found_b[warp]);
      seq_base = found_base[warp];
    }
  }
  uint32_t stage = 0, parity = 0;                           // of the next wait; the ring goes on from segment to segment

#pragma unroll 1
  for (uint64_t u = u0; u < u1;) {
    while (u >= seq_base + seq.units) {                     // (a sequence without rows has no units)
      seq_base += seq.units;
      seq = sequence_at<R>(p, seq.b + 1);
    }
    const uint64_t off = u - seq_base;
    const uint32_t span = seq.tiles + kSegmentCost;         // units of a segment: its cost, then its tiles
    const uint64_t segment = divide(off, span);
    const uint32_t x0 = (uint32_t)(off - segment * span), x1 = u1 - u < span - x0 ? x0 + (uint32_t)(u1 - u) : span;
    const uint32_t tile0 = x0 > kSegmentCost ? x0 - kSegmentCost : 0u, tile1 = x1 > kSegmentCost ? x1 - kSegmentCost : 0u;
    const uint64_t begin = u - x0 + kSegmentCost;           // its first tile on the line
    u += x1 - x0;
    if (tile0 == tile1) continue;                           // the stretch ends in front of its tiles
    const uint32_t head = (uint32_t)divide(segment, seq.row_tiles), row_tile = (uint32_t)(segment - (uint64_t)head * seq.row_tiles);
    const uint32_t row0 = row_tile * R, rows_all = seq.n * p.group;
    const uint32_t rows = rows_all - row0 < (uint32_t)R ? rows_all - row0 : (uint32_t)R;

    // Tokens that the first row sees (all rows see them) and that the last row sees.
    const int64_t all = seq.length - (int64_t)(seq.n - 1 - row0 / p.group), any = seq.length - (int64_t)(seq.n - 1 - (row0 + rows - 1) / p.group);
    const uint32_t see_all = all > 0 ? (uint32_t)all : 0u;
    const uint32_t see_any = any > 0 ? (uint32_t)any : 0u;
    uint32_t tile_end = (see_any + kCacheTile - 1) / kCacheTile;
    if (tile_end > tile1) tile_end = tile1;
    const uint32_t count = tile0 < tile_end ? tile_end - tile0 : 0u;
    const uint32_t clear = see_all / kCacheTile > tile0 ? see_all / kCacheTile - tile0 : 0u;      // tiles that every row sees whole
    // (A few tiles all go the way of those that are not seen whole: the code of the other way, cold, would take longer than it saves.)
    const uint32_t plain = count <= 4 ? 0u : clear < count ? clear : count;
    // ---- the warp's first copies: everything else of a segment's beginning goes on while they fly ---------------------------
    // Lane l knows where pairs l, l + 32, ... of the warp's tiles lie, and starts their copies.
    uint32_t pairs = (count + 1) / 2;
    auto look_up = [&](uint32_t i) -> const uint8_t* {
      if (i >= count) return nullptr;
      const uint32_t tile = tile0 + i, page = tile / p.c.page_tiles;
      int32_t at = __ldg(p.c.table + (uint64_t)seq.b * p.c.table_stride + page);
      if (at < 0 || (uint32_t)at >= p.c.n_pages) { atomicOr(p.c.status, QSGD_DEV_PAGE); at = 0; }
      return p.c.data + (uint64_t)at * p.c.page_stride + (uint64_t)head * p.c.head_stride + (uint64_t)(tile - page * p.c.page_tiles) * S::kTileBytes;
    };
    const uint8_t *source0 = look_up(2 * lane), *source1 = look_up(2 * lane + 1);
#pragma unroll 1
    for (uint32_t i = 0; i < S::kStages && i < pairs; ++i) {
      const uint32_t at = stage + i < S::kStages ? stage + i : stage + i - S::kStages;
      copy_tiles(lane == i, ring_u32 + at * 2 * S::kTileBytes, source0, source1, S::kTileBytes, bar_u32 + 8 * at);
    }


    // ---- queries: operands, sums of each group, and how far each row sees ------------------------------------------------
    uint32_t qf[NT][J][4][2];
    float qsum[NT][J][2], factor[NT][J][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint32_t r = 8 * nt + g;
      const bool live = r < rows;
      const uint32_t query = (row0 + r) / p.group, hh = (row0 + r) - query * p.group;
      const uint16_t* src = p.q + (uint64_t)(seq.start + query) * p.q_token + (uint64_t)(head * p.group + hh) * p.q_head + 16 * t;
      uint4 raw[J][2];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        raw[j][0] = raw[j][1] = make_uint4(0, 0, 0, 0);
        if (live) {
          raw[j][0] = __ldg(reinterpret_cast<const uint4*>(src + 64 * j));
          raw[j][1] = __ldg(reinterpret_cast<const uint4*>(src + 64 * j + 8));
        }
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float top_q = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t w[4] = {raw[j][h].x, raw[j][h].y, raw[j][h].z, raw[j][h].w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            top_q = fmaxf(top_q, fmaxf(fabsf(from_bits16<TYPE>(w[i] & 0xffffu)), fabsf(from_bits16<TYPE>(w[i] >> 16))));
        }
        top_q = fmaxf(top_q, __shfl_xor_sync(0xffffffffu, top_q, 1));
        top_q = fmaxf(top_q, __shfl_xor_sync(0xffffffffu, top_q, 2));
        // 2^(11 - e) for a largest number of [2^e, 2^(e + 1)); nothing to scale in a group of zeros, infinities or NaN
        const int32_t e = (int32_t)(__float_as_uint(top_q) >> 23) - 127;
        int32_t up = 11 - e;
        if (up > 120) up = top_q > 0.0f ? 120 : 0;
        if (e == 128) up = 0;
        const float times = __uint_as_float((uint32_t)(127 + up) << 23);
        const float back = p.scale_log2 * 1048576.0f * __uint_as_float((uint32_t)(127 - up) << 23);         // 2^20: see unpack
        factor[nt][j][0] = __shfl_sync(0xffffffffu, back, 8 * t);
        factor[nt][j][1] = __shfl_sync(0xffffffffu, back, 8 * t + 4);
        float sum = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t w[4] = {raw[j][h].x, raw[j][h].y, raw[j][h].z, raw[j][h].w};
          float x[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) { x[2 * i] = from_bits16<TYPE>(w[i] & 0xffffu) * times; x[2 * i + 1] = from_bits16<TYPE>(w[i] >> 16) * times; }
#pragma unroll
          for (int i = 0; i < 4; ++i) {                     // coordinates i and i + 4 of each word of eight
            sum += x[i] + x[i + 4];
            qf[nt][j][i][h] = pack16<QSGD_TYPE_F16>(x[i], x[i + 4]);
          }
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        sum *= 9.5367431640625e-07f;                        // 2^-20, as the codes
        qsum[nt][j][0] = __shfl_sync(0xffffffffu, sum, 8 * t);
        qsum[nt][j][1] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
      }
    }
    // How far each row sees; what lies behind the warp's tiles is not there to see. (Where only masked tiles look for it.)
    const uint32_t bound = tile_end * kCacheTile;
    if (lane < (uint32_t)R) {
      const int64_t far = lane < rows ? seq.length - (int64_t)(seq.n - 1 - (row0 + lane) / p.group) : 0;
      row_see[warp][lane] = far <= 0 ? 0u : far < (int64_t)bound ? (uint32_t)far : bound;
      if (lane == 0) row_see_any[warp] = see_any < bound ? see_any : bound;
    }
    __syncwarp();

    float o[NT][J][4][4], lsum[NT][2], osum[NT][J][2], top[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nt][j][i][0] = o[nt][j][i][1] = o[nt][j][i][2] = o[nt][j][i][3] = 0.0f;
        osum[nt][j][0] = osum[nt][j][1] = 0.0f;
      }
      lsum[nt][0] = lsum[nt][1] = 0.0f;
      top[nt][0] = top[nt][1] = kNoMax;
    }

    // ---- the warp's tiles, two at a time -------------------------------------------------------------------------------
    // Of each row and group: the power of two that p * step is multiplied by, and p * lo, until they are divided. It takes no p * step so far above 2^15,
    // and no p * lo above 2^25. And for each group a pair (lo, step): tokens up to it need no look at their p, which is 2^8 at most.
    float times[NT][J][2];
    uint32_t known[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      known[j] = 0;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) times[nt][j][0] = times[nt][j][1] = 64.0f / kLeastCap;
    }
    auto take_tiles = [&](auto masked_, const uint8_t* const tiles, const uint32_t first) {
      constexpr bool kMasked = decltype(masked_)::value;
      const uint32_t ka = token_of(g), kb = ka + 8;
      float sc[2][NT][4];                                   // scores of each tile: tokens ka, ka, kb, kb; rows 2t, 2t + 1, 2t, 2t + 1
      uint32_t pair[2][2][J];                               // of the values: tokens ka, kb
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t* const tile = tiles + h * S::kTileBytes;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sc[h][nt][0] = sc[h][nt][1] = sc[h][nt][2] = sc[h][nt][3] = 0.0f;
        uint32_t pair_a[J], pair_b[J];
        load_pairs<J>(reinterpret_cast<const uint32_t*>(tile + 8 * D) + ka * J, pair_a);
        load_pairs<J>(reinterpret_cast<const uint32_t*>(tile + 8 * D) + kb * J, pair_b);
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const uint2 ca = *reinterpret_cast<const uint2*>(tile + (j * 16 + ka) * 32 + 8 * t);
          const uint2 cb = *reinterpret_cast<const uint2*>(tile + (j * 16 + kb) * 32 + 8 * t);
          float acc[NT][4];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.0f;
          uint32_t ax[4], ay[4], bx[4], by[4];
          unpack(ca.x, ax); unpack(ca.y, ay); unpack(cb.x, bx); unpack(cb.y, by);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t a[4] = {ax[e], bx[e], ay[e], by[e]};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816(acc[nt], a, qf[nt][j][e][0], qf[nt][j][e][1]);
          }
          const float step_a = from_bits16<TYPE>(pair_a[j] >> 16), step_b = from_bits16<TYPE>(pair_b[j] >> 16);
          const float lo_a = from_bits16<TYPE>(pair_a[j] & 0xffffu), lo_b = from_bits16<TYPE>(pair_b[j] & 0xffffu);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[h][nt][e] = fmaf(factor[nt][j][e & 1], fmaf(e < 2 ? step_a : step_b, acc[nt][e], (e < 2 ? lo_a : lo_b) * qsum[nt][j][e & 1]), sc[h][nt][e]);
        }
        load_pairs<J>(reinterpret_cast<const uint32_t*>(tile + 17 * D) + ka * J, pair[h][0]);
        load_pairs<J>(reinterpret_cast<const uint32_t*>(tile + 17 * D) + kb * J, pair[h][1]);
      }

      // ---- softmax, against a maximum that is raised only when a score passes it by 2^8 ----------------------------------
      int32_t see[NT][2];                                                   // of the two tiles
      uint32_t see_any = 0;
      if (kMasked) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint2 both = *reinterpret_cast<const uint2*>(&row_see[warp][8 * nt + 2 * t]);
          see[nt][0] = (int32_t)(both.x - first); see[nt][1] = (int32_t)(both.y - first);
        }
        see_any = row_see_any[warp];
      }
      uint32_t seen = 0xffffffffu;                                          // bit 4 * (NT * h + nt) + e
      uint32_t widest[J];                                                   // the largest step and the largest lo (sign aside) of the lane's tokens
#pragma unroll
      for (int j = 0; j < J; ++j) widest[j] = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (kMasked && (int32_t)(16 * h + (e < 2 ? ka : kb)) >= see[nt][e & 1]) {
              seen &= ~(1u << (4 * (NT * h + nt) + e));
              sc[h][nt][e] = -INFINITY;
            }
          }
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (kMasked && first + 16 * h + (x ? kb : ka) >= see_any) pair[h][x][j] = 0;      // was never written, perhaps
            widest[j] = max_u16x2(widest[j], pair[h][x][j] & 0xffff7fffu);
          }
      }
      bool raise = false, wider = false;
#pragma unroll
      for (int j = 0; j < J; ++j) wider |= max_u16x2(widest[j], known[j]) != known[j];
      float high[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          high[nt][e] = fmaxf(fmaxf(sc[0][nt][e], sc[0][nt][e + 2]), fmaxf(sc[1][nt][e], sc[1][nt][e + 2]));
          raise |= high[nt][e] > top[nt][e] + 8.0f;
        }
      raise = __any_sync(0xffffffffu, raise || wider);
      if (raise) {
        // The lane's largest p times its largest size, which no p * size exceeds.
        bool over = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            over |= high[nt][e] > top[nt][e] + 8.0f;
            const float near = exp2_approx(high[nt][e] - top[nt][e] - 15.0f);
#pragma unroll
            for (int j = 0; j < J; ++j) over |= !(near * times[nt][j][e] * size_of_pair<TYPE>(widest[j]) <= 1.0f);      // (true of what is no number)
          }
        raise = __any_sync(0xffffffffu, over);
      }
      if (raise) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float m = fmaxf(fmaxf(sc[0][nt][e], sc[0][nt][e + 2]), fmaxf(sc[1][nt][e], sc[1][nt][e + 2]));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
            m = fmaxf(m, top[nt][e]);
            const float f = exp2_approx(top[nt][e] - m);
            top[nt][e] = m;
            lsum[nt][e] *= f;
            float p4[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) p4[x] = exp2_approx(sc[x >> 1][nt][e + 2 * (x & 1)] - m);
#pragma unroll
            for (int j = 0; j < J; ++j) {
              float size = 0.0f;                            // (what is no number is passed over: its products are none anyway)
#pragma unroll
              for (int x = 0; x < 4; ++x) size = fmaxf(size, p4[x] * size_of_pair<TYPE>(pair[x >> 1][x & 1][j]));
#pragma unroll
              for (int i = 4; i < 32; i <<= 1) size = fmaxf(size, __shfl_xor_sync(0xffffffffu, size, i));
              // The largest so far and now, as the next power of two, goes to 64.
              const float held = f * 64.0f * inverse_of_power(times[nt][j][e]), least = fminf(fmaxf(fmaxf(held, size), kLeastCap), kMostCap);
              const float cap = __uint_as_float((__float_as_uint(least) + 0x007fffffu) & 0xff800000u), inverse = inverse_of_power(cap);
              const float fo = held * inverse;              // (1 at most)
              times[nt][j][e] = 64.0f * inverse;
              osum[nt][j][e] *= fo;
#pragma unroll
              for (int r = 0; r < 4; ++r) { o[nt][j][r][e] *= fo; o[nt][j][r][e + 2] *= fo; }
            }
          }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          float most = times[0][j][0];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) most = fmaxf(most, fmaxf(times[nt][j][0], times[nt][j][1]));
          known[j] = pair_of_size<TYPE>(128.0f * inverse_of_power(most));          // 2^15 / 2^8
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[h][nt][e] = exp2_approx(sc[h][nt][e] - top[nt][e & 1]);
          lsum[nt][0] += sc[h][nt][0] + sc[h][nt][2];
          lsum[nt][1] += sc[h][nt][1] + sc[h][nt][3];
        }

      // ---- output ---------------------------------------------------------------------------------------------------------
      const uint32_t va = token_of(2 * t), vb = token_of(2 * t + 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t* const values = tiles + h * S::kTileBytes + 9 * D;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const float step_a = from_bits16<TYPE>(pair[h][0][j] >> 16), step_b = from_bits16<TYPE>(pair[h][1][j] >> 16);
          const float mid_a = fmaf(8.0f, step_a, from_bits16<TYPE>(pair[h][0][j] & 0xffffu));
          const float mid_b = fmaf(8.0f, step_b, from_bits16<TYPE>(pair[h][1][j] & 0xffffu));
          uint32_t bh[NT][2], bl[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float pr[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) pr[e] = sc[h][nt][e] * times[nt][j][e & 1];
            float w[4] = {pr[0] * step_a, pr[1] * step_a, pr[2] * step_b, pr[3] * step_b};
            if (kMasked) {                                  // what a row does not see may hold anything: no product with it
              float z[4] = {pr[0] * mid_a, pr[1] * mid_a, pr[2] * mid_b, pr[3] * mid_b};
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (!(seen >> (4 * (NT * h + nt) + e) & 1u)) w[e] = z[e] = 0.0f;
              osum[nt][j][0] += z[0] + z[2];
              osum[nt][j][1] += z[1] + z[3];
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) osum[nt][j][e & 1] = fmaf(pr[e], e < 2 ? mid_a : mid_b, osum[nt][j][e & 1]);
            }
            const uint32_t h0 = pack16<QSGD_TYPE_F16>(w[0], w[1]), h1 = pack16<QSGD_TYPE_F16>(w[2], w[3]);
            bh[nt][0] = transpose8x8(h0);
            bh[nt][1] = transpose8x8(h1);
            if (TYPE == QSGD_TYPE_F16) {
              bl[nt][0] = transpose8x8(pack16<QSGD_TYPE_F16>(w[0] - from_bits16<QSGD_TYPE_F16>(h0 & 0xffffu), w[1] - from_bits16<QSGD_TYPE_F16>(h0 >> 16)));
              bl[nt][1] = transpose8x8(pack16<QSGD_TYPE_F16>(w[2] - from_bits16<QSGD_TYPE_F16>(h1 & 0xffffu), w[3] - from_bits16<QSGD_TYPE_F16>(h1 >> 16)));
            }
          }
          const uint8_t* const codes = values + j * 512 + 4 * g;
          const uint32_t c0 = *reinterpret_cast<const uint32_t*>(codes + va * 32), c1 = *reinterpret_cast<const uint32_t*>(codes + vb * 32);
          const uint32_t c2 = *reinterpret_cast<const uint32_t*>(codes + (va + 8) * 32), c3 = *reinterpret_cast<const uint32_t*>(codes + (vb + 8) * 32);
          uint32_t lo01[4], hi01[4], lo23[4], hi23[4];
          unpack_centred(__byte_perm(c0, c1, 0x5410), lo01); unpack_centred(__byte_perm(c0, c1, 0x7632), hi01);
          unpack_centred(__byte_perm(c2, c3, 0x5410), lo23); unpack_centred(__byte_perm(c2, c3, 0x7632), hi23);
#pragma unroll
          for (int r = 0; r < 4; ++r) {                     // rows: coordinates 64 j + 8 g + r, and those + 4
            const uint32_t a[4] = {lo01[r], hi01[r], lo23[r], hi23[r]};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma16816(o[nt][j][r], a, bh[nt][0], bh[nt][1]);
              if (TYPE == QSGD_TYPE_F16) mma16816(o[nt][j][r], a, bl[nt][0], bl[nt][1]);
            }
          }
        }
      }
    };

#pragma unroll 1
    for (uint32_t i = 0; i < pairs; ++i) {
      if (!__all_sync(0xffffffffu, mbar_wait(bar_u32 + 8 * stage, parity, p.polls))) {
        // Said in the status word; the copy is waited for all the same, since it writes into the CTA's shared memory. One that does not land
        // within the built-in bound either ends the warp's work. (A way out of the loop here would cost 100 bytes of spilled registers.)
        late[warp] = 1;
        if (!__all_sync(0xffffffffu, mbar_wait(bar_u32 + 8 * stage, parity, kDrainPolls))) pairs = 0;
      }
      const uint32_t first = (tile0 + 2 * i) * kCacheTile;
      const uint8_t* const tiles = ring + stage * 2 * S::kTileBytes;
      // Some row does not see both tiles whole, or the second one lies behind the warp's stretch (and holds what was there before).
      if (2 * i + 2 > plain) take_tiles(Constant<true>(), tiles, first);
      else take_tiles(Constant<false>(), tiles, first);
      __syncwarp();                                         // the stage's readers are done
      const uint32_t next = i + S::kStages;
      if (next < pairs) {
        if ((next & 31u) == 0) { source0 = look_up(2 * (next + lane)); source1 = look_up(2 * (next + lane) + 1); }
        copy_tiles(lane == (next & 31u), ring_u32 + stage * 2 * S::kTileBytes, source0, source1, S::kTileBytes, bar_u32 + 8 * stage);
      }
      if (++stage == S::kStages) { stage = 0; parity ^= 1u; }
    }

    // ---- the segment's rows, or a part of them -----------------------------------------------------------------------------
    const bool from_front = tile0 == 0, to_end = tile1 == seq.tiles;
    const bool whole = from_front && to_end && p.direct <= 1;               // (a cluster's CTAs meet over every segment)
    const uint32_t slot = from_front ? 1u : 0u;             // a part without the segment's front is the stretch's first, one with it the last
    const Rows which{head, row0, rows, seq.start};
    float* const mine = reinterpret_cast<float*>(slot ? ring : ring + S::kRingSpace);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t r = 8 * nt + 2 * t + e;
        float l = lsum[nt][e];
#pragma unroll
        for (int m = 4; m < 32; m <<= 1) l += __shfl_xor_sync(0xffffffffu, l, m);
        uint64_t lse_at = 0;
        uint16_t* out = nullptr;
        float over = 0.0f;                                  // (sums that are not divided yet may lie outside fp32: times this, then times `held`)
        if (whole) {
          if (r < rows) {
            out = out_row(p, which, r, &lse_at);
            if (p.lse && g == 0) p.lse[lse_at] = log_sum(top[nt][e], l, 0.0f);
            over = saw(top[nt][e], l) ? 1.0f / l : 0.0f;
          }
        } else {
          over = p.part_times;
          if (g == 0) {
            part_m[slot][warp][r] = top[nt][e];
            part_l[slot][warp][r] = l * over;
          }
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const float held = inverse_of_power(times[nt][j][e]);         // undoes the power of two in o and osum
          float z = osum[nt][j][e];
#pragma unroll
          for (int m = 4; m < 32; m <<= 1) z += __shfl_xor_sync(0xffffffffu, z, m);
          float v[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = fmaf(o[nt][j][i][e], 512.0f, z) * over * held;                   // 2^9: see unpack_centred
            v[i + 4] = fmaf(o[nt][j][i][e + 2], 512.0f, z) * over * held;
          }
          if (out) {
            *reinterpret_cast<uint4*>(out + 64 * j + 8 * g) =
                make_uint4(pack16<TYPE>(v[0], v[1]), pack16<TYPE>(v[2], v[3]), pack16<TYPE>(v[4], v[5]), pack16<TYPE>(v[6], v[7]));
          } else if (!whole) {
            float* const at = mine + r * S::kRowFloats + 64 * j + 8 * g;
            *reinterpret_cast<float4*>(at) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(at + 4) = make_float4(v[4], v[5], v[6], v[7]);
          }
        }
      }
    if (!whole && lane == 0) {
      part_rows[slot][warp] = which;
      part_open[slot][warp] = to_end ? 1u : 2u;
      if (warp == 0 && slot == 0) { head_begin = begin; head_end = begin + seq.tiles; }
    }
  }
  __syncwarp();
  if (late[warp] && lane == 0) atomicOr(p.c.status, QSGD_DEV_TIMEOUT);

  // ---- what spans warps: joined, and written out where it ends in this CTA -------------------------------------------------
  __syncthreads();
  // Segment 0 begins in front of the CTA, segment k in warp k - 1. All threads go over all segments' rows. (Segments one after another, each waiting for
  // the latency of its reads, or a warp to each: 256 segments of 16 rows and 512 tokens took 37.5 us that way, 33.4 this.)
  if (warp == 0) {
    const uint32_t slot = lane ? 1u : 0u, w0 = lane ? lane - 1 : 0u;
    const bool open = lane <= kWarps && part_open[slot][w0] != 0;
    uint32_t w1 = w0;                                       // last warp that has some of the segment
    bool goes_on = open && part_open[slot][w0] == 2;
    while (goes_on && w1 + 1 < kWarps && part_open[0][w1 + 1]) goes_on = part_open[0][++w1] == 2;       // (the last warps may have no units)
    const uint32_t all = __ballot_sync(0xffffffffu, open);
    if (open) spans[__popc(all & ((1u << lane) - 1u))] = Span{(uint8_t)slot, (uint8_t)w0, (uint8_t)w1, (uint8_t)(slot && !goes_on)};
    if (lane == 0) n_spans = __popc(all);
  }
  __syncthreads();
  constexpr uint32_t kPieces = R * (D / 4);
  const uint32_t pieces = n_spans * kPieces;
#pragma unroll 1
  for (uint32_t i = tid; i < pieces; i += kThreads) {
    const Span span = spans[i / kPieces];
    const uint32_t r = i % kPieces / (D / 4), d4 = i % (D / 4), slot = span.slot, w0 = span.first;
    const Rows which = part_rows[slot][w0];
    if (r >= which.rows) continue;
    float m = part_m[slot][w0][r], l = part_l[slot][w0][r];
    float4 sum = *reinterpret_cast<const float4*>(smem + w0 * S::kPerWarp + (slot ? 0 : S::kRingSpace) + (r * S::kRowFloats + 4 * d4) * 4);
    for (uint32_t w = w0 + 1; w <= span.last; ++w) {
      const float wm = part_m[0][w][r], high = fmaxf(m, wm), f = exp2_approx(m - high), e = exp2_approx(wm - high);
      const float4 v = *reinterpret_cast<const float4*>(smem + w * S::kPerWarp + S::kRingSpace + (r * S::kRowFloats + 4 * d4) * 4);
      m = high;
      l = fmaf(e, part_l[0][w][r], f * l);
      sum.x = fmaf(e, v.x, f * sum.x); sum.y = fmaf(e, v.y, f * sum.y); sum.z = fmaf(e, v.z, f * sum.z); sum.w = fmaf(e, v.w, f * sum.w);
    }
    if (span.ends && p.direct <= 1) {
      uint64_t lse_at;
      uint16_t* const out = out_row(p, which, r, &lse_at);
      const float over = saw(m, l) ? 1.0f / l : 0.0f;
      *reinterpret_cast<uint2*>(out + 4 * d4) = make_uint2(pack16<TYPE>(sum.x * over, sum.y * over), pack16<TYPE>(sum.z * over, sum.w * over));
      if (p.lse && d4 == 0) p.lse[lse_at] = log_sum(m, l, p.part_lost);
    } else if (p.direct) {                                  // where the cluster's other CTAs look for it: nobody else's part, or this very place's
      *reinterpret_cast<float4*>(smem + S::kRingSpace + (r * S::kRowFloats + 4 * d4) * 4) = sum;
      if (d4 == 0) { cta_m[r] = m; cta_l[r] = l; }
    } else {
      float* const part = p.parts + ((uint64_t)blockIdx.x * 2 + slot) * part_floats(R, D);
      *reinterpret_cast<float4*>(part + r * D + 4 * d4) = sum;
      if (d4 == 0) { part[R * D + r] = m; part[R * D + R + r] = l; }
    }
  }
  JoinInfo info{};
  if (part_open[0][0] && !p.direct) {
    const uint32_t first = (uint32_t)(head_begin / per_cta);
    if (first + 1 == blockIdx.x) {                          // this CTA's start is the first such boundary inside the segment
      info.rows = part_rows[0][0];
      info.first = first;
      info.parts = (uint32_t)((head_end - 1) / per_cta) - first + 1;
    }
  }
  if (tid == 0 && !p.direct) p.join[blockIdx.x] = info;
  if (p.direct <= 1) return;

  // ---- a segment that a cluster has: each CTA joins the parts of some of the rows' coordinates --------------------------------
  cluster_barrier();
  const uint32_t segment = blockIdx.x / p.direct, rank = blockIdx.x % p.direct, row_tiles = (p.group + R - 1) / R;
  const uint32_t b = segment / (p.c.heads * row_tiles), rest = segment % (p.c.heads * row_tiles), row0 = rest % row_tiles * R;
  const Rows which{rest / row_tiles, row0, p.group - row0 < (uint32_t)R ? p.group - row0 : (uint32_t)R, b};
  for (uint32_t i = tid * p.direct + rank; i < which.rows * (D / 4); i += kThreads * p.direct) {
    const uint32_t r = i / (D / 4), d4 = i - r * (D / 4);
    float m = kNoMax, l = 0.0f;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (uint32_t c = 0; c < p.direct; ++c) {
      const float cm = cluster_load(smem_u32(&cta_m[r]), c), cl = cluster_load(smem_u32(&cta_l[r]), c);
      if (!saw(cm, cl)) continue;                           // a CTA without tiles has no part
      const float high = fmaxf(m, cm), f = exp2_approx(m - high), e = exp2_approx(cm - high);
      const float4 v = cluster_load4(smem_u32(smem + S::kRingSpace + (r * S::kRowFloats + 4 * d4) * 4), c);
      m = high;
      l = fmaf(e, cl, f * l);
      sum.x = fmaf(e, v.x, f * sum.x); sum.y = fmaf(e, v.y, f * sum.y); sum.z = fmaf(e, v.z, f * sum.z); sum.w = fmaf(e, v.w, f * sum.w);
    }
    uint64_t lse_at;
    uint16_t* const out = out_row(p, which, r, &lse_at);
    const float over = saw(m, l) ? 1.0f / l : 0.0f;
    *reinterpret_cast<uint2*>(out + 4 * d4) = make_uint2(pack16<TYPE>(sum.x * over, sum.y * over), pack16<TYPE>(sum.z * over, sum.w * over));
    if (p.lse && d4 == 0) p.lse[lse_at] = log_sum(m, l, p.part_lost);
  }
  cluster_barrier();                                        // no CTA leaves while another reads its shared memory
}

// Parts of a segment that several CTAs hold, one row to a CTA: a warp to every eighth part, each D / 32 coordinates a lane.
template <int TYPE, int D, int R>
__global__ void __launch_bounds__(kJoinThreads) cache_join_kernel(const __grid_constant__ AttendParams p, uint32_t n) {
  constexpr int V = D / 32;
  __shared__ float sum[kJoinWarps][D];
  __shared__ float part_m[kJoinWarps], part_l[kJoinWarps];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, r = blockIdx.x / n, cta = blockIdx.x - r * n;
  chain_wait();
  const JoinInfo j = p.join[cta];
  if (j.parts == 0 || r >= j.rows.rows) return;
  float m = kNoMax, l = 0.0f, o[V];
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = 0.0f;
  for (uint32_t k = warp; k < j.parts; k += kJoinWarps) {
    const float* part = p.parts + ((uint64_t)(j.first + k) * 2 + (k == 0 ? 1u : 0u)) * part_floats(R, D);
    const float pm = part[R * D + r], pl = part[R * D + R + r], top = fmaxf(m, pm), f = exp2_approx(m - top), e = exp2_approx(pm - top);
    l = fmaf(e, pl, l * f);
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = fmaf(e, part[r * D + 32 * i + lane], o[i] * f);
    m = top;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) sum[warp][32 * i + lane] = o[i];
  if (lane == 0) { part_m[warp] = m; part_l[warp] = l; }
  __syncthreads();
  if (threadIdx.x < D) {
    m = kNoMax;
    l = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < kJoinWarps; ++w) m = fmaxf(m, part_m[w]);
    float v = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < kJoinWarps; ++w) {
      const float f = exp2_approx(part_m[w] - m);
      l = fmaf(f, part_l[w], l);
      v = fmaf(f, sum[w][threadIdx.x], v);
    }
    uint64_t lse_at;
    uint16_t* const out = out_row(p, j.rows, r, &lse_at);
    out[threadIdx.x] = (uint16_t)to_bits16<TYPE>(saw(m, l) ? v / l : 0.0f);
    if (p.lse && threadIdx.x == 0) p.lse[lse_at] = log_sum(m, l, p.part_lost);
  }
}

template <int TYPE, int D, int NT>
int launch_attend(AttendParams& p, cudaStream_t stream) {
  using S = Shape<TYPE, D, NT>;
  static KernelSite site;
  auto kern = cache_attend_kernel<TYPE, D, NT>;
  int sms = 0, occ = 0;
  const int st = site.lookup(kern, S::kThreads, S::kSmem, &sms, &occ);
  if (st) return st;
  // Few segments, none long: a cluster of CTAs to each, as many as there are SMs for. Then there is no line of units to find one's place on, and
  // nothing to join behind.
  const uint64_t segments = (uint64_t)p.c.sequences * p.c.heads * ((p.group + S::kRows - 1) / S::kRows);
  const uint64_t longest = (uint64_t)p.c.table_pages * p.c.page_tiles * kCacheTile;
  p.direct = 0;
  if (!p.c.starts && segments <= kMostDirect) {
    uint32_t ctas = 1;
    while (ctas < kMostCluster && 2 * ctas * segments <= kMostDirect && 2 * ctas * kClusterTokens <= longest && (uint64_t)sms >= kMostDirect) ctas *= 2;
    if (longest <= (uint64_t)kDirectTokens * ctas) p.direct = ctas;
  }
  uint32_t grid = p.direct ? (uint32_t)segments * p.direct : (uint32_t)(sms * occ);
  if (grid > kMostCtas) grid = kMostCtas;
  {
    ScopedKernel sk(kKernCacheAttend, stream);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.direct ? p.direct : 1;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = launch_chaining_enabled() ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
    if (e != cudaSuccess || p.direct) return (int)e;
  }
  ScopedKernel sk(kKernCacheJoin, stream);
  return (int)launch_chained(cache_join_kernel<TYPE, D, S::kRows>, grid * S::kRows, kJoinThreads, 0, stream, p, grid);
}

template <int TYPE>
int dispatch(AttendParams& p, uint32_t dim, bool wide, cudaStream_t stream) {
  switch (dim) {
    case 64: return wide ? launch_attend<TYPE, 64, 2>(p, stream) : launch_attend<TYPE, 64, 1>(p, stream);
    case 128: return wide ? launch_attend<TYPE, 128, 2>(p, stream) : launch_attend<TYPE, 128, 1>(p, stream);
    case 192: return launch_attend<TYPE, 192, 1>(p, stream);
    default: return launch_attend<TYPE, 256, 1>(p, stream);
  }
}

}  // namespace

size_t cache_attend_workspace_bytes(uint32_t head_dim) {
  return kMostCtas * (sizeof(JoinInfo) + 2 * sizeof(float) * part_floats(kMostRowTile, head_dim));
}

int launch_cache_attend(const CacheView& view, uint32_t head_dim, int type, const AttendArgs& a, cudaStream_t stream) {
  if (cache_attend_wide_takes(view, head_dim, type, a.q_heads)) return launch_cache_attend_wide(view, head_dim, a, stream);
  AttendParams p;
  p.c = view;
  p.q = static_cast<const uint16_t*>(a.q);
  p.out = static_cast<uint16_t*>(a.out);
  p.q_token = a.q_token; p.q_head = a.q_head; p.out_token = a.out_token; p.out_head = a.out_head;
  p.lse = a.lse;
  p.q_heads = a.q_heads;
  p.group = a.q_heads / view.heads;
  p.scale_log2 = (float)((double)a.scale * 1.4426950408889634);
  p.polls = quantize_poll_limit();
  const int lost = attend_sums_lose(view);                  // (p against each part's maximum)
  p.part_lost = (float)lost;
  p.part_times = ldexpf(1.0f, -lost);
  p.join = reinterpret_cast<JoinInfo*>(a.workspace);
  p.parts = reinterpret_cast<float*>(a.workspace + kMostCtas * sizeof(JoinInfo));
  // 16 rows to a tile where a sequence has more than 8 on average: the codes are unpacked half as often.
  const bool wide = (uint64_t)view.rows * p.group > 8ull * view.sequences;
  return type == QSGD_TYPE_BF16 ? dispatch<QSGD_TYPE_BF16>(p, head_dim, wide, stream) : dispatch<QSGD_TYPE_F16>(p, head_dim, wide, stream);
}

}  // namespace qsgd
