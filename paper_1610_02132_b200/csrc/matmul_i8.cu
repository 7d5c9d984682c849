// Product in 8-bit integers for many rows: out[m][n] = (a_m . b_n) a_scale b_scale + bias on the fifth-generation tensor cores.
//
// Tiles of 128 x `width` of the output, each summed over K by tcgen05.mma (kind::i8, exact 32-bit sums in tensor memory). A persistent CTA per SM:
// one warp keeps a ring of stages (128 columns of 128 rows of a and `width` rows of b, 128-byte swizzle) filled by TMA, which puts zeros where a or b
// end; one warp issues the products (one lane of either, the others go round with it); four warps take finished sums out of tensor memory, scale them and store them, while the next tile's
// products run into the other half of tensor memory.
//
// The width is what leaves the SMs least idle (pick_width): 256 for large products, where it halves the traffic from L2 against 128; fewer columns,
// so that there is a tile for every SM, where rows are few: the bytes of b are then what bounds a product, and a narrow tile's ring holds as many of
// them in flight as a wide one's.
//
// All waits are bounded. One that runs out raises a flag in shared memory, at which every role leaves its loop; the CTA then waits for the
// copies and products in flight (bounded again), frees its tensor memory and returns with QSGD_DEV_TIMEOUT in the status word, if there is one.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "int8.cuh"

namespace qsgd {

namespace {

constexpr uint32_t kBM = 128, kBK = 128, kMostStages = 16, kThreads = 192, kEpilogueWarps = 4;
constexpr uint32_t kMostWidth = 256, kLeastWidth = 32;
constexpr uint32_t kRingBytes = 4 * (kBM + kMostWidth) * kBK;
// Stages on 1024-byte boundaries. A stage holds no more rows of a than there are; the products read 128 all the same, whatever lies behind (sums of
// rows that are not there go nowhere), so there is that much room behind the last stage.
constexpr uint32_t kSmem = kRingBytes + kBM * kBK + 1024;
constexpr uint32_t kDrainPolls = 1u << 22;                 // bound of the waits for copies and products in flight
// Up to kFewRows rows, and up to twice as many of small products, matmul_i8_few.cu, which has a tile of 8 rows read w once more: 32 rows of 16384 x 4096
// take 36.5 us there and 15.5 here, 16 rows 19.2 and 15.9; 16 rows of 8192 x 8192 27.3 and 21.5, of 4096 x 8192 13.5 and 20.6, of 8192 x 4096 15.2
// and 13.1, of 4096 x 4096 7.8 and 12.3, of 16384 x 1024 6.7 and 7.8.
constexpr uint32_t kFewRows = 8, kLargeCols = 8192, kLargeDepth = 2048;

struct GemmParams {
  MatmulArgs p;
  uint32_t m_tiles, n_tiles, k_steps;
  uint32_t width, stages;      // columns of a tile (a multiple of 16), stages of the ring
  uint32_t a_bytes;            // of a stage's rows of a
  uint32_t polls;              // bound of the roles' waits
  bool early;                  // the kernel ahead writes a and its scales only
  bool vector_out;             // rows of out begin on 16-byte boundaries
};

// Position in a ring of stages.
struct Ring {
  uint32_t stage = 0, parity = 0, fills = 0;
  __device__ __forceinline__ void next(uint32_t stages) {
    ++fills;
    if (++stage == stages) { stage = 0; parity ^= 1u; }
  }
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// False when the wait ran out or another role's has.
struct Waits {
  volatile uint32_t* given_up;
  uint32_t polls;
};
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const Waits& w) {
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
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Shared-memory descriptor of a tile whose rows are 128 bytes, 128-byte swizzle: 8 rows are 1024 bytes apart.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr) {
  return ((uint64_t)0x40004040u << 32) | (1u << 16) | ((addr >> 4) & 0x3fffu);
}
__device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
               "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t at, int32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(at));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// Tiles in an order that keeps those at work together close: columns of up to 16 row tiles.
__device__ __forceinline__ void tile_at(const GemmParams& g, uint32_t i, uint32_t* m, uint32_t* n) {
  constexpr uint32_t kBand = 16;
  const uint32_t per_band = kBand * g.n_tiles, band = i / per_band, rest = i - band * per_band;
  const uint32_t first = band * kBand, rows = g.m_tiles - first < kBand ? g.m_tiles - first : kBand;
  *n = rest / rows;
  *m = first + (rest - *n * rows);
}

template <int TYPE>
struct Out;
template <>
struct Out<QSGD_TYPE_F32> {
  typedef float T;
  static __device__ __forceinline__ T one(float v) { return v; }
};
template <>
struct Out<QSGD_TYPE_F16> {
  typedef __half T;
  static __device__ __forceinline__ T one(float v) { return __float2half_rn(v); }
};
template <>
struct Out<QSGD_TYPE_BF16> {
  typedef __nv_bfloat16 T;
  static __device__ __forceinline__ T one(float v) { return __float2bfloat16_rn(v); }
};

// 16 bytes of output from the values at v.
template <int TYPE>
__device__ __forceinline__ uint4 pack_out(const float* v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TYPE == QSGD_TYPE_F32) w[i] = __float_as_uint(v[i]);
    else if constexpr (TYPE == QSGD_TYPE_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads, 1) matmul_i8_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                               const __grid_constant__ GemmParams g) {
  typedef typename Out<TYPE>::T T;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t full[kMostStages], empty[kMostStages], sums_full[2], sums_empty[2];
  __shared__ uint32_t tmem_base, given_up;
  __shared__ float b_scale[kMostWidth], bias[kMostWidth];   // of the tile that is taken out
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const Waits waits{&given_up, g.polls};
  const uint32_t ring0 = (smem_u32(smem_raw) + 1023u) & ~1023u, stage_bytes = g.a_bytes + g.width * kBK;
  const uint32_t full0 = smem_u32(full), empty0 = smem_u32(empty), sums_full0 = smem_u32(sums_full), sums_empty0 = smem_u32(sums_empty);
  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < g.stages; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    for (uint32_t s = 0; s < 2; ++s) { mbar_init(sums_full0 + 8 * s, 1); mbar_init(sums_empty0 + 8 * s, kEpilogueWarps); }
    given_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0)                                            // all of tensor memory: two tiles of up to 256 columns
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(2 * kMostWidth) : "memory");
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_base;
  if (!g.early) chain_wait();

  const uint32_t tiles = g.m_tiles * g.n_tiles;
  if (warp == 0) {                                          // ---- fills the ring ------------------------------------------------
    // (The whole warp goes round here and in the next role, so that addresses are in uniform registers, and one lane issues: 37 rows on 5000 x 2885
    // take 10.2 us, 11.4 with one lane in the loops; 2048 on 8192 x 4096 take 52.9 and 53.7.)
    Ring r;
    bool fine = true;
    // Behind the library's own quantizing kernel: the first stages' rows of b are on their way before that has written a.
    uint32_t ahead = 0;
    if (g.early) {
      uint32_t m, n;
      tile_at(g, blockIdx.x, &m, &n);
      for (; ahead < g.stages && ahead < g.k_steps; ++ahead) {
        if (elected()) {
          const uint32_t bar = full0 + 8 * ahead;
          mbar_expect(bar, stage_bytes);
          tma_load(ring0 + ahead * stage_bytes + g.a_bytes, &map_b, ahead * kBK, n * g.width, bar);
        }
        __syncwarp();
      }
      chain_wait();
    }
    for (uint32_t i = blockIdx.x; i < tiles && fine; i += gridDim.x) {
      uint32_t m, n;
      tile_at(g, i, &m, &n);
      for (uint32_t k = 0; k < g.k_steps; ++k) {
        if (r.fills >= g.stages && !__all_sync(0xffffffffu, mbar_wait(empty0 + 8 * r.stage, r.parity ^ 1u, waits))) { fine = false; break; }
        if (elected()) {
          const uint32_t at = ring0 + r.stage * stage_bytes, bar = full0 + 8 * r.stage;
          if (r.fills >= ahead) {
            mbar_expect(bar, stage_bytes);
            tma_load(at + g.a_bytes, &map_b, k * kBK, n * g.width, bar);
          }
          tma_load(at, &map_a, k * kBK, m * kBM, bar);
        }
        __syncwarp();
        r.next(g.stages);
      }
    }
    // What is in flight lands before the CTA's shared memory goes away, whether anybody still waits for it or not.
    for (uint32_t back = 1; back <= g.stages && back <= r.fills; ++back) {
      const uint32_t fill = r.fills - back;
      for (uint32_t t = 0; t < kDrainPolls && !mbar_try(full0 + 8 * (fill % g.stages), (fill / g.stages) & 1u); ++t) {}
    }
  } else if (warp == 1) {                                   // ---- issues the products -------------------------------------------
    {
      const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((g.width >> 3) << 17) | ((kBM >> 4) << 24);     // s32 += s8 * s8
      Ring r;
      uint32_t done = 0;
      bool fine = true;
      for (uint32_t i = blockIdx.x; i < tiles && fine; i += gridDim.x, ++done) {
        const uint32_t half = done & 1u, use = done >> 1;
        if (use && !__all_sync(0xffffffffu, mbar_wait(sums_empty0 + 8 * half, (use - 1) & 1u, waits))) { fine = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (uint32_t k = 0; k < g.k_steps; ++k) {
          if (!__all_sync(0xffffffffu, mbar_wait(full0 + 8 * r.stage, r.parity, waits))) { fine = false; break; }
          if (elected()) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = ring0 + r.stage * stage_bytes;
            const uint64_t a = tile_desc(at), b = tile_desc(at + g.a_bytes);
#pragma unroll
            for (uint32_t x = 0; x < kBK / 32; ++x) mma_i8(tmem + half * kMostWidth, a + 2 * x, b + 2 * x, idesc, k != 0 || x != 0);
            tc_commit(empty0 + 8 * r.stage);
          }
          __syncwarp();
          r.next(g.stages);
        }
        if (fine && elected()) tc_commit(sums_full0 + 8 * half);
        __syncwarp();
      }
      // After a wait that ran out: products in flight are done before tensor memory is freed.
      if (!fine && r.fills) {
        const uint32_t fill = r.fills - 1;
        for (uint32_t t = 0; t < kDrainPolls && !mbar_try(empty0 + 8 * (fill % g.stages), (fill / g.stages) & 1u); ++t) {}
      }
    }
  } else {                                                  // ---- takes the sums out --------------------------------------------
    const uint32_t quarter = warp & 3u;                     // of tensor memory's lanes: a warp reaches those of its number modulo 4
    uint32_t done = 0;
    bool waited = !g.early, fine = true;
    for (uint32_t i = blockIdx.x; i < tiles; i += gridDim.x, ++done) {
      uint32_t m, n;
      tile_at(g, i, &m, &n);
      const uint32_t half = done & 1u;
      // The columns' scales come while the sums do. (All four warps meet twice a tile, whether they have given up or not.)
      asm volatile("bar.sync 1, 128;" ::: "memory");
      for (uint32_t c = threadIdx.x - 64; c < g.width; c += 128) {
        const uint32_t col = n * g.width + c < g.p.n ? n * g.width + c : g.p.n - 1;
        b_scale[c] = __ldg(g.p.b_scale + col);
        bias[c] = g.p.bias ? __ldg(g.p.bias + col) : 0.0f;
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
      if (!waited) { chain_wait(); waited = true; }
      fine = fine && __all_sync(0xffffffffu, mbar_wait(sums_full0 + 8 * half, (done >> 1) & 1u, waits));
      if (!fine) continue;                                  // (to the next tile's meetings, and no further)
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t row = m * kBM + 32 * quarter + lane;
      const bool live = row < g.p.m;
      const float a_scale = live ? __ldg(g.p.a_scale + row) : 0.0f;
      T* const out = static_cast<T*>(g.p.out) + (uint64_t)row * g.p.out_stride;
      if (m * kBM + 32 * quarter < g.p.m) {                 // (of the warp: some of its rows are there)
#pragma unroll 2
        for (uint32_t c = 0; c < g.width; c += 16) {
          const uint32_t col = n * g.width + c;
          if (col >= g.p.n) break;
          int32_t v[16];
          tmem_load16(tmem + half * kMostWidth + c + ((32 * quarter) << 16), v);
          if (live) {
            float y[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              y[x] = scaled_sum(v[x], a_scale, b_scale[c + x], bias[c + x]);
            }
            if (g.vector_out && col + 16 <= g.p.n) {
              constexpr int kPer = 16 / sizeof(T);
#pragma unroll
              for (int x = 0; x < 16; x += kPer) *reinterpret_cast<uint4*>(out + col + x) = pack_out<TYPE>(y + x);
            } else {
#pragma unroll
              for (int x = 0; x < 16; ++x)
                if (col + x < g.p.n) out[col + x] = Out<TYPE>::one(y[x]);
            }
          }
          __syncwarp();                                     // the next read of tensor memory is of the whole warp
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(sums_empty0 + 8 * half);
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 0) {
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kMostWidth));
  }
  if (threadIdx.x == 0 && given_up && g.p.status) atomicOr(g.p.status, QSGD_DEV_TIMEOUT);
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode_tiled(EncodeTiled* out) {
  static std::atomic<void*> known{nullptr};
  void* fn = known.load(std::memory_order_acquire);
  if (!fn) {
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return (int)e;
    if (found != cudaDriverEntryPointSuccess || !fn) return (int)cudaErrorNotSupported;
    known.store(fn, std::memory_order_release);
  }
  *out = reinterpret_cast<EncodeTiled>(fn);
  return 0;
}

// Rows of int8 in boxes of 128 columns x `box` rows.
int make_map(CUtensorMap* map, const int8_t* base, uint32_t cols, uint32_t rows, uint64_t stride, uint32_t box) {
  EncodeTiled encode;
  const int st = encode_tiled(&encode);
  if (st) return st;
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {stride};
  const cuuint32_t boxes[2] = {kBK, box}, ones[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(base), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? 0 : (int)cudaErrorInvalidValue;
}

// Columns of a tile. The tiles go round the SMs in rounds of equal length: a round takes as long as a tile has columns of b to bring in and to multiply
// with, and a part for a's rows and the tile's beginning and end.
uint32_t pick_width(uint32_t m_tiles, uint32_t a_rows, uint32_t n, uint32_t sms) {
  uint32_t best = kMostWidth;
  uint64_t least = ~0ull;
  for (uint32_t w = kMostWidth; w >= kLeastWidth; w -= 16) {
    const uint64_t tiles = (uint64_t)m_tiles * ((n + w - 1) / w), cost = (tiles + sms - 1) / sms * (w + a_rows / 2);
    if (cost < least) { least = cost; best = w; }
  }
  return best;
}

template <int TYPE>
int launch(const MatmulArgs& p, bool early, cudaStream_t stream) {
  static KernelSite site;
  int sms = 0, occ = 0;
  int st = site.lookup(matmul_i8_kernel<TYPE>, kThreads, kSmem, &sms, &occ);
  if (st) return st;
  GemmParams g;
  g.p = p;
  g.m_tiles = (p.m + kBM - 1) / kBM;
  const uint32_t a_rows = p.m < kBM ? (p.m + 7) / 8 * 8 : kBM;              // (8 rows of 128 bytes: the swizzle's period)
  g.a_bytes = a_rows * kBK;
  g.width = pick_width(g.m_tiles, a_rows, p.n, (uint32_t)sms);
  g.n_tiles = (p.n + g.width - 1) / g.width;
  g.k_steps = (p.k + kBK - 1) / kBK;
  g.stages = kRingBytes / (g.a_bytes + g.width * kBK);
  if (g.stages > kMostStages) g.stages = kMostStages;
  g.polls = quantize_poll_limit();
  g.early = early;
  g.vector_out = ((reinterpret_cast<uintptr_t>(p.out) | p.out_stride * (TYPE == QSGD_TYPE_F32 ? 4 : 2)) & 15u) == 0;
  CUtensorMap a, b;
  st = make_map(&a, p.a, p.k, p.m, p.a_stride, a_rows);
  if (!st) st = make_map(&b, p.b, p.k, p.n, p.b_stride, g.width);
  if (st) return st;
  const uint64_t tiles = (uint64_t)g.m_tiles * g.n_tiles;
  ScopedKernel sk(kKernMatmulI8, stream);
  return (int)launch_chained(matmul_i8_kernel<TYPE>, (uint32_t)(tiles < (uint64_t)sms ? tiles : (uint64_t)sms), kThreads, kSmem, stream, a, b, g);
}

}  // namespace

bool matmul_i8_many_takes(const MatmulArgs& p) {
  // TMA: rows on 16-byte boundaries. Tiles are counted in 32 bits.
  const bool aligned = ((reinterpret_cast<uintptr_t>(p.a) | reinterpret_cast<uintptr_t>(p.b) | p.a_stride | p.b_stride) & 15u) == 0;
  const uint64_t tiles = (uint64_t)((p.m + kBM - 1) / kBM) * ((p.n + kLeastWidth - 1) / kLeastWidth);
  return aligned && p.a_stride >= p.k && p.b_stride >= p.k && tiles < (1u << 30) && p.m > (p.n >= kLargeCols && p.k >= kLargeDepth ? kFewRows : 2 * kFewRows);
}

int launch_matmul_i8_many(const MatmulArgs& p, bool early, cudaStream_t stream) {
  switch (p.type) {
    case QSGD_TYPE_F32: return launch<QSGD_TYPE_F32>(p, early, stream);
    case QSGD_TYPE_F16: return launch<QSGD_TYPE_F16>(p, early, stream);
    default: return launch<QSGD_TYPE_BF16>(p, early, stream);
  }
}

}  // namespace qsgd
