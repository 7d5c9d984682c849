// Product in 8-bit integers for few rows of a (and for rows that begin anywhere): out[m][n] = (a_m . b_n) a_scale b_scale + bias.
//
// Bytes of b bound it: each is read once for up to 16 rows of a (up to 64 where rows begin anywhere). A CTA takes 16 rows of b (those of an m16n8k32 product) and its warps
// 64 columns of them in turn; a lane reads 16 bytes of two of its rows straight into registers, since the order of the columns inside a product does
// not matter as long as both operands agree. The warps meet in shared memory; integer sums have no order. CTAs are small so that a GPU full of them
// holds all the rows of b at once where they are not too many: 16384 rows are 1024 CTAs, 7 to an SM, and no second round is left half empty.
//
// Behind qsgd_linear_i8's own quantizing kernel this one starts while that still runs, and has its first bytes of b on the way before it waits for it.
//
// Rows that do not begin on 16-byte boundaries are read as 32-bit words that do, shifted into place. Such a word holds at least one
// byte of the row, so the read stays in its page; what does not belong to the row is cleared in a, and zeros make its products nothing.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "int8.cuh"

namespace qsgd {

namespace {

constexpr uint32_t kRowsB = 16, kStep = 64;

// 16 bytes of a row from column k on; only those in front of `cols` are the row's.
template <bool ALIGNED>
__device__ __forceinline__ uint4 load16(const int8_t* row, uint32_t k, uint32_t cols) {
  if (k >= cols) return make_uint4(0, 0, 0, 0);
  if (ALIGNED && k + 16 <= cols) return __ldg(reinterpret_cast<const uint4*>(row + k));
  const uintptr_t at = reinterpret_cast<uintptr_t>(row + k);
  const uint32_t shift = (uint32_t)(at & 3u) * 8u, have = (cols - k < 16 ? cols - k : 16) + (uint32_t)(at & 3u);   // bytes from the first word on
  const uint32_t* src = reinterpret_cast<const uint32_t*>(at & ~(uintptr_t)3u);
  uint32_t w[5];
#pragma unroll
  for (uint32_t i = 0; i < 5; ++i) w[i] = 4 * i < have ? __ldg(src + i) : 0u;
  return make_uint4(__funnelshift_r(w[0], w[1], shift), __funnelshift_r(w[1], w[2], shift), __funnelshift_r(w[2], w[3], shift),
                    __funnelshift_r(w[3], w[4], shift));
}

// Clears what lies behind column `cols`.
__device__ __forceinline__ uint32_t keep_front(uint32_t w, int32_t bytes) {
  return bytes >= 4 ? w : bytes <= 0 ? 0u : w & ((1u << (8 * bytes)) - 1u);
}

__device__ __forceinline__ void mma16832(int32_t (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void store_as(void* out, uint64_t at, float v, int type) {
  if (type == QSGD_TYPE_F32) static_cast<float*>(out)[at] = v;
  else if (type == QSGD_TYPE_F16) static_cast<__half*>(out)[at] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(v);
}

template <int NT, bool ALIGNED, uint32_t WARPS>
__global__ void __launch_bounds__(32 * WARPS) matmul_i8_few_kernel(const __grid_constant__ MatmulArgs p, bool early) {
  __shared__ int32_t sums[WARPS][8 * NT][kRowsB + 1];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, g = lane >> 2, t = lane & 3u;
  const uint32_t n0 = blockIdx.x * kRowsB, m0 = blockIdx.y * 8 * NT;
  int32_t acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0;
  const uint32_t r0 = n0 + g, r1 = n0 + g + 8;
  const int8_t* b0 = p.b + (uint64_t)(r0 < p.n ? r0 : p.n - 1) * p.b_stride;        // (rows behind the last are computed and dropped)
  const int8_t* b1 = p.b + (uint64_t)(r1 < p.n ? r1 : p.n - 1) * p.b_stride;
  constexpr int kAhead = ALIGNED ? 4 : 1;
  uint4 wb0[kAhead], wb1[kAhead];
  auto fetch = [&](uint32_t k0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t k = k0 + i * WARPS * kStep + 16 * t;
      wb0[i] = load16<ALIGNED>(b0, k, p.k);
      wb1[i] = load16<ALIGNED>(b1, k, p.k);
    }
  };
  if (!early) chain_wait();
  fetch(warp * kStep);
  if (early) chain_wait();                                  // b is older than the kernel ahead, a is what that writes
  for (uint32_t k0 = warp * kStep; k0 < p.k; k0 += kAhead * WARPS * kStep) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t k = k0 + i * WARPS * kStep + 16 * t;
      uint4 a[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint32_t m = m0 + 8 * nt + g;
        a[nt] = make_uint4(0, 0, 0, 0);
        if (m < p.m) {
          a[nt] = load16<ALIGNED>(p.a + (uint64_t)m * p.a_stride, k, p.k);
          if (k + 16 > p.k) {
            const int32_t left = (int32_t)(p.k - k);
            a[nt].x = keep_front(a[nt].x, left); a[nt].y = keep_front(a[nt].y, left - 4);
            a[nt].z = keep_front(a[nt].z, left - 8); a[nt].w = keep_front(a[nt].w, left - 12);
          }
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mma16832(acc[nt], wb0[i].x, wb1[i].x, wb0[i].y, wb1[i].y, a[nt].x, a[nt].y);
        mma16832(acc[nt], wb0[i].z, wb1[i].z, wb0[i].w, wb1[i].w, a[nt].z, a[nt].w);
      }
    }
    fetch(k0 + kAhead * WARPS * kStep);                     // (zeros behind the last column)
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    sums[warp][8 * nt + 2 * t][g] = acc[nt][0];
    sums[warp][8 * nt + 2 * t + 1][g] = acc[nt][1];
    sums[warp][8 * nt + 2 * t][g + 8] = acc[nt][2];
    sums[warp][8 * nt + 2 * t + 1][g + 8] = acc[nt][3];
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < 8 * NT * kRowsB; i += 32 * WARPS) {
    const uint32_t mm = i / kRowsB, nn = i % kRowsB;
    if (m0 + mm >= p.m || n0 + nn >= p.n) continue;
    int32_t sum = 0;
#pragma unroll
    for (uint32_t w = 0; w < WARPS; ++w) sum += sums[w][mm][nn];
    const float v = scaled_sum(sum, __ldg(p.a_scale + m0 + mm), __ldg(p.b_scale + n0 + nn), p.bias ? __ldg(p.bias + n0 + nn) : 0.0f);
    store_as(p.out, (uint64_t)(m0 + mm) * p.out_stride + n0 + nn, v, p.type);
  }
}

template <int NT, bool ALIGNED, uint32_t WARPS>
int launch_warps(const MatmulArgs& p, bool early, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((p.n + kRowsB - 1) / kRowsB, (p.m + 8 * NT - 1) / (8 * NT));
  cfg.blockDim = dim3(32 * WARPS);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = launch_chaining_enabled() ? 1 : 0;
  ScopedKernel sk(kKernMatmulI8Few, stream);
  return (int)cudaLaunchKernelEx(&cfg, matmul_i8_few_kernel<NT, ALIGNED, WARPS>, p, early);
}

template <int NT, bool ALIGNED>
int launch(const MatmulArgs& p, bool early, cudaStream_t stream) {
  int sms = 0;
  const int st = device_sms(&sms);
  if (st) return st;
  // Eight warps share a CTA's columns where CTAs are too few to fill the SMs with four.
  const uint64_t ctas = (uint64_t)((p.n + kRowsB - 1) / kRowsB) * ((p.m + 8 * NT - 1) / (8 * NT));
  return ctas < 6ull * sms ? launch_warps<NT, ALIGNED, 8>(p, early, stream) : launch_warps<NT, ALIGNED, 4>(p, early, stream);
}

}  // namespace

int launch_matmul_i8(const MatmulArgs& p, bool early, cudaStream_t stream) {
  if (matmul_i8_many_takes(p)) return launch_matmul_i8_many(p, early, stream);
  const bool aligned = ((reinterpret_cast<uintptr_t>(p.a) | reinterpret_cast<uintptr_t>(p.b) | p.a_stride | p.b_stride) & 15u) == 0;
  // The second grid axis takes 65535 tiles: more rows go in several launches.
  constexpr uint32_t kMostRows = 65535u * 8;
  for (uint32_t m0 = 0; m0 < p.m;) {
    MatmulArgs q = p;
    q.m = p.m - m0 < kMostRows ? p.m - m0 : kMostRows;
    q.a += (uint64_t)m0 * p.a_stride;
    q.a_scale += m0;
    q.out = static_cast<uint8_t*>(p.out) + (uint64_t)m0 * p.out_stride * (p.type == QSGD_TYPE_F32 ? 4 : 2);
    int st;
    if (aligned && q.m <= 16) st = q.m <= 8 ? launch<1, true>(q, early, stream) : launch<2, true>(q, early, stream);
    else if (q.m <= 8) st = launch<1, false>(q, early, stream);
    else if (q.m <= 32) st = launch<4, false>(q, early, stream);
    else st = launch<8, false>(q, early, stream);
    if (st) return st;
    m0 += q.m;
    early = false;
  }
  return 0;
}

}  // namespace qsgd
