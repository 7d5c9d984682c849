// Rows in 8 bits: scale = max|x| / 127, codes the whole numbers nearest to x * 127 / max|x|, of two as near the even one.
//
// A CTA to a row. The row is read once into registers (up to 8192 columns; what is behind those is read again, out of L2), its
// maximum goes round the CTA, and the codes are written: bytes in and out are all there is to do, so HBM bounds it where rows are many, and
// where they are few the latency of one read and one exchange.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <float.h>

#include "int8.cuh"

namespace qsgd {

namespace {

constexpr uint32_t kThreads = 256, kSpan = 8 * kThreads;    // columns that a CTA takes at a time
constexpr int kKept = 4;

struct RowsArgs {
  const void* x;
  int8_t* codes;
  float* scale;
  uint64_t rows, row_stride, codes_stride;
  uint32_t cols;
  bool release;
};

template <int TYPE>
struct Element;
template <>
struct Element<QSGD_TYPE_F32> {
  typedef float T;
  static __device__ __forceinline__ float get(T v) { return v; }
};
template <>
struct Element<QSGD_TYPE_F16> {
  typedef __half T;
  static __device__ __forceinline__ float get(T v) { return __half2float(v); }
};
template <>
struct Element<QSGD_TYPE_BF16> {
  typedef __nv_bfloat16 T;
  static __device__ __forceinline__ float get(T v) { return __bfloat162float(v); }
};

// Columns [c, c + 8) of a row, zeros behind its end. VECTOR: rows begin on 16-byte boundaries.
template <int TYPE, bool VECTOR>
__device__ __forceinline__ void load8(const typename Element<TYPE>::T* row, uint32_t c, uint32_t cols, float (&v)[8]) {
  typedef typename Element<TYPE>::T T;
  if (VECTOR && c + 8 <= cols) {
    T e[8];
    const uint4* src = reinterpret_cast<const uint4*>(row + c);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(e)[i] = __ldg(src + i);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = Element<TYPE>::get(e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? Element<TYPE>::get(row[c + i]) : 0.0f;
  }
}

// The product with the rounded factor is off by at most two roundings, 127 * 2^-23. Only so close to the middle between two codes (half the
// maximum lies on one) does the exact remainder decide, which fp64 holds.
__device__ __forceinline__ int32_t code_of(float v, float factor, float top) {
  const float q = v * factor, c = rintf(q);
  int32_t code = (int32_t)c;
  if (fabsf(q - c) > 0.4999f) {
    const double rest = 127.0 * (double)v - (double)code * (double)top, half = 0.5 * (double)top;
    if (fabs(rest) > half || (fabs(rest) == half && (code & 1))) code += rest > 0.0 ? 1 : -1;
  }
  return code;
}

template <bool VECTOR>
__device__ __forceinline__ void store8(int8_t* row, uint32_t c, uint32_t cols, const float (&v)[8], float factor, float top) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i >> 2] |= ((uint32_t)code_of(v[i], factor, top) & 0xffu) << (8 * (i & 3));
  if (VECTOR && c + 8 <= cols) {
    *reinterpret_cast<uint2*>(row + c) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) row[c + i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}

template <int TYPE, bool VECTOR>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const __grid_constant__ RowsArgs a) {
  typedef typename Element<TYPE>::T T;
  __shared__ float warp_top[kThreads / 32];
  const uint32_t c0 = 8 * threadIdx.x;
  chain_wait();
  // (The library's kernels else release no dependents: waiting CTAs slow running ones down. Here the running ones are a CTA to a row, 128 at most.)
  if (a.release) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* row = static_cast<const T*>(a.x) + r * a.row_stride;
    int8_t* out = a.codes + r * a.codes_stride;
    float kept[kKept][8];
    float top = 0.0f;
    bool fine = true;
#pragma unroll
    for (int s = 0; s < kKept; ++s) {
      const uint32_t c = c0 + s * kSpan;
      if (c < a.cols) {
        load8<TYPE, VECTOR>(row, c, a.cols, kept[s]);
#pragma unroll
        for (int i = 0; i < 8; ++i) { top = fmaxf(top, fabsf(kept[s][i])); fine &= fabsf(kept[s][i]) <= FLT_MAX; }
      }
    }
    for (uint32_t c = c0 + kKept * kSpan; c < a.cols; c += kSpan) {
      float v[8];
      load8<TYPE, VECTOR>(row, c, a.cols, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) { top = fmaxf(top, fabsf(v[i])); fine &= fabsf(v[i]) <= FLT_MAX; }
    }
    if (!fine) top = INFINITY;
#pragma unroll
    for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    if ((threadIdx.x & 31u) == 0) warp_top[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 32; ++w) top = fmaxf(top, warp_top[w]);
    fine = top <= FLT_MAX;
    const bool some = fine && top >= 127.0f * FLT_MIN;      // (a scale below the smallest normal number would lose its bits)
    const float factor = some ? 127.0f / top : 0.0f;
    if (threadIdx.x == 0) a.scale[r] = some ? top / 127.0f : fine ? 0.0f : NAN;
#pragma unroll
    for (int s = 0; s < kKept; ++s) {
      const uint32_t c = c0 + s * kSpan;
      if (c < a.cols) {
        if (!some) {
#pragma unroll
          for (int i = 0; i < 8; ++i) kept[s][i] = 0.0f;    // (NaN and infinity times zero would not be)
        }
        store8<VECTOR>(out, c, a.cols, kept[s], factor, top);
      }
    }
    for (uint32_t c = c0 + kKept * kSpan; c < a.cols; c += kSpan) {
      float v[8];
      load8<TYPE, VECTOR>(row, c, a.cols, v);
      if (!some) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
      }
      store8<VECTOR>(out, c, a.cols, v, factor, top);
    }
    __syncthreads();                                        // warp_top is written again
  }
}

template <int TYPE, bool VECTOR>
int launch(const RowsArgs& a, cudaStream_t stream) {
  static KernelSite site;
  int sms = 0, occ = 0;
  const int st = site.lookup(quantize_rows_kernel<TYPE, VECTOR>, kThreads, 0, &sms, &occ);
  if (st) return st;
  const uint64_t ctas = (uint64_t)sms * occ;
  ScopedKernel sk(kKernQuantizeRows, stream);
  return (int)launch_chained(quantize_rows_kernel<TYPE, VECTOR>, (uint32_t)(a.rows < ctas ? a.rows : ctas), kThreads, 0, stream, a);
}

}  // namespace

int launch_quantize_rows(const void* x, uint64_t rows, uint32_t cols, uint64_t row_stride, int type, int8_t* codes, uint64_t codes_stride,
                         float* scale, bool release, cudaStream_t stream) {
  const RowsArgs a{x, codes, scale, rows, row_stride, codes_stride, cols, release};
  const uint64_t size = type == QSGD_TYPE_F32 ? 4 : 2;
  const bool vector = ((reinterpret_cast<uintptr_t>(x) | row_stride * size) & 15u) == 0 &&
                      ((reinterpret_cast<uintptr_t>(codes) | codes_stride) & 7u) == 0;
  switch (type) {
    case QSGD_TYPE_F32: return vector ? launch<QSGD_TYPE_F32, true>(a, stream) : launch<QSGD_TYPE_F32, false>(a, stream);
    case QSGD_TYPE_F16: return vector ? launch<QSGD_TYPE_F16, true>(a, stream) : launch<QSGD_TYPE_F16, false>(a, stream);
    default: return vector ? launch<QSGD_TYPE_BF16, true>(a, stream) : launch<QSGD_TYPE_BF16, false>(a, stream);
  }
}

}  // namespace qsgd
