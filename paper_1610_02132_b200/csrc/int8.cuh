// Rows in 8-bit integers with a scale each, and their products: the internal launch interface.
#pragma once

#include "qsgd_common.cuh"

namespace qsgd {

int launch_quantize_rows(const void* x, uint64_t rows, uint32_t cols, uint64_t row_stride, int type, int8_t* codes, uint64_t codes_stride,
                         float* scale, bool release, cudaStream_t stream);
// release: the next kernel of the stream may start as soon as the kernels in front of this one are done. It waits for this one itself.

struct MatmulArgs {
  const int8_t* a;
  const int8_t* b;
  const float* a_scale;
  const float* b_scale;
  const float* bias;          // or nullptr
  void* out;
  uint64_t a_stride, b_stride, out_stride;
  uint32_t m, n, k;
  int type;
  uint32_t* status;           // or nullptr
};
// early: the kernel ahead is the one that writes a and its scales, launched with `release`; b, its scales and the bias are older.
int launch_matmul_i8(const MatmulArgs& args, bool early, cudaStream_t stream);

// For many rows (matmul_i8.cu): whether it takes a product, and the launch.
bool matmul_i8_many_takes(const MatmulArgs& args);
int launch_matmul_i8_many(const MatmulArgs& args, bool early, cudaStream_t stream);

#ifdef __CUDACC__
// The sum, scaled: in fp32, in this order, rounded to the output's type once.
__device__ __forceinline__ float scaled_sum(int32_t sum, float a_scale, float b_scale, float bias) {
  return __fadd_rn(__fmul_rn(__fmul_rn(__int2float_rn(sum), a_scale), b_scale), bias);
}
#endif

}  // namespace qsgd
