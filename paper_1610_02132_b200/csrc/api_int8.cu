// C ABI of the 8-bit rows and products: argument validation and dispatch. See include/qsgd.h for the contract of every entry point.
#include "int8.cuh"

using namespace qsgd;

namespace {

constexpr uint32_t kMostCols = 131071;                     // 128 * 128 * cols stays below 2^31

bool type_taken(int type) { return type == QSGD_TYPE_F32 || type == QSGD_TYPE_F16 || type == QSGD_TYPE_BF16; }
uint64_t size_of(int type) { return type == QSGD_TYPE_F32 ? 4 : 2; }

bool on(const void* p, uint64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Codes of m rows, on 16-byte boundaries, and their scales behind them.
uint64_t padded_cols(uint32_t cols) { return ((uint64_t)cols + 15) & ~15ull; }

}  // namespace

extern "C" {

int qsgd_quantize_rows(const void* x, uint64_t rows, uint32_t cols, uint64_t row_stride, int type, int8_t* codes, uint64_t codes_stride,
                       float* scale, qsgd_stream_t stream) {
  if (!type_taken(type)) return QSGD_ERR_TYPE;
  if (cols < 1 || cols > kMostCols || rows > 0x7fffffffull || row_stride >> 40 || codes_stride >> 40) return QSGD_ERR_SHAPE;
  if (rows > 1 && codes_stride < cols) return QSGD_ERR_SHAPE;
  if (rows == 0) return QSGD_OK;
  if (!x || !codes || !scale) return QSGD_ERR_NULL;
  if (!on(x, size_of(type)) || !on(scale, 4)) return QSGD_ERR_ALIGN;
  return launch_quantize_rows(x, rows, cols, row_stride, type, codes, codes_stride, scale, false, static_cast<cudaStream_t>(stream));
}

int qsgd_matmul_i8(const int8_t* a, uint64_t a_stride, const float* a_scale, const int8_t* b, uint64_t b_stride, const float* b_scale,
                   const float* bias, uint64_t m, uint64_t n, uint32_t cols, void* out, uint64_t out_stride, int type, uint32_t* status_dev,
                   qsgd_stream_t stream) {
  if (!type_taken(type)) return QSGD_ERR_TYPE;
  if (cols < 1 || cols > kMostCols || m > 0x7fffffffull || n > 0x7fffffffull || a_stride >> 40 || b_stride >> 40 || out_stride >> 40)
    return QSGD_ERR_SHAPE;
  if (m > 1 && out_stride < n) return QSGD_ERR_SHAPE;
  if (m == 0 || n == 0) return QSGD_OK;
  if (!a || !b || !a_scale || !b_scale || !out) return QSGD_ERR_NULL;
  if (!on(a_scale, 4) || !on(b_scale, 4) || !on(bias, 4) || !on(out, size_of(type))) return QSGD_ERR_ALIGN;
  const MatmulArgs args{a, b, a_scale, b_scale, bias, out, m > 1 ? a_stride : padded_cols(cols), n > 1 ? b_stride : padded_cols(cols),
                        out_stride, (uint32_t)m, (uint32_t)n, cols, type, status_dev};
  return launch_matmul_i8(args, false, static_cast<cudaStream_t>(stream));
}

size_t qsgd_linear_i8_workspace_bytes(uint64_t m, uint32_t cols) {
  if (cols < 1 || cols > kMostCols || m > 0x7fffffffull) return 0;
  return (size_t)(m * padded_cols(cols) + ((4 * m + 15) & ~15ull));
}

int qsgd_linear_i8(const void* x, uint64_t x_stride, int x_type, const int8_t* w, uint64_t w_stride, const float* w_scale, const float* bias,
                   uint64_t m, uint64_t n, uint32_t cols, void* out, uint64_t out_stride, int out_type, void* workspace,
                   uint32_t* status_dev, qsgd_stream_t stream) {
  if (!type_taken(x_type) || !type_taken(out_type)) return QSGD_ERR_TYPE;
  if (cols < 1 || cols > kMostCols || m > 0x7fffffffull || n > 0x7fffffffull || x_stride >> 40 || w_stride >> 40 || out_stride >> 40)
    return QSGD_ERR_SHAPE;
  if (m > 1 && out_stride < n) return QSGD_ERR_SHAPE;
  if (m == 0 || n == 0) return QSGD_OK;
  if (!x || !w || !w_scale || !out || !workspace) return QSGD_ERR_NULL;
  if (!on(workspace, 16) || !on(x, size_of(x_type)) || !on(w_scale, 4) || !on(bias, 4) || !on(out, size_of(out_type))) return QSGD_ERR_ALIGN;
  int8_t* codes = static_cast<int8_t*>(workspace);
  float* scale = reinterpret_cast<float*>(codes + m * padded_cols(cols));
  const MatmulArgs args{codes, w, scale, w_scale, bias, out, padded_cols(cols), n > 1 ? w_stride : padded_cols(cols), out_stride, (uint32_t)m,
                        (uint32_t)n, cols, out_type, status_dev};
  // Few rows: the product starts while the quantizing kernel still runs, and brings in w before it waits for it.
  const bool few = m <= 128;
  const int st = launch_quantize_rows(x, m, cols, x_stride, x_type, codes, padded_cols(cols), scale, few, static_cast<cudaStream_t>(stream));
  return st ? st : launch_matmul_i8(args, few, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
